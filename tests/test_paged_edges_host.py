"""The paged cache's binding without a GPU: what it refuses beside the tests of its C entry points (test_paged_host)."""
import pytest

from paper_2308_04623_amd import paged, ssd


def test_a_pools_tensors_cannot_be_replaced():
    """(The calls hold their addresses.)"""
    pages = object.__new__(paged.Pages)
    pages.data = data = object()
    pages.kind = ()
    for name in ("data", "scale", "page_rows", "code", "n_page", "kind", "_pool"):
        with pytest.raises(ssd.SSDError, match=name):
            setattr(pages, name, object())
    with pytest.raises(ssd.SSDError):
        del pages.data
    assert pages.data is data


def test_trees_whose_nodes_have_no_node_as_parent_are_refused():
    """(Such a node was at depth 1 for its position and a root for attention.)"""
    from types import SimpleNamespace

    import numpy as np

    from paper_2308_04623_amd.batch import Batch
    masks = lambda *parents: Batch.masks(SimpleNamespace(model=SimpleNamespace(device="cpu")), np.array(parents))  # noqa: E731
    assert masks([-1, 0, -2, 1, -1], [-2, -1, 1, 1, -3]).tolist() == [[1, 3, 0, 11, 16], [0, 2, 6, 10, 0]]
    for bad in ([-1, 0, -2, 2, 1], [-2, 0, 1, 2, 3], [-1, 0, 1, 3, 0], [-1, -3, 1, 0, 0]):
        with pytest.raises(ValueError, match="node"):
            masks([-1, 0, 1, 2, 3], bad)
