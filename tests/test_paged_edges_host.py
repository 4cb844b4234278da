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
