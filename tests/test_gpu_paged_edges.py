"""The paged cache's operators at calls that their documentation allows and a program seldom makes."""
import math

import numpy as np
import pytest

import paged_model as M
import test_gpu_paged as P

pytestmark = pytest.mark.gpu
env = P.env


# ---------------------------------------------------------------- commits

@pytest.mark.parametrize("dtype,code,rows,d,t", [("bf16", "int8", 32, 64, 2), ("f32", "int8", 32, 32, 7),
                                                 ("bf16", "e4m3", 64, 128, 1), ("f32", "e4m3", 128, 64, 33)])
def test_paths_that_name_rows_twice(env, dtype, code, rows, d, t):
    """Paths of 64 entries that name the same rows again: as many count as there are new rows, so the open page's rows stay in
    the tail (page_rows + t - 1 rows, the least there may be) until its codes are made of them."""
    torch, paged, _ = env
    b = 4
    batch = P.Batch(env, b, 6, 20, t, dtype, code, d=d, rows=rows)
    assert batch.kt.shape[3] == rows + t - 1
    for x in (batch.length, batch.host.length):
        x[:] = 0
    rng = np.random.default_rng(t)
    host_commit = batch.host.commit
    batch.host.commit = lambda path, n, *rest: host_commit([p[:t] for p in path], n, *rest)
    for step in range(3 * rows // t + 2):
        path = [(list(range(t)) * 64)[:64], [t - 1] * 64, rng.integers(0, t, 64).tolist(), list(range(t)) + [0] * (64 - t)]
        batch.step(path, [64, 40 + t, 64, max(t - 1, 1)])
    batch.open_rows()
    assert batch.host.length[0] == (3 * rows // t + 2) * t
