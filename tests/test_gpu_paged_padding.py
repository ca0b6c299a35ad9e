"""hawk_paged_attn on padded batches: rows that belong to no stream, in front and behind, hold large finite numbers (memory that
nobody wrote is as good as that).  They are loaded with the rows of the streams beside them and must not take part in anything.
Every kernel and launch shape; bounds as in test_gpu_paged_attn.py."""
import numpy as np
import pytest
import torch

from tests._paged import Batch
from tests.test_gpu_paged_attn import _binary_tree, _check, _run

pytestmark = pytest.mark.gpu

SHAPES = [
    ("a block per item, 8 warps", [4] * 8, [300] * 8, 4, 4, 64),
    ("a block per item, 4 warps", [5] * 16, [300] * 16, 20, 20, 64),
    ("equal shares of warps", [8] * 40, [200] * 40, 20, 20, 64),
    ("equal shares of wider items", [20] * 64, [200] * 64, 20, 20, 128),
    ("equal shares of blocks, single tokens", [1] * 7, [3000] * 7, 8, 2, 128),
    ("equal shares of blocks, single tokens at D = 64", [1, 0, 1], [5000, 9, 3111], 2, 2, 64),
    ("equal shares of blocks, 16 rows", [12, 9], [3000, 2000], 2, 2, 128),
    ("equal shares of blocks, 32 rows", [3, 5], [3000, 2000], 10, 2, 64),
    ("equal shares of blocks, 64 rows", [60, 41], [3000, 2000], 2, 2, 64),
    ("chunks, two query tiles", [300], [400], 2, 2, 128),
    ("chunks, one query tile", [100], [400], 2, 2, 64),
    ("chunks split over the keys", [100], [3000], 2, 2, 128),
    ("chunks and single tokens", [150, 1, 3], [400, 700, 90], 4, 2, 64),
]


@pytest.mark.parametrize("dtype,poison", [("bf16", 1e30), ("bf16", -3e10), ("fp16", 6e4)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: s[0])
def test_large_numbers_in_rows_of_no_stream(shape, dtype, poison):
    _, new, kv, H, H_kv, D = shape
    _check(Batch(new, kv, H, H_kv, D, 16, dtype, seed=90, front=5, back=70, poison=poison))


@pytest.mark.parametrize("n,H,H_kv,D", [(22, 2, 2, 128), (40, 1, 1, 64), (20, 12, 2, 64)])
def test_large_numbers_beside_a_tree(n, H, H_kv, D):
    _check(Batch([n, n // 2], [n + 2000, n // 2 + 1500], H, H_kv, D, 16, seed=91, back=70, poison=1e30), _binary_tree(n))


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: s[0])
def test_results_do_not_depend_on_rows_of_others(shape):
    """Bit for bit the same whatever the rows of no stream hold, and whatever the last stream's queries are for the others."""
    _, new, kv, H, H_kv, D = shape
    b = Batch(new, kv, H, H_kv, D, 16, seed=96, front=5, back=130, poison=0.0)
    begin, end = int(b.row_begin[0]), int(b.row_begin[-1])
    first, _ = _run(b)
    rows = torch.randn((b.T, H, D), generator=torch.Generator().manual_seed(97))
    for scale in (1.0, 30.0, 1e30):
        q = (rows * scale).to(b.dt)
        q[begin:end] = b.q[begin:end]
        b.q = q
        got, status = _run(b)
        assert status == 0 and np.array_equal(first[begin:end], got[begin:end])
    last = int(b.row_begin[-2])
    b.q[last:end] = (rows[last:end] * 30).to(b.dt)
    got, status = _run(b)
    assert status == 0 and np.array_equal(first[begin:last], got[begin:last])
