"""hawk_paged_attn on scores that rise or fall over the keys, in every launch shape of the kernel for few rows: a row's shift moves again
and again, with it every sum and accumulator, and the partial results that the joins fold have very different maxima.  (The same
for the other kernels: test_gpu_paged_shapes.py.)  The workspace's size tells the launch shape, so that each case says
which one it is for.  Bounds as in test_gpu_paged_attn.py."""
import pytest
import torch

from paper_2510_25739_b200 import binding
from tests._paged import Batch
from tests.test_gpu_paged_attn import _binary_tree, _check

pytestmark = pytest.mark.gpu

SMS, RECORD = 148, 32


def _shape(b):
    """Launch shape of the streams of few rows, from the workspace's size: ("group", 0) or ("shares", rows an item), with the other
    kernels' sizes refused."""
    group = b.H // b.H_kv
    few = min(b.max_new, b.T) * group
    size = binding.paged_attn_workspace_bytes(b.S, b.T, b.max_new, b.H, b.H_kv, b.D, b.max_kv)
    if few > 64:  # behind it the list of the chunk kernel: smaller than any of the sizes' differences
        lists = size
        for rpi in (8, 16, 24, 32):
            share = SMS * (12 if rpi == 8 else 8) * (RECORD + 2 * rpi * (b.D + 2) * 4)
            if 0 <= lists - share < 65536:
                return "shares", rpi
        raise AssertionError(size)
    if size == 0:
        return "group", 0
    assert size != SMS * (RECORD + 2 * 64 * (b.D + 2) * 4), "the 64-row kernel"
    for rpi in (8, 16, 24, 32):
        if size == SMS * (12 if rpi == 8 else 8) * (RECORD + 2 * rpi * (b.D + 2) * 4):
            return "shares", rpi
    raise AssertionError(size)


def _rising(b, seed=0):
    """Scores grow by 24 over a stream's keys, or fall by as much in every second stream, with noise on top."""
    g = torch.Generator().manual_seed(seed)
    base = torch.randint(0, 2, (b.D,), generator=g).float() * 2 - 1
    b.q = (base + 0.1 * torch.randn(b.q.shape, generator=g)).to(b.dt)
    for s, kv in enumerate(b.kv):
        at = torch.arange(kv) / max(kv, 1)
        ramp = 24 * b.D ** -0.5 * (at if s % 2 == 0 else 1 - at)
        keys = base * ramp[:, None] + 0.1 * torch.randn((b.H_kv, kv, b.D), generator=g)
        for j in range(b.need[s]):
            rows = min(b.page, kv - j * b.page)
            b.k_pages[int(b.block_table[s, j]), :, :rows] = keys[:, j * b.page:j * b.page + rows].to(b.dt)
    worst = 0
    for s, kv in enumerate(b.kv):
        ids, rows = b.block_table[s, :b.need[s]].long(), slice(int(b.row_begin[s]), int(b.row_begin[s + 1]))
        for h in range(b.H):
            keys = b.k_pages[ids, h // (b.H // b.H_kv)].reshape(-1, b.D)[:kv].float().abs()
            worst = max(worst, float((b.q[rows, h].float().abs() @ keys.T).max()) * b.D ** -0.5)
    assert worst * b.D < 4096  # D 2^-24 sum |q k| scale below 2^-12, as the bounds count it
    return b


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("new,kv,H,H_kv,D,shape", [
    ([4] * 8, [700] * 8, 4, 4, 64, ("group", 0)),               # 8 warps an item
    ([3] * 6, [400] * 6, 8, 8, 128, ("group", 0)),
    ([20] * 4, [600] * 4, 4, 4, 64, ("group", 0)),              # items of three column tiles
    ([5] * 16, [500] * 16, 20, 20, 64, ("group", 0)),           # 4 warps an item
    ([6] * 12, [400] * 12, 32, 32, 128, ("group", 0)),
    ([8] * 40, [333] * 40, 20, 20, 64, ("shares", 8)),
    ([7] * 30, [290] * 30, 20, 20, 128, ("shares", 8)),
    ([12] * 8, [900] * 8, 20, 20, 64, ("shares", 16)),
    ([14] * 31, [300] * 31, 20, 20, 128, ("shares", 16)),
    ([20] * 8, [700] * 8, 20, 20, 64, ("shares", 24)),
    ([20] * 31, [384] * 31, 20, 20, 128, ("shares", 24)),
    ([30] * 8, [1600] * 8, 20, 20, 64, ("shares", 32)),
    ([40] * 16, [500] * 16, 20, 20, 64, ("shares", 24)),        # two items a stream and head
    ([8, 1, 5, 8] * 5 + [140], [900, 700, 400, 33] * 5 + [300], 8, 8, 64, ("shares", 32)),   # beside a chunk
    ([22, 1, 9, 3] * 4 + [130], [900, 500, 300, 60] * 4 + [200], 4, 4, 128, ("shares", 24)),
])
def test_every_shape_of_the_rows_kernel(new, kv, H, H_kv, D, shape, dtype):
    b = Batch(new, kv, H, H_kv, D, 16, dtype, seed=100, back=3)
    assert _shape(b) == shape
    _check(_rising(b))


@pytest.mark.parametrize("n,S,kv,H,D,shape", [(7, 8, 300, 4, 64, ("group", 0)), (22, 30, 384, 20, 128, ("shares", 24)), (31, 8, 1500, 20, 64, ("shares", 32))])
def test_trees(n, S, kv, H, D, shape):
    b = Batch([n] * S, [n + kv] * S, H, H, D, 16, seed=101)
    assert _shape(b) == shape
    _check(_rising(b), _binary_tree(n))
