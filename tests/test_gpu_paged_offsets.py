"""Calls around the paged cache whose rows reach past 2^31 elements: queries, results and cache places behind that bound."""
import numpy as np
import pytest
import torch

from oracle import paged
from tests._paged import f64, half_step, rope_table

pytestmark = pytest.mark.gpu

ROWS, HEADS, D = 140_000, 128, 128  # 2.3 * 10^9 elements


@pytest.fixture(scope="module")
def rows():
    x = torch.empty((ROWS, HEADS, D), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(6)
    for at in range(0, ROWS, 10_000):
        x[at:at + 10_000].normal_(generator=g)
    yield x
    del x
    torch.cuda.empty_cache()


def test_norm_rope(rows):
    """The last rows of a long call are those of a call of their own, bit for bit; keys and values land far into the cache."""
    import paper_2510_25739_b200 as hawk
    w = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    table, position = rope_table(50, D).cuda(), (torch.arange(ROWS, device="cuda") % 50).int()
    tail = rows[-40:].clone()
    want, _ = hawk.qk_norm_rope(tail, None, position[-40:].contiguous(), table, norm="rms", q_weight=w)
    got, _ = hawk.qk_norm_rope(rows, None, position, table, norm="rms", q_weight=w)
    assert torch.equal(got[-40:], want)
    first, _ = hawk.qk_norm_rope(rows[:40], None, position[:40].contiguous(), table, norm="rms", q_weight=w)
    assert torch.equal(got[:40], first)
    pages = torch.zeros((17_500, HEADS, 8, D), dtype=torch.bfloat16, device="cuda")
    bt = torch.arange(17_500, dtype=torch.int32, device="cuda")[None, :]
    begin, kv = torch.tensor([0, ROWS], dtype=torch.int32, device="cuda"), torch.tensor([ROWS], dtype=torch.int32, device="cuda")
    del got
    hawk.rope_append(None, rows, rows, None, None, pages, pages, bt, begin, kv)
    assert torch.equal(pages[-1].transpose(0, 1), rows[-8:]) and torch.equal(pages[0].transpose(0, 1), rows[:8])


@pytest.mark.parametrize("n,H_kv", [(40, 128), (140, 128), (4, 8), (1, 128)])
def test_attention(rows, n, H_kv):
    """Streams of n rows and as many keys and a few: the first and the last against the plain form."""
    import paper_2510_25739_b200 as hawk
    S = min(ROWS // n, 4000)
    front = ROWS - S * n  # rows in front belong to nobody
    kv, page = n + 5, 16
    need = -(-kv // page)
    g = torch.Generator(device="cuda").manual_seed(n)
    kp, vp = (torch.empty((3 * need, H_kv, page, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2))
    bt = torch.stack([torch.arange(need) + need * (s % 3) for s in range(S)]).int().cuda()
    begin = (front + n * torch.arange(S + 1)).int().cuda()
    lens = torch.full((S,), kv, dtype=torch.int32, device="cuda")
    out = torch.full((ROWS, HEADS * D), 7.0, dtype=torch.bfloat16, device="cuda")
    hawk.paged_attn(rows, kp, vp, bt, begin, lens, n, kv, D ** -0.5, out=out)
    h = half_step(torch.bfloat16)
    assert front == 0 or (out[:front:997] == 7.0).all()
    for s in (0, S // 2, S - 1):
        r = slice(front + s * n, front + (s + 1) * n)
        want, size = paged.paged_attn(f64(rows[r]), f64(kp), f64(vp), bt[s:s + 1].cpu().numpy(), [0, n], [kv], D ** -0.5)
        got = f64(out[r]).reshape(n, HEADS, D)
        assert (np.abs(got - want) <= h * np.abs(want) + (h + 2.0 ** -11) * size).all()  # derived in test_gpu_paged_attn.py
