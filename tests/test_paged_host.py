"""Host-side refusals of the calls around the paged cache: every call below is refused (or a no-op) before the library
touches a device, so the pointers are never followed.  And the plain 64-bit forms, against closed forms."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import paged
from paper_2510_25739_b200 import binding, build
from tests._paged import PagedAttnArgs, QkRopeArgs, RopeAppendArgs

OK, E_NULL, E_SHAPE, E_ALIGN, E_UNSUP, E_WS, E_PARAM, E_CUDA = range(8)
P, ODD = 0x1000, 0x1004


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def _qk(**kw):
    a = QkRopeArgs()
    for name, _ in a._fields_:
        if name in ("q", "k", "q_out", "k_out", "q_weight", "k_weight", "q_bias", "k_bias", "position", "cos_sin"):
            setattr(a, name, P)
        elif name.endswith("row_stride"):
            setattr(a, name, 512)
        elif name.endswith("head_stride"):
            setattr(a, name, 64)
    a.T, a.H, a.H_kv, a.D, a.rot_dim, a.n_positions, a.norm, a.eps = 4, 8, 8, 64, 64, 100, 1, 1e-6
    for name, v in kw.items():
        setattr(a, name, v)
    return a


def test_norm_rope_refusals(lib):
    def call(**kw):
        return lib.hawk_qk_norm_rope(ctypes.byref(_qk(**kw)), None, None)

    assert lib.hawk_qk_norm_rope(None, None, None) == E_NULL
    assert call(T=0) == OK and call(H=0, H_kv=0) == OK
    assert call(T=-1) == E_SHAPE and call(n_positions=0) == E_SHAPE
    assert call(q=None) == E_NULL and call(k_out=None) == E_NULL and call(q_weight=None) == E_NULL and call(cos_sin=None) == E_NULL
    assert call(dtype=2) == E_PARAM and call(norm=3) == E_PARAM and call(eps=float("nan")) == E_PARAM and call(eps=-1.0) == E_PARAM
    assert call(D=96) == E_UNSUP and call(rot_dim=24) == E_UNSUP and call(rot_dim=128) == E_UNSUP
    assert call(q=ODD) == E_ALIGN and call(k_out=ODD) == E_ALIGN and call(k_weight=ODD) == E_ALIGN and call(cos_sin=ODD) == E_ALIGN
    assert call(q_row_stride=100) == E_ALIGN and call(k_out_head_stride=4) == E_ALIGN


def _append(**kw):
    a = RopeAppendArgs()
    a.qk = _qk(**kw.pop("qk", {}))
    for name, _ in a._fields_:
        if name in ("v", "k_pages", "v_pages", "block_table", "row_begin", "kv_len"):
            setattr(a, name, P)
        elif name.endswith("_stride"):
            setattr(a, name, 64)
    a.n_pages, a.page_size, a.S, a.table_width = 10, 16, 2, 3
    for name, v in kw.items():
        setattr(a, name, v)
    return a


def test_append_refusals(lib):
    def call(**kw):
        return lib.hawk_rope_append(ctypes.byref(_append(**kw)), None, None)

    assert lib.hawk_rope_append(None, None, None) == E_NULL
    assert call(S=0) == OK and call(qk=dict(T=0)) == OK
    assert call(S=-1) == E_SHAPE and call(page_size=0) == E_SHAPE and call(qk=dict(H_kv=0)) == E_SHAPE
    assert call(v=None) == E_NULL and call(k_pages=None) == E_NULL and call(row_begin=None) == E_NULL and call(qk=dict(k=None)) == E_NULL
    assert call(v=ODD) == E_ALIGN and call(v_pages=ODD) == E_ALIGN and call(k_page_row_stride=12) == E_ALIGN
    assert call(v_page_stride=12) == E_ALIGN and call(qk=dict(D=32)) == E_UNSUP and call(qk=dict(norm=-1)) == E_PARAM


def _attn(**kw):
    a = PagedAttnArgs()
    for name, _ in a._fields_:
        if name in ("q", "k_pages", "v_pages", "block_table", "row_begin", "kv_len", "out"):
            setattr(a, name, P)
        elif name.endswith("_stride"):
            setattr(a, name, 64)
    a.S, a.T, a.max_new, a.max_kv, a.H, a.H_kv, a.D, a.n_pages, a.page_size, a.table_width = 2, 10, 5, 160, 8, 8, 64, 20, 16, 10
    a.sm_scale = 0.125
    a.workspace, a.workspace_bytes = P, 1 << 40
    for name, v in kw.items():
        setattr(a, name, v)
    return a


def test_attn_refusals(lib):
    def call(**kw):
        return lib.hawk_paged_attn(ctypes.byref(_attn(**kw)), None, None)

    assert lib.hawk_paged_attn(None, None, None) == E_NULL
    assert call(S=0) == OK and call(T=0) == OK and call(max_new=0) == OK
    assert call(S=-1) == E_SHAPE and call(max_kv=-1) == E_SHAPE and call(max_kv=161) == E_SHAPE and call(n_pages=0) == E_SHAPE
    for name in ("q", "k_pages", "v_pages", "block_table", "row_begin", "kv_len", "out"):
        assert call(**{name: None}) == E_NULL
    assert call(dtype=7) == E_PARAM and call(sm_scale=0.0) == E_PARAM and call(sm_scale=float("nan")) == E_PARAM
    assert call(sm_scale=float("inf")) == E_PARAM
    assert call(D=96) == E_UNSUP and call(H=9) == E_UNSUP and call(H=129 * 8) == E_UNSUP and call(page_size=20) == E_UNSUP
    assert call(S=4097) == E_UNSUP and call(anc_mask=P, max_new=65, T=200) == E_UNSUP
    assert call(q=ODD) == E_ALIGN and call(out=ODD) == E_ALIGN and call(q_row_stride=68) == E_ALIGN and call(v_page_row_stride=4) == E_ALIGN
    assert call(q_row_stride=-64) == E_UNSUP
    need = lib.hawk_paged_attn_workspace_bytes(64, 512, 8, 8, 8, 64, 160)
    big = dict(S=64, T=512, max_new=8)
    assert need > 0 and call(workspace_bytes=need - 1, **big) == E_WS and call(workspace=None, **big) == E_WS
    assert call(workspace=0x1008, **big) == E_ALIGN


def test_attn_workspace(lib):
    ws = lib.hawk_paged_attn_workspace_bytes
    assert ws(0, 10, 5, 8, 8, 64, 160) == 0 and ws(2, 10, 5, 9, 8, 64, 160) == 0 and ws(2, 10, 5, 8, 8, 96, 160) == 0
    assert ws(2, 2, 1, 16, 16, 64, 129) == 0       # short items, a warp each
    assert ws(16, 80, 5, 20, 20, 64, 1149) == 0    # merged inside the block
    assert ws(128, 1024, 8, 20, 20, 64, 1032) > 0  # shares
    # more rows never need less
    sizes = [ws(3, 400, n, 4, 2, 64, 900) for n in (1, 8, 20, 33, 64, 65, 100, 400)]
    assert all(s >= 0 for s in sizes)
    # few query tiles over many keys: partial results of the key splits
    assert ws(1, 200, 200, 4, 2, 64, 8000) > ws(1, 200, 200, 4, 2, 64, 500)


def test_struct_fields_match_the_header():
    """Names and order of the argument structs against include/hawk.h."""
    import re
    from pathlib import Path
    text = (Path(__file__).resolve().parent.parent / "include" / "hawk.h").read_text()
    for struct, cls in (("hawk_qk_rope_args", QkRopeArgs), ("hawk_rope_append_args", RopeAppendArgs),
                        ("hawk_paged_attn_args", PagedAttnArgs)):
        body = re.search(r"typedef struct " + struct + r" \{(.*?)\} " + struct + ";", text, re.S).group(1)
        names = []
        for decl in re.sub(r"/\*.*?\*/", "", body, flags=re.S).split(";"):
            decl = re.sub(r"^\s*(const\s+)?(void|float|int32_t|uint64_t|int|size_t|long long|hawk_qk_rope_args)\b", "", decl.strip())
            names += [p.replace("*", "").strip() for p in decl.split(",") if p.strip()]
        assert names == [f[0] for f in cls._fields_]


def test_python_refusals():
    """Types, shapes, devices: refused before the library is called."""
    q = torch.zeros((2, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        binding.qk_norm_rope(q, q, None, None)
    with pytest.raises(ValueError, match="one of them"):
        binding.qk_norm_rope(None, None, None, None)
    with pytest.raises(ValueError, match="CUDA"):
        binding.paged_attn(q, q, q, q, q, q, 1, 1, 1.0)


# ---- the plain forms
def test_plain_rotation_is_a_rotation():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((4, 2, 8))
    angle = rng.uniform(0, 6, (9, 4))
    table = np.concatenate([np.cos(angle), np.sin(angle)], 1)
    for inter in (False, True):
        y, _ = paged.norm_rope(x, [0, 3, 8, 3], table, interleaved=inter)
        z = (x[..., 0::2] + 1j * x[..., 1::2]) if inter else (x[..., :4] + 1j * x[..., 4:])
        z = z * np.exp(1j * angle[[0, 3, 8, 3]])[:, None, :]
        want = np.stack([z.real, z.imag], -1).reshape(x.shape) if inter else np.concatenate([z.real, z.imag], -1)
        assert np.allclose(y, want, atol=1e-14)


def test_plain_norms():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 2, 16)) * 4 + 1
    y, _ = paged.norm_rope(x, None, None, "rms", 0.0, np.ones(16))
    assert np.allclose((y ** 2).mean(-1), 1)
    y, _ = paged.norm_rope(x, None, None, "layer", 0.0, np.ones(16), np.full(16, 0.5))
    assert np.allclose(y.mean(-1), 0.5) and np.allclose(y.var(-1), 1)


def test_plain_attention_closed_forms():
    rng = np.random.default_rng(2)
    kp, vp = rng.standard_normal((5, 1, 4, 8)), rng.standard_normal((5, 1, 4, 8))
    table = np.array([[3, 0, 4]])
    flat = np.concatenate([vp[3, 0], vp[0, 0], vp[4, 0]])
    # no queries' preference: the running mean of the values
    out, _ = paged.paged_attn(np.zeros((3, 1, 8)), kp, vp, table, [0, 3], [10], 1.0)
    for i in range(3):
        assert np.allclose(out[i, 0], flat[:8 + i].mean(0))
    # a chain's mask is the chain; a row without keys is zero; rows of nobody stay unset
    q = rng.standard_normal((4, 1, 8))
    a, _ = paged.paged_attn(q, kp, vp, table, [0, 3], [10], 0.3)
    b, _ = paged.paged_attn(q, kp, vp, table, [0, 3], [10], 0.3, [1, 3, 7])
    assert np.array_equal(a[:3], b[:3]) and np.isnan(a[3]).all()
    c, _ = paged.paged_attn(q, kp, vp, table, [0, 3], [2], 0.3)
    assert (c[0] == 0).all() and np.allclose(c[1, 0], flat[0])
