"""Host-side refusals of hawk_sample and hawk_pages_*: every call below is refused (or a no-op) before the library touches a device, so the
pointers are never followed.  And the plain 64-bit forms, against closed forms and invariants."""
import ctypes
import re
from pathlib import Path

import numpy as np
import pytest
import torch

from oracle import serving
from paper_2510_25739_b200 import binding, build
from tests import _serving as sv

OK, E_NULL, E_SHAPE, E_ALIGN, E_UNSUP, E_WS, E_PARAM, E_CUDA = range(8)
P, Q, ODD = 0x1000, 0x2000, 0x1004
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def _filled(cls, names, **kw):
    a = cls()
    for n in names:
        setattr(a, n, P)
    for n, v in kw.items():
        setattr(a, n, v)
    return a


def test_struct_fields_match_the_header():
    text = (Path(__file__).resolve().parent.parent / "include" / "hawk.h").read_text()
    for struct, cls in (("hawk_sample_args", sv.SampleArgs), ("hawk_pages_resize_args", sv.ResizeArgs), ("hawk_pages_fork_args", sv.ForkArgs),
                        ("hawk_pages_compact_args", sv.CompactArgs), ("hawk_page_tensors", sv.PageTensors),
                        ("hawk_pages_keep_args", sv.KeepArgs)):
        body = re.search(r"typedef struct " + struct + r" \{(.*?)\} " + struct + ";", text, re.S).group(1)
        names = []
        for decl in re.sub(r"/\*.*?\*/", "", body, flags=re.S).split(";"):
            decl = re.sub(r"^\s*(const\s+)?(void|float|int32_t|uint64_t|int|size_t|long long|hawk_page_tensors)\b", "", decl.strip())
            names += [p.replace("*", "").strip() for p in decl.split(",") if p.strip()]
        assert names == [f[0] for f in cls._fields_]


def test_sample_refusals(lib):
    def call(**kw):
        base = dict(dtype=2, R=3, V=100, v_begin=0, v_end=100, temperature=1.0, top_p=1.0, min_p=0.0, cfg_scale=1.0, row_stride=100,
                    uncond_row_stride=100, probs_row_stride=100)
        a = _filled(sv.SampleArgs, ("logits", "u", "token"), **{**base, **kw})
        return lib.hawk_sample(ctypes.byref(a), None, None)

    assert lib.hawk_sample(None, None, None) == E_NULL
    assert call(R=0) == OK and call(R=0, dtype=9) == OK
    assert call(R=-1) == E_SHAPE and call(v_end=101) == E_SHAPE and call(v_begin=-1) == E_SHAPE and call(v_begin=60, v_end=50) == E_SHAPE
    assert call(row_stride=-1) == E_SHAPE and call(uncond=P, uncond_row_stride=-4) == E_SHAPE and call(probs=P, probs_row_stride=99) == E_SHAPE
    for name in ("logits", "u", "token"):
        assert call(**{name: None}) == E_NULL
    assert call(dtype=3) == E_PARAM and call(dtype=-1) == E_PARAM
    assert call(temperature=-0.5) == E_PARAM and call(temperature=NAN) == E_PARAM and call(temperature=INF) == E_PARAM
    assert call(top_p=NAN) == E_PARAM and call(min_p=NAN) == E_PARAM
    assert call(uncond=P, cfg_scale=NAN) == E_PARAM and call(uncond=P, cfg_scale=INF) == E_PARAM
    assert call(v_begin=7, v_end=7) == E_UNSUP and call(V=300000, v_end=262145) == E_UNSUP and call(R=1 << 29) == E_UNSUP
    assert call(logits=0x1002) == E_ALIGN and call(probs=0x1002) == E_ALIGN and call(dtype=0, logits=0x1001) == E_ALIGN


def _resize(**kw):
    names = ("block_table", "kv_len", "new_len", "page_refs", "out_table", "out_len", "out_refs", "copies")
    return _filled(sv.ResizeArgs, names, **{**dict(S=2, table_width=4, n_pages=9, page_size=16), **kw})


def test_resize_refusals(lib):
    def call(**kw):
        return lib.hawk_pages_resize(ctypes.byref(_resize(**kw)), None, None)

    assert lib.hawk_pages_resize(None, None, None) == E_NULL
    assert call(S=0) == OK
    assert call(S=-1) == E_SHAPE and call(page_size=0) == E_SHAPE and call(n_pages=-1) == E_SHAPE and call(table_width=-2) == E_SHAPE
    for name in ("block_table", "kv_len", "new_len", "page_refs", "out_table", "out_len", "out_refs", "copies"):
        assert call(**{name: None}) == E_NULL
    assert call(S=4097) == E_UNSUP and call(n_pages=(1 << 20) + 1) == E_UNSUP and call(page_size=65537) == E_UNSUP
    assert call(S=4096, table_width=1 << 19) == E_UNSUP and call(table_width=1 << 16, page_size=1 << 15) == E_UNSUP
    assert call(page_refs=ODD) == E_ALIGN and call(out_refs=ODD) == E_ALIGN


def test_fork_refusals(lib):
    def call(**kw):
        names = ("block_table", "kv_len", "page_refs", "parent", "length", "out_refs")
        base = dict(S=2, S_out=3, table_width=4, n_pages=9, page_size=16, out_table=Q, out_len=Q)
        return lib.hawk_pages_fork(ctypes.byref(_filled(sv.ForkArgs, names, **{**base, **kw})), None, None)

    assert lib.hawk_pages_fork(None, None, None) == E_NULL
    assert call(S=0, S_out=0) == OK
    assert call(S_out=-1) == E_SHAPE and call(page_size=-3) == E_SHAPE
    for name in ("block_table", "kv_len", "page_refs", "parent", "out_table", "out_len", "out_refs"):
        assert call(**{name: None}) == E_NULL
    assert call(out_table=P) == E_PARAM and call(out_len=P) == E_PARAM
    assert call(S=4097) == E_UNSUP and call(S_out=4097) == E_UNSUP and call(out_refs=ODD) == E_ALIGN


def test_compact_refusals(lib):
    def call(**kw):
        names = ("block_table", "kv_len", "page_refs", "out_table", "out_refs", "copies", "top", "workspace")
        base = dict(S=2, table_width=4, n_pages=9, page_size=16, first_page=0, max_moves=3, workspace_bytes=1 << 30)
        return lib.hawk_pages_compact(ctypes.byref(_filled(sv.CompactArgs, names, **{**base, **kw})), None, None)

    ws = lib.hawk_pages_compact_workspace_bytes
    assert lib.hawk_pages_compact(None, None, None) == E_NULL
    assert call(max_moves=-1) == E_SHAPE and call(first_page=-1) == E_SHAPE and call(first_page=10) == E_SHAPE and call(n_pages=0) == E_SHAPE
    for name in ("block_table", "kv_len", "page_refs", "out_table", "out_refs", "copies"):
        assert call(**{name: None}) == E_NULL
    assert call(n_pages=(1 << 20) + 1) == E_UNSUP and call(max_moves=(1 << 20) + 1) == E_UNSUP
    assert call(workspace=None) == E_WS and call(workspace_bytes=ws(9, 3) - 1) == E_WS and call(workspace=0x1008) == E_ALIGN
    assert ws(0, 5) == 0 and ws(5, -1) == 0 and ws((1 << 20) + 1, 5) == 0
    assert ws(100, 0) > 0 and ws(100, 1000) == ws(100, 100) > ws(100, 10)


def _tensors(**kw):
    a = sv.PageTensors(layers=2, n_pages=9, H_kv=4, page_size=16, D=64, k_pages=P, v_pages=P)
    for n, _ in a._fields_:
        if n.endswith("_stride"):
            setattr(a, n, 64)
    for n, v in kw.items():
        setattr(a, n, v)
    return a


def test_copy_refusals(lib):
    def call(copies=P, n=3, **kw):
        return lib.hawk_pages_copy(ctypes.byref(_tensors(**kw)), copies, n, None, None)

    assert lib.hawk_pages_copy(None, P, 3, None, None) == E_NULL
    assert call(n=0) == OK and call(layers=0) == OK and call(n=0, D=7) == OK
    assert call(n=-1) == E_SHAPE and call(layers=-1) == E_SHAPE and call(H_kv=0) == E_SHAPE and call(n_pages=0) == E_SHAPE
    assert call(copies=None) == E_NULL and call(k_pages=None) == E_NULL and call(v_pages=None) == E_NULL
    assert call(D=12) == E_UNSUP and call(page_size=65537) == E_UNSUP and call(layers=32768) == E_UNSUP
    assert call(H_kv=65536, page_size=512) == E_UNSUP
    assert call(k_pages=ODD) == E_ALIGN and call(v_row_stride=68) == E_ALIGN and call(k_layer_stride=4) == E_ALIGN


def test_keep_refusals(lib):
    def call(pages=None, **kw):
        names = ("block_table", "row_begin", "kv_len", "path", "accept_len")
        a = _filled(sv.KeepArgs, names, **{**dict(S=4, B=2, table_width=4, path_width=3, first=1, out_len=Q), **kw})
        a.pages = _tensors(**(pages or {}))
        return lib.hawk_pages_keep(ctypes.byref(a), None, None)

    assert lib.hawk_pages_keep(None, None, None) == E_NULL
    assert call(S=0) == OK
    assert call(S=-1) == E_SHAPE and call(B=3) == E_SHAPE and call(B=0) == E_SHAPE and call(first=-1) == E_SHAPE and call(path_width=-1) == E_SHAPE
    for name in ("block_table", "row_begin", "kv_len", "accept_len", "out_len"):
        assert call(**{name: None}) == E_NULL
    assert call(out_len=P) == E_PARAM
    assert call(pages=dict(D=10)) == E_UNSUP and call(pages=dict(k_pages=None)) == E_NULL and call(pages=dict(v_pages=ODD)) == E_ALIGN


def test_python_refusals():
    x = torch.zeros((2, 8))
    i = torch.zeros((2, 4), dtype=torch.int32)
    for call in (lambda: binding.sample(x, x[0]), lambda: binding.pages_resize(i, i[0], i[0], i[0], 16),
                 lambda: binding.pages_fork(i, i[0], i[0], i[0], 16), lambda: binding.pages_compact(i, i[0], i[0], 16, 3),
                 lambda: binding.pages_copy(x.bfloat16(), x.bfloat16(), i), lambda: binding.pages_keep(None, None, None, i[0], i[0], None, i[0])):
        with pytest.raises(ValueError, match="CUDA"):
            call()


# ---- the plain forms
def test_plain_sampling_closed_forms():
    l = np.log([0.5, 0.25, 0.125, 0.125])
    for u, want in ((0.0, 0), (0.49, 0), (0.51, 1), (0.76, 2), (0.88, 3), (0.999, 3)):
        assert serving.sample_row(l, u)[0] == want
    assert serving.sample_row(l, 0.9, top_k=1)[0] == 0
    assert np.allclose(serving.sample_row(l, 0.9, top_k=2)[1], [2 / 3, 1 / 3, 0, 0])
    assert np.allclose(serving.sample_row(l, 0.9, top_k=3)[1], np.exp(l))          # ties with the third stay
    assert np.allclose(serving.sample_row(l, 0.9, top_p=0.6)[1], [2 / 3, 1 / 3, 0, 0])
    assert np.allclose(serving.sample_row(l, 0.9, top_p=0.8)[1], np.exp(l))
    assert np.allclose(serving.sample_row(l, 0.9, min_p=0.4)[1], [2 / 3, 1 / 3, 0, 0])
    assert np.allclose(serving.sample_row(l, 0.9, top_p=0.0)[1], [1, 0, 0, 0]) and np.allclose(serving.sample_row(l, 0.9, min_p=1.0)[1], [1, 0, 0, 0])
    assert np.allclose(serving.sample_row(l, 0.9, temperature=0.5)[1], np.exp(2 * l) / np.exp(2 * l).sum())
    assert serving.sample_row(l[::-1].copy(), 0.5, temperature=0.0)[0] == 3 and serving.sample_row([1.0, 3.0, 3.0], 0.9, temperature=0.0)[0] == 1
    assert serving.sample_row([-np.inf, np.nan, np.inf], 0.5)[0] == -1
    assert serving.sample_row([-np.inf, 2.0, np.nan], 0.0)[0] == 1


def test_plain_sampling_draws_from_its_probabilities():
    rng = np.random.default_rng(3)
    l = rng.standard_normal(12) * 2
    _, p, _ = serving.sample_row(l, 0.5, 0.8, 9, 0.95, 0.01)
    hits = np.bincount([serving.sample_row(l, (i + 0.5) / 4000, 0.8, 9, 0.95, 0.01)[0] for i in range(4000)], minlength=12)
    assert np.abs(hits / 4000 - p).max() <= 1 / 4000 + 1e-12  # an even grid of numbers: each id gets its share to a step


def test_plain_guidance():
    c, u = np.float32([1.5, -np.inf, 2.0, np.nan]), np.float32([0.5, 1.0, -np.inf, 0.0])
    got = serving.guided_logits(c, u, 3.0)
    assert got[0] == 3.5 and np.isneginf(got[1:]).all()


@pytest.mark.parametrize("seed", range(6))
def test_plain_pages_keep_their_counts(seed):
    """A long run of the plain forms: after each call the counts are those of the entries in use, and what streams see is what they wrote."""
    r = np.random.RandomState(seed)
    page, width, n_pages = int(r.randint(1, 9)), 12, 40
    st = sv.PageState(r.randint(0, page * 5 + 1, 5).tolist(), page, width, n_pages, share=2, seed=seed)
    table, lens, refs = st.table, list(st.lens), list(st.refs)
    content = {p: [object() for _ in range(page)] for p in range(n_pages)}

    def seen():
        return [[content[table[s][j // page]][j % page] for j in range(n)] for s, n in enumerate(lens)]

    def merge(out):
        return [[o if o is not None else t for o, t in zip(a, b)] for a, b in zip(out, table + [[-7] * width] * len(out))]

    for step in range(12):
        before = seen()
        what = step % 3
        if what == 0:
            new = [int(np.clip(n + r.randint(-2 * page, 2 * page + 1), 0, width * page)) for n in lens]
            out, got, refs, copies, _ = serving.resize(table, lens, new, refs, page)
            for a, b, n in copies:
                if a >= 0:
                    content[b][:n] = content[a][:n]
            table, old, lens = merge(out), lens, got
            after = seen()
            for s in range(len(lens)):
                assert after[s][:min(old[s], lens[s])] == before[s][:lens[s]]
        elif what == 1:
            parent = r.randint(-1, len(lens), len(lens) + int(r.randint(-1, 2))).tolist()
            length = r.randint(0, width * page, len(parent)).tolist()
            out, got, refs = serving.fork(table, lens, parent, refs, page, length)
            table, lens = merge(out), got
            assert all(a == (before[p][:n] if p >= 0 else []) for a, p, n in zip(seen(), parent, lens))
        else:
            out, refs, copies, top = serving.compact(table, lens, refs, page, 5)
            for a, b, n in copies:
                if a >= 0:
                    content[b][:n] = content[a][:n]
            table = merge(out)
            assert seen() == before and not any(refs[top:]) and (top == 0 or refs[top - 1] > 0)
        count = [0] * n_pages
        for s, n in enumerate(lens):
            for j in range(serving.pages(n, page)):
                count[table[s][j]] += 1
        assert count == refs


def test_plain_keep():
    lens, moves = serving.keep([0, 5, 5, 10], [20, 7, 30], [[2, 4], [-1, -1], [1, 3]], [2, 0, 1], 1)
    assert lens == [15 + 3, 7, 25 + 2] and moves == [(0, 17, 16), (0, 19, 17), (2, 26, 26)]
    assert serving.keep([0, 4], [10], None, [4], 1)[0] == [10]  # the last draft's row was never brought


# ---- bases that 32-bit elements cannot have (followed, they would fault)
@pytest.mark.parametrize("name", ["u", "token", "token_prob", "probs", "row_temperature", "row_top_k", "row_top_p", "row_min_p", "row_cfg_scale"])
def test_sample_refuses_misaligned_bases(lib, name):
    for off in (1, 2, 3):
        a = _filled(sv.SampleArgs, ("logits", "u", "token"), dtype=2, R=3, V=100, v_begin=0, v_end=100, temperature=1.0, top_p=1.0, cfg_scale=1.0,
                    row_stride=100, probs_row_stride=100, **{name: P + off})
        assert lib.hawk_sample(ctypes.byref(a), None, None) == E_ALIGN


def test_page_calls_refuse_misaligned_bases(lib):
    def fork(**kw):
        names = ("block_table", "kv_len", "page_refs", "parent", "length", "out_refs")
        base = dict(S=2, S_out=3, table_width=4, n_pages=9, page_size=16, out_table=Q, out_len=Q)
        return lib.hawk_pages_fork(ctypes.byref(_filled(sv.ForkArgs, names, **{**base, **kw})), None, None)

    def compact(**kw):
        names = ("block_table", "kv_len", "page_refs", "out_table", "out_refs", "copies", "top", "workspace")
        base = dict(S=2, table_width=4, n_pages=9, page_size=16, first_page=0, max_moves=3, workspace_bytes=1 << 30)
        return lib.hawk_pages_compact(ctypes.byref(_filled(sv.CompactArgs, names, **{**base, **kw})), None, None)

    def keep(**kw):
        names = ("block_table", "row_begin", "kv_len", "path", "accept_len")
        a = _filled(sv.KeepArgs, names, **{**dict(S=4, B=2, table_width=4, path_width=3, first=1, out_len=Q), **kw})
        a.pages = _tensors()
        return lib.hawk_pages_keep(ctypes.byref(a), None, None)

    for off in (1, 2, 3):
        for name in ("block_table", "kv_len", "new_len", "out_table", "out_len", "copies"):
            assert lib.hawk_pages_resize(ctypes.byref(_resize(**{name: P + off})), None, None) == E_ALIGN
        for name in ("block_table", "kv_len", "parent", "length", "out_table", "out_len"):
            assert fork(**{name: P + off}) == E_ALIGN
        for name in ("block_table", "kv_len", "out_table", "copies", "top"):
            assert compact(**{name: P + off}) == E_ALIGN
        assert lib.hawk_pages_copy(ctypes.byref(_tensors()), P + off, 3, None, None) == E_ALIGN
        for name in ("block_table", "row_begin", "kv_len", "path", "accept_len", "out_len"):
            assert keep(**{name: P + off}) == E_ALIGN


def test_only_tensors_with_elements_have_to_be_there(lib):
    """Without a GPU: a call that lacks a tensor without elements gets past the NULLs (here to the refusal of what comes behind them)."""
    assert lib.hawk_pages_resize(ctypes.byref(_resize(table_width=0, block_table=None, out_table=None, page_refs=ODD)), None, None) == E_ALIGN
    a = _filled(sv.ForkArgs, ("kv_len", "page_refs", "parent"), S=2, S_out=3, table_width=0, n_pages=9, page_size=16, out_len=Q, out_refs=ODD)
    assert lib.hawk_pages_fork(ctypes.byref(a), None, None) == E_ALIGN
    a = _filled(sv.CompactArgs, ("kv_len", "page_refs", "out_refs", "copies"), S=2, table_width=0, n_pages=9, page_size=16, max_moves=3)
    assert lib.hawk_pages_compact(ctypes.byref(a), None, None) == E_WS
    a = _filled(sv.KeepArgs, ("row_begin", "kv_len", "path", "accept_len"), S=4, B=2, table_width=0, path_width=3, first=1, out_len=Q)
    a.pages = _tensors(layers=0, k_pages=None, v_pages=None, k_row_stride=4)
    assert lib.hawk_pages_keep(ctypes.byref(a), None, None) == E_ALIGN
