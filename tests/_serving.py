"""States of a paged cache and rows of logits for the tests of sampling and of the page calls (inputs only, no arithmetic of the method),
and mirrors of their argument structs."""
import ctypes

import numpy as np
import torch

from oracle import serving


class PageState:
    """A block table, lengths and reference counts that agree: streams in groups of `share` start with the pages of their group's first
    stream, some up to their last page (just forked).  `held` pages have a count of the caller's own on top."""

    def __init__(self, lens, page, width, n_pages, share=1, seed=0, held=(), fresh=0.5):
        r = np.random.RandomState(seed)
        S = len(lens)
        self.page, self.n_pages = page, n_pages
        table = np.full((S, width), -7, np.int64)  # entries that are not in use hold nonsense
        ids = [p for p in r.permutation(n_pages) if p not in held]
        lens = list(lens)
        for s in range(S):
            need, first = serving.pages(lens[s], page), s - s % share
            shared = 0
            if s != first:
                common = min(lens[s], lens[first])
                shared = common // page
                if r.rand() < fresh:  # just forked: the same length, the partly filled page too
                    lens[s] = lens[first]
                    need = shared = serving.pages(lens[s], page)
                table[s, :shared] = table[first, :shared]
            for j in range(shared, need):
                table[s, j] = ids.pop()
        refs = np.zeros(n_pages, np.int64)
        for s in range(S):
            for j in range(serving.pages(lens[s], page)):
                refs[table[s, j]] += 1
        for p in held:
            refs[p] += 1
        self.lens, self.table, self.refs = lens, table.tolist(), refs.tolist()

    def cuda(self):
        return int32(self.table), int32(self.lens), int32(self.refs)


def int32(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def same_where_written(got, want):
    """The entries that the plain form wrote."""
    got = got.cpu().tolist()
    return all(w is None or g == w for a, b in zip(got, want) for g, w in zip(a, b))


def check_counts(table, lens, refs, page, held=()):
    """Every count is the number of entries in use that name the page."""
    refs = refs.cpu().numpy().copy()
    table, lens = table.cpu().numpy(), lens.cpu().numpy()
    for p in held:
        refs[p] -= 1
    for s in range(len(lens)):
        for j in range(serving.pages(int(lens[s]), page)):
            refs[table[s, j]] -= 1
    return not refs.any()


def pages_tensor(layers, n_pages, H, page, D, dtype=torch.bfloat16, layout="hrd", seed=0):
    """(k, v) [layers, n_pages, H, page, D] on the GPU in a layout: heads before rows, rows before heads, or keys and values of a page in one
    buffer; layers 0: without the first dimension."""
    g = torch.Generator().manual_seed(seed)
    L = max(1, layers)
    k, v = (torch.randn((L, n_pages, H, page, D), generator=g).to(dtype) for _ in range(2))
    if layout == "rhd":
        k, v = (x.transpose(2, 3).contiguous().cuda().transpose(2, 3) for x in (k, v))
    elif layout == "kv":
        both = torch.stack([k, v], 2).cuda()
        k, v = both[:, :, 0], both[:, :, 1]
    else:
        k, v = k.cuda(), v.cuda()
    return (k[0], v[0]) if layers == 0 else (k, v)


def exact_sample(logits, u, cfg_scale=None, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, begin=0, end=None):
    """serving.sample_row for each row: (token, prob, probs, margin, z of each id).  Settings are numbers or lists."""
    x = logits.float().cpu().numpy()
    end = x.shape[1] if end is None else end
    R = len(x) // (2 if cfg_scale is not None else 1)

    def each(v, r):
        v = v[r] if isinstance(v, (list, tuple, np.ndarray)) else v
        return float(np.float32(v))

    token, prob, probs, margin, zs = [], [], np.zeros((R, x.shape[1])), [], np.zeros((R, x.shape[1]))
    for r in range(R):
        l = x[r, begin:end]
        if cfg_scale is not None:
            l = serving.guided_logits(l, x[R + r, begin:end], each(cfg_scale, r))
        l = l.astype(np.float64)
        T = each(temperature, r)
        at, p, m = serving.sample_row(l, float(u[r]), T, int(each(top_k, r)), each(top_p, r), each(min_p, r))
        token.append(at + begin if at >= 0 else -1)
        prob.append(p[at] if at >= 0 else 0.0)
        probs[r, begin:end] = p
        margin.append(m)
        with np.errstate(invalid="ignore"):
            top = l[np.isfinite(l)].max() if np.isfinite(l).any() else 0.0
            z = (np.where(np.isfinite(l), l, top) - top) / (T if T > 0 else 1.0)
        zs[r, begin:end] = np.clip(z, -1e4, 0)
    return np.array(token), np.array(prob), probs, np.array(margin), zs


def prob_bound(p, z):
    """How far a probability in fp32 may be off: the rounding of l - max (half a step of a value of size |z| * T, so |z| * 2^-24 in the exponent
    times ln 2 in base 2, over ln 2 back), ex2.approx (2^-22), three multiplications and the factor's rounding (2^-22 together with
    what is left of the product's second part); weights below e^-32 of the largest count as 0."""
    return p * (np.abs(z) * 2.0 ** -23 + 2.0 ** -21) + np.exp(-31.9) + 1e-38


class SampleArgs(ctypes.Structure):
    """Mirror of hawk_sample_args (include/hawk.h)."""
    _fields_ = ([(n, ctypes.c_int) for n in ("dtype", "R", "V", "v_begin", "v_end", "top_k")]
                + [(n, ctypes.c_float) for n in ("temperature", "top_p", "min_p", "cfg_scale")]
                + [(n, ctypes.c_void_p) for n in ("logits", "uncond")]
                + [(n, ctypes.c_longlong) for n in ("row_stride", "uncond_row_stride")]
                + [(n, ctypes.c_void_p) for n in ("row_temperature", "row_top_p", "row_min_p", "row_cfg_scale", "row_top_k", "u", "token",
                                                  "token_prob", "probs")]
                + [("probs_row_stride", ctypes.c_longlong)])


class ResizeArgs(ctypes.Structure):
    """Mirror of hawk_pages_resize_args."""
    _fields_ = ([(n, ctypes.c_int) for n in ("S", "table_width", "n_pages", "page_size")]
                + [(n, ctypes.c_void_p) for n in ("block_table", "kv_len", "new_len", "page_refs", "out_table", "out_len", "out_refs", "copies")])


class ForkArgs(ctypes.Structure):
    """Mirror of hawk_pages_fork_args."""
    _fields_ = ([(n, ctypes.c_int) for n in ("S", "S_out", "table_width", "n_pages", "page_size")]
                + [(n, ctypes.c_void_p) for n in ("block_table", "kv_len", "page_refs", "parent", "length", "out_table", "out_len", "out_refs")])


class CompactArgs(ctypes.Structure):
    """Mirror of hawk_pages_compact_args."""
    _fields_ = ([(n, ctypes.c_int) for n in ("S", "table_width", "n_pages", "page_size", "first_page", "max_moves")]
                + [(n, ctypes.c_void_p) for n in ("block_table", "kv_len", "page_refs", "out_table", "out_refs", "copies", "top", "workspace")]
                + [("workspace_bytes", ctypes.c_size_t)])


class PageTensors(ctypes.Structure):
    """Mirror of hawk_page_tensors."""
    _fields_ = ([(n, ctypes.c_int) for n in ("layers", "n_pages", "H_kv", "page_size", "D")]
                + [(n, ctypes.c_void_p) for n in ("k_pages", "v_pages")]
                + [(f"{t}_{w}_stride", ctypes.c_longlong) for t in "kv" for w in ("layer", "page", "head", "row")])


class KeepArgs(ctypes.Structure):
    """Mirror of hawk_pages_keep_args."""
    _fields_ = ([("pages", PageTensors)] + [(n, ctypes.c_int) for n in ("S", "B", "table_width", "path_width", "first")]
                + [(n, ctypes.c_void_p) for n in ("block_table", "row_begin", "kv_len", "path", "accept_len", "out_len")])
