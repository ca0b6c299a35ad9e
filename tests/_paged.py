"""Ragged batches over a paged cache for the tests of the calls around it (inputs only, no arithmetic of the method)."""
import ctypes

import numpy as np
import torch

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


class Batch:
    """S streams with new[s] rows and kv[s] keys; pages handed out in random order; everything nobody owns is NaN: pages of
    no stream, page rows behind a stream's last key, rows of the call that belong to no stream (`front` and `back` of them)."""

    def __init__(self, new, kv, H, H_kv, D, page, dtype="bf16", seed=0, layout="hrd", front=0, back=0, packed=False, spare=3,
                 poison=float("nan")):
        g = torch.Generator().manual_seed(seed)
        self.dt = dt = DTYPES[dtype]
        self.new, self.kv, self.H, self.H_kv, self.D, self.page = list(new), list(kv), H, H_kv, D, page
        S = self.S = len(new)
        begin = np.concatenate([[front], front + np.cumsum(new)]).astype(np.int32)
        self.T = int(begin[-1]) + back
        self.row_begin = torch.from_numpy(begin)
        self.kv_len = torch.tensor(kv, dtype=torch.int32)
        need = [-(-l // page) if n else 0 for n, l in zip(new, kv)]
        width = max(1, -(-max(kv + [1]) // page))
        n_pages = sum(need) + spare
        order = torch.randperm(n_pages, generator=g)
        table = torch.full((S, width), -7, dtype=torch.int32)  # entries past the last used page hold nonsense
        at = 0
        for s in range(S):
            table[s, :need[s]] = order[at:at + need[s]].int()
            at += need[s]
        self.block_table, self.n_pages, self.need = table, n_pages, need

        def pages():
            x = torch.full((n_pages, H_kv, page, D), poison).to(dt)
            for s in range(S):
                for j in range(need[s]):
                    rows = min(page, kv[s] - j * page)
                    x[int(table[s, j]), :, :rows] = torch.randn((H_kv, rows, D), generator=g).to(dt)
            return x

        self.k_pages, self.v_pages = pages(), pages()
        heads = H + 2 * H_kv
        qkv = torch.randn((self.T, heads, D), generator=g).to(dt)
        qkv[:front] = poison
        qkv[int(begin[-1]):] = poison
        self.q, self.k, self.v = qkv[:, :H], qkv[:, H:H + H_kv], qkv[:, H + H_kv:]
        if not packed:
            self.q, self.k, self.v = self.q.contiguous(), self.k.contiguous(), self.v.contiguous()
        self.packed, self.layout = packed, layout
        self.max_new, self.max_kv = max(list(new) + [1]), max([l for n, l in zip(new, kv) if n] + [0])

    def cuda(self):
        """The tensors on the GPU, pages in the batch's layout: "hrd" heads before rows, "rhd" rows before heads, "kv" keys
        and values of a page in one buffer."""
        b = type("OnGpu", (), {})()
        if self.packed:
            whole = torch.cat([self.q, self.k, self.v], 1).cuda()
            b.q, b.k, b.v = whole[:, :self.H], whole[:, self.H:self.H + self.H_kv], whole[:, self.H + self.H_kv:]
        else:
            b.q, b.k, b.v = self.q.cuda(), self.k.cuda(), self.v.cuda()
        b.row_begin, b.kv_len, b.block_table = self.row_begin.cuda(), self.kv_len.cuda(), self.block_table.cuda()
        if self.layout == "rhd":
            b.k_pages = self.k_pages.transpose(1, 2).contiguous().cuda().transpose(1, 2)
            b.v_pages = self.v_pages.transpose(1, 2).contiguous().cuda().transpose(1, 2)
        elif self.layout == "kv":
            both = torch.stack([self.k_pages, self.v_pages], 1).cuda()
            b.k_pages, b.v_pages = both[:, 0], both[:, 1]
        else:
            b.k_pages, b.v_pages = self.k_pages.cuda(), self.v_pages.cuda()
        return b


def f64(t):
    return t.detach().double().cpu().numpy()


def half_step(dtype):
    """Largest relative error of one rounding to the type."""
    return torch.finfo(dtype).eps / 2


def rope_table(positions, rot, grid=0, seed=None):
    """fp32 [positions, rot]: cosines, then sines; one axis, or (grid columns) half of the angles by row and half by column."""
    half = rot // 2
    at = np.arange(positions, dtype=np.float64)
    if grid:
        f = 10000.0 ** (-np.arange(half // 2) / (half // 2))
        angle = np.concatenate([np.outer(at // grid, f), np.outer(at % grid, f)], 1)
    else:
        angle = np.outer(at, 10000.0 ** (-np.arange(half) / half))
    return torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32))


# ---- the argument structs of include/hawk.h, for the tests of the C ABI's refusals
class QkRopeArgs(ctypes.Structure):
    """Mirror of hawk_qk_rope_args (include/hawk.h)."""
    _fields_ = ([(n, ctypes.c_int) for n in ("dtype", "T", "H", "H_kv", "D", "norm", "per_head", "rot_dim", "n_positions",
                                             "interleaved")]
                + [("eps", ctypes.c_float)]
                + [(n, ctypes.c_void_p) for n in ("q", "k", "q_out", "k_out")]
                + [(f"{t}_{w}_stride", ctypes.c_longlong) for t in ("q", "k", "q_out", "k_out") for w in ("row", "head")]
                + [(n, ctypes.c_void_p) for n in ("q_weight", "k_weight", "q_bias", "k_bias", "position", "cos_sin")])


_PAGE_STRIDES = [(f"{t}_{w}_stride", ctypes.c_longlong) for t in "kv" for w in ("page", "page_head", "page_row")]


class RopeAppendArgs(ctypes.Structure):
    """Mirror of hawk_rope_append_args (include/hawk.h)."""
    _fields_ = ([("qk", QkRopeArgs), ("v", ctypes.c_void_p), ("v_row_stride", ctypes.c_longlong),
                 ("v_head_stride", ctypes.c_longlong), ("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p)]
                + _PAGE_STRIDES + [(n, ctypes.c_int) for n in ("n_pages", "page_size", "S", "table_width")]
                + [(n, ctypes.c_void_p) for n in ("block_table", "row_begin", "kv_len")])


class PagedAttnArgs(ctypes.Structure):
    """Mirror of hawk_paged_attn_args (include/hawk.h)."""
    _fields_ = ([(n, ctypes.c_int) for n in ("dtype", "S", "T", "max_new", "max_kv", "H", "H_kv", "D", "n_pages", "page_size",
                                             "table_width")]
                + [("sm_scale", ctypes.c_float), ("q", ctypes.c_void_p), ("q_row_stride", ctypes.c_longlong),
                   ("q_head_stride", ctypes.c_longlong), ("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p)]
                + _PAGE_STRIDES
                + [(n, ctypes.c_void_p) for n in ("block_table", "row_begin", "kv_len", "anc_mask", "out", "workspace")]
                + [("workspace_bytes", ctypes.c_size_t)])
