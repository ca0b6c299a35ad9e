// hawk_qk_norm_rope and hawk_rope_append: norm of every query and key head, position rotation, and (append) the rows'
// way into the paged cache, in one pass over the data.
//
// Bound by memory: 2 bytes in and 2 out per element, a handful of fp32 operations between, and per row one line of the
// cos/sin table that all heads of the row share.  A head of D elements belongs to D/16 neighbouring lanes, 16 elements
// each as two 16-byte chunks, so the norm's sums are two or three shuffles.  Lane j holds pairs 8j .. 8j+7 of the
// rotation in either pairing (half: chunks j and j + rot/16; interleaved: the 16 elements from 16j on), so a pair never
// crosses lanes and the 8 cosines and 8 sines stay in registers while the lanes walk over the heads of their row.
#include <math_constants.h>

#include "hawk_common.cuh"

namespace {

using namespace hawk;

constexpr int kThreads = 256;

struct RopeParams {
    const void *in[3];         // q, k, v (v: copied)
    void *out[3];              // q_out, k_out or k_pages, v_pages
    long long in_row[3], in_head[3], out_row[3], out_head[3];
    long long out_page[3];     // append: page stride of k_pages and v_pages
    const void *weight[2], *bias[2];
    const int32_t *position;
    const float *cos_sin;
    const int32_t *block_table, *row_begin, *kv_len;
    int heads_end[3];          // heads of q; of q and k; of q, k and v
    int T, norm, per_head, rot, n_positions, interleaved;
    int lanes_per_row, rows_per_block;
    int n_pages, page_size, S, table_width;
    float eps;
    int32_t *dev_status;
};

template <typename T16>
struct Two;
template <>
struct Two<__nv_bfloat16> {
    static __device__ __forceinline__ float2 get(uint32_t x)
    {
        return __bfloat1622float2(*reinterpret_cast<__nv_bfloat162 *>(&x));
    }
    static __device__ __forceinline__ uint32_t put(float a, float b) { return pack_bf16(a, b); }
};
template <>
struct Two<__half> {
    static __device__ __forceinline__ float2 get(uint32_t x) { return __half22float2(*reinterpret_cast<__half2 *>(&x)); }
    static __device__ __forceinline__ uint32_t put(float a, float b)
    {
        __half2 v = __floats2half2_rn(a, b);
        return *reinterpret_cast<uint32_t *>(&v);
    }
};

template <typename T16>
__device__ __forceinline__ void unpack8(const uint4 &u, float *x)
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = Two<T16>::get(w[i]);
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}

template <typename T16>
__device__ __forceinline__ uint4 pack8(const float *x)
{
    return make_uint4(Two<T16>::put(x[0], x[1]), Two<T16>::put(x[2], x[3]), Two<T16>::put(x[4], x[5]),
                      Two<T16>::put(x[6], x[7]));
}

template <typename T16, int D, bool kAppend>
__global__ void __launch_bounds__(kThreads) rope_kernel(const RopeParams P)
{
    constexpr int LH = D / 16;  // lanes of a head
    allow_dependent_launch();
    const int tid = threadIdx.x;
    const int local = tid / P.lanes_per_row, r = tid - local * P.lanes_per_row;
    const int j = r & (LH - 1);            // lanes_per_row is a multiple of LH, so a head's lanes are neighbours
    const int hstep = P.lanes_per_row / LH;
    const long long t_raw = static_cast<long long>(blockIdx.x) * P.rows_per_block + local;
    bool live = local < P.rows_per_block && t_raw < P.T;
    const int t = live ? static_cast<int>(t_raw) : 0;
    const int heads = P.heads_end[2];

    // element offsets of this lane's two chunks
    const int half = P.rot >> 1;
    const bool turns = 16 * j < P.rot;
    const int c0 = P.interleaved || !turns ? 16 * j : 8 * j;
    const int c1 = P.interleaved || !turns ? 16 * j + 8 : half + 8 * j;

    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    int flags = 0;
    auto load = [&](int h, uint4 &a, uint4 &b) {
        a = b = zero;
        if (!live || h >= heads) return;
        const int which = h < P.heads_end[0] ? 0 : h < P.heads_end[1] ? 1 : 2;
        const int hh = h - (which == 0 ? 0 : P.heads_end[which - 1]);
        const T16 *src = static_cast<const T16 *>(P.in[which]) + t * P.in_row[which] + hh * P.in_head[which];
        a = *reinterpret_cast<const uint4 *>(src + c0);
        b = *reinterpret_cast<const uint4 *>(src + c1);
    };
    grid_dependency_wait();
    // the first head's data travel while the row's place and its table line are looked up
    uint4 na, nb;
    load(r / LH, na, nb);

    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        cs[i] = 1.f;
        sn[i] = 0.f;
    }
    if (live && turns) {
        int pos = P.position[t];
        if (pos < 0 || pos >= P.n_positions) {
            flags |= HAWK_DEV_BAD_POSITION;
            pos = max(0, min(pos, P.n_positions - 1));
        }
        const float4 *cp = reinterpret_cast<const float4 *>(P.cos_sin + static_cast<long long>(pos) * P.rot + 8 * j);
        const float4 *sp = reinterpret_cast<const float4 *>(P.cos_sin + static_cast<long long>(pos) * P.rot + half + 8 * j);
        const float4 x0 = cp[0], x1 = cp[1], y0 = sp[0], y1 = sp[1];
        cs[0] = x0.x; cs[1] = x0.y; cs[2] = x0.z; cs[3] = x0.w;
        cs[4] = x1.x; cs[5] = x1.y; cs[6] = x1.z; cs[7] = x1.w;
        sn[0] = y0.x; sn[1] = y0.y; sn[2] = y0.z; sn[3] = y0.w;
        sn[4] = y1.x; sn[5] = y1.y; sn[6] = y1.z; sn[7] = y1.w;
    }

    bool in_cache = true;
    long long page = 0;
    int off = 0;
    if constexpr (kAppend) {
        // stream of the block's first row: how many streams end at or before it (one sweep of the block over row_begin,
        // instead of a search whose every step waits for the last); the few later rows walk on from there
        const int t0 = blockIdx.x * P.rows_per_block;
        int s = 0;
        for (int base = 0; base < P.S; base += kThreads) {
            const int i = base + tid;
            s += __syncthreads_count(i < P.S && P.row_begin[i + 1] <= t0);
        }
        while (s < P.S && P.row_begin[s + 1] <= t) ++s;
        int r0 = 0, r1 = 0;
        if (s < P.S) {
            r0 = P.row_begin[s];
            r1 = P.row_begin[s + 1];
        }
        if (!(r0 >= 0 && r0 <= t && t < r1 && r1 <= P.T)) {
            if (live && s < P.S && (r0 < 0 || r1 > P.T || r0 > r1)) flags |= HAWK_DEV_BAD_ROWS;
            live = false;  // a row of no stream
        }
        if (live) {
            const long long row = static_cast<long long>(P.kv_len[s]) - (r1 - r0) + (t - r0);
            if (row < 0 || row >= static_cast<long long>(P.table_width) * P.page_size) {
                flags |= HAWK_DEV_BAD_PREFIX;
                in_cache = false;
            } else {
                const int pg = static_cast<int>(row / P.page_size);
                off = static_cast<int>(row - static_cast<long long>(pg) * P.page_size);
                page = P.block_table[static_cast<long long>(s) * P.table_width + pg];
                if (page < 0 || page >= P.n_pages) {
                    flags |= HAWK_DEV_BAD_PAGE;
                    in_cache = false;
                }
            }
        }
    }

    const int rounds = (heads + hstep - 1) / hstep;  // the same for all lanes: the shuffles below take part together
    for (int it = 0, h = r / LH; it < rounds; ++it, h += hstep) {
        const uint4 ua = na, ub = nb;
        if (it + 1 < rounds) load(h + hstep, na, nb);
        const int which = h < P.heads_end[0] ? 0 : h < P.heads_end[1] ? 1 : 2;
        const int hh = h - (which == 0 ? 0 : P.heads_end[which - 1]);
        float x[16];
        unpack8<T16>(ua, x);
        unpack8<T16>(ub, x + 8);
        if (P.norm != HAWK_NORM_NONE) {
            if (P.norm == HAWK_NORM_LAYER) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) sum += x[i];
#pragma unroll
                for (int o = LH / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                const float mean = which == 2 ? 0.f : sum * (1.f / D);
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] -= mean;
            }
            float sq = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) sq = fmaf(x[i], x[i], sq);
#pragma unroll
            for (int o = LH / 2; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
            if (which < 2 && live && h < heads) {
                const float inv = rsqrtf(fmaf(sq, 1.f / D, P.eps));
                const long long wo = P.per_head ? static_cast<long long>(hh) * D : 0;
                const T16 *wp = static_cast<const T16 *>(P.weight[which]) + wo;
                float w[16];
                unpack8<T16>(*reinterpret_cast<const uint4 *>(wp + c0), w);
                unpack8<T16>(*reinterpret_cast<const uint4 *>(wp + c1), w + 8);
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = x[i] * inv * w[i];
                if (P.norm == HAWK_NORM_LAYER && P.bias[which]) {
                    const T16 *bp = static_cast<const T16 *>(P.bias[which]) + wo;
                    unpack8<T16>(*reinterpret_cast<const uint4 *>(bp + c0), w);
                    unpack8<T16>(*reinterpret_cast<const uint4 *>(bp + c1), w + 8);
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] += w[i];
                }
            }
        }
        if (!live || h >= heads) continue;
        T16 *dst = static_cast<T16 *>(P.out[which]) + hh * P.out_head[which];
        if (kAppend && which > 0) {
            if (!in_cache) continue;
            dst += page * P.out_page[which] + off * P.out_row[which];
        } else {
            dst += t * P.out_row[which];
        }
        uint4 ya = ua, yb = ub;  // v: the bits as they came
        if (which < 2) {
            if (turns) {
                if (P.interleaved) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float a = x[2 * i], b = x[2 * i + 1];
                        x[2 * i] = a * cs[i] - b * sn[i];
                        x[2 * i + 1] = b * cs[i] + a * sn[i];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float a = x[i], b = x[8 + i];
                        x[i] = a * cs[i] - b * sn[i];
                        x[8 + i] = b * cs[i] + a * sn[i];
                    }
                }
            }
            ya = pack8<T16>(x);
            yb = pack8<T16>(x + 8);
        }
        *reinterpret_cast<uint4 *>(dst + c0) = ya;
        *reinterpret_cast<uint4 *>(dst + c1) = yb;
    }
    if (flags && P.dev_status) atomicOr(P.dev_status, flags);
}

bool strides_ok(long long a, long long b) { return a % 8 == 0 && b % 8 == 0; }

hawk_status check_qk(const hawk_qk_rope_args &a, bool k_dense)
{
    if (a.T < 0 || a.H < 0 || a.H_kv < 0 || a.D < 0 || a.rot_dim < 0 || a.n_positions < 0) return HAWK_ERR_SHAPE;
    if (a.T == 0 || (a.H == 0 && a.H_kv == 0)) return HAWK_OK;
    if ((a.dtype != HAWK_BF16 && a.dtype != HAWK_F16) || a.norm < HAWK_NORM_NONE || a.norm > HAWK_NORM_LAYER)
        return HAWK_ERR_PARAM;
    if (a.norm != HAWK_NORM_NONE && !(a.eps >= 0.f && a.eps <= 3.4e38f)) return HAWK_ERR_PARAM;
    if ((a.D != 64 && a.D != 128) || a.rot_dim % 16 != 0 || a.rot_dim > a.D) return HAWK_ERR_UNSUPPORTED;
    if (a.H > (1 << 16) || a.H_kv > (1 << 16)) return HAWK_ERR_UNSUPPORTED;
    if (a.rot_dim > 0) {
        if (!a.position || !a.cos_sin) return HAWK_ERR_NULL;
        if (a.n_positions == 0) return HAWK_ERR_SHAPE;
        if (!hawk_host::aligned16(a.cos_sin)) return HAWK_ERR_ALIGN;
    }
    for (int w = 0; w < 2; ++w) {
        if ((w ? a.H_kv : a.H) == 0) continue;
        const void *in = w ? a.k : a.q, *out = w ? a.k_out : a.q_out;
        const void *weight = w ? a.k_weight : a.q_weight, *bias = w ? a.k_bias : a.q_bias;
        if (!in || ((w == 0 || k_dense) && !out)) return HAWK_ERR_NULL;
        if (a.norm != HAWK_NORM_NONE && !weight) return HAWK_ERR_NULL;
        if (!hawk_host::aligned16(in) || ((w == 0 || k_dense) && !hawk_host::aligned16(out))) return HAWK_ERR_ALIGN;
        if (a.norm != HAWK_NORM_NONE && (!hawk_host::aligned16(weight) || !hawk_host::aligned16(bias))) return HAWK_ERR_ALIGN;
        if (!(w ? strides_ok(a.k_row_stride, a.k_head_stride) : strides_ok(a.q_row_stride, a.q_head_stride)))
            return HAWK_ERR_ALIGN;
        if (w == 0 ? !strides_ok(a.q_out_row_stride, a.q_out_head_stride)
                   : k_dense && !strides_ok(a.k_out_row_stride, a.k_out_head_stride))
            return HAWK_ERR_ALIGN;
    }
    return HAWK_OK;
}

RopeParams params_of(const hawk_qk_rope_args &a, int32_t *dev_status)
{
    RopeParams P = {};
    P.in[0] = a.q;
    P.in[1] = a.k;
    P.out[0] = a.q_out;
    P.out[1] = a.k_out;
    P.in_row[0] = a.q_row_stride;
    P.in_head[0] = a.q_head_stride;
    P.in_row[1] = a.k_row_stride;
    P.in_head[1] = a.k_head_stride;
    P.out_row[0] = a.q_out_row_stride;
    P.out_head[0] = a.q_out_head_stride;
    P.out_row[1] = a.k_out_row_stride;
    P.out_head[1] = a.k_out_head_stride;
    P.weight[0] = a.q_weight;
    P.weight[1] = a.k_weight;
    P.bias[0] = a.q_bias;
    P.bias[1] = a.k_bias;
    P.position = a.position;
    P.cos_sin = a.cos_sin;
    P.T = a.T;
    P.norm = a.norm;
    P.per_head = a.per_head;
    P.rot = a.rot_dim;
    P.n_positions = a.n_positions;
    P.interleaved = a.interleaved;
    P.eps = a.eps;
    P.dev_status = dev_status;
    P.heads_end[0] = a.H;
    P.heads_end[1] = P.heads_end[2] = a.H + a.H_kv;
    return P;
}

hawk_status launch_rope(RopeParams &P, int D, int dtype, bool append, hawk_stream_t stream)
{
    if (!hawk_host::is_sm100(nullptr)) return HAWK_ERR_UNSUPPORTED;
    // a row's lanes: all heads at once if they fit a block, else the block walks over them in even rounds; rows with
    // few heads share a block
    const int lh = D / 16, heads = P.heads_end[2], fit = kThreads / lh;
    const int rounds = (heads + fit - 1) / fit;
    P.lanes_per_row = (heads + rounds - 1) / rounds * lh;
    P.rows_per_block = kThreads / P.lanes_per_row;
    const dim3 grid(static_cast<unsigned>((static_cast<long long>(P.T) + P.rows_per_block - 1) / P.rows_per_block));
    void (*kernel)(RopeParams);
    const bool bf = dtype == HAWK_BF16;
    if (D == 64)
        kernel = append ? (bf ? rope_kernel<__nv_bfloat16, 64, true> : rope_kernel<__half, 64, true>)
                        : (bf ? rope_kernel<__nv_bfloat16, 64, false> : rope_kernel<__half, 64, false>);
    else
        kernel = append ? (bf ? rope_kernel<__nv_bfloat16, 128, true> : rope_kernel<__half, 128, true>)
                        : (bf ? rope_kernel<__nv_bfloat16, 128, false> : rope_kernel<__half, 128, false>);
    return hawk_host::launch_dependent(kernel, grid, dim3(kThreads), 0, reinterpret_cast<cudaStream_t>(stream), P) ==
                   cudaSuccess
               ? HAWK_OK
               : HAWK_ERR_CUDA;
}

}  // namespace

extern "C" hawk_status hawk_qk_norm_rope(const hawk_qk_rope_args *a, int32_t *dev_status, hawk_stream_t stream)
{
    const hawk_host::NvtxRange nvtx_range("hawk_qk_norm_rope");
    if (!a) return HAWK_ERR_NULL;
    const hawk_status chk = check_qk(*a, true);
    if (chk != HAWK_OK) return chk;
    if (a->T == 0 || (a->H == 0 && a->H_kv == 0)) return HAWK_OK;
    RopeParams P = params_of(*a, dev_status);
    return launch_rope(P, a->D, a->dtype, false, stream);
}

extern "C" hawk_status hawk_rope_append(const hawk_rope_append_args *a, int32_t *dev_status, hawk_stream_t stream)
{
    const hawk_host::NvtxRange nvtx_range("hawk_rope_append");
    if (!a) return HAWK_ERR_NULL;
    if (a->S < 0 || a->n_pages < 0 || a->page_size < 0 || a->table_width < 0) return HAWK_ERR_SHAPE;
    const hawk_status chk = check_qk(a->qk, false);
    if (chk != HAWK_OK) return chk;
    if (a->qk.T == 0 || a->S == 0) return HAWK_OK;
    if (a->qk.H_kv < 1 || a->page_size < 1) return HAWK_ERR_SHAPE;
    if (!a->v || !a->k_pages || !a->v_pages || !a->block_table || !a->row_begin || !a->kv_len) return HAWK_ERR_NULL;
    if (!hawk_host::aligned16(a->v) || !hawk_host::aligned16(a->k_pages) || !hawk_host::aligned16(a->v_pages))
        return HAWK_ERR_ALIGN;
    if (!strides_ok(a->v_row_stride, a->v_head_stride) || !strides_ok(a->k_page_stride, a->k_page_head_stride) ||
        !strides_ok(a->v_page_stride, a->v_page_head_stride) || !strides_ok(a->k_page_row_stride, a->v_page_row_stride))
        return HAWK_ERR_ALIGN;
    RopeParams P = params_of(a->qk, dev_status);
    P.in[2] = a->v;
    P.in_row[2] = a->v_row_stride;
    P.in_head[2] = a->v_head_stride;
    P.out[1] = a->k_pages;
    P.out_row[1] = a->k_page_row_stride;
    P.out_head[1] = a->k_page_head_stride;
    P.out_page[1] = a->k_page_stride;
    P.out[2] = a->v_pages;
    P.out_row[2] = a->v_page_row_stride;
    P.out_head[2] = a->v_page_head_stride;
    P.out_page[2] = a->v_page_stride;
    P.heads_end[2] = a->qk.H + 2 * a->qk.H_kv;
    P.block_table = a->block_table;
    P.row_begin = a->row_begin;
    P.kv_len = a->kv_len;
    P.n_pages = a->n_pages;
    P.page_size = a->page_size;
    P.S = a->S;
    P.table_width = a->table_width;
    return launch_rope(P, a->qk.D, a->qk.dtype, true, stream);
}
