// hawk_qk_norm_rope and hawk_rope_append: norm of every query and key head, position rotation, and (append) the rows'
// way into the paged cache, in one pass over the data.
//
// Bound by memory: 2 bytes in and 2 out per element, a handful of fp32 operations between, and per row one line of the
// cos/sin table that all heads of the row share.  A head of D elements belongs to D/16 neighbouring lanes, 16 elements
// each as two 16-byte chunks, so the norm's sums are two or three shuffles.  Lane j holds pairs 8j .. 8j+7 of the
// rotation in either pairing (half: chunks j and j + rot/16; interleaved: the 16 elements from 16j on), so a pair never
// crosses lanes, and arithmetic runs on pairs of fp32 numbers (one instruction for two).
// A block owns a run of rows, as many as make the grid one wave (few rows: one pass, latency counts).  It first looks up, a
// thread a row, where the rows go (stream, page) and copies their table lines to shared memory.  Then a lane keeps one head
// (its weights in registers, one pointer in and one out) and goes down the rows with the loads of the next two under way,
// before it takes its next head.  (Rows outside, heads inside, was bound by instruction issue: 365 a 16-element piece with a
// layer norm, for pointers, weights and selections that this order hoists; 40 us against 31 for 4.7 k rows of 64 heads of 128.)
#include <type_traits>

#include "hawk_common.cuh"

namespace {

using namespace hawk;

constexpr int kThreads = 256;
constexpr int kBlocksPerSm = 2;

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
    int lanes_per_row, par, run;  // lanes of a row, rows a block has in hand at once, rows a block owns (a multiple of par)
    int n_pages, page_size, S, table_width;
    float eps;
    int32_t *dev_status;
};

template <typename T16>
__device__ __forceinline__ uint64_t unpack16(uint32_t x)  // two elements as a pair of fp32
{
    float2 f;
    if constexpr (sizeof(T16) == 2 && __is_same(T16, __nv_bfloat16)) f = __bfloat1622float2(*reinterpret_cast<__nv_bfloat162 *>(&x));
    else f = __half22float2(*reinterpret_cast<__half2 *>(&x));
    return pack2(f.x, f.y);
}

template <typename T16>
__device__ __forceinline__ uint32_t pack16(uint64_t v)
{
    const float2 f = unpack2(v);
    if constexpr (__is_same(T16, __nv_bfloat16)) return pack_bf16(f.x, f.y);
    const __half2 h = __floats2half2_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t *>(&h);
}

template <typename T16>
__device__ __forceinline__ void unpack8(const uint4 &u, uint64_t *x)
{
    x[0] = unpack16<T16>(u.x);
    x[1] = unpack16<T16>(u.y);
    x[2] = unpack16<T16>(u.z);
    x[3] = unpack16<T16>(u.w);
}

template <typename T16>
__device__ __forceinline__ uint4 pack8(const uint64_t *x)
{
    return make_uint4(pack16<T16>(x[0]), pack16<T16>(x[1]), pack16<T16>(x[2]), pack16<T16>(x[3]));
}

constexpr int kMaxRun = 64;  // rows of a block (one row a lane; runs of several rows a lane end at 32)

// Where a row of the block goes.
struct Place {
    int page, off;  // page id and row in it; page < 0: not into the cache
};

// kDirect: one row a lane (the block's run is what it has in hand at once); a lane reads its table line itself, straight
// from memory, which spares small calls a barrier and a trip through shared memory.
template <typename T16, int D, bool kAppend, int kNorm, bool kDirect>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) rope_kernel(const RopeParams P)
{
    constexpr int LH = D / 16;  // lanes of a head
    extern __shared__ float4 lines[];  // cos | sin of the block's rows: [run][rot]
    __shared__ Place place[kMaxRun];
    __shared__ int hist[kMaxRun], owned[kMaxRun], line_of[kMaxRun];
    allow_dependent_launch();
    const int tid = threadIdx.x;
    const int local = tid / P.lanes_per_row, r = tid - local * P.lanes_per_row;
    const int j = r & (LH - 1);  // lanes_per_row is a multiple of LH, so a head's lanes are neighbours
    const int hstep = P.lanes_per_row / LH;
    const int heads = P.heads_end[2], rounds = (heads + hstep - 1) / hstep;
    const long long t0 = static_cast<long long>(blockIdx.x) * P.run;
    const int rows = static_cast<int>(min(static_cast<long long>(P.run), P.T - t0));

    // element offsets of this lane's two chunks
    const int half = P.rot >> 1;
    const bool turns = 16 * j < P.rot;
    const int c0 = P.interleaved || !turns ? 16 * j : 8 * j;
    const int c1 = P.interleaved || !turns ? 16 * j + 8 : half + 8 * j;

    const int passes = (rows + P.par - 1) / P.par;  // rows local, local + par, ... of the block are this lane's
    auto tensor_of = [&](int h) { return h < P.heads_end[0] ? 0 : h < P.heads_end[1] ? 1 : 2; };

    // loads run ahead of the arithmetic by two rows, over the end of one head into the next
    const T16 *l_src = nullptr;
    long long l_step = 0;
    int l_pass = 0, l_round = 0;
    bool l_live = false;
    auto aim = [&]() {
        const int h = l_round * hstep + r / LH;
        l_live = local < P.par && h < heads;
        if (!l_live) return;
        const int which = tensor_of(h);
        const int hh = h - (which == 0 ? 0 : P.heads_end[which - 1]);
        l_step = P.in_row[which] * P.par;
        l_src = static_cast<const T16 *>(P.in[which]) + (t0 + local) * P.in_row[which] + hh * P.in_head[which];
    };
    struct Piece {
        uint4 a, b;
    };
    auto fetch = [&](Piece &p) {
        p.a = p.b = make_uint4(0u, 0u, 0u, 0u);
        if (l_live && local + l_pass * P.par < rows) {
            p.a = *reinterpret_cast<const uint4 *>(l_src + c0);
            p.b = *reinterpret_cast<const uint4 *>(l_src + c1);
        }
        l_src += l_step;
        if (++l_pass == passes) {
            l_pass = 0;
            ++l_round;
            aim();
        }
    };
    grid_dependency_wait();
    Piece p0, p1;
    aim();
    fetch(p0);
    fetch(p1);
    int flags = 0;
    auto line_at = [&](int row) {
        int pos = P.position[t0 + row];
        if (pos < 0 || pos >= P.n_positions) {
            flags |= HAWK_DEV_BAD_POSITION;
            pos = max(0, min(pos, P.n_positions - 1));
        }
        return pos;
    };
    const bool reads_line = kDirect && turns && local < P.par && local < rows;
    const int own_line = reads_line ? line_at(local) : 0;
    if (!kAppend && kDirect && flags && P.dev_status) atomicOr(P.dev_status, flags);
    flags = 0;

    // ---- the block's rows: place and table line
    if constexpr (kAppend) {
        // stream of row t0 + i: how many streams end at or before it, counted by all threads in one sweep over row_begin
        if (tid < kMaxRun) hist[tid] = 0;
        __syncthreads();
        int gone = 0;
        for (int s = tid; s < P.S; s += kThreads) {
            const long long e = P.row_begin[s + 1] - t0;
            if (e <= 0) ++gone;
            else if (e < rows) atomicAdd(&hist[e], 1);
        }
        gone = __reduce_add_sync(0xffffffffu, gone);
        if ((tid & 31) == 0 && gone) atomicAdd(&hist[0], gone);
        __syncthreads();
    }
    if ((kAppend || !kDirect) && tid < rows) {
        [[maybe_unused]] const int t = static_cast<int>(t0) + tid;
        if (P.rot > 0) line_of[tid] = line_at(tid);  // (a bad position of a row of no stream is forgotten below)
        if constexpr (kAppend) {
            int s = 0;
            for (int i = 0; i <= tid; ++i) s += hist[i];
            int r0 = 0, r1 = 0;
            if (s < P.S) {
                r0 = P.row_begin[s];
                r1 = P.row_begin[s + 1];
            }
            const bool mine = r0 >= 0 && r0 <= t && t < r1 && r1 <= P.T;
            Place pl = {-1, 0};
            if (mine) {
                const long long row = static_cast<long long>(P.kv_len[s]) - (r1 - r0) + (t - r0);
                if (row < 0 || row >= static_cast<long long>(P.table_width) * P.page_size) {
                    flags |= HAWK_DEV_BAD_PREFIX;
                } else {
                    const int pg = static_cast<int>(row / P.page_size);
                    pl.off = static_cast<int>(row - static_cast<long long>(pg) * P.page_size);
                    pl.page = P.block_table[static_cast<long long>(s) * P.table_width + pg];
                    if (pl.page < 0 || pl.page >= P.n_pages) {
                        flags |= HAWK_DEV_BAD_PAGE;
                        pl.page = -1;
                    }
                }
            } else {
                flags = s < P.S && (r0 < 0 || r1 > P.T || r0 > r1) ? HAWK_DEV_BAD_ROWS : 0;
            }
            place[tid] = pl;
            owned[tid] = mine;
        }
        if (flags && P.dev_status) atomicOr(P.dev_status, flags);
    }
    if (kAppend || !kDirect) __syncthreads();
    if (!kDirect && P.rot > 0) {
        const int per = P.rot >> 2;  // 16-byte pieces of a line
        for (int i = tid; i < rows * per; i += kThreads) {
            const int row = i / per, c = i - row * per;
            lines[i] = reinterpret_cast<const float4 *>(P.cos_sin)[static_cast<long long>(line_of[row]) * per + c];
        }
        __syncthreads();
    }

    // ---- the heads, one after the other, down the rows.  All lanes of a warp go through the loops together (the shuffles
    // below), those without a head or a row idle
    for (int round = 0; round < rounds; ++round) {
        const int h = round * hstep + r / LH;
        const bool has_head = local < P.par && h < heads;
        const int which = tensor_of(h);
        const int hh = h - (which == 0 ? 0 : P.heads_end[which - 1]);
        uint64_t w[8], bias[8];
        bool has_bias = false;
        if (kNorm != HAWK_NORM_NONE && which < 2 && has_head) {
            const long long wo = P.per_head ? static_cast<long long>(hh) * D : 0;
            const T16 *wp = static_cast<const T16 *>(P.weight[which]) + wo;
            unpack8<T16>(*reinterpret_cast<const uint4 *>(wp + c0), w);
            unpack8<T16>(*reinterpret_cast<const uint4 *>(wp + c1), w + 4);
            if (kNorm == HAWK_NORM_LAYER && P.bias[which]) {
                const T16 *bp = static_cast<const T16 *>(P.bias[which]) + wo;
                unpack8<T16>(*reinterpret_cast<const uint4 *>(bp + c0), bias);
                unpack8<T16>(*reinterpret_cast<const uint4 *>(bp + c1), bias + 4);
                has_bias = true;
            }
        }
        T16 *const out = static_cast<T16 *>(P.out[which]) + hh * P.out_head[which];
        const long long out_row = P.out_row[which], out_page = P.out_page[which];
        const bool to_cache = kAppend && which > 0;

        auto work = [&](int row, Piece &p) {
            const bool live = has_head && row < rows;
            uint64_t x[8];
            if (which < 2) {
                unpack8<T16>(p.a, x);
                unpack8<T16>(p.b, x + 4);
            }
            const uint4 ua = p.a, ub = p.b;
            fetch(p);
            if constexpr (kNorm != HAWK_NORM_NONE) {
                if (which >= 2) {  // v takes part in the shuffles only
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = 0;
                }
                if constexpr (kNorm == HAWK_NORM_LAYER) {
                    const float2 sf = unpack2(
                        add2(add2(add2(x[0], x[1]), add2(x[2], x[3])), add2(add2(x[4], x[5]), add2(x[6], x[7]))));
                    float sum = sf.x + sf.y;
#pragma unroll
                    for (int o = LH / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                    const float mean = sum * (-1.f / D);
                    const uint64_t m2 = pack2(mean, mean);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = add2(x[i], m2);
                }
                uint64_t q0 = mul2(x[0], x[0]), q1 = mul2(x[1], x[1]);
#pragma unroll
                for (int i = 2; i < 8; i += 2) {
                    q0 = fma2(x[i], x[i], q0);
                    q1 = fma2(x[i + 1], x[i + 1], q1);
                }
                const float2 qf = unpack2(add2(q0, q1));
                float sq = qf.x + qf.y;
#pragma unroll
                for (int o = LH / 2; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
                const float inv = rsqrtf(fmaf(sq, 1.f / D, P.eps));
                const uint64_t inv2 = pack2(inv, inv);
                if (has_bias) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = fma2(mul2(x[i], inv2), w[i], bias[i]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = mul2(mul2(x[i], inv2), w[i]);
                }
            }
            if (!live) return;
            T16 *dst;
            if constexpr (kAppend) {
                if (!owned[row]) return;
                if (to_cache) {
                    const Place pl = place[row];
                    if (pl.page < 0) return;
                    dst = out + pl.page * out_page + pl.off * out_row;
                } else {
                    dst = out + (t0 + row) * out_row;
                }
            } else {
                dst = out + (t0 + row) * out_row;
            }
            uint4 ya = ua, yb = ub;  // v: the bits as they came
            if (which < 2) {
                if (turns) {
                    const int per = P.rot >> 2, at = 2 * j, to_sin = half >> 2;
                    const float4 *line;  // (never one pointer for both kinds: that would make the loads generic ones)
                    if constexpr (kDirect) line = reinterpret_cast<const float4 *>(P.cos_sin) + static_cast<long long>(own_line) * per + at;
                    else line = lines + row * per + at;
                    const float4 ca = line[0], cb = line[1], sa = line[to_sin], sb = line[to_sin + 1];
                    const uint64_t cs[4] = {pack2(ca.x, ca.y), pack2(ca.z, ca.w), pack2(cb.x, cb.y), pack2(cb.z, cb.w)};
                    const uint64_t sn[4] = {pack2(sa.x, sa.y), pack2(sa.z, sa.w), pack2(sb.x, sb.y), pack2(sb.z, sb.w)};
                    if (P.interleaved) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {  // pair i: cosine i, the (i & 1)th of its couple
                            const float2 ab = unpack2(x[i]), c2 = unpack2(cs[i >> 1]), s2 = unpack2(sn[i >> 1]);
                            const float c = i & 1 ? c2.y : c2.x, s = i & 1 ? s2.y : s2.x;
                            x[i] = pack2(ab.x * c - ab.y * s, ab.y * c + ab.x * s);
                        }
                    } else {
                        const uint64_t minus = pack2(-1.f, -1.f);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint64_t a = x[i], b = x[4 + i];
                            x[i] = fma2(mul2(b, sn[i]), minus, mul2(a, cs[i]));
                            x[4 + i] = fma2(a, sn[i], mul2(b, cs[i]));
                        }
                    }
                }
                ya = pack8<T16>(x);
                yb = pack8<T16>(x + 4);
            }
            *reinterpret_cast<uint4 *>(dst + c0) = ya;
            *reinterpret_cast<uint4 *>(dst + c1) = yb;
        };
        for (int i = 0; i < passes; i += 2) {
            work(local + i * P.par, p0);
            if (i + 1 < passes) work(local + (i + 1) * P.par, p1);
        }
        if (passes & 1) {  // the pieces under way have changed places
            const Piece t = p0;
            p0 = p1;
            p1 = t;
        }
    }
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

// The formula of HAWK_NORM_RMS has no bias: one that is given is refused, not dropped.
bool has_stray_bias(const hawk_qk_rope_args &a)
{
    return a.norm == HAWK_NORM_RMS && ((a.H > 0 && a.q_bias) || (a.H_kv > 0 && a.k_bias));
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
    // a row's lanes: its heads in even rounds, as few as fit a block, or up to three more where that leaves fewer lanes
    // without work (48 heads of 128: 3 rounds of 2 x 128 lanes, not 2 of 192); rows with few heads share a block
    const int lh = D / 16, heads = P.heads_end[2], fit = kThreads / lh;
    const int least = (heads + fit - 1) / fit;
    int best = 0;
    for (int rounds = least; rounds <= least + 3 && rounds <= heads; ++rounds) {
        const int lanes = (heads + rounds - 1) / rounds * lh;
        const int par = kThreads / lanes < kMaxRun ? kThreads / lanes : kMaxRun;
        const int used = static_cast<int>(1000ll * par * heads * lh / (static_cast<long long>(kThreads) * rounds));
        // (more rounds have to gain a tenth; a call of few rows has nothing to gain)
        if (rounds == least || (used > best + best / 10 && P.T >= 2 * 148)) {
            best = used;
            P.lanes_per_row = lanes;
            P.par = par;
        }
    }
    // a block's run of rows: the grid is one wave where that needs no more rows than shared memory holds table lines for
    const long long wave = static_cast<long long>(kBlocksPerSm) * 148 * P.par;
    long long passes = (P.T + wave - 1) / wave;
    const long long most = 32 / P.par > 1 ? 32 / P.par : 1;
    if (passes > most) passes = most;
    P.run = static_cast<int>(passes * P.par);
    const dim3 grid(static_cast<unsigned>((static_cast<long long>(P.T) + P.run - 1) / P.run));
    const size_t smem = passes == 1 ? 0 : static_cast<size_t>(P.run) * P.rot * sizeof(float);
    void (*kernel)(RopeParams) = nullptr;
    auto pick = [&](auto type, auto dim, auto app, auto one) {
        using T16 = decltype(type);
        constexpr int kD = decltype(dim)::value;
        constexpr bool kA = decltype(app)::value, kOne = decltype(one)::value;
        kernel = P.norm == HAWK_NORM_NONE  ? rope_kernel<T16, kD, kA, HAWK_NORM_NONE, kOne>
                 : P.norm == HAWK_NORM_RMS ? rope_kernel<T16, kD, kA, HAWK_NORM_RMS, kOne>
                                           : rope_kernel<T16, kD, kA, HAWK_NORM_LAYER, kOne>;
    };
    auto pick_one = [&](auto type, auto dim, auto app) {
        if (passes == 1) pick(type, dim, app, std::true_type{});
        else pick(type, dim, app, std::false_type{});
    };
    auto pick_app = [&](auto type, auto dim) {
        if (append) pick_one(type, dim, std::true_type{});
        else pick_one(type, dim, std::false_type{});
    };
    auto pick_dim = [&](auto type) {
        if (D == 64) pick_app(type, std::integral_constant<int, 64>{});
        else pick_app(type, std::integral_constant<int, 128>{});
    };
    if (dtype == HAWK_BF16) pick_dim(__nv_bfloat16{});
    else pick_dim(__half{});
    return hawk_host::launch_dependent(kernel, grid, dim3(kThreads), smem, reinterpret_cast<cudaStream_t>(stream), P) ==
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
    if (has_stray_bias(*a)) return HAWK_ERR_PARAM;
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
    if (has_stray_bias(a->qk)) return HAWK_ERR_PARAM;
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
