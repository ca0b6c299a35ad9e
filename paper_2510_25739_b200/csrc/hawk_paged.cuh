// What the three kernels behind hawk_paged_attn share: the call's parameters, the view of one stream of the ragged batch,
// the 16-bit element types, and the launchers.
#pragma once

#include <math_constants.h>

#include "hawk_common.cuh"

namespace hawk {

// A pair of query tiles of a stream of many rows: what a block of the tile kernel works on (for one kv head).
struct PagedGroup {
    int s, r0, n, kv;  // stream, its first row, rows, keys; n = 0: behind the list's end
    int tok0;          // first position of the pair
    int pad[3];
};

// One launch of either kernel.
struct PagedParams {
    const void *q;
    void *out;
    const int32_t *row_begin, *kv_len, *block_table;
    const uint64_t *anc_mask;  // [max_new] or NULL
    float *part;               // partial results (layout: see each kernel)
    int32_t *records;          // rows kernel: one record of kRecordInts per worker
    long long part_floats, record_ints;  // room in the two (for the index checks of the debug build)
    long long q_row_stride, q_head_stride;
    int S, T, max_new, H, H_kv, group;
    int n_pages, page_size, table_width;
    int kv_cap;                // largest admissible kv_len
    int rows_few;              // a stream of at most this many rows per kv head goes to the rows kernel, others to the tile kernel
    int box_rows;              // cache rows of one TMA box: a divisor of the page size and of the tile
    int k_rows_inner, v_rows_inner;  // tensor maps are {D, rows, heads, pages} (1) or {D, heads, rows, pages} (0): the
                                     // dimension with the smaller stride comes first
    int row_blocks;            // rows kernel: blocks that do rows; one more makes the list below, where there is one
    PagedGroup *groups;        // [group_cap], longest first; NULL: no stream goes to the tile kernel
    int group_cap, tile_tok;   // tile_tok: positions a query tile holds
    int mid_tok;               // mid kernel: positions an item's queries are loaded for
    FastDiv div_page, div_group;
    float scale_log2;          // sm_scale * log2(e)
    int32_t *dev_status;
};

struct PagedStream {
    int r0, n, kv;  // first row, rows, keys (the rows' own included)
};

// Stream s of the batch, checked: a stream whose rows are not inside the call's is empty, a key count outside its range
// is clamped.  An idle stream's kv_len is not looked at.
__device__ __forceinline__ PagedStream paged_stream(const PagedParams &P, int s, int &flags)
{
    PagedStream st;
    const int r0 = P.row_begin[s], r1 = P.row_begin[s + 1];
    int kv = P.kv_len[s];
    st.r0 = r0;
    st.n = 0;
    st.kv = 0;
    if (r0 < 0 || r1 < r0 || r1 > P.T || r1 - r0 > P.max_new) {
        flags |= HAWK_DEV_BAD_ROWS;
        return st;
    }
    st.n = r1 - r0;
    if (st.n == 0) return st;
    if (kv < 0 || kv > P.kv_cap) {
        flags |= HAWK_DEV_BAD_PREFIX;
        kv = max(0, min(kv, P.kv_cap));
    }
    st.kv = kv;
    return st;
}

// The rows before `end` of a stream of n see keys of this many of its rows at most: a chain's up to themselves, a tree's nodes
// whatever their masks say.
__device__ __forceinline__ int paged_reach(const PagedParams &P, int n, int end) { return P.anc_mask ? n : min(n, end); }

__device__ __forceinline__ bool paged_is_few(const PagedParams &P, const PagedStream &st)
{
    return static_cast<long long>(st.n) * P.group <= P.rows_few;
}

// Softmax.  Maxima are kept as the products gave them, not yet scaled (partial results too), so nothing is lost in them.  The
// exponent of a score s under the shift m is one fma, s * scale - fl(m * scale): the rounding of that product is in every exponent of the
// row alike, as if the shift were another, and is under 2^-15 for shifts below this bound.  Beyond it (from 2^28 on it could exceed the 2^8
// that a probability may reach, from 2^31 on what fp32 holds) rows take (s - m) * scale, the difference being exact where it
// counts, for s near m; or they add what was lost, fl(m * scale) - m * scale, which fp32 holds exactly.  (That sum is off by 2^-24 of what
// was lost and of the exponent: under 2^-17 up to shifts of 2^30; beyond them scores are 2^6 and more apart or equal, and equal
// ones give 0.)  Decided for all rows of a warp or group at a renewal of their shifts.
constexpr float kFarShift = 512.f;  // base 2

__device__ __forceinline__ bool is_far(float m, float scale) { return m != -CUDART_INF_F && fabsf(m * scale) >= kFarShift; }

constexpr int kPagedTileKeys = 128;  // keys of a tile of the tile kernel
constexpr int kPlanBuckets = 256;

constexpr int kPlanWaves = 6;  // jobs of so many waves of blocks even out by themselves

// Makes the tile kernel's list: one block, `sh` holds kPlanBuckets + 1 ints.  Longest pair first (a counting sort over 256
// cost classes), so that no long job starts last; where the jobs are many waves of blocks, one stream after the other instead, each
// from its longest pair on, so that what runs together shares keys and values in L2 (799 against 822 us for 4 x 2048 rows
// over 8192 keys; for 7B chunks of 300 to 511 rows, under two waves, the sort takes 94 us to 84).
// A warp looks at 32 streams at once and deals their pairs out to its lanes.
__device__ __forceinline__ void paged_plan(const PagedParams &P, int *sh, int &flags)
{
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, warps = blockDim.x >> 5;
    const int per_pair = 2 * P.tile_tok;
    const float scale = (kPlanBuckets - 1) / (8.f * (P.kv_cap / kPagedTileKeys + 1));
    auto pairs_at = [&](int s, PagedStream &st) {  // pairs of stream s, 0 for one of the rows kernel's or none
        st = {0, 0, 0};
        if (s < P.S) st = paged_stream(P, s, flags);
        return st.n == 0 || paged_is_few(P, st) ? 0 : (st.n + per_pair - 1) / per_pair;
    };
    // visit(cost class, stream, first row, rows, keys, pair, place of the stream's last pair in plain order): for every pair
    auto each = [&](bool plain, auto &&visit) {
        for (int s0 = warp * 32; s0 < P.S; s0 += warps * 32) {
            PagedStream st;
            int before = 0;  // pairs of the streams before this lane's
            if (plain) {
                for (int s = lane; s < s0; s += 32) before += pairs_at(s, st);
                before = __reduce_add_sync(0xffffffffu, before);
            }
            const int mine = pairs_at(s0 + lane, st);
            int inc = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int u = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += u;
            }
            before += inc - mine;
            const int all = __shfl_sync(0xffffffffu, inc, 31);
            for (int i0 = 0; i0 < all; i0 += 32) {
                const int i = i0 + lane;  // pair of these 32 streams
                int b = 0;                // its stream: the first whose running sum is past i
#pragma unroll
                for (int step = 16; step; step >>= 1)
                    if (__shfl_sync(0xffffffffu, inc, b + step - 1) <= i) b += step;
                const int r0 = __shfl_sync(0xffffffffu, st.r0, b), n = __shfl_sync(0xffffffffu, st.n, b);
                const int kv = __shfl_sync(0xffffffffu, st.kv, b), pairs = __shfl_sync(0xffffffffu, mine, b);
                const int p = i - (__shfl_sync(0xffffffffu, inc, b) - pairs), at = __shfl_sync(0xffffffffu, before, b);
                if (i < all) {
                    // cost: key tiles that the pair's last position sees; one takes some 3400 cycles where both query tiles
                    // have rows, 2150 where only one does
                    const int keys = max(0, min(kv, kv - n + paged_reach(P, n, (p + 1) * per_pair)));
                    const int tiles = (keys + kPagedTileKeys - 1) / kPagedTileKeys;
                    const int cost = p * per_pair + P.tile_tok >= n ? 5 * tiles : 8 * tiles;
                    const int bucket = kPlanBuckets - 1 - min(kPlanBuckets - 1, static_cast<int>(cost * scale));
                    visit(bucket, s0 + b, r0, n, kv, p, at + pairs - 1 - p);
                }
                __syncwarp();
            }
        }
    };
    for (int i = tid; i < kPlanBuckets; i += blockDim.x) sh[i] = 0;
    __syncthreads();
    each(false, [&](int bucket, int, int, int, int, int, int) { atomicAdd(&sh[bucket], 1); });
    __syncthreads();
    if (warp == 0) {  // exclusive prefix sum, 8 classes a lane
        constexpr int kPer = kPlanBuckets / 32;
        int v[kPer], sum = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            v[i] = sh[lane * kPer + i];
            sum += v[i];
        }
        int inc = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += u;
        }
        if (lane == 31) sh[kPlanBuckets] = inc;
        int at = inc - sum;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            sh[lane * kPer + i] = at;
            at += v[i];
        }
    }
    __syncthreads();
    const int total = sh[kPlanBuckets];
    auto put = [&](int at, int s, int r0, int n, int kv, int p) {
        if (at >= P.group_cap) return;  // (the cap bounds every valid batch)
        *reinterpret_cast<int4 *>(P.groups + at) = make_int4(s, r0, n, kv);
        P.groups[at].tok0 = p * per_pair;
    };
    const bool plain = static_cast<long long>(total) * P.H_kv >= kPlanWaves * 148;
    each(plain, [&](int bucket, int s, int r0, int n, int kv, int p, int place) {
        put(plain ? place : atomicAdd(&sh[bucket], 1), s, r0, n, kv, p);
    });
    if (warp == 0)
        for (int i = total + lane; i < P.group_cap; i += 32) P.groups[i].n = 0;
}

// Box of cache rows (page, row inside it, kv head, 64-column half) into shared memory.
__device__ __forceinline__ void paged_load(void *dst, const CUtensorMap *map, int rows_inner, int half, int row, int head, int page,
                                           uint64_t *bar, uint64_t policy)
{
    tma_load_4d_hint(dst, map, half * 64, rows_inner ? row : head, rows_inner ? head : row, page, bar, policy);
}

template <typename T16>
struct Elem;
template <>
struct Elem<__nv_bfloat16> {
    static constexpr bool kBf16 = true;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack_bf16(lo, hi); }
    static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
    {
        mma_bf16_16816(d, a, b0, b1);
    }
};
template <>
struct Elem<__half> {
    static constexpr bool kBf16 = false;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<uint32_t *>(&v);
    }
    static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
    {
        mma_f16_16816(d, a, b0, b1);
    }
};

}  // namespace hawk

namespace hawk_host {

constexpr int kPagedSms = 148;  // launch shapes are planned for the B200's 148 SMs

// Tensor map over one of the page tensors with boxes of `box_rows` cache rows x 64 columns; *rows_inner as in PagedParams.
bool encode_pages(CUtensorMap *map, const hawk_paged_attn_args &a, bool values, int box_rows, int *rows_inner);

int paged_gcd(int a, int b);

constexpr int kPagedMaxStreams = 4096;  // the prefix sums are held in shared memory

// The mid kernel (up to 64 rows per kv head on tcgen05): rows per item it is built for that hold `rows` (16, 32, 64), and its
// launch (without the merge).
cudaError_t launch_paged_mid(const hawk_paged_attn_args &a, const hawk::PagedParams &base, int nr, cudaStream_t st);

// The tile kernel (tcgen05 tiles of query rows): bytes of its list and of its partial results, and its launch.
size_t paged_tile_workspace_bytes(int S, int T, int max_new, int H, int H_kv, int few, int D, int max_kv);
// Upper bound of the call's pairs of query tiles (the list's length); 0: more than the kernel can number.
int paged_tile_groups(int S, int T, int max_new, int H, int H_kv, int few);
cudaError_t launch_paged_tile(const hawk_paged_attn_args &a, const hawk::PagedParams &base, float *part, cudaStream_t st);

}  // namespace hawk_host
