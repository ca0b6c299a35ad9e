// hawk_paged_attn for streams that bring MANY rows (chunks of a prompt): tiles of query rows on the fifth-generation tensor
// cores, keys and values streamed page by page.
//
// A block owns one (stream, kv head, pair of 128-row query tiles).  The rows of a tile are (position, head of the group)
// pairs with the head running fastest, so grouped-query heads share every key and value tile.  Two query tiles a block
// halve the key/value bytes each flop asks of L2 and give the tensor pipe something to do while the other tile's
// scores are in softmax.  Warps:
//   0-3, 4-7  softmax of tile 0 and of tile 1: one query row a thread (row maxima and sums need no shuffles)
//   8         issues every tcgen05.mma:  S_t = Q_t K^T (both operands in shared memory), O_t += P_t V (P_t in tensor
//             memory, V in shared memory read along its rows)
//   9         loads: Q once, then K and V tiles of 128 keys into a ring, as boxes that stay inside a page
// Tensor memory: S_0, S_1 (128 columns each; P_t overwrites the first half of S_t in 16 bits), O_0, O_1 (D columns each).
// Order of the products: S_0(0) S_1(0) | P_0(i)V S_0(i+1) P_1(i)V S_1(i+1) | ..., so one tile's softmax runs under the
// other tile's two products, and when S_t(i) is complete so is O_t up to tile i-1: the softmax warps rescale O_t in
// place without any other handshake.  They do so only when a row's maximum has grown by more than 2^8 since the last
// time (any shift keeps the softmax exact as long as O and the sum use the same one; 2^8 leaves fp16 and fp32 ample room).
// Few blocks: the key range is split too, each split leaves (o, max, sum) in fp32 and a second kernel joins them.
#include <atomic>

#include "hawk_paged.cuh"

namespace {

using namespace hawk;

constexpr int kBM = 128, kBN = 128;
constexpr int kThreads = 320;
constexpr int kMaxSplits = 16;
constexpr int kMinSplitKeys = 512;  // shorter key ranges cost more in partial results than they gain in blocks

struct TileParams {
    PagedParams c;
    int tok;       // positions a query tile holds: 128 / group
    int n_split;
    int q_rows;    // rows of a query tile that are used: tok * group
    FastDiv div_split, div_hkv;
};

template <int D>
struct TileCfg {
    static constexpr int kHalves = D / 64;
    static constexpr int kHalfBytes = 128 * 128;           // [128 rows][64 columns]
    static constexpr int kTileBytes = kHalves * kHalfBytes;
    static constexpr int kStages = D == 128 ? 5 : 10;
    static constexpr size_t kSmem = 1024 + static_cast<size_t>(2 + kStages) * kTileBytes + 512;
};

// What the block works on.
struct TileJob {
    int s, hk, split;
    int r0, n, kv;
    int tok0;            // first position of the block's first query tile
    int nt[2];           // key tiles of each query tile, counted from tile `begin`
    int begin;           // first key tile of the split
    bool any;
};

// Pairs of query tiles of a stream that belongs to this kernel.
__device__ __forceinline__ int pairs_of(const TileParams &P, const PagedStream &st)
{
    if (st.n == 0 || paged_is_few(P.c, st)) return 0;
    return (st.n + 2 * P.tok - 1) / (2 * P.tok);
}

// Finds the block's job: the streams' pairs are numbered through; one sweep of the block over the streams.
__device__ __forceinline__ bool find_job(const TileParams &P, bool with_split, int *shared_sums, TileJob &job, int &flags)
{
    uint32_t split = 0, hk;
    const uint32_t pair_hk = with_split ? P.div_split.divmod(blockIdx.x, split) : blockIdx.x;
    const int pair = static_cast<int>(P.div_hkv.divmod(pair_hk, hk));
    job.split = static_cast<int>(split);
    job.hk = static_cast<int>(hk);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, warps = blockDim.x >> 5;
    int *found = shared_sums + 16;
    int running = 0;
    if (tid == 0) found[0] = -1;
    for (int base = 0; base < P.c.S && running <= pair; base += blockDim.x) {
        const int s = base + tid;
        int v = 0;
        if (s < P.c.S) v = pairs_of(P, paged_stream(P.c, s, flags));
        int inc = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += u;
        }
        if (lane == 31) shared_sums[warp] = inc;
        __syncthreads();
        int before = running, all = running;
        for (int w = 0; w < warps; ++w) {
            if (w < warp) before += shared_sums[w];
            all += shared_sums[w];
        }
        const int end = before + inc;
        if (v > 0 && pair >= end - v && pair < end) {
            found[0] = s;
            found[1] = pair - (end - v);
            found[2] = v;
        }
        running = all;
        __syncthreads();
    }
    __syncthreads();
    const int s = found[0];
    if (s < 0) return false;
    const PagedStream st = paged_stream(P.c, s, flags);
    job.s = s;
    job.r0 = st.r0;
    job.n = st.n;
    job.kv = st.kv;
    job.tok0 = (found[2] - 1 - found[1]) * 2 * P.tok;  // the pairs that see the most keys first
    const int pfx = st.kv - st.n;
    int end[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int first = job.tok0 + t * P.tok;
        const int last = min(st.n, first + P.tok) - 1;  // last position of the tile
        const int keys = first < st.n ? max(0, min(st.kv, pfx + last + 1)) : 0;
        end[t] = (keys + kBN - 1) / kBN;
    }
    const int all = max(end[0], end[1]);
    job.begin = static_cast<int>(static_cast<long long>(all) * job.split / P.n_split);
    const int stop = static_cast<int>(static_cast<long long>(all) * (job.split + 1) / P.n_split);
#pragma unroll
    for (int t = 0; t < 2; ++t) job.nt[t] = max(0, min(end[t], stop) - job.begin);
    job.any = job.nt[0] > 0 || job.nt[1] > 0;
    return true;
}

template <typename T16, int D>
__global__ void __launch_bounds__(kThreads, 1)
    paged_tile_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                      const __grid_constant__ CUtensorMap map_v, const TileParams P)
{
    using C = TileCfg<D>;
    using E = Elem<T16>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *q_smem = smem;                              // two query tiles
    uint8_t *ring = smem + 2 * C::kTileBytes;            // K and V tiles in turn
    uint64_t *bars = reinterpret_cast<uint64_t *>(ring + C::kStages * C::kTileBytes);
    uint64_t *full = bars, *empty = bars + C::kStages;
    uint64_t *q_full = bars + 2 * C::kStages, *s_full = q_full + 1, *p_ready = q_full + 3, *o_done = q_full + 5, *drain = q_full + 7;
    uint32_t *tmem_ptr = reinterpret_cast<uint32_t *>(drain + 1);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_ptr + 1);
    int *sums = reinterpret_cast<int *>(tmem_ptr + 2);   // [20]

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        mbar_init(q_full, 1);
        for (int t = 0; t < 2; ++t) {
            mbar_init(&s_full[t], 1);
            mbar_init(&p_ready[t], 4);
            mbar_init(&o_done[t], 1);
        }
        mbar_init(drain, 1);
        *abort_flag = 0;
        fence_mbar_init();
        fence_proxy_async();
        prefetch_tensormap(&map_q);
        prefetch_tensormap(&map_k);
        prefetch_tensormap(&map_v);
    }
    grid_dependency_wait();
    int flags = 0;
    TileJob job;
    const bool has_job = find_job(P, true, sums, job, flags);  // (block-uniform; also publishes the barriers)
    if (flags && blockIdx.x == 0 && P.c.dev_status) atomicOr(P.c.dev_status, flags);
    flags = 0;
    if (!has_job) return;
    if (warp == 8) {
        tmem_alloc(tmem_ptr, 512);
        tmem_relinquish();
    }
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = *tmem_ptr;
    const int nt_max = max(job.nt[0], job.nt[1]);
    const int pfx = job.kv - job.n;

    if (warp == 9) {
        // ------------------------------------------------------------------ loads
        bool ok = true;
        int issued = 0;  // ring stages armed
        if (job.any) {
            const uint64_t keep = l2_policy_evict_last();
            if (lane == 0) {
                const uint32_t bytes = (job.nt[0] > 0 ? 1 : 0) + (job.nt[1] > 0 ? 1 : 0);
                mbar_arrive_expect_tx(q_full, bytes * C::kHalves * P.q_rows * 128);
                for (int t = 0; t < 2; ++t)
                    if (job.nt[t] > 0)
                        for (int hf = 0; hf < C::kHalves; ++hf)
                            tma_load_4d(q_smem + t * C::kTileBytes + hf * C::kHalfBytes, &map_q, hf * 64, job.hk * P.c.group,
                                        job.r0 + job.tok0 + t * P.tok, 0, q_full);
            }
            const int need = static_cast<int>(P.c.div_page.div(static_cast<uint32_t>(job.kv + P.c.page_size - 1)));
            const int32_t *tb = P.c.block_table + static_cast<size_t>(job.s) * P.c.table_width;
            const int boxes = kBN / P.c.box_rows;
            int base = -64, cur = 0, nxt = 0;  // page ids base + lane and base + 32 + lane
            auto fetch = [&](int b) { return b + lane < need ? tb[b + lane] : 0; };
            for (int i = 0; i < nt_max && ok; ++i) {
                const int key0 = (job.begin + i) * kBN;
                const int live = min(boxes, (job.kv - key0 + P.c.box_rows - 1) / P.c.box_rows);
                for (int kind = 0; kind < 2 && ok; ++kind) {  // K, then V
                    const int st = issued % C::kStages;
                    const uint32_t round = issued / C::kStages;
                    if (round > 0) ok = mbar_wait(&empty[st], (round - 1) & 1u, abort_flag);
                    if (!ok) break;
                    uint8_t *dst = ring + st * C::kTileBytes;
                    if (lane == 0) {
                        const bool stall = kTestStallBytes != 0 && blockIdx.x == 0 && issued == 0;
                        mbar_arrive_expect_tx(&full[st], live * P.c.box_rows * 128 * C::kHalves + (stall ? kTestStallBytes : 0u));
                    }
                    ++issued;
                    for (int b = 0; b < live; ++b) {
                        uint32_t row;
                        const int pg = static_cast<int>(P.c.div_page.divmod(static_cast<uint32_t>(key0 + b * P.c.box_rows), row));
                        if (pg < base || pg >= base + 32) {
                            if (pg >= base + 32 && pg < base + 64) {
                                cur = nxt;
                                base += 32;
                            } else {
                                base = pg & ~31;
                                cur = fetch(base);
                            }
                            nxt = fetch(base + 32);
                        }
                        const int id = __shfl_sync(0xffffffffu, cur, pg - base);
                        if (id < 0 || id >= P.c.n_pages) flags |= HAWK_DEV_BAD_PAGE;  // (outside the tensor map: zeros)
                        if (lane == 0)
                            for (int hf = 0; hf < C::kHalves; ++hf)
                                paged_load(dst + hf * C::kHalfBytes + b * P.c.box_rows * 128, kind ? &map_v : &map_k,
                                           kind ? P.c.v_rows_inner : P.c.k_rows_inner, hf, static_cast<int>(row), job.hk, id,
                                           &full[st], keep);
                    }
                    // K's boxes of this tile come again for V: the table window may have moved on, which `base` notices
                }
            }
            if (!ok || *abort_flag) {
                // let what is in flight land (bounded) before the block retires
                *abort_flag = 1;
                mbar_wait(q_full, 0, nullptr);
                for (int i = max(0, issued - C::kStages); i < issued; ++i)
                    mbar_wait(&full[i % C::kStages], (i / C::kStages) & 1u, nullptr);
                flags |= HAWK_DEV_TIMEOUT;
            }
        }
        if (flags && lane == 0 && P.c.dev_status) atomicOr(P.c.dev_status, flags);
    } else if (warp == 8) {
        // ------------------------------------------------------------------ products
        constexpr uint32_t idesc_s = umma_idesc_f16kind(kBM, kBN, E::kBf16, false);
        constexpr uint32_t idesc_o = umma_idesc_f16kind(kBM, D, E::kBf16, true);
        const uint32_t q_addr = smem_u32(q_smem), ring_addr = smem_u32(ring);
        bool ok = true;
        auto wait_full = [&](int load) {  // load 2i: K tile i, 2i + 1: V tile i
            ok = ok && mbar_wait(&full[load % C::kStages], (load / C::kStages) & 1u, abort_flag);
        };
        auto scores = [&](int t, int i) {
            const uint32_t a = q_addr + t * C::kTileBytes, b = ring_addr + ((2 * i) % C::kStages) * C::kTileBytes;
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const uint32_t off = (kk >> 2) * C::kHalfBytes + (kk & 3) * 32;
                umma_bf16(tmem + t * kBN, umma_desc_k_major_sw128(a + off), umma_desc_k_major_sw128(b + off), idesc_s, kk > 0);
            }
            umma_commit(&s_full[t]);
        };
        auto values = [&](int t, int i) {
            const uint32_t b = ring_addr + ((2 * i + 1) % C::kStages) * C::kTileBytes;
#pragma unroll
            for (int kk = 0; kk < kBN / 16; ++kk)
                umma_f16_ts(tmem + 256 + t * D, tmem + t * kBN + kk * 8,
                            umma_desc_mn_major_sw128(b + kk * 2048, C::kHalfBytes), idesc_o, i > 0 || kk > 0);
            if (i + 1 == job.nt[t]) umma_commit(&o_done[t]);
        };
        if (job.any) {
            ok = mbar_wait(q_full, 0, abort_flag);
            wait_full(0);
            if (ok && lane == 0) {
                tcgen05_fence_after();
                for (int t = 0; t < 2; ++t)
                    if (job.nt[t] > 0) scores(t, 0);
                umma_commit(&empty[0]);
            }
            for (int i = 0; i < nt_max && ok; ++i) {
                wait_full(2 * i + 1);
                const int vst = (2 * i + 1) % C::kStages;
                const int left = job.kv - (job.begin + i) * kBN;  // keys of the tile that exist
                if (ok && left < kBN) {
                    // values behind the last key hold anything: zero them (0 * NaN is NaN)
                    uint8_t *v = ring + vst * C::kTileBytes;
                    for (int x = left * 8 + lane; x < kBN * 8; x += 32)
                        for (int hf = 0; hf < C::kHalves; ++hf)
                            *reinterpret_cast<uint4 *>(v + hf * C::kHalfBytes + x * 16) = make_uint4(0u, 0u, 0u, 0u);
                    fence_proxy_async();
                    __syncwarp();
                }
                for (int t = 0; t < 2 && ok; ++t) {
                    if (i < job.nt[t]) {
                        ok = mbar_wait(&p_ready[t], i & 1u, abort_flag);
                        if (ok && lane == 0) {
                            tcgen05_fence_after();
                            values(t, i);
                        }
                    }
                    if (i + 1 < job.nt[t]) {
                        wait_full(2 * i + 2);
                        if (ok && lane == 0) scores(t, i + 1);
                    }
                }
                if (ok && lane == 0) {
                    umma_commit(&empty[vst]);
                    if (i + 1 < nt_max) umma_commit(&empty[(2 * i + 2) % C::kStages]);
                }
            }
            // every product issued has finished before the block gives its tensor memory back
            __syncwarp();
            if (lane == 0) umma_commit(drain);
            if (!ok) *abort_flag = 1;
            if (!mbar_wait(drain, 0, nullptr)) ok = false;
            if (!ok && lane == 0 && P.c.dev_status) atomicOr(P.c.dev_status, HAWK_DEV_TIMEOUT);
        }
    } else {
        // ------------------------------------------------------------------ softmax and epilogue of query tile t
        const int t = warp >> 2;
        const int r = tid & 127;
        const uint32_t lane_off = static_cast<uint32_t>(warp & 3) << 21;  // 32 lanes of tensor memory per warp
        const uint32_t s_addr = tmem + lane_off + t * kBN, o_addr = tmem + lane_off + 256 + t * D;
        uint32_t hd;
        const int pos = job.tok0 + t * P.tok + static_cast<int>(P.c.div_group.divmod(static_cast<uint32_t>(r), hd));
        const bool valid = r < P.q_rows && pos < job.n;
        const int limit = min(job.kv, pfx + min(pos, job.n - 1) + 1);  // keys this row sees
        float m_run = -CUDART_INF_F, l_run = 0.f;
        const int nt = job.nt[t];
        bool ok = true;
        for (int i = 0; i < nt; ++i) {
            ok = mbar_wait(&s_full[t], i & 1u, abort_flag);
            if (!ok) break;
            tcgen05_fence_after();
            uint32_t u[4][32];
#pragma unroll
            for (int q = 0; q < 4; ++q) tmem_ld_32x32(s_addr + q * 32, u[q]);
            tmem_ld_wait();
            const int seen = limit - (job.begin + i) * kBN;
            if (seen < kBN) {
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int c = 0; c < 32; ++c)
                        if (q * 32 + c >= seen) u[q][c] = 0xff800000u;  // -inf
            }
            float mx[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                mx[q] = __uint_as_float(u[q][0]);
#pragma unroll
                for (int c = 1; c < 32; ++c) mx[q] = fmaxf(mx[q], __uint_as_float(u[q][c]));
            }
            const float m_new = fmaxf(m_run, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * P.c.scale_log2);
            if (i == 0) {
                m_run = m_new;
            } else if (__any_sync(0xffffffffu, m_new > m_run + 8.f)) {
                const float mu = m_new == -CUDART_INF_F ? 0.f : m_new;
                const float alpha = fast_exp2(m_run - mu);
                m_run = m_new;
                l_run *= alpha;
#pragma unroll
                for (int c0 = 0; c0 < D; c0 += 16) {
                    uint32_t o[16];
                    tmem_ld_32x16(o_addr + c0, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * alpha);
                    tmem_st_32x16(o_addr + c0, o);
                }
            }
            const float mu = m_run == -CUDART_INF_F ? 0.f : m_run;
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t pk[32];
#pragma unroll
                for (int c = 0; c < 32; ++c) {
                    const float x0 = __uint_as_float(u[half * 2 + (c >> 4)][(2 * c) & 31]);
                    const float x1 = __uint_as_float(u[half * 2 + (c >> 4)][(2 * c + 1) & 31]);
                    const float p0 = fast_exp2(fmaf(x0, P.c.scale_log2, -mu)), p1 = fast_exp2(fmaf(x1, P.c.scale_log2, -mu));
                    sum[c & 1] += p0;
                    sum[2 + (c & 1)] += p1;
                    pk[c] = E::pack(p0, p1);
                }
                tmem_st_32x32(s_addr + half * 32, pk);
            }
            l_run += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            tmem_st_wait();
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&p_ready[t]);
        }
        if (ok && nt > 0) ok = mbar_wait(&o_done[t], 0, abort_flag);
        if (!ok) *abort_flag = 1;
        tcgen05_fence_after();
        const long long row = job.r0 + static_cast<long long>(pos);
        const int h = job.hk * P.c.group + static_cast<int>(hd);
        const long long cell = row * P.c.H + h;
        // the tensor-memory loads below are for whole warps: rows that do not exist take part and store nothing
        if (P.n_split == 1) {
            const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
            T16 *dst = static_cast<T16 *>(P.c.out) + (valid ? cell * D : 0);
#pragma unroll
            for (int c0 = 0; c0 < D; c0 += 32) {
                uint32_t o[32];
                if (nt > 0) {
                    tmem_ld_32x32(o_addr + c0, o);
                    tmem_ld_wait();
                }
                if (valid && ok) {
#pragma unroll
                    for (int c = 0; c < 32; c += 8) {
                        uint32_t w[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            w[k] = nt == 0 || l_run == 0.f ? 0u
                                                           : E::pack(__uint_as_float(o[c + 2 * k]) * inv,
                                                                     __uint_as_float(o[c + 2 * k + 1]) * inv);
                        *reinterpret_cast<uint4 *>(dst + c0 + c) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
            }
        } else {
            const long long cells = static_cast<long long>(P.c.T) * P.c.H, at = job.split * cells + (valid ? cell : 0);
            float *dst = P.c.part + at * D;
            if (valid && ok)
                *reinterpret_cast<float2 *>(P.c.part + P.n_split * cells * D + at * 2) = make_float2(m_run, l_run);
            if (nt > 0) {  // (a split without keys has l = 0 and its o is not read)
#pragma unroll
                for (int c0 = 0; c0 < D; c0 += 32) {
                    uint32_t o[32];
                    tmem_ld_32x32(o_addr + c0, o);
                    tmem_ld_wait();
                    if (valid && ok) {
#pragma unroll
                        for (int c = 0; c < 32; c += 4)
                            *reinterpret_cast<uint4 *>(dst + c0 + c) = make_uint4(o[c], o[c + 1], o[c + 2], o[c + 3]);
                    }
                }
            }
        }
    }
    tcgen05_fence_before();
    __syncthreads();
    if (warp == 8) tmem_dealloc(tmem, 512);
}

// Joins the splits: a block per (pair of query tiles, kv head) as above, a warp per row.
template <typename T16, int D>
__global__ void __launch_bounds__(256) paged_tile_merge_kernel(const TileParams P)
{
    using E = Elem<T16>;
    constexpr int PER = D / 32;
    __shared__ int sums[20];
    allow_dependent_launch();
    TileJob job;
    int flags = 0;
    grid_dependency_wait();
    if (!find_job(P, false, sums, job, flags)) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long cells = static_cast<long long>(P.c.T) * P.c.H;
    const float *ml = P.c.part + P.n_split * cells * D;
    const int rows = min(2 * P.tok, job.n - job.tok0) * P.c.group;
    for (int r = warp; r < rows; r += 8) {
        uint32_t hd;
        const uint32_t pos = P.c.div_group.divmod(static_cast<uint32_t>(r), hd);
        const long long cell = (job.r0 + static_cast<long long>(job.tok0) + pos) * P.c.H + job.hk * P.c.group + static_cast<int>(hd);
        // lane x holds split x's maximum and sum (at most 16 splits)
        float2 mine = make_float2(-CUDART_INF_F, 0.f);
        if (lane < P.n_split) mine = *reinterpret_cast<const float2 *>(ml + (lane * cells + cell) * 2);
        const float m = warp_max(mine.y == 0.f ? -CUDART_INF_F : mine.x);
        const float mu = m == -CUDART_INF_F ? 0.f : m;
        const float f = mine.y == 0.f ? 0.f : fast_exp2(mine.x - mu);
        const float l = warp_sum(mine.y * f);
        const float scale = l == 0.f ? 0.f : f / l;
        float acc[PER];
#pragma unroll
        for (int c = 0; c < PER; ++c) acc[c] = 0.f;
        for (int x = 0; x < P.n_split; ++x) {
            const float w = __shfl_sync(0xffffffffu, scale, x);
            if (w == 0.f) continue;  // (its o may not have been written)
            const float *src = P.c.part + (x * cells + cell) * D + lane * PER;
#pragma unroll
            for (int c = 0; c < PER; c += 2) {
                const float2 v = *reinterpret_cast<const float2 *>(src + c);
                acc[c] = fmaf(v.x, w, acc[c]);
                acc[c + 1] = fmaf(v.y, w, acc[c + 1]);
            }
        }
        T16 *dst = static_cast<T16 *>(P.c.out) + cell * D + lane * PER;
#pragma unroll
        for (int c = 0; c < PER; c += 2) *reinterpret_cast<uint32_t *>(dst + c) = E::pack(acc[c], acc[c + 1]);
    }
}

// ---------------------------------------------------------------------------------------------- host side
struct TilePlan {
    int tok;
    long long pairs;  // upper bound of the call's pairs of query tiles
    int n_split;
};

TilePlan plan_tiles(int S, int T, int max_new, int H, int H_kv, int few, int max_kv)
{
    TilePlan p;
    const int group = H / H_kv;
    p.tok = kBM / group;
    const long long per = (max_new + 2ll * p.tok - 1) / (2 * p.tok);
    // streams with more than `few` rows per kv head: at most T / (few / group + 1) of them
    const long long many = T / (few / group + 1);
    const long long streams = many < S ? many : S;
    const long long a = streams * per, b = T / (2 * p.tok) + streams;
    p.pairs = a < b ? a : b;
    if (p.pairs < 1) p.pairs = 1;
    const long long blocks = p.pairs * H_kv;
    p.n_split = 1;
    if (2 * blocks <= hawk_host::kPagedSms) {
        long long n = hawk_host::kPagedSms / blocks;
        const long long by_keys = max_kv / kMinSplitKeys;
        n = n < by_keys ? n : by_keys;
        p.n_split = static_cast<int>(n < 1 ? 1 : n > kMaxSplits ? kMaxSplits : n);
    }
    return p;
}

template <typename T16, int D>
cudaError_t launch(const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv, const TileParams &P, long long pairs,
                   cudaStream_t st)
{
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    if (device < 0 || device >= 64) return cudaErrorInvalidDevice;
    static std::atomic<unsigned long long> attr_done{0};  // one bit per device
    if (!((attr_done.load(std::memory_order_relaxed) >> device) & 1ull)) {
        e = cudaFuncSetAttribute(paged_tile_kernel<T16, D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 static_cast<int>(TileCfg<D>::kSmem));
        if (e != cudaSuccess) return e;
        attr_done.fetch_or(1ull << device, std::memory_order_relaxed);
    }
    const unsigned base = static_cast<unsigned>(pairs * P.c.H_kv);
    e = hawk_host::launch_dependent(paged_tile_kernel<T16, D>, dim3(base * P.n_split), dim3(kThreads), TileCfg<D>::kSmem, st, mq,
                                    mk, mv, P);
    if (e != cudaSuccess || P.n_split == 1) return e;
    return hawk_host::launch_dependent(paged_tile_merge_kernel<T16, D>, dim3(base), dim3(256), 0, st, P);
}

}  // namespace

size_t hawk_host::paged_tile_workspace_bytes(int S, int T, int max_new, int H, int H_kv, int few, int D, int max_kv)
{
    const TilePlan p = plan_tiles(S, T, max_new, H, H_kv, few, max_kv);
    return p.n_split == 1 ? 0 : static_cast<size_t>(p.n_split) * T * H * (D + 2) * sizeof(float);
}

cudaError_t hawk_host::launch_paged_tile(const hawk_paged_attn_args &a, const PagedParams &base, float *part, cudaStream_t st,
                                         bool *refused)
{
    const TilePlan p = plan_tiles(a.S, a.T, base.max_new, a.H, a.H_kv, base.rows_few, a.max_kv);
    *refused = p.pairs * a.H_kv * p.n_split >= (1ll << 31);
    if (*refused) return cudaSuccess;
    TileParams P;
    P.c = base;
    P.c.part = part;
    P.tok = p.tok;
    P.q_rows = p.tok * base.group;
    P.n_split = p.n_split;
    P.div_split.set(static_cast<uint32_t>(p.n_split));
    P.div_hkv.set(static_cast<uint32_t>(a.H_kv));
    P.c.box_rows = paged_gcd(a.page_size, kBN);
    CUtensorMap mq, mk, mv;
    const uint64_t row = 2ull * a.q_row_stride, head = 2ull * a.q_head_stride;
    if (!encode_16bit_4d_sw128(&mq, a.q, a.dtype == HAWK_BF16, {static_cast<uint64_t>(a.D), static_cast<uint64_t>(a.H),
                                                                static_cast<uint64_t>(a.T), 1},
                               {head, row, row}, base.group, p.tok, 1) ||
        !encode_pages(&mk, a, false, P.c.box_rows, &P.c.k_rows_inner) ||
        !encode_pages(&mv, a, true, P.c.box_rows, &P.c.v_rows_inner))
        return cudaErrorInvalidValue;
    if (a.dtype == HAWK_BF16)
        return a.D == 64 ? launch<__nv_bfloat16, 64>(mq, mk, mv, P, p.pairs, st) : launch<__nv_bfloat16, 128>(mq, mk, mv, P, p.pairs, st);
    return a.D == 64 ? launch<__half, 64>(mq, mk, mv, P, p.pairs, st) : launch<__half, 128>(mq, mk, mv, P, p.pairs, st);
}
