// hawk_paged_attn for streams that bring MANY rows (chunks of a prompt): tiles of query rows on the fifth-generation tensor
// cores, keys and values streamed page by page.
//
// A block owns one (stream, kv head, pair of 128-row query tiles).  The rows of a tile are (position, head of the group)
// pairs with the head running fastest, so grouped-query heads share every key and value tile.  Two accumulation slots a
// block give the tensor pipe something to do while the other slot's scores are in softmax, and a pair of query tiles
// halves the key/value bytes each flop asks of L2.  Where only one query tile has rows, both slots work on it, the even key
// tiles in slot 0 and the odd ones in slot 1, and are joined at the end.  Warps:
//   0-3, 4-7  softmax of slot 0 and of slot 1: one query row a thread (row maxima and sums need no shuffles)
//   8         issues every tcgen05.mma:  S_t = Q_t K^T (both operands in shared memory), O_t += P_t V (P_t in tensor
//             memory, V in shared memory read along its rows)
//   9, 10     loads: Q once and K tiles of 128 keys, V tiles, each its part of the ring, as boxes that stay inside a page, a box a lane
// Tensor memory: S_0, S_1 (128 columns each; P_t overwrites the first half of S_t in 16 bits), O_0, O_1 (D columns each).
// Order of the products: S_0(0) S_1(0) | P_0(i)V S_0(i+1) P_1(i)V S_1(i+1) | ..., so one slot's softmax runs under the
// other slot's two products, and when S_t(i) is complete so is O_t up to tile i-1: the softmax warps rescale O_t in
// place without any other handshake.  They do so only when a row's maximum has grown by more than 2^8 since the last
// time (any shift keeps the softmax exact as long as O and the sum use the same one; 2^8 leaves fp16 and fp32 ample room).
// P is handed over in two halves, so that P V starts on the first 64 keys while the others are in the exponential.
// At D = 64 the exponentials bound the loop (128 x 128 of them a tile against 512 cycles of products): every fourth pair
// is computed on the FMA pipe instead, 2^x = 2^n 2^f with n the nearest integer and a degree-4 polynomial for 2^f on
// [-1/2, 1/2] (least squares on Chebyshev points, relative error 2.6e-6); 4 x 2048 rows over 8192 keys, 32 heads sharing 8: 726 to
// 702 us.  At D = 128 it gains nothing (790 against 794).
// Measured there in a graph of back-to-back calls: 1.2 PFLOP/s at D = 128, 0.72 of the measured burst peak (called alone 931 us,
// 1.03 PFLOP/s).  What it took: MMAs issued under a predicate with
// descriptors stepped by their low word (980 to 790 us; see umma_f16_ss_if).  Two score buffers of 64 keys a slot, so that the next
// scores never wait for P V, came to 916 us: products of 64 columns read Q from shared memory twice as often.
// Jobs come from a list that one extra block of the rows kernel (which every call launches before this one) makes: a block reads
// one record instead of searching the batch, and the longest jobs start first.
// One warp issued a tile's boxes of 16 keys (32 at D = 128) one lane after the other, some 90 cycles each, which paced a single query
// tile; two warps took 4 x 128 rows over 2816 keys from 53 to 43 us (pairs of query tiles, which need half as many: 138 to 139).
// Measured and taken back: results leaving as whole rows through shared memory (140 to 146 us for 16 x 511 rows over 600 keys: row by
// row the stores need nobody to wait for them); tensor memory taken before the job is known (148).
// Few blocks: the key range is split too, each split leaves (o, max, sum) in fp32 and a second kernel joins them.
// Measured and taken back: one persistent block per SM over equal shares of all key tiles.  Changing segments inside a block
// costs what changing blocks does (some 10 k cycles of draining, epilogue, queries and first scores), cuts add partial results,
// and the clock under the power cap was lower: 868 against 793 us for the prefill above, 137 against 119 for 4 x 512 rows.
#include <atomic>

#include "hawk_paged.cuh"

namespace {

using namespace hawk;

constexpr int kBM = 128, kBN = 128;
constexpr int kThreads = 384;        // three warpgroups; the third has one warp for the products and two for the loads
constexpr int kRegsSoftmax = 224, kRegsOther = 56;  // of the 168 a thread that the block starts with (2 x 224 + 56 = 3 x 168)
constexpr int kMaxSplits = 16;
constexpr int kMinSplitKeys = 512;  // shorter key ranges cost more in partial results than they gain in blocks

struct TileParams {
    PagedParams c;
    const PagedGroup *groups;  // the call's pairs of query tiles, longest first
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
    // partial result of a block: o as [D / 4][256 rows][4], so that a warp's rows are neighbours, then (max, sum) of the rows
    static constexpr int kPartFloats = 2 * kBM * (D + 2);
    static constexpr size_t kSmem = 1024 + static_cast<size_t>(2 + kStages) * kTileBytes + 512 + 1024 /* max, sum of slot 1's rows */;
};

// What the block works on.
struct TileJob {
    int s, hk, split;
    int r0, n, kv;
    int tok0;            // first position of the block's first query tile
    int nt[2];           // key tiles of each slot
    int tiles;           // key tiles of the block, counted from tile `begin`
    int begin;           // first key tile of the split
    bool single;         // one query tile, its key tiles dealt out to the two slots
};

// The block's job (or, without `with_split`, its group and kv head) from the sorted list; false behind the list's end.
__device__ __forceinline__ bool find_job(const TileParams &P, bool with_split, TileJob &job)
{
    uint32_t split = 0, hk;
    const uint32_t group_hk = with_split ? P.div_split.divmod(blockIdx.x, split) : blockIdx.x;
    const uint32_t rank = P.div_hkv.divmod(group_hk, hk);
    const int4 a = *reinterpret_cast<const int4 *>(P.groups + rank);
    const int2 b = *reinterpret_cast<const int2 *>(reinterpret_cast<const int4 *>(P.groups + rank) + 1);
    PagedStream st;
    job.s = a.x;
    job.r0 = a.y;
    job.n = st.n = a.z;
    job.kv = st.kv = a.w;
    job.tok0 = b.x;
    job.split = static_cast<int>(split);
    job.hk = static_cast<int>(hk);
    if (job.n == 0) return false;  // (the list ends with an empty record)
    const int pfx = st.kv - st.n;
    int end[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int first = job.tok0 + t * P.tok;
        const int keys = first < st.n ? max(0, min(st.kv, pfx + paged_reach(P.c, st.n, first + P.tok))) : 0;
        end[t] = (keys + kBN - 1) / kBN;
    }
    const int all = max(end[0], end[1]);
    job.begin = static_cast<int>(static_cast<long long>(all) * job.split / P.n_split);
    const int stop = static_cast<int>(static_cast<long long>(all) * (job.split + 1) / P.n_split);
#pragma unroll
    for (int t = 0; t < 2; ++t) job.nt[t] = max(0, min(end[t], stop) - job.begin);
    job.tiles = max(job.nt[0], job.nt[1]);
    job.single = job.tok0 + P.tok >= st.n;
    if (job.single) {
        job.nt[0] = (job.tiles + 1) / 2;
        job.nt[1] = job.tiles / 2;
    }
    return true;
}

// 2^x of two numbers on the FMA pipe, -126 <= x < 127 (smaller ones give 2^-126).
__device__ __forceinline__ float2 exp2_fma(uint64_t x2)
{
    float2 x = unpack2(x2);
    x.x = fmaxf(x.x, -126.f);
    x.y = fmaxf(x.y, -126.f);
    const uint64_t v = pack2(x.x, x.y);
    constexpr float kRound = 12582912.f;  // 1.5 * 2^23: adding it leaves the nearest integer in the low mantissa bits
    const uint64_t n = add2(v, pack2(kRound, kRound));
    const uint64_t f = add2(v, fma2(n, pack2(-1.f, -1.f), pack2(kRound, kRound)));  // x - nearest integer
    uint64_t p = fma2(pack2(0.0095701f, 0.0095701f), f, pack2(0.05591786f, 0.05591786f));
    p = fma2(p, f, pack2(0.24024745f, 0.24024745f));
    p = fma2(p, f, pack2(0.69312181f, 0.69312181f));
    p = fma2(p, f, pack2(0.99999926f, 0.99999926f));
    const float2 pf = unpack2(p), nf = unpack2(n);
    return make_float2(__int_as_float(__float_as_int(pf.x) + (__float_as_int(nf.x) << 23)),
                       __int_as_float(__float_as_int(pf.y) + (__float_as_int(nf.y) << 23)));
}

// Bits c = 0 .. 31 of a tree row: may it see the key `rel + c` places behind the prefix?  (rel < 0: some lie in the prefix.)
__device__ __forceinline__ uint32_t tree_word(int rel, uint64_t nodes)
{
    if (rel <= -32) return 0xffffffffu;
    if (rel < 0) return static_cast<uint32_t>(nodes << -rel) | ((1u << -rel) - 1u);
    return rel < 64 ? static_cast<uint32_t>(nodes >> rel) : 0u;
}

// mbar_wait of a whole warp: true for all its lanes or for none, so that the warp stays together when a wait gives up.
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity, volatile int *abort_flag)
{
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
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
    uint8_t *q_smem = smem;                              // two query tiles; at the end slot 1's O of a single tile
    uint8_t *ring = smem + 2 * C::kTileBytes;            // K and V tiles in turn
    float2 *ml_smem = reinterpret_cast<float2 *>(ring + C::kStages * C::kTileBytes);  // [128]
    uint64_t *bars = reinterpret_cast<uint64_t *>(ml_smem + 128);
    uint64_t *full = bars, *empty = bars + C::kStages;
    uint64_t *q_full = bars + 2 * C::kStages, *s_full = q_full + 1, *p_ready = q_full + 3, *o_done = q_full + 7, *drain = q_full + 9;
    uint32_t *tmem_ptr = reinterpret_cast<uint32_t *>(drain + 1);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_ptr + 1);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 9 * 32) {  // (the warp that loads: it starts before the others are told)
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        mbar_init(q_full, 1);
        for (int t = 0; t < 2; ++t) {
            mbar_init(&s_full[t], 1);
            mbar_init(&p_ready[2 * t], 4);
            mbar_init(&p_ready[2 * t + 1], 4);
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
    if (!find_job(P, true, job)) return;  // (block-uniform)
    if (warp == 8) {
        tmem_alloc(tmem_ptr, 512);
        tmem_relinquish();
    }
    if (warp == 9) {
        __syncwarp();
        // The barriers are there; the loads need nothing else.  (Named barrier 2, not 0: this warp does not wait here, and a job
        // without keys or a slow tensor-memory allocation can bring it to the block's last barrier before the others pass this one.)
        asm volatile("bar.arrive 2, %0;" ::"n"(kThreads) : "memory");
    } else {
        tcgen05_fence_before();
        asm volatile("bar.sync 2, %0;" ::"n"(kThreads) : "memory");
        tcgen05_fence_after();
    }
    constexpr uint32_t tmem = 0;  // all 512 columns are the block's: its tensor memory starts at lane 0, column 0
    const int pfx = job.kv - job.n;

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
        // stages for keys, the others are for values: a single query tile starts on two key tiles, a pair holds value tiles longer
        const int key_stages = job.single ? (C::kStages + 1) / 2 : C::kStages / 2;
        if (warp == 9 || warp == 10) {
            // -------------------------------------------------------------- loads: queries and keys, or values
            const bool values = warp == 10;
            bool ok = true;
            int issued = 0;  // tiles of this warp
            if (job.tiles > 0) {
                // Keys and values that few other blocks read pass through L2 marked evict-first, which makes room without a search: 7B
                // chunks of 300 to 511 rows 70 us against 78 kept, 8 x 512 rows of 32 heads on 8 over 2048 keys 159 against
                // 164.  From 32 pairs of query tiles on it pays to keep them (794 against 815 us for 4 x 2048 rows of 32
                // heads on 8 over 8192 keys; 16 pairs: the same).
                const uint64_t policy = job.n > 32 * P.tok ? l2_policy_evict_last() : l2_policy_evict_first();
                // lane l loads 64-column half l % halves of box l / halves of every tile (at most 32 of them: boxes have
                // 8 rows or more); its page id is fetched three tiles ahead
                const CUtensorMap *map = values ? &map_v : &map_k;
                const int rows_inner = values ? P.c.v_rows_inner : P.c.k_rows_inner;
                const int hf = lane % C::kHalves;
                const int box_key = lane / C::kHalves * P.c.box_rows;
                const int32_t *tb = P.c.block_table + static_cast<size_t>(job.s) * P.c.table_width;
                auto key_of = [&](int i) { return (job.begin + i) * kBN + box_key; };
                auto has_box = [&](int i) { return i < job.tiles && box_key < kBN && key_of(i) < job.kv; };
                auto page_id = [&](int i) {
                    return has_box(i) ? tb[P.c.div_page.div(static_cast<uint32_t>(key_of(i)))] : 0;
                };
                const int base = values ? key_stages : 0, depth = values ? C::kStages - key_stages : key_stages;
                int at = 0;         // stage of tile i, and the parity of its use
                uint32_t use = 0;
                int id[4] = {page_id(0), page_id(1), page_id(2), 0};  // (on their way while Q is asked for)
                if (!values && lane == 0) {
                    const int q_tiles = job.single ? 1 : 2;
                    mbar_arrive_expect_tx(q_full, q_tiles * C::kHalves * P.q_rows * 128);
                    for (int t = 0; t < q_tiles; ++t)
                        for (int hf = 0; hf < C::kHalves; ++hf)
                            tma_load_4d(q_smem + t * C::kTileBytes + hf * C::kHalfBytes, &map_q, hf * 64, job.hk * P.c.group,
                                        job.r0 + job.tok0 + t * P.tok, 0, q_full);
                }
                for (int i = 0; i < job.tiles; ++i) {
                    id[3] = page_id(i + 3);
                    const int st = base + at;
                    if (i >= depth) ok = warp_wait(&empty[st], use ^ 1u, abort_flag);
                    if (!ok) break;
                    const int rows = min(kBN, (job.kv - (job.begin + i) * kBN + P.c.box_rows - 1) & -P.c.box_rows);
                    if (lane == 0) {
                        // (test builds only: the first tile of the first block is armed for more bytes than arrive)
                        const bool stall = kTestStallBytes != 0 && blockIdx.x == 0 && i == 0 && !values;
                        mbar_arrive_expect_tx(&full[st], rows * 128 * C::kHalves + (stall ? kTestStallBytes : 0u));
                    }
                    __syncwarp();
                    ++issued;
                    if (has_box(i)) {
                        if (id[0] < 0 || id[0] >= P.c.n_pages) flags |= HAWK_DEV_BAD_PAGE;  // (outside the tensor map: zeros)
                        uint32_t row;
                        P.c.div_page.divmod(static_cast<uint32_t>(key_of(i)), row);
                        paged_load(ring + st * C::kTileBytes + hf * C::kHalfBytes + box_key * 128, map, rows_inner, hf,
                                   static_cast<int>(row), job.hk, id[0], &full[st], policy);
                    }
                    __syncwarp();
                    id[0] = id[1];
                    id[1] = id[2];
                    id[2] = id[3];
                    if (++at == depth) {
                        at = 0;
                        use ^= 1u;
                    }
                }
                // what is in flight lands before the block retires, whoever gives up later (bounded waits)
                if (!ok) *abort_flag = 1;
                if (!values) ok = warp_wait(q_full, 0, nullptr) && ok;
                for (int i = max(0, issued - depth); i < issued; ++i)
                    ok = warp_wait(&full[base + i % depth], (i / depth) & 1u, nullptr) && ok;
                if (!ok) flags |= HAWK_DEV_TIMEOUT;
            }
            if (flags && P.c.dev_status) atomicOr(P.c.dev_status, flags);
        } else if (warp == 8 && job.tiles > 0) {
            // -------------------------------------------------------------- products
            constexpr uint32_t idesc_s = umma_idesc_f16kind(kBM, kBN, E::kBf16, false);
            constexpr uint32_t idesc_o = umma_idesc_f16kind(kBM, D, E::kBf16, true);
            const uint32_t lead = elect_one();
            // broadcasts: what the loop runs on is warp-uniform for the compiler too (uniform registers, no divergence)
            const int nt0 = __shfl_sync(0xffffffffu, job.nt[0], 0), nt1 = __shfl_sync(0xffffffffu, job.nt[1], 0);
            const int tiles = __shfl_sync(0xffffffffu, job.tiles, 0);
            const int all_keys = __shfl_sync(0xffffffffu, job.kv - job.begin * kBN, 0);  // keys from the block's first tile on
            const bool single = __shfl_sync(0xffffffffu, static_cast<int>(job.single), 0) != 0;
            const uint64_t qd = umma_desc_k_major_sw128(smem_u32(q_smem)), kd = umma_desc_k_major_sw128(smem_u32(ring)),
                           vd = umma_desc_mn_major_sw128(smem_u32(ring), C::kHalfBytes);
            const uint32_t q_lo = static_cast<uint32_t>(qd), k_lo = static_cast<uint32_t>(kd), v_lo = static_cast<uint32_t>(vd);
            const uint32_t qk_hi = static_cast<uint32_t>(qd >> 32), v_hi = static_cast<uint32_t>(vd >> 32);
            bool ok = warp_wait(q_full, 0, abort_flag);
            const int n_key = __shfl_sync(0xffffffffu, key_stages, 0);
            int k_at = 0, v_at = n_key;
            uint32_t k_use = 0, v_use = 0;
            auto acquire = [&](bool values) {  // the next tile of keys or of values
                const int st = values ? v_at : k_at;
                ok = ok && warp_wait(&full[st], values ? v_use : k_use, abort_flag);
                if (values && ++v_at == C::kStages) {
                    v_at = n_key;
                    v_use ^= 1u;
                }
                if (!values && ++k_at == n_key) {
                    k_at = 0;
                    k_use ^= 1u;
                }
                return st;
            };
            auto release = [&](int st) {
                if (ok) umma_commit_if(lead, &empty[st]);
            };
            auto scores = [&](int t, int st) {
                if (!ok) return;
                const uint32_t a = q_lo + ((single ? 0 : t * C::kTileBytes) >> 4);
                const uint32_t b = k_lo + ((st * C::kTileBytes) >> 4);
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    constexpr int kHalf16 = C::kHalfBytes >> 4;
                    const uint32_t off = (kk >> 2) * kHalf16 + (kk & 3) * 2;
                    umma_f16_ss_if(lead, tmem + t * kBN, a + off, qk_hi, b + off, qk_hi, idesc_s, kk > 0);
                }
                umma_commit_if(lead, &s_full[t]);
            };
            auto values = [&](int t, int i, int st) {
                const uint32_t b = v_lo + ((st * C::kTileBytes) >> 4);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    ok = ok && warp_wait(&p_ready[2 * t + half], i & 1u, abort_flag);
                    if (!ok) return;
                    tcgen05_fence_after();
#pragma unroll
                    for (int kk = half * 4; kk < half * 4 + 4; ++kk)
                        umma_f16_ts_if(lead, tmem + 256 + t * D, tmem + t * kBN + kk * 8, b + kk * 128, v_hi, idesc_o, i > 0 || kk > 0);
                }
                if (i + 1 == (t == 0 ? nt0 : nt1)) umma_commit_if(lead, &o_done[t]);
            };
            auto clean = [&](int tile, int st) {
                // values behind the last key hold anything: zero them (0 * NaN is NaN)
                const int left = all_keys - tile * kBN;  // keys of the tile that exist
                if (!ok || left >= kBN) return;
                uint8_t *v = ring + st * C::kTileBytes;
                for (int x = left * 8 + lane; x < kBN * 8; x += 32)
                    for (int hf = 0; hf < C::kHalves; ++hf)
                        *reinterpret_cast<uint4 *>(v + hf * C::kHalfBytes + x * 16) = make_uint4(0u, 0u, 0u, 0u);
                fence_proxy_async();
                __syncwarp();
            };
            if (single) {
                int st = acquire(false);
                scores(0, st);
                release(st);
                if (tiles > 1) {
                    st = acquire(false);
                    scores(1, st);
                    release(st);
                }
                for (int j = 0; j < tiles && ok; ++j) {
                    const int t = j & 1, v = acquire(true);
                    clean(j, v);
                    values(t, j >> 1, v);
                    release(v);
                    if (j + 2 < tiles) {
                        const int k = acquire(false);
                        scores(t, k);
                        release(k);
                    }
                }
            } else {
                int k = acquire(false);
                if (nt0 > 0) scores(0, k);
                if (nt1 > 0) scores(1, k);
                release(k);
                for (int i = 0; i < tiles && ok; ++i) {
                    const int v = acquire(true);
                    clean(i, v);
                    if (i < nt0) values(0, i, v);
                    if (i + 1 < tiles) k = acquire(false);
                    if (i + 1 < nt0) scores(0, k);
                    if (i < nt1) values(1, i, v);
                    release(v);
                    if (i + 1 < nt1) scores(1, k);
                    if (i + 1 < tiles) release(k);
                }
            }
            // every product issued has finished before the block gives its tensor memory back
            __syncwarp();
            umma_commit_if(lead, drain);
            if (!ok) *abort_flag = 1;
            if (!warp_wait(drain, 0, nullptr)) ok = false;
            if (!ok && lane == 0 && P.c.dev_status) atomicOr(P.c.dev_status, HAWK_DEV_TIMEOUT);
        }
    } else {
        // ------------------------------------------------------------------ softmax and epilogue of slot t
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
        const int t = warp >> 2;
        const int r = tid & 127;
        const uint32_t lane_off = static_cast<uint32_t>(warp & 3) << 21;  // 32 lanes of tensor memory per warp
        const uint32_t s_addr = tmem + lane_off + t * kBN, o_addr = tmem + lane_off + 256 + t * D;
        uint32_t hd;
        const int pos = job.tok0 + (job.single ? 0 : t * P.tok) + static_cast<int>(P.c.div_group.divmod(static_cast<uint32_t>(r), hd));
        const bool valid = r < P.q_rows && pos < job.n;
        // keys this row sees: all up to itself in a chain; in a tree all in front of the chunk, and the nodes of its mask
        uint64_t nodes = 0;
        int limit = min(job.kv, pfx + min(pos, job.n - 1) + 1);
        if (P.c.anc_mask) {
            limit = pfx;
            nodes = P.c.anc_mask[min(pos, job.n - 1)];
            if (job.n < 64) nodes &= (1ull << job.n) - 1;
        }
        const int first = job.begin + (job.single ? t : 0), stride = job.single ? 2 : 1;  // key tiles of the slot
        const uint64_t scale2 = pack2(P.c.scale_log2, P.c.scale_log2);
        float m_run = -CUDART_INF_F, l_run = 0.f;
        const int nt = job.nt[t];
        bool ok = true;
        uint32_t u[4][32];
        float m_new = 0.f;
        auto take_scores = [&](int i) {  // tile i's scores, masked, and the row's maximum with them
            ok = warp_wait(&s_full[t], i & 1u, abort_flag);
            if (!ok) return false;
            tcgen05_fence_after();
#pragma unroll
            for (int q = 0; q < 4; ++q) tmem_ld_32x32(s_addr + q * 32, u[q]);
            tmem_ld_wait();
            const int seen = limit - (first + i * stride) * kBN;
            if (seen < kBN) {
                if (P.c.anc_mask) {
                    // (seen counts the keys in front of the tree here)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const uint32_t open = tree_word(q * 32 - seen, nodes);
#pragma unroll
                        for (int c = 0; c < 32; ++c)
                            if (!(open >> c & 1u)) u[q][c] = 0xff800000u;
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
#pragma unroll
                        for (int c = 0; c < 32; ++c)
                            if (q * 32 + c >= seen) u[q][c] = 0xff800000u;  // -inf
                }
            }
            __syncwarp();  // (whole-warp tensor-memory instructions follow)
            float mx[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                mx[q] = __uint_as_float(u[q][0]);
#pragma unroll
                for (int c = 1; c < 32; ++c) mx[q] = fmaxf(mx[q], __uint_as_float(u[q][c]));
            }
            m_new = fmaxf(m_run, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])));
            return true;
        };
        auto renew = [&](int i) {  // m_new becomes the shift
            if (i > 0) {
                const float mu = m_new == -CUDART_INF_F ? 0.f : m_new;
                const float alpha = fast_exp2((m_run - mu) * P.c.scale_log2);
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
            m_run = m_new;
        };
        auto exponentials = [&](uint64_t shift2) {  // the tile's probabilities, handed over in halves, and their sum
            uint64_t sum_a = 0, sum_b = 0;        // (two zeros each)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t pk[32];
#pragma unroll
                for (int c = 0; c < 32; ++c) {
                    const int q = half * 2 + (c >> 4), e = (2 * c) & 31;
                    const uint64_t x2 = fma2(pack2(__uint_as_float(u[q][e]), __uint_as_float(u[q][e + 1])), scale2, shift2);
                    float2 p;
                    if (D == 64 && c % 4 == 3) {
                        p = exp2_fma(x2);
                    } else {
                        p = unpack2(x2);
                        p.x = fast_exp2(p.x);
                        p.y = fast_exp2(p.y);
                    }
                    if (c & 1) sum_b = add2(sum_b, pack2(p.x, p.y));
                    else sum_a = add2(sum_a, pack2(p.x, p.y));
                    pk[c] = E::pack(p.x, p.y);
                }
                tmem_st_32x32(s_addr + half * 32, pk);
                tmem_st_wait();
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_ready[2 * t + half]);
            }
            const float2 sums2 = unpack2(add2(sum_a, sum_b));
            l_run += sums2.x + sums2.y;
        };
        // The same for far shifts (see kFarShift), differences first.  A small loop over 32 columns that takes the scores from tensor
        // memory again (a part's probabilities go over scores that it has read): as long as the loop above, its code alone cost jobs
        // of few tiles 5 %.
        auto far_exponentials = [&](int i) {
            const int seen = limit - (first + i * stride) * kBN;
            const float minus = m_run == -CUDART_INF_F ? 0.f : -m_run;
            const uint64_t minus2 = pack2(minus, minus);
            uint64_t sum = 0;
#pragma unroll 1
            for (int q = 0; q < 4; ++q) {
                uint32_t w[32], pk[16];
                __syncwarp();
                tmem_ld_32x32(s_addr + q * 32, w);
                tmem_ld_wait();
                const int left = seen - q * 32;
                const uint32_t open = P.c.anc_mask ? tree_word(-left, nodes) : left >= 32 ? 0xffffffffu : left <= 0 ? 0u : (1u << left) - 1u;
#pragma unroll
                for (int c = 0; c < 32; ++c)
                    if (!(open >> c & 1u)) w[c] = 0xff800000u;
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    float2 p = unpack2(mul2(add2(pack2(__uint_as_float(w[2 * c]), __uint_as_float(w[2 * c + 1])), minus2), scale2));
                    p.x = fast_exp2(p.x);
                    p.y = fast_exp2(p.y);
                    sum = add2(sum, pack2(p.x, p.y));
                    pk[c] = E::pack(p.x, p.y);
                }
                __syncwarp();
                tmem_st_32x16(s_addr + q * 16, pk);
                tmem_st_wait();
                if (q & 1) {
                    tcgen05_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&p_ready[2 * t + (q >> 1)]);
                }
            }
            const float2 sums2 = unpack2(sum);
            l_run += sums2.x + sums2.y;
        };
        // what the fma adds to a row's scores: minus the shift, or for a row without one so much that any score is too high (-inf stays
        // -inf)
        constexpr float kNoShift = 3e38f;
        float sh = kNoShift;
        for (int i = 0; i < nt; ++i) {
            if (!take_scores(i)) break;
            // (a tile's last rows may be another stream's or nobody's: they have no vote)
            if (__any_sync(0xffffffffu, valid && fmaf(m_new, P.c.scale_log2, sh) > 8.f)) {
                renew(i);
                sh = m_run == -CUDART_INF_F ? kNoShift : -m_run * P.c.scale_log2;
                // far shifts are renewed at every tile, so that the loop's usual way knows nothing of them (a flag in it cost the
                // prefill 2 % at D = 128 and 5 % at D = 64; this way 0 and 1)
                if (__any_sync(0xffffffffu, valid && is_far(m_run, P.c.scale_log2))) {
                    far_exponentials(i);
                    sh = kNoShift;  // (so that the next tile comes here again)
                    continue;
                }
            }
            exponentials(pack2(sh, sh));
        }
        if (ok && nt > 0) ok = warp_wait(&o_done[t], 0, abort_flag);
        if (ok && job.single && job.tiles > 1) ok = warp_wait(&o_done[t ^ 1], 0, abort_flag);  // (Q is free then)
        if (!ok) *abort_flag = 1;
        tcgen05_fence_after();
        if (m_run == -CUDART_INF_F && l_run == l_run) l_run = 0.f;  // a row that has seen no key (NaN scores: NaN)
        // the tensor-memory loads below are for whole warps: rows that do not exist take part and store nothing
        float f_own = 1.f, f_other = 0.f;  // weights of the two slots' O where they are joined
        auto other_at = [&](int c) {       // 16-byte chunk c of row r of slot 1's O (the chunk index turned by the row: no conflicts)
            return reinterpret_cast<uint4 *>(q_smem) + r * (D / 4) + (c ^ (r & (D / 4 - 1)));
        };
        if (job.single) {
            if (t == 1) {
                ml_smem[r] = make_float2(m_run, l_run);
                if (nt > 0) {
#pragma unroll
                    for (int c0 = 0; c0 < D; c0 += 32) {
                        uint32_t o[32];
                        tmem_ld_32x32(o_addr + c0, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int c = 0; c < 32; c += 4) *other_at((c0 + c) / 4) = make_uint4(o[c], o[c + 1], o[c + 2], o[c + 3]);
                    }
                }
            }
            asm volatile("bar.sync 1, 256;" ::: "memory");
            if (t == 0) {
                const float2 o = ml_smem[r];
                const float m = fmaxf(m_run, o.x);
                const float mu = m == -CUDART_INF_F ? 0.f : m;
                f_own = l_run == 0.f ? 0.f : fast_exp2((m_run - mu) * P.c.scale_log2);
                f_other = o.y == 0.f ? 0.f : fast_exp2((o.x - mu) * P.c.scale_log2);
                l_run = l_run * f_own + o.y * f_other;
                m_run = m;
            }
        }
        if (!job.single || t == 0) {
            const long long row = job.r0 + static_cast<long long>(pos);
            const long long cell = row * P.c.H + job.hk * P.c.group + static_cast<int>(hd);
            const bool join = job.single && job.nt[1] > 0;
            const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
            T16 *dst = static_cast<T16 *>(P.c.out) + (valid ? cell * D : 0);
            float *part = P.c.part + static_cast<size_t>(blockIdx.x) * C::kPartFloats;
            const int prow = (job.single ? 0 : t * kBM) + r;
            if (P.n_split > 1 && !HAWK_IN_BOUNDS(P.c.dev_status, part - P.c.part + C::kPartFloats - 1, P.c.part_floats)) ok = false;
            if (P.n_split > 1 && valid && ok) *reinterpret_cast<float2 *>(part + 2 * kBM * D + 2 * prow) = make_float2(m_run, l_run);
            // (a split without keys has sum 0 and its o is not read)
            if (nt > 0 || P.n_split == 1) {
#pragma unroll
                for (int c0 = 0; c0 < D; c0 += 32) {
                    uint32_t o[32];
                    __syncwarp();  // (rows that store and rows that do not, together again)
                    if (nt > 0) {
                        tmem_ld_32x32(o_addr + c0, o);
                        tmem_ld_wait();
                    }
#pragma unroll
                    for (int c = 0; c < 32; c += 4) {
                        float v[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[k] = l_run == 0.f ? 0.f : __uint_as_float(o[c + k]);
                        if (join) {
                            const uint4 x = *other_at((c0 + c) / 4);
                            // (a slot without mass for this row may hold anything)
                            v[0] = (f_own == 0.f ? 0.f : v[0] * f_own) + (f_other == 0.f ? 0.f : __uint_as_float(x.x) * f_other);
                            v[1] = (f_own == 0.f ? 0.f : v[1] * f_own) + (f_other == 0.f ? 0.f : __uint_as_float(x.y) * f_other);
                            v[2] = (f_own == 0.f ? 0.f : v[2] * f_own) + (f_other == 0.f ? 0.f : __uint_as_float(x.z) * f_other);
                            v[3] = (f_own == 0.f ? 0.f : v[3] * f_own) + (f_other == 0.f ? 0.f : __uint_as_float(x.w) * f_other);
                        }
#pragma unroll
                        for (int k = 0; k < 4; ++k) o[c + k] = __float_as_uint(v[k]);
                    }
                    if (!valid || !ok) continue;
                    if (!HAWK_IN_BOUNDS(P.c.dev_status, cell * D + c0 + 31, static_cast<long long>(P.c.T) * P.c.H * D)) continue;
                    if (P.n_split == 1) {
#pragma unroll
                        for (int c = 0; c < 32; c += 8) {
                            uint32_t w[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                w[k] = E::pack(__uint_as_float(o[c + 2 * k]) * inv, __uint_as_float(o[c + 2 * k + 1]) * inv);
                            *reinterpret_cast<uint4 *>(dst + c0 + c) = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                    } else {
#pragma unroll
                        for (int c = 0; c < 32; c += 4)
                            *reinterpret_cast<uint4 *>(part + ((c0 + c) / 4 * 2 * kBM + prow) * 4) =
                                make_uint4(o[c], o[c + 1], o[c + 2], o[c + 3]);
                    }
                }
            }
        }
    }
    __syncwarp();
    tcgen05_fence_before();
    __syncthreads();
    if (warp == 8) tmem_dealloc(*tmem_ptr, 512);
}

// Joins the splits: 8 blocks per (pair of query tiles, kv head), 32 rows each, a row a lane and the head dimension dealt out to
// the warps.
template <typename T16, int D>
__global__ void __launch_bounds__(256) paged_tile_merge_kernel(const TileParams P)
{
    using E = Elem<T16>;
    using C = TileCfg<D>;
    constexpr int PER = D / 32;  // 16-byte pieces of a row that a warp takes: D / 4 over 8 warps
    allow_dependent_launch();
    grid_dependency_wait();
    TileJob job;
    if (!find_job(P, false, job)) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int prow = blockIdx.y * 32 + lane, tile = prow / kBM;
    uint32_t hd;
    const int pos = job.tok0 + tile * P.tok + static_cast<int>(P.c.div_group.divmod(static_cast<uint32_t>(prow - tile * kBM), hd));
    if (prow - tile * kBM >= P.q_rows || pos >= job.n) return;
    const float *parts = P.c.part + static_cast<size_t>(blockIdx.x) * P.n_split * C::kPartFloats;
    float m = -CUDART_INF_F;
    for (int x = 0; x < P.n_split; ++x) {
        const float2 v = *reinterpret_cast<const float2 *>(parts + static_cast<size_t>(x) * C::kPartFloats + 2 * kBM * D + 2 * prow);
        if (v.y != 0.f) m = fmaxf(m, v.x);
    }
    float4 acc[PER];
    float l = 0.f;
#pragma unroll
    for (int c = 0; c < PER; ++c) acc[c] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
    for (int x = 0; x < P.n_split; ++x) {
        const float *p = parts + static_cast<size_t>(x) * C::kPartFloats;
        const float2 v = *reinterpret_cast<const float2 *>(p + 2 * kBM * D + 2 * prow);
        const float f = v.y == 0.f ? 0.f : fast_exp2((v.x - m) * P.c.scale_log2);
        l = fmaf(v.y, f, l);
#pragma unroll
        for (int c = 0; c < PER; ++c) {
            const float4 o = *reinterpret_cast<const float4 *>(p + ((warp * PER + c) * 2 * kBM + prow) * 4);
            if (f == 0.f) continue;  // (its o may not have been written)
            acc[c].x = fmaf(o.x, f, acc[c].x);
            acc[c].y = fmaf(o.y, f, acc[c].y);
            acc[c].z = fmaf(o.z, f, acc[c].z);
            acc[c].w = fmaf(o.w, f, acc[c].w);
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const long long at = ((job.r0 + static_cast<long long>(pos)) * P.c.H + job.hk * P.c.group + static_cast<int>(hd)) * D + warp * PER * 4;
    T16 *dst = static_cast<T16 *>(P.c.out) + at;
    if (!HAWK_IN_BOUNDS(P.c.dev_status, at, static_cast<long long>(P.c.T) * P.c.H * D) ||
        !HAWK_IN_BOUNDS(P.c.dev_status, at + PER * 4 - 1, static_cast<long long>(P.c.T) * P.c.H * D))
        return;
#pragma unroll
    for (int c = 0; c < PER; ++c)
        *reinterpret_cast<uint2 *>(dst + 4 * c) =
            make_uint2(E::pack(acc[c].x * inv, acc[c].y * inv), E::pack(acc[c].z * inv, acc[c].w * inv));
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
    return hawk_host::launch_dependent(paged_tile_merge_kernel<T16, D>, dim3(base, 2 * kBM / 32), dim3(256), 0, st, P);
}

}  // namespace

size_t hawk_host::paged_tile_workspace_bytes(int S, int T, int max_new, int H, int H_kv, int few, int D, int max_kv)
{
    const TilePlan p = plan_tiles(S, T, max_new, H, H_kv, few, max_kv);
    const size_t list = static_cast<size_t>(p.pairs) * sizeof(PagedGroup);
    if (p.n_split == 1) return list;
    return list + static_cast<size_t>(p.pairs) * H_kv * p.n_split * sizeof(float) *
                      (D == 64 ? TileCfg<64>::kPartFloats : TileCfg<128>::kPartFloats);
}

int hawk_host::paged_tile_groups(int S, int T, int max_new, int H, int H_kv, int few)
{
    const long long pairs = plan_tiles(S, T, max_new, H, H_kv, few, 0).pairs;
    return pairs * H_kv * kMaxSplits < (1ll << 31) ? static_cast<int>(pairs) : 0;
}

cudaError_t hawk_host::launch_paged_tile(const hawk_paged_attn_args &a, const PagedParams &base, float *part, cudaStream_t st)
{
    const TilePlan p = plan_tiles(a.S, a.T, base.max_new, a.H, a.H_kv, base.rows_few, a.max_kv);
    TileParams P;
    P.c = base;
    P.groups = base.groups;
    P.c.part = part + static_cast<size_t>(p.pairs) * sizeof(PagedGroup) / sizeof(float);
    P.c.part_floats = p.n_split == 1 ? 0
                                     : static_cast<long long>(p.pairs) * a.H_kv * p.n_split *
                                           (a.D == 64 ? TileCfg<64>::kPartFloats : TileCfg<128>::kPartFloats);
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
