// hawk_paged_attn for calls of up to 64 rows per kv head: a few dozen (candidate trees, drafted blocks under grouped heads),
// or any number where the streams are few and long.
//
// Up to 64 rows share every key, so the call is bound by reading keys and values once, but past 8 rows the products are too
// many for warp-level MMAs to keep that pace.  Here the KEYS sit on the 128-row operand of tcgen05 and the rows on the
// narrow one:
//   S^T [128 keys x rows] = K Q^T          both operands as stored;       a thread of the softmax warps has one key
//   O   [rows x D]       += P V,  P^T in shared memory as [key][64 rows]: a thread writes its key's probabilities as whole
//                                  16-byte pieces, and both operands are read along their rows ("MN-major")
// The 64 columns of P are half as many rows as the operand has; its upper half reads the lower one again (a stride of 0) and is
// never looked at.  One block per SM walks an equal share of the list of 128-key tiles; a tile's scores are under way while the tile
// before is in softmax, O is there twice, so that one item's epilogue runs under the next item's products.  Warps:
//   0-3, 4-7  softmax of the rows' first and second half (a key a thread in each)
//   8, 9      epilogue: a row a lane
//   10        products    11, 12  loads of keys and of values (one warp for both issued a tile's 32 boxes of 16 keys in 3000
//             cycles, which set the pace)
// A row's shift m (see the rows kernel: it moves only when a score exceeds it by 2^8) is exact at an item's first tile, from a
// reduction across the warps; after that a vote of the four warps is all that a tile costs.  A tile renews its shifts once at most,
// whatever the scores then look like (they may exceed a new shift by what its rounding lost, again and again).  The query box
// of a short item ends in rows that are another stream's or nobody's: their shift is -inf, so that they have no vote.
// Row sums stay in the threads (a key each) until the item ends.
// Measured (D = 128, 16-row pages): 256 items of 8000 keys in 164 us at 32 rows and 172 at 60, 98 and 93 % of the rate of a
// copy; of 2400 keys 58 and 64 us against 49 of reading: some 5 us before the first product and 4 of join.  What paces a tile is
// the loads up to 32 rows and the softmax warps above.  At D = 64 a tile is 16 KB + 16 KB and the softmax sets the pace at any rows
// (256 items of 8000 keys, 24 rows: 110 us against 80).
#include <atomic>

#include "hawk_paged.cuh"

namespace {

using namespace hawk;

constexpr int kThreads = 416;
constexpr int kKeys = kPagedTileKeys;
constexpr float kLazy = 8.f;
// What is added to the scores of a row without a maximum: any finite one is then too high, and a masked one stays -inf.
constexpr float kNoShift = 3e38f;

template <int D, int NR>
struct MidCfg {
    static constexpr int kHalves = D / 64;
    static constexpr int kHalfBytes = kKeys * 128;
    static constexpr int kTileBytes = kHalves * kHalfBytes;
    static constexpr int kStages = D == 128 ? 4 : 8;  // half for keys, half for values
    static constexpr int kRing = kStages / 2;
    static constexpr int kQHalfBytes = NR * 128;
    static constexpr int kQBytes = kHalves * kQHalfBytes;
    static constexpr int kPBytes = kKeys * 128;
    // float m[2][64], alpha[64], shift[64], lost[64], wmax[2][4][32], sums[2][2][4][32]; uint64 masks[64]; barriers; small things
    static constexpr int kSmallBytes = 2 * 64 * 4 + 3 * 64 * 4 + 3 * 2 * 4 * 32 * 4 + 64 * 8 + (2 * kStages + 18) * 8 + 256;
    static constexpr size_t smem(int S)
    {
        return 1024 + static_cast<size_t>(kStages) * kTileBytes + 2 * kQBytes + 2 * kPBytes + kSmallBytes +
               (static_cast<size_t>(S) + 1) * sizeof(int);
    }
};

// Position in the list of tiles: stream, kv head, tile.
struct Cursor {
    int s, hk, tile;
    int r0, n, kv, nt;  // of the stream
    int left;           // tiles left in the share, this one included
};

__device__ __forceinline__ int tiles_of(int kv) { return max(1, (kv + kKeys - 1) / kKeys); }

__device__ __forceinline__ void enter_stream(Cursor &c, const PagedParams &P, int &flags)
{
    const PagedStream st = paged_stream(P, c.s, flags);
    c.r0 = st.r0;
    c.n = st.n;
    c.kv = st.kv;
    c.nt = tiles_of(st.kv);
}

__device__ __forceinline__ void advance(Cursor &c, const PagedParams &P, const int *prefix, int &flags)
{
    --c.left;
    ++c.tile;
    if (c.tile == c.nt && c.left > 0) {
        c.tile = 0;
        if (++c.hk == P.H_kv) {
            c.hk = 0;
            // (tiles are left, so a stream with some follows; the bound holds even if the lengths change under the call)
            do c.s = min(c.s + 1, P.S - 1);
            while (c.s < P.S - 1 && prefix[c.s + 1] == prefix[c.s]);
            enter_stream(c, P, flags);
        }
    }
}

__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity, volatile int *abort_flag)
{
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
}

// Is the predicate true in any of the 128 threads that meet at barrier `id`?
__device__ __forceinline__ bool group_any(int id, bool pred)
{
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.or.pred q, %2, 128, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"(static_cast<uint32_t>(pred)), "r"(id)
        : "memory");
    return r != 0;
}

__device__ __forceinline__ void group_sync(int id) { asm volatile("barrier.cta.sync %0, 128;" ::"r"(id) : "memory"); }

__device__ __forceinline__ float warp_redux_max(float x)
{
    float y;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
    return y;
}

template <int N>
__device__ __forceinline__ void tmem_ld_row(uint32_t addr, uint32_t (&u)[N])
{
    if constexpr (N == 32) {
        tmem_ld_32x32(addr, u);
    } else if constexpr (N == 16) {
        tmem_ld_32x16(addr, u);
    } else {
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7])
                     : "r"(addr)
                     : "memory");
    }
}

template <typename T16, int D, int NR>
__global__ void __launch_bounds__(kThreads, 1)
    paged_mid_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ CUtensorMap map_v, const PagedParams P)
{
    using C = MidCfg<D, NR>;
    using E = Elem<T16>;
    constexpr int NH = NR / 2;  // rows of a softmax group
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *ring = smem;
    uint8_t *q_smem = ring + C::kStages * C::kTileBytes;  // two items' queries
    uint8_t *p_smem = q_smem + 2 * C::kQBytes;            // two tiles' P^T
    float *m_smem = reinterpret_cast<float *>(p_smem + 2 * C::kPBytes);  // [2 items][64]: group g's row r at 32 g + r
    float *alpha = m_smem + 128;                                      // [64]
    float *shift = alpha + 64;                                        // [64]: what a row adds to its scores
    float *lost = shift + 64;                                         // [64]: what that sum of a row's maximum lacks to 0
    float *wmax = lost + 64;                                          // [2 groups][4 warps][32]
    float *sums = wmax + 256;                                         // [2 items][2 groups][4 warps][32]
    uint64_t *masks = reinterpret_cast<uint64_t *>(sums + 512);       // [64]: block rows that a row sees
    uint64_t *full = masks + 64, *empty = full + C::kStages;
    uint64_t *q_full = empty + C::kStages /* [2] */, *q_empty = q_full + 2, *s_full = q_full + 4, *p_ready = q_full + 6,
             *p_free = q_full + 8, *o_full = q_full + 10, *o_empty = q_full + 12, *l_ready = q_full + 14,
             *drain = q_full + 16;
    uint32_t *tmem_ptr = reinterpret_cast<uint32_t *>(drain + 1);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_ptr + 1);
    int *wsum = reinterpret_cast<int *>(tmem_ptr + 2);  // [16]
    int *any_far = wsum + 16;                           // [2 groups]: some row's shift is (see kFarShift)
    int *prefix = any_far + 2;                          // [S + 1]
    static_assert(2 * 64 * 4 + 3 * 64 * 4 + 768 * 4 + 64 * 8 + (2 * C::kStages + 17) * 8 + 8 + 64 + 8 <= C::kSmallBytes, "");

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&q_full[b], 1);
            mbar_init(&q_empty[b], 1);
            mbar_init(&s_full[b], 1);
            mbar_init(&p_ready[b], 8);
            mbar_init(&p_free[b], 1);
            mbar_init(&o_full[b], 1);
            mbar_init(&o_empty[b], 2);
            mbar_init(&l_ready[b], 8);
        }
        mbar_init(drain, 1);
        *abort_flag = 0;
        fence_mbar_init();
        prefetch_tensormap(&map_q);
        prefetch_tensormap(&map_k);
        prefetch_tensormap(&map_v);
    }
    // zeros where the queries of short items leave rows unwritten
    for (int i = tid; i < 2 * C::kQBytes / 16; i += kThreads) reinterpret_cast<uint4 *>(q_smem)[i] = make_uint4(0, 0, 0, 0);
    fence_proxy_async();
    grid_dependency_wait();
    int flags = 0;

    // ---- prefix sum over the streams' tiles, and this block's share
    int running = 0;
    for (int base = 0; base < P.S; base += kThreads) {
        const int s = base + tid;
        int v = 0;
        if (s < P.S) {
            const PagedStream st = paged_stream(P, s, flags);
            if (st.n > 0) v = P.H_kv * tiles_of(st.kv);
        }
        int inc = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += u;
        }
        if (lane == 31) wsum[warp] = inc;
        __syncthreads();
        int before = running, all = running;
#pragma unroll
        for (int x = 0; x < kThreads / 32; ++x) {
            if (x < warp) before += wsum[x];
            all += wsum[x];
        }
        if (s < P.S) prefix[s + 1] = before + inc;
        running = all;
        __syncthreads();
    }
    if (tid == 0) prefix[0] = 0;
    __syncthreads();
    if (flags && P.dev_status && blockIdx.x == 0) atomicOr(P.dev_status, flags);
    flags = 0;
    const int total = running, W = max(1, min(P.row_blocks, total / 2));
    const int w = static_cast<int>(blockIdx.x);
    Cursor first;
    first.s = first.hk = first.tile = first.r0 = first.n = first.kv = first.left = 0;
    first.nt = 1;
    if (w < W && total > 0) {
        const int f = static_cast<int>(static_cast<long long>(w) * total / W);
        first.left = static_cast<int>(static_cast<long long>(w + 1) * total / W) - f;
        int lo = 0, hi = P.S;  // prefix[lo] <= f < prefix[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (prefix[mid] <= f) lo = mid;
            else hi = mid;
        }
        first.s = lo;
        enter_stream(first, P, flags);
        const int loc = f - prefix[lo];
        first.hk = loc / first.nt;
        first.tile = loc - first.hk * first.nt;
    }
    if (tid == 0 && HAWK_IN_BOUNDS(P.dev_status, (w + 1) * 8 - 1, P.record_ints)) {
        int32_t *rec = P.records + static_cast<size_t>(w) * 8;
        *reinterpret_cast<int4 *>(rec) = make_int4(first.tile, first.nt, first.r0, first.n);
        *reinterpret_cast<int4 *>(rec + 4) = make_int4(first.hk, 0, total, W);
    }
    if (first.left == 0) return;  // (block-uniform)
    if (warp == 10) {
        tmem_alloc(tmem_ptr, 512);
        tmem_relinquish();
    }
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    // tensor memory, all of it the block's: scores [2][64 columns], then O [2][D]
    constexpr uint32_t kO = 128, kOStride = D;

    if (warp >= 11) {
        // ------------------------------------------------------------------ loads: queries and keys, or values
        const bool values = warp == 12;
        const int base = values ? C::kRing : 0;  // the stages of this warp
        bool ok = true;
        int issued = 0, items = 0;
        const uint64_t policy = l2_policy_evict_first();
        const CUtensorMap *map = values ? &map_v : &map_k;
        const int rows_inner = values ? P.v_rows_inner : P.k_rows_inner;
        const int hf = lane % C::kHalves, box_key = lane / C::kHalves * P.box_rows;
        auto key_of = [&](const Cursor &c) { return c.tile * kKeys + box_key; };
        auto has_box = [&](const Cursor &c) { return c.left > 0 && box_key < kKeys && key_of(c) < c.kv; };
        auto page_id = [&](const Cursor &c) {
            return has_box(c) ? P.block_table[static_cast<size_t>(c.s) * P.table_width + P.div_page.div(static_cast<uint32_t>(key_of(c)))]
                              : 0;
        };
        Cursor c = first;
        int pg = page_id(c);
        while (c.left > 0) {
            Cursor next = c;
            advance(next, P, prefix, flags);
            const int pg_next = page_id(next);  // under way while this tile's boxes go out
            if (!values && (issued == 0 || c.tile == 0)) {
                const int b = items & 1;
                if (items >= 2) ok = ok && warp_wait(&q_empty[b], ((items >> 1) - 1) & 1u, abort_flag);
                if (!ok) break;
                if (lane == 0) {
                    mbar_arrive_expect_tx(&q_full[b], C::kHalves * P.mid_tok * P.group * 128);
                    for (int h2 = 0; h2 < C::kHalves; ++h2)
                        tma_load_4d(q_smem + b * C::kQBytes + h2 * C::kQHalfBytes, &map_q, h2 * 64, c.hk * P.group, c.r0, 0, &q_full[b]);
                }
                __syncwarp();
                ++items;
            }
            const int st = base + issued % C::kRing, round = issued / C::kRing;
            if (round > 0) ok = ok && warp_wait(&empty[st], (round - 1) & 1u, abort_flag);
            if (!ok) break;
            const int rows = max(0, min(kKeys, c.kv - c.tile * kKeys) + P.box_rows - 1) & -P.box_rows;
            if (lane == 0) {
                // (test builds only: the first tile of the first share is armed for more bytes than arrive)
                const bool stall = kTestStallBytes != 0 && blockIdx.x == 0 && issued == 0 && !values;
                mbar_arrive_expect_tx(&full[st], rows * 128 * C::kHalves + (stall ? kTestStallBytes : 0u));
            }
            __syncwarp();
            ++issued;
            if (has_box(c)) {
                if (pg < 0 || pg >= P.n_pages) flags |= HAWK_DEV_BAD_PAGE;  // (outside the tensor map: zeros)
                uint32_t row;
                P.div_page.divmod(static_cast<uint32_t>(key_of(c)), row);
                paged_load(ring + st * C::kTileBytes + hf * C::kHalfBytes + box_key * 128, map, rows_inner, hf,
                           static_cast<int>(row), c.hk, pg, &full[st], policy);
            }
            __syncwarp();
            c = next;
            pg = pg_next;
        }
        // what is in flight lands before the block retires, whoever gives up later (bounded waits)
        if (!ok) *abort_flag = 1;
        for (int i = max(0, items - 2); i < items; ++i) ok = warp_wait(&q_full[i & 1], (i >> 1) & 1u, nullptr) && ok;
        for (int i = max(0, issued - C::kRing); i < issued; ++i)
            ok = warp_wait(&full[base + i % C::kRing], (i / C::kRing) & 1u, nullptr) && ok;
        if (!ok) flags |= HAWK_DEV_TIMEOUT;
        if (flags && P.dev_status) atomicOr(P.dev_status, flags);
    } else if (warp == 10) {
        // ------------------------------------------------------------------ products
        constexpr uint32_t kAlongRows = 1u << 15;  // A operand read along its rows
        constexpr uint32_t idesc_s = umma_idesc_f16kind(128, NR, E::kBf16, false);
        constexpr uint32_t idesc_o = umma_idesc_f16kind(128, D, E::kBf16, true) | kAlongRows;
        const uint32_t lead = elect_one();
        const uint64_t kd = umma_desc_k_major_sw128(smem_u32(ring)), qd = umma_desc_k_major_sw128(smem_u32(q_smem)),
                       pd = umma_desc_mn_major_sw128(smem_u32(p_smem), 0), vd = umma_desc_mn_major_sw128(smem_u32(ring), C::kHalfBytes);
        const uint32_t k_lo = static_cast<uint32_t>(kd), q_lo = static_cast<uint32_t>(qd), p_lo = static_cast<uint32_t>(pd),
                       v_lo = static_cast<uint32_t>(vd);
        const uint32_t kq_hi = static_cast<uint32_t>(kd >> 32), mn_hi = static_cast<uint32_t>(pd >> 32);
        bool ok = true;
        auto acquire = [&](int j, bool values) {  // tile j's stage
            const int st = (values ? C::kRing : 0) + j % C::kRing;
            ok = ok && warp_wait(&full[st], (j / C::kRing) & 1u, abort_flag);
            return st;
        };
        auto scores = [&](int j, int item, bool first_tile, bool last_tile) {  // S of tile j
            if (first_tile) ok = ok && warp_wait(&q_full[item & 1], (item >> 1) & 1u, abort_flag);
            const int st = acquire(j, false);
            if (!ok) return;
            tcgen05_fence_after();
            const uint32_t ka = k_lo + ((st * C::kTileBytes) >> 4), qb = q_lo + (((item & 1) * C::kQBytes) >> 4);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const uint32_t a = (kk >> 2) * (C::kHalfBytes >> 4) + (kk & 3) * 2;
                const uint32_t b = (kk >> 2) * (C::kQHalfBytes >> 4) + (kk & 3) * 2;
                umma_f16_ss_if(lead, (j & 1) * 64, ka + a, kq_hi, qb + b, kq_hi, idesc_s, kk > 0);
            }
            umma_commit_if(lead, &s_full[j & 1]);
            umma_commit_if(lead, &empty[st]);
            if (last_tile) umma_commit_if(lead, &q_empty[item & 1]);
        };
        Cursor c = first;
        int tiles = __shfl_sync(0xffffffffu, first.left, 0), item = 0;
        bool begins = true;  // tile j is its item's first in the share
        scores(0, 0, true, c.tile + 1 == c.nt || c.left == 1);
        for (int j = 0; j < tiles && ok; ++j) {
            // broadcasts: what the loop runs on is warp-uniform for the compiler too
            const bool ends = __shfl_sync(0xffffffffu, static_cast<int>(c.tile + 1 == c.nt || c.left == 1), 0) != 0;
            const int left = __shfl_sync(0xffffffffu, max(0, c.kv - c.tile * kKeys), 0);  // keys of the tile that exist
            if (j + 1 < tiles) {
                Cursor nx = c;
                advance(nx, P, prefix, flags);
                const bool nx_ends = __shfl_sync(0xffffffffu, static_cast<int>(nx.tile + 1 == nx.nt || nx.left == 1), 0) != 0;
                scores(j + 1, ends ? item + 1 : item, ends, nx_ends);
                c = nx;
            }
            const int st = acquire(j, true);
            if (ok && left < kKeys) {
                // values behind the last key hold anything: zero them (0 * NaN is NaN)
                uint8_t *v = ring + st * C::kTileBytes;
                for (int x = left * 8 + lane; x < kKeys * 8; x += 32)
                    for (int h2 = 0; h2 < C::kHalves; ++h2)
                        *reinterpret_cast<uint4 *>(v + h2 * C::kHalfBytes + x * 16) = make_uint4(0u, 0u, 0u, 0u);
                fence_proxy_async();
                __syncwarp();
            }
            const int ob = item & 1;
            if (begins && item >= 2) ok = ok && warp_wait(&o_empty[ob], ((item >> 1) - 1) & 1u, abort_flag);
            ok = ok && warp_wait(&p_ready[j & 1], (j >> 1) & 1u, abort_flag);
            if (ok) {
                tcgen05_fence_after();
                const uint32_t pa = p_lo + (((j & 1) * C::kPBytes) >> 4), vb = v_lo + ((st * C::kTileBytes) >> 4);
                const uint32_t o = kO + ob * kOStride;
#pragma unroll
                for (int kk = 0; kk < kKeys / 16; ++kk)
                    umma_f16_ss_if(lead, o, pa + kk * 128, mn_hi, vb + kk * 128, mn_hi, idesc_o, !begins || kk > 0);
                umma_commit_if(lead, &p_free[j & 1]);
                umma_commit_if(lead, &empty[st]);
                if (ends) umma_commit_if(lead, &o_full[ob]);
            }
            begins = ends;
            if (ends) ++item;
        }
        __syncwarp();
        umma_commit_if(lead, drain);
        if (!ok) *abort_flag = 1;
        if (!warp_wait(drain, 0, nullptr)) ok = false;
        if (!ok && lane == 0 && P.dev_status) atomicOr(P.dev_status, HAWK_DEV_TIMEOUT);
    } else if (warp >= 8) {
        // ------------------------------------------------------------------ epilogue of group g's rows
        const int g = warp - 8;
        const uint32_t lane_off = static_cast<uint32_t>(g) << 21;
        bool ok = true;
        Cursor c = first;
        for (int item = 0; ok && c.left > 0; ++item) {
            const int ob = item & 1;
            const int tb = c.tile, take = min(c.nt - c.tile, c.left), n = c.n, r0 = c.r0, hk = c.hk;
            const bool whole = tb == 0 && take == c.nt;
            c.tile += take - 1;
            c.left -= take - 1;
            advance(c, P, prefix, flags);
            ok = warp_wait(&o_full[ob], (item >> 1) & 1u, abort_flag);
            if (!ok) break;
            tcgen05_fence_after();
            const int r = g * NH + lane;  // row of the item
            bool valid = lane < NH && r < n * P.group;
            uint32_t hd;
            const uint32_t pos = P.div_group.divmod(static_cast<uint32_t>(valid ? r : 0), hd);
            const uint32_t o_addr = lane_off + kO + ob * kOStride;
            ok = warp_wait(&l_ready[ob], (item >> 1) & 1u, abort_flag);
            if (!ok) break;
            const float *ls = sums + ((ob * 2 + g) * 4) * 32 + lane;
            const float l = (ls[0] + ls[32]) + (ls[64] + ls[96]);
            const float inv = l == 0.f ? 0.f : 1.f / l;  // (a row that has seen no key: zeros)
            T16 *dst = static_cast<T16 *>(P.out) + ((r0 + static_cast<long long>(pos)) * P.H + hk * P.group + static_cast<int>(hd)) * D;
            float *part = P.part + (static_cast<size_t>(w) * 2 + (item > 0 ? 1 : 0)) * 64 * (D + 2);
            if (!whole && !HAWK_IN_BOUNDS(P.dev_status, part - P.part + 64 * (D + 2) - 1, P.part_floats)) valid = false;
            if (valid && !whole) *reinterpret_cast<float2 *>(part + 64 * D + 2 * r) = make_float2(m_smem[ob * 64 + g * 32 + lane], l);
#pragma unroll
            for (int c0 = 0; c0 < D; c0 += 32) {
                uint32_t o[32];
                __syncwarp();  // (rows that store and rows that do not, together again)
                tmem_ld_32x32(o_addr + c0, o);
                tmem_ld_wait();
                if (!valid) continue;
                if (whole) {
                    if (!HAWK_IN_BOUNDS(P.dev_status, dst - static_cast<T16 *>(P.out) + c0 + 31, static_cast<long long>(P.T) * P.H * D))
                        continue;
#pragma unroll
                    for (int x = 0; x < 32; x += 8) {
                        uint32_t y[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            y[i] = l == 0.f ? 0u : E::pack(__uint_as_float(o[x + 2 * i]) * inv, __uint_as_float(o[x + 2 * i + 1]) * inv);
                        *reinterpret_cast<uint4 *>(dst + c0 + x) = make_uint4(y[0], y[1], y[2], y[3]);
                    }
                } else {
#pragma unroll
                    for (int x = 0; x < 32; x += 4)
                        *reinterpret_cast<uint4 *>(part + r * D + c0 + x) = make_uint4(o[x], o[x + 1], o[x + 2], o[x + 3]);
                }
            }
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&o_empty[ob]);
        }
        if (!ok) *abort_flag = 1;
    } else {
        // ------------------------------------------------------------------ softmax of group g's rows, a key a thread
        const int g = warp >> 2, wg = warp & 3, key = tid & 127, bar_id = 1 + g;
        const uint32_t lane_off = static_cast<uint32_t>(wg) << 21;
        bool ok = true;
        Cursor c = first;
        int item = 0;
        bool begins = true;
        bool far = false;       // some row's shift is (see kFarShift)
        uint64_t lsum[NH / 2];  // of this thread's keys, two rows a register pair
        const int tiles = first.left;
        for (int j = 0; j < tiles; ++j) {
            const int b = j & 1, ob = item & 1;
            const int pfx = c.kv - c.n, key0 = c.tile * kKeys;
            if (begins) {
                // the rows' masks, and no maximum yet (the epilogue of the item before the last has read its own)
                if (item >= 2) ok = ok && warp_wait(&o_empty[ob], ((item >> 1) - 1) & 1u, abort_flag);
                if (key < NH) {
                    const int r = g * NH + key;
                    uint64_t m = 0;
                    if (r < c.n * P.group) {
                        const int pos = static_cast<int>(P.div_group.div(static_cast<uint32_t>(r)));
                        m = P.anc_mask ? P.anc_mask[pos] : pos >= 63 ? ~0ull : (2ull << pos) - 1;
                        if (c.n < 64) m &= (1ull << c.n) - 1;
                    }
                    masks[g * 32 + key] = m;
                    m_smem[ob * 64 + g * 32 + key] = -CUDART_INF_F;
                    any_far[g] = 0;
                    shift[g * 32 + key] = r < c.n * P.group ? kNoShift : -CUDART_INF_F;
                }
#pragma unroll
                for (int r2 = 0; r2 < NH / 2; ++r2) lsum[r2] = 0;
                far = false;
                group_sync(bar_id);
            }
            ok = ok && warp_wait(&s_full[b], (j >> 1) & 1u, abort_flag);
            tcgen05_fence_after();
            __syncwarp();  // (whole-warp tensor-memory instructions here and below)
            uint32_t u[NH];
            tmem_ld_row<NH>(lane_off + b * 64 + g * NH, u);
            tmem_ld_wait();
            if (key0 + kKeys > pfx) {
                const int rel = key0 + key - pfx;
                if (rel >= 0) {
#pragma unroll
                    for (int r = 0; r < NH; ++r)
                        if (rel >= 64 || !((masks[g * 32 + r] >> rel) & 1ull)) u[r] = 0xff800000u;  // -inf
                }
            }
            bool renewed = false;
            const uint64_t scale2 = pack2(P.scale_log2, P.scale_log2);
            const ulonglong2 *s4 = reinterpret_cast<const ulonglong2 *>(shift + g * 32);
            float x[NH];
            for (;;) {
                float top = -CUDART_INF_F;
#pragma unroll
                for (int r4 = 0; r4 < NH / 4; ++r4) {
                    const ulonglong2 m = s4[r4];
                    const uint32_t *s = u + 4 * r4;
                    const float2 lo = unpack2(fma2(pack2(__uint_as_float(s[0]), __uint_as_float(s[1])), scale2, m.x)),
                                 hi = unpack2(fma2(pack2(__uint_as_float(s[2]), __uint_as_float(s[3])), scale2, m.y));
                    x[4 * r4] = lo.x;
                    x[4 * r4 + 1] = lo.y;
                    x[4 * r4 + 2] = hi.x;
                    x[4 * r4 + 3] = hi.y;
                    top = fmaxf(fmaxf(top, fmaxf(lo.x, lo.y)), fmaxf(hi.x, hi.y));
                }
                if (renewed) {
                    if (far) {
#pragma unroll
                        for (int r = 0; r < NH; ++r) x[r] += lost[g * 32 + r];
                    }
                    // once a tile, whatever the scores still are.  The vote: a warp that gave up takes the others along, and the next
                    // item's shifts wait until all have read this one's
                    ok = !group_any(bar_id, !ok);
                    break;
                }
                // one vote for all: a score too high, far shifts (renewed at every tile), or a wait of this warp that gave up
                if (!group_any(bar_id, begins || far || top > kLazy || !ok)) break;
                // new maxima: across the lanes, then across the four warps
                float mine = -CUDART_INF_F;
#pragma unroll
                for (int r = 0; r < NH; ++r) {
                    const float v = warp_redux_max(__uint_as_float(u[r]));
                    if (lane == r) mine = v;
                }
                wmax[(g * 4 + wg) * 32 + lane] = mine;
                group_sync(bar_id);
                if (key < NH) {
                    const float *wm = wmax + g * 128 + key;
                    const float m_old = m_smem[ob * 64 + g * 32 + key];
                    const float m_new = fmaxf(m_old, fmaxf(fmaxf(wm[0], wm[32]), fmaxf(wm[64], wm[96])));
                    const bool none = m_new == -CUDART_INF_F;
                    const float sh = none ? kNoShift : -m_new * P.scale_log2;
                    m_smem[ob * 64 + g * 32 + key] = m_new;
                    if (g * NH + key < c.n * P.group) {
                        shift[g * 32 + key] = sh;
                        if (is_far(m_new, P.scale_log2)) any_far[g] = 1;
                    }
                    lost[g * 32 + key] = none ? 0.f : -fmaf(m_new, P.scale_log2, sh);
                    alpha[g * 32 + key] = none ? 1.f : fast_exp2((m_old - m_new) * P.scale_log2);
                }
                group_sync(bar_id);
                far = any_far[g] != 0;  // (until the item ends)
#pragma unroll
                for (int r2 = 0; r2 < NH / 2; ++r2) {
                    const float2 a2 = *reinterpret_cast<const float2 *>(alpha + g * 32 + 2 * r2);
                    lsum[r2] = mul2(lsum[r2], pack2(a2.x, a2.y));
                }
                if (!begins && wg == g && ok) {
                    // O's lanes of this group: its last product done, the next not started (P of this tile is not out)
                    ok = warp_wait(&p_free[b ^ 1], ((j - 1) >> 1) & 1u, abort_flag);
                    tcgen05_fence_after();
                    const float a = lane < NH ? alpha[g * 32 + lane] : 1.f;
                    __syncwarp();
#pragma unroll
                    for (int c0 = 0; c0 < D; c0 += 16) {
                        uint32_t o[16];
                        tmem_ld_32x16(lane_off + kO + ob * kOStride + c0, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * a);
                        tmem_st_32x16(lane_off + kO + ob * kOStride + c0, o);
                    }
                    tmem_st_wait();
                }
                renewed = true;
            }
            if (!ok) break;  // (uniform: see the votes)
            if (j >= 2) ok = ok && warp_wait(&p_free[b], ((j >> 1) - 1) & 1u, abort_flag);
            uint8_t *prow = p_smem + b * C::kPBytes + key * 128;
#pragma unroll
            for (int r8 = 0; r8 < NH / 8; ++r8) {
                uint32_t y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p0 = fast_exp2(x[8 * r8 + 2 * i]), p1 = fast_exp2(x[8 * r8 + 2 * i + 1]);
                    lsum[4 * r8 + i] = add2(lsum[4 * r8 + i], pack2(p0, p1));
                    y[i] = E::pack(p0, p1);
                }
                *reinterpret_cast<uint4 *>(prow + (((g * 4 + r8) ^ (key & 7)) << 4)) = make_uint4(y[0], y[1], y[2], y[3]);
            }
            fence_proxy_async();
            tcgen05_fence_before();
            __syncwarp();
            if (ok && lane == 0) mbar_arrive(&p_ready[b]);
            begins = c.tile + 1 == c.nt;
            if (begins || c.left == 1) {
                // the segment ends: the rows' sums over the warp's keys, a row a lane (or a few lanes)
                float v[NH];
#pragma unroll
                for (int r2 = 0; r2 < NH / 2; ++r2) {
                    const float2 l2 = unpack2(lsum[r2]);
                    v[2 * r2] = l2.x;
                    v[2 * r2 + 1] = l2.y;
                }
                int o = 16;
#pragma unroll
                for (int half = NH / 2; half >= 1; half >>= 1, o >>= 1) {
                    const bool upper = lane & o;
#pragma unroll
                    for (int i = 0; i < half; ++i) {
                        const float keep = upper ? v[i + half] : v[i], give = upper ? v[i] : v[i + half];
                        v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
                    }
                }
                for (; o >= 1; o >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
                if (lane % (32 / NH) == 0) sums[((ob * 2 + g) * 4 + wg) * 32 + lane / (32 / NH)] = v[0];
                __syncwarp();
                if (ok && lane == 0) mbar_arrive(&l_ready[ob]);
            }
            if (begins) ++item;
            advance(c, P, prefix, flags);
        }
        if (!ok) *abort_flag = 1;
    }
    __syncwarp();
    tcgen05_fence_before();
    __syncthreads();
    if (warp == 10) tmem_dealloc(*tmem_ptr, 512);
}

template <typename T16, int D, int NR>
cudaError_t launch_n(const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv, const PagedParams &P, cudaStream_t st)
{
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    if (device < 0 || device >= 64) return cudaErrorInvalidDevice;
    static std::atomic<unsigned long long> attr_done{0};  // one bit per device
    if (!((attr_done.load(std::memory_order_relaxed) >> device) & 1ull)) {
        e = cudaFuncSetAttribute(paged_mid_kernel<T16, D, NR>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 static_cast<int>(MidCfg<D, NR>::smem(hawk_host::kPagedMaxStreams)));
        if (e != cudaSuccess) return e;
        attr_done.fetch_or(1ull << device, std::memory_order_relaxed);
    }
    return hawk_host::launch_dependent(paged_mid_kernel<T16, D, NR>, dim3(P.row_blocks), dim3(kThreads),
                                       MidCfg<D, NR>::smem(P.S), st, mq, mk, mv, P);
}

template <typename T16, int D>
cudaError_t launch(int nr, const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv, const PagedParams &P, cudaStream_t st)
{
    if (nr == 16) return launch_n<T16, D, 16>(mq, mk, mv, P, st);
    if (nr == 32) return launch_n<T16, D, 32>(mq, mk, mv, P, st);
    return launch_n<T16, D, 64>(mq, mk, mv, P, st);
}

}  // namespace

cudaError_t hawk_host::launch_paged_mid(const hawk_paged_attn_args &a, const PagedParams &base, int nr, cudaStream_t st)
{
    PagedParams P = base;
    const int tile_tok = nr / P.group;  // positions of an item
    P.box_rows = paged_gcd(a.page_size, kKeys);
    CUtensorMap mq, mk, mv;
    const uint64_t row = 2ull * a.q_row_stride, head = 2ull * a.q_head_stride;
    if (!encode_16bit_4d_sw128(&mq, a.q, a.dtype == HAWK_BF16, {static_cast<uint64_t>(a.D), static_cast<uint64_t>(a.H),
                                                                static_cast<uint64_t>(a.T), 1},
                               {head, row, row}, base.group, tile_tok, 1) ||
        !encode_pages(&mk, a, false, P.box_rows, &P.k_rows_inner) || !encode_pages(&mv, a, true, P.box_rows, &P.v_rows_inner))
        return cudaErrorInvalidValue;
    P.mid_tok = tile_tok;
    if (a.dtype == HAWK_BF16)
        return a.D == 64 ? launch<__nv_bfloat16, 64>(nr, mq, mk, mv, P, st) : launch<__nv_bfloat16, 128>(nr, mq, mk, mv, P, st);
    return a.D == 64 ? launch<__half, 64>(nr, mq, mk, mv, P, st) : launch<__half, 128>(nr, mq, mk, mv, P, st);
}
