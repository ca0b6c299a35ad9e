// hawk_paged_attn: attention of a ragged batch of new rows over a paged key/value cache.  This file holds the entry point
// and the kernel for FEW rows per kv head (decode steps, drafted blocks, small candidate trees).  Streams of more than 64
// rows per kv head go to the tile kernel in hawk_paged_tile.cu, each by its own row count; the others of a call go to the
// kernel here or, in calls without such streams, to the one in hawk_paged_mid.cu, by the call's sizes (plan_rows).
//
// With few rows the call is bound by reading every key and value once (r flops per byte for r rows per kv head), so the
// kernel is organised like the dense verify attention: a flat list of key tiles cut into equal shares, one per warp of a
// persistent grid, every warp its own TMA pipeline, transposed products S^T = K Q^T and O^T = V^T P^T on warp-level MMAs
// with the keys on the 16-row operand, running maximum and sum in registers.  What paging and ragged batches change:
//   - The list is built on the device from row_begin and kv_len (a prefix sum over the streams in shared memory, one
//     pass of the block), so every share holds the same number of tiles that exist, however uneven the streams are.
//   - A tile is loaded as boxes that each stay inside one page.  The page ids sit in registers, 32 of them across the
//     warp's lanes and the next 32 on their way, so no load waits for the block table in the middle of a stream.
//   - Boxes that lie wholly behind the stream's last key are not loaded (their table entries may be anything).
//   - A share that holds part of an item leaves an fp32 partial and a record of what it is part of; the merge kernel
//     works from the records alone and needs neither the lengths nor the prefix sum again.
#include <atomic>
#include <type_traits>

#include "hawk_paged.cuh"

namespace {

using namespace hawk;

// Launch shapes (WARPS pipelines per block, STAGES tiles deep, 8 KB a stage).
//   shares: one block per SM, every warp an equal share of the list; items may be cut, the merge kernel follows.  Items
//           of one 8-row column tile leave registers for 12 warps of 2 stages, wider ones for 8 of 3.
//   group : one item per block, split evenly over its warps, which merge in shared memory.  8 warps of 3 stages and one
//           block per SM, or (one column tile) 4 of 2 and three blocks per SM.
// group needs no second kernel and no partial results in memory, so it is taken whenever the items fit the GPU at once
// and are not so few and long that most SMs would idle (plan_rows has the rules and what both sides measured).
__host__ __device__ constexpr int shares_warps(int nqt) { return nqt == 1 ? 12 : 8; }
__host__ __device__ constexpr int shares_stages(int nqt) { return nqt == 1 ? 2 : 3; }
constexpr int kMinShareTiles = 2;    // shorter shares would only add partial results to merge
constexpr float kLazy = 8.f;         // log2 units by which a score may exceed the softmax shift
constexpr int kStageBytes = 8192;
constexpr int kMaxStreams = hawk_host::kPagedMaxStreams;
constexpr int kMaxKv = 1 << 30;      // key positions, rounded up to tiles, stay 32-bit numbers (and no cache of one stream is longer)
constexpr int kRecordInts = 8;       // start tile, tiles of the item, first row, rows, kv head, row chunk, total tiles, workers

template <int D>
struct Tile {
    static constexpr int kHalves = D / 64;
    static constexpr int kKeys = kStageBytes / (4 * D);  // keys of a stage: 32 (D = 64), 16 (D = 128)
    static constexpr int kSubBytes = kKeys * 128;        // [keys][64 columns]
};

// Rows per item: what one warp's registers hold beside the accumulators.
__host__ __device__ constexpr int rows_max(int D) { return D == 64 ? 32 : 24; }

constexpr size_t rows_smem(int warps, int stages, int S)
{
    return 1024 + static_cast<size_t>(warps) * stages * (kStageBytes + sizeof(uint64_t)) + 64 + 64 +
           (static_cast<size_t>(S) + 1) * sizeof(int);
}

// Position in the list of tiles: stream, kv head, row chunk, tile of that item.
struct Cursor {
    int s, hk, chunk, tile;
    int r0, n, kv, nt, chunks;  // of the stream
    int left;                   // tiles left in the share, this one included
};

template <int D>
__device__ __forceinline__ int tiles_of(int kv)
{
    return max(1, (kv + Tile<D>::kKeys - 1) / Tile<D>::kKeys);  // (a stream without keys still has rows to write)
}

template <int D, int RPI>
__device__ __forceinline__ int items_of(const PagedParams &P, const PagedStream &st)
{
    return st.n == 0 || !paged_is_few(P, st) ? 0 : P.H_kv * ((st.n * P.group + RPI - 1) / RPI);
}

template <int D, int RPI>
__device__ __forceinline__ void enter_stream(Cursor &c, const PagedParams &P, int &flags)
{
    const PagedStream st = paged_stream(P, c.s, flags);
    c.r0 = st.r0;
    c.n = st.n;
    c.kv = st.kv;
    c.nt = tiles_of<D>(st.kv);
    c.chunks = (st.n * P.group + RPI - 1) / RPI;
}

__device__ __forceinline__ long long share_begin(long long g, long long T, int W) { return g * T / W; }

template <typename T16, int D, int NQT, int kWarps, int kStages, bool kGroup>
__global__ void __launch_bounds__(kWarps * 32, kWarps == 4 ? 3 : 1)
    paged_rows_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                      const PagedParams P)
{
    using C = Tile<D>;
    using E = Elem<T16>;
    constexpr int TK = C::kKeys, KB = TK / 16, DB = D / 16, RPI = NQT * 8;
    constexpr bool kShares = !kGroup;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + kWarps * kStages * kStageBytes);
    volatile int *has_part = reinterpret_cast<volatile int *>(bars + kWarps * kStages);  // [16], group shape
    int *wsum = const_cast<int *>(has_part) + 16;                                        // [16]
    int *prefix = wsum + 16;                                                             // [S + 1]

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < kWarps * kStages; ++i) mbar_init(&bars[i], 1);
        for (int i = 0; i < 16; ++i) has_part[i] = 0;
        fence_mbar_init();
        fence_proxy_async();
        prefetch_tensormap(&map_k);
        prefetch_tensormap(&map_v);
    }
    grid_dependency_wait();
    int flags = 0;
    if (P.groups && static_cast<int>(blockIdx.x) == P.row_blocks) {  // the block that makes the tile kernel's list
        __syncthreads();
        paged_plan(P, reinterpret_cast<int *>(smem), flags);
        if (flags && P.dev_status) atomicOr(P.dev_status, flags);
        return;
    }

    // ---- prefix sum over the streams: of their tiles (shares) or of their items (group)
    int running = 0;
    for (int base = 0; base < P.S; base += kWarps * 32) {
        const int s = base + tid;
        int v = 0;
        if (s < P.S) {
            const PagedStream st = paged_stream(P, s, flags);
            v = items_of<D, RPI>(P, st);
            if (kShares) v *= tiles_of<D>(st.kv);
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
        for (int w2 = 0; w2 < kWarps; ++w2) {
            if (w2 < warp) before += wsum[w2];
            all += wsum[w2];
        }
        if (s < P.S) prefix[s + 1] = before + inc;
        running = all;
        __syncthreads();
    }
    if (tid == 0) prefix[0] = 0;
    __syncthreads();
    if (flags && P.dev_status && blockIdx.x == 0) atomicOr(P.dev_status, flags);
    flags = 0;

    // ---- this warp's share
    const int total = running;
    int W = 0, w = 0, f = 0, len = 0;
    if (kShares) {
        W = max(1, min(P.row_blocks * kWarps, total / kMinShareTiles));
        w = static_cast<int>(blockIdx.x) * kWarps + warp;
        if (w < W) {
            f = static_cast<int>(share_begin(w, total, W));
            len = static_cast<int>(share_begin(w + 1, total, W)) - f;
        }
    } else {
        w = f = static_cast<int>(blockIdx.x);
        len = w < total ? 1 : 0;
    }
    Cursor cc;
    cc.s = cc.hk = cc.chunk = cc.tile = cc.left = cc.r0 = cc.n = cc.kv = 0;
    cc.nt = cc.chunks = 1;
    if (len > 0) {
        int lo = 0, hi = P.S;  // prefix[lo] <= f < prefix[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (prefix[mid] <= f) lo = mid;
            else hi = mid;
        }
        cc.s = lo;
        enter_stream<D, RPI>(cc, P, flags);
        int item = f - prefix[lo];
        if (kShares) {
            const int loc = item;
            item = loc / cc.nt;
            cc.tile = loc - item * cc.nt;
            cc.left = len;
        } else {
            cc.tile = static_cast<int>(static_cast<long long>(cc.nt) * warp / kWarps);
            cc.left = static_cast<int>(static_cast<long long>(cc.nt) * (warp + 1) / kWarps) - cc.tile;
        }
        cc.hk = item / cc.chunks;
        cc.chunk = item - cc.hk * cc.chunks;
    }
    if (kShares && lane == 0 && HAWK_IN_BOUNDS(P.dev_status, (w + 1) * kRecordInts - 1, P.record_ints)) {
        int32_t *rec = P.records + static_cast<size_t>(w) * kRecordInts;
        *reinterpret_cast<int4 *>(rec) = make_int4(cc.tile, cc.nt, cc.r0, cc.n);
        *reinterpret_cast<int4 *>(rec + 4) = make_int4(cc.hk, cc.chunk, total, W);
    }
    if (!kGroup && cc.left == 0) return;
    const Cursor head = cc;  // group shape: the block's item

    uint8_t *ring = smem + warp * kStages * kStageBytes;
    uint64_t *full_bar = bars + warp * kStages;
    const uint32_t ring_u32 = smem_u32(ring);
    uint64_t policy = 0;
    if (lane == 0) policy = l2_policy_evict_first();

    auto advance = [&](Cursor &c) {
        --c.left;
        ++c.tile;
        if (c.tile == c.nt && c.left > 0) {
            c.tile = 0;
            if (++c.chunk == c.chunks) {
                c.chunk = 0;
                if (++c.hk == P.H_kv) {
                    c.hk = 0;
                    // (tiles are left, so a stream with some follows; the bound holds even if the lengths change under the call)
                    do c.s = min(c.s + 1, P.S - 1);
                    while (c.s < P.S - 1 && prefix[c.s + 1] == prefix[c.s]);
                    enter_stream<D, RPI>(c, P, flags);
                }
            }
        }
    };

    // ---- issue side: page ids of the stream, 32 at a time across the lanes
    int pg_s = -1, pg_base = 0, pg_cur = 0, pg_nxt = 0, first_s = -1, pg_first = 0;
    auto page_of = [&](const Cursor &c, int pg) {
        if (pg_s != c.s || pg < pg_base || pg >= pg_base + 32) {
            const int need = static_cast<int>(P.div_page.div(static_cast<uint32_t>(c.kv + P.page_size - 1)));
            const int32_t *tb = P.block_table + static_cast<size_t>(c.s) * P.table_width;
            auto fetch = [&](int base) { return base + lane < need ? tb[base + lane] : 0; };
            if (pg_s == c.s && pg >= pg_base + 32 && pg < pg_base + 64) {
                pg_cur = pg_nxt;
                pg_base += 32;
            } else {
                pg_base = pg & ~31;
                if (pg_base == 0 && first_s == c.s) {
                    pg_cur = pg_first;
                } else {
                    pg_cur = fetch(pg_base);
                    if (pg_base == 0) {
                        pg_first = pg_cur;
                        first_s = c.s;
                    }
                }
            }
            pg_s = c.s;
            pg_nxt = fetch(pg_base + 32);
        }
        return __shfl_sync(0xffffffffu, pg_cur, pg - pg_base);
    };
    int box_pg = 0, box_row = 0;  // page index and row in it of the next box
    if (cc.left > 0) {
        uint32_t row;
        box_pg = static_cast<int>(P.div_page.divmod(static_cast<uint32_t>(cc.tile) * TK, row));
        box_row = static_cast<int>(row);
    }
    bool first_issue = true;
    auto issue = [&](const Cursor &c, int st) {
        if (c.tile == 0) box_pg = box_row = 0;
        const int bytes_box = P.box_rows * 128;
        const int live = max(0, min(TK, c.kv - c.tile * TK) + P.box_rows - 1) & -P.box_rows;  // rows of the boxes to load
        uint8_t *kd = ring + st * kStageBytes;
        uint8_t *vd = kd + C::kHalves * C::kSubBytes;
        if (lane == 0) {
            // (test builds only: the first tile of the first share is armed for more bytes than arrive)
            const bool stall = kTestStallBytes != 0 && blockIdx.x == 0 && warp == 0 && first_issue;
            mbar_arrive_expect_tx(&full_bar[st], live * 128 * 2 * C::kHalves + (stall ? kTestStallBytes : 0u));
        }
        first_issue = false;
        for (int off = 0; off < live * 128; off += bytes_box) {
            const int id = page_of(c, box_pg);
            if (id < 0 || id >= P.n_pages) flags |= HAWK_DEV_BAD_PAGE;  // (outside the tensor map: zeros)
            if (lane == 0) {
#pragma unroll
                for (int hf = 0; hf < C::kHalves; ++hf) {
                    paged_load(kd + hf * C::kSubBytes + off, &map_k, P.k_rows_inner, hf, box_row, c.hk, id, &full_bar[st], policy);
                    paged_load(vd + hf * C::kSubBytes + off, &map_v, P.v_rows_inner, hf, box_row, c.hk, id, &full_bar[st], policy);
                }
            }
            box_row += P.box_rows;
            if (box_row >= P.page_size) {
                box_row = 0;
                ++box_pg;
            }
        }
    };
    Cursor ci = cc;
    int in_flight = 0;
#pragma unroll
    for (int i = 0; i < kStages; ++i) {
        if (ci.left > 0) {
            issue(ci, i);
            advance(ci);
            ++in_flight;
        }
    }

    // ---- consume side; fragment coordinates: g = lane / 4, tq = lane % 4
    //   S^T block (16 keys x 8 rows): keys g and g + 8, rows 2tq and 2tq + 1 of the column tile
    //   O^T block (16 dims x 8 rows): dims g and g + 8, rows 2tq and 2tq + 1
    const int g = lane >> 2, tq = lane & 3;
    const int lm_mi = lane >> 3, lm_r = lane & 7;
    uint32_t k_off[DB], v_off[DB];  // ldmatrix rows of this lane (128-byte swizzle: chunk index XOR row modulo 8)
#pragma unroll
    for (int kk = 0; kk < DB; ++kk) {
        const int kc = 2 * kk + (lm_mi >> 1), vc = 2 * kk + (lm_mi & 1);
        k_off[kk] = (kc >> 3) * C::kSubBytes + ((lm_mi & 1) * 8 + lm_r) * 128 + (((kc & 7) ^ lm_r) << 4);
        v_off[kk] = (vc >> 3) * C::kSubBytes + ((lm_mi >> 1) * 8 + lm_r) * 128 + (((vc & 7) ^ lm_r) << 4);
    }

    uint32_t qb[NQT][DB][2];
    float ot[NQT][DB][4];
    float mrun[NQT][2], lrun[NQT][2];
    bool far = false;                     // some row's shift is (see kFarShift)
    int hk = 0, row0 = 0, nrows = 0;      // of the segment's item: kv head, first row of the chunk, rows
    int seg_r0 = 0, seg_tile = 0;
    bool seg_first = true, open = false;  // first segment of the share; a segment is being worked on

    auto q_row = [&](int r) {  // element offset of row r of the chunk in q
        uint32_t hd;
        const uint32_t pos = P.div_group.divmod(static_cast<uint32_t>(row0 + r), hd);
        return (seg_r0 + static_cast<long long>(pos)) * P.q_row_stride + (hk * P.group + static_cast<int>(hd)) * P.q_head_stride;
    };
    auto out_row = [&](int r, int first_row, int kv_head, int chunk_row0) {
        uint32_t hd;
        const uint32_t pos = P.div_group.divmod(static_cast<uint32_t>(chunk_row0 + r), hd);
        return ((first_row + static_cast<long long>(pos)) * P.H + kv_head * P.group + static_cast<int>(hd)) * D;
    };
    [[maybe_unused]] const long long out_elems = static_cast<long long>(P.T) * P.H * D;

    // Writes the finished segment: the result if it held the whole item, else an fp32 partial.
    auto flush = [&](bool complete) {
#pragma unroll
        for (int nq = 0; nq < NQT; ++nq)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float l = lrun[nq][c];
                l += __shfl_xor_sync(0xffffffffu, l, 4);
                l += __shfl_xor_sync(0xffffffffu, l, 8);
                l += __shfl_xor_sync(0xffffffffu, l, 16);
                lrun[nq][c] = l;
            }
        if (complete) {
#pragma unroll
            for (int nq = 0; nq < NQT; ++nq) {
                // a row that saw no key has no mass: zeros
                const float inv0 = lrun[nq][0] == 0.f ? 0.f : 1.f / lrun[nq][0];
                const float inv1 = lrun[nq][1] == 0.f ? 0.f : 1.f / lrun[nq][1];
                const int r = nq * 8 + g;
                const bool valid = r < nrows;
                const long long o = valid ? out_row(r, seg_r0, hk, row0) : 0;
                T16 *dst = static_cast<T16 *>(P.out) + o + 2 * tq;
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    const uint32_t lo = movmatrix_trans(E::pack(ot[nq][db][0] * inv0, ot[nq][db][1] * inv1));
                    const uint32_t hi = movmatrix_trans(E::pack(ot[nq][db][2] * inv0, ot[nq][db][3] * inv1));
                    if (valid && HAWK_IN_BOUNDS(P.dev_status, o + 2 * tq + db * 16 + 9, out_elems)) {
                        *reinterpret_cast<uint32_t *>(dst + db * 16) = lo;
                        *reinterpret_cast<uint32_t *>(dst + db * 16 + 8) = hi;
                    }
                }
            }
            return;
        }
        // group shape: the ring is free by now (every copy issued has been consumed) and takes the partial
        float *ps = kGroup ? reinterpret_cast<float *>(ring)
                           : P.part + (static_cast<size_t>(w) * 2 + (seg_first ? 0 : 1)) * RPI * (D + 2);
        static_assert(!kGroup || RPI * (D + 2) * 4 <= kStages * kStageBytes, "a partial fits the ring");
        if (!kGroup && !HAWK_IN_BOUNDS(P.dev_status, ps - P.part + RPI * (D + 2) - 1, P.part_floats)) return;
        if (kGroup && lane == 0) has_part[warp] = 1;
#pragma unroll
        for (int nq = 0; nq < NQT; ++nq)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int r = nq * 8 + 2 * tq + c;
                if (r < nrows) {
                    float *pr = ps + r * D;
#pragma unroll
                    for (int db = 0; db < DB; ++db) {
                        pr[db * 16 + g] = ot[nq][db][c];
                        pr[db * 16 + 8 + g] = ot[nq][db][2 + c];
                    }
                    if (g == 0)
                        *reinterpret_cast<float2 *>(ps + RPI * D + 2 * r) = make_float2(mrun[nq][c], lrun[nq][c]);
                }
            }
    };

    int st = 0;
    uint32_t ph = 0;
    bool ok = true;
    while (cc.left > 0) {
        if (!open) {
            // ---- a new segment: this item's queries, empty state
            open = true;
            far = false;
            hk = cc.hk;
            row0 = cc.chunk * RPI;
            nrows = min(RPI, cc.n * P.group - row0);
            seg_r0 = cc.r0;
            seg_tile = cc.tile;
#pragma unroll
            for (int nq = 0; nq < NQT; ++nq) {
                const int r = nq * 8 + g;
                const bool valid = r < nrows;
                const T16 *qr = static_cast<const T16 *>(P.q) + (valid ? q_row(r) : 0) + 2 * tq;
#pragma unroll
                for (int kk = 0; kk < DB; ++kk) {
                    qb[nq][kk][0] = valid ? *reinterpret_cast<const uint32_t *>(qr + kk * 16) : 0u;
                    qb[nq][kk][1] = valid ? *reinterpret_cast<const uint32_t *>(qr + kk * 16 + 8) : 0u;
                }
#pragma unroll
                for (int db = 0; db < DB; ++db) ot[nq][db][0] = ot[nq][db][1] = ot[nq][db][2] = ot[nq][db][3] = 0.f;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    mrun[nq][c] = -CUDART_INF_F;
                    lrun[nq][c] = 0.f;
                }
            }
        }
        const int kv = cc.kv, pfx = kv - cc.n;  // (pfx < 0: the first rows see nothing)
        const int key0 = cc.tile * TK;
        ok = mbar_wait(&full_bar[st], ph, nullptr);
        if (!ok) break;
        const uint32_t kbase = ring_u32 + st * kStageBytes;
        const uint32_t vbase = kbase + C::kHalves * C::kSubBytes;

        // The tile's products and softmax for the first NQ column tiles: an item may have fewer rows than its place in the call holds
        // (single tokens beside chunks of a prompt), and then pays for one.
        auto columns = [&](auto active) {
            constexpr int NQ = decltype(active)::value;
            // ---- S^T = K Q^T
            float sc[NQ][KB][4];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
                for (int nq = 0; nq < NQ; ++nq) sc[nq][kb][0] = sc[nq][kb][1] = sc[nq][kb][2] = sc[nq][kb][3] = 0.f;
#pragma unroll
                for (int kk = 0; kk < DB; ++kk) {
                    uint32_t ka[4];
                    ldmatrix_x4(ka, kbase + kb * 2048 + k_off[kk]);
#pragma unroll
                    for (int nq = 0; nq < NQ; ++nq) E::mma(sc[nq][kb], ka, qb[nq][kk][0], qb[nq][kk][1]);
                }
            }
            // ---- masks, at the tiles that reach past the prefix (keys behind the stream's last one among them)
            if (key0 + TK > pfx) {
#pragma unroll
                for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const uint32_t r = static_cast<uint32_t>(min(row0 + nq * 8 + 2 * tq + c, cc.n * P.group - 1));
                        const int pos = static_cast<int>(P.div_group.div(r));
                        const uint64_t m = P.anc_mask ? P.anc_mask[pos] : 0ull;
                        auto visible = [&](int key) {
                            const int rel = key - pfx;
                            if (!P.anc_mask) return rel <= pos;
                            return rel < 0 || (rel < cc.n && rel < 64 && ((m >> rel) & 1ull));
                        };
#pragma unroll
                        for (int kb = 0; kb < KB; ++kb) {
                            const int key = key0 + kb * 16 + g;
                            if (!visible(key)) sc[nq][kb][c] = -CUDART_INF_F;
                            if (!visible(key + 8)) sc[nq][kb][2 + c] = -CUDART_INF_F;
                        }
                    }
            }
            // ---- running softmax per row, base 2.  The shift m may be any number as long as o, the sum and p share it; it
            // is renewed only when a score exceeds it by more than kLazy, so that almost every tile goes without the
            // reduction across lanes and without touching o (p stays below 2^kLazy: far inside fp16, bf16 and fp32)
            bool grows = false;
            float mx[NQ][2];
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float m = -CUDART_INF_F;
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) m = fmaxf(m, fmaxf(sc[nq][kb][c], sc[nq][kb][2 + c]));
                    mx[nq][c] = m;
                    grows |= (m - mrun[nq][c]) * P.scale_log2 > kLazy;  // (no score yet and none now: NaN, no)
                }
            }
            if (__any_sync(0xffffffffu, grows)) {
                bool is = false;
#pragma unroll
                for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float m = mx[nq][c];
#pragma unroll
                        for (int o = 4; o < 32; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
                        m = fmaxf(m, mrun[nq][c]);
                        const float a = fast_exp2((mrun[nq][c] - (m == -CUDART_INF_F ? 0.f : m)) * P.scale_log2);
                        mrun[nq][c] = m;
                        is |= is_far(m, P.scale_log2);
                        lrun[nq][c] *= a;
#pragma unroll
                        for (int db = 0; db < DB; ++db) {
                            ot[nq][db][c] *= a;
                            ot[nq][db][2 + c] *= a;
                        }
                    }
                far = __any_sync(0xffffffffu, is);
            }
            uint32_t pb[NQ][KB][2];
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq) {
                const float mu0 = mrun[nq][0] == -CUDART_INF_F ? 0.f : mrun[nq][0];
                const float mu1 = mrun[nq][1] == -CUDART_INF_F ? 0.f : mrun[nq][1];
                float sh0 = -mu0 * P.scale_log2, sh1 = -mu1 * P.scale_log2;
                if (far) {
                    sh0 = sh1 = 0.f;
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) {
                        sc[nq][kb][0] -= mu0;
                        sc[nq][kb][1] -= mu1;
                        sc[nq][kb][2] -= mu0;
                        sc[nq][kb][3] -= mu1;
                    }
                }
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
                    const float p0 = fast_exp2(fmaf(sc[nq][kb][0], P.scale_log2, sh0));
                    const float p1 = fast_exp2(fmaf(sc[nq][kb][1], P.scale_log2, sh1));
                    const float p2 = fast_exp2(fmaf(sc[nq][kb][2], P.scale_log2, sh0));
                    const float p3 = fast_exp2(fmaf(sc[nq][kb][3], P.scale_log2, sh1));
                    lrun[nq][0] += p0 + p2;
                    lrun[nq][1] += p1 + p3;
                    pb[nq][kb][0] = movmatrix_trans(E::pack(p0, p1));
                    pb[nq][kb][1] = movmatrix_trans(E::pack(p2, p3));
                }
            }
            // ---- O^T += V^T P^T; values behind the last key hold anything (or are an earlier tile's): zeroed, 0 * NaN is NaN
            const bool ragged = key0 + TK > kv;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                const int kleft = kv - (key0 + kb * 16);
                if (ragged && kleft <= 0) break;
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    uint32_t va[4];
                    ldmatrix_x4_trans(va, vbase + kb * 2048 + v_off[db]);
                    if (ragged && kleft < 16) {
                        const int ka = 2 * tq, kb2 = 2 * tq + 8;
                        const uint32_t ma = (ka < kleft ? 0x0000ffffu : 0u) | (ka + 1 < kleft ? 0xffff0000u : 0u);
                        const uint32_t mb = (kb2 < kleft ? 0x0000ffffu : 0u) | (kb2 + 1 < kleft ? 0xffff0000u : 0u);
                        va[0] &= ma;
                        va[1] &= ma;
                        va[2] &= mb;
                        va[3] &= mb;
                    }
#pragma unroll
                    for (int nq = 0; nq < NQ; ++nq) E::mma(ot[nq][db], va, pb[nq][kb][0], pb[nq][kb][1]);
                }
            }
        };
        if (NQT > 1 && nrows <= 8) columns(std::integral_constant<int, 1>{});
        else columns(std::integral_constant<int, NQT>{});
        __syncwarp();
        --in_flight;
        if (ci.left > 0) {
            fence_proxy_async();  // the warp's reads of the stage come before the copy that overwrites it
            issue(ci, st);
            advance(ci);
            ++in_flight;
        }
        const bool item_ends = cc.tile + 1 == cc.nt;
        if (item_ends || cc.left == 1) {
            flush(!kGroup && item_ends && seg_tile == 0);
            seg_first = false;
            open = false;
        }
        advance(cc);
        if (++st == kStages) {
            st = 0;
            ph ^= 1u;
        }
    }
    if (!ok) {
        flags |= HAWK_DEV_TIMEOUT;
        for (int i = 0; i < in_flight; ++i) {  // let the copies still in flight land (bounded) before the block retires
            mbar_wait(&full_bar[st], ph, nullptr);
            if (++st == kStages) {
                st = 0;
                ph ^= 1u;
            }
        }
    }
    if (flags && lane == 0 && P.dev_status) atomicOr(P.dev_status, flags);

    if constexpr (kGroup) {
        // ---- the warps' partial results of the block's item, folded in share order from shared memory
        __syncthreads();
        if (head.n == 0) return;
        constexpr int PER = D / 32;
        const int kvh = head.hk, c_row0 = head.chunk * RPI;
        const int rows = min(RPI, head.n * P.group - c_row0);
        for (int r = warp; r < rows; r += kWarps) {
            float acc[PER];
#pragma unroll
            for (int c = 0; c < PER; ++c) acc[c] = 0.f;
            float mm = -CUDART_INF_F, ll = 0.f;
            for (int gg = 0; gg < kWarps; ++gg) {
                if (!has_part[gg]) continue;  // (fewer tiles than warps)
                const float *ps = reinterpret_cast<const float *>(smem + gg * kStages * kStageBytes);
                const float2 m_l = *reinterpret_cast<const float2 *>(ps + RPI * D + 2 * r);
                const float mn = fmaxf(mm, m_l.x);
                const float mu = mn == -CUDART_INF_F ? 0.f : mn;
                const float f_old = fast_exp2((mm - mu) * P.scale_log2), f_new = fast_exp2((m_l.x - mu) * P.scale_log2);
                mm = mn;
                ll = ll * f_old + m_l.y * f_new;
#pragma unroll
                for (int c = 0; c < PER; ++c) acc[c] = acc[c] * f_old + ps[r * D + lane * PER + c] * f_new;
            }
            const float inv = ll == 0.f ? 0.f : 1.f / ll;
            const long long o = out_row(r, head.r0, kvh, c_row0) + lane * PER;
            T16 *dst = static_cast<T16 *>(P.out) + o;
            if (!HAWK_IN_BOUNDS(P.dev_status, o, out_elems) || !HAWK_IN_BOUNDS(P.dev_status, o + PER - 1, out_elems)) continue;
#pragma unroll
            for (int c = 0; c < PER; c += 2)
                *reinterpret_cast<uint32_t *>(dst + c) = E::pack(acc[c] * inv, acc[c + 1] * inv);
        }
    }
}

// Merges the items that were cut.  Worker g stands for the item its share starts inside of, if its predecessor's share
// holds that item's first tile; contribution 0 is the predecessor's last segment, contribution c the first segment of
// worker g + c - 1, until the item's tiles are used up.  Everything comes from the records.
// A block looks at 8 neighbouring workers and deals its 8 warps out to those among them that stand for an item: one warp
// each when all do (items shorter than a share: two contributions), all 8 on one item when it is the only one (an item
// spread over dozens of shares), joined in shared memory.  A warp takes 8 rows (4 at D = 128: registers), its lanes across the head dimension, and has
// two contributions' loads under way at a time.  (One warp per worker and row instead, 1775 to 3549 blocks most of which
// only looked at a record, took 5 us at 8 rows an item and 8 us at 24.)
constexpr int kMergeWorkers = 8;
__host__ __device__ constexpr int merge_rows(int D) { return D == 64 ? 8 : 4; }

template <typename T16, int D, int RPI>
__global__ void __launch_bounds__(256, 3) paged_merge_kernel(const PagedParams P, int workers_max)
{
    using E = Elem<T16>;
    constexpr int PER = D / 32, RW = merge_rows(D);
    __shared__ float joined[8][RW * (D + 2)];
    allow_dependent_launch();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g0 = blockIdx.x * kMergeWorkers + 1, r0g = blockIdx.y * RW;  // first worker, first row of the item
    grid_dependency_wait();
    // lane i < 8 looks at worker g0 + i
    const int mine = g0 + (lane & 7);
    int4 a = make_int4(0, 1, 0, 0), b = make_int4(0, 0, 0, 1);
    if (mine < workers_max) {
        a = *reinterpret_cast<const int4 *>(P.records + static_cast<size_t>(mine) * kRecordInts);
        b = *reinterpret_cast<const int4 *>(P.records + static_cast<size_t>(mine) * kRecordInts + 4);
    }
    const int total = b.z, W = b.w;
    const int sb = static_cast<int>(share_begin(mine, total, W));
    const int before = sb - static_cast<int>(share_begin(mine - 1, total, W));
    const bool stands = lane < 8 && mine < W && a.x > 0 && a.x <= before;
    const unsigned act = __ballot_sync(0xffffffffu, stands);
    const int n_act = __popc(act);
    if (n_act == 0) return;
    const int wpi = n_act == 1 ? 8 : n_act == 2 ? 4 : n_act <= 4 ? 2 : 1;  // warps per item
    const int idx = warp / wpi, sub = warp - idx * wpi;
    const bool work = idx < n_act;
    const int src = work ? __fns(act, 0, idx + 1) : 0;
    const int tile = __shfl_sync(0xffffffffu, a.x, src), nt = __shfl_sync(0xffffffffu, a.y, src);
    const int first_row = __shfl_sync(0xffffffffu, a.z, src), n = __shfl_sync(0xffffffffu, a.w, src);
    const int hk = __shfl_sync(0xffffffffu, b.x, src), row0 = __shfl_sync(0xffffffffu, b.y, src) * RPI + r0g;
    const int sb_g = __shfl_sync(0xffffffffu, sb, src), before_g = __shfl_sync(0xffffffffu, before, src);
    const int all = __shfl_sync(0xffffffffu, total, src), workers = __shfl_sync(0xffffffffu, W, src);
    const int g = g0 + src, end = sb_g - tile + nt;  // one past the item's last tile in the list
    const int rows = work ? min(RW, min(RPI, n * P.group - (row0 - r0g)) - r0g) : 0;

    float acc[RW][PER], mm[RW], ll[RW];
#pragma unroll
    for (int r = 0; r < RW; ++r) {
        mm[r] = -CUDART_INF_F;
        ll[r] = 0.f;
#pragma unroll
        for (int c = 0; c < PER; ++c) acc[r][c] = 0.f;
    }
    auto exists = [&](int c) {
        if (c == 0) return true;
        const int gg = g + c - 1;
        return gg < workers && static_cast<int>(share_begin(gg, all, workers)) < end;
    };
    auto slot_of = [&](int c) {
        const int slot = c == 0 ? (g - 1) * 2 + (tile == before_g ? 0 : 1) : (g + c - 1) * 2;
        return P.part + static_cast<size_t>(slot) * RPI * (D + 2);
    };
    struct Piece {
        float2 ml;  // lane r: of row r
        float v[RW][PER];
    };
    auto fetch = [&](Piece &p, const float *ps) {
        p.ml = make_float2(-CUDART_INF_F, 0.f);
        if (lane < rows) p.ml = *reinterpret_cast<const float2 *>(ps + RPI * D + 2 * (r0g + lane));
#pragma unroll
        for (int r = 0; r < RW; ++r) {
            if (r < rows) {
                const float *pr = ps + (r0g + r) * D + lane * PER;
                if constexpr (PER == 2) {
                    const float2 x = *reinterpret_cast<const float2 *>(pr);
                    p.v[r][0] = x.x;
                    p.v[r][1] = x.y;
                } else {
                    const float4 x = *reinterpret_cast<const float4 *>(pr);
                    p.v[r][0] = x.x;
                    p.v[r][1] = x.y;
                    p.v[r][PER - 2] = x.z;
                    p.v[r][PER - 1] = x.w;
                }
            }
        }
    };
    auto fold_row = [&](int r, float m, float l, const float (&v)[PER]) {
        const float mn = fmaxf(mm[r], m);
        const float mu = mn == -CUDART_INF_F ? 0.f : mn;
        const float f_old = fast_exp2((mm[r] - mu) * P.scale_log2), f_new = fast_exp2((m - mu) * P.scale_log2);
        mm[r] = mn;
        ll[r] = ll[r] * f_old + l * f_new;
#pragma unroll
        for (int c = 0; c < PER; ++c) acc[r][c] = acc[r][c] * f_old + v[c] * f_new;
    };
    auto fold = [&](const Piece &p) {
#pragma unroll
        for (int r = 0; r < RW; ++r) {
            const float m = __shfl_sync(0xffffffffu, p.ml.x, r), l = __shfl_sync(0xffffffffu, p.ml.y, r);
            if (r < rows) fold_row(r, m, l, p.v[r]);
        }
    };
    if (rows > 0) {
        for (int c = sub; exists(c); c += 2 * wpi) {
            Piece p0, p1;
            const bool two = exists(c + wpi);
            fetch(p0, slot_of(c));
            if (two) fetch(p1, slot_of(c + wpi));
            fold(p0);
            if (two) fold(p1);
        }
    }
    if (wpi > 1) {  // (block-uniform)
#pragma unroll
        for (int r = 0; r < RW; ++r) {
#pragma unroll
            for (int c = 0; c < PER; ++c) joined[warp][r * D + lane * PER + c] = acc[r][c];
            if (lane == 0) {
                joined[warp][RW * D + 2 * r] = mm[r];
                joined[warp][RW * D + 2 * r + 1] = ll[r];
            }
        }
        __syncthreads();
        if (sub > 0) return;
        for (int o = 1; o < wpi; ++o) {
            const float *j = joined[warp + o];
#pragma unroll
            for (int r = 0; r < RW; ++r) {
                float v[PER];
#pragma unroll
                for (int c = 0; c < PER; ++c) v[c] = j[r * D + lane * PER + c];
                fold_row(r, j[RW * D + 2 * r], j[RW * D + 2 * r + 1], v);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < RW; ++r) {
        if (r >= rows) break;
        const float inv = ll[r] == 0.f ? 0.f : 1.f / ll[r];
        uint32_t hd;
        const uint32_t pos = P.div_group.divmod(static_cast<uint32_t>(row0 + r), hd);
        T16 *dst = static_cast<T16 *>(P.out) +
                   ((first_row + static_cast<long long>(pos)) * P.H + hk * P.group + static_cast<int>(hd)) * D + lane * PER;
        if (!HAWK_IN_BOUNDS(P.dev_status, dst - static_cast<T16 *>(P.out) + PER - 1, static_cast<long long>(P.T) * P.H * D)) continue;
#pragma unroll
        for (int c = 0; c < PER; c += 2)
            *reinterpret_cast<uint32_t *>(dst + c) = E::pack(acc[r][c] * inv, acc[r][c + 1] * inv);
    }
}

// ---------------------------------------------------------------------------------------------- host side
enum Shape { kShapeShares, kShapeGroup4, kShapeGroup8, kShapeMid };

struct RowsPlan {
    Shape shape;
    int rpi, grid;
};

// The kernel with the keys on tcgen05 in place of this file's?  It costs the same up to 64 rows (1.5 us a 128-key tile of a block
// at D = 128), this one more with each column tile of 8 rows, and its shares, a block each instead of a warp each, leave a tenth
// of the partial results.  But each of its items costs a few us once, and at D = 64, where a tile is half the bytes, it
// does not keep up with reading.  Measured, us, that kernel / this one, for (streams x kv heads) items of so many keys:
//   D = 128, 256 of 2400   8 rows 57 / 50    12: 58 / 63    24: 58 / 64    32: 59 / 114   60: 64 / 158
//            256 of 600    12 rows 23 / 26   24: 25 / 32    60: 35 / 53
//            1280 of 400   12 rows 56 / 54   24: 66 / 61    32: 67 / 104   40: 98 / 104   60: 107 / 146
//            56 of 20000    1 row  95 / 97    8: 95 / 101   32: 96 / 195
//            8 of 12000     1 row  19 / 28    8: 20 / 32    1 of 20000: 1 row 16 / 45
//            in place of group, 32 of 1500: 32 rows 17 / 20;  64 of 1200: 12 rows 17 / 17, 32: 19 / 18;  128 of 1500: 12 rows 26 / 21
//   D = 64,  256 of 2400   12 rows 40 / 37   32: 45 / 47    60: 58 / 72
//            320 of 500    12 rows 21 / 20   32: 24 / 28    40: 31 / 27   60: 33 / 34;   1280 of 400: 24 rows 64 / 37
//            8 of 12000     1 row  16 / 25    8: 18 / 34    40: 24 / 30
// From host-known bounds only, so that the workspace query and the launch agree.
bool mid_pays(bool shares, long long items, int rows, int D, int max_kv)
{
    const bool light = items * ((max_kv + kPagedTileKeys - 1) / kPagedTileKeys) <= 12 * hawk_host::kPagedSms;
    const bool few = items <= hawk_host::kPagedSms / 2;
    if (D == 128) {
        if (!shares) return few && rows > 8 && max_kv >= 1536;
        return few || (rows > 8 && (rows > 24 || light || max_kv >= 512));
    }
    return shares && ((rows > 32 && max_kv >= 1024) || (light && (few || (rows > 24 && rows <= 32))));
}

// `chunks_too`: some streams may be the tile kernel's, and the bound on the others' rows is then only that kernel's threshold.
RowsPlan plan_rows(int S, int rows, int H_kv, int D, int max_kv, bool chunks_too)
{
    RowsPlan p;
    const int cap = rows_max(D), tk = kStageBytes / (4 * D);
    const int chunks = (rows + cap - 1) / cap;
    p.rpi = ((rows + chunks - 1) / chunks + 7) / 8 * 8;
    const long long items = static_cast<long long>(S) * H_kv * ((rows + p.rpi - 1) / p.rpi);
    const int tiles = max_kv < 1 ? 1 : (max_kv + tk - 1) / tk;
    p.shape = kShapeShares;
    p.grid = hawk_host::kPagedSms;
    // at most one item per SM, a block each.  Shares spread the same tiles over all SMs but pay some 4 us for partial results
    // and their merge: with 80 items of 8 rows at D = 64 blocks take 13.9 / 22.8 / 40.2 us at 65 / 129 / 257 tiles an item, shares
    // 16.7 / 23.3 / 36.7; with 32 items the two cross at 65 tiles, with 144 they never do (97 against 103 us at 513)
    if (items <= hawk_host::kPagedSms && (items >= 120 || tiles <= 40 + items)) {
        p.shape = kShapeGroup8;
        p.grid = static_cast<int>(items);
    } else if (p.rpi <= 8 && items > hawk_host::kPagedSms && items <= 3 * hawk_host::kPagedSms) {
        // (320 items of 36 tiles: 17.9 us against 22.8 as shares; 400 of 257: 131 against 142)
        p.shape = kShapeGroup4;
        p.grid = static_cast<int>(items);
    }
    // Beside chunks of a prompt the other streams bring single tokens or drafted blocks as a rule, a column tile or two here and a fixed
    // 64 rows there: 60 tokens over 3000 keys of 32 heads of 64 beside a chunk of 300 rows 256 against 405 us, 200 over 700 keys of 8
    // heads of 128 122 against 146, 16 blocks of 5 rows 45 against 61; 30 trees of 22 rows 73 against 69.
    if (!chunks_too && mid_pays(p.shape == kShapeShares, static_cast<long long>(S) * H_kv, rows, D, max_kv)) {
        p.shape = kShapeMid;
        p.grid = hawk_host::kPagedSms;
        p.rpi = rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
    }
    return p;
}

size_t rows_workspace_bytes(const RowsPlan &p, int D)
{
    if (p.shape == kShapeMid)
        return static_cast<size_t>(hawk_host::kPagedSms) * (kRecordInts * sizeof(int32_t) + 2ull * 64 * (D + 2) * sizeof(float));
    if (p.shape != kShapeShares) return 0;
    return static_cast<size_t>(hawk_host::kPagedSms) * shares_warps(p.rpi / 8) * (kRecordInts * sizeof(int32_t) + 2ull * p.rpi * (D + 2) * sizeof(float));
}

template <typename T16, int D, int NQT, int WARPS, int STAGES, bool GROUP>
cudaError_t launch_shape(const CUtensorMap &mk, const CUtensorMap &mv, const PagedParams &P, int grid, cudaStream_t st)
{
    const size_t smem = rows_smem(WARPS, STAGES, P.S);
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    if (device < 0 || device >= 64) return cudaErrorInvalidDevice;
    static std::atomic<unsigned long long> attr_done{0};  // one bit per device
    if (!((attr_done.load(std::memory_order_relaxed) >> device) & 1ull)) {
        // (group: no more streams than items)
        const size_t most = rows_smem(WARPS, STAGES, GROUP ? hawk_host::kPagedSms * 3 : kMaxStreams);
        e = cudaFuncSetAttribute(paged_rows_kernel<T16, D, NQT, WARPS, STAGES, GROUP>,
                                 cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(most));
        if (e != cudaSuccess) return e;
        attr_done.fetch_or(1ull << device, std::memory_order_relaxed);
    }
    return hawk_host::launch_dependent(paged_rows_kernel<T16, D, NQT, WARPS, STAGES, GROUP>,
                                       dim3(grid + (P.groups ? 1 : 0)), dim3(WARPS * 32), smem,
                                       st, mk, mv, P);
}

template <typename T16, int D, int RPI>
cudaError_t launch_merge(const PagedParams &P, int workers, cudaStream_t st)
{
    return hawk_host::launch_dependent(paged_merge_kernel<T16, D, RPI>,
                                       dim3((workers - 1 + kMergeWorkers - 1) / kMergeWorkers, RPI / merge_rows(D)), dim3(256), 0, st,
                                       P, workers);
}

template <typename T16, int D, int NQT>
cudaError_t launch_rows(const CUtensorMap &mk, const CUtensorMap &mv, const PagedParams &P, const RowsPlan &p, cudaStream_t st)
{
    if (p.shape == kShapeGroup8) return launch_shape<T16, D, NQT, 8, 3, true>(mk, mv, P, p.grid, st);
    if constexpr (NQT == 1)
        if (p.shape == kShapeGroup4) return launch_shape<T16, D, NQT, 4, 2, true>(mk, mv, P, p.grid, st);
    constexpr int kW = shares_warps(NQT);
    cudaError_t e = launch_shape<T16, D, NQT, kW, shares_stages(NQT), false>(mk, mv, P, p.grid, st);
    if (e != cudaSuccess) return e;
    return launch_merge<T16, D, NQT * 8>(P, hawk_host::kPagedSms * kW, st);
}

template <typename T16, int D>
cudaError_t launch_rows_n(const CUtensorMap &mk, const CUtensorMap &mv, const PagedParams &P, const RowsPlan &p, cudaStream_t st)
{
    switch (p.rpi / 8) {
        case 1: return launch_rows<T16, D, 1>(mk, mv, P, p, st);
        case 2: return launch_rows<T16, D, 2>(mk, mv, P, p, st);
        case 3: return launch_rows<T16, D, 3>(mk, mv, P, p, st);
        case 4:
            if constexpr (D == 64) return launch_rows<T16, D, 4>(mk, mv, P, p, st);
    }
    return cudaErrorInvalidValue;
}

// Rows per kv head up to which a stream goes to the rows kernel.
constexpr int kFewRows = 64;

size_t align16(size_t n) { return (n + 15) / 16 * 16; }

}  // namespace

int hawk_host::paged_gcd(int a, int b)
{
    while (b) {
        const int t = a % b;
        a = b;
        b = t;
    }
    return a;
}

bool hawk_host::encode_pages(CUtensorMap *map, const hawk_paged_attn_args &a, bool values, int box_rows, int *rows_inner)
{
    const uint64_t row = 2ull * (values ? a.v_page_row_stride : a.k_page_row_stride);
    const uint64_t head = 2ull * (values ? a.v_page_head_stride : a.k_page_head_stride);
    const uint64_t page = 2ull * (values ? a.v_page_stride : a.k_page_stride);
    const uint64_t D = a.D, R = a.page_size, H = a.H_kv, N = a.n_pages;
    *rows_inner = row <= head ? 1 : 0;
    if (*rows_inner)
        return encode_16bit_4d_sw128(map, values ? a.v_pages : a.k_pages, a.dtype == HAWK_BF16, {D, R, H, N},
                                     {row, head, page}, box_rows, 1, 1);
    return encode_16bit_4d_sw128(map, values ? a.v_pages : a.k_pages, a.dtype == HAWK_BF16, {D, H, R, N}, {head, row, page}, 1,
                                 box_rows, 1);
}

extern "C" size_t hawk_paged_attn_workspace_bytes(int S, int T, int max_new, int H, int H_kv, int D, int max_kv)
{
    if (S <= 0 || T <= 0 || max_new <= 0 || H <= 0 || H_kv <= 0 || H % H_kv != 0 || (D != 64 && D != 128) || max_kv < 0 ||
        max_kv > kMaxKv || S > kMaxStreams || H / H_kv > 128)
        return 0;
    if (max_new > T) max_new = T;
    const long long rows = static_cast<long long>(max_new) * (H / H_kv);
    const long long few = rows < kFewRows ? rows : kFewRows;
    const size_t a = rows_workspace_bytes(plan_rows(S, static_cast<int>(few), H_kv, D, max_kv, rows > kFewRows), D);
    const size_t b = rows > kFewRows ? hawk_host::paged_tile_workspace_bytes(S, T, max_new, H, H_kv, kFewRows, D, max_kv) : 0;
    return align16(a) + b;
}

extern "C" hawk_status hawk_paged_attn(const hawk_paged_attn_args *args, int32_t *dev_status, hawk_stream_t stream)
{
    const hawk_host::NvtxRange nvtx_range("hawk_paged_attn");
    if (!args) return HAWK_ERR_NULL;
    const hawk_paged_attn_args &a = *args;
    if (a.S < 0 || a.T < 0 || a.max_new < 0 || a.max_kv < 0 || a.H < 0 || a.H_kv < 0 || a.D < 0 || a.n_pages < 0 ||
        a.page_size < 0 || a.table_width < 0)
        return HAWK_ERR_SHAPE;
    if (a.S == 0 || a.T == 0 || a.max_new == 0) return HAWK_OK;
    if (!a.q || !a.k_pages || !a.v_pages || !a.block_table || !a.row_begin || !a.kv_len || !a.out) return HAWK_ERR_NULL;
    if (a.dtype != HAWK_BF16 && a.dtype != HAWK_F16) return HAWK_ERR_PARAM;
    if ((a.D != 64 && a.D != 128) || a.H < 1 || a.H_kv < 1 || a.H % a.H_kv != 0 || a.H / a.H_kv > 128 || a.page_size < 8 ||
        a.page_size % 8 != 0 || a.S > kMaxStreams || a.max_kv > kMaxKv || (a.anc_mask && a.max_new > 64))
        return HAWK_ERR_UNSUPPORTED;
    if (a.n_pages < 1 || a.max_kv > static_cast<long long>(a.table_width) * a.page_size) return HAWK_ERR_SHAPE;
    if (!(a.sm_scale > 0.f) || isinf(a.sm_scale)) return HAWK_ERR_PARAM;
    if (!hawk_host::aligned16(a.q) || !hawk_host::aligned16(a.k_pages) || !hawk_host::aligned16(a.v_pages) ||
        !hawk_host::aligned16(a.out))
        return HAWK_ERR_ALIGN;
    const long long strides[8] = {a.q_row_stride,  a.q_head_stride,      a.k_page_stride,    a.k_page_head_stride,
                                  a.v_page_stride, a.v_page_head_stride, a.k_page_row_stride, a.v_page_row_stride};
    for (long long s : strides) {
        if (s % 8 != 0) return HAWK_ERR_ALIGN;
        if (s < 0 || s >= (1ll << 38)) return HAWK_ERR_UNSUPPORTED;
    }
    const int group = a.H / a.H_kv, max_new = a.max_new < a.T ? a.max_new : a.T;
    const long long rows_all = static_cast<long long>(max_new) * group;
    const bool tiles = rows_all > kFewRows;
    const int rows = static_cast<int>(tiles ? kFewRows : rows_all);
    const RowsPlan plan = plan_rows(a.S, rows, a.H_kv, a.D, a.max_kv, tiles);
    // list positions are 32-bit numbers
    const int tk = kStageBytes / (4 * a.D);
    if (static_cast<double>(a.S) * a.H_kv * ((rows + plan.rpi - 1) / plan.rpi) * (a.max_kv / tk + 1) >= 2147483000.0 ||
        static_cast<double>(a.T) * group >= 2147483000.0)
        return HAWK_ERR_UNSUPPORTED;
    const int groups = tiles ? hawk_host::paged_tile_groups(a.S, a.T, max_new, a.H, a.H_kv, rows) : 0;
    if (tiles && groups == 0) return HAWK_ERR_UNSUPPORTED;
    const size_t rows_ws = rows_workspace_bytes(plan, a.D);
    const size_t need = hawk_paged_attn_workspace_bytes(a.S, a.T, a.max_new, a.H, a.H_kv, a.D, a.max_kv);
    if (need > 0) {
        if (!a.workspace || a.workspace_bytes < need) return HAWK_ERR_WORKSPACE;
        if (!hawk_host::aligned16(a.workspace)) return HAWK_ERR_ALIGN;
    }
    if (!hawk_host::is_sm100(nullptr)) return HAWK_ERR_UNSUPPORTED;

    PagedParams P = {};
    P.q = a.q;
    P.out = a.out;
    P.row_begin = a.row_begin;
    P.kv_len = a.kv_len;
    P.block_table = a.block_table;
    P.anc_mask = a.anc_mask;
    P.records = static_cast<int32_t *>(a.workspace);
    P.record_ints = static_cast<long long>(hawk_host::kPagedSms) * (plan.shape == kShapeMid ? 1 : shares_warps(plan.rpi / 8)) * kRecordInts;
    P.part = reinterpret_cast<float *>(P.records + P.record_ints);
    P.part_floats = static_cast<long long>(rows_ws / sizeof(float)) - P.record_ints;
    P.q_row_stride = a.q_row_stride;
    P.q_head_stride = a.q_head_stride;
    P.S = a.S;
    P.T = a.T;
    P.max_new = max_new;
    P.H = a.H;
    P.H_kv = a.H_kv;
    P.group = group;
    P.n_pages = a.n_pages;
    P.page_size = a.page_size;
    P.table_width = a.table_width;
    P.kv_cap = a.max_kv;
    P.rows_few = rows;
    P.div_page.set(static_cast<uint32_t>(a.page_size));
    P.div_group.set(static_cast<uint32_t>(group));
    P.scale_log2 = a.sm_scale * 1.4426950408889634f;
    P.dev_status = dev_status;
    P.row_blocks = plan.grid;
    if (tiles) {
        P.groups = reinterpret_cast<PagedGroup *>(static_cast<uint8_t *>(a.workspace) + align16(rows_ws));
        P.group_cap = groups;
        P.tile_tok = 128 / group;
    }
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);

    if (plan.shape == kShapeMid) {
        if (hawk_host::launch_paged_mid(a, P, plan.rpi, st) != cudaSuccess) return HAWK_ERR_CUDA;
        cudaError_t e;
        if (a.dtype == HAWK_BF16)
            e = a.D == 64 ? launch_merge<__nv_bfloat16, 64, 64>(P, hawk_host::kPagedSms, st)
                          : launch_merge<__nv_bfloat16, 128, 64>(P, hawk_host::kPagedSms, st);
        else
            e = a.D == 64 ? launch_merge<__half, 64, 64>(P, hawk_host::kPagedSms, st)
                          : launch_merge<__half, 128, 64>(P, hawk_host::kPagedSms, st);
        if (e != cudaSuccess) return HAWK_ERR_CUDA;
    } else {
        CUtensorMap mk, mv;
        P.box_rows = hawk_host::paged_gcd(a.page_size, tk);
        if (!hawk_host::encode_pages(&mk, a, false, P.box_rows, &P.k_rows_inner) ||
            !hawk_host::encode_pages(&mv, a, true, P.box_rows, &P.v_rows_inner))
            return HAWK_ERR_CUDA;
        cudaError_t e;
        if (a.dtype == HAWK_BF16)
            e = a.D == 64 ? launch_rows_n<__nv_bfloat16, 64>(mk, mv, P, plan, st) : launch_rows_n<__nv_bfloat16, 128>(mk, mv, P, plan, st);
        else
            e = a.D == 64 ? launch_rows_n<__half, 64>(mk, mv, P, plan, st) : launch_rows_n<__half, 128>(mk, mv, P, plan, st);
        if (e != cudaSuccess) return HAWK_ERR_CUDA;
    }
    if (tiles && hawk_host::launch_paged_tile(a, P, reinterpret_cast<float *>(P.groups), st) != cudaSuccess) return HAWK_ERR_CUDA;
    return HAWK_OK;
}
