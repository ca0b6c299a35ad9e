// The paged cache between two steps: hawk_pages_resize, hawk_pages_fork, hawk_pages_compact (its state: block table, lengths, a count of
// references a page), hawk_pages_copy and hawk_pages_keep (rows of its pages).
//
// The paper has no paged cache; these are the bookkeeping and the copies that the calls around one need between two verify steps.
//
// The state is small (a few hundred KB at most) and every step of the bookkeeping needs the one before it: releases, then the free
// pages, then who gets them.  So resize and compact are ONE launch of one cluster: 8 blocks that share the scan of the counts,
// meet at cluster barriers (some 0.6 us each; another launch costs 1.5 to 2) and exchange one number a block through
// distributed shared memory.  What a free page is called is found by prefix sums over bit masks in shared memory, not by atomics, so
// results do not depend on the launch.  All of it is bound by latency: a launch, two or three barriers and as many dependent loads.
#include <climits>

#include "hawk_common.cuh"

namespace {

using hawk_host::aligned16;

constexpr int kBookBlocks = 8;       // of the cluster (the largest that every device runs)
constexpr int kBookThreads = 1024;
constexpr int kBookWarps = kBookThreads / 32;
constexpr int kMaxStreams = 4096;    // their prefix sums are held in shared memory
constexpr int kMaxPages = 1 << 20;   // a block's share of them as bit masks too
constexpr int kSlice = kMaxPages / kBookBlocks;

struct Div {  // number of pages of `keys` keys
    hawk::FastDiv page;
    __device__ __forceinline__ int pages(int keys) const { return static_cast<int>(page.div(static_cast<uint32_t>(keys) + page.d - 1)); }
};

__device__ __forceinline__ int warp_inclusive(int v)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += u;
    }
    return v;
}

// Exclusive prefix sum over the block's threads; *total: of all.  `sh` holds kBookWarps ints.
__device__ __forceinline__ int block_exclusive(int v, int *sh, int *total)
{
    const int inc = warp_inclusive(v), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();  // (sh may still be read from the sum before)
    if (lane == 31) sh[warp] = inc;
    __syncthreads();
    const int mine = sh[lane < kBookWarps ? lane : 0];
    const int sums = warp_inclusive(lane < kBookWarps ? mine : 0);
    *total = __shfl_sync(0xffffffffu, sums, kBookWarps - 1);
    const int before = warp > 0 ? __shfl_sync(0xffffffffu, sums, warp - 1) : 0;
    return before + inc - v;
}

// Barrier of the cluster (lanes that a branch parted come together first).
__device__ __forceinline__ void meet()
{
    __syncwarp();
    hawk::cluster_sync_all();
}

// Takes one reference of a page back; a count that is 0 already stays so.
__device__ __forceinline__ void release(int32_t *refs, int page, int n_pages, int &flags)
{
    if (page < 0 || page >= n_pages) {
        flags |= HAWK_DEV_BAD_PAGE;
    } else if (atomicSub(refs + page, 1) <= 0) {
        atomicAdd(refs + page, 1);
        flags |= HAWK_DEV_BAD_PAGE;
    }
}

__device__ __forceinline__ void report(int32_t *dev_status, int flags)
{
    if (flags && dev_status) atomicOr(dev_status, flags);
}

// A block's share of the pages, in whole runs of 128 (what a warp looks at in one go): [first, end).
__device__ __forceinline__ void slice_of(int n_pages, int rank, int &first, int &end)
{
    const int per = ((n_pages + kBookBlocks - 1) / kBookBlocks + 127) & ~127;
    first = min(n_pages, rank * per);
    end = min(n_pages, first + per);
}

// Which pages of the block's share satisfy `is(count, page)`: bit i of bits[w] stands for page first + 32 w + i.  Returns this thread's
// part of their number.
template <class F>
__device__ __forceinline__ int mark_pages(const int32_t *refs, int first, int end, uint32_t *bits, F &&is)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int count = 0;
    for (int p0 = first + warp * 128; p0 < end; p0 += kBookWarps * 128) {
        const int p = p0 + 4 * lane;
        uint32_t four = 0;
        if (p + 3 < end) {
            const int4 c = __ldcg(reinterpret_cast<const int4 *>(refs + p));
            four = (is(c.x, p) ? 1u : 0u) | (is(c.y, p + 1) ? 2u : 0u) | (is(c.z, p + 2) ? 4u : 0u) | (is(c.w, p + 3) ? 8u : 0u);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (p + i < end && is(__ldcg(refs + p + i), p + i)) four |= 1u << i;
        }
        count += __popc(four);
        uint32_t word = four << (4 * (lane & 7));
        word |= __shfl_xor_sync(0xffffffffu, word, 1);
        word |= __shfl_xor_sync(0xffffffffu, word, 2);
        word |= __shfl_xor_sync(0xffffffffu, word, 4);
        if ((lane & 7) == 0) bits[(p0 - first) / 32 + lane / 8] = word;
    }
    return count;
}

// The blocks' numbers `mine` (thread 0's): how many the blocks before this one have, and all.  A cluster barrier.
__device__ __forceinline__ void exchange_counts(int mine, int *slot, int rank, int &before, int &total)
{
    if (threadIdx.x == 0) *slot = mine;
    meet();
    before = total = 0;
#pragma unroll
    for (int r = 0; r < kBookBlocks; ++r) {
        const int n = static_cast<int>(hawk::ld_cluster_u32(hawk::map_shared_to_cta(slot, r)));
        if (r < rank) before += n;
        total += n;
    }
}

// ---------------------------------------------------------------------------------------------- resize
struct ResizeParams {
    const int32_t *table, *kv, *next, *refs;
    int32_t *out_table, *out_len, *out_refs, *copies;
    int S, W, n_pages;
    Div div;
    int32_t *dev_status;
};

struct ResizeShared {
    uint32_t bits[kSlice / 32];
    int end[kMaxStreams];    // running sum of the pages that streams need
    int kv[kMaxStreams];     // keys now; -1: the stream stays as it is (its lengths are out of range)
    int have[kMaxStreams];   // pages now, times two, plus one where the last is copied
    int sums[kBookWarps];
    int slot, any;
};

__global__ void __launch_bounds__(kBookThreads, 1) resize_kernel(ResizeParams P)
{
    extern __shared__ __align__(16) unsigned char smem_raw[];
    ResizeShared &sh = *reinterpret_cast<ResizeShared *>(smem_raw);
    hawk::allow_dependent_launch();
    hawk::grid_dependency_wait();
    const int tid = threadIdx.x, lane = tid & 31, rank = static_cast<int>(hawk::cluster_cta_rank());
    const int worker = rank * kBookWarps + (tid >> 5);  // warp of the cluster
    constexpr int kWorkers = kBookBlocks * kBookWarps;
    const long long cap = static_cast<long long>(P.W) * P.div.page.d;
    int flags = 0, first, end;
    slice_of(P.n_pages, rank, first, end);

    // ---- lengths; entries that stay; counts to where they are kept.  Everything that is decided is decided by the lengths as they
    // were on entry, which every block reads before the barrier in front of the writes.
    if (tid == 0) sh.any = 0;
    __syncthreads();
    bool shrinks = false;
    for (int s = tid; s < P.S; s += kBookThreads) {
        const int old = P.kv[s], next = P.next[s];
        const bool ok = old >= 0 && old <= cap && next >= 0 && next <= cap;
        if (!ok) flags |= HAWK_DEV_BAD_PREFIX;
        sh.kv[s] = ok ? old : -1;
        shrinks |= ok && next < old;
    }
    if (shrinks) sh.any = 1;
    const bool moved_refs = P.out_refs != P.refs;
    if (moved_refs) {
        for (int i = first / 4 + tid; i < end / 4; i += kBookThreads)
            reinterpret_cast<int4 *>(P.out_refs)[i] = reinterpret_cast<const int4 *>(P.refs)[i];
        for (int i = (end & ~3) + tid; i < end; i += kBookThreads) P.out_refs[i] = P.refs[i];
    }
    __syncthreads();
    const bool any = sh.any != 0;  // the same in all blocks
    if (any && moved_refs) meet();

    // ---- streams that shrink release pages
    if (any || P.out_table != P.table) {
        for (int s = worker; s < P.S; s += kWorkers) {
            const int old = sh.kv[s];
            if (old < 0) continue;
            const int next = P.next[s], have = P.div.pages(old), stay = next < old ? P.div.pages(next) : have;
            const size_t row = static_cast<size_t>(s) * P.W;
            if (P.out_table != P.table)
                for (int j = lane; j < stay; j += 32) P.out_table[row + j] = P.table[row + j];
            for (int j = stay + lane; j < have; j += 32) release(P.out_refs, P.table[row + j], P.n_pages, flags);
        }
    }
    if (any || moved_refs) meet();

    // ---- what every stream needs (each block for itself), and the free pages of the block's share
    int need[kMaxStreams / kBookThreads], sum = 0;
#pragma unroll
    for (int i = 0; i < kMaxStreams / kBookThreads; ++i) {
        const int s = tid * (kMaxStreams / kBookThreads) + i;
        need[i] = 0;
        if (s >= P.S) continue;
        const int old = sh.kv[s];
        int have = 0, copy = 0;
        if (old >= 0) {
            const int next = P.next[s];
            uint32_t part;
            have = P.div.pages(old);
            P.div.page.divmod(static_cast<uint32_t>(old), part);
            if (next > old) {
                if (part != 0) {
                    const int page = P.table[static_cast<size_t>(s) * P.W + have - 1];
                    if (page < 0 || page >= P.n_pages) flags |= HAWK_DEV_BAD_PAGE;
                    else copy = __ldcg(P.out_refs + page) > 1;
                }
                need[i] = P.div.pages(next) - have + copy;
            }
        }
        sh.have[s] = have * 2 + copy;
        sum += need[i];
    }
    int total_need, total_free, free_before, mine;
    int run = block_exclusive(sum, sh.sums, &total_need);
#pragma unroll
    for (int i = 0; i < kMaxStreams / kBookThreads; ++i) {
        const int s = tid * (kMaxStreams / kBookThreads) + i;
        run += need[i];
        if (s < P.S) sh.end[s] = run;
    }
    const int words = (end - first + 31) / 32;
    int count = mark_pages(P.out_refs, first, end, sh.bits, [](int c, int) { return c == 0; });
    (void)block_exclusive(count, sh.sums, &mine);  // (its barriers publish bits and end)
    exchange_counts(mine, &sh.slot, rank, free_before, total_free);

    // ---- the free pages of the share to the streams whose turn they are
    if (free_before < total_need && total_need > 0) {
        const int per = (words + kBookThreads - 1) / kBookThreads;  // consecutive words a thread
        int in = 0, dummy;
        for (int w = tid * per; w < min(words, (tid + 1) * per); ++w) in += __popc(sh.bits[w]);
        int r = free_before + block_exclusive(in, sh.sums, &dummy);
        for (int w = tid * per; w < min(words, (tid + 1) * per) && r < total_need; ++w) {
            for (uint32_t m = sh.bits[w]; m && r < total_need; m &= m - 1, ++r) {
                const int page = first + w * 32 + __ffs(m) - 1;
                int lo = 0, hi = P.S - 1;  // the first stream whose running sum is past r
                while (lo < hi) {
                    const int mid = (lo + hi) / 2;
                    if (sh.end[mid] > r) hi = mid;
                    else lo = mid + 1;
                }
                if (sh.end[lo] > total_free) continue;  // this stream and all behind it stay as they were
                const int copy = sh.have[lo] & 1, have = sh.have[lo] >> 1;
                const int at = r - (lo > 0 ? sh.end[lo - 1] : 0);
                const int j = have - copy + at;
                const size_t e = static_cast<size_t>(lo) * P.W + j;
                if (!HAWK_IN_BOUNDS(P.dev_status, j, P.W) || !HAWK_IN_BOUNDS(P.dev_status, page, P.n_pages)) continue;
                if (copy && at == 0) {
                    const int from = P.table[e];
                    uint32_t part;
                    P.div.page.divmod(static_cast<uint32_t>(sh.kv[lo]), part);
                    P.copies[3 * lo] = from;
                    P.copies[3 * lo + 1] = page;
                    P.copies[3 * lo + 2] = static_cast<int>(part);
                    release(P.out_refs, from, P.n_pages, flags);
                }
                P.out_table[e] = page;
                P.out_refs[page] = 1;
            }
        }
    }
    for (int s = rank * kBookThreads + tid; s < P.S; s += kBookBlocks * kBookThreads) {
        const int needs = sh.end[s] - (s > 0 ? sh.end[s - 1] : 0);
        const bool served = needs == 0 || sh.end[s] <= total_free;
        if (!served) flags |= HAWK_DEV_NO_PAGES;
        if (!(sh.have[s] & 1) || !served) {
            P.copies[3 * s] = -1;
            P.copies[3 * s + 1] = -1;
            P.copies[3 * s + 2] = 0;
        }
        if (sh.kv[s] < 0) {
            if (P.out_len != P.kv) P.out_len[s] = P.kv[s];
        } else {
            const int next = P.next[s];
            P.out_len[s] = served ? next : sh.kv[s];
        }
    }
    report(P.dev_status, flags);
    meet();  // nobody leaves while its numbers are read
}

// ---------------------------------------------------------------------------------------------- fork
struct ForkParams {
    const int32_t *table, *kv, *parent, *length;
    int32_t *out_table, *out_len, *refs;
    int S, S_out, W, n_pages;
    Div div;
    int32_t *dev_status;
};

__global__ void __launch_bounds__(256) copy_ints_kernel(const int32_t *from, int32_t *to, int n)
{
    hawk::allow_dependent_launch();
    hawk::grid_dependency_wait();
    const int i = (blockIdx.x * 256 + threadIdx.x) * 4;
    if (i + 3 < n) {
        *reinterpret_cast<int4 *>(to + i) = *reinterpret_cast<const int4 *>(from + i);
    } else {
        for (int k = i; k < n; ++k) to[k] = from[k];
    }
}

// A block of 128 lanes takes one stream's entries, old and new: entry j of out stream t is its parent's; the count of a page that t
// named before and names still (a stream that goes on) is not touched at all.
__global__ void __launch_bounds__(128) fork_kernel(ForkParams P)
{
    hawk::allow_dependent_launch();
    hawk::grid_dependency_wait();
    const int t = blockIdx.x, tid = threadIdx.x;
    const long long cap = static_cast<long long>(P.W) * P.div.page.d;
    int flags = 0;
    auto keys_of = [&](int s) {
        const int kv = P.kv[s];
        if (kv >= 0 && kv <= cap) return kv;
        flags |= HAWK_DEV_BAD_PREFIX;
        return 0;
    };
    int from = -1, take = 0;
    if (t < P.S_out) {
        from = P.parent[t];
        if (from < -1 || from >= P.S) {
            flags |= HAWK_DEV_BAD_ROWS;
            from = -1;
        }
        int keys = from < 0 ? 0 : keys_of(from);
        if (P.length && from >= 0) {
            const int most = P.length[t];
            if (most < 0) flags |= HAWK_DEV_BAD_PREFIX;
            keys = min(keys, max(most, 0));
        }
        take = P.div.pages(keys);
        if (tid == 0) P.out_len[t] = keys;
    }
    const int held = t < P.S ? P.div.pages(keys_of(t)) : 0;
    const int same = from == t ? min(take, held) : 0;  // entries that go on
    const size_t row = static_cast<size_t>(t) * P.W, source = static_cast<size_t>(max(from, 0)) * P.W;
    for (int j = tid; j < take; j += 128) {
        const int page = P.table[source + j];
        P.out_table[row + j] = page;
        if (j < same) continue;
        if (page < 0 || page >= P.n_pages) flags |= HAWK_DEV_BAD_PAGE;
        else atomicAdd(P.refs + page, 1);
    }
    for (int j = same + tid; j < held; j += 128) {
        const int page = P.table[row + j];
        if (page < 0 || page >= P.n_pages) flags |= HAWK_DEV_BAD_PAGE;
        else atomicSub(P.refs + page, 1);
    }
    report(P.dev_status, flags);
}

// ---------------------------------------------------------------------------------------------- compact
struct CompactParams {
    const int32_t *table, *kv, *refs;
    int32_t *out_table, *out_refs, *copies, *top;
    int32_t *to, *from;   // [moves + 1] the lowest free pages, ascending, and the highest in use, descending
    int32_t *place;       // [n_pages] place in the lists of the pages that move
    int S, W, n_pages, first_page, moves;
    Div div;
    int32_t *dev_status;
};

struct CompactShared {
    uint32_t used[kSlice / 32];
    int sums[kBookWarps];
    int slot_used, slot_free;
};

__global__ void __launch_bounds__(kBookThreads, 1) compact_kernel(CompactParams P)
{
    extern __shared__ __align__(16) unsigned char smem_raw[];
    CompactShared &sh = *reinterpret_cast<CompactShared *>(smem_raw);
    hawk::allow_dependent_launch();
    hawk::grid_dependency_wait();
    const int tid = threadIdx.x, lane = tid & 31, rank = static_cast<int>(hawk::cluster_cta_rank());
    const long long cap = static_cast<long long>(P.W) * P.div.page.d;
    int flags = 0, first, end;
    slice_of(P.n_pages, rank, first, end);
    if (P.out_refs != P.refs) {
        for (int i = first / 4 + tid; i < end / 4; i += kBookThreads)
            reinterpret_cast<int4 *>(P.out_refs)[i] = reinterpret_cast<const int4 *>(P.refs)[i];
        for (int i = (end & ~3) + tid; i < end; i += kBookThreads) P.out_refs[i] = P.refs[i];
    }
    const int words = (end - first + 31) / 32;
    // pages of the share from first_page on
    const int from_page = P.first_page;
    const int count = mark_pages(P.refs, first, end, sh.used, [=](int c, int p) { return c != 0 && p >= from_page; });
    int mine, used_before, used, free_before, free_all;
    (void)block_exclusive(count, sh.sums, &mine);
    const int eligible = max(0, end - max(first, from_page));
    if (tid == 0) sh.slot_free = eligible - mine;
    exchange_counts(mine, &sh.slot_used, rank, used_before, used);
    free_before = free_all = 0;
#pragma unroll
    for (int r = 0; r < kBookBlocks; ++r) {
        const int n = static_cast<int>(hawk::ld_cluster_u32(hawk::map_shared_to_cta(&sh.slot_free, r)));
        if (r < rank) free_before += n;
        free_all += n;
    }

    // ---- the lowest free pages and the highest in use, by rank
    const int lists = P.moves + 1;
    const int per = (words + kBookThreads - 1) / kBookThreads;
    const int w0 = tid * per, w1 = min(words, w0 + per);
    int in = 0, open = 0, dummy;
    auto free_bits = [&](int w) {  // of word w: not in use, inside the share, from first_page on
        const int p = first + w * 32;
        uint32_t m = ~sh.used[w];
        if (end - p < 32) m &= (1u << (end - p)) - 1;
        if (from_page > p) m &= from_page - p >= 32 ? 0u : ~((1u << (from_page - p)) - 1);
        return m;
    };
    for (int w = w0; w < w1; ++w) {
        in += __popc(sh.used[w]);
        open += __popc(free_bits(w));
    }
    int u = used_before + block_exclusive(in, sh.sums, &dummy), f = free_before + block_exclusive(open, sh.sums, &dummy);
    for (int w = w0; w < w1; ++w) {
        const int p = first + w * 32;
        if (used - u - __popc(sh.used[w]) < lists) {  // (the word's last page in use is of this rank from the top)
            for (uint32_t m = sh.used[w]; m; m &= m - 1, ++u) {
                const int i = used - 1 - u;
                if (i < lists && HAWK_IN_BOUNDS(P.dev_status, i, lists)) P.from[i] = p + __ffs(m) - 1;
            }
        } else {
            u += __popc(sh.used[w]);
        }
        for (uint32_t m = f < lists ? free_bits(w) : 0u; m; m &= m - 1, ++f)
            if (f < lists && HAWK_IN_BOUNDS(P.dev_status, f, lists)) P.to[f] = p + __ffs(m) - 1;
    }
    meet();

    // ---- moves: pairs of the lists for as long as they go down (once one does not, none behind it does)
    const int pairs = min(P.moves, min(used, free_all));
    int down = 0, moved;
    for (int i = tid; i < pairs; i += kBookThreads) down += __ldcg(P.to + i) < __ldcg(P.from + i);
    (void)block_exclusive(down, sh.sums, &moved);  // each block counts them for itself
    for (int i = rank * kBookThreads + tid; i < P.moves; i += kBookBlocks * kBookThreads) {
        int a = -1, b = -1;
        if (i < moved) {
            a = __ldcg(P.from + i);
            b = __ldcg(P.to + i);
            P.out_refs[b] = P.refs[a];
            P.out_refs[a] = 0;
            P.place[a] = i;
        }
        P.copies[3 * i] = a;
        P.copies[3 * i + 1] = b;
        P.copies[3 * i + 2] = a < 0 ? 0 : static_cast<int>(P.div.page.d);
    }
    if (P.top && rank == 0 && tid == 0) {
        int top = from_page;  // behind the highest page in use: one that stayed, or the last that moved in
        if (moved < used) top = max(top, __ldcg(P.from + moved) + 1);
        if (moved > 0) top = max(top, __ldcg(P.to + moved - 1) + 1);
        *P.top = top;
    }
    const int lowest = moved > 0 ? __ldcg(P.from + moved - 1) : INT_MAX;  // pages in use from here on have moved
    meet();

    // ---- the new ids into the table
    if (moved == 0 && P.out_table == P.table) {
        report(P.dev_status, flags);
        return;  // (moved is the same in all blocks, and no block reads another's shared memory any more)
    }
    for (int s = rank * kBookWarps + (tid >> 5); s < P.S; s += kBookBlocks * kBookWarps) {
        const int kv = P.kv[s];
        if (kv < 0 || kv > cap) {
            flags |= HAWK_DEV_BAD_PREFIX;
            continue;
        }
        const int n = P.div.pages(kv);
        const size_t row = static_cast<size_t>(s) * P.W;
        for (int j = lane; j < n; j += 32) {
            int page = P.table[row + j];
            if (page < 0 || page >= P.n_pages) flags |= HAWK_DEV_BAD_PAGE;
            else if (page >= lowest) {
                const int i = __ldcg(P.place + page);  // (no more than a guess for a page that the counts say is free)
                if (i >= 0 && i < moved && __ldcg(P.from + i) == page) page = __ldcg(P.to + i);
                else flags |= HAWK_DEV_BAD_PAGE;
            }
            P.out_table[row + j] = page;
        }
    }
    report(P.dev_status, flags);
}

// ---------------------------------------------------------------------------------------------- rows of pages
struct PageSide {
    uint4 *base;
    long long layer, page, head, row;  // strides in 16-byte pieces
};

struct PageParams {
    PageSide side[2];  // keys, values
    int n_pages, H, page_size, pieces;  // pieces of 16 bytes a row of a head
    hawk::FastDiv div_pieces, div_inner, div_page;
    int inner[2];  // 1: rows are the inner dimension of a side's pages, 0: heads are
    int32_t *dev_status;
};

constexpr int kCopyThreads = 256;
constexpr int kCopyUnroll = 8;  // loads in flight a thread
constexpr int kCopyPieces = 2 * kCopyThreads * kCopyUnroll;  // of a block: 64 KB

// Block (x, y, z): entry x; keys or values of layer y / 2; z: which kCopyPieces of the page.  Pieces are taken in the order of memory.
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(PageParams P, const int32_t *copies)
{
    hawk::allow_dependent_launch();
    hawk::grid_dependency_wait();
    const int a = copies[3 * static_cast<size_t>(blockIdx.x)], b = copies[3 * static_cast<size_t>(blockIdx.x) + 1];
    const int rows = min(copies[3 * static_cast<size_t>(blockIdx.x) + 2], P.page_size);
    if (a < 0) return;
    if (a >= P.n_pages || b < 0 || b >= P.n_pages) {
        if (threadIdx.x == 0) report(P.dev_status, HAWK_DEV_BAD_PAGE);
        return;
    }
    if (rows <= 0) return;
    const PageSide &side = P.side[blockIdx.y & 1];
    const bool inner = P.inner[blockIdx.y & 1] != 0;
    uint4 *layer = side.base + (blockIdx.y >> 1) * side.layer;
    const uint4 *from = layer + a * side.page;
    uint4 *to = layer + b * side.page;
    const uint32_t all = static_cast<uint32_t>(P.H) * P.page_size * P.pieces;
    const uint32_t last = min(all, (blockIdx.z + 1) * static_cast<uint32_t>(kCopyPieces));
    for (uint32_t c0 = blockIdx.z * static_cast<uint32_t>(kCopyPieces) + threadIdx.x; c0 < last; c0 += kCopyThreads * kCopyUnroll) {
        uint4 v[kCopyUnroll];
        long long at[kCopyUnroll];
#pragma unroll
        for (int i = 0; i < kCopyUnroll; ++i) {
            const uint32_t c = c0 + i * kCopyThreads;
            at[i] = -1;
            if (c >= last) continue;
            uint32_t piece, low;
            const uint32_t cell = P.div_pieces.divmod(c, piece);
            uint32_t high;
            if (inner) high = P.div_page.divmod(cell, low);
            else high = P.div_inner.divmod(cell, low);
            const int row = static_cast<int>(inner ? low : high), head = static_cast<int>(inner ? high : low);
            if (row >= rows) continue;
            at[i] = head * side.head + row * side.row + piece;
            v[i] = __ldcs(from + at[i]);
        }
#pragma unroll
        for (int i = 0; i < kCopyUnroll; ++i)
            if (at[i] >= 0) __stcs(to + at[i], v[i]);
    }
}

struct KeepParams {
    PageParams pages;
    const int32_t *table, *row_begin, *kv, *path, *accept_len;
    int32_t *out_len;
    int S, B, W, path_width, first;
    int columns;  // blocks along z share a stream's columns
};

constexpr int kKeepThreads = 128;
constexpr int kKeepRows = 64;   // rows whose places are held at a time
constexpr int kKeepUnroll = 8;

// Block (x, y, z): stream x; keys or values of layer y / 2; z: a share of the columns (16 bytes of a row of a head).  A thread moves its
// column's rows one batch after the other, all loads of a batch before its stores.  The path ascends from `first` on, so row first + i is not
// behind row path[i], and no row is written before it was read.
__global__ void __launch_bounds__(kKeepThreads) keep_kernel(KeepParams P)
{
    __shared__ long long src[kKeepRows], dst[kKeepRows];
    hawk::allow_dependent_launch();
    hawk::grid_dependency_wait();
    const int s = blockIdx.x, tid = threadIdx.x, of = s % P.B;
    const bool leader = blockIdx.y == 0 && blockIdx.z == 0;
    const int r0 = P.row_begin[s], r1 = P.row_begin[s + 1], kv = P.kv[s], accepted = P.accept_len[of];
    const int32_t *path = P.path ? P.path + static_cast<size_t>(of) * P.path_width : nullptr;
    const long long n = static_cast<long long>(r1) - r0;
    int flags = 0, length = kv, moves = 0;
    if (r0 < 0 || n < 0) flags = HAWK_DEV_BAD_ROWS;
    else if (n > 0) {
        if (kv < n || (path && kv > static_cast<long long>(P.W) * P.pages.page_size)) flags = HAWK_DEV_BAD_PREFIX;
        else if (accepted < 0 || (path && accepted > P.path_width)) flags = HAWK_DEV_BAD_TREE;
        else {
            length = static_cast<int>(kv - n + min(n, static_cast<long long>(P.first) + accepted));
            moves = path ? accepted : 0;
        }
    }
    const int base = static_cast<int>(kv - n);
    if (path && moves > 0) {  // does it ascend, from `first` on, below n?
        bool bad = false;
        for (int i = tid; i < moves; i += kKeepThreads) {
            const int p = path[i];
            bad |= p >= n || p < (i == 0 ? P.first : path[i - 1] + 1);
        }
        if (__syncthreads_or(bad)) {
            flags = HAWK_DEV_BAD_TREE;
            length = kv;
            moves = 0;
        }
    }
    if (leader && tid == 0) {
        P.out_len[s] = length;
        report(P.pages.dev_status, flags);
    }
    if (moves == 0) return;
    const PageSide &side = P.pages.side[blockIdx.y & 1];
    uint4 *layer = side.base + (blockIdx.y >> 1) * side.layer;
    const int columns = P.pages.H * P.pages.pieces;
    for (int i0 = 0; i0 < moves; i0 += kKeepRows) {
        const int rows = min(kKeepRows, moves - i0);
        if (i0 > 0) __syncthreads();
        if (tid < rows) {
            const int i = i0 + tid;
            uint32_t in_a, in_b;
            const uint32_t ja = P.pages.div_page.divmod(static_cast<uint32_t>(base + path[i]), in_a);
            const uint32_t jb = P.pages.div_page.divmod(static_cast<uint32_t>(base + P.first + i), in_b);
            long long a = -1, b = -1;
            if (path[i] != P.first + i && HAWK_IN_BOUNDS(P.pages.dev_status, ja, P.W) && HAWK_IN_BOUNDS(P.pages.dev_status, jb, P.W)) {
                const int pa = P.table[static_cast<size_t>(s) * P.W + ja], pb = P.table[static_cast<size_t>(s) * P.W + jb];
                if (pa < 0 || pa >= P.pages.n_pages || pb < 0 || pb >= P.pages.n_pages) {
                    if (leader) report(P.pages.dev_status, HAWK_DEV_BAD_PAGE);
                } else {
                    a = pa * side.page + static_cast<long long>(in_a) * side.row;
                    b = pb * side.page + static_cast<long long>(in_b) * side.row;
                }
            }
            src[tid] = a;
            dst[tid] = b;
        }
        __syncthreads();
        for (int c = blockIdx.z * kKeepThreads + tid; c < columns; c += P.columns * kKeepThreads) {
            uint32_t piece;
            const uint32_t head = P.pages.div_pieces.divmod(static_cast<uint32_t>(c), piece);
            uint4 *column = layer + head * side.head + piece;
            for (int i = 0; i < rows; i += kKeepUnroll) {
                uint4 v[kKeepUnroll];
#pragma unroll
                for (int k = 0; k < kKeepUnroll; ++k)
                    if (i + k < rows && src[i + k] >= 0) v[k] = column[src[i + k]];
#pragma unroll
                for (int k = 0; k < kKeepUnroll; ++k)
                    if (i + k < rows && src[i + k] >= 0) column[dst[i + k]] = v[k];
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------- host side
hawk_status check_state(int S, int W, int n_pages, int page_size)
{
    if (S < 0 || W < 0 || n_pages < 0 || page_size < 0) return HAWK_ERR_SHAPE;
    if (page_size < 1) return HAWK_ERR_SHAPE;
    if (S > kMaxStreams || n_pages > kMaxPages || page_size > 65536) return HAWK_ERR_UNSUPPORTED;
    if (static_cast<long long>(S) * W >= (1ll << 31) || static_cast<long long>(W) * page_size >= (1ll << 31) - 65536)
        return HAWK_ERR_UNSUPPORTED;
    return HAWK_OK;
}

Div make_div(int page_size)
{
    Div d;
    d.page.set(static_cast<uint32_t>(page_size));
    return d;
}

hawk_status done(cudaError_t e) { return e == cudaSuccess ? HAWK_OK : HAWK_ERR_CUDA; }

// Lets `kernel` use `bytes` of shared memory on the current device (asked once for each).
template <class K>
bool allow_smem(K *kernel, size_t bytes, unsigned long long (&seen))
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    const unsigned long long bit = 1ull << (dev & 63);
    if (__atomic_load_n(&seen, __ATOMIC_ACQUIRE) & bit && dev < 64) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes)) != cudaSuccess) return false;
    __atomic_fetch_or(&seen, bit, __ATOMIC_RELEASE);
    return true;
}

hawk_status check_pages(const hawk_page_tensors &p)
{
    if (p.layers < 0 || p.n_pages < 0 || p.H_kv < 0 || p.page_size < 0 || p.D < 0) return HAWK_ERR_SHAPE;
    if (p.H_kv < 1 || p.page_size < 1 || p.D < 1 || p.n_pages < 1) return HAWK_ERR_SHAPE;
    if (p.D % 8 != 0 || p.D > 65536 || p.page_size > 65536 || p.layers > 32767) return HAWK_ERR_UNSUPPORTED;
    if (p.H_kv > 65536 || static_cast<long long>(p.H_kv) * p.page_size > (1ll << 30) / p.D) return HAWK_ERR_UNSUPPORTED;
    if (!p.k_pages || !p.v_pages) return HAWK_ERR_NULL;
    if (!aligned16(p.k_pages) || !aligned16(p.v_pages)) return HAWK_ERR_ALIGN;
    const long long strides[] = {p.k_layer_stride, p.k_page_stride, p.k_head_stride, p.k_row_stride,
                                 p.v_layer_stride, p.v_page_stride, p.v_head_stride, p.v_row_stride};
    for (long long s : strides)
        if (s % 8 != 0) return HAWK_ERR_ALIGN;
    return HAWK_OK;
}

PageParams page_params(const hawk_page_tensors &p, int32_t *dev_status)
{
    PageParams P = {};
    P.side[0] = {static_cast<uint4 *>(p.k_pages), p.k_layer_stride / 8, p.k_page_stride / 8, p.k_head_stride / 8, p.k_row_stride / 8};
    P.side[1] = {static_cast<uint4 *>(p.v_pages), p.v_layer_stride / 8, p.v_page_stride / 8, p.v_head_stride / 8, p.v_row_stride / 8};
    P.inner[0] = p.k_row_stride <= p.k_head_stride;
    P.inner[1] = p.v_row_stride <= p.v_head_stride;
    P.n_pages = p.n_pages;
    P.H = p.H_kv;
    P.page_size = p.page_size;
    P.pieces = p.D / 8;
    P.div_pieces.set(static_cast<uint32_t>(P.pieces));
    P.div_inner.set(static_cast<uint32_t>(p.H_kv));
    P.div_page.set(static_cast<uint32_t>(p.page_size));
    P.dev_status = dev_status;
    return P;
}

}  // namespace

extern "C" hawk_status hawk_pages_resize(const hawk_pages_resize_args *a, int32_t *dev_status, hawk_stream_t stream)
{
    const hawk_host::NvtxRange nvtx_range("hawk_pages_resize");
    if (!a) return HAWK_ERR_NULL;
    const hawk_status chk = check_state(a->S, a->table_width, a->n_pages, a->page_size);
    if (chk != HAWK_OK) return chk;
    if (a->S == 0 && (a->n_pages == 0 || a->page_refs == a->out_refs)) return HAWK_OK;
    if (a->S > 0 && (!a->block_table || !a->kv_len || !a->new_len || !a->out_table || !a->out_len || !a->copies)) return HAWK_ERR_NULL;
    if (a->n_pages > 0 && (!a->page_refs || !a->out_refs)) return HAWK_ERR_NULL;
    if (!aligned16(a->page_refs) || !aligned16(a->out_refs)) return HAWK_ERR_ALIGN;
    if (!hawk_host::is_sm100(nullptr)) return HAWK_ERR_UNSUPPORTED;
    static unsigned long long seen = 0;
    if (!allow_smem(resize_kernel, sizeof(ResizeShared), seen)) return HAWK_ERR_CUDA;
    ResizeParams P = {a->block_table, a->kv_len, a->new_len, a->page_refs, a->out_table, a->out_len, a->out_refs, a->copies,
                      a->S, a->table_width, a->n_pages, make_div(a->page_size), dev_status};
    return done(hawk_host::launch_dependent_clusters(resize_kernel, kBookBlocks, dim3(kBookBlocks), dim3(kBookThreads),
                                                     sizeof(ResizeShared), reinterpret_cast<cudaStream_t>(stream), P));
}

extern "C" hawk_status hawk_pages_fork(const hawk_pages_fork_args *a, int32_t *dev_status, hawk_stream_t stream)
{
    const hawk_host::NvtxRange nvtx_range("hawk_pages_fork");
    if (!a) return HAWK_ERR_NULL;
    hawk_status chk = check_state(a->S, a->table_width, a->n_pages, a->page_size);
    if (chk == HAWK_OK) chk = check_state(a->S_out, a->table_width, a->n_pages, a->page_size);
    if (chk != HAWK_OK) return chk;
    const bool move = a->n_pages > 0 && a->page_refs != a->out_refs;
    if (a->S == 0 && a->S_out == 0 && !move) return HAWK_OK;
    if (a->S > 0 && (!a->block_table || !a->kv_len)) return HAWK_ERR_NULL;
    if (a->S_out > 0 && (!a->parent || !a->out_table || !a->out_len)) return HAWK_ERR_NULL;
    if (a->n_pages > 0 && (!a->page_refs || !a->out_refs)) return HAWK_ERR_NULL;
    if (!aligned16(a->page_refs) || !aligned16(a->out_refs)) return HAWK_ERR_ALIGN;
    if ((a->S_out > 0 && a->S > 0) && (a->out_table == a->block_table || a->out_len == a->kv_len)) return HAWK_ERR_PARAM;
    if (!hawk_host::is_sm100(nullptr)) return HAWK_ERR_UNSUPPORTED;
    const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (move) {
        const int per = 256 * 4;
        const cudaError_t e = hawk_host::launch_dependent(copy_ints_kernel, dim3((a->n_pages + per - 1) / per), dim3(256), 0, st,
                                                          a->page_refs, a->out_refs, a->n_pages);
        if (e != cudaSuccess) return HAWK_ERR_CUDA;
    }
    const int streams = a->S > a->S_out ? a->S : a->S_out;
    if (streams == 0) return HAWK_OK;
    ForkParams P = {a->block_table, a->kv_len, a->parent, a->length, a->out_table, a->out_len, a->out_refs,
                    a->S, a->S_out, a->table_width, a->n_pages, make_div(a->page_size), dev_status};
    return done(hawk_host::launch_dependent(fork_kernel, dim3(streams), dim3(128), 0, st, P));
}

extern "C" size_t hawk_pages_compact_workspace_bytes(int n_pages, int max_moves)
{
    if (n_pages < 1 || n_pages > kMaxPages || max_moves < 0) return 0;
    const size_t moves = max_moves < n_pages ? max_moves : n_pages;
    return sizeof(int32_t) * (static_cast<size_t>(n_pages) + 2 * (moves + 1));
}

extern "C" hawk_status hawk_pages_compact(const hawk_pages_compact_args *a, int32_t *dev_status, hawk_stream_t stream)
{
    const hawk_host::NvtxRange nvtx_range("hawk_pages_compact");
    if (!a) return HAWK_ERR_NULL;
    const hawk_status chk = check_state(a->S, a->table_width, a->n_pages, a->page_size);
    if (chk != HAWK_OK) return chk;
    if (a->first_page < 0 || a->max_moves < 0) return HAWK_ERR_SHAPE;
    if (a->max_moves > kMaxPages) return HAWK_ERR_UNSUPPORTED;
    if (a->S > 0 && (!a->block_table || !a->kv_len || !a->out_table)) return HAWK_ERR_NULL;
    if (a->n_pages > 0 && (!a->page_refs || !a->out_refs)) return HAWK_ERR_NULL;
    if (a->max_moves > 0 && !a->copies) return HAWK_ERR_NULL;
    if (!aligned16(a->page_refs) || !aligned16(a->out_refs) || !aligned16(a->workspace)) return HAWK_ERR_ALIGN;
    if (a->n_pages > 0 && (!a->workspace || a->workspace_bytes < hawk_pages_compact_workspace_bytes(a->n_pages, a->max_moves)))
        return HAWK_ERR_WORKSPACE;
    if (!hawk_host::is_sm100(nullptr)) return HAWK_ERR_UNSUPPORTED;
    static unsigned long long seen = 0;
    if (!allow_smem(compact_kernel, sizeof(CompactShared), seen)) return HAWK_ERR_CUDA;
    CompactParams P = {};
    P.table = a->block_table;
    P.kv = a->kv_len;
    P.refs = a->page_refs;
    P.out_table = a->out_table;
    P.out_refs = a->out_refs;
    P.copies = a->copies;
    P.top = a->top;
    const int lists = (a->max_moves < a->n_pages ? a->max_moves : a->n_pages) + 1;
    P.to = static_cast<int32_t *>(a->workspace);
    P.from = P.to + lists;
    P.place = P.from + lists;
    P.S = a->S;
    P.W = a->table_width;
    P.n_pages = a->n_pages;
    P.first_page = a->first_page < a->n_pages ? a->first_page : a->n_pages;
    P.moves = a->max_moves;
    P.div = make_div(a->page_size);
    P.dev_status = dev_status;
    return done(hawk_host::launch_dependent_clusters(compact_kernel, kBookBlocks, dim3(kBookBlocks), dim3(kBookThreads),
                                                     sizeof(CompactShared), reinterpret_cast<cudaStream_t>(stream), P));
}

extern "C" hawk_status hawk_pages_copy(const hawk_page_tensors *pages, const int32_t *copies, int n_copies, int32_t *dev_status,
                                       hawk_stream_t stream)
{
    const hawk_host::NvtxRange nvtx_range("hawk_pages_copy");
    if (!pages) return HAWK_ERR_NULL;
    if (n_copies < 0 || pages->layers < 0) return HAWK_ERR_SHAPE;
    if (n_copies == 0 || pages->layers == 0) return HAWK_OK;
    const hawk_status chk = check_pages(*pages);
    if (chk != HAWK_OK) return chk;
    if (!copies) return HAWK_ERR_NULL;
    if (!hawk_host::is_sm100(nullptr)) return HAWK_ERR_UNSUPPORTED;
    const PageParams P = page_params(*pages, dev_status);
    const long long all = static_cast<long long>(P.H) * P.page_size * P.pieces;
    const dim3 grid(n_copies, 2 * pages->layers, static_cast<unsigned>((all + kCopyPieces - 1) / kCopyPieces));
    return done(hawk_host::launch_dependent(copy_kernel, grid, dim3(kCopyThreads), 0, reinterpret_cast<cudaStream_t>(stream), P, copies));
}

extern "C" hawk_status hawk_pages_keep(const hawk_pages_keep_args *a, int32_t *dev_status, hawk_stream_t stream)
{
    const hawk_host::NvtxRange nvtx_range("hawk_pages_keep");
    if (!a) return HAWK_ERR_NULL;
    if (a->S < 0 || a->B < 0 || a->path_width < 0 || a->first < 0 || a->table_width < 0) return HAWK_ERR_SHAPE;
    if (a->S == 0) return HAWK_OK;
    if (a->B < 1 || a->S % a->B != 0) return HAWK_ERR_SHAPE;
    if (!a->row_begin || !a->kv_len || !a->accept_len || !a->out_len) return HAWK_ERR_NULL;
    if (a->out_len == a->kv_len) return HAWK_ERR_PARAM;
    KeepParams P = {};
    int layers = 1;
    if (a->path) {
        const hawk_status chk = check_pages(a->pages);
        if (chk != HAWK_OK) return chk;
        if (!a->block_table) return HAWK_ERR_NULL;
        if (static_cast<long long>(a->S) * a->table_width >= (1ll << 31) ||
            static_cast<long long>(a->table_width) * a->pages.page_size >= (1ll << 31) - 65536)
            return HAWK_ERR_UNSUPPORTED;
        P.pages = page_params(a->pages, dev_status);
        layers = a->pages.layers > 1 ? a->pages.layers : 1;
        if (a->pages.layers == 0) P.pages.H = 0;  // (lengths only)
    }
    if (!hawk_host::is_sm100(nullptr)) return HAWK_ERR_UNSUPPORTED;
    P.pages.dev_status = dev_status;
    P.table = a->block_table;
    P.row_begin = a->row_begin;
    P.kv = a->kv_len;
    P.path = a->path;
    P.accept_len = a->accept_len;
    P.out_len = a->out_len;
    P.S = a->S;
    P.B = a->B;
    P.W = a->table_width;
    P.path_width = a->path_width;
    P.first = a->first;
    const int blocks = a->path ? (P.pages.H * P.pages.pieces + kKeepThreads - 1) / kKeepThreads : 1;
    P.columns = blocks < 1 ? 1 : blocks > 16 ? 16 : blocks;
    const dim3 grid(a->S, a->path ? 2 * layers : 1, P.columns);
    return done(hawk_host::launch_dependent(keep_kernel, grid, dim3(kKeepThreads), 0, reinterpret_cast<cudaStream_t>(stream), P));
}
