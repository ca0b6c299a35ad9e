// The paged cache between two steps: hawk_pages_resize, hawk_pages_fork, hawk_pages_compact (its state: block table, lengths, a count of
// references a page), hawk_pages_copy and hawk_pages_keep (rows of its pages).
//
// The paper has no paged cache; these are the bookkeeping and the copies that the calls around one need between two verify steps.
//
// The state is small (a few hundred KB at most) and every step of the bookkeeping needs the one before it: releases, then the free
// pages, then who gets them.  So resize and compact are ONE launch of one cluster: 8 blocks that share the scan of the counts,
// meet at two cluster barriers (some 0.6 us each; another launch costs 1.5 to 2) and exchange one number a block through
// distributed shared memory.  What a free page is called is found by prefix sums over bit masks in shared memory, not by atomics, so
// results do not depend on the launch.  All of it is bound by latency: a launch, the barriers, and chains of dependent loads (lengths,
// table, counts) of some 0.7 us each.  256 streams that share pages, 131 of which need a copy: 9.9 us in a graph of such calls, 14.8 under
// ncu with cold caches (a thread that handed out the free pages of a word of the bit mask one after the other took 26 where this took 12.7).
// The copies are bound by HBM: 2735 pages of 82 KB (keys and values) in 71 us, 6.3 TB/s read and written, 0.97 of what a plain copy
// reaches.  Fork is one block a stream (one block for small states) with four entries a thread in flight, its counts by atomics without a result (512 streams,
// 239 thousand entries: 6.1 us in a graph, 8.0 under ncu); keep moves rows through registers, eight a thread in flight (128 trees of 64 nodes, 4 layers: 7 us for 26 MB,
// bound by the chain lengths -> table -> rows).
#include <climits>

#include "hawk_common.cuh"

namespace {

using hawk_host::aligned16;
using hawk_host::aligned4;

constexpr int kBookBlocks = 8;       // of the cluster (the largest that every device runs)
constexpr int kBookThreads = 1024;
constexpr int kBookWarps = kBookThreads / 32;
constexpr int kMaxStreams = 4096;    // their prefix sums are held in shared memory
constexpr int kMaxPages = 1 << 20;   // a block's share of them as bit masks too
constexpr int kSlice = kMaxPages / kBookBlocks;
// States up to here go to one block: 2 streams over 28 pages 8.1 us in a cluster, 7.4 in one block; 12 streams over 600 pages packed 12 and 8;
// but 256 streams over 3922 pages 12.7 and 17, 128 over 12300 packed 14 and 28.
constexpr int kSmallPages = 2048, kSmallEntries = 4096;

struct Div {  // number of pages of `keys` keys
    hawk::FastDiv page;
    __device__ __forceinline__ int pages(int keys) const { return static_cast<int>(page.div(static_cast<uint32_t>(keys) + page.d - 1)); }
};

template <typename N>
__device__ __forceinline__ N warp_inclusive(N v)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const N u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += u;
    }
    return v;
}

// Exclusive prefix sum over the block's threads; *total: of all.  `sh` holds kBookWarps numbers.
template <typename N>
__device__ __forceinline__ N block_exclusive(N v, N *sh, N *total)
{
    const N inc = warp_inclusive(v);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();  // (sh may still be read from the sum before)
    if (lane == 31) sh[warp] = inc;
    __syncthreads();
    static_assert(kBookWarps == 32, "a sum a lane");
    const N sums = warp_inclusive(sh[lane]);
    *total = __shfl_sync(0xffffffffu, sums, kBookWarps - 1);
    const N before = __shfl_sync(0xffffffffu, sums, warp > 0 ? warp - 1 : 0);
    return (warp > 0 ? before : N(0)) + inc - v;
}

// Sum over the block's threads.
__device__ __forceinline__ int block_sum(int v, int *sh)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    v = __reduce_add_sync(0xffffffffu, v);
    __syncthreads();  // (sh may still be read from the sum before)
    if (lane == 0) sh[warp] = v;
    __syncthreads();
    return __reduce_add_sync(0xffffffffu, sh[lane]);
}

// Barrier of the cluster (lanes that a branch parted come together first).
template <int kBlocks>
__device__ __forceinline__ void meet()
{
    if (kBlocks == 1) {
        __syncthreads();
    } else {
        __syncwarp();
        hawk::cluster_sync_all();
    }
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
template <int kBlocks>
__device__ __forceinline__ void slice_of(int n_pages, int rank, int &first, int &end)
{
    const int per = ((n_pages + kBlocks - 1) / kBlocks + 127) & ~127;
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

// The blocks' numbers `mine`: how many the blocks before this one have, and all.  A cluster barrier.
template <int kBlocks>
__device__ __forceinline__ void exchange_counts(int mine, int *slot, int rank, int &before, int &total)
{
    before = 0;
    total = mine;
    if (kBlocks == 1) {
        __syncthreads();
        return;
    }
    if (threadIdx.x == 0) *slot = mine;
    meet<kBlocks>();
    total = 0;
#pragma unroll
    for (int r = 0; r < kBlocks; ++r) {
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
    uint32_t bits[kSlice / 32];  // the share's free pages
    int before[kSlice / 32];     // free pages of the share in front of each word
    int end[kMaxStreams];        // running sum of the pages that streams need
    int kv[kMaxStreams], next[kMaxStreams];  // lengths, `next` the old one where the new one is out of range; -1: the old one is
    int last[kMaxStreams];       // the page that a stream grows into, -1: none
    int sums[kBookWarps];
    int slot;
};

// The n-th set bit (from 0) of a word that has it.
__device__ __forceinline__ int nth_bit(uint32_t word, int n)
{
    int at = 0;
#pragma unroll
    for (int half = 16; half; half >>= 1) {
        const int low = __popc((word >> at) & ((1u << half) - 1));
        if (n >= low) {
            n -= low;
            at += half;
        }
    }
    return at;
}

// The first entry of a non-decreasing array that is past r.
__device__ __forceinline__ int first_past(const int *ends, int n, int r)
{
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (ends[mid] > r) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// Everything that the block reads of the state as it was on entry it reads before the first barrier of the cluster, and nobody writes the
// state in place before it (but a block the counts of its own share of the pages).
template <int kBlocks>
__global__ void __launch_bounds__(kBookThreads, 1) resize_kernel(ResizeParams P)
{
    extern __shared__ __align__(16) unsigned char smem_raw[];
    ResizeShared &sh = *reinterpret_cast<ResizeShared *>(smem_raw);
    hawk::allow_dependent_launch();
    hawk::grid_dependency_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = kBlocks == 1 ? 0 : static_cast<int>(hawk::cluster_cta_rank());
    const long long cap = static_cast<long long>(P.W) * P.div.page.d;
    int flags = 0, first, end;
    slice_of<kBlocks>(P.n_pages, rank, first, end);

    // ---- lengths, pages that streams grow into; the share's counts to where they are kept
    if (P.out_refs != P.refs) {
        for (int i = first / 4 + tid; i < end / 4; i += kBookThreads)
            reinterpret_cast<int4 *>(P.out_refs)[i] = reinterpret_cast<const int4 *>(P.refs)[i];
        for (int i = max(first, end & ~3) + tid; i < end; i += kBookThreads) P.out_refs[i] = P.refs[i];
    }
    for (int s = tid; s < P.S; s += kBookThreads) {
        int old = P.kv[s], next = P.next[s];
        const bool held = old >= 0 && old <= cap;
        if (!held || next < 0 || next > cap) {  // the stream stays as it is
            flags |= HAWK_DEV_BAD_PREFIX;
            next = old = held ? old : -1;
        }
        int last = -1;
        if (next > old) {
            uint32_t part;
            const int full = static_cast<int>(P.div.page.divmod(static_cast<uint32_t>(old), part));
            if (part != 0) {
                last = P.table[static_cast<size_t>(s) * P.W + full];
                if (last < 0 || last >= P.n_pages) {
                    flags |= HAWK_DEV_BAD_PAGE;
                    last = -1;
                }
            }
        }
        sh.kv[s] = old;
        sh.next[s] = next;
        sh.last[s] = last;
    }
    __syncthreads();

    // ---- streams that shrink: each block releases what lies in its share (all look through the entries, which is less than a barrier
    // costs unless very many are released); entries that stay, where the table goes elsewhere
    for (int s = warp; s < P.S; s += kBookWarps) {
        const int old = sh.kv[s], next = sh.next[s];
        if (next >= old) continue;
        const int have = P.div.pages(old);
        const size_t row = static_cast<size_t>(s) * P.W;
        for (int j = P.div.pages(next) + lane; j < have; j += 32) {
            const int page = P.table[row + j];
            if (page < 0 || page >= P.n_pages) flags |= HAWK_DEV_BAD_PAGE;
            else if (page >= first && page < end) release(P.out_refs, page, P.n_pages, flags);
        }
    }
    if (P.out_table != P.table) {
        for (int s = rank * kBookWarps + warp; s < P.S; s += kBlocks * kBookWarps) {
            const int old = sh.kv[s];
            if (old < 0) continue;
            const int stay = P.div.pages(min(old, sh.next[s]));
            const size_t row = static_cast<size_t>(s) * P.W;
            for (int j = lane; j < stay; j += 128) {  // (four loads in flight)
                int page[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) page[k] = j + 32 * k < stay ? P.table[row + j + 32 * k] : 0;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (j + 32 * k < stay) P.out_table[row + j + 32 * k] = page[k];
            }
        }
    }
    __syncthreads();

    // ---- the share's free pages
    const int words = (end - first + 31) / 32;
    (void)mark_pages(P.out_refs, first, end, sh.bits, [](int c, int) { return c == 0; });
    __syncthreads();
    const int per = (words + kBookThreads - 1) / kBookThreads, w0 = min(words, tid * per), w1 = min(words, w0 + per);
    int in = 0, mine, free_before, total_free, total_need;
    for (int w = w0; w < w1; ++w) in += __popc(sh.bits[w]);
    int at = block_exclusive(in, sh.sums, &mine);
    for (int w = w0; w < w1; ++w) {
        at += __popc(sh.bits[w]);
        sh.before[w] = at;  // (with the word's own)
    }
    exchange_counts<kBlocks>(mine, &sh.slot, rank, free_before, total_free);

    // ---- what every stream needs: each block for itself
    constexpr int kPer = kMaxStreams / kBookThreads;
    const int streams = (P.S + kBookThreads - 1) / kBookThreads;  // a thread
    int need[kPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int s = tid * streams + i;
        need[i] = 0;
        if (i >= streams || s >= P.S) continue;
        const int old = sh.kv[s], next = sh.next[s];
        if (next <= old) continue;
        need[i] = P.div.pages(next) - P.div.pages(old);
        // A count of 0 contradicts the entry.  (The block whose share the page is in sees it for certain: only that one may hand the page out, behind
        // this loop.)
        const int count = sh.last[s] >= 0 ? __ldcg(P.out_refs + sh.last[s]) : 1;
        if (count <= 0) flags |= HAWK_DEV_BAD_PAGE;
        if (count > 1) ++need[i];
        else sh.last[s] = -1;  // (from here on: the page that is copied)
        sum += need[i];
    }
    int run = block_exclusive(sum, sh.sums, &total_need);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int s = tid * streams + i;
        run += need[i];
        if (i < streams && s < P.S) sh.end[s] = run;
    }
    __syncthreads();

    // ---- the share's free pages to the streams whose turn they are, a page a thread
    for (int i = tid; i < mine && free_before + i < total_need; i += kBookThreads) {
        const int r = free_before + i, word = first_past(sh.before, words, i);
        const int page = first + word * 32 + nth_bit(sh.bits[word], i - (word > 0 ? sh.before[word - 1] : 0));
        const int s = first_past(sh.end, P.S, r);
        if (sh.end[s] > total_free) continue;  // this stream and all behind it stay as they were
        const int old = sh.kv[s], copied = sh.last[s], nth = r - (s > 0 ? sh.end[s - 1] : 0);
        const int j = P.div.pages(old) + nth - (copied >= 0);
        if (!HAWK_IN_BOUNDS(P.dev_status, j, P.W) || !HAWK_IN_BOUNDS(P.dev_status, page, P.n_pages)) continue;
        if (copied >= 0 && nth == 0) {
            uint32_t part;
            P.div.page.divmod(static_cast<uint32_t>(old), part);
            P.copies[3 * s] = copied;
            P.copies[3 * s + 1] = page;
            P.copies[3 * s + 2] = static_cast<int>(part);
        }
        P.out_table[static_cast<size_t>(s) * P.W + j] = page;
        P.out_refs[page] = 1;
    }
    meet<kBlocks>();  // (the counts of shared pages have been looked at by all; nobody's numbers are read any more)
    for (int s = rank * kBookThreads + tid; s < P.S; s += kBlocks * kBookThreads) {
        const int needs = sh.end[s] - (s > 0 ? sh.end[s - 1] : 0);
        const bool served = needs == 0 || sh.end[s] <= total_free;
        if (!served) flags |= HAWK_DEV_NO_PAGES;
        const int copied = sh.next[s] > sh.kv[s] && served ? sh.last[s] : -1;
        if (copied >= 0) {
            release(P.out_refs, copied, P.n_pages, flags);
        } else {
            P.copies[3 * s] = -1;
            P.copies[3 * s + 1] = -1;
            P.copies[3 * s + 2] = 0;
        }
        if (sh.kv[s] >= 0) P.out_len[s] = served ? sh.next[s] : sh.kv[s];
        else if (P.out_len != P.kv) P.out_len[s] = P.kv[s];
    }
    report(P.dev_status, flags);
}

// ---------------------------------------------------------------------------------------------- fork
struct ForkParams {
    const int32_t *table, *kv, *parent, *length, *page_refs;
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

constexpr int kForkThreads = 128;

// `kLanes` threads take one stream's entries, old and new, four a thread in flight: entry j of out stream t is its parent's; the count of a page that t
// named before and names still (a stream that goes on) is not touched at all.  Returns what is to be flagged.
template <int kLanes>
__device__ __forceinline__ int fork_stream(const ForkParams &P, int t, int tid, int32_t *refs)
{
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
    constexpr int kFlight = 4;
    const int most = max(take, held);
    for (int j0 = tid; j0 < most; j0 += kLanes * kFlight) {
        int now[kFlight], was[kFlight];
#pragma unroll
        for (int k = 0; k < kFlight; ++k) {
            const int j = j0 + k * kLanes;
            now[k] = j < take ? P.table[source + j] : 0;
            was[k] = j >= same && j < held ? P.table[row + j] : 0;
        }
#pragma unroll
        for (int k = 0; k < kFlight; ++k) {
            const int j = j0 + k * kLanes;
            if (j < take) {
                P.out_table[row + j] = now[k];
                if (now[k] < 0 || now[k] >= P.n_pages) flags |= HAWK_DEV_BAD_PAGE;
                else if (j >= same) atomicAdd(refs + now[k], 1);
            }
            if (j >= same && j < held) {
                if (was[k] < 0 || was[k] >= P.n_pages) flags |= HAWK_DEV_BAD_PAGE;
                else atomicSub(refs + was[k], 1);
            }
        }
    }
    return flags;
}

__global__ void __launch_bounds__(kForkThreads) fork_kernel(ForkParams P)
{
    hawk::allow_dependent_launch();
    hawk::grid_dependency_wait();
    report(P.dev_status, fork_stream<kForkThreads>(P, blockIdx.x, threadIdx.x, P.refs));
}

// Small states whose counts go to another tensor: one block, a warp a stream, the changes of the counts in shared memory, so that no launch
// ahead has to copy them.  In a graph 2.0 -> 1.7 us for 2 streams over 64 pages and 2.5 -> 2.0 for 16 over 700, launched one by one 4.3 -> 3.1; but
// 2.6 and 3.2 for 16 streams of 256 entries, 2.6 and 3.8 for 64 of 64.  At the bounds, 32 streams of 128 entries: over 64 pages 4.0 -> 2.5 in a graph, over
// 700 3.0 -> 2.6, over 4096 2.7 -> 2.8, and one by one 5.0 -> 3.1 for each.
constexpr int kForkStreams = kBookWarps, kForkWidth = 128, kForkPages = 4 * kBookThreads;

__global__ void __launch_bounds__(kBookThreads) fork_small_kernel(ForkParams P)
{
    __shared__ __align__(16) int32_t changes[kForkPages];
    const int page = 4 * threadIdx.x, warp = threadIdx.x >> 5;  // four pages a thread
    const bool all = page + 3 < P.n_pages;
    hawk::allow_dependent_launch();
    *reinterpret_cast<int4 *>(changes + page) = make_int4(0, 0, 0, 0);
    hawk::grid_dependency_wait();
    int4 refs = make_int4(0, 0, 0, 0);
    if (all) refs = *reinterpret_cast<const int4 *>(P.page_refs + page);
    __syncthreads();
    int flags = 0;
    if (warp < max(P.S, P.S_out)) flags = fork_stream<32>(P, warp, threadIdx.x & 31, changes);
    __syncthreads();
    if (all) {
        const int4 d = *reinterpret_cast<const int4 *>(changes + page);
        *reinterpret_cast<int4 *>(P.refs + page) = make_int4(refs.x + d.x, refs.y + d.y, refs.z + d.z, refs.w + d.w);
    } else {
        for (int p = page; p < P.n_pages; ++p) P.refs[p] = P.page_refs[p] + changes[p];
    }
    report(P.dev_status, flags);
}

// ---------------------------------------------------------------------------------------------- compact
struct CompactParams {
    const int32_t *table, *kv, *refs;
    int32_t *out_table, *out_refs, *copies, *top;
    int32_t *to, *from;   // [lists] the lowest free pages, ascending, and the highest in use, descending
    int32_t *place;       // [n_pages] place in the lists of the pages that may move
    int32_t *counts;      // [kBookBlocks] pages in use of each share that lie behind where the pages in use would end
    int S, W, n_pages, first_page, moves;
    Div div;
    hawk::FastDiv div_runs;  // runs of 128 entries a stream
    int32_t *dev_status;
};

struct CompactShared {
    uint32_t used[kSlice / 32];
    int sums[kBookWarps];
    uint32_t packed[kBookWarps];
    int slot_used, slot_free;
};

// Packed, the pages in use end at `border`: those behind it have to move, and as many free ones lie in front of it.  Both lists are made
// by rank; then every block knows all it needs, and the moves and the new ids are written without another barrier.
template <int kBlocks>
__global__ void __launch_bounds__(kBookThreads, 1) compact_kernel(CompactParams P)
{
    extern __shared__ __align__(16) unsigned char smem_raw[];
    CompactShared &sh = *reinterpret_cast<CompactShared *>(smem_raw);
    hawk::allow_dependent_launch();
    hawk::grid_dependency_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = kBlocks == 1 ? 0 : static_cast<int>(hawk::cluster_cta_rank());
    const long long cap = static_cast<long long>(P.W) * P.div.page.d;
    int flags = 0, first, end;
    slice_of<kBlocks>(P.n_pages, rank, first, end);
    if (P.out_refs != P.refs) {
        for (int i = first / 4 + tid; i < end / 4; i += kBookThreads)
            reinterpret_cast<int4 *>(P.out_refs)[i] = reinterpret_cast<const int4 *>(P.refs)[i];
        for (int i = max(first, end & ~3) + tid; i < end; i += kBookThreads) P.out_refs[i] = P.refs[i];
    }
    const int words = (end - first + 31) / 32;
    const int from_page = P.first_page;
    const int count = mark_pages(P.refs, first, end, sh.used, [=](int c, int p) { return c != 0 && p >= from_page; });
    int mine = count, used_before, used, free_before, free_all;
    mine = block_sum(mine, sh.sums);
    const int eligible = max(0, end - max(first, from_page));
    if (tid == 0) sh.slot_free = eligible - mine;
    exchange_counts<kBlocks>(mine, &sh.slot_used, rank, used_before, used);
    free_before = 0;
    free_all = eligible - mine;
    if (kBlocks > 1) {
        free_all = 0;
#pragma unroll
        for (int r = 0; r < kBlocks; ++r) {
            const int n = static_cast<int>(hawk::ld_cluster_u32(hawk::map_shared_to_cta(&sh.slot_free, r)));
            if (r < rank) free_before += n;
            free_all += n;
        }
    }

    // ---- the lowest free pages and the highest in use, by rank; a word a thread
    const int border = from_page + used, lists = P.moves + 1;
    int behind = 0, u = 0, f = 0;
    for (int w0 = 0; w0 < words; w0 += kBookThreads) {
        const int w = w0 + tid, p = first + w * 32;
        uint32_t in = 0, open = 0;
        if (w < words) {
            in = sh.used[w];
            open = ~in;  // of the share, from first_page on
            if (end - p < 32) open &= (1u << (end - p)) - 1;
            if (from_page > p) open &= from_page - p >= 32 ? 0u : ~((1u << (from_page - p)) - 1);
        }
        uint32_t both;  // of kBookThreads words: 2^15 pages at most, so that the two numbers fit one
        const uint32_t at = block_exclusive(static_cast<uint32_t>(__popc(in)) << 16 | __popc(open), sh.packed, &both);
        int i_u = used_before + u + static_cast<int>(at >> 16), i_f = free_before + f + static_cast<int>(at & 0xffff);
        u += static_cast<int>(both >> 16);
        f += static_cast<int>(both & 0xffff);
        for (uint32_t m = in; m; m &= m - 1, ++i_u) {
            const int page = p + __ffs(m) - 1, i = used - 1 - i_u;  // rank from the top
            behind += page >= border;
            if (i < lists && HAWK_IN_BOUNDS(P.dev_status, i, lists)) {
                P.from[i] = page;
                P.place[page] = i;
            }
        }
        for (uint32_t m = i_f < lists && p < border ? open : 0u; m; m &= m - 1, ++i_f)
            if (i_f < lists && HAWK_IN_BOUNDS(P.dev_status, i_f, lists)) P.to[i_f] = p + __ffs(m) - 1;
    }
    behind = block_sum(behind, sh.sums);
    if (kBlocks > 1 && tid == 0) P.counts[rank] = behind;
    meet<kBlocks>();
    int moved = kBlocks > 1 ? 0 : behind;
    if (kBlocks > 1) {
#pragma unroll
        for (int r = 0; r < kBlocks; ++r) moved += __ldcg(P.counts + r);
    }
    const int all_moves = moved;
    moved = min(moved, P.moves);

    // ---- moves
    for (int i = rank * kBookThreads + tid; i < P.moves; i += kBlocks * kBookThreads) {
        int a = -1, b = -1;
        if (i < moved) {
            a = __ldcg(P.from + i);
            b = __ldcg(P.to + i);
            P.out_refs[b] = P.refs[a];
            P.out_refs[a] = 0;
        }
        P.copies[3 * i] = a;
        P.copies[3 * i + 1] = b;
        P.copies[3 * i + 2] = a < 0 ? 0 : static_cast<int>(P.div.page.d);
    }
    if (P.top && rank == 0 && tid == 0) *P.top = moved == all_moves ? border : __ldcg(P.from + moved) + 1;

    // ---- the new ids into the table: runs of 128 entries a warp (in place with nothing to move too, for what is to be flagged)
    const int lowest = moved > 0 ? __ldcg(P.from + moved - 1) : INT_MAX;  // pages in use from here on move
    const int runs = P.S * static_cast<int>(P.div_runs.d);
    for (int t = rank * kBookWarps + warp; t < runs; t += kBlocks * kBookWarps) {
        uint32_t part;
        const int s = static_cast<int>(P.div_runs.divmod(static_cast<uint32_t>(t), part)), j0 = static_cast<int>(part) * 128 + lane;
        const int kv = P.kv[s];
        if (kv < 0 || kv > cap) {
            flags |= HAWK_DEV_BAD_PREFIX;
            continue;
        }
        const int n = P.div.pages(kv);
        const size_t row = static_cast<size_t>(s) * P.W;
        int page[4], i[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) page[k] = j0 + 32 * k < n ? P.table[row + j0 + 32 * k] : 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            i[k] = -1;
            if (page[k] < 0 || page[k] >= P.n_pages) flags |= HAWK_DEV_BAD_PAGE;
            else if (page[k] >= lowest) i[k] = __ldcg(P.place + page[k]);  // (a guess, for a page that the counts say is free)
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (j0 + 32 * k >= n) continue;
            if (page[k] >= lowest && page[k] < P.n_pages) {
                if (i[k] >= 0 && i[k] < moved && __ldcg(P.from + i[k]) == page[k]) page[k] = __ldcg(P.to + i[k]);
                else flags |= HAWK_DEV_BAD_PAGE;
            }
            P.out_table[row + j0 + 32 * k] = page[k];
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
constexpr int kCopyPieces = kCopyThreads * kCopyUnroll;  // of a block, 32 KB, or twice as many in calls of many blocks

// Block (x, y, z): entry x; keys or values of layer y / 2; z: which `share` pieces of the page.  Pieces are taken in the order of memory.
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(PageParams P, const int32_t *copies, uint32_t share)
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
    const uint32_t last = min(all, (blockIdx.z + 1) * share);
    for (uint32_t c0 = blockIdx.z * share + threadIdx.x; c0 < last; c0 += kCopyThreads * kCopyUnroll) {
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
bool allow_smem(K *kernel, size_t bytes, unsigned long long &seen)
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    const unsigned long long bit = 1ull << (dev & 63);
    if (__atomic_load_n(&seen, __ATOMIC_ACQUIRE) & bit && dev < 64) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes)) != cudaSuccess) return false;
    __atomic_fetch_or(&seen, bit, __ATOMIC_RELEASE);
    return true;
}

// The bookkeeping kernels: a cluster, or one block for small states, which then needs no barrier of a cluster.
template <class P>
hawk_status launch_book(void (*many)(P), void (*one)(P), unsigned long long &seen, unsigned long long &seen_one, size_t smem, const P &p,
                        cudaStream_t st)
{
    const bool small = p.n_pages <= kSmallPages && static_cast<long long>(p.S) * p.W <= kSmallEntries;
    if (small) {
        if (!allow_smem(one, smem, seen_one)) return HAWK_ERR_CUDA;
        return done(hawk_host::launch_dependent(one, dim3(1), dim3(kBookThreads), smem, st, p));
    }
    if (!allow_smem(many, smem, seen)) return HAWK_ERR_CUDA;
    return done(hawk_host::launch_dependent_clusters(many, kBookBlocks, dim3(kBookBlocks), dim3(kBookThreads), smem, st, p));
}

hawk_status check_pages(const hawk_page_tensors &p)
{
    if (p.layers < 0 || p.n_pages < 0 || p.H_kv < 0 || p.page_size < 0 || p.D < 0) return HAWK_ERR_SHAPE;
    if (p.H_kv < 1 || p.page_size < 1 || p.D < 1 || p.n_pages < 1) return HAWK_ERR_SHAPE;
    if (p.D % 8 != 0 || p.D > 65536 || p.page_size > 65536 || p.layers > 32767) return HAWK_ERR_UNSUPPORTED;
    if (p.H_kv > 65536 || static_cast<long long>(p.H_kv) * p.page_size > (1ll << 30) / p.D) return HAWK_ERR_UNSUPPORTED;
    if (p.layers > 0 && (!p.k_pages || !p.v_pages)) return HAWK_ERR_NULL;
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
    if (a->S > 0 && (!a->kv_len || !a->new_len || !a->out_len || !a->copies)) return HAWK_ERR_NULL;
    if (a->S > 0 && a->table_width > 0 && (!a->block_table || !a->out_table)) return HAWK_ERR_NULL;
    if (a->n_pages > 0 && (!a->page_refs || !a->out_refs)) return HAWK_ERR_NULL;
    if (!aligned16(a->page_refs) || !aligned16(a->out_refs)) return HAWK_ERR_ALIGN;
    if (!aligned4(a->block_table, a->kv_len, a->new_len, a->out_table, a->out_len, a->copies)) return HAWK_ERR_ALIGN;
    if (!hawk_host::is_sm100(nullptr)) return HAWK_ERR_UNSUPPORTED;
    ResizeParams P = {a->block_table, a->kv_len, a->new_len, a->page_refs, a->out_table, a->out_len, a->out_refs, a->copies,
                      a->S, a->table_width, a->n_pages, make_div(a->page_size), dev_status};
    static unsigned long long seen = 0, seen_one = 0;
    return launch_book(resize_kernel<kBookBlocks>, resize_kernel<1>, seen, seen_one, sizeof(ResizeShared), P,
                       reinterpret_cast<cudaStream_t>(stream));
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
    const bool wide = a->table_width > 0;
    if (a->S > 0 && ((wide && !a->block_table) || !a->kv_len)) return HAWK_ERR_NULL;
    if (a->S_out > 0 && (!a->parent || (wide && !a->out_table) || !a->out_len)) return HAWK_ERR_NULL;
    if (a->n_pages > 0 && (!a->page_refs || !a->out_refs)) return HAWK_ERR_NULL;
    if (!aligned16(a->page_refs) || !aligned16(a->out_refs)) return HAWK_ERR_ALIGN;
    if (!aligned4(a->block_table, a->kv_len, a->parent, a->length, a->out_table, a->out_len)) return HAWK_ERR_ALIGN;
    if ((a->S_out > 0 && a->S > 0) && ((wide && a->out_table == a->block_table) || a->out_len == a->kv_len)) return HAWK_ERR_PARAM;
    if (!hawk_host::is_sm100(nullptr)) return HAWK_ERR_UNSUPPORTED;
    const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const int streams = a->S > a->S_out ? a->S : a->S_out;
    ForkParams P = {a->block_table, a->kv_len, a->parent, a->length, a->page_refs, a->out_table, a->out_len, a->out_refs,
                    a->S, a->S_out, a->table_width, a->n_pages, make_div(a->page_size), dev_status};
    if (move && streams > 0 && streams <= kForkStreams && a->table_width <= kForkWidth && a->n_pages <= kForkPages)
        return done(hawk_host::launch_dependent(fork_small_kernel, dim3(1), dim3(kBookThreads), 0, st, P));
    if (move) {
        const int per = 256 * 4;
        const cudaError_t e = hawk_host::launch_dependent(copy_ints_kernel, dim3((a->n_pages + per - 1) / per), dim3(256), 0, st,
                                                          a->page_refs, a->out_refs, a->n_pages);
        if (e != cudaSuccess) return HAWK_ERR_CUDA;
    }
    if (streams == 0) return HAWK_OK;
    return done(hawk_host::launch_dependent(fork_kernel, dim3(streams), dim3(kForkThreads), 0, st, P));
}

extern "C" size_t hawk_pages_compact_workspace_bytes(int n_pages, int max_moves)
{
    if (n_pages < 1 || n_pages > kMaxPages || max_moves < 0) return 0;
    const size_t moves = max_moves < n_pages ? max_moves : n_pages;
    return sizeof(int32_t) * (static_cast<size_t>(n_pages) + 2 * (moves + 1) + kBookBlocks);
}

extern "C" hawk_status hawk_pages_compact(const hawk_pages_compact_args *a, int32_t *dev_status, hawk_stream_t stream)
{
    const hawk_host::NvtxRange nvtx_range("hawk_pages_compact");
    if (!a) return HAWK_ERR_NULL;
    const hawk_status chk = check_state(a->S, a->table_width, a->n_pages, a->page_size);
    if (chk != HAWK_OK) return chk;
    if (a->n_pages < 1 || a->first_page < 0 || a->first_page > a->n_pages || a->max_moves < 0) return HAWK_ERR_SHAPE;
    if (a->max_moves > kMaxPages) return HAWK_ERR_UNSUPPORTED;
    if (a->S > 0 && (!a->kv_len || (a->table_width > 0 && (!a->block_table || !a->out_table)))) return HAWK_ERR_NULL;
    if (!a->page_refs || !a->out_refs) return HAWK_ERR_NULL;
    if (a->max_moves > 0 && !a->copies) return HAWK_ERR_NULL;
    if (!aligned16(a->page_refs) || !aligned16(a->out_refs) || !aligned16(a->workspace)) return HAWK_ERR_ALIGN;
    if (!aligned4(a->block_table, a->kv_len, a->out_table, a->copies, a->top)) return HAWK_ERR_ALIGN;
    if (!a->workspace || a->workspace_bytes < hawk_pages_compact_workspace_bytes(a->n_pages, a->max_moves))
        return HAWK_ERR_WORKSPACE;
    if (!hawk_host::is_sm100(nullptr)) return HAWK_ERR_UNSUPPORTED;
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
    P.counts = P.place + a->n_pages;
    P.div_runs.set(static_cast<uint32_t>(a->table_width > 128 ? (a->table_width + 127) / 128 : 1));
    P.S = a->S;
    P.W = a->table_width;
    P.n_pages = a->n_pages;
    P.first_page = a->first_page;
    P.moves = a->max_moves;
    P.div = make_div(a->page_size);
    P.dev_status = dev_status;
    static unsigned long long seen = 0, seen_one = 0;
    return launch_book(compact_kernel<kBookBlocks>, compact_kernel<1>, seen, seen_one, sizeof(CompactShared), P,
                       reinterpret_cast<cudaStream_t>(stream));
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
    if (!aligned4(copies)) return HAWK_ERR_ALIGN;
    if (!hawk_host::is_sm100(nullptr)) return HAWK_ERR_UNSUPPORTED;
    const PageParams P = page_params(*pages, dev_status);
    const long long all = static_cast<long long>(P.H) * P.page_size * P.pieces;
    // 2735 pages of 40 KB: 72 us with a page in two blocks, 68 in one; 16 pages of 98 KB: 5.2 us in twice as many blocks, 6.0 else.  A grid has
    // 65535 blocks along z at most: the largest pages (2^27 pieces) take the larger share in any call.
    const bool many = static_cast<long long>(n_copies) * 2 * pages->layers >= 4 * 148 || all > 65535ll * kCopyPieces;
    const long long share = many ? 2 * kCopyPieces : kCopyPieces;
    const dim3 grid(n_copies, 2 * pages->layers, static_cast<unsigned>((all + share - 1) / share));
    return done(hawk_host::launch_dependent(copy_kernel, grid, dim3(kCopyThreads), 0, reinterpret_cast<cudaStream_t>(stream), P, copies,
                                            static_cast<uint32_t>(share)));
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
    if (!aligned4(a->row_begin, a->kv_len, a->accept_len, a->path, a->out_len)) return HAWK_ERR_ALIGN;
    KeepParams P = {};
    int layers = 1;
    if (a->path) {
        const hawk_status chk = check_pages(a->pages);
        if (chk != HAWK_OK) return chk;
        if (a->table_width > 0 && !a->block_table) return HAWK_ERR_NULL;
        if (!aligned4(a->block_table)) return HAWK_ERR_ALIGN;
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
