// What the two kernels behind hawk_paged_attn share: the call's parameters, the view of one stream of the ragged batch,
// the 16-bit element types, and the launchers.
#pragma once

#include <math_constants.h>

#include "hawk_common.cuh"

namespace hawk {

// One launch of either kernel.
struct PagedParams {
    const void *q;
    void *out;
    const int32_t *row_begin, *kv_len, *block_table;
    const uint64_t *anc_mask;  // [max_new] or NULL
    float *part;               // partial results (layout: see each kernel)
    int32_t *records;          // rows kernel: one record of kRecordInts per worker
    long long q_row_stride, q_head_stride;
    int S, T, max_new, H, H_kv, group;
    int n_pages, page_size, table_width;
    int kv_cap;                // largest admissible kv_len
    int rows_few;              // a stream of at most this many rows per kv head goes to the rows kernel, others to the tile kernel
    int box_rows;              // cache rows of one TMA box: a divisor of the page size and of the tile
    int k_rows_inner, v_rows_inner;  // tensor maps are {D, rows, heads, pages} (1) or {D, heads, rows, pages} (0): the
                                     // dimension with the smaller stride comes first
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

__device__ __forceinline__ bool paged_is_few(const PagedParams &P, const PagedStream &st)
{
    return static_cast<long long>(st.n) * P.group <= P.rows_few;
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

// The chunk kernel (tcgen05 tiles of query rows): bytes of its partial results, and its launch.
size_t paged_tile_workspace_bytes(int S, int T, int max_new, int H, int H_kv, int few, int D, int max_kv);
cudaError_t launch_paged_tile(const hawk_paged_attn_args &a, const hawk::PagedParams &base, float *part, cudaStream_t st,
                              bool *refused);

}  // namespace hawk_host
