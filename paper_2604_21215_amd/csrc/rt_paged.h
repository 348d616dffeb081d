// Internal interface of the paged-cache kernels (rt_paged.hip).
#pragma once
#include "rt_common.h"
#include "rt_paged_index.h"

namespace rt {

// Rows of cached pairs on the caller's side: row (s, n) starts s * seq_stride + n * pos_stride elements behind the pointer, heads contiguous.
struct PairRows {
    const int32_t *first, *count;   // [S]: first position (negative: idle), rows (null: all N)
    int S, N;
    long long seq_stride, pos_stride;
};

// One new token per sequence against its cached rows.
struct PagedAttention {
    int S, H, max_len;
    const int32_t *lens;
    float scale, alibi;
    // query and pair: storage dtype rows (stand-alone call) ...
    const void *q, *kt, *vt;
    long long q_stride, kv_stride, out_stride;
    void *out;
    float *lse;
    // ... or [S][3 d] fp32 raw or finished [q | k_tmp | v_tmp] (the layer's step), with the outputs the base case reads
    const float *qkv;
    const void *g_q, *g_k;
    int normalise;            // qkRMS of q and k_tmp is still to be taken
    float eps;
    float *attn_cat;
    bf16_t *op_a;             // or null
    int op_fragments;
    // partial states [S][H][n_splits]
    float *pm, *pl, *po;
    SplitPlan plan;
};

template <typename T> hipError_t cache_write_launch(const PagedCache &C, const PairRows &R, int H, const void *k, const void *v, hipStream_t st);
template <typename T> hipError_t cache_read_launch(const PagedCache &C, const PairRows &R, int H, void *k, void *v, hipStream_t st);
size_t paged_partials_bytes();
void paged_partials(PagedAttention &A, void *slab);
template <typename T> hipError_t paged_attention_launch(const PagedCache &C, const PagedAttention &A, hipStream_t st);
// The last part of a paged step on the plain-ALU products: the pairs of fp32 rows kv [S][2 d] (raw) into their pages and the rows of y_new
// into y, for sequences that are not idle.
template <typename T>
hipError_t paged_finish_launch(const PagedCache &C, const LayerDims &D, const int32_t *pos, int max_pos, const float *kv, const void *g_k,
                               const void *y_new, void *y, hipStream_t st);
// The products of a step for the widths and types that step_mm_supported leaves out, and for batches they take (rt_paged_products.hip).
template <typename T> hipError_t paged_qkv_launch(const LayerDims &D, const Weights &W, const Scratch &S, const void *x_t, hipStream_t st);
template <typename T>
hipError_t paged_base_case_launch(const LayerDims &D, const Weights &W, const Scratch &S, const void *x_t, void *y_new, hipStream_t st);

}  // namespace rt
