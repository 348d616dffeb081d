// The matrix products of a decoding step from pages for fp32 layers, for widths that the stack engine's matrix-core products do not cover (d
// or d_hidden no multiple of 256), and for the batches in which they are the faster ones (paged_products_take): out[b][o] = epilogue(sum_k W[o][k] in[b][k]), every row of the batch in one launch.
#include "rt_base_case.h"
#include "rt_paged.h"
#include "rt_ll.h"

namespace rt {

// Products of 16 outputs, 16 batch rows and 32 indices: lane (i = lane % 16, g = lane / 16) holds indices 8 g .. + 7 of row i of either side.
// bf16 weights: one instruction of 16 x 16 x 32 for the inputs' heads (rounded to bf16) and one for their remainders, which leaves 2^-17
// of an input.  fp32: eight of 16 x 16 x 4 in fp32, instruction j taking the lanes' element j.
typedef float f32x2_t __attribute__((ext_vector_type(2)));
template <typename T> struct Side;
template <> struct Side<bf16_t> {
    Frag w;
    __device__ __forceinline__ void load(const bf16_t *p, bool in) { w.u = in ? *reinterpret_cast<const uint4 *>(p) : make_uint4(0u, 0u, 0u, 0u); }
};
template <> struct Side<float> {
    float w[8];
    __device__ __forceinline__ void load(const float *p, bool in)
    {
        load8(p, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = in ? w[e] : 0.f;
    }
};
template <typename T> struct Input;
template <> struct Input<bf16_t> {
    Frag hi, lo;
    __device__ __forceinline__ void set(const float (&v)[8])
    {
        uint32_t h[4], r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const f32x2_t a = {v[2 * e], v[2 * e + 1]};
            h[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(a, bf16x2_t));
            const f32x2_t b = {v[2 * e] - __uint_as_float(h[e] << 16), v[2 * e + 1] - __uint_as_float(h[e] & 0xFFFF0000u)};
            r[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(b, bf16x2_t));
        }
        hi.u = make_uint4(h[0], h[1], h[2], h[3]);
        lo.u = make_uint4(r[0], r[1], r[2], r[3]);
    }
    __device__ __forceinline__ f32x4_t product(const Side<bf16_t> &s, f32x4_t acc) const { return mfma16(s.w, hi, mfma16(s.w, lo, acc)); }
};
template <> struct Input<float> {
    float x[8];
    __device__ __forceinline__ void set(const float (&v)[8])
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = v[e];
    }
    __device__ __forceinline__ f32x4_t product(const Side<float> &s, f32x4_t acc) const
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(s.w[e], x[e], acc, 0, 0, 0);
        return acc;
    }
};

// A workgroup owns 16 NO outputs of 16 batch rows; its eight wavefronts take every eighth block of 32 indices, their sums meet in LDS and
// are added in wavefront order.  An input row's elements are split once per workgroup (NO tiles share them), and with do_norm their squares
// are summed on the way: 1 / rms scales the finished sums, the gain multiplies the elements.
// Bound: for few rows the dependent trips to memory, hence 16 outputs per workgroup (NO = 1) where 64 would leave compute units idle.
// Rows past n_first and 2 n_first come from Wb and Wc (n_first a multiple of 16).  grid (ceil(n_out / (16 NO)), ceil(B / 16)), block 512.
template <typename T, typename IN_T, int EPI, int NO>
__global__ __launch_bounds__(512) void paged_product_kernel(const T *__restrict__ Wa, const T *__restrict__ Wb, const T *__restrict__ Wc,
                                                            int n_first, int n_out, int K, const IN_T *__restrict__ in, int B,
                                                            const T *__restrict__ gain, float eps, int do_norm, float alpha,
                                                            const T *__restrict__ res_T, const float *__restrict__ res_f,
                                                            float *__restrict__ out_f, T *__restrict__ out_T)
{
    __shared__ f32x4_t part[8][NO][64];
    __shared__ float ssq[8][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4;
    const int row0 = blockIdx.x * 16 * NO, b = min((int)blockIdx.y * 16 + i, B - 1);   // rows past the batch repeat its last one (dropped)
    const T *w[NO];
#pragma unroll
    for (int t = 0; t < NO; ++t) {
        const int o0 = min(row0 + 16 * t, (n_out - 1) / 16 * 16), which = o0 / n_first;
        const T *m = Wa;
        if (which == 1) m = Wb;
        if (which == 2) m = Wc;
        w[t] = m + (size_t)(min(o0 + i, n_out - 1) - which * n_first) * K;
    }
    const IN_T *x = in + (size_t)b * K;
    f32x4_t acc[NO];
#pragma unroll
    for (int t = 0; t < NO; ++t) acc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float ss = 0.f;
    const bool use_gain = do_norm && gain;
    // two blocks at a time, both requested before the first is used; the second may lie past the end (zeros).  Rows lie a power of two of
    // bytes apart more often than not, so that the same block of all rows is behind one channel of the cache: every workgroup starts at
    // another block (d = 1024, 16 rows: 50.7 -> 48.8 us for the whole step)
    const int nblk = (K + 31) / 32, turn = (int)((blockIdx.x * 4 + blockIdx.y * 2) % (unsigned)nblk);
    for (int j0 = wave; j0 < nblk; j0 += 2 * 8) {
        Side<T> s[2][NO];
        float v[2][8], gn[2][8];
        bool inside[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int j = j0 + 8 * u, at = j + turn < nblk ? j + turn : j + turn - nblk;
            inside[u] = j < nblk && 32 * at + 8 * g < K;   // K is a multiple of eight
            const int k = inside[u] ? 32 * at + 8 * g : 0;
#pragma unroll
            for (int t = 0; t < NO; ++t) s[u][t].load(w[t] + k, inside[u]);
            load8(x + k, v[u]);
            if (use_gain) load8(gain + k, gn[u]);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[u][e] = inside[u] ? v[u][e] : 0.f;
                if (do_norm) ss = fmaf(v[u][e], v[u][e], ss);
                if (use_gain) v[u][e] *= gn[u][e];
            }
            Input<T> f;
            f.set(v[u]);
#pragma unroll
            for (int t = 0; t < NO; ++t) acc[t] = f.product(s[u][t], acc[t]);
        }
    }
    if (do_norm) {
        ss += xor16(ss);
        ss += xor32(ss);
        if (g == 0) ssq[wave][i] = ss;
    }
#pragma unroll
    for (int t = 0; t < NO; ++t) part[wave][t][lane] = acc[t];
    __syncthreads();
    if (wave >= NO) return;
    const int o = row0 + 16 * wave + 4 * g;
    f32x4_t sum = part[0][wave][lane];
#pragma unroll
    for (int p = 1; p < 8; ++p) sum += part[p][wave][lane];
    float v[4] = {sum[0], sum[1], sum[2], sum[3]};
    if (do_norm) {
        float tot = 0.f;
#pragma unroll
        for (int p = 0; p < 8; ++p) tot += ssq[p][i];
        const float rinv = rsqrtf(tot / (float)K + eps);
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] *= rinv;
    }
    if (o >= n_out || (int)blockIdx.y * 16 + i >= B) return;
    const size_t at = (size_t)b * n_out + o;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (EPI == EPI_WO) v[r] = to_f32(res_T[at + r]) + alpha * v[r];
        if (EPI == EPI_W1) v[r] = gelu_erf(v[r]);
        if (EPI == EPI_W2) v[r] = res_f[at + r] + alpha * v[r];
    }
    *reinterpret_cast<float4 *>(out_f + at) = make_float4(v[0], v[1], v[2], v[3]);
    if (EPI == EPI_W2) {
#pragma unroll
        for (int r = 0; r < 4; ++r) out_T[at + r] = from_f32_any<T>(v[r]);
    }
}

template <typename T, typename IN_T, int EPI>
static void product(const void *Wa, const void *Wb, const void *Wc, int n_first, int n_out, int K, const IN_T *in, const LayerDims &D, const void *gain,
                    int do_norm, const void *res_T, const float *res_f, float *out_f, void *out_T, hipStream_t st)
{
    const int cols = (D.B + 15) / 16;
#define RT_PRODUCT(NO)                                                                                                                      \
    hipLaunchKernelGGL((paged_product_kernel<T, IN_T, EPI, NO>), dim3((n_out + 16 * NO - 1) / (16 * NO), cols), dim3(512), 0, st, (const T *)Wa, \
                       (const T *)Wb, (const T *)Wc, n_first, n_out, K, in, D.B, (const T *)gain, D.eps, do_norm, D.alpha, (const T *)res_T, \
                       res_f, out_f, (T *)out_T)
    if (paged_product_tiles(n_out, D.B) == 4) RT_PRODUCT(4);
    else RT_PRODUCT(1);
#undef RT_PRODUCT
}

// raw [q | k_tmp | v_tmp] of x_t [B][d] into S.qkv_raw
template <typename T> hipError_t paged_qkv_launch(const LayerDims &D, const Weights &W, const Scratch &S, const void *x_t, hipStream_t st)
{
    product<T, T, EPI_KV>(W.Wq, W.Wk, W.Wv, D.d, 3 * D.d, D.d, (const T *)x_t, D, W.g_attn, !D.norm_free, nullptr, nullptr, S.qkv_raw, nullptr, st);
    return hipGetLastError();
}
// from the attention output S.attn_cat: h, the MLP, y_new [B][d] and the raw pair S.kv_raw
template <typename T>
hipError_t paged_base_case_launch(const LayerDims &D, const Weights &W, const Scratch &S, const void *x_t, void *y_new, hipStream_t st)
{
    const int d = D.d, F = D.F, norm = !D.norm_free;
    product<T, float, EPI_WO>(W.Wo, W.Wo, W.Wo, d, d, d, S.attn_cat, D, nullptr, 0, x_t, nullptr, S.h, nullptr, st);
    product<T, float, EPI_W1>(W.W1, W.W1, W.W1, F, F, d, S.h, D, W.g_mlp, norm, nullptr, nullptr, S.u, nullptr, st);
    product<T, float, EPI_W2>(W.W2, W.W2, W.W2, d, d, F, S.u, D, nullptr, 0, nullptr, S.h, S.z, y_new, st);
    product<T, float, EPI_KV>(W.Wk, W.Wv, W.Wv, d, 2 * d, d, S.z, D, W.g_kv, norm, nullptr, nullptr, S.kv_raw, nullptr, st);
    return hipGetLastError();
}
#define RT_PRODUCTS_FOR(T)                                                                                                              \
    template hipError_t paged_qkv_launch<T>(const LayerDims &, const Weights &, const Scratch &, const void *, hipStream_t);             \
    template hipError_t paged_base_case_launch<T>(const LayerDims &, const Weights &, const Scratch &, const void *, void *, hipStream_t);
RT_PRODUCTS_FOR(float)
RT_PRODUCTS_FOR(bf16_t)
#undef RT_PRODUCTS_FOR

}  // namespace rt
