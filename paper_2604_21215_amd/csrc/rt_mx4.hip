// The read-out of a stack with 4-bit weights: blocks of 32 weights of a row share a scale 2^e, a weight is a sign and one of
// 0, 1/2, 1, 3/2, 2, 3, 4, 6 (the MX format with 4-bit elements, E2M1 codes and E8M0 scales): 17 bytes for 32 weights.
#include "rt_mx4.h"
#include "rt_mfma_device.h"

#include <cmath>

namespace rt {

// ---------------------------------------------------------------- packing (host)
static uint8_t e2m1_code(double u)   // nearest, ties to the even code
{
    const double a = std::fabs(u);
    int c;
    if (a <= 0.25) c = 0;
    else if (a < 0.75) c = 1;
    else if (a <= 1.25) c = 2;
    else if (a < 1.75) c = 3;
    else if (a <= 2.5) c = 4;
    else if (a < 3.5) c = 5;
    else if (a <= 5.0) c = 6;
    else c = 7;
    return (uint8_t)(c | (u < 0 && c ? 8 : 0));
}
static double e2m1_value(uint8_t c)
{
    static const double v[8] = {0, 0.5, 1, 1.5, 2, 3, 4, 6};
    return c & 8 ? -v[c & 7] : v[c & 7];
}

bool mx4_pack_host(const void *W, bool bf16, long long rows, int cols, uint8_t *codes, uint8_t *exps)
{
    auto weight = [&](long long i) -> float {
        if (!bf16) return ((const float *)W)[i];
        const uint32_t u = (uint32_t)((const uint16_t *)W)[i] << 16;
        float f;
        memcpy(&f, &u, 4);
        return f;
    };
    for (long long i = 0; i < rows * cols; ++i)
        if (!std::isfinite(weight(i))) return false;
    for (long long b = 0; b < rows * (cols / kMx4Block); ++b) {
        double w[kMx4Block], top = 0;
        for (int i = 0; i < kMx4Block; ++i) {
            w[i] = weight(b * kMx4Block + i);
            top = std::fmax(top, std::fabs(w[i]));
        }
        int e = 0;
        if (top > 0) {
            // the smallest scale that reaches the largest weight, or one below (which cuts it to 6): the smaller squared error
            (void)std::frexp(top / 6.0, &e);
            if (std::ldexp(6.0, e - 1) >= top) --e;
            if (e < -126) e = -126;
            double err[2] = {0, 0};
            for (int t = 0; t < 2; ++t)
                for (int i = 0; i < kMx4Block; ++i) {
                    const double u = std::ldexp(w[i], t - e), r = u - e2m1_value(e2m1_code(u));
                    err[t] += std::ldexp(r * r, -2 * t);
                }
            if (e > -126 && err[1] < err[0]) --e;
        }
        exps[b] = (uint8_t)(e + 127);
        for (int i = 0; i < kMx4Block; i += 2)
            codes[b * (kMx4Block / 2) + i / 2] =
                (uint8_t)(e2m1_code(std::ldexp(w[i], -e)) | (e2m1_code(std::ldexp(w[i + 1], -e)) << 4));
    }
    return true;
}

// ---------------------------------------------------------------- logits (device)
// logits[b][v] = sum_k W[v][k] n_b[k], n_b = g z_b / rms(z_b): D[16 vocabulary rows][16 batch columns] += W[16][32] n^T[32][16].
// The weights are exact in bf16 (two bits and a power of two) and one instruction turns two codes into two bf16 with their scale; the rows
// n_b are staged as three bf16 parts whose sum holds all 24 bits, so the logits carry fp32 accuracy: every weight fragment feeds three
// matrix instructions.  A lane holds one whole block of a row: its 16 bytes of codes are four fragments, and the contraction index is dealt
// so that slot 8 g + e of instruction j is k = 32 (4 step + g) + 8 j + e for lane group g.
// grid (<= row tiles / 4, batch tiles of bt), block 256, LDS 3 bt ld bf16.
typedef __bf16 bf16x2v_t __attribute__((ext_vector_type(2)));
constexpr size_t kMxMaxLds = 152 * 1024;

__host__ __device__ static inline int mx_ld(int d) { return (d + 127) / 128 * 128 + 8; }   // a row's elements in LDS
static_assert(3 * ((kMx4MaxWidth + 127) / 128 * 128 + 8) * 2 <= kMxMaxLds, "the widest row");

template <int BYTE> __device__ __forceinline__ uint32_t two_weights(uint32_t codes, float scale)
{
    const bf16x2v_t r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, BYTE);
    return __builtin_bit_cast(uint32_t, r);
}

template <typename T>
__global__ __launch_bounds__(256) void mx4_head_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ exps,
                                                       const T *__restrict__ gain, const T *__restrict__ z, long long z_stride,
                                                       float *__restrict__ logits, int B, int d, int vocab, float eps, int norm_free, int bt)
{
    extern __shared__ __align__(16) unsigned char mx_smem[];
    bf16_t *zs = reinterpret_cast<bf16_t *>(mx_smem);   // [3][bt][ld]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = lane & 15, g = lane >> 4;
    const int b0 = blockIdx.y * bt, nb = min(bt, B - b0), ld = mx_ld(d);
    const int blocks = d / kMx4Block, steps = (d + 127) / 128;
    for (int b = wave; b < nb; b += 4) {
        const T *zr = z + (long long)(b0 + b) * z_stride;
        float ss = 0.f;
        for (int k = lane; k < d; k += 64) { const float v = to_f32(zr[k]); ss = fmaf(v, v, ss); }
        ss = wave_sum(ss);
        const float rinv = norm_free ? 1.f : rsqrtf(ss / (float)d + eps);
        for (int k = lane; k < ld; k += 64) {
            float v = 0.f;
            if (k < d) v = to_f32(zr[k]) * (rinv * ((gain && !norm_free) ? to_f32(gain[k]) : 1.f));
            // by truncation, as a value beyond the largest bf16 has a finite head then; every difference is exact
            const uint32_t p0 = __float_as_uint(v) & 0xFFFF0000u;
            const float r1 = (p0 & 0x7F800000u) == 0x7F800000u ? 0.f : v - __uint_as_float(p0);   // an infinity has no remainder
            const uint32_t p1 = __float_as_uint(r1) & 0xFFFF0000u;
            const uint32_t p2 = __float_as_uint(r1 - __uint_as_float(p1));
            zs[(size_t)b * ld + k] = v == v ? (bf16_t)(p0 >> 16) : (bf16_t)0x7FC0;
            zs[(size_t)(bt + b) * ld + k] = (bf16_t)(p1 >> 16);
            zs[(size_t)(2 * bt + b) * ld + k] = (bf16_t)(p2 >> 16);
        }
    }
    __syncthreads();
    const int cb = min(col, nb - 1);   // columns beyond the batch repeat its last row (their results are dropped)
    const bf16_t *zh = zs + (size_t)cb * ld + 32 * g, *zm = zh + (size_t)bt * ld, *zl = zm + (size_t)bt * ld;
    const int tiles = (vocab + 15) / 16;
    for (int tile = blockIdx.x * 4 + wave; tile < tiles; tile += gridDim.x * 4) {
        const size_t row = (size_t)min(tile * 16 + col, vocab - 1);
        const uint8_t *cr = codes + row * (d / 2), *er = exps + row * blocks;
        constexpr f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
        f32x4_t low = zero, head[4] = {zero, zero, zero, zero};   // middle and tail parts: 2^-8 of the sum, in one chain
        for (int st = 0; st < steps; ++st) {
            const int blk = 4 * st + g, at = min(blk, blocks - 1);
            uint4 c4 = *reinterpret_cast<const uint4 *>(cr + (size_t)at * 16);
            const int byte = er[at];
            if (blk >= blocks) c4 = make_uint4(0u, 0u, 0u, 0u);
            const float scale = __uint_as_float((uint32_t)byte << 23);
            const bool odd = byte == 0 || byte == 255;   // no scale: the block reads as NaN
            const uint32_t cw[4] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                Frag a, x;
                a.u = make_uint4(two_weights<0>(cw[j], scale), two_weights<1>(cw[j], scale), two_weights<2>(cw[j], scale),
                                 two_weights<3>(cw[j], scale));
                if (odd) a.u = make_uint4(0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u);
                const int k = 128 * st + 8 * j;
                x.u = *reinterpret_cast<const uint4 *>(zl + k); low = mfma16(a, x, low);
                x.u = *reinterpret_cast<const uint4 *>(zm + k); low = mfma16(a, x, low);
                x.u = *reinterpret_cast<const uint4 *>(zh + k); head[j] += mfma16(a, x, zero);
            }
        }
        const f32x4_t top = (head[0] + head[1]) + (head[2] + head[3]);
        f32x4_t acc = top + low;
        // an infinite product of one part with zero or the other sign in the others is no part of the sum: the head's product stands
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[r] = acc[r] == acc[r] ? acc[r] : top[r];
        if (col < nb) {
            const int v0 = tile * 16 + 4 * g;
            float *out = logits + (size_t)(b0 + col) * vocab + v0;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (v0 + r < vocab) out[r] = acc[r];
        }
    }
}

template <typename T>
hipError_t mx4_head_launch(const uint8_t *codes, const uint8_t *exps, const void *g, const void *z, long long z_stride, float *logits, int B,
                           int d, int vocab, float eps, int norm_free, hipStream_t st)
{
    int bt = (int)(kMxMaxLds / ((size_t)3 * mx_ld(d) * 2));
    bt = bt > 16 ? 16 : bt;
    bt = bt > B ? B : bt;
    const size_t lds = (size_t)3 * bt * mx_ld(d) * 2;
    hipError_t e = hipFuncSetAttribute((const void *)mx4_head_kernel<T>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kMxMaxLds);
    if (e != hipSuccess) return e;
    const int tiles = (vocab + 15) / 16, want = (tiles + 3) / 4;
    const int fit = (int)((size_t)160 * 1024 / lds), resident = 256 * (fit > 8 ? 8 : fit);
    hipLaunchKernelGGL(mx4_head_kernel<T>, dim3(want < resident ? want : resident, (B + bt - 1) / bt), dim3(256), lds, st, codes, exps,
                       (const T *)g, (const T *)z, z_stride, logits, B, d, vocab, eps, norm_free, bt);
    return hipGetLastError();
}
template hipError_t mx4_head_launch<float>(const uint8_t *, const uint8_t *, const void *, const void *, long long, float *, int, int, int,
                                           float, int, hipStream_t);
template hipError_t mx4_head_launch<bf16_t>(const uint8_t *, const uint8_t *, const void *, const void *, long long, float *, int, int, int,
                                            float, int, hipStream_t);

}  // namespace rt
