// The read-out of a stack with 4-bit weights: blocks of 32 weights of a row share a scale 2^e, a weight is a sign and one of
// 0, 1/2, 1, 3/2, 2, 3, 4, 6 (the MX format with 4-bit elements, E2M1 codes and E8M0 scales): 17 bytes for 32 weights.
#include "rt_mx4.h"
#include "rt_ll.h"

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
// logits[b][v] = sum_k W[v][k] n_b[k], n_b = g z_b / rms(z_b): products of 16 batch rows, 16 vocabulary rows and 32 indices.
// The weights are exact in bf16 (two bits and a power of two), and one instruction turns two codes into two bf16 with their scale.  A lane
// holds one whole block of a row: its 16 bytes of codes are four fragments, and the contraction index is dealt so that slot 8 g + e of
// instruction j is k = 128 slice + 32 g + 8 j + e for lane group g.
// The rows must not lose what fp32 logits hold, so an element enters as bf16 parts that add up to all of it: one part for bf16 rows without a
// gain, two for bf16 rows with one (a product of two eight-bit significands has sixteen), three for fp32.
typedef __bf16 bf16x2v_t __attribute__((ext_vector_type(2)));

template <int BYTE> __device__ __forceinline__ uint32_t two_weights(uint32_t codes, float scale)
{
    const bf16x2v_t r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, BYTE);
    return __builtin_bit_cast(uint32_t, r);
}

__device__ __forceinline__ Frag weight_fragment(uint32_t codes, float scale)
{
    Frag f;
    f.u = make_uint4(two_weights<0>(codes, scale), two_weights<1>(codes, scale), two_weights<2>(codes, scale), two_weights<3>(codes, scale));
    return f;
}

// v as the sum of PARTS bf16 values, by truncation: a value beyond the largest bf16 has a finite head then, and every difference is exact.
// Two parts are taken of rows that are normalised: what is not finite reaches the logits through the row's 1 / rms.
template <int PARTS> __device__ __forceinline__ void split_parts(float v, uint32_t (&p)[PARTS])
{
    float r = v;
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        p[i] = __float_as_uint(r) & 0xFFFF0000u;
        r -= __uint_as_float(p[i]);
        if (PARTS > 2) r = (p[i] & 0x7F800000u) == 0x7F800000u ? 0.f : r;   // an infinity has no remainder
    }
    if (PARTS > 2 && v != v) p[0] = 0x7FC00000u;
}

__device__ __forceinline__ void eight(const uint4 (&r)[1], float (&f)[8])
{
    const uint32_t w[4] = {r[0].x, r[0].y, r[0].z, r[0].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) { f[2 * e] = __uint_as_float(w[e] << 16); f[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u); }
}
__device__ __forceinline__ void eight(const uint4 (&r)[2], float (&f)[8])
{
    const uint32_t w[8] = {r[0].x, r[0].y, r[0].z, r[0].w, r[1].x, r[1].y, r[1].z, r[1].w};
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(w[e]);
}

// The rows stay in registers and the matrix streams past them.  A workgroup has a wavefront per slice of 128 indices (up to WMAX, each with SL
// slices): it holds the fragments of its slices for 16 CT batch rows, made from z once, and per tile of 16 vocabulary rows loads 16 bytes per
// lane and slice, turns them into four fragments and feeds 4 CT PARTS matrix instructions.  The slices' partial tiles meet in LDS, RT tiles at
// a time, and are summed in slice order; the row's 1 / rms is applied to the sum.  No element of z is read or split twice by a workgroup, and
// nothing but partial tiles goes through LDS.
// Bound: for few rows the matrix (17 bytes per 32 weights; one row, d = 1024, 32768 vocabulary rows: 8.5 us = 2.1 TB/s, of which some 4 us are
// the launch and the first trip to memory); for 64 rows the chain of loads, conversions, products and sums that the two wavefronts of a SIMD
// walk through (50001 vocabulary rows: 24.1 us, the matrix units busy for 22 % of it; with rows staged in LDS and the matrix read once per 16
// rows 187).  Every further batch tile of 16 CT rows reads the matrix again: 128 rows 43.3 us, 200 78.6; fp32, 64 rows (two tiles) 55.3, 200 162;
// 64 rows of d = 2048 (two tiles) 58.8, of 4096 (four) 265.
// 32 columns and twice the wavefronts: 32 us; two tiles per barrier at 64 columns: 24.6.
// grid (<= groups of RT tiles, batch tiles of 16 CT), block 64 NW.
template <typename T, int PARTS, int CT, int SL, int RT, int WMAX>
__global__ __launch_bounds__(64 * WMAX) void mx4_rows_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ exps,
                                                       const T *__restrict__ gain, const T *__restrict__ z, long long z_stride,
                                                       float *__restrict__ logits, int B, int d, int vocab, float eps, int norm_free)
{
    extern __shared__ __align__(16) unsigned char mx_smem[];
    const int NW = blockDim.x >> 6;
    float *ssq = reinterpret_cast<float *>(mx_smem);                                 // [WMAX][16 CT] sums of squares, slice by slice
    f32x4_t *part = reinterpret_cast<f32x4_t *>(mx_smem + (WMAX + 1) * 16 * CT * 4);          // [2][RT][NW][16 CT][4]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int b0 = blockIdx.y * 16 * CT, blocks = d / kMx4Block;
    const int groups = (vocab + 16 * RT - 1) / (16 * RT);
    int blk[SL];
#pragma unroll
    for (int s = 0; s < SL; ++s) blk[s] = 4 * (wave + s * NW) + g;   // this lane's block of a row in each slice

    uint4 wc[RT][SL];
    int we[RT][SL];
    uint4 nc[RT][SL];
    int ne[RT][SL];
    auto request = [&](int grp) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const size_t row = (size_t)min((grp * RT + t) * 16 + col, vocab - 1);
#pragma unroll
            for (int s = 0; s < SL; ++s) {
                const int at = min(blk[s], blocks - 1);
                nc[t][s] = *reinterpret_cast<const uint4 *>(codes + row * (d / 2) + (size_t)at * 16);
                ne[t][s] = exps[row * blocks + at];
            }
        }
    };
    // loads come back in order: the first rows, then the matrix, which is on its way while the rows are split
    constexpr int kRaw = sizeof(T) / 2;   // 16-byte pieces of eight elements
    uint4 znext[4][kRaw], graw[SL][4][kRaw];
    const bool has_gain = PARTS == 2 || (PARTS == 3 && gain);
    auto request_rows = [&](int c, int s) {
        const T *zr = z + min(b0 + 16 * c + col, B - 1) * z_stride;   // columns beyond the batch repeat its last row (their results are dropped)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int r = 0; r < kRaw; ++r) {
                const int k = min(blk[s], blocks - 1) * kMx4Block + 8 * j + r * (16 / (int)sizeof(T));
                znext[j][r] = *reinterpret_cast<const uint4 *>(zr + k);
                if (c == 0 && has_gain) graw[s][j][r] = *reinterpret_cast<const uint4 *>(gain + k);
            }
    };
    request_rows(0, 0);
    __builtin_amdgcn_sched_barrier(0);
    int grp = blockIdx.x;
    request(grp);
    __builtin_amdgcn_sched_barrier(0);

    Frag x[CT][SL][4][PARTS];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        float ss = 0.f;
#pragma unroll
        for (int s = 0; s < SL; ++s) {
            uint4 zraw[4][kRaw];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int r = 0; r < kRaw; ++r) zraw[j][r] = znext[j][r];
            if (s + 1 < SL) request_rows(c, s + 1);
            else if (c + 1 < CT) request_rows(c + 1, 0);
            const bool in = blk[s] < blocks;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (!in) {   // past the row's end
#pragma unroll
                    for (int r = 0; r < kRaw; ++r) zraw[j][r] = make_uint4(0u, 0u, 0u, 0u);
                }
                float v[8], gn[8];
                eight(zraw[j], v);
                if (has_gain) eight(graw[s][j], gn);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    ss = fmaf(v[e], v[e], ss);
                    if (has_gain) v[e] *= gn[e];
                }
                if (PARTS == 1) {   // bf16 as it is
                    x[c][s][j][0].u = zraw[j][0];
                    continue;
                }
                uint32_t p[8][PARTS];
#pragma unroll
                for (int e = 0; e < 8; ++e) split_parts<PARTS>(v[e], p[e]);
#pragma unroll
                for (int i = 0; i < PARTS; ++i) {
                    uint4 &u = x[c][s][j][i].u;
                    u = make_uint4((p[0][i] >> 16) | p[1][i], (p[2][i] >> 16) | p[3][i], (p[4][i] >> 16) | p[5][i], (p[6][i] >> 16) | p[7][i]);
                    asm("" : "+v"(u.x), "+v"(u.y), "+v"(u.z), "+v"(u.w));   // packed here: two values a register from now on
                }
            }
            __builtin_amdgcn_sched_barrier(0);   // one block's loads at a time: the fragments take the registers
        }
        ss += xor16(ss);
        ss += xor32(ss);
        if (g == 0) ssq[wave * 16 * CT + 16 * c + col] = ss;
    }
    __syncthreads();
    float *rinv = ssq + WMAX * 16 * CT;   // [16 CT]
    if (threadIdx.x < 16 * CT) {
        float ss = 0.f;
        for (int w = 0; w < NW; ++w) ss += ssq[w * 16 * CT + threadIdx.x];
        rinv[threadIdx.x] = norm_free ? 1.f : rsqrtf(ss / (float)d + eps);   // read behind the loop's barrier
    }
    // Sums of a group's partial tiles: a thread takes one vocabulary row of four batch rows, neighbours neighbouring vocabulary rows.
    constexpr int kOut = 16 * RT * 4 * CT;
    auto finish = [&](const f32x4_t *src, int group) {
        for (int o = threadIdx.x; o < kOut; o += blockDim.x) {
            const int v = group * RT * 16 + o % (16 * RT), t = (o >> 4) % RT, q = o / (16 * RT);
            if (b0 + 4 * q >= B || v >= vocab) continue;
            const f32x4_t *p = src + (t * NW * 4 * CT + q) * 16 + (o & 15);
            f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w0 = 0; w0 < WMAX; w0 += 8) {
                if (w0 >= NW) break;
                f32x4_t s[8];
#pragma unroll
                for (int w = 0; w < 8; ++w) s[w] = p[min(w0 + w, NW - 1) * 4 * CT * 16];   // eight on the way before the first is added
#pragma unroll
                for (int w = 0; w < 8; ++w)
                    if (w0 + w < NW) sum += s[w];
            }
            float *out = logits + (size_t)(b0 + 4 * q) * vocab + v;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (b0 + 4 * q + r < B) out[(size_t)r * vocab] = sum[r] * rinv[4 * q + r];
        }
    };
    // Half of the wavefronts finish the group before while the other half, on the same SIMDs, keep the matrix units busy, and the other way
    // round: one barrier per group, partial tiles in two halves.
    const bool early = (wave & 4) == 0;
    int last = -1;
    for (int buf = 0; grp < groups; buf ^= 1) {
        f32x4_t *dst = part + buf * RT * NW * 16 * CT * 4, *prev = part + (buf ^ 1) * RT * NW * 16 * CT * 4;
        const int now = grp;
        grp += gridDim.x;
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int s = 0; s < SL; ++s) { wc[t][s] = nc[t][s]; we[t][s] = ne[t][s]; }
        if (grp < groups) request(grp);   // a whole group ahead
        if (early && last >= 0) finish(prev, last);
        // the fragments of one slice of one tile ahead of the products: the conversions take a fourth of the vector rate, and the matrix
        // units have work meanwhile
        Frag a[2][4];
        unsigned long long odd[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) odd[t] = 0;
        auto convert = [&](Frag(&f)[4], int u) {   // past a row's end the rows' fragments are zero: any block of the row will do
            const uint4 c4 = wc[u / SL][u % SL];
            const int byte = we[u / SL][u % SL];
            const float scale = __uint_as_float((uint32_t)byte << 23);
            f[0] = weight_fragment(c4.x, scale);
            f[1] = weight_fragment(c4.y, scale);
            f[2] = weight_fragment(c4.z, scale);
            f[3] = weight_fragment(c4.w, scale);
            odd[u / SL] |= __ballot(byte == 0 || byte == 255);   // no scale: the row's logits are NaN
        };
        convert(a[0], 0);
        f32x4_t acc[CT];
#pragma unroll
        for (int u = 0; u < RT * SL; ++u) {
            const int t = u / SL, s = u % SL;
            if (u + 1 < RT * SL) convert(a[(u + 1) & 1], u + 1);
            if (s == 0) {
#pragma unroll
                for (int c = 0; c < CT; ++c) acc[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            }
#pragma unroll
            for (int i = PARTS - 1; i >= 0; --i)   // the smallest part first
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int c = 0; c < CT; ++c) acc[c] = mfma16(x[c][s][j][i], a[u & 1][j], acc[c]);
            if (s == SL - 1) {
                if (odd[t]) {
                    const unsigned long long rows = odd[t] | odd[t] >> 16 | odd[t] >> 32 | odd[t] >> 48;
                    if (rows >> col & 1) {
#pragma unroll
                        for (int c = 0; c < CT; ++c) acc[c] = f32x4_t{} + __uint_as_float(0x7FC00000u);
                    }
                }
#pragma unroll
                for (int c = 0; c < CT; ++c) dst[((t * NW + wave) * 4 * CT + 4 * c + g) * 16 + col] = acc[c];   // batch rows 4 g .., vocabulary row col
            }
        }
        if (!early && last >= 0) finish(prev, last);
        last = now;
        __syncthreads();
        if (grp >= groups) finish(dst, now);
    }
}

template <typename T, int PARTS, int CT, int SL, int RT, int WMAX>
static hipError_t mx4_rows_go(const uint8_t *codes, const uint8_t *exps, const T *g, const T *z, long long z_stride, float *logits, int B, int d,
                              int vocab, float eps, int norm_free, hipStream_t st)
{
    const int slices = (d + 127) / 128, NW = (slices + SL - 1) / SL;
    const size_t lds = (WMAX + 1) * 16 * CT * 4 + (size_t)2 * RT * NW * 16 * CT * 16 * 4;
    const hipError_t e = hipFuncSetAttribute((const void *)mx4_rows_kernel<T, PARTS, CT, SL, RT, WMAX>, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    if (e != hipSuccess) return e;
    const int groups = (vocab + 16 * RT - 1) / (16 * RT), chunks = (B + 16 * CT - 1) / (16 * CT);
    const int most = CT >= 4 ? 256 : 512;
    hipLaunchKernelGGL((mx4_rows_kernel<T, PARTS, CT, SL, RT, WMAX>), dim3(groups < most ? groups : most, chunks), dim3(64 * NW), lds, st, codes, exps, g, z,
                       z_stride, logits, B, d, vocab, eps, norm_free);
    return hipGetLastError();
}

// ---- rows too wide for registers (d > 4096, fp32 > 2048) or off 16 bytes: staged in LDS as three parts, a tile of rows at a time.
// Bound: the chain of LDS reads and products of one wavefront's tile; 32768 vocabulary rows: one bf16 row of d = 8192 155 us (the matrix at 0.9
// TB/s), 16 rows 936 (three to a tile), one fp32 row of d = 4096 64.
// grid (<= row tiles / 4, batch tiles of bt), block 256, LDS 3 bt ld bf16.
constexpr size_t kMxMaxLds = 152 * 1024;

__host__ __device__ static inline int mx_ld(int d) { return (d + 127) / 128 * 128 + 8; }   // a row's elements in LDS
static_assert(3 * ((kMx4MaxWidth + 127) / 128 * 128 + 8) * 2 <= kMxMaxLds, "the widest row");

template <typename T>
__global__ __launch_bounds__(256) void mx4_wide_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ exps,
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
            uint32_t p[3];
            split_parts<3>(v, p);
#pragma unroll
            for (int i = 0; i < 3; ++i) zs[(size_t)(i * bt + b) * ld + k] = (bf16_t)(p[i] >> 16);
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
                Frag a = weight_fragment(cw[j], scale), x;
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
    const T *gt = norm_free ? nullptr : (const T *)g, *zt = (const T *)z;
#define RT_MX4_GO(PARTS, CT, SL, RT_, WMAX) \
    return mx4_rows_go<T, PARTS, CT, SL, RT_, WMAX>(codes, exps, gt, zt, z_stride, logits, B, d, vocab, eps, norm_free, st)
    // the rows' 16-byte loads: anything else goes the way of the wide rows
    const bool wide = d > 4096 || (z_stride * (long long)sizeof(T)) % 16 != 0 || ((uintptr_t)z & 15) != 0 || ((uintptr_t)g & 15) != 0;
    if (wide) {
    } else if constexpr (sizeof(T) == 2) {
        if (gt) {
            if (d <= 1024) { if (B <= 16) RT_MX4_GO(2, 1, 1, 4, 8); if (B <= 32) RT_MX4_GO(2, 2, 1, 2, 8); RT_MX4_GO(2, 4, 1, 1, 8); }
            if (d <= 2048) { if (B <= 16) RT_MX4_GO(2, 1, 1, 2, 16); RT_MX4_GO(2, 2, 1, 1, 16); }
            RT_MX4_GO(2, 1, 2, 1, 16);
        } else {
            if (d <= 1024) { if (B <= 16) RT_MX4_GO(1, 1, 1, 4, 8); if (B <= 32) RT_MX4_GO(1, 2, 1, 2, 8); RT_MX4_GO(1, 4, 1, 1, 8); }
            if (d <= 2048) { if (B <= 16) RT_MX4_GO(1, 1, 1, 2, 16); RT_MX4_GO(1, 2, 1, 1, 16); }
            RT_MX4_GO(1, 1, 2, 1, 16);
        }
    } else {
        if (d <= 1024) { if (B <= 16) RT_MX4_GO(3, 1, 1, 4, 8); RT_MX4_GO(3, 2, 1, 2, 8); }
        if (d <= 2048) RT_MX4_GO(3, 1, 1, 1, 16);
    }
#undef RT_MX4_GO
    int bt = (int)(kMxMaxLds / ((size_t)3 * mx_ld(d) * 2));
    bt = bt > 16 ? 16 : bt;
    bt = bt > B ? B : bt;
    const size_t lds = (size_t)3 * bt * mx_ld(d) * 2;
    hipError_t e = hipFuncSetAttribute((const void *)mx4_wide_kernel<T>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kMxMaxLds);
    if (e != hipSuccess) return e;
    const int tiles = (vocab + 15) / 16, want = (tiles + 3) / 4;
    const int fit = (int)((size_t)160 * 1024 / lds), resident = 256 * (fit > 8 ? 8 : fit);
    hipLaunchKernelGGL(mx4_wide_kernel<T>, dim3(want < resident ? want : resident, (B + bt - 1) / bt), dim3(256), lds, st, codes, exps,
                       (const T *)g, (const T *)z, z_stride, logits, B, d, vocab, eps, norm_free, bt);
    return hipGetLastError();
}
template hipError_t mx4_head_launch<float>(const uint8_t *, const uint8_t *, const void *, const void *, long long, float *, int, int, int,
                                           float, int, hipStream_t);
template hipError_t mx4_head_launch<bf16_t>(const uint8_t *, const uint8_t *, const void *, const void *, long long, float *, int, int, int,
                                            float, int, hipStream_t);

}  // namespace rt
