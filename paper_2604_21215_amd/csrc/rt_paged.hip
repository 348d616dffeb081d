// Serving from pages: rows of cached pairs written (in the storage dtype or in eight bits) and read back, the attention of one new token
// per sequence over its pages, and the end of a decoding step that caches its pair there.
//
// A page holds page_len positions of one sequence, head by head: [pages][H][page_len][64].  A head's run of page_len rows is contiguous
// (2 KB and more in bf16), so a wavefront that walks one head's positions reads whole cache lines also where a row is only the 64 bytes
// of eight bits.
#include "rt_paged.h"
#include "rt_ll.h"

#include <type_traits>

namespace rt {

// ---------------------------------------------------------------- rows of 64 values, 16 bytes of them per lane
template <typename T> constexpr int kLanesPerRow = 64 * (int)sizeof(T) / 16;   // fp32 16, bf16 8, int8 4
template <typename T> constexpr int kPerLane = 16 / (int)sizeof(T);

// sum / maximum over the lanes of a row (4, 8 or 16 neighbouring lanes: inside a row of 16 lanes, no LDS crossbar)
template <int LPR> __device__ __forceinline__ float row_sum(float v)
{
    v += dpp_f(v, 0);
    v += dpp_f(v, 1);
    if (LPR >= 8) v += dpp_f(v, 2);
    if (LPR >= 16) v += dpp_f(v, 3);
    return v;
}
template <int LPR> __device__ __forceinline__ uint32_t row_max_bits(uint32_t v)
{
    v = max(v, __float_as_uint(dpp_f(__uint_as_float(v), 0)));
    v = max(v, __float_as_uint(dpp_f(__uint_as_float(v), 1)));
    if (LPR >= 8) v = max(v, __float_as_uint(dpp_f(__uint_as_float(v), 2)));
    if (LPR >= 16) v = max(v, __float_as_uint(dpp_f(__uint_as_float(v), 3)));
    return v;
}

// neighbours inside a row of 16 lanes, eight and four lanes on (every lane of the row gets the sum in the end)
__device__ __forceinline__ float ror8(float v) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x128, 0xF, 0xF, true)); }
__device__ __forceinline__ float ror4(float v) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x124, 0xF, 0xF, true)); }
// a summed over the lanes' halves in the low half (the even rows of 16), b in the high half (the odd rows)
__device__ __forceinline__ float add_halves32(float a, float b)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float add_halves16(float a, float b)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ void widen(const uint4 &r, float (&f)[4], const float *)
{
    f[0] = __uint_as_float(r.x); f[1] = __uint_as_float(r.y); f[2] = __uint_as_float(r.z); f[3] = __uint_as_float(r.w);
}
__device__ __forceinline__ void widen(const uint4 &r, float (&f)[8], const bf16_t *)
{
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) { f[2 * e] = __uint_as_float(w[e] << 16); f[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u); }
}
__device__ __forceinline__ void widen(const uint4 &r, float (&f)[16], const int8_t *)
{
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int b = 0; b < 4; ++b) f[4 * e + b] = (float)(int8_t)(w[e] >> (8 * b));
}

// ---------------------------------------------------------------- rows into pages and back
// The position of row n of sequence s, or -1 where there is none: an idle sequence, a row past its count.  at_end: positions that the
// sequence's line of the table has room for.
__device__ __forceinline__ int row_position(const PairRows &R, int s, int n, long long at_end, bool *outside)
{
    const int first = R.first[s];
    const int cnt = R.count ? min(R.count[s], R.N) : R.N;
    *outside = false;
    if (first < 0 || n >= cnt) return -1;
    if ((long long)first + n >= at_end) { *outside = true; return -1; }
    return first + n;
}

// One row of one head per 4, 8 or 16 lanes, its keys and its values.  Rows of a workgroup: tiles of eight consecutive positions (one where
// a call has fewer), head after head, so that both the 128 bytes of a head read and the runs of a page written are neighbours.
// Bound: memory; a large copy reaches 4.9 TB/s.  16 heads, over three sets of rows in turn, write / read: 8 sequences of 2048 positions in bf16
// (134 MB) 30.5 us = 4.4 TB/s / 28.5 = 4.7, bf16 and 8 bits (101 MB) 24.3 = 4.2 / 25.8 = 3.9, fp32 (268 MB) 54.3 = 4.9 / 52.7 = 5.1, fp32 and
// 8 bits (168 MB) 38.8 = 4.3 / 44.1 = 3.8; four times as many sequences 4.3 to 4.6 / 4.3 to 5.3 TB/s.  grid (row groups, S), block 256.
template <typename T, bool BITS8, int TILE>
__global__ __launch_bounds__(256) void cache_write_kernel(const PagedCache C, const PairRows R, int H, const T *__restrict__ k,
                                                          const T *__restrict__ v)
{
    constexpr int LPR = kLanesPerRow<T>, PL = kPerLane<T>;
    const int c = threadIdx.x % LPR, s = blockIdx.y;
    const unsigned r = blockIdx.x * (256 / LPR) + threadIdx.x / LPR;   // [tile of positions][head][position in the tile]
    const unsigned th = r / TILE;
    const int n = (int)(th / (unsigned)H) * TILE + (int)(r % TILE), h = (int)(th % (unsigned)H);
    if (n >= R.N) return;
    bool outside;
    const int pos = row_position(R, s, n, C.table_stride << C.lg, &outside);
    if (pos < 0) return;
    const int page = C.table[s * C.table_stride + (pos >> C.lg)];
    if (!page_ok(page, C.pages)) return;
    const size_t row = pool_row(page, H, h, C.lg, pos & ((1 << C.lg) - 1));
    const long long src = s * R.seq_stride + n * R.pos_stride + h * kHeadDim + c * PL;
    const uint4 kr = *reinterpret_cast<const uint4 *>(k + src), vr = *reinterpret_cast<const uint4 *>(v + src);
    if (!BITS8) {
        *reinterpret_cast<uint4 *>((T *)C.K + row * kHeadDim + c * PL) = kr;
        *reinterpret_cast<uint4 *>((T *)C.V + row * kHeadDim + c * PL) = vr;
        return;
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        float f[PL];
        widen(w ? vr : kr, f, (const T *)nullptr);
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < PL; ++e) top = max(top, __float_as_uint(f[e]) & 0x7FFFFFFFu);
        const int byte = row_exponent(row_max_bits<LPR>(top));
        if (__builtin_expect(byte == kLargestStep, 0)) {   // a branch of its own: as part of every code it costs 5 % of a large call
#pragma unroll
            for (int e = 0; e < PL; ++e) f[e] = row_clip(f[e]);
        }
        uint32_t packed[PL / 4];
#pragma unroll
        for (int e = 0; e < PL; ++e) {
            if (e % 4 == 0) packed[e / 4] = 0;
            packed[e / 4] |= (uint32_t)(row_code(f[e], byte) & 255) << (8 * (e % 4));
        }
        uint32_t *dst = reinterpret_cast<uint32_t *>((int8_t *)(w ? C.V : C.K) + row * kHeadDim + c * PL);
#pragma unroll
        for (int e = 0; e < PL / 4; ++e) dst[e] = packed[e];
        if (c == 0) (w ? C.Vx : C.Kx)[row] = (uint8_t)byte;
    }
}

template <typename T, bool BITS8, int TILE>
__global__ __launch_bounds__(256) void cache_read_kernel(const PagedCache C, const PairRows R, int H, T *__restrict__ k,
                                                         T *__restrict__ v)
{
    constexpr int LPR = kLanesPerRow<T>, PL = kPerLane<T>;
    const int c = threadIdx.x % LPR, s = blockIdx.y;
    const unsigned r = blockIdx.x * (256 / LPR) + threadIdx.x / LPR, th = r / TILE;
    const int n = (int)(th / (unsigned)H) * TILE + (int)(r % TILE), h = (int)(th % (unsigned)H);
    if (n >= R.N) return;
    bool outside;
    const int pos = row_position(R, s, n, C.table_stride << C.lg, &outside);
    if (pos < 0 && !outside) return;
    const int page = outside ? -1 : C.table[s * C.table_stride + (pos >> C.lg)];
    const bool ok = page_ok(page, C.pages);   // no such page: the row reads as NaN
    const size_t row = ok ? pool_row(page, H, h, C.lg, pos & ((1 << C.lg) - 1)) : 0;
    const long long dst = s * R.seq_stride + n * R.pos_stride + h * kHeadDim + c * PL;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        float f[PL];
        uint4 raw = make_uint4(0u, 0u, 0u, 0u);
        if (!BITS8) {
            if (ok) raw = *reinterpret_cast<const uint4 *>((const T *)(w ? C.V : C.K) + row * kHeadDim + c * PL);
            else if (sizeof(T) == 4) raw = make_uint4(0x7FC00000u, 0x7FC00000u, 0x7FC00000u, 0x7FC00000u);
            else raw = make_uint4(0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u);
            *reinterpret_cast<uint4 *>((w ? v : k) + dst) = raw;
            continue;
        }
        const float step = __uint_as_float(exponent_step_bits(ok ? (w ? C.Vx : C.Kx)[row] : 255));
        const uint32_t *src = reinterpret_cast<const uint32_t *>((const int8_t *)(w ? C.V : C.K) + row * kHeadDim + c * PL);
#pragma unroll
        for (int e = 0; e < PL / 4; ++e) {
            const uint32_t u = src[e];
#pragma unroll
            for (int b = 0; b < 4; ++b) f[4 * e + b] = (float)(int8_t)(u >> (8 * b)) * step;
        }
        T o[PL];
#pragma unroll
        for (int e = 0; e < PL; ++e) o[e] = from_f32_any<T>(f[e]);   // exact: codes have seven bits
        __builtin_memcpy(&raw, o, 16);
        *reinterpret_cast<uint4 *>((w ? v : k) + dst) = raw;
    }
}

template <typename T, int TILE> static dim3 rows_grid(const PairRows &R, int H)
{
    const long long rows = (long long)((R.N + TILE - 1) / TILE) * TILE * H, per = 256 / kLanesPerRow<T>;
    return dim3((unsigned)((rows + per - 1) / per), (unsigned)R.S);
}
template <typename T, int TILE> static void cache_write_go(const PagedCache &C, const PairRows &R, int H, const T *k, const T *v, hipStream_t st)
{
    const dim3 grid = rows_grid<T, TILE>(R, H);
    if (C.Kx) hipLaunchKernelGGL((cache_write_kernel<T, true, TILE>), grid, dim3(256), 0, st, C, R, H, k, v);
    else hipLaunchKernelGGL((cache_write_kernel<T, false, TILE>), grid, dim3(256), 0, st, C, R, H, k, v);
}
template <typename T, int TILE> static void cache_read_go(const PagedCache &C, const PairRows &R, int H, T *k, T *v, hipStream_t st)
{
    const dim3 grid = rows_grid<T, TILE>(R, H);
    if (C.Kx) hipLaunchKernelGGL((cache_read_kernel<T, true, TILE>), grid, dim3(256), 0, st, C, R, H, k, v);
    else hipLaunchKernelGGL((cache_read_kernel<T, false, TILE>), grid, dim3(256), 0, st, C, R, H, k, v);
}
template <typename T> hipError_t cache_write_launch(const PagedCache &C, const PairRows &R, int H, const void *k, const void *v, hipStream_t st)
{
    if (R.N >= 8) cache_write_go<T, 8>(C, R, H, (const T *)k, (const T *)v, st);
    else cache_write_go<T, 1>(C, R, H, (const T *)k, (const T *)v, st);
    return hipGetLastError();
}
template <typename T> hipError_t cache_read_launch(const PagedCache &C, const PairRows &R, int H, void *k, void *v, hipStream_t st)
{
    if (R.N >= 8) cache_read_go<T, 8>(C, R, H, (T *)k, (T *)v, st);
    else cache_read_go<T, 1>(C, R, H, (T *)k, (T *)v, st);
    return hipGetLastError();
}

// ---------------------------------------------------------------- attention of one new token
// out = sum_j softmax_j(scale <q, k_j> - slope (n - j)) v_j over the n cached rows and the pair of the token itself (distance 0).
// One pass with a running maximum and sum, kept per group of lanes that shares a row (4, 8 or 16 of them): nothing crosses the groups
// inside the loop.  The running maximum starts at the lowest finite number, so an empty row needs no special case: its sum is 0.
constexpr float kLowest = -3.402823466e38f;
__device__ __forceinline__ float exp_diff(float a, float m) { return __expf(a - m); }

// q and the pair of (s, h) as 64 values, one per lane
template <typename T, bool STEP> struct TokenRows {
    float q, kt, vt;
    bool pair;
    __device__ __forceinline__ TokenRows(const PagedAttention &A, int s, int h)
    {
        const int lane = threadIdx.x & 63;
        if (STEP) {
            const int d = A.H * kHeadDim;
            const float *r = A.qkv + (size_t)s * 3 * d + h * kHeadDim + lane;
            q = r[0]; kt = r[d]; vt = r[2 * d];
            pair = true;
            if (A.normalise) {
                q = head_norm(q, (const T *)A.g_q, h, A.eps);
                kt = head_norm(kt, (const T *)A.g_k, h, A.eps);
            }
        } else {
            q = to_f32(((const T *)A.q)[s * A.q_stride + h * kHeadDim + lane]);
            pair = A.kt != nullptr;
            kt = pair ? to_f32(((const T *)A.kt)[s * A.kv_stride + h * kHeadDim + lane]) : 0.f;
            vt = pair ? to_f32(((const T *)A.vt)[s * A.kv_stride + h * kHeadDim + lane]) : 0.f;
        }
    }
    static __device__ __forceinline__ float head_norm(float v, const T *g, int h, float eps)
    {
        return v * rsqrtf(fast_sum(v * v) / (float)kHeadDim + eps) * (g ? to_f32(g[h * kHeadDim + (threadIdx.x & 63)]) : 1.f);
    }
};

// The finished row of (s, h): lane = dimension, (m, l, o) the state over the cached rows; bad: NaN.
template <typename T, bool STEP>
__device__ __forceinline__ void finish_row(const PagedAttention &A, int s, int h, const TokenRows<T, STEP> &t, float m, float l, float o, bool bad)
{
    const int lane = threadIdx.x & 63;
    if (t.pair) {
        const float z = A.scale * fast_sum(t.q * t.kt), mx = fmaxf(m, z);
        const float e0 = exp_diff(m, mx), e1 = exp_diff(z, mx);
        l = fmaf(l, e0, e1);
        o = fmaf(o, e0, e1 * t.vt);
        m = mx;
    }
    float a = l == 0.f ? 0.f : o / l;
    if (bad) a = __uint_as_float(0x7FC00000u);
    if (STEP) {
        const int d = A.H * kHeadDim;
        if (A.attn_cat) A.attn_cat[(size_t)s * d + h * kHeadDim + lane] = a;
        if (A.op_a) {
            const bf16_t hi = f32_to_bf16_any(a);
            const ulonglong2 oo = operand_offsets(A.op_fragments != 0, A.S, d, s, h * kHeadDim + lane);
            A.op_a[oo.x] = hi;
            A.op_a[oo.y] = f32_to_bf16_any(a - bf16_to_f32(hi));
        }
    } else {
        ((T *)A.out)[s * A.out_stride + h * kHeadDim + lane] = from_f32_any<T>(a);
        if (A.lse && lane == 0) A.lse[(size_t)s * A.H + h] = bad ? __uint_as_float(0x7FC00000u) : (l == 0.f ? -INFINITY : m + logf(l));
    }
}

// C: type of the cached values (T or int8_t).  Workgroup = (h, s, split), heads first: consecutive workgroups go to different XCDs, and all
// heads of a sequence have the same work, while the late splits of a ragged batch are mostly empty (splits first, and eight of them: an
// XCD gets one split of every sequence, 512 pairs of up to 8000 positions: 125 us instead of 98).  Its wavefronts share the split's rows in
// as many runs.
// A wavefront loads 64 rows of keys and of values (fp32: 32), or 16 where no more are left, before it computes on them; the other wavefronts of
// its SIMD cover the trip (a second chunk on the way in registers leaves two wavefronts a SIMD and is slower: 8 bits, 64 sequences of up to
// 2000: 28 -> 31 us).
// Bound: memory, and for ragged batches of few sequences the longest of them.  16 heads, over three sets of pages in turn: 200 sequences of up
// to 4096 positions in bf16, 1.63 GB in 281 us = 5.8 TB/s, in 8 bits 868 MB in 188 = 4.6; 64 of up to 2000 in 8 bits 123 MB in 34.9 = 3.5,
// all of 2000 266 MB in 58.9 = 4.5 (in bf16 4.5 and 5.3, in fp32 4.5 and 5.5).  What the last-level cache holds is faster: that one set again
// and again 28.1.  One sequence of 37: 4.1 us, three dependent trips.
template <typename T, typename C, bool STEP, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void paged_attention_kernel(const PagedCache P, const PagedAttention A)
{
    constexpr int LPR = kLanesPerRow<C>, PL = kPerLane<C>, RPL = 64 / LPR, NL = sizeof(C) == 1 ? 4 : 8, CH = NL * RPL, SMALL = 16 / RPL;
    constexpr bool Q8 = sizeof(C) == 1;
    __shared__ float sm[WAVES], sl[WAVES];
    __shared__ float so[WAVES][kHeadDim];
    __shared__ int sbad[WAVES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int split = blockIdx.z, h = blockIdx.x, s = blockIdx.y;
    const int lo = split * A.plan.split_len;
    const bool one = A.plan.n_splits == 1;
    // requested together: the length, the token's rows, the table's first 64 entries of this split (whether they are needed or not)
    const int32_t *line = P.table + s * P.table_stride;
    const int n = A.lens[s];
    int base = lo >> P.lg, have = 64;   // lane i holds the entry of page base + i of the sequence, i < have
    int entry = line[min((long long)base + lane, P.table_stride - 1)];
    TokenRows<T, STEP> tok(A, s, h);
    if (n < 0 || n > A.max_len) {
        if (split == 0 && wave == 0 && (STEP || n > 0)) {   // an idle row of a step: zeros for the products; too long: NaN
            tok.pair = false;
            finish_row<T, STEP>(A, s, h, tok, kLowest, 0.f, 0.f, n > 0);
        }
        return;
    }
    if (lo >= n && !one) return;   // no rows here; the join counts the splits in the same way
    const int hi = min(n, lo + A.plan.split_len);
    // this wavefront's run: its share of the rows, in whole chunks where there is more than one for each
    const int unit = hi - lo > WAVES * 16 ? CH : 16;
    const int share = ((hi - lo + WAVES * unit - 1) / (WAVES * unit)) * unit;
    const int wlo = lo + wave * share, whi = min(hi, wlo + share);

    const int c = lane % LPR, g = lane / LPR;
    float q[PL];
#pragma unroll
    for (int e = 0; e < PL; ++e) q[e] = __shfl(tok.q, c * PL + e, 64);
    float m = kLowest, l = 0.f, o[PL];
#pragma unroll
    for (int e = 0; e < PL; ++e) o[e] = 0.f;
    const float slope = alibi_slope(A.alibi, h, A.H);
    bool bad = false;
    const int last_page = max(n - 1, 0) >> P.lg, page_mask = (1 << P.lg) - 1;
    auto check_entries = [&] {   // entries that name no page are not followed; the ones that this run needs make the row NaN
        const bool wrong = !page_ok(entry, P.pages);
        if (wrong) entry = 0;
        const int p = base + lane;
        bad = bad || __any(wrong && p >= (wlo >> P.lg) && p <= last_page && ((long long)p << P.lg) < whi);
    };
    check_entries();
    auto chunk = [&](int r0, auto loads) {
        constexpr int N = decltype(loads)::value;
        uint4 kr[N], vr[N];
        float ks[N], vs[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = r0 + i * RPL;
            const int page = __builtin_amdgcn_readlane(entry, min(r >> P.lg, last_page) - base);
            const size_t row = pool_row(page, A.H, h, P.lg, r & page_mask) + g;
            kr[i] = *reinterpret_cast<const uint4 *>((const C *)P.K + row * kHeadDim + c * PL);
            vr[i] = *reinterpret_cast<const uint4 *>((const C *)P.V + row * kHeadDim + c * PL);
            if (Q8) {
                ks[i] = __uint_as_float(exponent_step_bits(P.Kx[row]));
                vs[i] = __uint_as_float(exponent_step_bits(P.Vx[row]));
            }
        }
        float z[N], mx = m;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float f[PL], acc = 0.f;
            widen(kr[i], f, (const C *)nullptr);
#pragma unroll
            for (int e = 0; e < PL; ++e) acc = fmaf(q[e], f[e], acc);
            acc = row_sum<LPR>(acc) * A.scale;
            if (Q8) acc *= ks[i];
            const int r = r0 + i * RPL + g;
            z[i] = r < whi ? fmaf(-slope, (float)(n - r), acc) : -INFINITY;
            mx = fmaxf(mx, z[i]);
        }
        const float f0 = exp_diff(m, mx);
        l *= f0;
#pragma unroll
        for (int e = 0; e < PL; ++e) o[e] *= f0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float p = exp_diff(z[i], mx);
            l += p;
            float f[PL];
            widen(vr[i], f, (const C *)nullptr);
            const bool in = r0 + i * RPL + g < whi;   // what lies behind the last row may be anything
            const float w = Q8 ? (in ? p * vs[i] : 0.f) : p;
#pragma unroll
            for (int e = 0; e < PL; ++e) o[e] = fmaf(w, Q8 || in ? f[e] : 0.f, o[e]);
        }
        m = mx;
    };
    for (int r0 = wlo; r0 < whi; r0 += CH) {
        if ((min(r0 + CH, whi) - 1) >> P.lg >= base + have) {
            base = r0 >> P.lg;
            entry = line[min(base + lane, last_page)];
            check_entries();
        }
        if (whi - r0 > 16) chunk(r0, std::integral_constant<int, NL>{});
        else chunk(r0, std::integral_constant<int, SMALL>{});
    }
    // the groups' states meet inside the wavefront: their maximum, then the sums, each exchange halving what a lane holds of o
    float mw = fmaxf(m, xor32(m));
    mw = fmaxf(mw, xor16(mw));
    if (LPR <= 8) mw = fmaxf(mw, ror8(mw));
    if (LPR <= 4) mw = fmaxf(mw, ror4(mw));
    const float wgt = exp_diff(m, mw);
    l *= wgt;
    l += xor32(l);
    l += xor16(l);
    if (LPR <= 8) l += ror8(l);
    if (LPR <= 4) l += ror4(l);
#pragma unroll
    for (int e = 0; e < PL; ++e) o[e] *= wgt;
#pragma unroll
    for (int e = 0; e < PL / 2; ++e) o[e] = add_halves32(o[e], o[e + PL / 2]);
#pragma unroll
    for (int e = 0; e < PL / 4; ++e) {
        o[e] = add_halves16(o[e], o[e + PL / 4]);
        if (LPR <= 8) o[e] += ror8(o[e]);
        if (LPR <= 4) o[e] += ror4(o[e]);
    }
    if ((lane & 15) < LPR) {
        const int at = c * PL + (lane & 32 ? PL / 2 : 0) + (lane & 16 ? PL / 4 : 0);
#pragma unroll
        for (int e = 0; e < PL / 4; ++e) so[wave][at + e] = o[e];
    }
    if (lane == 0) { sm[wave] = mw; sl[wave] = l; sbad[wave] = bad; }
    // the wavefronts' states in LDS
    __syncthreads();
    if (wave != 0) return;
    float M = lane < WAVES ? sm[lane] : kLowest;
    M = fast_max(M);
    const float f = lane < WAVES ? exp_diff(sm[lane], M) : 0.f;
    const float L0 = fast_sum(lane < WAVES ? sl[lane] * f : 0.f);
    const bool any_bad = __any(lane < WAVES && sbad[lane]);
    float O = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) O = fmaf(so[i][lane], lane_bcast(f, i), O);
    float L = L0;
    if (one) {
        finish_row<T, STEP>(A, s, h, tok, M, L, O, any_bad);
        return;
    }
    if (any_bad) L = __uint_as_float(0x7FC00000u);
    const size_t idx = ((size_t)s * A.H + h) * A.plan.n_splits + split;
    if (lane == 0) { A.pm[idx] = M; A.pl[idx] = L; }
    A.po[idx * kHeadDim + lane] = O;
}

// The splits of every (s, h) joined, one wavefront each: the largest maximum first, then the weighted sums in split order.  The stored
// sums are requested before the maxima are known, 64 splits at a time, four per instruction (sixteen lanes each).
// grid ceil(S H / 4), block 256.
template <typename T, bool STEP> __global__ __launch_bounds__(256) void paged_join_kernel(const PagedAttention A)
{
    const int lane = threadIdx.x & 63, sh = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (sh >= A.S * A.H) return;
    const int s = sh / A.H, h = sh % A.H, all = A.plan.n_splits;
    const float *pm = A.pm + (size_t)sh * all, *pl = A.pl + (size_t)sh * all;
    const float *po = A.po + (size_t)sh * all * kHeadDim + (lane & 15) * 4;
    const int n = A.lens[s];
    TokenRows<T, STEP> tok(A, s, h);
    float m = kLowest, l = 0.f;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    if (n < 0 || n > A.max_len) return;   // done by the splits' launch
    const int ns = (n + A.plan.split_len - 1) / A.plan.split_len;
    for (int i0 = 0; i0 < ns; i0 += 64) {
        const int i = min(i0 + lane, all - 1);
        const float mi = pm[i], li = pl[i];
        constexpr int kHalf = 8;
        f32x4_t v[2][kHalf];
#pragma unroll
        for (int k = 0; k < kHalf; ++k) v[0][k] = *reinterpret_cast<const f32x4_t *>(po + (size_t)min(i0 + 4 * k + (lane >> 4), all - 1) * kHeadDim);
        if (ns - i0 > 32) {
#pragma unroll
            for (int k = 0; k < kHalf; ++k)
                v[1][k] = *reinterpret_cast<const f32x4_t *>(po + (size_t)min(i0 + 32 + 4 * k + (lane >> 4), all - 1) * kHeadDim);
        }
        const bool in = i0 + lane < ns;
        const float mx = fmaxf(m, fast_max(in ? mi : kLowest)), f0 = exp_diff(m, mx);
        const float w = in ? exp_diff(mi, mx) : 0.f;
        l = fmaf(l, f0, fast_sum(in ? w * li : 0.f));
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r] *= f0;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (half && ns - i0 <= 32) break;
#pragma unroll
            for (int k = 0; k < kHalf; ++k) {
                const int j = 32 * half + 4 * k + (lane >> 4);
                const float wj = __shfl(w, j, 64);
                const bool there = i0 + j < ns;   // what was not written may be anything
#pragma unroll
                for (int r = 0; r < 4; ++r) o[r] = fmaf(wj, there ? v[half][k][r] : 0.f, o[r]);
            }
        }
        m = mx;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        o[r] += xor16(o[r]);
        o[r] += xor32(o[r]);
    }
    const int src = lane >> 2;   // the lane that holds dimensions 4 (lane / 4) ..
    const float o0 = __shfl(o[0], src, 64), o1 = __shfl(o[1], src, 64), o2 = __shfl(o[2], src, 64), o3 = __shfl(o[3], src, 64);
    finish_row<T, STEP>(A, s, h, tok, m, l, lane & 2 ? (lane & 1 ? o3 : o2) : (lane & 1 ? o1 : o0), false);
}

size_t paged_partials_bytes() { return (size_t)kMaxPartials * (kHeadDim + 2) * 4; }
void paged_partials(PagedAttention &A, void *slab)
{
    A.po = (float *)slab;
    A.pm = A.po + (size_t)kMaxPartials * kHeadDim;
    A.pl = A.pm + kMaxPartials;
}

template <typename T, bool STEP, int WAVES> static void attention_go(const PagedCache &C, const PagedAttention &A, hipStream_t st)
{
    const dim3 grid((unsigned)A.H, (unsigned)A.S, (unsigned)A.plan.n_splits);
    if (C.Kx) hipLaunchKernelGGL((paged_attention_kernel<T, int8_t, STEP, WAVES>), grid, dim3(64 * WAVES), 0, st, C, A);
    else hipLaunchKernelGGL((paged_attention_kernel<T, T, STEP, WAVES>), grid, dim3(64 * WAVES), 0, st, C, A);
}
template <typename T, bool STEP> static hipError_t attention_launch(const PagedCache &C, const PagedAttention &A, hipStream_t st)
{
    if (A.plan.waves == 16) attention_go<T, STEP, 16>(C, A, st);
    else attention_go<T, STEP, 4>(C, A, st);
    if (A.plan.n_splits > 1)
        hipLaunchKernelGGL((paged_join_kernel<T, STEP>), dim3((unsigned)((A.S * A.H + 3) / 4)), dim3(256), 0, st, A);
    return hipGetLastError();
}
template <typename T> hipError_t paged_attention_launch(const PagedCache &C, const PagedAttention &A, hipStream_t st)
{
    return A.qkv ? attention_launch<T, true>(C, A, st) : attention_launch<T, false>(C, A, st);
}

// ---------------------------------------------------------------- the end of a paged step
// One wavefront per (s, h): qkRMS of the key, the pair into its page row (rounded once from fp32, to the
// storage dtype or to codes), and the head's slice of y.  grid (H, S), block 64.
template <typename T>
__global__ __launch_bounds__(64) void paged_finish_kernel(const PagedCache C, const int32_t *__restrict__ pos_of, int max_pos,
                                                          const float *__restrict__ kv, const T *__restrict__ g_k, int normalise, int H,
                                                          float eps, const T *__restrict__ y_new, T *__restrict__ y)
{
    const int lane = threadIdx.x, h = blockIdx.x, s = blockIdx.y, d = H * kHeadDim;
    const int pos = pos_of[s];
    if (pos < 0) return;
    const size_t yo = (size_t)s * d + h * kHeadDim + lane;
    y[yo] = y_new[yo];
    if (pos > max_pos) return;
    const int page = C.table[s * C.table_stride + (pos >> C.lg)];
    if (!page_ok(page, C.pages)) return;
    const size_t row = pool_row(page, H, h, C.lg, pos & ((1 << C.lg) - 1));
    float k = kv[(size_t)s * 2 * d + h * kHeadDim + lane];
    const float v = kv[(size_t)s * 2 * d + d + h * kHeadDim + lane];
    if (normalise) k = TokenRows<T, true>::head_norm(k, g_k, h, eps);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const float u = w ? v : k;
        if (!C.Kx) { ((T *)(w ? C.V : C.K))[row * kHeadDim + lane] = from_f32_any<T>(u); continue; }
        uint32_t top = __float_as_uint(u) & 0x7FFFFFFFu;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
        const int byte = row_exponent(top);
        ((int8_t *)(w ? C.V : C.K))[row * kHeadDim + lane] = (int8_t)row_code(byte == kLargestStep ? row_clip(u) : u, byte);
        if (lane == 0) (w ? C.Vx : C.Kx)[row] = (uint8_t)byte;
    }
}
template <typename T>
hipError_t paged_finish_launch(const PagedCache &C, const LayerDims &D, const int32_t *pos, int max_pos, const float *kv, const void *g_k,
                               const void *y_new, void *y, hipStream_t st)
{
    hipLaunchKernelGGL(paged_finish_kernel<T>, dim3((unsigned)D.H, (unsigned)D.B), dim3(64), 0, st, C, pos, max_pos, kv, (const T *)g_k,
                       !D.norm_free, D.H, D.eps, (const T *)y_new, (T *)y);
    return hipGetLastError();
}

#define RT_PAGED_FOR(T)                                                                                                          \
    template hipError_t cache_write_launch<T>(const PagedCache &, const PairRows &, int, const void *, const void *, hipStream_t); \
    template hipError_t cache_read_launch<T>(const PagedCache &, const PairRows &, int, void *, void *, hipStream_t);            \
    template hipError_t paged_attention_launch<T>(const PagedCache &, const PagedAttention &, hipStream_t);                      \
    template hipError_t paged_finish_launch<T>(const PagedCache &, const LayerDims &, const int32_t *, int, const float *,       \
                                               const void *, const void *, void *, hipStream_t);
RT_PAGED_FOR(float)
RT_PAGED_FOR(bf16_t)
#undef RT_PAGED_FOR

}  // namespace rt
