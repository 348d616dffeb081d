// Arithmetic of the paged cache that is the same on the host and on the device (plain C++, no HIP types): where a row lies,
// which exponent an 8-bit row takes, and how a call's positions are cut into splits.
#pragma once
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#if defined(__HIPCC__)
#define RT_BOTH __host__ __device__ __forceinline__
#else
#define RT_BOTH inline
#endif

namespace rt {

constexpr int kMinPage = 16, kMaxPage = 1024;   // positions of a page: a power of two in this range

// Row (of 64 values) of position j of a page, head h, in a pool [pages][H][page_len][64] with page_len = 2^lg.
RT_BOTH size_t pool_row(int page, int H, int h, int lg, int j) { return ((((size_t)page * (size_t)H) + (size_t)h) << lg) + (size_t)j; }

// A pool of pages as the kernels see it.
struct PagedCache {
    void *K, *V;              // [pages][H][page_len][64]: storage dtype, or int8 codes
    uint8_t *Kx, *Vx;         // [pages][H][page_len] exponent bytes, or null
    const int32_t *table;     // [S][table_stride]
    long long table_stride;
    int pages, lg;            // page_len = 2^lg
};

// Where a decoding step caches its pairs instead of rows K, V: sequence s at position pos[s] (negative: idle, nothing is written for it).
struct StepPages {
    PagedCache C;
    const int32_t *pos;   // null: no pages
    int max_pos;
};

// Work-items in x of the launch over N rows of S sequences: a lane for every 16 bytes of a row, positions in tiles of eight.  A grid has
// fewer than 2^32 of them.
RT_BOTH int64_t pair_row_lanes(int64_t N, int64_t H, int64_t storage_bytes) { return (N + 7) / 8 * 8 * H * (64 * storage_bytes / 16); }
constexpr int64_t kMaxRowLanes = ((int64_t)1 << 32) - 256;   // whole workgroups of 256

// A page table's entry is used only if it names a page of the pool.
RT_BOTH bool page_ok(int entry, int pages) { return (uint32_t)entry < (uint32_t)pages; }

// 8-bit rows: the values u of a row are held as codes rint(u 2^-e), |code| <= 127, with the smallest e >= -126 for which
// max |u| <= 127 2^e, and the byte e + 127.  Steps are powers of two: u 2^-e and code 2^e are exact, so a code never depends on how a
// quotient was rounded, and what is read back is exact in bf16 as well (seven bits).  Byte 0: all values are 0.  Byte 255: a value of
// the row is not finite; the row reads as NaN.  At the largest step, 2^122 (byte 249), the code 64 would read as 2^128: codes end at 63 there.
// top: the largest of the row's values as bits, sign cleared (as integers these order like the values, NaN above all).
RT_BOTH int row_exponent(uint32_t top)
{
    const int E = (int)(top >> 23);
    if (E == 255) return 255;
    if (top == 0) return 0;
    // top = 1.m 2^(E-127): 1.m 2^6 <= 127 holds up to m = 0x7E0000
    const int byte = E - 6 + ((top & 0x7FFFFFu) > 0x7E0000u ? 1 : 0);
    return byte < 1 ? 1 : byte;
}
RT_BOTH uint32_t exponent_step_bits(int byte) { return byte == 255 ? 0x7FC00000u : (uint32_t)byte << 23; }          // 2^e, 0 or NaN
RT_BOTH uint32_t exponent_inverse_bits(int byte) { return byte == 0 || byte == 255 ? 0u : (uint32_t)(254 - byte) << 23; }   // 2^-e, or 0
constexpr int kLargestStep = 249;
RT_BOTH float row_clip(float u) { return fminf(fmaxf(u, -0x1.f8p127f), 0x1.f8p127f); }   // to 63 steps of the largest
RT_BOTH int row_code(float u, int byte)   // the code of a value (clipped, if the byte is kLargestStep) of a row with this byte
{
    const uint32_t inv_bits = exponent_inverse_bits(byte);
    float inv;
    __builtin_memcpy(&inv, &inv_bits, 4);
    return byte == 255 ? 0 : (int)rintf(u * inv);
}

// How the positions below max_len of S sequences and H heads are cut: workgroups of `waves` wavefronts and split_len positions each (the last
// one shorter).  A cut costs a second launch and a stored state per part; a workgroup of sixteen wavefronts has as many loads on the way as four
// of four and needs no second launch, but fills a compute unit by itself and idles where it has less than a chunk for each wavefront.
//   Few pairs of a sequence and a head (at most kFewPairs), up to kWhole16 positions (up to kLong16 from half as many pairs on): sixteen
//   wavefronts, one part.  Up to 256 positions four have enough to do.
//   Else few pairs are cut until the chip has something to do (kWantGroups workgroups, parts of kShort positions and more), and all of them into
//   parts of about kLong, which bounds how long one sequence of a ragged batch keeps its workgroup after the others are done.
//   Many pairs, long rows in the storage dtype (kMany16 positions, between the 2000 and the 4000 measured below): sixteen
//   wavefronts again, which end their sequences four times as early.
// MI355X, us per call on the same inputs again and again, S H pairs of up to so many positions, waves * parts (bf16 unless said):
//   16 pairs, 500: 4*1 6.0, 16*1 5.6;  1000: 4*1 8.7, 4*4 7.7, 16*1 7.3;  2000: 4*1 14.3, 4*8 7.8, 16*1 10.5;  14 pairs, 513, fp32: 4*1 7.7, 16*1 5.8;
//   64 pairs, 1000: 4*4 8.0, 16*1 7.3;  2000: 4*8 8.6, 16*1 10.6;  8000: 4*1 62, 4*16 17.6, 16*4 17.0;
//   256 pairs, 500: 4*1 6.2, 16*1 5.9;  1000: 4*1 10.6, 16*1 8.1;  2000: 4*4 18.1, 16*1 14.8;  4000: 4*8 26.6, 16*1 24.0;  8000: 4*8 44, 16*1 44;
//   512 pairs, 500: 4*1 9.8, 16*1 11.4;  2000: 4*1 27.8, 4*4 29.7, 16*1 26.3;  768 pairs, 1000: 4*1 20.1, 16*1 20.5;  4000: 4*4 76.8, 16*1 71.0;
//   1024 pairs, 2000, 8 bits: 4*1 28.5, 16*1 33.3;  3200 pairs, 4096: 4*1 298, 4*4 294, 16*1 281;  8 bits: 4*1 184, 4*4 177, 16*1 193;
//   1600 pairs, 8000, 8 bits: 4*1 188, 4*8 160, 16*1 176;  32 pairs, 100001: 4*1 1015, 4*8 152, 4*32 118, 4*64 117, 16*8 111.
// In 8 bits, few pairs: 16 pairs, 500: 4*1 6.0, 16*1 6.0;  1000: 4*1 8.3, 4*4 7.6, 16*1 7.6;  2000: 4*1 12.8, 4*8 7.8, 16*1 10.8;
//   128 pairs, 1000: 4*1 8.3, 16*1 7.6;  2000: 4*8 10.8, 16*1 11.0;  4000: 4*1 26.1, 4*8 15.0, 4*16 14.3, 16*1 18.1, 16*2 15.7;
//   256 pairs, 1000: 4*1 8.5, 16*1 7.9;  2000: 4*1 15.2, 4*8 14.2, 16*1 11.9;  4000: 4*1 28.5, 4*8 21.1, 16*1 20.4;
//   many pairs: 512, 4000: 4*1 33.7, 4*8 30.6, 16*1 30.1;  1024, 4000: 4*1 52.8, 4*4 48.3, 16*1 57.9.
// fp32: 16 pairs, 300: 4*1 6.2, 16*1 5.6;  1000: 4*1 11.0, 4*4 8.4, 16*1 8.7;  2000: 4*1 18.3, 4*8 8.3, 16*1 13.3;
//   256 pairs, 1000: 4*1 15.9, 16*1 14.1;  2000: 4*1 26.6, 16*1 23.7;  4000: 4*1 53, 4*16 45.9, 16*1 45.0;  320, 8000: 4*1 186, 4*8 150, 16*1 145;
//   512 pairs, 2000: 4*1 52.1, 16*1 49.5;  3200: 4*1 92, 4*4 87, 16*1 88;  4000: 4*1 112, 4*4 106, 16*1 106, 16*2 101;  1024, 4000: 4*1 199, 4*4 188, 16*1 197.
struct SplitPlan {
    int split_len, n_splits, waves;
};
constexpr int kMaxPartials = 65536;    // stored partial states of a call: S * H * n_splits if n_splits > 1
constexpr int kSplitUnit = 256;        // four wavefronts of 64 positions
constexpr int kFewPairs = 256, kWhole16 = 1280, kLong16 = 4096, kMany16 = 3200;
constexpr int kWantGroups = 768, kShort = 256, kWhole = 640, kLong = 1024;
RT_BOTH SplitPlan split_plan(int max_len, int S, int H, bool eight_bits)
{
    const int64_t pairs = (int64_t)S * H;
    const bool few = pairs <= kFewPairs && max_len > 256 && max_len <= (2 * pairs > kFewPairs ? kLong16 : kWhole16);
    const bool many = pairs > kFewPairs && !eight_bits && max_len >= kMany16;
    int64_t n = kWantGroups / pairs;
    const int64_t most = max_len <= kWhole ? 1 : (max_len + kShort - 1) / kShort;
    if (n > most) n = most;
    if (n < max_len / kLong) n = max_len / kLong;
    if (few) n = 1;
    if (many) n = max_len / (2 * kLong16);
    if (n > kMaxPartials / pairs) n = kMaxPartials / pairs;
    if (n < 1) n = 1;
    int64_t len = ((int64_t)max_len + n - 1) / n;
    len = (len + kSplitUnit - 1) / kSplitUnit * kSplitUnit;
    if (len < kSplitUnit) len = kSplitUnit;
    SplitPlan p;
    p.split_len = (int)len;
    p.n_splits = (int)(((int64_t)max_len + len - 1) / len);
    if (p.n_splits < 1) p.n_splits = 1;
    p.waves = few || many ? 16 : 4;
    return p;
}

// The products of a step.  Where both kinds can run: those of rt_paged_products.hip read the rows as fp32 and start 16 outputs by 16 rows at a
// time, the stack engine's prepare operand rows in one product for the next.  MI355X, us per step (up to 500 cached positions, bf16), these /
// the others: d = 1024, 1 row 39.1 / 35.2, 4 rows 41.3 / 42.5, 8 43.9 / 51.1, 16 48.8 / 63.6, 32 56.8 / 76.1, 64 66.7 / 70.6, 128 101 / 82,
// 200 157 / 108;  d = 512, 1 row 28.6 / 28.1, 8 31.3 / 35.1, 32 36.1 / 45.6, 128 51.5 / 57.2, 200 71.4 / 63.1;  d = 256, 4 rows 27.2 / 27.0,
// 16 30.4 / 33.4, 200 47.4 / 49.4.
RT_BOTH bool paged_products_take(int B, int d) { return B >= 8 && (int64_t)B * d <= 65536; }
// Tiles of 16 outputs that a workgroup of rt_paged_products.hip owns: four share the splitting of their input rows, but only where that leaves
// every compute unit a workgroup.  us per step, by this rule / one tile everywhere / four: bf16, d = 1024, 32 rows 55.7 / 55.0 / 71.7, 64 rows 68.1 /
// 74.3 / 79.1;  d = 320, 200 rows 54.4 / 56.9 / 54.6;  fp32, d = 1024, 64 rows 85.0 / 88.6 / 119.1, 128 rows 138 / 147 / 153;  but d = 576, 400 rows
// 134 / 157 / 118, whose Wo and W2 just miss the line.
RT_BOTH int paged_product_tiles(int n_out, int B) { return (int64_t)((n_out + 63) / 64) * ((B + 15) / 16) >= 256 ? 4 : 1; }

}  // namespace rt
