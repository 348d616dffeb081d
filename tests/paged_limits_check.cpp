// CPU checks of the paged cache at the ends of its ranges: codes of 8-bit rows next to the largest and the smallest numbers.
#include "rt_paged_args.h"

#include <cmath>
#include <cstdio>
#include <cstring>
#include <initializer_list>

using namespace rt;

#define EXPECT(cond)                                                                  \
    do {                                                                              \
        if (!(cond)) { printf("line %d: %s\n", __LINE__, #cond); return 1; }          \
    } while (0)

static float from_bits(uint32_t u) { float f; memcpy(&f, &u, 4); return f; }
static uint32_t bits_of(float f) { uint32_t u; memcpy(&u, &f, 4); return u; }

// Every finite row reads as finite values: off by max(max |u| / 127, 2^-127) at most, or held as 63 2^122 past 63.5 2^122.
static int codes()
{
    const double edge = std::ldexp(63.5, 122);
    for (uint32_t E = 0; E < 255; ++E)
        for (int i = 0; i < 4000; ++i) {
            uint32_t m = i < 1000 ? (uint32_t)i : (i < 2000 ? 0x7FFFFFu - (uint32_t)(i - 1000) : (i < 3000 ? 0x7E0000u + (uint32_t)i - 2500u : (uint32_t)i * 2137u & 0x7FFFFFu));
            const uint32_t top = E << 23 | m;
            const int byte = row_exponent(top);
            const float big = from_bits(top), step = from_bits(exponent_step_bits(byte));
            const float of_row[] = {big, big / 2, big * 0.7f, big / 3, big * 0.996f, 0.f};   // values that such a row may hold
            for (float u : of_row)
                for (float s : {1.f, -1.f}) {
                    const int c = row_code(byte == kLargestStep ? row_clip(s * u) : s * u, byte);
                    const float got = (float)c * step;
                    EXPECT(c >= -127 && c <= 127 && std::isfinite(got));
                    EXPECT((bits_of(got) & 0xFFFFu) == 0);   // exact in bf16
                    const double off = std::fabs((double)got - (double)s * (double)u);
                    if ((double)u > edge) EXPECT(got == s * std::ldexp(63.f, 122) && off <= (double)u / 63);
                    else EXPECT(off <= std::fmax((double)big / 127, std::ldexp(1.0, -127)) && off <= (double)step / 2);
                }
        }
    EXPECT(row_code(INFINITY, 255) == 0 && row_code(NAN, 255) == 0 && row_code(0.f, 0) == 0);
    return 0;
}

// What the checks accept can be launched: fewer than 2^32 work-items in x, in whole workgroups (rows_grid: a workgroup of 256 takes 32 rows in
// bf16 and 16 in fp32, positions in tiles of eight from N = 8 on).
static int launches()
{
    const char *msg;
    const int32_t *ints = (const int32_t *)(uintptr_t)(1ull << 40);
    for (int dtype : {RT_BF16, RT_F32})
        for (int H : {1, 255, 256, 257, 511, 512, 513, 1000, 18631, 4096, 100000}) {
            rt_config c = {};
            c.n_heads = H; c.head_dim = 64; c.d_model = 64 * H; c.max_batch = 1; c.dtype = dtype;
            const int per = dtype == RT_BF16 ? 32 : 16;
            const int64_t limit = dtype == RT_BF16 ? 1ll << 29 : 1ll << 28;
            const int mid = (int)(limit / H);
            for (int N : {1, 7, 8, 9, 14408, mid - 9, mid - 8, mid - 7, mid - 1, mid, mid + 1, mid + 9, (1 << 20) - 7, 1 << 20, (1 << 20) + 1}) {
                if (N < 1) continue;
                const int64_t d = c.d_model;
                const bool ok = check_pair_rows(c, PoolRanges{}, ints, 1, N, (const void *)(2ull << 50), (const void *)(3ull << 50), d, d, false, &msg) == RT_OK;
                const int64_t rows = N >= 8 ? (int64_t)((N + 7) / 8) * 8 * H : (int64_t)N * H, items = (rows + per - 1) / per * 256;
                if (ok) EXPECT(items < 1ll << 32 && N <= 1 << 20);
                EXPECT(ok == (N <= 1 << 20 && (int64_t)(N + 7) / 8 * 8 * H <= limit - per));
            }
        }
    return 0;
}

int main(int argc, char **argv)
{
    const char *what = argc > 1 ? argv[1] : "";
    if (!strcmp(what, "codes")) return codes();
    if (!strcmp(what, "launches")) return launches();
    return 2;
}
