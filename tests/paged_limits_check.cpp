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

static char *at(uint64_t v) { return (char *)(uintptr_t)v; }   // addresses are compared, never followed

// What a call writes must not be what it reads while it writes: lengths, positions, the page table, the gain of the read-out.
static int overlaps()
{
    const char *msg;
    PoolRanges R;
    rt_config c = {};
    c.d_model = 256; c.n_heads = 4; c.head_dim = 64; c.max_batch = 8; c.dtype = RT_BF16;
    rt_paged_cache p = {};
    p.K = at(1ull << 40); p.V = at(2ull << 40); p.table = (const int32_t *)at(5ull << 40);
    p.table_stride = 10; p.pages = 20; p.page_len = 32;
    EXPECT(check_pool(c, &p, 3, &R, &msg) == RT_OK);
    rt_paged_cache inside = p;
    inside.table = (const int32_t *)at((1ull << 40) + 64);
    EXPECT(check_pool(c, &inside, 3, &R, &msg) == RT_ERR_INVALID_ARG);
    inside.table = (const int32_t *)at((2ull << 40) - 84);      // the third line's first entry is the pool's first byte
    EXPECT(check_pool(c, &inside, 3, &R, &msg) == RT_OK);
    inside.table = (const int32_t *)at((2ull << 40) - 80);
    EXPECT(check_pool(c, &inside, 3, &R, &msg) == RT_ERR_INVALID_ARG && check_pool(c, &inside, 2, &R, &msg) == RT_OK);
    // positions are 32-bit numbers: the last one that a line may name is 2^31 - 1
    rt_paged_cache wide = p;
    wide.page_len = 1024; wide.table_stride = 1 << 21;
    EXPECT(check_pool(c, &wide, 1, &R, &msg) == RT_OK);
    wide.table_stride = (1 << 21) + 1;
    EXPECT(check_pool(c, &wide, 1, &R, &msg) == RT_ERR_INVALID_ARG);
    wide.page_len = 16; wide.table_stride = 1 << 26;
    EXPECT(check_pool(c, &wide, 1, &R, &msg) == RT_OK);
    EXPECT(check_pool(c, &p, 3, &R, &msg) == RT_OK);

    char *k = at(7ull << 40), *v = at(8ull << 40), *q = at(9ull << 40), *out = at(10ull << 40);
    const int32_t *ints = (const int32_t *)at(6ull << 40);
    auto rows = [&](const int32_t *first, const int32_t *count, const int32_t *table, bool outputs) {
        return check_pair_rows(c, R, first, 3, 5, k, v, 256, 768, outputs, &msg, count, table, 10);
    };
    for (bool outputs : {false, true}) {
        EXPECT(rows(ints, nullptr, p.table, outputs) == RT_OK && rows(ints, ints, p.table, outputs) == RT_OK);
        for (char *w : {k, v, (char *)p.K + 100, (char *)p.V}) {
            const bool written = outputs == (w == k || w == v);
            const int32_t *i = (const int32_t *)(w + 512);
            EXPECT((rows(i, nullptr, p.table, outputs) == RT_OK) == !written && (rows(ints, i, p.table, outputs) == RT_OK) == !written);
            EXPECT((rows(ints, nullptr, i, outputs) == RT_OK) == !written);
        }
    }
    float *lse = (float *)at(11ull << 40);
    auto attn = [&](const int32_t *lens, void *o, float *l) {
        return check_paged_attention(c, &p, R, 3, lens, 100, q, 256, k, v, 256, o, 256, l, &msg);
    };
    EXPECT(attn(ints, out, lse) == RT_OK && attn(ints, out, nullptr) == RT_OK);
    EXPECT(attn((const int32_t *)(out + 4), out, lse) == RT_ERR_INVALID_ARG && attn((const int32_t *)(lse + 11), out, lse) == RT_ERR_INVALID_ARG);
    EXPECT(attn(ints, (void *)(p.table + 23), lse) == RT_ERR_INVALID_ARG && attn(ints, (void *)(p.table + 24), lse) == RT_OK);   // 4 entries of the last line
    EXPECT(attn(ints, out, (float *)p.table) == RT_ERR_INVALID_ARG);
    auto step = [&](const int32_t *pos, void *y) { return check_paged_step(c, &p, R, q, 3, pos, 100, y, &msg); };
    EXPECT(step(ints, out) == RT_OK && step((const int32_t *)out + 2, out) == RT_ERR_INVALID_ARG);
    EXPECT(step((const int32_t *)p.K, out) == RT_ERR_INVALID_ARG && step(ints, (void *)p.table) == RT_ERR_INVALID_ARG);
    const uint8_t *codes = (const uint8_t *)at(12ull << 40), *exps = (const uint8_t *)at(13ull << 40);
    auto head = [&](int vocab, const void *g) { return check_mx4_head(c, codes, exps, vocab, q, 256, 8, lse, &msg, g); };
    EXPECT(head(100, k) == RT_OK && head(100, nullptr) == RT_OK && head(100, lse + 799) == RT_ERR_INVALID_ARG && head(100, lse + 800) == RT_OK);
    EXPECT(head(100, (char *)lse - 511) == RT_ERR_INVALID_ARG && head(100, (char *)lse - 512) == RT_OK);
    EXPECT(head(INT32_MAX, k) == RT_ERR_INVALID_ARG && head(INT32_MAX - 63, k) == RT_ERR_INVALID_ARG && head(INT32_MAX - 64, k) == RT_OK);
    return 0;
}

int main(int argc, char **argv)
{
    const char *what = argc > 1 ? argv[1] : "";
    if (!strcmp(what, "codes")) return codes();
    if (!strcmp(what, "launches")) return launches();
    if (!strcmp(what, "overlaps")) return overlaps();
    return 2;
}
