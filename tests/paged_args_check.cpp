// CPU checks of the paged cache's arithmetic (rt_paged_index.h) and of its entry points' argument checks (rt_paged_args.h).
#include "rt_paged_args.h"

#include <cmath>
#include <cstdio>
#include <initializer_list>
#include <cstring>

using namespace rt;

#define EXPECT(cond)                                                                  \
    do {                                                                              \
        if (!(cond)) { printf("line %d: %s\n", __LINE__, #cond); return 1; }          \
    } while (0)

static float from_bits(uint32_t u) { float f; memcpy(&f, &u, 4); return f; }

static int exponents()
{
    EXPECT(row_exponent(0) == 0 && row_exponent(0x7F800000u) == 255 && row_exponent(0x7FC00000u) == 255 && row_exponent(0x7FFFFFFFu) == 255);
    uint32_t seed = 12345;
    for (int i = 0; i < 2000000; ++i) {
        seed = seed * 1664525u + 1013904223u;
        uint32_t top = seed & 0x7FFFFFFFu;
        if (i < 2000) top = (uint32_t)i;                                   // the smallest
        else if (i < 4000) top = ((uint32_t)(i % 255) << 23) | (0x7E0000u + (uint32_t)(i / 255) - 11u);   // next to 127 / 128
        if (top == 0 || top >= 0x7F800000u) continue;
        const int byte = row_exponent(top);
        EXPECT(byte >= 1 && byte <= 249);
        const double t = from_bits(top), step = std::ldexp(1.0, byte - 127);
        EXPECT(t <= 127 * step);
        EXPECT(byte == 1 || t > 127 * step / 2);
        EXPECT(from_bits(exponent_step_bits(byte)) == (float)step && from_bits(exponent_inverse_bits(byte)) == (float)(1 / step));
        EXPECT(std::nearbyint(t / step) <= 127);
    }
    EXPECT(from_bits(exponent_step_bits(0)) == 0.f && std::isnan(from_bits(exponent_step_bits(255))));
    EXPECT(exponent_inverse_bits(0) == 0 && exponent_inverse_bits(255) == 0);
    return 0;
}

static int rows()
{
    // every row of a small pool once; entries of a table that name no page
    bool seen[3 * 5 * 16] = {};
    for (int page = 0; page < 3; ++page)
        for (int h = 0; h < 5; ++h)
            for (int j = 0; j < 16; ++j) {
                const size_t r = pool_row(page, 5, h, 4, j);
                EXPECT(r < sizeof(seen) && !seen[r]);
                seen[r] = true;
            }
    EXPECT(pool_row(1 << 20, 200, 199, 10, 1023) == ((size_t)(1 << 20) * 200 + 199) * 1024 + 1023);   // beyond 32 bits
    EXPECT(page_ok(0, 1) && page_ok(6, 7) && !page_ok(7, 7) && !page_ok(-1, 7) && !page_ok(INT32_MIN, 7) && !page_ok(INT32_MAX, 7));
    return 0;
}

static int plans()
{
    const int lens[] = {0, 1, 37, 255, 256, 257, 1000, 4096, 5000, 100001, 1 << 20}, seqs[] = {1, 2, 7, 64, 200, 1024}, heads[] = {1, 2, 12, 16, 128};
    for (int len : lens)
        for (int S : seqs)
            for (int H : heads)
                for (bool eight_bits : {false, true}) {
                    const SplitPlan p = split_plan(len, S, H, eight_bits);
                    EXPECT(p.waves == 4 || p.waves == 16);
                    EXPECT(p.n_splits >= 1 && p.split_len >= kSplitUnit && p.split_len % kSplitUnit == 0);
                    EXPECT((int64_t)p.n_splits * p.split_len >= len);
                    EXPECT(p.n_splits == 1 || (int64_t)(p.n_splits - 1) * p.split_len < len);
                    EXPECT(p.n_splits == 1 || (int64_t)p.n_splits * S * H <= kMaxPartials);
                }
    return 0;
}

static rt_config config(int dtype = RT_BF16)
{
    rt_config c = {};
    c.d_model = 256; c.n_heads = 4; c.head_dim = 64; c.d_hidden = 1024; c.max_batch = 8; c.max_seq = 1; c.dtype = dtype;
    return c;
}
static char *at(uint64_t v) { return (char *)(uintptr_t)v; }   // addresses are compared, never followed
static rt_paged_cache pool_of(int bits)
{
    rt_paged_cache p = {};
    p.K = at(1ull << 40); p.V = at(2ull << 40);
    if (bits) { p.K_exp = (uint8_t *)at(3ull << 40); p.V_exp = (uint8_t *)at(4ull << 40); }
    p.table = (const int32_t *)at(5ull << 40);
    p.table_stride = 10; p.pages = 20; p.page_len = 32; p.bits = bits;
    return p;
}

static int refusals()
{
    const char *msg;
    PoolRanges R;
    const rt_config cfg = config();
    rt_paged_cache p = pool_of(0), q8 = pool_of(8);
    EXPECT(check_pool(cfg, &p, 3, &R, &msg) == RT_OK && check_pool(cfg, &q8, 3, &R, &msg) == RT_OK);
    auto bad = [&](rt_paged_cache c, int S, rt_status want) { return check_pool(cfg, &c, S, &R, &msg) == want && msg[0]; };
#define CHANGED(from, stmt, S, want) { rt_paged_cache c = from; stmt; EXPECT(bad(c, S, want)); }
    EXPECT(check_pool(cfg, nullptr, 1, &R, &msg) == RT_ERR_INVALID_ARG);
    CHANGED(p, c.K = nullptr, 1, RT_ERR_INVALID_ARG) CHANGED(p, c.V = nullptr, 1, RT_ERR_INVALID_ARG)
    CHANGED(p, c.table = nullptr, 1, RT_ERR_INVALID_ARG) CHANGED(p, c.bits = 4, 1, RT_ERR_UNSUPPORTED)
    CHANGED(p, c.bits = 8, 1, RT_ERR_INVALID_ARG) CHANGED(q8, c.bits = 0, 1, RT_ERR_INVALID_ARG)
    CHANGED(q8, c.V_exp = nullptr, 1, RT_ERR_INVALID_ARG) CHANGED(p, c.pages = 0, 1, RT_ERR_INVALID_ARG)
    CHANGED(p, c.page_len = 24, 1, RT_ERR_INVALID_ARG) CHANGED(p, c.page_len = 8, 1, RT_ERR_INVALID_ARG)
    CHANGED(p, c.page_len = 2048, 1, RT_ERR_INVALID_ARG) CHANGED(p, c.table_stride = 0, 1, RT_ERR_INVALID_ARG)
    CHANGED(p, (void)0, 0, RT_ERR_INVALID_ARG) CHANGED(p, (void)0, 70000, RT_ERR_INVALID_ARG)
    CHANGED(p, c.K = at((1ull << 40) + 8), 1, RT_ERR_INVALID_ARG) CHANGED(p, c.V = at((1ull << 40) + 1024), 1, RT_ERR_INVALID_ARG)
    CHANGED(q8, c.K_exp = (uint8_t *)at((2ull << 40) + 5), 1, RT_ERR_INVALID_ARG)

    EXPECT(check_pool(cfg, &p, 3, &R, &msg) == RT_OK);
    const int32_t *ints = (const int32_t *)at(6ull << 40);
    char *k = at(7ull << 40), *v = at(8ull << 40);
    auto rows = [&](int S, int N, void *k_, void *v_, int64_t ss, int64_t ps, bool outputs) {
        return check_pair_rows(cfg, R, ints, S, N, k_, v_, ss, ps, outputs, &msg);
    };
    EXPECT(rows(3, 5, k, v, 256, 3 * 256, true) == RT_OK && rows(3, 5, k, v, 5 * 256, 256, true) == RT_OK && rows(1, 1, k, v, 0, 0, true) == RT_OK);
    EXPECT(check_pair_rows(cfg, R, nullptr, 3, 5, k, v, 256, 768, false, &msg) == RT_ERR_INVALID_ARG);
    EXPECT(rows(3, 0, k, v, 256, 768, false) == RT_ERR_INVALID_ARG && rows(3, (1 << 20) + 1, k, v, 256, 768, false) == RT_ERR_INVALID_ARG);
    EXPECT(rows(3, 5, k, nullptr, 256, 768, false) == RT_ERR_INVALID_ARG && rows(3, 5, k + 8, v, 256, 768, false) == RT_ERR_INVALID_ARG);
    EXPECT(rows(3, 5, k, v, 255, 768, false) == RT_ERR_INVALID_ARG && rows(3, 5, k, v, 260, 1024, false) == RT_ERR_INVALID_ARG);
    EXPECT(rows(3, 5, k, v, 256, -768, false) == RT_ERR_INVALID_ARG && rows(3, 5, at(1ull << 40) - 256, v, 256, 768, false) == RT_ERR_INVALID_ARG);
    EXPECT(rows(3, 5, k, v, 256, 256, false) == RT_OK && rows(3, 5, k, v, 256, 256, true) == RT_ERR_INVALID_ARG);   // read twice / written twice
    EXPECT(rows(3, 5, k, k, 256, 768, false) == RT_OK && rows(3, 5, k, k, 256, 768, true) == RT_ERR_INVALID_ARG);
    EXPECT(rows(3, 5, k, k + 512, 512, 3 * 512, true) == RT_OK);            // [N][S][2][d]
    EXPECT(rows(3, 5, k, k + 3 * 512, 256, 6 * 256, true) == RT_OK);        // [N][2][S][d]
    EXPECT(rows(3, 5, k, k + 256, 512, 3 * 512, true) == RT_ERR_INVALID_ARG);
    EXPECT(rows(1, 1, k, k + 256, 0, 0, true) == RT_ERR_INVALID_ARG && rows(1, 1, k, k + 512, 0, 0, true) == RT_OK);

    char *q = at(9ull << 40), *out = at(10ull << 40);
    float *lse = (float *)at(11ull << 40);
    auto attn = [&](int S, int len, void *q_, int64_t qs, void *kt, void *vt, int64_t kvs, void *o, int64_t os, float *l) {
        return check_paged_attention(cfg, &p, R, S, ints, len, q_, qs, kt, vt, kvs, o, os, l, &msg);
    };
    EXPECT(attn(8, 320, q, 256, k, v, 256, out, 256, lse) == RT_OK && attn(1, 0, q, 256, nullptr, nullptr, 0, out, 300, nullptr) == RT_OK);
    EXPECT(attn(9, 320, q, 256, k, v, 256, out, 256, lse) == RT_ERR_INVALID_ARG && attn(8, 321, q, 256, k, v, 256, out, 256, lse) == RT_ERR_INVALID_ARG);
    EXPECT(attn(8, -1, q, 256, k, v, 256, out, 256, lse) == RT_ERR_INVALID_ARG && attn(8, 9, nullptr, 256, k, v, 256, out, 256, lse) == RT_ERR_INVALID_ARG);
    EXPECT(attn(8, 9, q, 256, k, nullptr, 256, out, 256, lse) == RT_ERR_INVALID_ARG && attn(8, 9, q, 255, k, v, 256, out, 256, lse) == RT_ERR_INVALID_ARG);
    EXPECT(attn(8, 9, q, 256, k, v, 0, out, 256, lse) == RT_ERR_INVALID_ARG && attn(8, 9, q, 256, k, v, 256, out, 128, lse) == RT_ERR_INVALID_ARG);
    EXPECT(attn(8, 9, q, 256, k, v, 256, q + 64, 256, lse) == RT_ERR_INVALID_ARG && attn(8, 9, q, 256, k, v, 256, v, 256, lse) == RT_ERR_INVALID_ARG);
    EXPECT(attn(8, 9, q, 256, k, v, 256, at(2ull << 40), 256, lse) == RT_ERR_INVALID_ARG && attn(8, 9, q, 256, k, v, 256, out, 256, (float *)out) == RT_ERR_INVALID_ARG);

    auto step = [&](void *x, int S, const int32_t *pos, int most, void *y) { return check_paged_step(cfg, &p, R, x, S, pos, most, y, &msg); };
    EXPECT(step(q, 8, ints, 319, out) == RT_OK && step(q, 8, ints, 320, out) == RT_ERR_INVALID_ARG && step(q, 8, ints, -1, out) == RT_ERR_INVALID_ARG);
    EXPECT(step(q, 9, ints, 5, out) == RT_ERR_INVALID_ARG && step(q, 8, nullptr, 5, out) == RT_ERR_INVALID_ARG && step(q, 8, ints, 5, q + 512) == RT_ERR_INVALID_ARG);
    EXPECT(step(q + 8, 8, ints, 5, out) == RT_ERR_INVALID_ARG && step(q, 8, ints, 5, out + 8) == RT_ERR_INVALID_ARG);
    EXPECT(step(at(1ull << 40), 8, ints, 5, out) == RT_ERR_INVALID_ARG && step(q, 8, ints, 5, nullptr) == RT_ERR_INVALID_ARG);

    const uint8_t *codes = (const uint8_t *)at(12ull << 40), *exps = (const uint8_t *)at(13ull << 40);
    auto head = [&](const uint8_t *c, const uint8_t *e, int vocab, const void *z, int64_t zs, int B, float *l) {
        return check_mx4_head(cfg, c, e, vocab, z, zs, B, l, &msg);
    };
    EXPECT(head(codes, exps, 100, q, 256, 8, lse) == RT_OK && head(codes + 8, exps, 100, q, 256, 8, lse) == RT_ERR_INVALID_ARG);
    EXPECT(head(codes, nullptr, 100, q, 256, 8, lse) == RT_ERR_INVALID_ARG && head(codes, exps, 0, q, 256, 8, lse) == RT_ERR_INVALID_ARG);
    EXPECT(head(codes, exps, 100, q, 255, 8, lse) == RT_ERR_INVALID_ARG && head(codes, exps, 100, q, 256, 9, lse) == RT_ERR_INVALID_ARG);
    EXPECT(head(codes, exps, 100, q, 256, 8, (float *)q) == RT_ERR_INVALID_ARG && head(codes, exps, 100, q, 256, 8, (float *)exps) == RT_ERR_INVALID_ARG);
    rt_config big = cfg;
    big.d_model = 25920;
    EXPECT(check_mx4_head(big, codes, exps, 100, q, 25920, 8, lse, &msg) == RT_ERR_UNSUPPORTED);
    return 0;
}

int main(int argc, char **argv)
{
    const char *what = argc > 1 ? argv[1] : "";
    if (!strcmp(what, "exponents")) return exponents();
    if (!strcmp(what, "rows")) return rows();
    if (!strcmp(what, "plans")) return plans();
    if (!strcmp(what, "refusals")) return refusals();
    return 2;
}
