// Host-side checks of the paged-cache and 4-bit entry points: everything that can be told from the arguments, before anything is
// enqueued.  Plain C++ (the CPU tests compile it by itself); msg receives the reason.
#pragma once
#include "../../include/rt.h"
#include "rt_paged_index.h"

#include <stddef.h>
#include <stdint.h>

namespace rt {

constexpr int kMx4Block = 32;          // weights that share a scale
constexpr int kMx4MaxWidth = 25856;    // three bf16 parts of a row fit in LDS

struct ByteRange {
    const void *p;
    size_t bytes;
};
inline bool ranges_meet(const ByteRange &a, const ByteRange &b)
{
    const char *pa = (const char *)a.p, *pb = (const char *)b.p;
    return a.p && b.p && pa < pb + b.bytes && pb < pa + a.bytes;
}
inline bool on16(const void *p) { return ((uintptr_t)p & 15) == 0; }
inline int64_t storage_bytes(const rt_config &cfg) { return cfg.dtype == RT_BF16 ? 2 : 4; }

// The four arrays of a pool (the last two null in the storage dtype).
struct PoolRanges {
    ByteRange r[4];
    bool meets(const ByteRange &o) const { return ranges_meet(r[0], o) || ranges_meet(r[1], o) || ranges_meet(r[2], o) || ranges_meet(r[3], o); }
};

// The lines of S sequences in a table of which the last line's first `entries` count.
inline ByteRange table_range(const rt_paged_cache &cache, int32_t S, int64_t entries)
{
    return {cache.table, (size_t)(((int64_t)(S - 1) * cache.table_stride + (entries < 1 ? 1 : entries)) * 4)};
}
inline ByteRange ints_range(const int32_t *p, int32_t S) { return {p, (size_t)S * 4}; }

inline rt_status check_pool(const rt_config &cfg, const rt_paged_cache *cache, int32_t S, PoolRanges *out, const char **msg)
{
    *msg = "null cache pointer";
    if (!cache || !cache->K || !cache->V || !cache->table) return RT_ERR_INVALID_ARG;
    *msg = "a cache holds the storage dtype (bits 0) or 8 bits";
    if (cache->bits != 0 && cache->bits != 8) return RT_ERR_UNSUPPORTED;
    *msg = "K_exp and V_exp belong to a cache of 8 bits, and to no other";
    if ((cache->bits == 8) != (cache->K_exp != nullptr) || (cache->bits == 8) != (cache->V_exp != nullptr)) return RT_ERR_INVALID_ARG;
    *msg = "pages >= 1 and page_len a power of two from 16 to 1024 are required";
    if (cache->pages < 1 || cache->page_len < kMinPage || cache->page_len > kMaxPage || (cache->page_len & (cache->page_len - 1)) != 0)
        return RT_ERR_INVALID_ARG;
    *msg = "1 <= S <= 65535 and 1 <= table_stride <= 2^26 are required";
    if (S < 1 || S > 65535 || cache->table_stride < 1 || cache->table_stride > (1 << 26)) return RT_ERR_INVALID_ARG;
    *msg = "a line of the table may name 2^31 positions at most";
    if (cache->table_stride * cache->page_len > (int64_t)1 << 31) return RT_ERR_INVALID_ARG;
    *msg = "K and V of a cache must lie on 16 bytes";
    if (!on16(cache->K) || !on16(cache->V)) return RT_ERR_INVALID_ARG;
    const size_t rows = (size_t)cache->pages * (size_t)cfg.n_heads * (size_t)cache->page_len;
    const size_t bytes = rows * 64 * (cache->bits == 8 ? 1 : (size_t)storage_bytes(cfg));
    *out = {{{cache->K, bytes}, {cache->V, bytes}, {cache->K_exp, rows}, {cache->V_exp, rows}}};
    *msg = "the arrays of a cache must not overlap";
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < i; ++j)
            if (ranges_meet(out->r[i], out->r[j])) return RT_ERR_INVALID_ARG;
    *msg = "the page table must not overlap the pages";
    if (out->meets(table_range(*cache, S, 1))) return RT_ERR_INVALID_ARG;
    *msg = "";
    return RT_OK;
}

// Rows of pairs on the caller's side; outputs: rows that are written must not overlap one another.
inline rt_status check_pair_rows(const rt_config &cfg, const PoolRanges &pool, const int32_t *first, int32_t S, int32_t N, const void *k,
                                 const void *v, int64_t seq_stride, int64_t pos_stride, bool outputs, const char **msg,
                                 const int32_t *count = nullptr, const int32_t *table = nullptr, int64_t table_stride = 0)
{
    const int64_t d = cfg.d_model, E = storage_bytes(cfg), most = (int64_t)1 << 40;
    *msg = "null pointer";
    if (!first || !k || !v) return RT_ERR_INVALID_ARG;
    *msg = "1 <= N <= 2^20 and N (rounded up to a multiple of 8) n_heads <= 2^29 - 32 (bf16) or 2^28 - 16 (fp32) are required";
    if (N < 1 || N > (1 << 20) || pair_row_lanes(N, cfg.n_heads, E) > kMaxRowLanes) return RT_ERR_INVALID_ARG;
    *msg = "rows are at least d_model elements apart";
    if ((S > 1 && seq_stride < d) || (N > 1 && pos_stride < d) || seq_stride < 0 || pos_stride < 0 || seq_stride > most || pos_stride > most)
        return RT_ERR_INVALID_ARG;
    *msg = "rows of pairs must lie on 16 bytes";
    if (!on16(k) || !on16(v) || seq_stride * E % 16 != 0 || pos_stride * E % 16 != 0) return RT_ERR_INVALID_ARG;
    const size_t span = (size_t)(((int64_t)(S - 1) * seq_stride + (int64_t)(N - 1) * pos_stride + d) * E);
    const ByteRange kr = {k, span}, vr = {v, span};
    *msg = "the rows must not overlap the cache";
    if (pool.meets(kr) || pool.meets(vr)) return RT_ERR_INVALID_ARG;
    const ByteRange ints[3] = {ints_range(first, S), ints_range(count, S), {table, (size_t)((S - 1) * table_stride + 1) * 4}};
    *msg = "first, count and the page table must not overlap what is written";
    for (const ByteRange &r : ints)
        if (outputs ? ranges_meet(kr, r) || ranges_meet(vr, r) : pool.meets(r)) return RT_ERR_INVALID_ARG;
    if (outputs) {
        *msg = "the rows of different sequences overlap";
        if (S > 1 && N > 1 && seq_stride < (int64_t)(N - 1) * pos_stride + d && pos_stride < (int64_t)(S - 1) * seq_stride + d)
            return RT_ERR_INVALID_ARG;
        // k and v may be slices of one tensor: then the rows of one lie in the gaps of the other, between neighbouring rows or
        // between the runs of the outer index
        *msg = "k and v overlap";
        if (ranges_meet(kr, vr)) {
            const int64_t off = ((const char *)v - (const char *)k) / E, gap = off < 0 ? -off : off;
            const bool seq_inner = N == 1 || (S > 1 && seq_stride <= pos_stride);
            const int64_t inner = seq_inner ? seq_stride : pos_stride, outer = seq_inner ? pos_stride : seq_stride;
            const int64_t n_in = seq_inner ? S : N, n_out = seq_inner ? N : S, run = (n_in - 1) * inner + d;
            const bool between_rows = n_in > 1 && gap >= d && gap + d <= inner, between_runs = n_out > 1 && gap >= run && gap + run <= outer;
            if (!between_rows && !between_runs) return RT_ERR_INVALID_ARG;
        }
    }
    *msg = "";
    return RT_OK;
}

inline rt_status check_paged_attention(const rt_config &cfg, const rt_paged_cache *cache, const PoolRanges &pool, int32_t S, const int32_t *lens,
                                       int32_t max_len, const void *q, int64_t q_stride, const void *k_t, const void *v_t, int64_t kv_stride,
                                       const void *out, int64_t out_stride, const float *lse, const char **msg)
{
    const int64_t d = cfg.d_model, E = storage_bytes(cfg), most = (int64_t)1 << 40;
    *msg = "null pointer";
    if (!lens || !q || !out) return RT_ERR_INVALID_ARG;
    *msg = "k_t and v_t are given together or not at all";
    if ((k_t == nullptr) != (v_t == nullptr)) return RT_ERR_INVALID_ARG;
    *msg = "S out of range [1, max_batch]";
    if (S > cfg.max_batch) return RT_ERR_INVALID_ARG;
    *msg = "max_len out of range [0, min(2^20, table_stride page_len)]";
    if (max_len < 0 || max_len > (1 << 20) || max_len > cache->table_stride * cache->page_len) return RT_ERR_INVALID_ARG;
    *msg = "rows are at least d_model elements apart";
    if (q_stride < d || out_stride < d || (k_t && kv_stride < d) || q_stride > most || out_stride > most || (k_t && kv_stride > most))
        return RT_ERR_INVALID_ARG;
    auto rows = [&](const void *p, int64_t stride) { return ByteRange{p, p ? (size_t)(((S - 1) * stride + d) * E) : 0}; };
    const ByteRange o = rows(out, out_stride), l = {lse, (size_t)S * (size_t)cfg.n_heads * 4};
    const ByteRange in[3] = {rows(q, q_stride), rows(k_t, kv_stride), rows(v_t, kv_stride)};
    *msg = "out and lse must not overlap an input or each other";
    if (ranges_meet(o, l) || pool.meets(o) || pool.meets(l)) return RT_ERR_INVALID_ARG;
    for (const ByteRange &r : in)
        if (ranges_meet(o, r) || ranges_meet(l, r)) return RT_ERR_INVALID_ARG;
    const ByteRange n = ints_range(lens, S), t = table_range(*cache, S, (max_len + cache->page_len - 1) / cache->page_len);
    if (ranges_meet(o, n) || ranges_meet(l, n) || ranges_meet(o, t) || ranges_meet(l, t)) return RT_ERR_INVALID_ARG;
    *msg = "";
    return RT_OK;
}

inline rt_status check_paged_step(const rt_config &cfg, const rt_paged_cache *cache, const PoolRanges &pool, const void *x_t, int32_t S,
                                  const int32_t *pos, int32_t max_pos, const void *y_t, const char **msg)
{
    *msg = "null tensor pointer";
    if (!x_t || !pos || !y_t) return RT_ERR_INVALID_ARG;
    *msg = "S out of range [1, max_batch]";
    if (S > cfg.max_batch) return RT_ERR_INVALID_ARG;
    *msg = "max_pos out of range [0, min(2^20, table_stride page_len - 1)]";
    if (max_pos < 0 || max_pos > (1 << 20) || max_pos >= cache->table_stride * cache->page_len) return RT_ERR_INVALID_ARG;
    *msg = "x_t and y_t must lie on 16 bytes";
    if (!on16(x_t) || !on16(y_t)) return RT_ERR_INVALID_ARG;
    const size_t bytes = (size_t)S * (size_t)cfg.d_model * (size_t)storage_bytes(cfg);
    const ByteRange x = {x_t, bytes}, y = {y_t, bytes};
    *msg = "the cache, x_t, y_t must not overlap";
    if (ranges_meet(x, y) || pool.meets(x) || pool.meets(y)) return RT_ERR_INVALID_ARG;
    const ByteRange n = ints_range(pos, S);
    *msg = "pos and the page table must not overlap y_t or the cache";
    if (ranges_meet(y, n) || pool.meets(n) || ranges_meet(y, table_range(*cache, S, max_pos / cache->page_len + 1))) return RT_ERR_INVALID_ARG;
    *msg = "";
    return RT_OK;
}

inline rt_status check_mx4_head(const rt_config &cfg, const uint8_t *codes, const uint8_t *exps, int32_t vocab, const void *z, int64_t z_stride,
                                int32_t B, const float *logits, const char **msg, const void *g_final = nullptr)
{
    const int64_t d = cfg.d_model;
    *msg = "null pointer";
    if (!codes || !exps || !z || !logits) return RT_ERR_INVALID_ARG;
    *msg = "1 <= vocab < 2^31 - 64, 1 <= B <= max_batch and z_stride >= d_model are required";
    if (vocab < 1 || vocab >= INT32_MAX - 63 || B < 1 || B > cfg.max_batch || z_stride < d || z_stride > (int64_t)1 << 40) return RT_ERR_INVALID_ARG;
    *msg = "the codes must lie on 16 bytes";
    if (!on16(codes)) return RT_ERR_INVALID_ARG;
    *msg = "rt_lm_head_mx4 covers d_model <= 25856";
    if (d > kMx4MaxWidth) return RT_ERR_UNSUPPORTED;
    const ByteRange l = {logits, (size_t)B * (size_t)vocab * 4};
    *msg = "logits must not overlap an input";
    if (ranges_meet(l, {z, (size_t)(((B - 1) * z_stride + d) * storage_bytes(cfg))}) ||
        ranges_meet(l, {codes, (size_t)vocab * (size_t)d / 2}) || ranges_meet(l, {exps, (size_t)vocab * (size_t)d / kMx4Block}) ||
        ranges_meet(l, {g_final, (size_t)(d * storage_bytes(cfg))}))
        return RT_ERR_INVALID_ARG;
    *msg = "";
    return RT_OK;
}

}  // namespace rt
