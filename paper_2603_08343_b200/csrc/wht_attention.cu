// C ABI of the serving attention (see include/wht_attention.h): argument checks and the split of work.
#include <algorithm>

#include "attn_host.h"
#include "kv_append_kernels.cuh"
#include "select_kernels.cuh"

namespace {

using namespace wht_host;
using wht::AppendParams;
using wht::AttnParams;
using wht::SelectParams;
using wht::UmmaAttnParams;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
size_t elem(int dtype) { return dtype == WHT_F32 ? 4 : 2; }
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

int page_shift_of(int32_t page) { return page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : page == 128 ? 7 : -1; }

// Rows of a strided [T x H x D] tensor start on 16-byte boundaries.
bool strides_ok(const void* p, int64_t st, int64_t sh, int dtype) {
    const int64_t unit = 16 / static_cast<int64_t>(elem(dtype));
    return aligned16(p) && st % unit == 0 && sh % unit == 0;
}

int check_shape(int64_t T, int32_t Hq, int32_t Hkv, int32_t D, int64_t num_pages, int32_t page, int dtype) {
    if (dtype != WHT_F32 && dtype != WHT_BF16) return WHT_ERR_BAD_DTYPE;
    if (D != 64 && D != 96 && D != 128) return WHT_ERR_BAD_DIM;
    if (Hkv < 1 || Hq < Hkv || Hq % Hkv != 0 || Hq / Hkv > 64 || Hq > 65536) return WHT_ERR_BAD_DIM;
    // (tiled copies count a cache's rows in 31 bits; one of more rows would not fit the device's memory)
    if (page_shift_of(page) < 0 || num_pages < 0 || num_pages > 0x7fffffff / page / Hkv) return WHT_ERR_BAD_DIM;
    if (T < 0 || T * Hq > 0x7fffffff) return WHT_ERR_BAD_T;
    return WHT_OK;
}

int check_batch(int64_t T, int32_t B, int32_t max_q_len, int32_t table_width, int32_t page, bool ragged) {
    if (B < 0 || max_q_len < 1 || table_width < 0 || static_cast<int64_t>(table_width) * page > 0x7fffffff) return WHT_ERR_BAD_DIM;
    if (max_q_len > (1 << 20) || (!ragged && (T != B || max_q_len != 1))) return WHT_ERR_BAD_T;
    return WHT_OK;
}

// 8-row tiles per unit of the paged kernel
int row_tiles(int64_t rows) { return rows <= 8 ? 1 : rows <= 16 ? 2 : 4; }

// How the paged kernel divides a set of units of up to `keys` keys: warps per unit, and key ranges (splits).
// No warp gets fewer than four 16-key chunks: its own set-up and the join would cost more than they save.
struct Division {
    int wpu, splits;
};
// bf16 units of one 8-row tile: twelve warps an SM can be resident, seven or eight take all that memory gives, and a second wave that
// the units do not fill costs more than it brings.  So as many warps per unit, then ranges, as stay within one wave of up to
// 8.75 warps an SM.  D = 128, 8 key heads, us for (warps . ranges): 64 sequences x 2048 keys 98 (1.1) 82.6 (2.1) 94 (4.1) 90.6 (4.2); 8 x 16384
// 180 (4.1) 98.6 (4.2) 85.6 (4.4) 89.4 (4.6); 32 x 4096 96.5 (2.1) 82.2 (4.1) 98 (4.2); 128 x 1024 86.5 (1.1) 96 (2.1).  Beyond
// one wave long lists take four warps (200 x 2048: 237, with one 247), short ones a warp each (no join, no waiting).
// More rows or fp32: eight (four) warps are resident, bound by products as well.
Division divide(int64_t units, int64_t keys, int nr, int dtype, int sms) {
    const int64_t chunks = ceil_div(keys, 16);
    Division d{1, 1};
    if (nr == 1 && dtype == WHT_BF16) {
        const int64_t wave = 35ll * sms / 4;
        if (units > wave) return Division{chunks >= 32 && units <= 24 * sms ? 4 : 1, 1};
        while (d.wpu < 4 && units * d.wpu * 2 <= wave && chunks >= 4 * 2 * d.wpu) d.wpu *= 2;
        if (d.wpu == 4) d.splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(8ll * sms / (units * 4), chunks / 16)));
        return d;
    }
    const int64_t slots = 8ll * sms;
    while (d.wpu < 4 && units * d.wpu < 3 * slots && chunks >= 4 * 2 * d.wpu) d.wpu *= 2;
    if (d.wpu == 4) d.splits = static_cast<int>(std::max<int64_t>(1, std::min(slots / (units * 4), chunks / 16)));
    return d;
}

// Whether each unit gets a block of eight warps, so that nothing is left to join: short lists, and few enough units that fill the
// machine at a block each.  us, in brackets with four warps a unit and ranges, 8 key heads of 4 rows, D = 128:
//   own pages  bf16  1 x 512 keys 8.5 (12.8), 1 x 2048 18.5 (12.4), 4 x 4096 30.8 (21.8), 9 x 2048 20.5 (22.7), 18 x 8192 97 (102)
//              fp32  1 x 1024 32.9 (18.5), 9 x 8192 237 (180), 18 x 512 27 (37), 18 x 8192 243 (342), 40 tokens of 2 x 512 (80 units) 61 (102)
//   selection  bf16  1 x 1024 16.4 (20.5), 1 x 2048 23.5 (18.8), 9 x 2048 27.1 (31.8), 18 x 2048 39.0 (43.4)
//              fp32  1 x 256 18.6 (21.2), 1 x 512 25.4 (24.7), 1 x 1024 37.3 (25.9), 18 x 1024 47.8 (63.9)
bool block_each(int64_t units, int64_t keys, int dtype, int sms) {
    const bool f32 = dtype == WHT_F32;
    const int64_t chunks = ceil_div(keys, 16 * 8);  // of a warp
    return units <= sms && (chunks <= (f32 ? 3 : 8) || (f32 ? 2 * units > sms : 4 * units > 3 * sms));
}

struct PrefixPlan {
    int prefix_nr, prefix_row_tiles, prefix_wpu, prefix_splits, own_nr, own_row_tiles, own_wpu, own_splits, parts;
    bool joint;                                 // small: every sequence walks the prefix itself
    bool umma;                                  // the prefix on the tcgen05 kernel
    int umma_splits, umma_row_blocks, same_rows;
    size_t bytes;
};

// Rows per key head from which the tcgen05 kernel takes the prefix.  Up to 32 rows are one unit of the paged kernel, which then reads
// each key once as well (16 heads x 16384 keys: 32 rows 48 us, here 46); above, it reads them once per 32 rows (48 rows: 63 us, here 49).
constexpr int kUmmaMinRows = 33;
constexpr int kUmmaMinKeys = 256;

// Key ranges of the tcgen05 kernel: the number that makes the whole call shortest by a small model of it.  Its blocks take an
// SM each; the sequences' own pages (own_bytes of keys and values) run beside it on the SMs that are left, then on all.
// Measured at 1.5 GHz under load: 6 us for a block's set-up and result and 1.8 (D = 64) to 2.2 us per tile of 128 keys;
// 54 GB/s per SM for the own pages next to it, 6000 GB/s alone.  256 x 32768 keys with 150 keys of their own, 32 heads: 3 ranges
// (96 blocks) are best, 4 (128 blocks) take 5% more, 9 (two waves) 12% more; 64 x 8192 with 256, 8 key heads: 10 ranges 40.5 us,
// 11 42.7 us, 15 45 us, 18 53 us.
int umma_splits_for(int64_t units, int64_t tiles, int tiles_per_step, int32_t D, double own_bytes, int sms) {
    const double tile_us = (D > 64 ? 2.2 : 1.8) * tiles_per_step;
    double best_us = 1e30;
    int best = 1;
    for (int64_t n = 1; n <= tiles && n <= 64; ++n) {
        const int64_t blocks = units * n, waves = ceil_div(blocks, sms);
        const double umma_us = static_cast<double>(waves) * (6.0 + tile_us * static_cast<double>(ceil_div(tiles, n)));
        const double beside = waves == 1 ? 54e3 * static_cast<double>(sms - blocks) * umma_us : 0.0;  // bytes
        const double us = umma_us + (own_bytes > beside ? (own_bytes - beside) / 6e6 : 0.0);
        if (us < best_us) {
            best_us = us;
            best = static_cast<int>(n);
        }
    }
    return best;
}

PrefixPlan plan_prefix(int64_t prefix_len, int32_t table_width, int64_t T, int32_t B, int32_t max_q_len, int32_t Hq, int32_t Hkv,
                       int32_t D, int32_t page, int dtype, bool umma_allowed, int sms) {
    PrefixPlan f{};
    const int group = Hq / Hkv;
    const int64_t own_rows = static_cast<int64_t>(max_q_len) * group;
    f.own_nr = row_tiles(own_rows);
    f.own_row_tiles = static_cast<int>(ceil_div(own_rows, 8 * f.own_nr));
    const Division own = divide(static_cast<int64_t>(B) * Hkv * f.own_row_tiles, static_cast<int64_t>(table_width) * page, f.own_nr, dtype, sms);
    f.own_wpu = own.wpu;
    f.own_splits = own.splits;
    f.prefix_nr = f.prefix_wpu = 1;
    if (prefix_len == 0 && block_each(static_cast<int64_t>(B) * Hkv * f.own_row_tiles, static_cast<int64_t>(table_width) * page, dtype, sms)) {
        f.own_wpu = 8;
        f.own_splits = 1;
    }
    // Small calls are all latency: one launch in which eight warps per unit walk the prefix and then the sequence's own pages beats a
    // prefix part and a join as long as no warp has more than 6 chunks (fp32, whose chunks take twice as long and more: 2) and the units
    // fit the machine at once.  2 sequences x 16 heads, D = 64, 40 own keys: 512 prefix keys 8.2 us against 10.3, 1000 keys 10.3
    // both, 2000 keys 14.4 against 11.3; fp32: 128 keys 8.3 against 12.3, 512 keys 14.4 against 12.3.
    const int64_t own_units = static_cast<int64_t>(B) * Hkv * f.own_row_tiles;
    const int64_t all_keys = prefix_len + static_cast<int64_t>(table_width) * page;
    f.joint = prefix_len > 0 && own_units <= sms && all_keys <= 16 * 8 * (dtype == WHT_F32 ? 2 : 6);
    if (f.joint) {
        f.own_wpu = 8;
        f.own_splits = f.parts = 1;
        return f;
    }
    f.umma = umma_allowed && dtype == WHT_BF16 && T * group >= kUmmaMinRows && prefix_len >= kUmmaMinKeys;
    if (f.umma) {
        f.same_rows = T * group <= 128;
        f.umma_row_blocks = static_cast<int>(ceil_div(T * group, 256));
        // with the same rows in both tiles a block takes two key tiles at a time
        // (the lengths are on the device: sequences are taken to fill 0.6 of their tables' width)
        const double own_bytes = 0.6 * B * Hkv * static_cast<double>(table_width) * page * D * 4.0;
        f.umma_splits = umma_splits_for(static_cast<int64_t>(Hkv) * f.umma_row_blocks, ceil_div(prefix_len, f.same_rows ? 256 : 128),
                                        1, D, own_bytes, sms);
    } else if (prefix_len > 0) {
        f.prefix_nr = row_tiles(T * group);
        f.prefix_row_tiles = static_cast<int>(ceil_div(T * group, 8 * f.prefix_nr));
        const Division pre = divide(static_cast<int64_t>(f.prefix_row_tiles) * Hkv, prefix_len, f.prefix_nr, dtype, sms);
        f.prefix_wpu = pre.wpu;
        f.prefix_splits = pre.splits;
    }
    f.parts = f.prefix_splits + f.own_splits + (f.same_rows ? 2 : 1) * f.umma_splits;
    const size_t rows = static_cast<size_t>(T) * Hq;
    f.bytes = f.parts > 1 ? up256(rows * f.parts * sizeof(float2)) + rows * f.parts * D * sizeof(float) : 0;
    return f;
}

struct SelectPlan {
    int nr, row_tiles, wpu, splits;
    size_t scores_bytes, bytes;
};

SelectPlan plan_select(int32_t table_width, int32_t select, int64_t T, int32_t Hq, int32_t Hkv, int32_t D, int32_t page, int dtype, int sms) {
    SelectPlan f{};
    const int group = Hq / Hkv;
    f.nr = row_tiles(group);
    f.row_tiles = static_cast<int>(ceil_div(group, 8 * f.nr));
    const int64_t units = T * Hkv * f.row_tiles, keys = static_cast<int64_t>(std::min(select, table_width)) * page;
    Division d = divide(units, keys, f.nr, dtype, sms);
    if (block_each(units, keys, dtype, sms)) d = Division{8, 1};
    f.wpu = d.wpu;
    f.splits = d.splits;
    f.scores_bytes = up256(static_cast<size_t>(T) * Hkv * table_width * sizeof(int32_t));
    const size_t rows = static_cast<size_t>(T) * Hq;
    f.bytes = f.scores_bytes + (f.splits > 1 ? up256(rows * f.splits * sizeof(float2)) + rows * f.splits * D * sizeof(float) : 0);
    return f;
}

void set_parts(AttnParams& p, unsigned char* at, int64_t rows) {
    if (p.parts <= 1) return;
    p.part_ml = reinterpret_cast<float2*>(at);
    p.part_o = reinterpret_cast<float*>(at + up256(static_cast<size_t>(rows) * p.parts * sizeof(float2)));
}

int join(const AttnParams& p, int dtype, int32_t D, cudaStream_t s) {
    if (p.parts <= 1) return WHT_OK;
    return dtype == WHT_F32 ? launch_attn_join<float>(p, D, s) : launch_attn_join<__nv_bfloat16>(p, D, s);
}

}  // namespace

extern "C" {

int wht_kv_append(const void* k, int64_t k_stride_t, int64_t k_stride_h, const void* v, int64_t v_stride_t, int64_t v_stride_h,
                  const void* q, int64_t q_stride_t, int64_t q_stride_h, void* q_out, const int64_t* slots,
                  const int32_t* positions, const float* cos_table, const float* sin_table, void* k_cache, void* v_cache,
                  int8_t* summary, const float* summary_scale, int64_t T, int32_t Hq, int32_t Hkv, int32_t D, int32_t rot,
                  int32_t interleaved, int64_t max_pos, int64_t num_pages, int32_t page, int dtype, void* stream) {
    int rc = check_shape(T, q ? Hq : Hkv, Hkv, D, num_pages, page, dtype);
    if (rc != WHT_OK) return rc;
    if (rot < 0 || rot > D || rot % 16 != 0 || (rot > 0 && max_pos < 1)) return WHT_ERR_BAD_DIM;
    if ((q == nullptr) != (q_out == nullptr)) return WHT_ERR_NULL;
    if (T == 0) return WHT_OK;
    if (!k || !v || !slots || !k_cache || !v_cache) return WHT_ERR_NULL;
    if (rot > 0 && (!positions || !cos_table || !sin_table)) return WHT_ERR_NULL;
    if (summary && !summary_scale) return WHT_ERR_NULL;
    if (!strides_ok(k, k_stride_t, k_stride_h, dtype) || !strides_ok(v, v_stride_t, v_stride_h, dtype) ||
        (q && !strides_ok(q, q_stride_t, q_stride_h, dtype)) || !aligned16(q_out) || !aligned16(k_cache) || !aligned16(v_cache) ||
        !aligned16(summary) || !aligned16(cos_table) || !aligned16(sin_table))
        return WHT_ERR_MISALIGNED;
    int dev = 0, sms = 0;
    rc = device_info(&dev, &sms);
    if (rc != WHT_OK) return rc;
    AppendParams p{};
    p.k = k; p.v = v; p.q = q;
    p.k_st = k_stride_t; p.k_sh = k_stride_h;
    p.v_st = v_stride_t; p.v_sh = v_stride_h;
    p.q_st = q_stride_t; p.q_sh = q_stride_h;
    p.q_out = q_out; p.k_cache = k_cache; p.v_cache = v_cache;
    p.slots = slots; p.positions = positions; p.cos_t = cos_table; p.sin_t = sin_table;
    p.summary = summary; p.summary_scale = summary_scale;
    p.T = T; p.max_pos = max_pos; p.num_slots = num_pages * page;
    p.hq = q ? Hq : 0; p.hkv = Hkv; p.d = D; p.rot = rot; p.page_shift = page_shift_of(page);
    return launch_append(p, dtype, interleaved != 0, sms, static_cast<cudaStream_t>(stream));
}

size_t wht_attn_prefix_workspace_bytes(int64_t prefix_len, int32_t table_width, int64_t T, int32_t B, int32_t max_q_len, int32_t Hq,
                                       int32_t Hkv, int32_t D, int32_t page, int dtype) {
    int dev = 0, sms = 0;
    if (check_shape(T, Hq, Hkv, D, 0, page, dtype) != WHT_OK || check_batch(T, B, max_q_len, table_width, page, true) != WHT_OK ||
        prefix_len < 0 || device_info(&dev, &sms) != WHT_OK)
        return 0;
    // either form of the prefix may be taken (the tcgen05 one has conditions that are not known here)
    return std::max(plan_prefix(prefix_len, table_width, T, B, max_q_len, Hq, Hkv, D, page, dtype, true, sms).bytes,
                    plan_prefix(prefix_len, table_width, T, B, max_q_len, Hq, Hkv, D, page, dtype, false, sms).bytes);
}

int wht_attn_prefix(const void* q, int64_t q_stride_t, int64_t q_stride_h, const void* k_cache, const void* v_cache,
                    const int32_t* prefix_pages, int64_t prefix_len, const int32_t* page_table, int32_t table_width,
                    const int32_t* kv_lens, const int32_t* q_start, void* out, int64_t T, int32_t B, int32_t max_q_len,
                    int32_t Hq, int32_t Hkv, int32_t D, int64_t num_pages, int32_t page, float scale, int dtype,
                    void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_shape(T, Hq, Hkv, D, num_pages, page, dtype);
    if (rc == WHT_OK) rc = check_batch(T, B, max_q_len, table_width, page, q_start != nullptr);
    if (rc != WHT_OK) return rc;
    if (prefix_len < 0 || prefix_len > 0x7fffff00) return WHT_ERR_BAD_T;
    if (T == 0) return WHT_OK;
    if (!q || !k_cache || !v_cache || !out || !kv_lens || (table_width > 0 && !page_table) || (prefix_len > 0 && !prefix_pages))
        return WHT_ERR_NULL;
    if (!strides_ok(q, q_stride_t, q_stride_h, dtype) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out) || !aligned16(workspace))
        return WHT_ERR_MISALIGNED;
    int dev = 0, sms = 0;
    rc = device_info(&dev, &sms);
    if (rc != WHT_OK) return rc;
    if (num_pages < 1) return WHT_ERR_BAD_DIM;
    const bool umma_allowed = scale > 0.0f;  // the tcgen05 kernel finds a row's maximum before it scales
    const PrefixPlan f = plan_prefix(prefix_len, table_width, T, B, max_q_len, Hq, Hkv, D, page, dtype, umma_allowed, sms);
    if (f.bytes > 0 && (!workspace || workspace_bytes < f.bytes)) return WHT_ERR_WORKSPACE;
    AttnParams p{};
    p.q = q; p.k_cache = k_cache; p.v_cache = v_cache;
    p.q_st = q_stride_t; p.q_sh = q_stride_h;
    p.out = out;
    p.parts = f.parts;
    set_parts(p, static_cast<unsigned char*>(workspace), T * Hq);
    p.prefix_pages = prefix_pages; p.prefix_len = prefix_len;
    p.prefix_splits = f.prefix_splits; p.prefix_row_tiles = f.prefix_row_tiles; p.prefix_nr = f.prefix_nr; p.prefix_wpu = f.prefix_wpu;
    p.page_table = page_table; p.kv_lens = kv_lens; p.q_start = q_start;
    p.table_width = table_width; p.B = B; p.max_q_len = max_q_len;
    p.own_splits = f.own_splits; p.own_row_tiles = f.own_row_tiles; p.own_nr = f.own_nr; p.own_wpu = f.own_wpu;
    p.joint = f.joint;
    p.T = T; p.num_pages = num_pages;
    p.hq = Hq; p.hkv = Hkv; p.group = Hq / Hkv; p.page_shift = page_shift_of(page);
    p.scale_log2 = scale * wht::kLog2e;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (f.umma) {
        const UmmaAttnParams up{p, f.umma_splits, f.umma_row_blocks, f.same_rows};
        rc = launch_attn_umma_prefix(up, D, dev, s);
        if (rc != WHT_OK) return rc;
    }
    rc = dtype == WHT_F32 ? launch_attn_prefix<float>(p, D, dev, f.umma, s) : launch_attn_prefix<__nv_bfloat16>(p, D, dev, f.umma, s);
    return rc != WHT_OK ? rc : join(p, dtype, D, s);
}

size_t wht_attn_select_workspace_bytes(int32_t table_width, int32_t select, int64_t T, int32_t B, int32_t max_q_len, int32_t Hq,
                                       int32_t Hkv, int32_t D, int32_t page, int dtype) {
    int dev = 0, sms = 0;
    if (check_shape(T, Hq, Hkv, D, 0, page, dtype) != WHT_OK || check_batch(T, B, max_q_len, table_width, page, true) != WHT_OK ||
        select < 1 || select > 1024 || device_info(&dev, &sms) != WHT_OK)
        return 0;
    return plan_select(table_width, select, T, Hq, Hkv, D, page, dtype, sms).bytes;
}

int wht_attn_select(const void* q, int64_t q_stride_t, int64_t q_stride_h, const void* k_cache, const void* v_cache,
                    const int8_t* summary, const int32_t* page_table, int32_t table_width, const int32_t* kv_lens,
                    const int32_t* q_start, int32_t select, void* out, int32_t* pages_out, int64_t T, int32_t B,
                    int32_t max_q_len, int32_t Hq, int32_t Hkv, int32_t D, int64_t num_pages, int32_t page, float scale,
                    int dtype, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_shape(T, Hq, Hkv, D, num_pages, page, dtype);
    if (rc == WHT_OK) rc = check_batch(T, B, max_q_len, table_width, page, q_start != nullptr);
    if (rc != WHT_OK) return rc;
    if (select < 1 || select > 1024 || table_width > 49152) return WHT_ERR_BAD_DIM;
    if (T == 0) return WHT_OK;
    if (num_pages < 1) return WHT_ERR_BAD_DIM;
    if (!q || !k_cache || !v_cache || !summary || !out || !pages_out || !kv_lens || (table_width > 0 && !page_table)) return WHT_ERR_NULL;
    if (!strides_ok(q, q_stride_t, q_stride_h, dtype) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(summary) ||
        !aligned16(out) || !aligned16(workspace))
        return WHT_ERR_MISALIGNED;
    int dev = 0, sms = 0;
    rc = device_info(&dev, &sms);
    if (rc != WHT_OK) return rc;
    const SelectPlan f = plan_select(table_width, select, T, Hq, Hkv, D, page, dtype, sms);
    if (f.bytes > 0 && (!workspace || workspace_bytes < f.bytes)) return WHT_ERR_WORKSPACE;
    SelectParams sp{};
    AttnParams& p = sp.a;
    p.q = q; p.k_cache = k_cache; p.v_cache = v_cache;
    p.q_st = q_stride_t; p.q_sh = q_stride_h;
    p.out = out;
    p.parts = f.splits;
    set_parts(p, static_cast<unsigned char*>(workspace) + f.scores_bytes, T * Hq);
    p.page_table = page_table; p.kv_lens = kv_lens; p.q_start = q_start;
    p.table_width = table_width; p.B = B; p.max_q_len = max_q_len;
    p.own_splits = f.splits; p.own_row_tiles = f.row_tiles; p.own_nr = f.nr; p.own_wpu = f.wpu;
    p.chosen = pages_out; p.select = select;
    p.T = T; p.num_pages = num_pages;
    p.hq = Hq; p.hkv = Hkv; p.group = Hq / Hkv; p.page_shift = page_shift_of(page);
    p.scale_log2 = scale * wht::kLog2e;
    sp.summary = summary;
    sp.scores = static_cast<int32_t*>(workspace);
    sp.pages = pages_out;
    sp.stride = table_width;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    rc = launch_select(sp, dtype, D, s);
    if (rc == WHT_OK) rc = dtype == WHT_F32 ? launch_attn_chosen<float>(p, D, dev, s) : launch_attn_chosen<__nv_bfloat16>(p, D, dev, s);
    return rc != WHT_OK ? rc : join(p, dtype, D, s);
}

int wht_attn_device_status(void) {
    unsigned any = 0;
    for (auto take : {take_attn_error_append, take_attn_error_paged_bf16, take_attn_error_paged_f32, take_attn_error_select,
                      take_attn_error_umma}) {
        unsigned flag = 0;
        const int rc = take(&flag);
        if (rc != WHT_OK) return rc;
        any |= flag;
    }
    for (auto take : {take_device_error_attn_umma, take_device_error_attn_paged_bf16, take_device_error_attn_paged_f32}) {
        unsigned waits = 0;
        const int rc = take(&waits);
        if (rc != WHT_OK) return rc;
        if (waits) any |= wht::kAttnErrWait;
    }
    return any & wht::kAttnErrIndex ? WHT_ERR_DEVICE_INDEX : any ? WHT_ERR_DEVICE_WAIT : WHT_OK;
}

}  // extern "C"
