// How a call of the serving attention divides its work: warps per unit, key ranges, which kernel takes the prefix, and the workspace
// that follows from it.  Host arithmetic alone (no CUDA), so that every shape can be checked without a device.
#pragma once
#include <algorithm>
#include <cstddef>
#include <cstdint>

#include "../../include/wht_attention.h"

namespace wht_plan {

inline long long div_up(long long a, long long b) { return (a + b - 1) / b; }
inline size_t up256(size_t n) { return (n + 255) / 256 * 256; }
constexpr size_t kPartStats = 2 * sizeof(float);  // a partial result's maximum and sum

// 8-row tiles per unit of the paged kernel
inline int row_tiles(int64_t rows) { return rows <= 8 ? 1 : rows <= 16 ? 2 : 4; }

// How the paged kernel divides a set of units (one at least) of up to `keys` keys: warps per unit, and key ranges (splits).
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
inline Division divide(int64_t units, int64_t keys, int nr, int dtype, int sms) {
    const int64_t chunks = div_up(keys, 16);
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
inline bool block_each(int64_t units, int64_t keys, int dtype, int sms) {
    const bool f32 = dtype == WHT_F32;
    const int64_t chunks = div_up(keys, 16 * 8);  // of a warp
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
inline int umma_splits_for(int64_t units, int64_t tiles, int32_t D, double own_bytes, int sms) {
    const double tile_us = D > 64 ? 2.2 : 1.8;
    double best_us = 1e30;
    int best = 1;
    for (int64_t n = 1; n <= tiles && n <= 64; ++n) {
        const int64_t blocks = units * n, waves = div_up(blocks, sms);
        const double umma_us = static_cast<double>(waves) * (6.0 + tile_us * static_cast<double>(div_up(tiles, n)));
        const double beside = waves == 1 ? 54e3 * static_cast<double>(sms - blocks) * umma_us : 0.0;  // bytes
        const double us = umma_us + (own_bytes > beside ? (own_bytes - beside) / 6e6 : 0.0);
        if (us < best_us) {
            best_us = us;
            best = static_cast<int>(n);
        }
    }
    return best;
}

inline PrefixPlan plan_prefix(int64_t prefix_len, int32_t table_width, int64_t T, int32_t B, int32_t max_q_len, int32_t Hq, int32_t Hkv,
                              int32_t D, int32_t page, int dtype, bool umma_allowed, int sms) {
    PrefixPlan f{};
    if (T == 0) return f;  // nothing is launched
    const int group = Hq / Hkv;
    const int64_t own_rows = static_cast<int64_t>(max_q_len) * group;
    f.own_nr = row_tiles(own_rows);
    f.own_row_tiles = static_cast<int>(div_up(own_rows, 8 * f.own_nr));
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
        f.umma_row_blocks = static_cast<int>(div_up(T * group, 256));
        // with the same rows in both tiles a block takes two key tiles at a time
        // (the lengths are on the device: sequences are taken to fill 0.6 of their tables' width)
        const double own_bytes = 0.6 * B * Hkv * static_cast<double>(table_width) * page * D * 4.0;
        f.umma_splits = umma_splits_for(static_cast<int64_t>(Hkv) * f.umma_row_blocks, div_up(prefix_len, f.same_rows ? 256 : 128),
                                        D, own_bytes, sms);
    } else if (prefix_len > 0) {
        f.prefix_nr = row_tiles(T * group);
        f.prefix_row_tiles = static_cast<int>(div_up(T * group, 8 * f.prefix_nr));
        const Division pre = divide(static_cast<int64_t>(f.prefix_row_tiles) * Hkv, prefix_len, f.prefix_nr, dtype, sms);
        f.prefix_wpu = pre.wpu;
        f.prefix_splits = pre.splits;
    }
    f.parts = f.prefix_splits + f.own_splits + (f.same_rows ? 2 : 1) * f.umma_splits;
    const size_t rows = static_cast<size_t>(T) * Hq;
    f.bytes = f.parts > 1 ? up256(rows * f.parts * kPartStats) + rows * f.parts * D * sizeof(float) : 0;
    return f;
}

struct SelectPlan {
    int nr, row_tiles, wpu, splits;
    bool one_kernel;       // scores and picks in one kernel, which needs no memory for the scores
    size_t scores_bytes, bytes;
};

inline SelectPlan plan_select(int32_t table_width, int32_t select, int64_t T, int32_t B, int32_t max_q_len, int32_t Hq, int32_t Hkv,
                              int32_t D, int32_t page, int dtype, int sms) {
    SelectPlan f{};
    if (T == 0) return f;  // nothing is launched
    const int group = Hq / Hkv;
    f.nr = row_tiles(group);
    f.row_tiles = static_cast<int>(div_up(group, 8 * f.nr));
    const int64_t units = T * Hkv * f.row_tiles, keys = static_cast<int64_t>(std::min(select, table_width)) * page;
    Division d = divide(units, keys, f.nr, dtype, sms);
    if (block_each(units, keys, dtype, sms)) d = Division{8, 1};
    f.wpu = d.wpu;
    f.splits = d.splits;
    // One kernel where its blocks' scores fit shared memory, unless a few blocks would have to read long tables alone.  Whole call, 8 key
    // heads, pages of 16, one kernel against two: 1 x 256 pages 15.9 us (17.2), 1 x 512 18.6 (18.2), 1 x 1024 29.5 (20.6), 1 x 2048 43.0 (21.3), 4 x 2048
    // 42.5 (32.3), 16 x 2048 57.0 (51.1), 64 x 2048 100.7 (105.3), 300 prompt tokens of 1500 pages 110 (163).
    const int tq = max_q_len == 1 ? 1 : 16;  // queries of a block
    const int64_t blocks = static_cast<int64_t>(B) * div_up(max_q_len, tq) * Hkv;
    f.one_kernel = static_cast<int64_t>(table_width) * tq * 4 <= 96 * 1024 && (table_width <= 512 || blocks >= 128);
    f.scores_bytes = f.one_kernel ? 0 : up256(static_cast<size_t>(T) * Hkv * table_width * sizeof(int32_t));
    const size_t rows = static_cast<size_t>(T) * Hq;
    f.bytes = f.scores_bytes + (f.splits > 1 ? up256(rows * f.splits * kPartStats) + rows * f.splits * D * sizeof(float) : 0);
    return f;
}

}  // namespace wht_plan
