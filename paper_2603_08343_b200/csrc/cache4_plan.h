// How a call of the attention over the 4-bit cache divides its work, and the workspace that follows from it.  Host arithmetic alone (no
// CUDA), so that every shape can be checked without a device.
#pragma once
#include <cmath>

#include "attn_plan.h"

namespace wht_plan {

// 8-row tiles of a unit.  (Four take a quarter of the instructions for the codes, but 255 registers, so that eight warps fit an SM: 8 x 64 questions over 5000
// keys 62 us against 51, 100 tokens over 1000 25 us against 11; only 128 tokens over 30000 keys, 242 against 271, are better off.)
inline int row_tiles4(int64_t rows) { return rows <= 8 ? 1 : 2; }
// One-warp blocks that an SM holds at once.
constexpr int resident4(int row_tiles, bool f32) { return row_tiles * (f32 ? 2 : 1) > 2 ? 8 : row_tiles * (f32 ? 2 : 1) > 1 ? 12 : 16; }

constexpr int kLeastRun4 = 8;  // tiles of 16 keys: a shorter run would not pay for its start and its part of the join
constexpr int kGrain4 = 1;     // log2 of the tiles in which work is counted: a step of the kernel takes two

// Prompts of bf16 queries on tcgen05: rows of a unit, log2 of the tiles of a grain (a step takes 64 keys), blocks that an SM holds.
constexpr int kUmma4Rows = 256, kUmma4Grain = 2, kUmma4Resident = 1;
// Whether the tcgen05 kernel is the faster one, by a small model of both, in us (D = 128; less for fewer channels): a start of 28, 1.75 a step of 256 rows and
// 64 keys in a block and 8 a further unit of it, against 10 and 0.085 an SM for 16 rows and 16 keys in the kernel of few rows.  Lengths are on the device: as
// if the tokens were spread evenly and the tables full, with a quarter in hand, since lengths that are not favour the kernel of few rows.
// us, tcgen05 and the other: 128 tokens of 4 rows over 30000 keys, 8 key heads, 121 (275); 2048 over 4000 219 (528); 64 over 20000 66 (108); 100 over 10000
// 61 (86); 16 x 128 over up to 2000 100 (138); 8 x 64 over up to 5000, 4 key heads, D = 96, 54 (54); 400 over 800 39 (41); 256 over 300 25 (25).
inline bool umma4_pays(int64_t keys, int64_t T, int32_t B, int group, int32_t Hkv, int32_t D, int sms) {
    const int64_t rows = (T + B - 1) / B * group;
    const double heads = static_cast<double>(B) * Hkv, k = static_cast<double>(keys);
    const double units = heads * static_cast<double>((rows + kUmma4Rows - 1) / kUmma4Rows), units_few = heads * static_cast<double>((rows + 15) / 16);
    const double umma = 12.0 + D / 8.0 + (0.45 + 0.0102 * D) * std::ceil(units * (k / 64) / sms) + 8.0 * units / sms;
    const double other = 10.0 + (0.045 + D / 3200.0) * units_few * (k / 16) / sms;
    return 1.25 * umma < other;
}

struct Attend4Plan {
    bool umma;
    int row_tiles, warps, grain, least, part_rows;
    size_t ml_bytes, o_bytes, lse_bytes, scores_bytes, bytes;
};

inline Attend4Plan plan_attend4(int32_t table_width, int64_t T, int32_t B, int32_t max_q_len, int32_t Hq, int32_t Hkv, int32_t D,
                                int32_t page, int dtype, bool weigh, int sms) {
    Attend4Plan f{};
    if (T == 0) return f;
    const int group = Hq / Hkv;
    f.umma = dtype == WHT_BF16 && static_cast<int64_t>(max_q_len) * group > 16 && umma4_pays(static_cast<int64_t>(table_width) * page, T, B, group, Hkv, D, sms);
    f.row_tiles = row_tiles4(static_cast<int64_t>(max_q_len) * group);
    const int rows = f.umma ? kUmma4Rows : 8 * f.row_tiles;
    f.part_rows = static_cast<int>(std::min<int64_t>(rows, static_cast<int64_t>(max_q_len) * group));
    // as many runs as fit the machine at once, unless the tables hold too few keys for that
    // (a sequence's last row tile may be a short one; offsets that let sequences overlap, which no call should have, may make for more units: the
    // kernels then stay within their bounds)
    const double units = static_cast<double>(Hkv) * std::min(static_cast<double>(B) * div_up(std::min<int64_t>(max_q_len, T) * group, rows),
                                                             static_cast<double>(div_up(T * group, rows) + B));
    const double tiles = units * static_cast<double>(std::max<int64_t>(1, static_cast<int64_t>(table_width) * page / 16));
    const double runs = std::max(1.0, tiles / kLeastRun4 + 1.0);
    const int most = sms * (f.umma ? kUmma4Resident : resident4(f.row_tiles, dtype == WHT_F32));
    f.warps = runs < most ? static_cast<int>(runs) : most;
    // grains are counted in 32 bits, with room for a run's worth beyond the last (wide tables of many sequences take larger ones)
    f.grain = f.umma ? kUmma4Grain : kGrain4;
    while (units * static_cast<double>(div_up(static_cast<int64_t>(table_width) * page, 16ll << f.grain) + 1) > 2147483647.0 && f.grain < 26) ++f.grain;
    f.least = std::max(1, kLeastRun4 >> f.grain);
    f.ml_bytes = up256(static_cast<size_t>(2) * f.warps * f.part_rows * kPartStats);
    f.o_bytes = static_cast<size_t>(2) * f.warps * f.part_rows * D * sizeof(float);
    f.lse_bytes = weigh ? up256(static_cast<size_t>(T) * Hq * sizeof(float)) : 0;
    // the scores of few rows are kept for the received weight, in a gigabyte at most
    const double scores = 4.0 * f.part_rows * B * Hkv * static_cast<double>(table_width) * page;
    f.scores_bytes = weigh && f.row_tiles == 1 && scores <= 1073741824.0 ? static_cast<size_t>(scores) : 0;
    f.bytes = f.ml_bytes + up256(f.o_bytes) + f.lse_bytes + f.scores_bytes;
    return f;
}

}  // namespace wht_plan
