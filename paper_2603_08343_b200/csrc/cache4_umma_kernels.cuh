// Attention of prompts over the cache held in 4 bits, on the tcgen05 tensor core (bf16 queries).
//
// The formulas are those of cache4_attend_kernels.cuh.  A unit is 256 rows (token, query head) of one sequence and key head, two tiles of 128, so that
// with the queries as one operand and the codes of 64 keys as the other both products are dense:
//     S = Q C^T (bf16: codes 0 .. 15 are exact)    P = exp2(score - m) step' as fp16, over S in tensor memory    O += P (C' - z) (fp16)
// with O in tensor memory too.  Codes become numbers on their way from the cache to shared memory, once per 256 rows: a half word masked and
// joined with the exponent of 128 (bf16) or 1024 (fp16), less that number (and, of a value, less z); values' odd codes stay 16 times too large until the end.
// The tensor core truncates as it adds: every kFoldUmma4 steps a row's O moves to a sum in the workspace, where it is added with rounding (512 tokens over
// 100000 keys 1115 us with it, 1091 without; every 32 steps 1161).
//
// A block of 13 warps has an SM to itself:
//   warps 0 .. 3, 4 .. 7  softmax of the two tiles, a row a thread; the queries, and the results
//   warps 8, 9            the codes of the keys of a step, a key a thread            warps 10, 11  of the values; and (step, lo) of both
//   warp 12               issues the products, the tiles in turn, so that one tile's softmax runs under the other's products
// K, V, S and P have two buffers each.  All roles walk the same runs of grains as the kernel for few rows, a run a block, and leave the same parts.
// The scores, and with them the weights, are all of a thread's own: the reference m moves without asking others, but for the
// reads and writes of O, which a warp makes together.
//
// Operands lie in the 128-byte swizzle: rows of 64 channels, 16-byte pieces permuted by the row.  Channels of a piece of keys stand in the
// order in which their codes fall out of a word, and so do the queries'; the results' are put right when they are written.
//
// What bounds it: the softmax warps.  A step of both tiles takes 2800 clocks, 2100 of them the weights of 64 keys (64 exponentials, 7 packed operations a pair of
// keys, two of a warp's reads of (step, lo)), 1000 the products.  128 tokens of 32 heads over 30000 keys of 8 key heads 121 us (0.5 PFLOP/s; 275 in the kernel of few rows),
// 2048 tokens over 4000 219 us (528).  Slower: blocks of one tile, two an SM (96 registers a thread, 150 us), the issuing warp's loops not unrolled (a product
// takes 100 clocks to issue, 133 us), (step, lo) unpacked by the softmax warps (147 us).
//
// Waits are bounded as in umma_kernels.cuh.
#pragma once
#include "attn_umma_kernels.cuh"
#include "cache4_attend_kernels.cuh"

namespace wht {

constexpr int kUmma4Threads = 416;
constexpr int kUmma4Rows = 256, kUmma4Keys = 64;
constexpr float kMostUmma4 = 32768.0f;  // of the products of a row and 64 keys together
constexpr int kFoldUmma4 = 64;          // steps of which the tensor core holds the sum: 4096 keys

template <int D>
struct Umma4Geo {
    static constexpr int BOXES = D > 64 ? 2 : 1;              // of 64 channels
    static constexpr int Q_BOX = 128 * 128, BOX = kUmma4Keys * 128;
    static constexpr int TILE = BOXES * BOX;                  // 64 keys or values
    static constexpr int Q_TILE = BOXES * Q_BOX;              // 128 rows
    static constexpr int OFF_K = 2 * Q_TILE;
    static constexpr int OFF_V = OFF_K + 2 * TILE;
    static constexpr int OFF_ROWS = OFF_V + 2 * TILE;         // [2][32 pairs of keys][steps, los of the keys, of the values]
    static constexpr int OFF_BARS = OFF_ROWS + 2 * 1024;
    static constexpr int NBARS = 19;
    static constexpr int OFF_MISC = OFF_BARS + NBARS * 8;
    static constexpr int BYTES = OFF_MISC + 16;
    static constexpr int O_COLS = D > 64 ? 128 : 64;
};

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint32_t minus_bf162(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// Eight codes of a word as bf16 pairs (code i, code 4 + i), and less `even` as fp16 pairs, the odd ones times 16 (less `odd`).
__device__ __forceinline__ uint4 codes_bf16(uint32_t w) {
    auto two = [](uint32_t x) { return minus_bf162((x & 0x000f000fu) | 0x43004300u, 0x43004300u); };
    return make_uint4(two(w), two(w >> 4), two(w >> 8), two(w >> 12));
}
__device__ __forceinline__ uint4 codes_f16(uint32_t w, uint32_t even, uint32_t odd) {
    auto low = [&](uint32_t x) { return minus_half2((x & 0x000f000fu) | 0x64006400u, even); };
    auto high = [&](uint32_t x) { return minus_half2((x & 0x00f000f0u) | 0x64006400u, odd); };
    return make_uint4(low(w), high(w), low(w >> 8), high(w >> 8));
}
// Piece c of row r of an operand in the 128-byte swizzle, `box` bytes between blocks of 64 channels.
__device__ __forceinline__ int piece_of(int box, int r, int c) { return (c >> 3) * box + r * 128 + (((c & 7) ^ (r & 7)) << 4); }

// Two barriers at once.
__device__ __forceinline__ bool warp_poll_both(uint64_t* x, uint64_t* y, uint32_t parity, volatile uint32_t* abort_flag) {
    const bool there = mbar_try_wait(x, parity) & mbar_try_wait(y, parity);
    if (__all_sync(kFullMask, there)) return true;
    return warp_poll_or_abort(x, parity, abort_flag) && warp_poll_or_abort(y, parity, abort_flag);
}

template <int D>
__global__ void __launch_bounds__(kUmma4Threads, 1)
attn4_umma_kernel(const Attn4Params p) {
    using Geo = Umma4Geo<D>;
    extern __shared__ __align__(1024) unsigned char umma4_smem[];
    const AttnParams& a = p.a;
    unsigned char* smem = umma4_smem;
    if (smem_u32(smem) & 1023u) {  // the swizzle counts on it (dynamic shared memory starts on such a boundary)
        attn_report(kAttnErrWait);
        return;
    }
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + Geo::OFF_BARS);
    uint64_t *k_full = bars, *k_free = bars + 2, *v_full = bars + 4, *v_free = bars + 6;             // [buffer]
    uint64_t *s_full = bars + 8, *p_ready = bars + 12, *q_full = bars + 16, *all_done = bars + 18;    // [tile][buffer], q_full [tile]
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + Geo::OFF_MISC);
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(smem + Geo::OFF_MISC + 4);
    uint32_t* far = reinterpret_cast<uint32_t*>(smem + Geo::OFF_MISC + 8);      // [buffer] whether what z stands for is large for a value, a half word a warp
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(kFullMask, tid >> 5, 0);

    // (tensor memory is taken after the kernel before, which may want it too, and before the one after may start)
    grid_dependency_wait();
    if (warp == 12) {
        tmem_alloc(tmem_slot, 512);
        tmem_relinquish();
    }
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(k_full + i, 2);
            mbar_init(v_full + i, 2);
            mbar_init(k_free + i, 1);
            mbar_init(v_free + i, 1);
            mbar_init(q_full + i, 4);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(s_full + i, 1);
            mbar_init(p_ready + i, 4);
        }
        mbar_init(all_done, 1);
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (a.q_start != nullptr && warp == 8)
        for (int head = blockIdx.x; head < a.hkv; head += gridDim.x) attn_uncovered<__nv_bfloat16, D>(a, head);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(kFullMask, *tmem_slot, 0);
    grid_launch_dependents();                                        // (never before the wait: the join reads lengths and offsets ahead of its own)

    unsigned run;
    const Place4 home = find_run4(p, kUmma4Rows, blockIdx.x, run);
    const unsigned run_begin = run * blockIdx.x, run_end = min(run_begin + run, home.total);
    // Every role walks the run: f(segment, end, least limit, steps, number of the first step) returns whether to go on.
    auto walk = [&](auto f) {
        unsigned at = run_begin, before = home.before, first = 0;
        for (int b = home.b; at < run_end && b < a.B; ++b) {
            const Share4 s(a, b, kUmma4Rows, p.grain);
            const unsigned cost = s.cost(a.hkv);
            while (at < run_end && at - before < cost) {
                const unsigned unit = (at - before) / s.grains, start = before + unit * s.grains;
                Segment4 u;
                u.token0 = s.token0;
                u.count = s.count;
                u.keys = s.keys;
                u.table = a.page_table + static_cast<int64_t>(b) * a.table_width;
                u.head = static_cast<int>(unit / s.row_tiles);
                u.row0 = static_cast<int>(unit - u.head * s.row_tiles) * kUmma4Rows;
                const unsigned g0 = at - start, g1 = min(run_end - start, s.grains);
                u.tile0 = static_cast<int>(g0 << p.grain);
                u.tile1 = static_cast<int>(g1 << p.grain);
                u.slot = g0 > 0 ? 2ll * blockIdx.x : g1 < s.grains ? 2ll * blockIdx.x + 1 : -1;
                u.scores = nullptr;
                const int rows = u.count * a.group, first_limit = u.keys - u.count + 1;
                const int last_row = min(rows, u.row0 + kUmma4Rows) - 1;
                const int end = static_cast<int>(min(static_cast<int64_t>(u.tile1) * kTileKeys, static_cast<int64_t>(first_limit + last_row / a.group)));
                const int steps = max(0, (end - u.tile0 * kTileKeys + kUmma4Keys - 1) / kUmma4Keys);
                if (!f(u, end, steps, first)) return;
                first += steps;
                at = start + g1;
            }
            before += cost;
        }
    };

    if (warp >= 8 && warp < 12) {
        // codes of one key (value) a thread and step
        const bool values = warp >= 10;
        const int kk = tid & 63, j = kk & 15;
        const float zero_code = j & 1 ? 7.0f : 8.0f;                 // z of this key; 1024 + z and 1024 + 16 z, twice
        const uint32_t even = j & 1 ? 0x64076407u : 0x64086408u, odd = j & 1 ? 0x64706470u : 0x64806480u;
        constexpr int LOADS = D / 32;                                // 16 bytes each
        uint64_t *full = values ? v_full : k_full, *free_bar = values ? v_free : k_free;
        walk([&](const Segment4& u, int end, int steps, unsigned first) {
            const int shift = a.page_shift - 4, in_page = (1 << shift) - 1;
            const int last_tile = max(0, (end - 1) >> 4);
            // codes one step ahead, page numbers two
            uint4 raw[LOADS], next[LOADS];
            uint2 row = make_uint2(0, 0), next_row = make_uint2(0, 0);
            auto tile_of = [&](int i) { return min(u.tile0 + i * (kUmma4Keys / kTileKeys) + (kk >> 4), last_tile); };   // (behind the end: any key, nobody sees it)
            auto look = [&](int i) { return i < steps ? u.table[tile_of(i) >> shift] : 0; };
            auto fetch = [&](int i, int pg) {
                if (pg < 0 || pg >= a.num_pages) {
                    attn_report(kAttnErrIndex);
                    pg = 0;
                }
                const unsigned char* tile = p.cache + (((static_cast<int64_t>(pg) * a.hkv + u.head) << shift) + (tile_of(i) & in_page)) * tile4_bytes(D);
                if (!values) {
#pragma unroll
                    for (int n = 0; n < LOADS; ++n) next[n] = *(reinterpret_cast<const uint4*>(tile + j * (D / 2)) + n);
                } else {
                    const int place = value4_place(j);
#pragma unroll
                    for (int n = 0; n < LOADS; ++n)
                        next[n] = *reinterpret_cast<const uint4*>(tile + 8 * D + (D == 128 ? place * 64 + n * 16 : n < 2 ? place * 32 + n * 16 : 512 + place * 16));
                    next_row = *reinterpret_cast<const uint2*>(tile + tile4_rows(D) + j * 8);
                }
            };
            int page = look(0);
            if (steps > 0) fetch(0, page);
            page = look(1);
            for (int i = 0; i < steps; ++i) {
                const unsigned step = first + i, buf = step & 1, phase = (step >> 1) & 1;
#pragma unroll
                for (int n = 0; n < LOADS; ++n) raw[n] = next[n];
                row = next_row;
                if (i + 1 < steps) fetch(i + 1, page);
                page = look(i + 2);
                if (!warp_poll_or_abort(free_bar + buf, phase ^ 1u, abort_flag)) return false;
                unsigned char* to = smem + (values ? Geo::OFF_V : Geo::OFF_K) + buf * Geo::TILE;
                if (!values) {
                    // word [c4][g] holds the channels 32 g + 8 c4 .. + 7
#pragma unroll
                    for (int n = 0; n < LOADS * 4; ++n) {
                        const uint32_t w = n % 4 == 0 ? raw[n / 4].x : n % 4 == 1 ? raw[n / 4].y : n % 4 == 2 ? raw[n / 4].z : raw[n / 4].w;
                        const int c4 = n / (D / 32), g = n % (D / 32);
                        *reinterpret_cast<uint4*>(to + piece_of(Geo::BOX, kk, g * 4 + c4)) = codes_bf16(w);
                    }
                } else {
                    // D = 128: piece u of 8 bytes, halves g = 0 .. 3; else word u, halves g = 0, 1, and (D = 96) half u, g = 2
#pragma unroll
                    for (int n = 0; n < LOADS * 4; ++n) {
                        const uint32_t w = n % 4 == 0 ? raw[n / 4].x : n % 4 == 1 ? raw[n / 4].y : n % 4 == 2 ? raw[n / 4].z : raw[n / 4].w;
                        if constexpr (D == 128) {
                            const int at = 2 * ((n >> 1) ^ (j & 4)) + (n & 1);
                            *reinterpret_cast<uint4*>(to + piece_of(Geo::BOX, kk, at)) = codes_f16(w, even, odd);
                        } else if (n < 8) {
                            *reinterpret_cast<uint4*>(to + piece_of(Geo::BOX, kk, n)) = codes_f16(w, even, odd);
                        } else {
                            const uint32_t lo = (w & 0xffffu) | (w << 12), hi = (w >> 16) | ((w >> 4) & 0x0ffff000u);   // codes 0 and 1 (2 and 3) side by side
                            auto two = [&](uint32_t x) { return minus_half2((x & 0x000f000fu) | 0x64006400u, even); };
                            *reinterpret_cast<uint4*>(to + piece_of(Geo::BOX, kk, n)) = make_uint4(two(lo), two(lo >> 8), two(hi), two(hi >> 8));
                        }
                    }
                    float* rows = reinterpret_cast<float*>(smem + Geo::OFF_ROWS + buf * 1024) + (kk >> 1) * 8 + (kk & 1);
                    rows[0] = step4_of(row.x);
                    rows[2] = lo4_of(row.x);
                    rows[4] = step4_of(row.y);
                    const float base_value = value4_of(row.y, zero_code);
                    rows[6] = base_value;
                    const bool large = __any_sync(kFullMask, fabsf(base_value) > kLargeBase4);
                    if (lane == 0) reinterpret_cast<unsigned short*>(far + buf)[warp & 1] = large;
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(full + buf);
            }
            return true;
        });
    } else if (warp == 12) {
        constexpr uint32_t qk_idesc = umma_attn_idesc(kUmma4Keys, false);
        constexpr uint32_t pv_idesc = umma_attn_idesc(D, true) & ~((1u << 7) | (1u << 10));      // fp16 operands
        const uint64_t q_desc = umma_desc_sw128(smem_u32(smem), 16), k_desc0 = umma_desc_sw128(smem_u32(smem) + Geo::OFF_K, 16);
        const uint64_t v_desc0 = umma_desc_sw128(smem_u32(smem) + Geo::OFF_V, Geo::BOX);
        unsigned segment = 0;
        walk([&](const Segment4& u, int, int steps, unsigned first) {
            if (steps == 0) return true;
            // (a tile without rows has no products, but its barriers go on: all follow every phase)
            const bool both = u.count * a.group - u.row0 > 128;
            for (int w = 0; w < 2; ++w)
                if (!warp_poll_or_abort(q_full + w, segment & 1u, abort_flag)) return false;
            ++segment;
            // (tiles and buffers by unrolled loops, so that descriptors are known sums of uniform registers)
            auto scores = [&](auto tile, int i, uint32_t buf, uint32_t phase) {
                constexpr int w = decltype(tile)::value;
                if (w == 0 && !warp_poll_or_abort(k_full + buf, phase, abort_flag)) return false;
                tc_fence_after();
                const uint64_t k_desc = k_desc0 + static_cast<uint64_t>(buf * (Geo::TILE >> 4));
                const uint32_t s_cols = tmem + w * 256 + buf * 64;
                if (elect_one()) {
                    if (w == 0 || both) {
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            constexpr int kQBox = Geo::Q_BOX, kBox = Geo::BOX, kTile = Geo::Q_TILE;
                            umma_bf16(s_cols, q_desc + static_cast<uint64_t>((w * kTile + (k >> 2) * kQBox + (k & 3) * 32) >> 4),
                                      k_desc + static_cast<uint64_t>(((k >> 2) * kBox + (k & 3) * 32) >> 4), qk_idesc, k > 0);
                        }
                    }
                    umma_commit(s_full + 2 * w + buf);
                    if (w == 1) umma_commit(k_free + buf);
                }
                __syncwarp();
                return true;
            };
            auto values = [&](auto tile, int i, uint32_t buf, uint32_t phase) {
                constexpr int w = decltype(tile)::value;
                if (!warp_poll_or_abort(p_ready + 2 * w + buf, phase, abort_flag)) return false;
                tc_fence_after();
                const uint64_t v_desc = v_desc0 + static_cast<uint64_t>(buf * (Geo::TILE >> 4));
                const uint32_t p_cols = tmem + w * 256 + buf * 64;
                if (elect_one()) {
                    if (w == 0 || both) {
#pragma unroll
                        for (int k = 0; k < kUmma4Keys / 16; ++k)
                            umma_bf16_a_tmem(tmem + w * 256 + 128, p_cols + k * 8, v_desc + k * 128, pv_idesc, i > 0 || k > 0);
                    }
                    if (w == 1) umma_commit(v_free + buf);
                }
                __syncwarp();
                return true;
            };
            constexpr std::integral_constant<int, 0> tile0{};
            constexpr std::integral_constant<int, 1> tile1{};
            for (int i = 0; i < 2 && i < steps; ++i) {
                const uint32_t step = first + i, buf = step & 1, phase = (step >> 1) & 1;
                if (!scores(tile0, i, buf, phase) || !scores(tile1, i, buf, phase)) return false;
            }
            for (int i = 0; i < steps; ++i) {
                const uint32_t step = first + i, buf = step & 1, phase = (step >> 1) & 1;
                const bool more = i + 2 < steps;
                // the tensor core runs products in order: the next scores may overwrite the weights just used
                if (!warp_poll_or_abort(v_full + buf, phase, abort_flag) || !values(tile0, i, buf, phase) || (more && !scores(tile0, i + 2, buf, phase ^ 1)) ||
                    !values(tile1, i, buf, phase) || (more && !scores(tile1, i + 2, buf, phase ^ 1)))
                    return false;
            }
            return true;
        });
        if (elect_one()) umma_commit(all_done);
        __syncwarp();
        if (!mbar_wait_bounded(all_done, 0)) *abort_flag = 1;
    } else {
        const int local = tid, w = warp >> 2;                        // row of the unit; tile
        const uint32_t lanes = (static_cast<uint32_t>((warp & 3) * 32) << 16) + w * 256;
        const uint32_t o_cols = tmem + 128 + lanes;
        s_full += 2 * w;
        p_ready += 2 * w;
        const float sl = a.scale_log2;
        walk([&](const Segment4& u, int end, int steps, unsigned first) {
            const int rows = u.count * a.group, row = u.row0 + local, tok = row / a.group;
            if (w == 1 && rows - u.row0 <= 128) {                        // a tile without rows
                if (steps > 0 && lane == 0) mbar_arrive(q_full + w);
                for (int i = 0; i < steps; ++i) {
                    const unsigned step = first + i, buf = step & 1, phase = (step >> 1) & 1;
                    if (!warp_poll_both(v_full + buf, s_full + buf, phase, abort_flag)) return false;
                    if (lane == 0) mbar_arrive(p_ready + buf);
                }
                return true;
            }
            const int first_limit = u.keys - u.count + 1;
            // (rows that are not there see zeros)
            const int limit = row < rows ? min(end, first_limit + tok) : end, least_limit = min(end, first_limit + (u.row0 + 128 * w) / a.group);
            const int64_t at = (u.token0 + tok) * a.hq + static_cast<int64_t>(u.head) * a.group + (row - tok * a.group);
            float m = -INFINITY, l = 0.0f, r = 0.0f, qs = 0.0f;
            if (steps > 0) {
                // this row's queries, their sum, and their place in the operand
                const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q) + (u.token0 + tok) * a.q_st +
                                           (static_cast<int64_t>(u.head) * a.group + (row - tok * a.group)) * a.q_sh;
#pragma unroll 8
                for (int c = 0; c < D / 8; ++c) {
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (row < rows) v = *(reinterpret_cast<const uint4*>(src) + c);
                    qs += ((bf16lo_to_f32(v.x) + bf16hi_to_f32(v.x)) + (bf16lo_to_f32(v.y) + bf16hi_to_f32(v.y))) +
                          ((bf16lo_to_f32(v.z) + bf16hi_to_f32(v.z)) + (bf16lo_to_f32(v.w) + bf16hi_to_f32(v.w)));
                    *reinterpret_cast<uint4*>(smem + w * Geo::Q_TILE + piece_of(Geo::Q_BOX, local & 127, c)) =
                        make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
                }
                qs *= sl;
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(q_full + w);
            }
            // Sums of O from the steps before the last fold, in the reference of that time: [four channels][row] for a warp, in the part that the unit leaves (one that
            // leaves none uses the place of the part that goes on, which is written after it).
            const int part_lanes = min(32, p.part_rows - warp * 32);
            float* kept = a.part_o + ((u.slot >= 0 ? u.slot : 2ll * blockIdx.x + 1) * p.part_rows + warp * 32) * D + lane * 4;
            float kept_m = 0.0f, kept_l = 0.0f, kept_r = 0.0f;           // (and those of l and r)
            // last: O becomes the whole sum; else the sum takes O, which begins anew
            auto fold = [&](bool begun, bool last) {
                const float f = m > kept_m ? exp2_fast(kept_m - m) : 1.0f;
#pragma unroll 1
                for (int c = 0; c < D; c += 16) {
                    float o[16];
                    float* to = kept + c * part_lanes;
                    tmem_ld16(o_cols + c, o);
                    float4 x[4] = {};
                    if (begun && row < rows)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = *reinterpret_cast<const float4*>(to + e * 4 * part_lanes);
                    tmem_wait_ld();
                    uint32_t z[16];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[e] = make_float4(fmaf(x[e].x, f, o[4 * e]), fmaf(x[e].y, f, o[4 * e + 1]), fmaf(x[e].z, f, o[4 * e + 2]), fmaf(x[e].w, f, o[4 * e + 3]));
                        if (!last && row < rows) *reinterpret_cast<float4*>(to + e * 4 * part_lanes) = x[e];
                        z[4 * e] = last ? __float_as_uint(x[e].x) : 0;
                        z[4 * e + 1] = last ? __float_as_uint(x[e].y) : 0;
                        z[4 * e + 2] = last ? __float_as_uint(x[e].z) : 0;
                        z[4 * e + 3] = last ? __float_as_uint(x[e].w) : 0;
                    }
                    tmem_st16(o_cols + c, z);
                }
                tmem_wait_st();
                kept_m = m;
                kept_l = fmaf(kept_l, f, l);
                kept_r = fmaf(kept_r, f, r);
                l = last ? kept_l : 0.0f;
                r = last ? kept_r : 0.0f;
            };
            for (int i = 0; i < steps;) {
                if (i > 0) {
                    const unsigned before = first + i - 1;
                    if (!warp_poll_or_abort(v_free + (before & 1), (before >> 1) & 1u, abort_flag)) return false;
                    tc_fence_after();
                    fold(i > kFoldUmma4, false);
                }
                const int stop = min(steps, i + kFoldUmma4);
#pragma unroll 1
                for (; i < stop; ++i) {
                    const unsigned step = first + i, buf = step & 1, phase = (step >> 1) & 1;
                    const int base = u.tile0 * kTileKeys + i * kUmma4Keys;
                    const bool mask = base + kUmma4Keys > least_limit;
                    if (!warp_poll_both(v_full + buf, s_full + buf, phase, abort_flag)) return false;
                    tc_fence_after();
                    const uint32_t s_cols = tmem + buf * 64 + lanes;
                    const float4* par = reinterpret_cast<const float4*>(smem + Geo::OFF_ROWS + buf * 1024);   // two keys, then their values
                    uint32_t y[32];
                    float sx, sy, sr;
                    auto weigh = [&](auto masked) {
                        const uint64_t sl2 = pair(sl, sl), qs2 = pair(qs, qs), m2 = pair(-m, -m);
                        uint64_t sx2 = 0, sy2 = 0, sr2 = 0;
#pragma unroll
                        for (int c0 = 0; c0 < kUmma4Keys; c0 += 16) {
                            float s[16];
                            tmem_ld16(s_cols + c0, s);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; e += 2) {
                                const float4 key = par[c0 + e], val = par[c0 + e + 1];
                                float x0, x1, y0, y1;
                                unpair(fma2(mul2(pair(key.x, key.y), pair(s[e], s[e + 1])), sl2, fma2(pair(key.z, key.w), qs2, m2)), x0, x1);
                                x0 = exp2_fast(x0);
                                x1 = exp2_fast(x1);
                                uint64_t x2 = pair(x0, x1), lo2 = pair(val.z, val.w), y2 = mul2(x2, pair(val.x, val.y));
                                if constexpr (masked.value) {
                                    const bool see0 = base + c0 + e < limit, see1 = base + c0 + e + 1 < limit;
                                    unpair(y2, y0, y1);
                                    x2 = pair(see0 ? x0 : 0.0f, see1 ? x1 : 0.0f);
                                    lo2 = pair(see0 ? val.z : 0.0f, see1 ? val.w : 0.0f);
                                    y2 = pair(see0 ? y0 : 0.0f, see1 ? y1 : 0.0f);
                                }
                                sx2 = add2(sx2, x2);
                                sy2 = add2(sy2, y2);
                                sr2 = fma2(x2, lo2, sr2);
                                unpair(y2, y0, y1);
                                y[(c0 + e) / 2] = pack_half2(y0, y1);
                            }
                        }
                        float p0, p1;
                        unpair(sx2, p0, p1);
                        sx = p0 + p1;
                        unpair(sy2, p0, p1);
                        sy = p0 + p1;
                        unpair(sr2, p0, p1);
                        sr = p0 + p1;
                    };
                    // A segment's first step, and later the rare case that some row's weights or products have grown too far: the row's reference moves so
                    // that its largest product becomes 2^6.  O and the sums follow.  (Once a step: what is NaN stays NaN.)
                    bool moved = false;
                    for (;;) {
                        if (i > 0 || moved) {
                            if (mask) weigh(std::true_type{});
                            else weigh(std::false_type{});
                            if (moved || __all_sync(kFullMask, sx + fabsf(sr) <= kMostWeight4 && sy <= kMostUmma4)) break;
                        } else {
                            sx = INFINITY;
                            sr = sy = 0.0f;
                        }
                        const bool moves = !(sx + fabsf(sr) <= kMostWeight4 && sy <= kMostUmma4);
                        float top = -INFINITY, heavy = -INFINITY;
#pragma unroll 1
                        for (int c0 = 0; c0 < kUmma4Keys; c0 += 16) {
                            float s[16];
                            tmem_ld16(s_cols + c0, s);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; e += 2) {
                                const float4 key = par[c0 + e], val = par[c0 + e + 1];
                                const float z0 = fmaf(key.x * s[e], sl, key.z * qs), z1 = fmaf(key.y * s[e + 1], sl, key.w * qs);
                                if (base + c0 + e < limit) {
                                    top = fmaxf(top, z0);
                                    heavy = fmaxf(heavy, z0 + __log2f(val.x));
                                }
                                if (base + c0 + e + 1 < limit) {
                                    top = fmaxf(top, z1);
                                    heavy = fmaxf(heavy, z1 + __log2f(val.y));
                                }
                            }
                        }
                        float wide = top;
                        if (far[buf] != 0) {
#pragma unroll 1
                            for (int c0 = 0; c0 < kUmma4Keys; c0 += 16) {
                                float s[16];
                                tmem_ld16(s_cols + c0, s);
                                tmem_wait_ld();
#pragma unroll
                                for (int e = 0; e < 16; e += 2) {
                                    const float4 key = par[c0 + e], val = par[c0 + e + 1];
                                    if (base + c0 + e < limit) wide = fmaxf(wide, fmaf(key.x * s[e], sl, key.z * qs) + __log2f(fabsf(val.z)));
                                    if (base + c0 + e + 1 < limit) wide = fmaxf(wide, fmaf(key.y * s[e + 1], sl, key.w * qs) + __log2f(fabsf(val.w)));
                                }
                            }
                        }
                        float to = fmaxf(heavy > -INFINITY ? heavy - 6.0f : top, wide - 90.0f);
                        to = moves ? fmaxf(to, m) : m;
                        const float f = to > m ? exp2_fast(m - to) : 1.0f;
                        m = to;
                        l *= f;
                        r *= f;
                        if (i > 0) {
                            if (!warp_poll_or_abort(v_free + ((step - 1) & 1), ((step - 1) >> 1) & 1u, abort_flag)) return false;
                            tc_fence_after();
#pragma unroll 1
                            for (int c = 0; c < Geo::O_COLS; c += 16) {
                                float o[16];
                                tmem_ld16(o_cols + c, o);
                                tmem_wait_ld();
                                uint32_t z[16];
#pragma unroll
                                for (int e = 0; e < 16; ++e) z[e] = __float_as_uint(o[e] * f);
                                tmem_st16(o_cols + c, z);
                            }
                        }
                        moved = true;
                    }
                    l += sx;
                    r += sr;
                    tmem_st16(s_cols, y);
                    tmem_st16(s_cols + 16, y + 16);
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_ready + buf);
                }
            }
            if (steps > 0) {
                const unsigned step = first + steps - 1;
                if (!warp_poll_or_abort(v_free + (step & 1), (step >> 1) & 1u, abort_flag)) return false;
                tc_fence_after();
                if (steps > kFoldUmma4) fold(true, true);
                __syncwarp();                                            // (others write this row's part)
            }
            const float inv = u.slot >= 0 ? 1.0f : l > 0.0f ? 1.0f / l : 0.0f;
            // 32 channels at a time through this warp's rows of the queries' place, which no product reads any more: a row's four channels after the
            // other go there, whole lines of 128 bytes (fp32) leave (a row a thread straight to memory: 16000 clocks a unit against 6000)
            unsigned char* stage = smem + w * Geo::Q_TILE + (warp & 3) * 4096;
            const int there = rows - u.row0 - warp * 32 - (lane >> 3);           // row 4 k of this lane is there if 4 k < there
            const int groups = rows - u.row0 > warp * 32 ? D / 32 : 0;
            const int64_t part0 = (u.slot * p.part_rows + warp * 32 + (lane >> 3)) * D + (lane & 7) * 4;
            int line[8];                                                         // rows of the output, from the sequence's and head's first on
            if (u.slot < 0) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int out_row = u.row0 + warp * 32 + (lane >> 3) + 4 * k, t = out_row / a.group;
                    line[k] = t * a.hq + out_row - t * a.group;
                }
            }
            __nv_bfloat16* out0 = static_cast<__nv_bfloat16*>(a.out) + (u.token0 * a.hq + static_cast<int64_t>(u.head) * a.group) * D + (lane & 7) * 4;
            const unsigned char* from = stage + (lane >> 3) * 128;
            const int piece0 = ((lane & 7) ^ (lane >> 3)) << 4;
#pragma unroll 1
            for (int g = 0; g < groups; ++g) {
                // D = 128: column 16 u + 8 (g / 2) + 2 i + (g & 1) is channel 32 g + 4 u + i; else column 8 u + 2 i + g, and (D = 96) the last 32 as they are
                const bool plain = D == 96 && g == 2;
#pragma unroll
                for (int v0 = 0; v0 < 8; v0 += 4) {
                    float o[4][8] = {};
                    if (steps > 0) {
#pragma unroll
                        for (int v = 0; v < 4; ++v) tmem_ld8(o_cols + (D == 128 ? 16 * (v0 + v) + 8 * (g >> 1) : plain ? 64 + 4 * (v0 + v) : 8 * (v0 + v)), o[v]);
                        tmem_wait_ld();
                    }
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        float4 x = g & 1 ? make_float4(o[v][1], o[v][3] * 0.0625f, o[v][5], o[v][7] * 0.0625f)
                                         : make_float4(o[v][0], o[v][2] * 0.0625f, o[v][4], o[v][6] * 0.0625f);
                        if (plain) x = make_float4(o[v][0], o[v][1], o[v][2], o[v][3]);
                        *reinterpret_cast<float4*>(stage + lane * 128 + (((v0 + v) ^ (lane & 7)) << 4)) =
                            make_float4((x.x + r) * inv, (x.y + r) * inv, (x.z + r) * inv, (x.w + r) * inv);
                    }
                }
                __syncwarp();
                float4 x[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = *reinterpret_cast<const float4*>(from + k * 512 + (piece0 ^ ((k & 1) << 6)));
                if (u.slot >= 0) {
                    float* to = a.part_o + part0 + g * 32;
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (4 * k < there) *reinterpret_cast<float4*>(to + k * 4 * D) = x[k];
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (4 * k < there)
                            *reinterpret_cast<uint2*>(out0 + static_cast<int64_t>(line[k]) * D + g * 32) = make_uint2(pack_bf16x2(x[k].x, x[k].y), pack_bf16x2(x[k].z, x[k].w));
                }
                __syncwarp();
            }
            tc_fence_before();
            if (row < rows) {
                if (u.slot >= 0) a.part_ml[u.slot * p.part_rows + local] = make_float2(m, l);
                else if (p.lse) p.lse[at] = l > 0.0f || l != l ? m + log2f(l) : INFINITY;
            }
            return true;
        });
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 12) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

}  // namespace wht
