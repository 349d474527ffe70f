// Shared-prefix attention of many rows on the tcgen05 tensor core (bf16).
//
// Every row (token, query head) of a key head sees the same prefix, so with R rows the two products are dense
// [R x D] x [D x L] and [R x L] x [L x D]: 4 D flops per row and key against 4 D bytes per key, i.e. R flops a byte.
// From about 250 rows on that is the tensor core's balance, and the exponentials (one per row and key,
// 16 a clock and SM) weigh as much as the products.
//
// A block of 11 warps owns 256 rows of one key head as two tiles of 128, and a range of keys:
//   warps 0..3, 4..7   softmax of tile 0 / tile 1: one thread per row
//   warps 8, 9         issue the products of tile 0 / tile 1;   warp 10   copies keys and values (TMA, a ring of 128-key tiles)
// and runs steps of one tile and 128 keys, the two tiles taking turns, so that one tile's softmax runs under the other's products:
//   S = Q K^T            into tensor memory (128 lanes x 128 fp32 columns)
//   P = exp2(S - m)      read by the row's thread, rounded to bf16 and written over S
//   O += P V             P from tensor memory, V from shared memory, O stays in tensor memory (D columns)
// The reference maximum m of a row is that of its first 64 keys and moves only when 64 weights add up to more than 2^14: large
// weights are as exact in bf16 and fp32 as weights up to 1, O, which sits in tensor memory, is rescaled a few times per row at
// most instead of once per tile, and the common path needs no maximum at all.  The weights are handed over in halves of 64 keys, so that
// the second product of the first half runs under the exponentials of the second.  With 128 rows or fewer both tiles hold the SAME rows and take alternate key tiles; they
// leave as two parts.
//
// Keys and values arrive as page-high boxes of 64 channels in the 128-byte swizzle; K is the K-major operand of the
// first product and V, the same way in memory, the MN-major operand of the second.  For D = 96 the second box reaches over
// the row's end, where the copy fills zeros, and is used up to channel 96.
//
// Waits are bounded as in umma_kernels.cuh; every copy is one block's own, from this GPU's memory.
#pragma once
#include <cuda.h>

#include "attn_kernels.cuh"
#include "umma_kernels.cuh"

namespace wht {

constexpr int kUmmaAttnThreads = 352;
constexpr float kLargestHalf = 16384.0f;  // 2^14: sum of 64 weights from which a row's reference maximum moves

template <int D>
struct UmmaAttnGeo {
    static constexpr int HALVES = D > 64 ? 2 : 1;             // 64-channel boxes per row
    static constexpr int BOX = 128 * 128;                     // bytes of 128 rows of one box
    static constexpr int TILE = HALVES * BOX;                 // a tile of 128 rows: queries, keys or values
    static constexpr int STAGES = HALVES == 2 ? 5 : 8;
    static constexpr int OFF_RING = 2 * TILE;
    static constexpr int OFF_BARS = OFF_RING + STAGES * TILE;
    static constexpr int NBARS = 2 * STAGES + 10 + 2;
    static constexpr int OFF_MISC = OFF_BARS + NBARS * 8;
    static constexpr int BYTES = OFF_MISC + 16 + 1024;        // and what aligning the start to 1024 bytes takes
    static constexpr int O_COLS = D > 64 ? 128 : 64;
};

// Shared-memory operand in the 128-byte swizzle: 8-row groups 1024 bytes apart (both majors); `lead` is the distance of 64-channel
// blocks for the MN-major operand (unused for the K-major one, whose instructions stay within a block).
__device__ __forceinline__ uint64_t umma_desc_sw128(uint32_t addr, uint32_t lead) {
    uint64_t d = static_cast<uint64_t>((addr & 0x3FFFFu) >> 4);
    d |= static_cast<uint64_t>(lead >> 4) << 16;
    d |= static_cast<uint64_t>(1024 >> 4) << 32;
    d |= static_cast<uint64_t>(1) << 46;
    d |= static_cast<uint64_t>(2) << 61;
    return d;
}
__host__ __device__ constexpr uint32_t umma_attn_idesc(int n, bool b_mn_major) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (b_mn_major ? 1u << 16 : 0u) | (static_cast<uint32_t>(n >> 3) << 17) |
           (static_cast<uint32_t>(128 >> 4) << 24);
}

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}

// ---- two fp32 values in one instruction
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
    return d;
}
__device__ __forceinline__ void unpair(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
constexpr float kExp2C0 = 0.9999992847f, kExp2C1 = 0.6931217909f, kExp2C2 = 0.2402474433f, kExp2C3 = 0.05591785908f, kExp2C4 = 0.0095701003f;
// 2^x for two values on the multiply-add pipe: x = n + f with n the nearest whole number, 2^f by a polynomial of degree 4
// on [-1/2, 1/2] (least relative error, 2.6e-6: a thousandth of the rounding to bf16 that follows), 2^n from its exponent bits.
// Held to [-126, 127]; NaN stays NaN.
__device__ __forceinline__ uint64_t exp2_poly2(uint64_t x) {
    float a, b;
    unpair(x, a, b);
    asm("max.NaN.f32 %0, %0, %1;\n\tmin.NaN.f32 %0, %0, %2;" : "+f"(a) : "f"(-126.0f), "f"(127.0f));
    asm("max.NaN.f32 %0, %0, %1;\n\tmin.NaN.f32 %0, %0, %2;" : "+f"(b) : "f"(-126.0f), "f"(127.0f));
    x = pair(a, b);
    constexpr float kRound = 12582912.0f;  // 1.5 * 2^23: adding it leaves the nearest whole number in the low bits
    const uint64_t r = add2(x, pair(kRound, kRound));
    const uint64_t f = add2(x, mul2(add2(r, pair(-kRound, -kRound)), pair(-1.0f, -1.0f)));
    uint64_t y = fma2(f, pair(kExp2C4, kExp2C4), pair(kExp2C3, kExp2C3));
    y = fma2(y, f, pair(kExp2C2, kExp2C2));
    y = fma2(y, f, pair(kExp2C1, kExp2C1));
    y = fma2(y, f, pair(kExp2C0, kExp2C0));
    float ra, rb;
    unpair(r, ra, rb);
    return mul2(y, pair(__uint_as_float((__float_as_uint(ra) << 23) + 0x3f800000u), __uint_as_float((__float_as_uint(rb) << 23) + 0x3f800000u)));
}

// Bounded wait that polls without a pause: the products and the softmax hand over to each other every thousand clocks or so, and
// a parked wait answered some 400 clocks late (measured).  Gives up like wait_or_abort.
__device__ __forceinline__ bool poll_or_abort(uint64_t* bar, uint32_t parity, volatile uint32_t* abort_flag) {
    for (uint32_t i = 0; i < (1u << 24); ++i) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(smem_u32(bar)), "r"(parity)
            : "memory");
        if (ok) return true;
        if ((i & 255u) == 255u && *abort_flag) return false;
    }
    *abort_flag = 1;
    atomicExch(&g_wht_device_error, kDeviceErrWaitExpired);
    return false;
}
__device__ __forceinline__ bool warp_poll_or_abort(uint64_t* bar, uint32_t parity, volatile uint32_t* abort_flag) {
    return __all_sync(kFullMask, poll_or_abort(bar, parity, abort_flag));
}

__device__ __forceinline__ bool elect_one() {
    uint32_t is;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
    return is != 0;
}

// one lane's row of weights
struct SoftmaxRow {
    float m = 0.0f;  // reference maximum, in units of the raw scores
    float l = 0.0f;
};

template <int D>
__global__ void __launch_bounds__(kUmmaAttnThreads, 1)
attn_umma_prefix_kernel(const UmmaAttnParams up, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
    using Geo = UmmaAttnGeo<D>;
    extern __shared__ unsigned char umma_attn_smem[];
    const AttnParams& p = up.a;
    unsigned char* smem = umma_attn_smem + ((1024u - (smem_u32(umma_attn_smem) & 1023u)) & 1023u);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + Geo::OFF_BARS);
    uint64_t* kv_full = bars;
    uint64_t* kv_empty = bars + Geo::STAGES;
    uint64_t* s_full = bars + 2 * Geo::STAGES;   // [2] scores of a tile's step are in tensor memory
    uint64_t* p_ready = s_full + 2;              // [2] its weights are
    uint64_t* o_done = s_full + 4;               // [2] its second product is complete
    uint64_t* p_half = s_full + 6;               // [2] the weights of its first 64 keys are
    uint64_t* o_half = s_full + 8;               // [2] the product of those is complete
    uint64_t* all_done = s_full + 10;            // [2] every product issued for a tile is complete
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + Geo::OFF_MISC);
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(smem + Geo::OFF_MISC + 4);

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int b = blockIdx.x;
    const int split = b % up.splits;
    b /= up.splits;
    const int row0 = (b % up.row_blocks) * 256;
    const int head = b / up.row_blocks;
    const int rows = static_cast<int>(p.T) * p.group;
    int key0, key1;
    attn_part(static_cast<int>(p.prefix_len), 128, up.splits, split, key0, key1);
    const int tiles = (key1 - key0 + 127) / 128;
    const bool same = up.same_rows != 0;
    // Steps of row tile w: step i takes key tile i, or, where both tiles hold the same rows, every second one.
    auto steps_of = [&](int w) { return same ? (tiles - w + 1) / 2 : tiles; };
    auto key_tile = [&](int w, int i) { return same ? 2 * i + w : i; };
    // Where item 2 i (keys) or 2 i + 1 (values) of row tile w's step i lies: all stages in turn; with the same rows each
    // tile has half of the stages to itself.  Either way a waiting warp follows every phase of a stage's barrier that it looks at: on
    // a barrier that other items pass through unseen, a wait by parity could be answered by an earlier phase.
    struct Place {
        int stage;
        uint32_t parity;
    };
    auto place_of = [&](int w, int item) {
        constexpr int kHalf = Geo::STAGES / 2;
        return same ? Place{w * kHalf + item % kHalf, static_cast<uint32_t>(item / kHalf) & 1u}
                    : Place{item % Geo::STAGES, static_cast<uint32_t>(item / Geo::STAGES) & 1u};
    };

    grid_launch_dependents();
    if (warp == 8) {
        tmem_alloc(tmem_slot, 512);
        tmem_relinquish();
    }
    if (tid == 10 * 32) {
        for (int s = 0; s < Geo::STAGES; ++s) {
            mbar_init(kv_full + s, 1);
            mbar_init(kv_empty + s, same ? 1 : 2);  // as many row tiles read it
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(s_full + s, 1);
            mbar_init(p_ready + s, 4);
            mbar_init(p_half + s, 4);
            mbar_init(o_done + s, 1);
            mbar_init(o_half + s, 1);
            mbar_init(all_done + s, 1);
        }
        *abort_flag = 0;
        fence_mbar_init();
    }
    // queries: 128-byte rows of 64 channels, chunks permuted by the row as the copies' swizzle does
    {
        const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p.q);
        constexpr int CH = Geo::HALVES * 8;
        // eight chunks a thread at a time, all loads in flight
        constexpr int BATCH = 8;
        for (int i0 = tid; i0 < 256 * CH; i0 += BATCH * kUmmaAttnThreads) {
            uint4 v[BATCH];
#pragma unroll
            for (int e = 0; e < BATCH; ++e) {
                const int i = i0 + e * kUmmaAttnThreads, r = i / CH, c = i % CH;
                const int row = row0 + (same ? r & 127 : r);
                v[e] = make_uint4(0, 0, 0, 0);
                if (i < 256 * CH && row < rows && c * 8 < D) {
                    const int tok = row / p.group;
                    v[e] = __ldg(reinterpret_cast<const uint4*>(q + tok * p.q_st + (static_cast<int64_t>(head) * p.group + (row - tok * p.group)) * p.q_sh) + c);
                }
            }
#pragma unroll
            for (int e = 0; e < BATCH; ++e) {
                const int i = i0 + e * kUmmaAttnThreads, r = i / CH, c = i % CH;
                unsigned char* dst = smem + (r >> 7) * Geo::TILE + (c >> 3) * Geo::BOX + (r & 127) * 128 + (((c & 7) ^ (r & 7)) << 4);
                if (i < 256 * CH) *reinterpret_cast<uint4*>(dst) = v[e];
            }
        }
        fence_async_smem();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const uint32_t ring = smem_u32(smem) + Geo::OFF_RING;

    if (warp == 10) {
        if (lane == 0) {
            // the items in the order in which the products take them
            const int list = static_cast<int>((p.prefix_len + (1 << p.page_shift) - 1) >> p.page_shift);
            const int page = 1 << p.page_shift;
            bool ok = true;
            int loaded = 0;
            for (int item = 0; ok && item < 2 * steps_of(0); ++item) {
                for (int w = 0; ok && w < (same ? 2 : 1); ++w) {
                    if (item >= 2 * steps_of(w)) break;
                    const Place at = place_of(w, item);
                    ok = wait_or_abort(kv_empty + at.stage, at.parity ^ 1u, abort_flag);
                    if (!ok) break;
                    const CUtensorMap* map = item & 1 ? &v_map : &k_map;
                    const int first = (key0 + key_tile(w, item >> 1) * 128) >> p.page_shift;
                    const int n = min(128 >> p.page_shift, list - first);
                    mbar_expect_tx(kv_full + at.stage, static_cast<uint32_t>(n * page * 128 * Geo::HALVES));
                    for (int i = 0; i < n; ++i) {
                        int pg = __ldg(p.prefix_pages + first + i);
                        if (pg < 0 || pg >= p.num_pages) {
                            attn_report(kAttnErrIndex);
                            pg = 0;
                        }
                        const int y = (pg * p.hkv + head) << p.page_shift;
#pragma unroll
                        for (int h = 0; h < Geo::HALVES; ++h)
                            tma_load_2d(ring + at.stage * Geo::TILE + h * Geo::BOX + i * page * 128, map, h * 64, y, kv_full + at.stage);
                    }
                    ++loaded;
                }
            }
            if (!ok) {  // given up: the copies in flight still write this block's memory
                for (int k = 0, item = 0; k < loaded; ++item)
                    for (int w = 0; w < (same ? 2 : 1) && k < loaded; ++w) {
                        if (item >= 2 * steps_of(w)) break;
                        if (k++ < loaded - Geo::STAGES) continue;
                        const Place at = place_of(w, item);
                        mbar_wait_bounded(kv_full + at.stage, at.parity);
                    }
            }
        }
    } else if (warp >= 8) {
        // One warp per row tile issues its products.  The whole warp walks the loop and one elected lane issues, so that
        // descriptors and barrier addresses stay in uniform registers (from a single lane's code each product took 100
        // clocks to issue, more than the 64 it runs).
        const int w = warp - 8;
        const int n = steps_of(w);
        constexpr uint32_t qk_idesc = umma_attn_idesc(128, false), pv_idesc = umma_attn_idesc(D, true);
        const uint64_t q_desc = umma_desc_sw128(smem_u32(smem) + w * Geo::TILE, 16);
        const uint32_t s_cols = tmem + w * 128, o_cols = tmem + 256 + w * Geo::O_COLS;
        bool ok = true;
        auto scores = [&](int i) {   // S of the tile's step i
            const Place at = place_of(w, 2 * i);
            if (!warp_poll_or_abort(kv_full + at.stage, at.parity, abort_flag)) return false;
            tc_fence_after();
            const uint64_t k_desc = umma_desc_sw128(ring + at.stage * Geo::TILE, 16);
            if (elect_one()) {
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    constexpr int kBox = Geo::BOX;
                    const uint64_t off = static_cast<uint64_t>(((k >> 2) * kBox + (k & 3) * 32) >> 4);
                    umma_bf16(s_cols, q_desc + off, k_desc + off, qk_idesc, k > 0);
                }
                umma_commit(s_full + w);
                umma_commit(kv_empty + at.stage);
            }
            __syncwarp();
            return true;
        };
        if (n > 0) ok = scores(0);
        for (int i = 0; ok && i < n; ++i) {
            const Place at = place_of(w, 2 * i + 1);
            ok = warp_poll_or_abort(kv_full + at.stage, at.parity, abort_flag) &&
                 warp_poll_or_abort(p_half + w, static_cast<uint32_t>(i) & 1u, abort_flag);
            if (!ok) break;
            tc_fence_after();
            const uint64_t v_desc = umma_desc_sw128(ring + at.stage * Geo::TILE, Geo::BOX);
            if (elect_one()) {
#pragma unroll
                for (int k = 0; k < 4; ++k) umma_bf16_a_tmem(o_cols, s_cols + k * 8, v_desc + k * 128, pv_idesc, i > 0 || k > 0);
                umma_commit(o_half + w);
            }
            __syncwarp();
            ok = warp_poll_or_abort(p_ready + w, static_cast<uint32_t>(i) & 1u, abort_flag);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int k = 4; k < 8; ++k) umma_bf16_a_tmem(o_cols, s_cols + k * 8, v_desc + k * 128, pv_idesc, 1);
                umma_commit(o_done + w);
                umma_commit(kv_empty + at.stage);
            }
            __syncwarp();
            // the tensor core runs a tile's products in order: the next scores may overwrite the weights just used
            if (i + 1 < n) ok = scores(i + 1);
        }
        if (elect_one()) umma_commit(all_done + w);
        __syncwarp();
        if (!mbar_wait_bounded(all_done + w, 0)) *abort_flag = 1;
    } else if (warp < 8) {
        const int w = warp >> 2;
        const int r = row0 + (same ? 0 : w * 128) + (warp & 3) * 32 + lane;
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t s_cols = tmem + w * 128 + lanes, o_cols = tmem + 256 + w * Geo::O_COLS + lanes;
        const float sl = p.scale_log2;
        const int n = steps_of(w);
        SoftmaxRow st;
        bool ok = true;
        for (int i = 0; i < n; ++i) {
            const int valid = min(128, key1 - key0 - key_tile(w, i) * 128);
            ok = warp_poll_or_abort(s_full + w, static_cast<uint32_t>(i) & 1u, abort_flag);
            if (!ok) break;
            tc_fence_after();
            uint32_t x[64];      // the half of the tile at hand
            auto load_half = [&](int c0) {
#pragma unroll
                for (int c = 0; c < 64; c += 32) tmem_ld32(s_cols + c0 + c, x + c);
                tmem_wait_ld();
                if (valid < c0 + 64) {
#pragma unroll
                    for (int c = 0; c < 64; ++c)
                        if (c0 + c >= valid) x[c] = 0xff800000u;  // -infinity
                }
            };
            // Weights of the half, against the reference maximum, into the columns from c0 / 2 on; returns their sum.  One pair in four takes the
            // polynomial, so that the exponential unit (4 a clock and scheduler) and the multiply-add pipe finish together.
            const uint64_t sl2 = pair(sl, sl);
            auto weights = [&](int c0) {
                const uint64_t off2 = pair(-st.m * sl, -st.m * sl);
                uint64_t sum[2] = {0, 0};
#pragma unroll
                for (int c = 0; c < 64; c += 32) {
                    uint32_t y[16];
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        uint64_t v = fma2(pair(__uint_as_float(x[c + e]), __uint_as_float(x[c + e + 1])), sl2, off2);
                        float a, b;
                        if ((e & 7) == 6) {
                            v = exp2_poly2(v);
                            unpair(v, a, b);
                        } else {
                            unpair(v, a, b);
                            a = exp2_fast(a);
                            b = exp2_fast(b);
                            v = pair(a, b);
                        }
                        sum[(e >> 1) & 1] = add2(sum[(e >> 1) & 1], v);
                        y[e / 2] = pack_bf16x2(a, b);
                    }
                    tmem_st16(s_cols + (c0 + c) / 2, y);
                }
                float a, b;
                unpair(add2(sum[0], sum[1]), a, b);
                return a + b;
            };
            auto half_max = [&]() {
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < 64; c += 8)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top[e] = max3(top[e], __uint_as_float(x[c + e]), __uint_as_float(x[c + 4 + e]));
                return fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
            };
            // The rare case: some row's weights have grown past kLargestHalf.  Its reference moves to the half's maximum; the products issued so far (`bar`) are waited for, and O and l are scaled.
            auto move_reference = [&](bool move, uint64_t* bar, uint32_t parity) {
                if (!warp_poll_or_abort(bar, parity, abort_flag)) return false;
                tc_fence_after();
                const float mx = fmaxf(st.m, half_max());
                const float f = move ? exp2_fast((st.m - mx) * sl) : 1.0f;
                if (move) st.m = mx;
                st.l *= f;
#pragma unroll 1
                for (int c = 0; c < D; c += 16) {
                    float o[16];
                    tmem_ld16(o_cols + c, o);
                    tmem_wait_ld();
                    uint32_t y[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) y[e] = __float_as_uint(o[e] * f);
                    tmem_st16(o_cols + c, y);
                }
                return true;
            };
            load_half(0);
            if (i == 0) st.m = half_max();
            float sum = weights(0);
            if (__any_sync(kFullMask, sum > kLargestHalf) && i > 0) {
                ok = move_reference(sum > kLargestHalf, o_done + w, static_cast<uint32_t>(i - 1) & 1u);
                if (!ok) break;
                sum = weights(0);
            }
            st.l += sum;
            if (valid < 128) {
                // the tile's last rows hold keys that nobody sees, or nothing at all: their values become 0 so that a
                // weight of 0 takes nothing from them
                const Place at = place_of(w, 2 * i + 1);
                ok = warp_poll_or_abort(kv_full + at.stage, at.parity, abort_flag);
                if (!ok) break;
                unsigned char* v = smem + Geo::OFF_RING + at.stage * Geo::TILE;
                for (int e = (warp & 3) * 32 + lane; e < (128 - valid) * 8 * Geo::HALVES; e += 128) {
                    const int row = valid + e / (8 * Geo::HALVES), c = e % (8 * Geo::HALVES);
                    *reinterpret_cast<uint4*>(v + (c >> 3) * Geo::BOX + row * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
                }
                fence_async_smem();
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_half + w);
            load_half(64);
            sum = weights(64);
            if (__any_sync(kFullMask, sum > kLargestHalf)) {
                ok = move_reference(sum > kLargestHalf, o_half + w, static_cast<uint32_t>(i) & 1u);
                if (!ok) break;
                sum = weights(64);
            }
            st.l += sum;
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_ready + w);
        }
        if (ok && n > 0) {
            ok = warp_poll_or_abort(o_done + w, static_cast<uint32_t>(n - 1) & 1u, abort_flag);
            tc_fence_after();
        }
        if (ok) {
            const int tok = r / p.group;
            const int64_t at = static_cast<int64_t>(tok) * p.hq + head * p.group + (r - tok * p.group);
            const int part = same ? 2 * split + w : split;
            const int64_t slot = static_cast<int64_t>(part) * p.T * p.hq + at;
#pragma unroll 1
            for (int c = 0; c < D; c += 16) {
                float o[16];
                if (n > 0) {
                    tmem_ld16(o_cols + c, o);
                    tmem_wait_ld();
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = 0.0f;
                }
                if (r < rows) {
#pragma unroll
                    for (int e = 0; e < 16; e += 4)
                        *reinterpret_cast<float4*>(p.part_o + slot * D + c + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                }
            }
            if (r < rows) p.part_ml[slot] = n > 0 ? make_float2(st.m * sl, st.l) : make_float2(-INFINITY, 0.0f);
        }
        tc_fence_before();
    }
    __syncwarp();
    __syncthreads();
    if (warp == 8) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

}  // namespace wht
