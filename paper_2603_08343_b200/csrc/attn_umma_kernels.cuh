// Shared-prefix attention of many rows on the tcgen05 tensor core (bf16).
//
// Every row (token, query head) of a key head sees the same prefix, so with R rows the two products are dense
// [R x D] x [D x L] and [R x L] x [L x D]: 4 D flops per row and key against 4 D bytes per key, i.e. R flops a byte.
// From about 250 rows on that is the tensor core's balance, and the exponentials (one per row and key,
// 16 a clock and SM) weigh as much as the products.
//
// A block of 18 warps owns 256 rows of one key head as two tiles of 128, and a range of keys:
//   warps 0..7, 8..15  softmax of tile 0 / tile 1: a row's 128 keys of a step belong to two threads, 64 each
//   warp 16            issues the products;   warp 17   copies keys and values (TMA, a ring of 128-key tiles)
// and runs steps of one tile and 128 keys, the two tiles strictly in turn, so that one tile's softmax runs under the other's products:
//   S = Q K^T            into tensor memory (128 lanes x 128 fp32 columns)
//   P = exp2(S - m)      read by the row's threads, rounded to bf16 and written over S
//   O += P V             P from tensor memory, V from shared memory, O stays in tensor memory (D columns)
// The reference maximum m of a row is that of its first tile and moves (once a step at most) only when a half's 64 weights add up to more than 2^14: large
// weights are as exact in bf16 and fp32 as weights up to 1, O, which sits in tensor memory, is rescaled a few times per row at
// most instead of once per tile, and the common path needs no maximum at all.  The weights are one bf16 term here: a second
// product for the second term would cost what the first does.  With 128 rows or fewer both tiles hold the SAME rows and take alternate
// key tiles; they leave as two parts.
//
// Measured, 256 rows x 32768 keys x 32 heads, D = 128: 128 to 145 us (1.07 to 0.95 PFLOP/s, with the SM clock), 178 in the first form; eight
// softmax warps instead of sixteen 191, warp numbers not known to be uniform 163 (a product then takes 100 clocks to issue, not
// 30).  A step takes 3400 clocks, 1600 of them a tile's weights, which is what bounds it: exponentials, multiply-adds and tensor-memory
// reads of 256 x 128 scores.  Short ranges (512 keys a block) spend 5.9k clocks before the first scores and 5k on the result.
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

constexpr int kUmmaAttnThreads = 576;
constexpr int kStartBarrier = 3;  // (0: the whole block at its end; 1, 2: the two tiles' votes)
constexpr float kLargestHalf = 16384.0f;  // 2^14: sum of 64 weights from which a row's reference maximum moves
// 2^29: largest reference in the exponents.  Beyond, a row's two largest scores, if they differ at all, are 32 or more apart in its units: all weight
// is the largest one's under any scale that leaves them so, and with this one the rounding of m * scale (below 64) cannot take it to 0.
constexpr float kLargestReference = 536870912.0f;

template <int D>
struct UmmaAttnGeo {
    static constexpr int HALVES = D > 64 ? 2 : 1;             // 64-channel boxes per row
    static constexpr int BOX = 128 * 128;                     // bytes of 128 rows of one box
    static constexpr int TILE = HALVES * BOX;                 // a tile of 128 rows: queries, keys or values
    static constexpr int STAGES = HALVES == 2 ? 5 : 8;
    static constexpr int OFF_RING = 2 * TILE;
    static constexpr int OFF_BARS = OFF_RING + STAGES * TILE;
    static constexpr int NBARS = 2 * STAGES + 6 + 1;
    static constexpr int OFF_MISC = OFF_BARS + NBARS * 8;
    static constexpr int OFF_MAX = OFF_MISC + 16;             // [2 tiles][2 halves][128 rows] fp32
    static constexpr int OFF_IDS = OFF_MAX + 2048;            // page numbers on their way to the copies
    static constexpr int BYTES = OFF_IDS + 64 * 4;
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

// Bounded wait on the barriers that products and softmax hand over by, every thousand clocks or so.  try_wait lets the
// hardware hold the warp and wake it when the phase ends; polling with test_wait instead floods the unit that answers it (and
// copies between registers and tensor memory go through), and made everything else in the block slower (measured).
// Gives up like wait_or_abort.
__device__ __forceinline__ bool poll_or_abort(uint64_t* bar, uint32_t parity, volatile uint32_t* abort_flag) {
    for (uint32_t i = 0; i < (1u << 20); ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if (*abort_flag) return false;
        if (i > 4096) __nanosleep(256);
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

// Vote of the 256 threads that hold a row tile (both halves of its keys), and a barrier among them.
__device__ __forceinline__ bool tile_any(int w, bool flag) {
    uint32_t any;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(any)
        : "r"(flag ? 1u : 0u), "r"(w + 1)
        : "memory");
    return any != 0;
}

// 32 bytes in one store: a thread's row is its own, so narrower stores would write half sectors
__device__ __forceinline__ void store_sector(float* p, const float* v) {
    asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]),
                 "f"(v[5]), "f"(v[6]), "f"(v[7])
                 : "memory");
}

template <int D>
__global__ void __launch_bounds__(kUmmaAttnThreads, 1)
attn_umma_prefix_kernel(const UmmaAttnParams up, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
    using Geo = UmmaAttnGeo<D>;
    extern __shared__ __align__(1024) unsigned char umma_attn_smem[];
    const AttnParams& p = up.a;
    unsigned char* smem = umma_attn_smem;
    if (smem_u32(smem) & 1023u) {  // the swizzle counts on it (dynamic shared memory starts on such a boundary)
        attn_report(kAttnErrWait);
        return;
    }
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + Geo::OFF_BARS);
    uint64_t* kv_full = bars;
    uint64_t* kv_empty = bars + Geo::STAGES;
    uint64_t* s_full = bars + 2 * Geo::STAGES;   // [2] scores of a tile's step are in tensor memory
    uint64_t* p_ready = s_full + 2;              // [2] its weights are
    uint64_t* o_done = s_full + 4;               // [2] its second product is complete
    uint64_t* all_done = s_full + 6;             // every product issued is complete
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + Geo::OFF_MISC);
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(smem + Geo::OFF_MISC + 4);

    // The warp's number by way of a shuffle, so that the compiler knows it to be the same for the whole warp: descriptors then
    // stay in uniform registers and a product takes 30 clocks to issue instead of 100, and 64 to run (128 x 128 x 16).
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(kFullMask, tid >> 5, 0);
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
    if (warp == 16) {
        tmem_alloc(tmem_slot, 512);
        tmem_relinquish();
    }
    // The copies, by warp 17: the items in the order in which the products take them.  Page numbers come 32 at a time, one per lane,
    // and the next 32 are on their way while these are used.
    int item = 0, of = 0, loaded = 0;
    const int list = static_cast<int>((p.prefix_len + (1 << p.page_shift) - 1) >> p.page_shift);
    int filled = key0 >> p.page_shift, ahead = -1;  // list entries below `filled` have been put into `ids`; `ahead`: this lane's next one
    int32_t* ids = reinterpret_cast<int32_t*>(smem + Geo::OFF_IDS);
    auto fetch_ids = [&]() { ahead = filled + lane < list ? __ldg(p.prefix_pages + filled + lane) : 0; };
    auto copy_items = [&]() {
        const int page = 1 << p.page_shift;
        for (; item < 2 * steps_of(0); ++item, of = 0) {
            for (; of < (same ? 2 : 1); ++of) {
                if (item >= 2 * steps_of(of)) break;
                const Place at = place_of(of, item);
                const int first = (key0 + key_tile(of, item >> 1) * 128) >> p.page_shift;
                const int n = min(128 >> p.page_shift, list - first);
                while (filled < first + n) {
                    int pg = ahead;
                    if (pg < 0 || pg >= p.num_pages) {
                        attn_report(kAttnErrIndex);
                        pg = 0;
                    }
                    ids[(filled + lane) & 63] = pg;
                    filled += 32;
                    fetch_ids();
                    __syncwarp();
                }
                if (!__all_sync(kFullMask, wait_or_abort(kv_empty + at.stage, at.parity ^ 1u, abort_flag))) return false;
                const CUtensorMap* map = item & 1 ? &v_map : &k_map;
                if (lane == 0) {
                    mbar_expect_tx(kv_full + at.stage, static_cast<uint32_t>(n * page * 128 * Geo::HALVES));
                    for (int i = 0; i < n; ++i) {
                        const int y = (ids[(first + i) & 63] * p.hkv + head) << p.page_shift;
#pragma unroll
                        for (int h = 0; h < Geo::HALVES; ++h)
                            tma_load_2d(smem_u32(smem) + Geo::OFF_RING + at.stage * Geo::TILE + h * Geo::BOX + i * page * 128, map, h * 64, y,
                                        kv_full + at.stage);
                    }
                }
                __syncwarp();
                ++loaded;
            }
        }
        return true;
    };
    if (warp == 17) fetch_ids();
    if (tid == 17 * 32) {
        for (int s = 0; s < Geo::STAGES; ++s) {
            mbar_init(kv_full + s, 1);
            mbar_init(kv_empty + s, same ? 1 : 2);  // as many row tiles read it
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(s_full + s, 1);
            mbar_init(p_ready + s, 8);
            mbar_init(o_done + s, 1);
        }
        mbar_init(all_done, 1);
        *abort_flag = 0;
        fence_mbar_init();
    }
    // queries, by the softmax warps: 128-byte rows of 64 channels, chunks permuted by the row as the copies' swizzle does
    if (warp < 16) {
        const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p.q);
        constexpr int CH = Geo::HALVES * 8, BATCH = 256 * CH / 512;   // chunks a row and a thread, all loads in flight
        constexpr int STEP = 512 / CH;           // rows from one chunk of a thread to its next
        const int c = tid % CH, step_tok = STEP / p.group, step_in = STEP % p.group;
        int row = row0 + tid / CH, tok = row / p.group, in = row - tok * p.group;
        uint4 v[BATCH];
#pragma unroll
        for (int e = 0; e < BATCH; ++e) {
            if (same && e == BATCH / 2) {        // the second tile has the first one's rows
                row -= 128;
                tok = row / p.group;
                in = row - tok * p.group;
            }
            v[e] = make_uint4(0, 0, 0, 0);
            if (row < rows && c * 8 < D)
                v[e] = __ldg(reinterpret_cast<const uint4*>(q + tok * p.q_st + (static_cast<int64_t>(head) * p.group + in) * p.q_sh) + c);
            row += STEP;
            tok += step_tok;
            in += step_in;
            if (in >= p.group) {
                in -= p.group;
                ++tok;
            }
        }
#pragma unroll
        for (int e = 0; e < BATCH; ++e) {
            const int r = tid / CH + e * STEP;
            unsigned char* dst = smem + (r >> 7) * Geo::TILE + (c >> 3) * Geo::BOX + (r & 127) * 128 + (((c & 7) ^ (r & 7)) << 4);
            *reinterpret_cast<uint4*>(dst) = v[e];
        }
        fence_async_smem();
    }
    // The copying warp needs nothing from the others: it says that the barriers are set up and goes on.  (Waiting here as well, after
    // it had filled the ring, held the first scores up by 3600 clocks.)  The barrier has a number of its own: where the ring takes all
    // copies of a block at once, this warp comes to the block's last barrier while others are still here.
    tc_fence_before();
    if (warp == 17) {
        __threadfence_block();
        __syncwarp();
        asm volatile("bar.arrive %0, %1;" ::"n"(kStartBarrier), "n"(kUmmaAttnThreads) : "memory");
    } else {
        asm volatile("bar.sync %0, %1;" ::"n"(kStartBarrier), "n"(kUmmaAttnThreads) : "memory");
    }
    tc_fence_after();
    const uint32_t tmem = warp == 17 ? 0u : __shfl_sync(kFullMask, *tmem_slot, 0);
    const uint32_t ring = smem_u32(smem) + Geo::OFF_RING;

    if (warp == 17) {
        if (!copy_items()) {  // given up: the copies in flight still write this block's memory
            for (int k = 0, j = 0; k < loaded; ++j)
                for (int w = 0; w < (same ? 2 : 1) && k < loaded; ++w) {
                    if (j >= 2 * steps_of(w)) break;
                    if (k++ < loaded - Geo::STAGES) continue;
                    const Place at = place_of(w, j);
                    mbar_wait_bounded(kv_full + at.stage, at.parity);
                }
        }
    } else if (warp == 16) {
        // One warp issues all products, the tiles strictly in turn: a tile's second product and its next scores go to the tensor core as
        // one piece, so that its softmax starts while the other tile's piece runs.  (With a warp per tile the two tiles shared
        // the tensor core, ended together and then shared the exponential unit: no overlap, measured.)  The whole warp walks the loop
        // and one elected lane issues, so that descriptors and barrier addresses stay in uniform registers.
        constexpr uint32_t qk_idesc = umma_attn_idesc(128, false), pv_idesc = umma_attn_idesc(D, true);
        const uint64_t q_desc0 = umma_desc_sw128(smem_u32(smem), 16);
        const int n0 = steps_of(0), n1 = steps_of(1);
        bool ok = true;
        auto scores = [&](int w, int i) {   // S of tile w's step i
            const Place at = place_of(w, 2 * i);
            if (!warp_poll_or_abort(kv_full + at.stage, at.parity, abort_flag)) return false;
            tc_fence_after();
            const uint64_t q_desc = q_desc0 + static_cast<uint64_t>(w * (Geo::TILE >> 4));
            const uint64_t k_desc = umma_desc_sw128(ring + at.stage * Geo::TILE, 16);
            if (elect_one()) {
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    constexpr int kBox = Geo::BOX;
                    const uint64_t off = static_cast<uint64_t>(((k >> 2) * kBox + (k & 3) * 32) >> 4);
                    umma_bf16(tmem + w * 128, q_desc + off, k_desc + off, qk_idesc, k > 0);
                }
                umma_commit(s_full + w);
                umma_commit(kv_empty + at.stage);
            }
            __syncwarp();
            return true;
        };
        if (n0 > 0) ok = scores(0, 0);
        if (ok && n1 > 0) ok = scores(1, 0);
        for (int i = 0; ok && i < n0; ++i) {
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                if (w == 1 && i >= n1) break;
                const uint32_t o_cols = tmem + 256 + w * Geo::O_COLS, p_cols = tmem + w * 128;
                const Place at = place_of(w, 2 * i + 1);
                ok = ok && warp_poll_or_abort(kv_full + at.stage, at.parity, abort_flag) &&
                     warp_poll_or_abort(p_ready + w, static_cast<uint32_t>(i) & 1u, abort_flag);
                if (!ok) break;
                tc_fence_after();
                const uint64_t v_desc = umma_desc_sw128(ring + at.stage * Geo::TILE, Geo::BOX);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) umma_bf16_a_tmem(o_cols, p_cols + k * 8, v_desc + k * 128, pv_idesc, i > 0 || k > 0);
                    umma_commit(o_done + w);
                    umma_commit(kv_empty + at.stage);
                }
                __syncwarp();
                // the tensor core runs a tile's products in order: the next scores may overwrite the weights just used
                if (i + 1 < (w ? n1 : n0)) ok = scores(w, i + 1);
                if (!ok) break;
            }
        }
        if (elect_one()) umma_commit(all_done);
        __syncwarp();
        if (!mbar_wait_bounded(all_done, 0)) *abort_flag = 1;
    } else {
        // 16 softmax warps: tile w, half h of the keys; warp & 3 says which 32 lanes of tensor memory it may read
        const int w = warp >> 3, h = (warp >> 2) & 1;
        const int lane_row = (warp & 3) * 32 + lane;
        const int r = row0 + (same ? 0 : w * 128) + lane_row;
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t s_cols = tmem + w * 128 + h * 64 + lanes, p_cols = tmem + w * 128 + h * 32 + lanes;
        const uint32_t o_cols = tmem + 256 + w * Geo::O_COLS + lanes;
        constexpr int O_HALF = D / 2;            // each half's warps scale and write half of the channels
        float* maxima = reinterpret_cast<float*>(smem + Geo::OFF_MAX) + w * 256;
        const float sl = p.scale_log2;
        const int n = steps_of(w);
        float m = 0.0f, l = 0.0f;                // reference maximum in units of the raw scores (the same in both halves), this half's sum
        float slope = sl;                        // the row's scale in the exponents
        bool ok = true;
        for (int i = 0; i < n; ++i) {
            const int valid = min(128, key1 - key0 - key_tile(w, i) * 128) - h * 64;  // of this half's 64 keys
            ok = ok && warp_poll_or_abort(s_full + w, static_cast<uint32_t>(i) & 1u, abort_flag);
            tc_fence_after();
            auto load = [&](uint32_t (&x)[32], int c0) {
                tmem_ld32(s_cols + c0, x);
                tmem_wait_ld();
                if (valid < c0 + 32) {
#pragma unroll
                    for (int c = 0; c < 32; ++c)
                        if (c0 + c >= valid) x[c] = 0xff800000u;  // -infinity
                }
            };
            // The half's weights against the reference m slope, rounded up so that none passes 1, as bf16 pairs.  Returns the sum of what the
            // pairs hold: the result is then a mean with just these weights, and that of a row with one key that counts is its value.
            uint32_t y[32];
            auto weights = [&]() {
                const float off = -__fmul_ru(m, slope);
                const uint64_t off2 = pair(off, off), sl2 = pair(slope, slope);
                uint64_t sum[2] = {0, 0};
#pragma unroll
                for (int c = 0; c < 64; c += 32) {
                    uint32_t x[32];
                    load(x, c);
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float a, b;
                        unpair(fma2(pair(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), sl2, off2), a, b);
                        a = exp2_fast(a);
                        b = exp2_fast(b);
                        const uint32_t ab = pack_bf16x2(a, b);
                        y[(c + e) / 2] = ab;
                        sum[(e >> 1) & 1] = add2(sum[(e >> 1) & 1], pair(__uint_as_float(ab << 16), __uint_as_float(ab & 0xffff0000u)));
                    }
                }
                float a, b;
                unpair(add2(sum[0], sum[1]), a, b);
                return a + b;
            };
            // One vote of both halves' warps per round: nobody stores weights before all agree on the reference.  (A wait that ran
            // out also ends up here, so that all leave together: the votes are barriers.)  The reference moves once per step at most: it is
            // the tile's maximum then, whatever the sum that follows.
            float sum = 0.0f;
            bool gave_up = false;
            for (bool moved = false;; moved = true) {
                if (i > 0 || moved) {
                    sum = weights();
                    if (!tile_any(w, !ok || (!moved && sum > kLargestHalf))) break;
                }
                // The first tile, and later the rare case that some row's weights have grown past kLargestHalf: the row's
                // reference moves to the maximum of the tile.  O and l follow; its products so far are waited for.
                float top = -INFINITY;
#pragma unroll 1
                for (int c = 0; c < 64; c += 32) {
                    uint32_t x[32];
                    load(x, c);
#pragma unroll
                    for (int e = 0; e < 32; e += 2) top = max3(top, __uint_as_float(x[e]), __uint_as_float(x[e + 1]));
                }
                maxima[h * 128 + lane_row] = top;
                if (i > 0) ok = ok && warp_poll_or_abort(o_done + w, static_cast<uint32_t>(i - 1) & 1u, abort_flag);
                if ((gave_up = tile_any(w, !ok))) break;
                top = fmaxf(maxima[lane_row], maxima[128 + lane_row]);
                if (i == 0) {
                    m = top;
                } else {
                    tc_fence_after();
                    const bool higher = top > m;
                    const float f = higher ? exp2_fast(__fsub_rn(__fmul_ru(m, sl), __fmul_ru(top, sl))) : 1.0f;
                    if (higher) m = top;
                    l *= f;
#pragma unroll 1
                    for (int c = h * O_HALF; c < (h + 1) * O_HALF; c += 16) {
                        float o[16];
                        tmem_ld16(o_cols + c, o);
                        tmem_wait_ld();
                        uint32_t z[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) z[e] = __float_as_uint(o[e] * f);
                        tmem_st16(o_cols + c, z);
                    }
                }
                slope = fabsf(m * sl) > kLargestReference ? kLargestReference / fabsf(m) : sl;
            }                   // (the next vote also says that everyone has read the maxima)
            if (gave_up) break;
            l += sum;
            tmem_st16(p_cols, y);
            tmem_st16(p_cols + 16, y + 16);
            if (valid < 64) {
                // the tile's last rows hold keys that nobody sees, or nothing at all: their values become 0 so that a
                // weight of 0 takes nothing from them
                const Place at = place_of(w, 2 * i + 1);
                ok = ok && warp_poll_or_abort(kv_full + at.stage, at.parity, abort_flag);
                unsigned char* v = smem + Geo::OFF_RING + at.stage * Geo::TILE + h * 64 * 128;
                const int from = max(0, valid);
                for (int e = lane_row; e < (64 - from) * 8 * Geo::HALVES; e += 128) {
                    const int row = from + e / (8 * Geo::HALVES), c = e % (8 * Geo::HALVES);
                    *reinterpret_cast<uint4*>(v + (c >> 3) * Geo::BOX + row * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
                }
                fence_async_smem();
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_ready + w);
        }
        if (n > 0) ok = ok && warp_poll_or_abort(o_done + w, static_cast<uint32_t>(n - 1) & 1u, abort_flag);
        tc_fence_after();
        if (!tile_any(w, !ok)) {
            const int tok = r / p.group;
            const int64_t at = static_cast<int64_t>(tok) * p.hq + head * p.group + (r - tok * p.group);
            const int part = same ? 2 * split + w : split;
            const int64_t slot = static_cast<int64_t>(part) * p.T * p.hq + at;
#pragma unroll 1
            for (int c = h * O_HALF; c < (h + 1) * O_HALF; c += 16) {
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
                    for (int e = 0; e < 16; e += 8) store_sector(p.part_o + slot * D + c + e, o + e);
                }
            }
            if (h == 1) maxima[128 + lane_row] = l;
            tile_any(w, false);
            if (h == 0 && r < rows) p.part_ml[slot] = n > 0 ? make_float2(__fmul_ru(m, sl), l + maxima[128 + lane_row]) : make_float2(-INFINITY, 0.0f);
        }
        tc_fence_before();
    }
    __syncwarp();
    __syncthreads();
    if (warp == 16) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

}  // namespace wht
