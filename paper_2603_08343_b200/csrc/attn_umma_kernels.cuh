// Shared-prefix attention of many rows on the tcgen05 tensor core (bf16).
//
// Every row (token, query head) of a key head sees the same prefix, so with R rows the two products are dense
// [R x D] x [D x L] and [R x L] x [L x D]: 4 D flops per row and key against 4 D bytes per key, i.e. R flops a byte.
// From about 250 rows on that is the tensor core's balance, and the exponentials (one per row and key,
// 16 a clock and SM) weigh as much as the products.
//
// A block of 10 warps owns 256 rows of one key head as two tiles of 128, and a range of keys:
//   warps 0..3, 4..7   softmax of tile 0 / tile 1: one thread per row
//   warp 8             issues the products;   warp 9   copies keys and values (TMA, a ring of 128-key tiles)
// and runs steps of one tile and 128 keys, the two tiles taking turns, so that one tile's softmax runs under the other's products:
//   S = Q K^T            into tensor memory (128 lanes x 128 fp32 columns)
//   P = exp2(S - m)      read by the row's thread, rounded to bf16 and written over S
//   O += P V             P from tensor memory, V from shared memory, O stays in tensor memory (D columns)
// The reference maximum m of a row moves only when a score exceeds it by more than 2^8 (kSlack): weights up to 2^8 are as
// exact in bf16 and fp32 as weights up to 1, and O, which sits in tensor memory, is rescaled a few times per row
// instead of once per tile.  With 128 rows or fewer both tiles hold the SAME rows and take alternate key tiles; they
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

constexpr int kUmmaAttnThreads = 320;

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
    uint64_t* all_done = s_full + 6;             // every product issued is complete
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
    const int steps = same ? tiles : 2 * tiles;  // step j: tile j & 1 of the rows; key tile j (same rows) or j / 2

    grid_launch_dependents();
    if (warp == 8) {
        tmem_alloc(tmem_slot, 512);
        tmem_relinquish();
    }
    if (tid == 9 * 32) {
        for (int s = 0; s < Geo::STAGES; ++s) {
            mbar_init(kv_full + s, 1);
            mbar_init(kv_empty + s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(s_full + s, 1);
            mbar_init(p_ready + s, 4);
            mbar_init(o_done + s, 1);
        }
        mbar_init(all_done, 1);
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

    if (warp == 9) {
        if (lane == 0) {
            // The ring's items in the order in which the products take them: K of steps 0 and 1, then V of step j and K of
            // step j + 2, each key tile once.
            const int list = static_cast<int>((p.prefix_len + (1 << p.page_shift) - 1) >> p.page_shift);
            const int page = 1 << p.page_shift;
            int item = 0;
            bool ok = true;
            auto load = [&](const CUtensorMap* map, int t) {
                const int s = item % Geo::STAGES;
                const uint32_t ph = static_cast<uint32_t>(item / Geo::STAGES) & 1u;
                if (!wait_or_abort(kv_empty + s, ph ^ 1u, abort_flag)) return false;
                const int first = (key0 + t * 128) >> p.page_shift;
                const int n = min(128 >> p.page_shift, list - first);
                mbar_expect_tx(kv_full + s, static_cast<uint32_t>(n * page * 128 * Geo::HALVES));
                for (int i = 0; i < n; ++i) {
                    int pg = __ldg(p.prefix_pages + first + i);
                    if (pg < 0 || pg >= p.num_pages) {
                        attn_report(kAttnErrIndex);
                        pg = 0;
                    }
                    const int y = (pg * p.hkv + head) << p.page_shift;
#pragma unroll
                    for (int h = 0; h < Geo::HALVES; ++h)
                        tma_load_2d(ring + s * Geo::TILE + h * Geo::BOX + i * page * 128, map, h * 64, y, kv_full + s);
                }
                ++item;
                return true;
            };
            if (same) {
                for (int j = -2; ok && j < tiles; ++j) {
                    if (j >= 0) ok = load(&v_map, j);
                    if (ok && j + 2 < tiles) ok = load(&k_map, j + 2);
                }
            } else {
                for (int t = -1; ok && t < tiles; ++t) {
                    if (ok && t >= 0) ok = load(&v_map, t);
                    if (ok && t + 1 < tiles) ok = load(&k_map, t + 1);
                }
            }
            if (!ok) {  // given up: the copies in flight still write this block's memory
                for (int i = item > Geo::STAGES ? item - Geo::STAGES : 0; i < item; ++i)
                    mbar_wait_bounded(kv_full + i % Geo::STAGES, static_cast<uint32_t>(i / Geo::STAGES) & 1u);
            }
        }
    } else if (warp == 8) {
        if (lane == 0) {
            constexpr uint32_t qk_idesc = umma_attn_idesc(128, false), pv_idesc = umma_attn_idesc(D, true);
            const uint32_t q_addr = smem_u32(smem);
            // ring item of key tile t's keys and values, in the loader's order
            auto k_item = [&](int t) { return same ? (t < 2 ? t : 2 * t - 1) : 2 * t; };
            auto v_item = [&](int t) { return same ? (t == tiles - 1 ? 2 * t + 1 : 2 * t + 2) : 2 * t + 1; };
            bool ok = true;
            auto scores = [&](int j) {   // S of step j
                const int w = j & 1, t = same ? j : j >> 1;
                const int item = k_item(t), s = item % Geo::STAGES;
                if (!wait_or_abort(kv_full + s, static_cast<uint32_t>(item / Geo::STAGES) & 1u, abort_flag)) return false;
                tc_fence_after();
                const uint32_t k_addr = ring + s * Geo::TILE;
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint32_t off = (k >> 2) * Geo::BOX + (k & 3) * 32;
                    umma_bf16(tmem + w * 128, umma_desc_sw128(q_addr + w * Geo::TILE + off, 16), umma_desc_sw128(k_addr + off, 16),
                              qk_idesc, k > 0);
                }
                umma_commit(s_full + w);
                if (same || w == 1) umma_commit(kv_empty + s);
                return true;
            };
            for (int j = 0; ok && j < 2 && j < steps; ++j) ok = scores(j);
            for (int j = 0; ok && j < steps; ++j) {
                const int w = j & 1, t = same ? j : j >> 1, i = j >> 1;
                const int item = v_item(t), s = item % Geo::STAGES;
                ok = wait_or_abort(p_ready + w, static_cast<uint32_t>(i) & 1u, abort_flag) &&
                     wait_or_abort(kv_full + s, static_cast<uint32_t>(item / Geo::STAGES) & 1u, abort_flag);
                if (!ok) break;
                tc_fence_after();
                const uint32_t v_addr = ring + s * Geo::TILE;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    umma_bf16_a_tmem(tmem + 256 + w * Geo::O_COLS, tmem + w * 128 + k * 8, umma_desc_sw128(v_addr + k * 2048, Geo::BOX),
                                     pv_idesc, i > 0 || k > 0);
                umma_commit(o_done + w);
                if (same || w == 1) umma_commit(kv_empty + s);
                // the tensor core runs its products in order: the next scores may overwrite the weights just used
                if (j + 2 < steps) ok = scores(j + 2);
            }
            umma_commit(all_done);
            if (!mbar_wait_bounded(all_done, 0)) *abort_flag = 1;
        }
    } else {
        const int w = warp >> 2;
        const int r = row0 + (same ? 0 : w * 128) + (warp & 3) * 32 + lane;
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t s_cols = tmem + w * 128 + lanes, o_cols = tmem + 256 + w * Geo::O_COLS + lanes;
        const float sl = p.scale_log2;
        const int n = steps > w ? (steps - w + 1) / 2 : 0;
        SoftmaxRow st;
        bool ok = true;
        for (int i = 0; i < n; ++i) {
            const int t = same ? 2 * i + w : i;
            const int valid = min(128, key1 - key0 - t * 128);
            ok = warp_wait_or_abort(s_full + w, static_cast<uint32_t>(i) & 1u, abort_flag);
            if (!ok) break;
            tc_fence_after();
            uint32_t x[128];
#pragma unroll
            for (int c = 0; c < 128; c += 32) tmem_ld32(s_cols + c, x + c);
            tmem_wait_ld();
            if (valid < 128) {
#pragma unroll
                for (int c = 0; c < 128; ++c)
                    if (c >= valid) x[c] = 0xff800000u;  // -infinity
            }
            float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int c = 0; c < 128; c += 8)
#pragma unroll
                for (int e = 0; e < 4; ++e) top[e] = max3(top[e], __uint_as_float(x[c + e]), __uint_as_float(x[c + 4 + e]));
            const float mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
            if (i == 0) {
                st.m = mx;
            } else {
                const bool move = (mx - st.m) * sl > kSlack;
                if (__any_sync(kFullMask, move)) {
                    ok = warp_wait_or_abort(o_done + w, static_cast<uint32_t>(i - 1) & 1u, abort_flag);
                    if (!ok) break;
                    tc_fence_after();
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
                    tmem_wait_st();
                }
            }
            const uint64_t off2 = pair(-st.m * sl, -st.m * sl), sl2 = pair(sl, sl);
            uint64_t sum[2] = {0, 0};
#pragma unroll
            for (int c = 0; c < 128; c += 32) {
                uint32_t y[16];
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    float a, b;
                    unpair(fma2(pair(__uint_as_float(x[c + e]), __uint_as_float(x[c + e + 1])), sl2, off2), a, b);
                    a = exp2_fast(a);
                    b = exp2_fast(b);
                    sum[(e >> 1) & 1] = add2(sum[(e >> 1) & 1], pair(a, b));
                    y[e / 2] = pack_bf16x2(a, b);
                }
                tmem_st16(s_cols + c / 2, y);
            }
            {
                float a, b;
                unpair(add2(sum[0], sum[1]), a, b);
                st.l += a + b;
            }
            if (valid < 128) {
                // the tile's last rows hold keys that nobody sees, or nothing at all: their values become 0 so that a
                // weight of 0 takes nothing from them
                const int item = same ? (t == tiles - 1 ? 2 * t + 1 : 2 * t + 2) : 2 * t + 1;
                const int s = item % Geo::STAGES;
                ok = warp_wait_or_abort(kv_full + s, static_cast<uint32_t>(item / Geo::STAGES) & 1u, abort_flag);
                if (!ok) break;
                unsigned char* v = smem + Geo::OFF_RING + s * Geo::TILE;
                for (int e = (warp & 3) * 32 + lane; e < (128 - valid) * 8 * Geo::HALVES; e += 128) {
                    const int row = valid + e / (8 * Geo::HALVES), c = e % (8 * Geo::HALVES);
                    *reinterpret_cast<uint4*>(v + (c >> 3) * Geo::BOX + row * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
                }
                fence_async_smem();
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_ready + w);
        }
        if (ok && n > 0) {
            ok = warp_wait_or_abort(o_done + w, static_cast<uint32_t>(n - 1) & 1u, abort_flag);
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
