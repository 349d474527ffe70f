// Paged-cache append with the position rotation.
//
//     k'[i] = k[i] cos - k[j] sin      k'[j] = k[j] cos + k[i] sin          pairs (i, j) = (i, i + R/2) or (2i, 2i + 1)
//
// A pass over memory: every element is read once and written once, at most three operations each, so DRAM (prompts)
// or the launch itself (single tokens) bounds it.  A thread owns 16 elements of one row, the two halves of eight
// pairs, so every access is 128 bits wide and no value crosses threads.  The angles' rows (R * 4 bytes a token) are shared by all heads
// of a token and come from the caches.
//
// With page summaries the keys are walked by page instead: one warp takes the run of tokens that a call adds
// to one page for one head, keeps the channels' least and largest whole values in registers as 16-bit pairs, folds
// the rows of the warp by shuffles and joins the page's stored summary once.  No atomics: a run has one owner.
#pragma once
#include "attn_common.cuh"

namespace wht {

struct AppendParams {
    const void *k, *v, *q;
    int64_t k_st, k_sh, v_st, v_sh, q_st, q_sh;
    void *q_out, *k_cache, *v_cache;
    const int64_t* slots;
    const int32_t* positions;
    const float *cos_t, *sin_t;
    int8_t* summary;
    const float* summary_scale;
    int64_t T, max_pos, num_slots;
    int hq, hkv, d, rot, page_shift;
    int rows;            // rows per token that the flat part handles: hq (q) [+ hkv (k)] + hkv (v)
    int tile;            // tokens per block of the flat part
    int flat_x, flat_y;  // its blocks: token tiles, and blocks per tile
    int run_tile;        // tokens per block of the page part
};

__device__ __forceinline__ void load16(const float* p, float (&v)[16]) {
    load8(p, reinterpret_cast<float(&)[8]>(v[0]));
    load8(p + 8, reinterpret_cast<float(&)[8]>(v[8]));
}

template <typename T>
__device__ __forceinline__ T* row_of(void* base, int64_t off) { return static_cast<T*>(base) + off; }
template <typename T>
__device__ __forceinline__ const T* row_of(const void* base, int64_t off) { return static_cast<const T*>(base) + off; }

// The value a stored element has: rounded to the type.
__device__ __forceinline__ float stored(float x, const float*) { return x; }
__device__ __forceinline__ float stored(float x, const __nv_bfloat16*) { return __bfloat162float(__float2bfloat16_rn(x)); }

// One item of a row: 16 elements as two groups of eight, at lo and hi.  Items below rot/16 turn; the pairs are
// (lo[i], hi[i]) (halves) or neighbours (interleaved); the others pass through.
template <typename T, bool INTERLEAVED>
struct RowItem {
    int lo, hi;      // element offsets of the two groups
    int angle;       // offset of the eight angles, or -1
    __device__ __forceinline__ RowItem(int item, int rot) {
        if (item < rot / 16) {
            angle = item * 8;
            lo = INTERLEAVED ? item * 16 : item * 8;
            hi = INTERLEAVED ? lo + 8 : lo + rot / 2;
        } else {
            angle = -1;
            lo = item * 16;
            hi = lo + 8;
        }
    }
    __device__ __forceinline__ void turn(float (&a)[8], float (&b)[8], const float* cos_row, const float* sin_row) const {
        if (angle < 0) return;
        float c[8], s[8];
        load8(cos_row + angle, c);
        load8(sin_row + angle, s);
        if constexpr (INTERLEAVED) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                rotate(a[2 * i], a[2 * i + 1], c[i], s[i]);
                rotate(b[2 * i], b[2 * i + 1], c[4 + i], s[4 + i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) rotate(a[i], b[i], c[i], s[i]);
        }
    }
    // every product and sum rounded on its own: the stored keys are a function of the inputs alone
    __device__ __forceinline__ static void rotate(float& x, float& y, float c, float s) {
        const float x2 = __fsub_rn(__fmul_rn(x, c), __fmul_rn(y, s));
        y = __fadd_rn(__fmul_rn(y, c), __fmul_rn(x, s));
        x = x2;
    }
};

__device__ __forceinline__ int64_t append_position(const AppendParams& p, int64_t t) {
    if (p.rot == 0) return 0;
    const int64_t pos = __ldg(p.positions + t);
    if (pos < 0 || pos >= p.max_pos) {
        attn_report(kAttnErrIndex);
        return pos < 0 ? 0 : p.max_pos - 1;
    }
    return pos;
}
// The token's slot, or -1 for padding and for slots outside the cache (reported).
__device__ __forceinline__ int64_t append_slot(const AppendParams& p, int64_t t) {
    const int64_t s = __ldg(reinterpret_cast<const long long*>(p.slots) + t);
    if (s >= p.num_slots) {
        attn_report(kAttnErrIndex);
        return -1;
    }
    return s < 0 ? -1 : s;
}
__device__ __forceinline__ int64_t cache_offset(const AppendParams& p, int64_t slot, int head) {
    const int64_t page = slot >> p.page_shift, place = slot & ((1 << p.page_shift) - 1);
    return (((page * p.hkv + head) << p.page_shift) + place) * p.d;
}

// Flat part: queries, values and (without summaries) keys, item by item.
template <typename T, bool INTERLEAVED, bool SUMMARY>
__device__ __forceinline__ void append_flat(const AppendParams& p, int block) {
    const int per_row = p.d / 16, per_token = p.rows * per_row;
    const int bx = block / p.flat_y, by = block - bx * p.flat_y;
    const int64_t t0 = static_cast<int64_t>(bx) * p.tile;
    const int count = static_cast<int>(p.T - t0 < p.tile ? p.T - t0 : p.tile) * per_token;
    for (int j = by * blockDim.x + threadIdx.x; j < count; j += p.flat_y * blockDim.x) {
        const int dt = j / per_token;
        int r = j - dt * per_token;
        int row = r / per_row;
        const RowItem<T, INTERLEAVED> it(r - row * per_row, p.rot);
        const int64_t t = t0 + dt;
        const T* src;
        T* dst;
        bool turns = true;
        if (row < p.hq) {
            src = row_of<T>(p.q, t * p.q_st + row * p.q_sh);
            dst = row_of<T>(p.q_out, (t * p.hq + row) * p.d);
        } else {
            row -= p.hq;
            const int64_t slot = append_slot(p, t);
            if (slot < 0) continue;
            if (!SUMMARY && row < p.hkv) {
                src = row_of<T>(p.k, t * p.k_st + row * p.k_sh);
                dst = row_of<T>(p.k_cache, cache_offset(p, slot, row));
            } else {
                if (!SUMMARY) row -= p.hkv;
                src = row_of<T>(p.v, t * p.v_st + row * p.v_sh);
                dst = row_of<T>(p.v_cache, cache_offset(p, slot, row));
                turns = false;
            }
        }
        float a[8], b[8];
        load8(src + it.lo, a);
        load8(src + it.hi, b);
        if (turns && it.angle >= 0) {
            const int64_t pos = append_position(p, t);
            it.turn(a, b, p.cos_t + pos * (p.rot / 2), p.sin_t + pos * (p.rot / 2));
        }
        store8(dst + it.lo, a);
        store8(dst + it.hi, b);
    }
}

__device__ __forceinline__ unsigned pack_s16(int lo, int hi) {
    return (static_cast<unsigned>(lo) & 0xffffu) | (static_cast<unsigned>(hi) << 16);
}

// Page part: this warp's runs of one head.
template <typename T, bool INTERLEAVED>
__device__ __forceinline__ void append_pages(const AppendParams& p, int64_t tile0, int head) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int per_row = p.d / 16;
    int rows = 1;  // rows of a warp's step: a power of two, so that they fold by shuffles
    while (rows * 2 * per_row <= 32) rows *= 2;
    const int sub = lane / per_row;
    const RowItem<T, INTERLEAVED> it(lane - sub * per_row, p.rot);
    const bool active = sub < rows;
    // which of the tile's tokens begin a run
    int64_t page = -1, before = -1;
    if (lane < p.run_tile && tile0 + lane < p.T) {
        const int64_t s = append_slot(p, tile0 + lane);
        if (s >= 0) page = s >> p.page_shift;
        if (tile0 + lane > 0) {
            const int64_t s1 = append_slot(p, tile0 + lane - 1);
            if (s1 >= 0) before = s1 >> p.page_shift;
        }
    }
    unsigned leaders = __ballot_sync(kFullMask, page >= 0 && page != before);
    const float scale = __ldg(p.summary_scale + head);
    for (int n = 0; leaders; ++n) {
        const int l = __ffs(leaders) - 1;
        leaders &= leaders - 1;
        if (n % warps != warp) continue;
        const int64_t first = tile0 + l;
        const int64_t run_page = __shfl_sync(kFullMask, page, l);
        // the run's length: the tokens that follow on the same page
        int len = 1;
        for (;;) {
            const int64_t t = first + len + lane;
            bool same = false;
            if (t < p.T) {
                const int64_t s = append_slot(p, t);
                same = s >= 0 && (s >> p.page_shift) == run_page;
            }
            const unsigned other = ~__ballot_sync(kFullMask, same);
            if (other) {
                len += __ffs(other) - 1;
                break;
            }
            len += 32;
        }
        unsigned least[8], most[8];  // 16 channels as 16-bit pairs
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            least[i] = pack_s16(127, 127);
            most[i] = pack_s16(-127, -127);
        }
#pragma unroll 2
        for (int r = sub; r < len; r += rows) {
            if (!active) break;
            const int64_t t = first + r;
            const int64_t slot = append_slot(p, t);
            const T* src = row_of<T>(p.k, t * p.k_st + head * p.k_sh);
            T* dst = row_of<T>(p.k_cache, cache_offset(p, slot, head));
            float a[8], b[8];
            load8(src + it.lo, a);
            load8(src + it.hi, b);
            if (it.angle >= 0) {
                const int64_t pos = append_position(p, t);
                it.turn(a, b, p.cos_t + pos * (p.rot / 2), p.sin_t + pos * (p.rot / 2));
            }
            store8(dst + it.lo, a);
            store8(dst + it.hi, b);
            int w[16];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = max(-127, min(127, __float2int_rn(__fmul_rn(stored(a[i], src), scale))));
                w[8 + i] = max(-127, min(127, __float2int_rn(__fmul_rn(stored(b[i], src), scale))));
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const unsigned x = pack_s16(w[2 * i], w[2 * i + 1]);
                least[i] = __vmins2(least[i], x);
                most[i] = __vmaxs2(most[i], x);
            }
        }
        for (int step = rows / 2; step >= 1; step >>= 1) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                least[i] = __vmins2(least[i], __shfl_down_sync(kFullMask, least[i], step * per_row));
                most[i] = __vmaxs2(most[i], __shfl_down_sync(kFullMask, most[i], step * per_row));
            }
        }
        if (lane < per_row) {
            const bool anew = (append_slot(p, first) & ((1 << p.page_shift) - 1)) == 0;
            int8_t* at = p.summary + ((run_page * p.hkv + head) * 2) * p.d;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                int8_t* lo = at + (half ? it.hi : it.lo);
                int8_t* hi = lo + p.d;
                uint2 old_lo, old_hi, new_lo, new_hi;
                if (!anew) {
                    old_lo = *reinterpret_cast<const uint2*>(lo);
                    old_hi = *reinterpret_cast<const uint2*>(hi);
                }
                unsigned wl[2], wh[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {  // four channels: two pairs to four bytes
                    const unsigned l0 = least[half * 4 + 2 * j], l1 = least[half * 4 + 2 * j + 1];
                    const unsigned h0 = most[half * 4 + 2 * j], h1 = most[half * 4 + 2 * j + 1];
                    wl[j] = __byte_perm(l0, l1, 0x6420);
                    wh[j] = __byte_perm(h0, h1, 0x6420);
                }
                new_lo = make_uint2(wl[0], wl[1]);
                new_hi = make_uint2(wh[0], wh[1]);
                if (!anew) {
                    new_lo = make_uint2(__vmins4(new_lo.x, old_lo.x), __vmins4(new_lo.y, old_lo.y));
                    new_hi = make_uint2(__vmaxs4(new_hi.x, old_hi.x), __vmaxs4(new_hi.y, old_hi.y));
                }
                *reinterpret_cast<uint2*>(lo) = new_lo;
                *reinterpret_cast<uint2*>(hi) = new_hi;
            }
        }
    }
}

constexpr int kAppendThreads = 256;

template <typename T, bool INTERLEAVED, bool SUMMARY>
__global__ void __launch_bounds__(kAppendThreads)
kv_append_kernel(const AppendParams p) {
    const int flat = p.flat_x * p.flat_y;
    if (SUMMARY && static_cast<int>(blockIdx.x) >= flat) {
        const int b = static_cast<int>(blockIdx.x) - flat;
        append_pages<T, INTERLEAVED>(p, static_cast<int64_t>(b / p.hkv) * p.run_tile, b % p.hkv);
        return;
    }
    append_flat<T, INTERLEAVED, SUMMARY>(p, blockIdx.x);
}

}  // namespace wht
