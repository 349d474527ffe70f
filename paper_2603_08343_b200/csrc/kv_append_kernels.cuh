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
    int q_blocks, kv_blocks;  // blocks of heads
    int tile;                 // tokens per tile of the flat part
    int flat_x, flat_y;       // its thread blocks: token tiles, and blocks per tile
    int run_tile;             // tokens per block of the page part
    int run_heads;            // heads per block of the page part
};

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
    __device__ __forceinline__ void turn(float (&a)[8], float (&b)[8], const float (&c)[8], const float (&s)[8]) const {
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

// Eight stored elements as they lie in memory, so that several loads can be in flight in few registers.
template <typename T>
struct Raw8 {
    uint4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) w[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
    }
    __device__ __forceinline__ void store(T* p) const {
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) reinterpret_cast<uint4*>(p)[i] = w[i];
    }
    __device__ __forceinline__ void widen(float (&v)[8]) const {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                v[4 * i] = __uint_as_float(w[i].x); v[4 * i + 1] = __uint_as_float(w[i].y);
                v[4 * i + 2] = __uint_as_float(w[i].z); v[4 * i + 3] = __uint_as_float(w[i].w);
            }
        } else {
            v[0] = bf16lo_to_f32(w[0].x); v[1] = bf16hi_to_f32(w[0].x);
            v[2] = bf16lo_to_f32(w[0].y); v[3] = bf16hi_to_f32(w[0].y);
            v[4] = bf16lo_to_f32(w[0].z); v[5] = bf16hi_to_f32(w[0].z);
            v[6] = bf16lo_to_f32(w[0].w); v[7] = bf16hi_to_f32(w[0].w);
        }
    }
};

// Heads that a thread takes one after the other, all loads in flight at once; they share the angles.
template <typename T>
constexpr int kHeadBlock = sizeof(T) == 4 ? 2 : 4;

// Flat part: queries, values and (without summaries) keys, item by item.
template <typename T, bool INTERLEAVED, bool SUMMARY>
__device__ __forceinline__ void append_flat(const AppendParams& p, int block) {
    constexpr int HB = kHeadBlock<T>;
    const int per_row = p.d / 16;
    const int per_token = (p.q_blocks + (SUMMARY ? 1 : 2) * p.kv_blocks) * per_row;
    const int bx = block / p.flat_y, by = block - bx * p.flat_y;
    const int64_t t0 = static_cast<int64_t>(bx) * p.tile;
    const int count = static_cast<int>(p.T - t0 < p.tile ? p.T - t0 : p.tile) * per_token;
    const int j = by * blockDim.x + threadIdx.x;
    if (j >= count) return;
    const int dt = j / per_token;
    const int r = j - dt * per_token;
    int rb = r / per_row;
    const RowItem<T, INTERLEAVED> it(r - rb * per_row, p.rot);
    const int64_t t = t0 + dt;
    const T* src;
    T* dst;
    int64_t step, out_step;  // from head to head
    int heads;
    bool turns = it.angle >= 0;
    int64_t pos = 0;
    if (turns) pos = append_position(p, t);
    if (rb < p.q_blocks) {
        const int h = rb * HB;
        heads = p.hq - h;
        src = row_of<T>(p.q, t * p.q_st + h * p.q_sh);
        dst = row_of<T>(p.q_out, (t * p.hq + h) * p.d);
        step = p.q_sh;
        out_step = p.d;
    } else {
        rb -= p.q_blocks;
        const int64_t slot = append_slot(p, t);
        if (slot < 0) return;
        const bool is_k = !SUMMARY && rb < p.kv_blocks;
        if (!SUMMARY && !is_k) rb -= p.kv_blocks;
        const int h = rb * HB;
        heads = p.hkv - h;
        src = is_k ? row_of<T>(p.k, t * p.k_st + h * p.k_sh) : row_of<T>(p.v, t * p.v_st + h * p.v_sh);
        dst = row_of<T>(is_k ? p.k_cache : p.v_cache, cache_offset(p, slot, h));
        step = is_k ? p.k_sh : p.v_sh;
        out_step = static_cast<int64_t>(p.d) << p.page_shift;
        turns = turns && is_k;
    }
    Raw8<T> lo[HB], hi[HB];
#pragma unroll
    for (int i = 0; i < HB; ++i) {
        if (i < heads) {
            lo[i].load(src + i * step + it.lo);
            hi[i].load(src + i * step + it.hi);
        }
    }
    if (!turns) {
#pragma unroll
        for (int i = 0; i < HB; ++i) {
            if (i < heads) {
                lo[i].store(dst + i * out_step + it.lo);
                hi[i].store(dst + i * out_step + it.hi);
            }
        }
        return;
    }
    float c[8], s[8];
    load8(p.cos_t + pos * (p.rot / 2) + it.angle, c);
    load8(p.sin_t + pos * (p.rot / 2) + it.angle, s);
#pragma unroll
    for (int i = 0; i < HB; ++i) {
        if (i < heads) {
            float a[8], b[8];
            lo[i].widen(a);
            hi[i].widen(b);
            it.turn(a, b, c, s);
            store8(dst + i * out_step + it.lo, a);
            store8(dst + i * out_step + it.hi, b);
        }
    }
}

__device__ __forceinline__ unsigned pack_s16(int lo, int hi) {
    return (static_cast<unsigned>(lo) & 0xffffu) | (static_cast<unsigned>(hi) << 16);
}

// Page part: the warps of a block share the tile's runs and the block's heads.
template <typename T, bool INTERLEAVED>
__device__ __forceinline__ void append_pages(const AppendParams& p, int64_t tile0, int head0) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int per_row = p.d / 16;
    int rows = 1;  // rows of a warp's step: a power of two, so that they fold by shuffles
    while (rows * 2 * per_row <= 32) rows *= 2;
    const int sub = lane / per_row;
    const RowItem<T, INTERLEAVED> it(lane - sub * per_row, p.rot);
    const bool active = sub < rows;
    const int heads = min(p.run_heads, p.hkv - head0);
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
    const unsigned leaders = __ballot_sync(kFullMask, page >= 0 && page != before);
    const int pairs = __popc(leaders) * heads;
    for (int pair = warp; pair < pairs; pair += warps) {
        const int head = head0 + pair % heads;
        const int l = __fns(leaders, 0, pair / heads + 1);
        const float scale = __ldg(p.summary_scale + head);
        const int64_t first = tile0 + l;
        const int64_t run_page = __shfl_sync(kFullMask, page, l);
        unsigned least[8], most[8];  // 16 channels as 16-bit pairs
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            least[i] = pack_s16(127, 127);
            most[i] = pack_s16(-127, -127);
        }
        int first_place = 0;
        const T* src = row_of<T>(p.k, head * p.k_sh);
        T* dst = row_of<T>(p.k_cache, cache_offset(p, run_page << p.page_shift, head));
        // 32 tokens at a time: the lanes read their slots and positions at once, and find where the run ends
        for (int64_t c0 = first;; c0 += 32) {
            int place = -1;
            int pos = 0;
            if (c0 + lane < p.T) {
                const int64_t s = append_slot(p, c0 + lane);
                if (s >= 0 && (s >> p.page_shift) == run_page) place = static_cast<int>(s & ((1 << p.page_shift) - 1));
                pos = static_cast<int>(append_position(p, c0 + lane));
            }
            const unsigned other = ~__ballot_sync(kFullMask, place >= 0);
            const int n = other ? __ffs(other) - 1 : 32;
            if (c0 == first) first_place = __shfl_sync(kFullMask, place, 0);
#pragma unroll 2
            for (int r0 = 0; r0 < n; r0 += rows) {
                const int r = r0 + sub;
                const int at = __shfl_sync(kFullMask, place, r & 31), ps = __shfl_sync(kFullMask, pos, r & 31);
                if (!active || r >= n) continue;
                const T* row = src + (c0 + r) * p.k_st;
                Raw8<T> lo, hi;
                lo.load(row + it.lo);
                hi.load(row + it.hi);
                float a[8], b[8];
                if (it.angle >= 0) {
                    float c[8], s[8];
                    load8(p.cos_t + static_cast<int64_t>(ps) * (p.rot / 2) + it.angle, c);
                    load8(p.sin_t + static_cast<int64_t>(ps) * (p.rot / 2) + it.angle, s);
                    lo.widen(a);
                    hi.widen(b);
                    it.turn(a, b, c, s);
                } else {
                    lo.widen(a);
                    hi.widen(b);
                }
                store8(dst + at * p.d + it.lo, a);
                store8(dst + at * p.d + it.hi, b);
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
            if (n < 32) break;
        }
        for (int step = rows / 2; step >= 1; step >>= 1) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                least[i] = __vmins2(least[i], __shfl_down_sync(kFullMask, least[i], step * per_row));
                most[i] = __vmaxs2(most[i], __shfl_down_sync(kFullMask, most[i], step * per_row));
            }
        }
        if (lane < per_row) {
            const bool anew = first_place == 0;
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
    // (the page blocks come first: theirs is the longer work)
    const int page_blocks = static_cast<int>(gridDim.x) - flat;
    if (SUMMARY && static_cast<int>(blockIdx.x) < page_blocks) {
        const int hb = (p.hkv + p.run_heads - 1) / p.run_heads;
        const int tile = static_cast<int>(blockIdx.x) / hb;
        append_pages<T, INTERLEAVED>(p, static_cast<int64_t>(tile) * p.run_tile, (static_cast<int>(blockIdx.x) - tile * hb) * p.run_heads);
        return;
    }
    append_flat<T, INTERLEAVED, SUMMARY>(p, static_cast<int>(blockIdx.x) - page_blocks);
}

}  // namespace wht
