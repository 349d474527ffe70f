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
// to one page for one head, keeps the channels' least and largest values in registers, folds the rows of the warp by
// shuffles and joins the page's stored summary once.  No atomics: a run has one owner.
//
// Measured: 16384 tokens, 16 heads of 64 and as many key heads, bf16: 38 us without summaries (5.4 TB/s), 54 with them, where a warp's walk
// of its run is a chain of waits; one token 6.1 us, 256 tokens of 32 heads 4.9 us, both the launch; 3001 fp32 tokens 22.5 us.
// Slower: a team of warps per run (57), the ranges in a second kernel that reads the stored keys back (55, and 16.5 instead of 7.5
// for 256 tokens).
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
    int page_blocks;          // thread blocks of the page part
};

template <typename T>
__device__ __forceinline__ T* row_of(void* base, int64_t off) { return static_cast<T*>(base) + off; }
template <typename T>
__device__ __forceinline__ const T* row_of(const void* base, int64_t off) { return static_cast<const T*>(base) + off; }

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

// WRITTEN: by ordinary loads, for kernels that may be resident while the kernel before writes what they read.
template <bool WRITTEN = false>
__device__ __forceinline__ int append_position(const AppendParams& p, int64_t t) {
    return p.rot == 0 ? 0 : WRITTEN ? p.positions[t] : __ldg(p.positions + t);
}
// The position held to the table: for tokens that use theirs (a dropped token's may be anything).
__device__ __forceinline__ int checked_position(const AppendParams& p, int pos) {
    if (p.rot != 0 && (pos < 0 || pos >= p.max_pos)) {
        attn_report(kAttnErrIndex);
        return pos < 0 ? 0 : static_cast<int>(p.max_pos - 1);
    }
    return pos;
}
// The token's slot, or -1 for padding and for slots outside the cache (reported).
template <bool WRITTEN = false>
__device__ __forceinline__ int64_t append_slot(const AppendParams& p, int64_t t) {
    const int64_t s = WRITTEN ? p.slots[t] : __ldg(reinterpret_cast<const long long*>(p.slots) + t);
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
    __device__ __forceinline__ void load_written(const T* p) {     // by ordinary loads
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
    }
    __device__ __forceinline__ void narrow(const float (&v)[8]) {  // rounded to the type
        if constexpr (sizeof(T) == 4) {
            w[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
            w[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
        } else {
            w[0] = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
        }
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
    int pos = turns ? append_position(p, t) : 0;  // (asked for beside the slot, checked once it is known to be used)
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
    pos = checked_position(p, pos);
    float c[8], s[8];
    load8(p.cos_t + static_cast<int64_t>(pos) * (p.rot / 2) + it.angle, c);
    load8(p.sin_t + static_cast<int64_t>(pos) * (p.rot / 2) + it.angle, s);
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

// ---- page part ----
// The least and the largest of 16 channels' stored values.  c() is monotonic, so they can be found on the values themselves, for bf16
// two to an instruction, and made whole numbers once per run (on whole numbers this part took 36 instructions per element and
// a third of the kernel's time).
template <typename T>
struct Range {
    static constexpr int N = 16;
    float least[N], most[N];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            least[i] = INFINITY;
            most[i] = -INFINITY;
        }
    }
    __device__ __forceinline__ void join(const Raw8<T>& lo, const Raw8<T>& hi) {
        float a[8], b[8];
        lo.widen(a);
        hi.widen(b);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            least[i] = fminf(least[i], a[i]);
            most[i] = fmaxf(most[i], a[i]);
            least[8 + i] = fminf(least[8 + i], b[i]);
            most[8 + i] = fmaxf(most[8 + i], b[i]);
        }
    }
    __device__ __forceinline__ void fold(int lanes) {  // with the lane `lanes` further on
#pragma unroll
        for (int i = 0; i < N; ++i) {
            least[i] = fminf(least[i], __shfl_down_sync(kFullMask, least[i], lanes));
            most[i] = fmaxf(most[i], __shfl_down_sync(kFullMask, most[i], lanes));
        }
    }
    __device__ __forceinline__ void get(int i, float& lo, float& hi) const {
        lo = least[i];
        hi = most[i];
    }
};
template <>
struct Range<__nv_bfloat16> {
    static constexpr int N = 8;  // pairs
    __nv_bfloat162 least[N], most[N];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            least[i] = __halves2bfloat162(__ushort_as_bfloat16(0x7f80), __ushort_as_bfloat16(0x7f80));
            most[i] = __halves2bfloat162(__ushort_as_bfloat16(0xff80), __ushort_as_bfloat16(0xff80));
        }
    }
    __device__ __forceinline__ void join(const Raw8<__nv_bfloat16>& lo, const Raw8<__nv_bfloat16>& hi) {
        const unsigned w[8] = {lo.w[0].x, lo.w[0].y, lo.w[0].z, lo.w[0].w, hi.w[0].x, hi.w[0].y, hi.w[0].z, hi.w[0].w};
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162*>(&w[i]);
            least[i] = __hmin2(least[i], x);
            most[i] = __hmax2(most[i], x);
        }
    }
    __device__ __forceinline__ void fold(int lanes) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            least[i] = __hmin2(least[i], __shfl_down_sync(kFullMask, least[i], lanes));
            most[i] = __hmax2(most[i], __shfl_down_sync(kFullMask, most[i], lanes));
        }
    }
    __device__ __forceinline__ void get(int i, float& lo, float& hi) const {
        lo = __bfloat162float(i & 1 ? least[i / 2].y : least[i / 2].x);
        hi = __bfloat162float(i & 1 ? most[i / 2].y : most[i / 2].x);
    }
};

// The warps of a block share the tile's runs and the block's heads.
template <typename T, bool INTERLEAVED>
__device__ __forceinline__ void append_pages(const AppendParams& p, int64_t tile0, int head0) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int per_row = p.d / 16;                      // 4, 6 or 8 lanes
    const int rows = per_row == 4 ? 8 : 4;             // rows of a warp's step: a power of two, so that they fold by shuffles
    const int lane_row = lane / per_row;
    const RowItem<T, INTERLEAVED> it(lane - lane_row * per_row, p.rot);
    const int heads = min(p.run_heads, p.hkv - head0);
    // which of the tile's tokens begin a run, and which runs go on after their first token
    int64_t page = -1, before = -1, after = -1;
    if (lane < p.run_tile && tile0 + lane < p.T) {
        const int64_t s = append_slot(p, tile0 + lane);
        const int64_t s1 = tile0 + lane > 0 ? append_slot(p, tile0 + lane - 1) : -1;
        const int64_t s2 = tile0 + lane + 1 < p.T ? append_slot(p, tile0 + lane + 1) : -1;
        if (s >= 0) page = s >> p.page_shift;
        if (s1 >= 0) before = s1 >> p.page_shift;
        if (s2 >= 0) after = s2 >> p.page_shift;
    }
    const unsigned leaders = __ballot_sync(kFullMask, page >= 0 && page != before);
    const unsigned longer = __ballot_sync(kFullMask, page >= 0 && page != before && page == after);
    // A warp's rows are tokens of one head, or, where every run is a single token (a decode step), heads of one token.
    const int across = longer ? 1 : rows;              // heads of a warp
    const int row_step = rows / across, sub = lane_row % row_step;
    const int groups = (heads + across - 1) / across;
    // (run, group) pairs are dealt to the warps in turn
    unsigned left = leaders;
    for (int group = warp; left; group += warps) {
        while (group >= groups && left) {
            group -= groups;
            left &= left - 1;
        }
        if (!left) break;
        const int l = __ffs(left) - 1;
        const int hb = group * across + lane_row / row_step;
        const bool mine = lane_row < rows && hb < heads;
        const int head = head0 + (mine ? hb : 0);
        const int64_t first = tile0 + l;
        const int64_t run_page = __shfl_sync(kFullMask, page, l);
        Range<T> range;
        range.clear();
        int first_place = 0;
        const T* src = row_of<T>(p.k, head * p.k_sh);
        T* dst = row_of<T>(p.k_cache, cache_offset(p, run_page << p.page_shift, head));
        // 32 tokens at a time: the lanes read their slots and positions at once, and find where the run ends
        for (int64_t c0 = first;; c0 += 32) {
            int place = -1;
            int pos = 0;
            if (c0 + lane < p.T) {
                const int64_t s = append_slot(p, c0 + lane);
                pos = append_position(p, c0 + lane);
                if (s >= 0 && (s >> p.page_shift) == run_page) {
                    place = static_cast<int>(s & ((1 << p.page_shift) - 1));
                    pos = checked_position(p, pos);
                }
            }
            const unsigned other = ~__ballot_sync(kFullMask, place >= 0);
            const int n = other ? __ffs(other) - 1 : 32;
            if (c0 == first) first_place = __shfl_sync(kFullMask, place, 0);
            const T* row = src + (c0 + sub) * p.k_st;
            const int64_t next_row = row_step * p.k_st;
#pragma unroll 2
            for (int r0 = 0; r0 < n; r0 += row_step, row += next_row) {
                const int r = r0 + sub;
                const int to = __shfl_sync(kFullMask, place, r & 31), ps = __shfl_sync(kFullMask, pos, r & 31);
                if (r >= n || !mine) continue;
                Raw8<T> lo, hi;
                lo.load(row + it.lo);
                hi.load(row + it.hi);
                if (it.angle >= 0) {
                    float c[8], s[8], a[8], b[8];
                    load8(p.cos_t + static_cast<int64_t>(ps) * (p.rot / 2) + it.angle, c);
                    load8(p.sin_t + static_cast<int64_t>(ps) * (p.rot / 2) + it.angle, s);
                    lo.widen(a);
                    hi.widen(b);
                    it.turn(a, b, c, s);
                    lo.narrow(a);
                    hi.narrow(b);
                }
                lo.store(dst + to * p.d + it.lo);
                hi.store(dst + to * p.d + it.hi);
                range.join(lo, hi);
            }
            if (n < 32) break;
        }
        for (int step = row_step / 2; step >= 1; step >>= 1) range.fold(step * per_row);
        if (!mine || sub != 0) continue;
        const bool anew = first_place == 0;
        const float scale = __ldg(p.summary_scale + head);
        int8_t* at = p.summary + ((run_page * p.hkv + head) * 2) * p.d;
        auto whole = [&](float x) { return max(-127, min(127, __float2int_rn(__fmul_rn(x, scale)))); };
#pragma unroll
        for (int w = 0; w < 4; ++w) {                  // four channels at a time
            unsigned wl = 0, wh = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float lo, hi;
                range.get(4 * w + i, lo, hi);
                const int a = whole(lo), b = whole(hi);  // (a negative scale turns them round)
                wl |= (static_cast<unsigned>(min(a, b)) & 0xffu) << (8 * i);
                wh |= (static_cast<unsigned>(max(a, b)) & 0xffu) << (8 * i);
            }
            unsigned* to = reinterpret_cast<unsigned*>(at + (w < 2 ? it.lo : it.hi) + 4 * (w & 1));
            if (!anew) {
                wl = __vmins4(wl, to[0]);
                wh = __vmaxs4(wh, to[p.d / 4]);
            }
            to[0] = wl;
            to[p.d / 4] = wh;
        }
    }
}

constexpr int kAppendThreads = 256;

template <typename T, bool INTERLEAVED, bool SUMMARY>
__global__ void __launch_bounds__(kAppendThreads, SUMMARY ? 3 : 4)
kv_append_kernel(const AppendParams p) {
    const int block = static_cast<int>(blockIdx.x);
    if constexpr (SUMMARY) {
        // Page blocks wait more than they move, flat blocks the other way round: spread evenly among each other they share the SMs.
        const long long pages = p.page_blocks, total = gridDim.x;
        const int before = static_cast<int>(block * pages / total), after = static_cast<int>((block + 1) * pages / total);
        if (after > before) {
            const int hb = (p.hkv + p.run_heads - 1) / p.run_heads, tile = before / hb;
            append_pages<T, INTERLEAVED>(p, static_cast<int64_t>(tile) * p.run_tile, (before - tile * hb) * p.run_heads);
            return;
        }
        append_flat<T, INTERLEAVED, true>(p, block - before);
    } else {
        append_flat<T, INTERLEAVED, false>(p, block);
    }
}

}  // namespace wht
