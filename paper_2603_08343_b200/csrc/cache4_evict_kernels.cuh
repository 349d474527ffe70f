// Eviction: for each sequence and key head the first keys, the last ones and the heaviest of those between move into pages of their own.
//
// Two kernels.  The choice, a block per sequence and key head: the weights as ordered whole numbers; the spare-th largest found by
// three counts of 11, 11 and 10 bits; then one walk in the order of the keys that lists what stays (above the threshold, or at it while there is
// room: the lowest first).  Its bytes are 4 a key; what it costs is the chain of counts and scans, so that the weights are asked for all at once
// and the first 16384 stay in registers from there to the walk: 256 blocks over up to 16384 keys 29 us.
// (Copies of the counters for fewer collisions were slower.)
// The move, a warp per 16 kept keys: a tile is gathered from wherever its rows lie and written as one piece, 2 (D + 8) bytes a row
// moved, which memory bounds: 1048576 rows of 128 channels, keys and values, 57 us behind the choice, 5.0 TB/s.
#pragma once
#include "cache4_common.cuh"

namespace wht {

struct Evict4Params {
    AttnParams a;            // page_table, table_width, kv_lens, B, hkv, page_shift, num_pages
    unsigned char* cache;
    const int32_t* out_table;
    int out_width;           // pages
    const float* weights;    // [B x Hkv x table_width * page]
    float* weights_out;      // [B x Hkv x out_width * page]
    int32_t *lens_out, *kept;  // [B], [B x Hkv x budget]
    int budget, first, last;
};

constexpr int kEvictBins = 2048;

// Ordered whole numbers: NaN the least, -0 as 0.
__device__ __forceinline__ unsigned ordered4(float x) {
    if (x != x) return 0;
    const unsigned u = __float_as_uint(x == 0.0f ? 0.0f : x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sum over the threads before this one, and over all (two barriers).
template <int THREADS>
__device__ __forceinline__ unsigned block_scan4(unsigned x, unsigned* warp_sums, unsigned& all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned upto = x;
#pragma unroll
    for (int i = 1; i < 32; i <<= 1) {
        const unsigned y = __shfl_up_sync(kFullMask, upto, i);
        if (lane >= i) upto += y;
    }
    if (lane == 31) warp_sums[warp] = upto;
    __syncthreads();
    unsigned sums = lane < THREADS / 32 ? warp_sums[lane] : 0;       // (every warp adds them up: 32 at a time by shuffles)
#pragma unroll
    for (int i = 1; i < THREADS / 32; i <<= 1) {
        const unsigned y = __shfl_up_sync(kFullMask, sums, i);
        if (lane >= i) sums += y;
    }
    all = __shfl_sync(kFullMask, sums, THREADS / 32 - 1);
    unsigned before = __shfl_sync(kFullMask, sums, max(warp - 1, 0));
    if (warp == 0) before = 0;
    __syncthreads();
    return before + upto - x;
}

// Four neighbouring weights from key i on; what lies behind the n-th is 0.
__device__ __forceinline__ float4 weights4(const float* w, int i, int n) {
    if (i + 3 < n) return *reinterpret_cast<const float4*>(w + i);
    return make_float4(i < n ? w[i] : 0.0f, i + 1 < n ? w[i + 1] : 0.0f, i + 2 < n ? w[i + 2] : 0.0f, 0.0f);
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS)
kv_evict4_choose_kernel(const Evict4Params p) {
    constexpr int TILE = 4 * THREADS, HELD = 16384 / TILE;  // keys of a step, and steps whose weights stay in registers
    __shared__ unsigned bins[kEvictBins];
    __shared__ unsigned warp_sums[THREADS / 32];
    __shared__ unsigned found[2];                      // the bin that holds the threshold, and what is above it
    const AttnParams& a = p.a;
    const int tid = threadIdx.x;
    const int b = blockIdx.x / a.hkv, head = blockIdx.x % a.hkv;
    grid_dependency_wait();
    grid_launch_dependents();
    const int n = attn_length(a, b);
    const int keep = min(p.budget, n);
    const int from = min(p.first, n), to = max(from, n - p.last);    // the keys between, of which the heaviest `spare` stay
    const int spare = keep - (n - (to - from));
    const int64_t width = static_cast<int64_t>(a.table_width) << a.page_shift;
    const float* w = p.weights + (static_cast<int64_t>(b) * a.hkv + head) * width;
    const int64_t out_keys = static_cast<int64_t>(p.out_width) << a.page_shift;
    float* w_out = p.weights_out + (static_cast<int64_t>(b) * a.hkv + head) * out_keys;
    int32_t* kept = p.kept + (static_cast<int64_t>(b) * a.hkv + head) * p.budget;
    if (head == 0 && tid == 0) p.lens_out[b] = keep;
    float4 held[HELD];
#pragma unroll
    for (int r = 0; r < HELD; ++r) held[r] = weights4(w, r * TILE + 4 * tid, n);
    // f(first key, four weights) for every step
    auto walk = [&](auto f) {
#pragma unroll
        for (int r = 0; r < HELD; ++r)
            if (r * TILE < n) f(r * TILE + 4 * tid, held[r]);
        for (int base = HELD * TILE; base < n; base += TILE) f(base + 4 * tid, weights4(w, base + 4 * tid, n));
    };

    const bool chosen = spare < to - from;             // (otherwise all stay)
    unsigned threshold = 0, ties = 0;
    if (chosen && spare > 0) {
        unsigned known = 0, mask = 0, want = static_cast<unsigned>(spare);
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, count = pass == 2 ? 1024 : 2048;
            for (int i = tid; i < count; i += THREADS) bins[i] = 0;
            __syncthreads();
            walk([&](int i, const float4& v) {
                const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const unsigned key = ordered4(x[e]);
                    if (i + e >= from && i + e < to && (key & mask) == known) atomicAdd(&bins[(key >> shift) & (count - 1)], 1u);
                }
            });
            __syncthreads();
            // from the top: each thread a few bins, the highest first
            const int per = (count + THREADS - 1) / THREADS, top = count - 1 - tid * per;
            unsigned mine = 0;
            for (int i = 0; i < per; ++i) mine += bins[top - i];
            unsigned all;
            unsigned above = block_scan4<THREADS>(mine, warp_sums, all);
            if (above < want && above + mine >= want) {
                for (int i = 0; i < per; ++i) {
                    const unsigned c = bins[top - i];
                    if (above + c >= want) {
                        found[0] = static_cast<unsigned>(top - i);
                        found[1] = above;
                        break;
                    }
                    above += c;
                }
            }
            __syncthreads();
            known |= found[0] << shift;
            mask |= static_cast<unsigned>(count - 1) << shift;
            want -= found[1];
        }
        threshold = known;
        ties = want;                                   // of the keys at the threshold, this many stay
    }

    unsigned written = 0, tied = 0;
    walk([&](int i0, const float4& v) {
        const float x[4] = {v.x, v.y, v.z, v.w};
        unsigned above = 0, at = 0;                    // bits: stays in any case; at the threshold
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = i0 + e;
            if (i >= n) continue;
            if (!chosen || i < from || i >= to) {
                above |= 1u << e;
            } else if (spare > 0) {
                const unsigned key = ordered4(x[e]);
                if (key > threshold) above |= 1u << e;
                else if (key == threshold) at |= 1u << e;
            }
        }
        unsigned all;
        const unsigned before = block_scan4<THREADS>(static_cast<unsigned>(__popc(above)) | static_cast<unsigned>(__popc(at)) << 16, warp_sums, all);
        unsigned rank = tied + (before >> 16);         // of this thread's first key at the threshold
        unsigned place = written + (before & 0xffffu) + (min(rank, ties) - min(tied, ties));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            bool stays = above >> e & 1u;
            if (at >> e & 1u) stays = rank++ < ties;
            if (!stays) continue;
            kept[place] = i0 + e;
            w_out[place] = x[e];
            ++place;
        }
        written += (all & 0xffffu) + (min(tied + (all >> 16), ties) - min(tied, ties));
        tied += all >> 16;
    });
    for (int64_t i = keep + tid; i < p.budget; i += THREADS) kept[i] = -1;
    for (int64_t i = keep + tid; i < out_keys; i += THREADS) w_out[i] = 0.0f;
}

// Where 16-byte piece `piece` of row j lies in a tile: the codes of the key, then those of the value.
template <int D>
__device__ __forceinline__ int piece4_at(int j, int piece) {
    constexpr int KEY = D / 32;                        // pieces of a key's codes, and of a value's
    if (piece < KEY) return j * (D / 2) + piece * 16;
    const int u = piece - KEY;
    if constexpr (D == 128) return 8 * D + value4_place(j) * 64 + ((u * 16) ^ ((j & 4) << 3));
    return u < 2 ? 8 * D + value4_place(j) * 32 + u * 16 : 8 * D + 512 + value4_place(j) * 16;
}

constexpr int kMove4Warps = 4;

template <int D>
__global__ void __launch_bounds__(32 * kMove4Warps)
kv_evict4_move_kernel(const Evict4Params p) {
    constexpr int PIECES = D / 16, MINE = PIECES / 2;  // of a row, and of a lane: all of them in flight at once
    const AttnParams& a = p.a;
    const int lane = threadIdx.x & 31;
    const int tiles = (p.budget + kTileKeys - 1) / kTileKeys;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * kMove4Warps + (threadIdx.x >> 5);
    grid_dependency_wait();
    grid_launch_dependents();
    const int64_t bh = unit / tiles;
    const int tile = static_cast<int>(unit - bh * tiles);
    const int b = static_cast<int>(bh / a.hkv), head = static_cast<int>(bh - static_cast<int64_t>(b) * a.hkv);
    if (b >= a.B) return;
    const int shift = a.page_shift - 4, in_page = (1 << shift) - 1;
    // lanes 0 .. 15: where each row comes from
    int64_t from = -1;                                 // tile of the cache * 16 + row
    const int at = tile * kTileKeys + lane;
    if (lane < kTileKeys && at < p.budget) {
        const int key = __ldcg(p.kept + bh * p.budget + at);
        if (key >= 0) {
            const int t = key >> 4;
            int pg = a.page_table[static_cast<int64_t>(b) * a.table_width + (t >> shift)];
            if (pg < 0 || pg >= a.num_pages) {
                attn_report(kAttnErrIndex);
                pg = 0;
            }
            from = ((((static_cast<int64_t>(pg) * a.hkv + head) << shift) + (t & in_page)) << 4) + (key & 15);
        }
    }
    if (!__any_sync(kFullMask, from >= 0)) return;
    const int out = p.out_table[static_cast<int64_t>(b) * p.out_width + (tile >> shift)];
    if (out < 0 || out >= a.num_pages) {
        attn_report(kAttnErrIndex);
        return;
    }
    unsigned char* to = p.cache + (((static_cast<int64_t>(out) * a.hkv + head) << shift) + (tile & in_page)) * tile4_bytes(D);
    uint4 got[MINE];
    uint2 row = make_uint2(0, 0);
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        const int n = i * 32 + lane, j = n / PIECES;
        const int64_t src = __shfl_sync(kFullMask, from, j);
        got[i] = make_uint4(0, 0, 0, 0);
        if (src >= 0) got[i] = *reinterpret_cast<const uint4*>(p.cache + (src >> 4) * tile4_bytes(D) + piece4_at<D>(static_cast<int>(src & 15), n - j * PIECES));
    }
    if (from >= 0) row = *reinterpret_cast<const uint2*>(p.cache + (from >> 4) * tile4_bytes(D) + tile4_rows(D) + (from & 15) * 8);
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        const int n = i * 32 + lane, j = n / PIECES;
        if (__shfl_sync(kFullMask, from, j) >= 0) *reinterpret_cast<uint4*>(to + piece4_at<D>(j, n - j * PIECES)) = got[i];
    }
    if (from >= 0) *reinterpret_cast<uint2*>(to + tile4_rows(D) + lane * 8) = row;
}

}  // namespace wht
