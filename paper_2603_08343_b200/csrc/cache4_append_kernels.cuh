// Append to the cache held in 4 bits: rotation, quantisation, write; and the rows that the cache holds, read back.
//
//     q' = rotation(q)     row k' = rotation(k), row v: lo, step and codes (cache4_common.cuh)
//
// A pass over memory: each element is read once; queries are written as they came, keys and values in a quarter of the bytes or less.
// Four lanes (D = 64) or eight own a row, 16 channels each as two groups of eight, so that a rotation's pairs never cross
// lanes, the row's extremes take two or three shuffles, and each group of eight channels is one word of codes.  A thread takes the same channels of
// several heads, all loads in flight at once; they share the angles.
#pragma once
#include "cache4_common.cuh"
#include "kv_append_kernels.cuh"

namespace wht {

struct Append4Params {
    AppendParams a;          // k_cache, v_cache, summary unused
    unsigned char* cache;
    int q_groups, kv_groups; // groups of heads that a thread takes
    int per_token;           // q_groups + 2 * kv_groups
};

// where the tile of a slot's row lies, and its place in the tile
__device__ __forceinline__ unsigned char* tile4_of(unsigned char* cache, int64_t slot, int head, int hkv, int page_shift, int d) {
    const int64_t page = slot >> page_shift;
    const int place = static_cast<int>(slot & ((1 << page_shift) - 1));
    return cache + (((page * hkv + head) << (page_shift - 4)) + (place >> 4)) * tile4_bytes(d);
}

template <typename T>
constexpr int kHeads4 = sizeof(T) == 4 ? 2 : 4;
constexpr int kAppend4Threads = 256;

template <typename T, bool INTERLEAVED, int D>
__global__ void __launch_bounds__(kAppend4Threads)
kv_append4_kernel(const Append4Params p) {
    constexpr int HB = kHeads4<T>;
    constexpr int LANES = D == 64 ? 4 : 8;             // of a row
    const AppendParams& a = p.a;
    const int64_t job = (static_cast<int64_t>(blockIdx.x) * kAppend4Threads + threadIdx.x) / LANES;
    const int item = threadIdx.x % LANES;
    const int64_t t = job / p.per_token;
    int group = static_cast<int>(job - t * p.per_token);
    const bool there = t < a.T && item < D / 16;       // (no lane leaves: rows fold by shuffles)
    const RowItem<T, INTERLEAVED> it(item < D / 16 ? item : 0, a.rot);
    const bool is_q = group < p.q_groups;
    bool turns = there && it.angle >= 0;
    int pos = turns ? append_position(a, t) : 0;
    int64_t slot = 0;
    const T* src = nullptr;
    int64_t step = 0;
    int h0 = 0, heads = 0;
    bool is_k = false;
    if (there) {
        if (is_q) {
            h0 = group * HB;
            heads = a.hq - h0;
            src = row_of<T>(a.q, t * a.q_st + h0 * a.q_sh);
            step = a.q_sh;
        } else {
            group -= p.q_groups;
            is_k = group < p.kv_groups;
            if (!is_k) group -= p.kv_groups;
            slot = append_slot(a, t);
            h0 = group * HB;
            heads = slot < 0 ? 0 : a.hkv - h0;
            src = is_k ? row_of<T>(a.k, t * a.k_st + h0 * a.k_sh) : row_of<T>(a.v, t * a.v_st + h0 * a.v_sh);
            step = is_k ? a.k_sh : a.v_sh;
            turns = turns && is_k && slot >= 0;
        }
    }
    Raw8<T> lo[HB], hi[HB];
#pragma unroll
    for (int i = 0; i < HB; ++i) {
        if (i < heads) {
            lo[i].load(src + i * step + it.lo);
            hi[i].load(src + i * step + it.hi);
        }
    }
    float c[8], s[8];
    if (turns) {
        pos = checked_position(a, pos);
        load8(a.cos_t + static_cast<int64_t>(pos) * (a.rot / 2) + it.angle, c);
        load8(a.sin_t + static_cast<int64_t>(pos) * (a.rot / 2) + it.angle, s);
    }
    const int place = static_cast<int>(slot & 15);
#pragma unroll
    for (int i = 0; i < HB; ++i) {
        float x[8], y[8];
        bool finite = true;
        float least = INFINITY, most = -INFINITY;
        const bool mine = i < heads;
        if (mine) {
            lo[i].widen(x);
            hi[i].widen(y);
            if (turns) it.turn(x, y, c, s);
            if (is_q) {
                T* dst = row_of<T>(a.q_out, (t * a.hq + h0 + i) * D);
                store8(dst + it.lo, x);
                store8(dst + it.hi, y);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    least = fminf(least, fminf(x[e], y[e]));
                    most = fmaxf(most, fmaxf(x[e], y[e]));
                    finite = finite && fabsf(x[e]) < INFINITY && fabsf(y[e]) < INFINITY;
                }
            }
        }
#pragma unroll
        for (int n = 1; n < LANES; n <<= 1) {
            least = fminf(least, __shfl_xor_sync(kFullMask, least, n));
            most = fmaxf(most, __shfl_xor_sync(kFullMask, most, n));
        }
        bool bad = !finite;
#pragma unroll
        for (int n = 1; n < LANES; n <<= 1) bad = bad || __shfl_xor_sync(kFullMask, static_cast<int>(bad), n);
        if (!mine || is_q) continue;
        const Hold4 hold(least, most, !bad);
        unsigned char* tile = tile4_of(p.cache, slot, h0 + i, a.hkv, a.page_shift, D);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int channel = half ? it.hi : it.lo, g = channel >> 5, u = (channel >> 2) & 7;  // u even
            unsigned w = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) w |= hold.code(half ? y[e] : x[e]) << (4 * e);
            if (is_k) {
                *reinterpret_cast<unsigned*>(tile + key4_at(D, place, g, u)) = w;
            } else {
                *reinterpret_cast<unsigned short*>(tile + value4_at(D, place, g, u)) = static_cast<unsigned short>(w);
                *reinterpret_cast<unsigned short*>(tile + value4_at(D, place, g, u + 1)) = static_cast<unsigned short>(w >> 16);
            }
        }
        if (item == 0) *reinterpret_cast<unsigned*>(tile + tile4_rows(D) + place * 8 + (is_k ? 0 : 4)) = hold.word();
    }
}

struct Read4Params {
    const unsigned char* cache;
    const int64_t* slots;
    void *k, *v;             // [n x Hkv x D]
    int64_t n, num_slots;
    int hkv, page_shift;
};

// A thread: eight channels of a key and of the value beside it.
template <typename T, int D>
__global__ void __launch_bounds__(256)
kv_read4_kernel(const Read4Params p) {
    constexpr int PER = D / 8;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t row = i / PER;                       // slot number * hkv + head
    const int octet = static_cast<int>(i - row * PER);
    const int64_t at = row / p.hkv;
    if (at >= p.n) return;
    const int head = static_cast<int>(row - at * p.hkv);
    int64_t slot = __ldg(reinterpret_cast<const long long*>(p.slots) + at);
    if (slot >= p.num_slots) {
        attn_report(kAttnErrIndex);
        slot = -1;
    }
    float k[8], v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) k[e] = v[e] = 0.0f;
    if (slot >= 0) {
        const unsigned char* tile = tile4_of(const_cast<unsigned char*>(p.cache), slot, head, p.hkv, p.page_shift, D);
        const int j = static_cast<int>(slot & 15), g = octet >> 2, u = 2 * (octet & 3);
        const unsigned kw = __ldg(reinterpret_cast<const unsigned*>(tile + key4_at(D, j, g, u)));
        const unsigned vw = __ldg(reinterpret_cast<const unsigned short*>(tile + value4_at(D, j, g, u))) |
                            static_cast<unsigned>(__ldg(reinterpret_cast<const unsigned short*>(tile + value4_at(D, j, g, u + 1)))) << 16;
        const uint2 w = __ldg(reinterpret_cast<const uint2*>(tile + tile4_rows(D) + j * 8));
        const float ks = step4_of(w.x), kl = lo4_of(w.x), vs = step4_of(w.y), vl = lo4_of(w.y);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            k[e] = __fadd_rn(kl, __fmul_rn(ks, static_cast<float>((kw >> (4 * e)) & 15u)));
            v[e] = __fadd_rn(vl, __fmul_rn(vs, static_cast<float>((vw >> (4 * e)) & 15u)));
        }
    }
    store8(static_cast<T*>(p.k) + row * D + octet * 8, k);
    store8(static_cast<T*>(p.v) + row * D + octet * 8, v);
}

}  // namespace wht
