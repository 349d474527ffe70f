// Selection of pages by a whole-number score.
//
//     q8 = rint(q * (127 * (1 / max|q|)))      score(page) = sum_channels up . most(page) + down . least(page)
//     up = sum over the heads of the positive q8, down = of the negative: the heads of a key head add up first,
// so a page costs two products of length D whatever the group.  Sums of whole numbers have no order: the scores, and
// so the selection, are the same for every batch shape and split.
//
// attn_select_kernel does both for a block's queries where their scores fit shared memory and there are blocks enough; else
// attn_score_kernel: one thread per page, its summary (2 D bytes) in registers, the queries' sums in shared memory as
// base-64 digits (two signed bytes each), four dp4a chains per query.  A block takes up to TQ tokens of a
// sequence, so that prompts read each summary once per TQ queries; single tokens stream summaries at the rate of memory.
// attn_pick_kernel: one block per query and key head.  The threshold is built bit by bit from the top (the scores less
// their minimum, so only as many steps as their range has bits), each step a count over the block; then one ordered pass
// writes the pages above it and, lowest first, as many that equal it as are still wanted.
//
// Measured (D = 128, pages of 64): 64 sequences of up to 512 pages, 8 key heads, 24 us for 50 MB of summaries, a chain of short
// phases (queries, page numbers, eight rounds of summaries, the pick); one sequence of 64 pages 5.4 us; 2048 prompt tokens of 193 pages, 4 key
// heads, 28 us.
#pragma once
#include "attn_kernels.cuh"

namespace wht {

struct SelectParams {
    AttnParams a;           // queries, tables, lengths
    const int8_t* summary;  // [num_pages x Hkv x 2 x D]
    int32_t* scores;        // [T x Hkv x stride], for the two kernels
    int32_t* pages;         // [T x Hkv x select]
    int stride;             // candidates a row has room for (the table's width)
    int token_tiles;        // token tiles per sequence
    int chunks;             // blocks of pages
};

constexpr int kScoreThreads = 128;

template <typename T>
__device__ __forceinline__ float load_f32(const T* p) {
    if constexpr (std::is_same<T, float>::value) return __ldg(p);
    else return __bfloat162float(*p);
}

template <typename T, int D, int TQ>
__global__ void __launch_bounds__(kScoreThreads)
attn_score_kernel(const SelectParams sp) {
    __shared__ __align__(16) int8_t digits[TQ][4][D];
    const AttnParams& p = sp.a;
    grid_launch_dependents();
    int64_t b = blockIdx.x;
    const int chunk = static_cast<int>(b % sp.chunks);
    b /= sp.chunks;
    const int head = static_cast<int>(b % p.hkv);
    b /= p.hkv;
    const int tile = static_cast<int>(b % sp.token_tiles), seq = static_cast<int>(b / sp.token_tiles);
    int64_t first;
    int count;
    attn_tokens(p, seq, first, count);
    const int n = min(TQ, count - tile * TQ);
    if (n <= 0) return;
    const int64_t t0 = first + tile * TQ;
    // own page of each token: the pages before it are candidates
    const int64_t place0 = static_cast<int64_t>(attn_length(p, seq)) - count + tile * TQ;
    const int64_t last = place0 + n - 1;
    const int most = last < 0 ? 0 : static_cast<int>(last >> p.page_shift);
    if (most <= p.select - 1 || chunk * kScoreThreads >= most) return;  // all are taken / no page of this chunk is before a token

    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int C = D / 32;
    for (int i = warp; i < n; i += kScoreThreads / 32) {
        const T* q = static_cast<const T*>(p.q) + (t0 + i) * p.q_st + static_cast<int64_t>(head) * p.group * p.q_sh;
        float top = 0.0f;
        for (int g = 0; g < p.group; ++g)
#pragma unroll
            for (int c = 0; c < C; ++c) top = fmaxf(top, fabsf(load_f32(q + g * p.q_sh + lane + 32 * c)));
#pragma unroll
        for (int k = 16; k; k >>= 1) top = fmaxf(top, __shfl_xor_sync(kFullMask, top, k));
        const float r = top > 1e-30f ? __fmul_rn(__frcp_rn(top), 127.0f) : 0.0f;
        int up[C], down[C];
#pragma unroll
        for (int c = 0; c < C; ++c) up[c] = down[c] = 0;
        for (int g = 0; g < p.group; ++g)
#pragma unroll
            for (int c = 0; c < C; ++c) {
                // (an infinite or NaN query gives no number: 0)
                const int v = max(-127, min(127, __float2int_rn(__fmul_rn(load_f32(q + g * p.q_sh + lane + 32 * c), r))));
                up[c] += max(v, 0);
                down[c] += min(v, 0);
            }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int uh = (up[c] + 32) >> 6, dh = (down[c] + 32) >> 6;
            digits[i][0][lane + 32 * c] = static_cast<int8_t>(uh);
            digits[i][1][lane + 32 * c] = static_cast<int8_t>(up[c] - uh * 64);
            digits[i][2][lane + 32 * c] = static_cast<int8_t>(dh);
            digits[i][3][lane + 32 * c] = static_cast<int8_t>(down[c] - dh * 64);
        }
    }
    __syncthreads();
    const int page = chunk * kScoreThreads + threadIdx.x;
    if (page >= most) return;
    int phys = __ldg(p.page_table + static_cast<int64_t>(seq) * p.table_width + page);
    if (phys < 0 || phys >= p.num_pages) {
        attn_report(kAttnErrIndex);
        phys = 0;
    }
    constexpr int V = D / 16;
    uint4 least[V], largest[V];
    const uint4* row = reinterpret_cast<const uint4*>(sp.summary + (static_cast<int64_t>(phys) * p.hkv + head) * 2 * D);
#pragma unroll
    for (int v = 0; v < V; ++v) least[v] = __ldg(row + v);
#pragma unroll
    for (int v = 0; v < V; ++v) largest[v] = __ldg(row + V + v);
    for (int i = 0; i < n; ++i) {
        const int64_t mine = (place0 + i) >> p.page_shift;
        if (place0 + i < 0 || page >= mine) continue;
        int hi = 0, lo = 0;
        auto dot = [](const uint4& x, const uint4& y, int acc) {
            acc = __dp4a(static_cast<int>(x.x), static_cast<int>(y.x), acc);
            acc = __dp4a(static_cast<int>(x.y), static_cast<int>(y.y), acc);
            acc = __dp4a(static_cast<int>(x.z), static_cast<int>(y.z), acc);
            return __dp4a(static_cast<int>(x.w), static_cast<int>(y.w), acc);
        };
#pragma unroll
        for (int v = 0; v < V; ++v) {
            hi = dot(*reinterpret_cast<const uint4*>(&digits[i][0][v * 16]), largest[v], hi);
            lo = dot(*reinterpret_cast<const uint4*>(&digits[i][1][v * 16]), largest[v], lo);
            hi = dot(*reinterpret_cast<const uint4*>(&digits[i][2][v * 16]), least[v], hi);
            lo = dot(*reinterpret_cast<const uint4*>(&digits[i][3][v * 16]), least[v], lo);
        }
        sp.scores[((t0 + i) * p.hkv + head) * sp.stride + page] = hi * 64 + lo;
    }
}

// ---- scoring and picking in one kernel, where the candidates of a block's queries fit shared memory ----
constexpr int kSelectThreads = 256;

// The k best of n scores (n > k), ties to the lowest, ascending; then page n itself.  By one warp, scores in shared memory;
// R: rounds of 32 that are held in registers (n <= 32 R), 0: read again in every step.
template <int R>
__device__ __forceinline__ void warp_pick(const int32_t* score, int n, int k, int32_t* out) {
    const int lane = threadIdx.x & 31;
    int least = 0x7fffffff, most = -0x7fffffff - 1;
    for (int i = lane; i < n; i += 32) {
        least = min(least, score[i]);
        most = max(most, score[i]);
    }
    least = __reduce_min_sync(kFullMask, least);
    most = __reduce_max_sync(kFullMask, most);
    // scores counted from the least one, plus 1: what is no candidate is 0 and reaches no threshold
    uint32_t held[R > 0 ? R : 1];
#pragma unroll
    for (int j = 0; j < R; ++j) held[j] = lane + 32 * j < n ? static_cast<uint32_t>(score[lane + 32 * j]) - static_cast<uint32_t>(least) + 1u : 0u;
    auto value = [&](int i) { return i < n ? static_cast<uint32_t>(score[i]) - static_cast<uint32_t>(least) + 1u : 0u; };
    auto reached = [&](uint32_t want) {  // how many scores reach it
        int c = 0;
        if constexpr (R > 0) {
#pragma unroll
            for (int j = 0; j < R; ++j) c += held[j] >= want;
        } else {
            for (int i = lane; i < n; i += 32) c += value(i) >= want;
        }
        return __reduce_add_sync(kFullMask, c);
    };
    // the largest threshold that at least k scores reach, bit by bit
    uint32_t cut = 0;
    bool exact = false;
    for (int bit = 31 - __clz(static_cast<int>(static_cast<uint32_t>(most) - static_cast<uint32_t>(least) + 1u)); bit >= 0 && !exact; --bit) {
        const int c = reached(cut | (1u << bit));
        if (c >= k) {
            cut |= 1u << bit;
            exact = c == k;
        }
    }
    int wanted = exact ? 0 : k - reached(cut + 1u);  // of those that equal the threshold
    const unsigned before = (1u << lane) - 1u;
    int written = 0;
    auto round = [&](int i0, uint32_t v) {
        const bool above = exact ? v >= cut : v > cut, equal = !exact && v == cut;
        const unsigned equals = __ballot_sync(kFullMask, equal);
        const bool take = above || (equal && __popc(equals & before) < wanted);
        wanted = max(0, wanted - __popc(equals));
        const unsigned taken = __ballot_sync(kFullMask, take);
        if (take) out[written + __popc(taken & before)] = i0 + lane;
        written += __popc(taken);
    };
    if constexpr (R > 0) {
#pragma unroll
        for (int j = 0; j < R; ++j)
            if (32 * j < n) round(32 * j, held[j]);
    } else {
        for (int i0 = 0; i0 < n; i0 += 32) round(i0, value(i0 + lane));
    }
    if (lane == 0) out[k] = n;
}

__device__ __forceinline__ void mma_s8_16832(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// TQ = 1: single tokens, four threads per page and dp4a, the summaries on their way while the query is made whole numbers.
// TQ = 16: prompts, 16 queries as the rows of an int8 matrix product with 8 pages, digits and summaries as they lie in memory
// (the contraction index is permuted so that a lane's 16 bytes of a page are its operands of two instructions).
template <typename T, int D, int TQ>
__global__ void __launch_bounds__(kSelectThreads, TQ > 1 ? 2 : 4)
attn_select_kernel(const SelectParams sp) {
    constexpr int ROW = 2 * D + (TQ > 1 ? 64 : 0);           // bytes of a query's digits (most | least), padded against bank conflicts
    __shared__ __align__(16) int8_t digits[2][TQ][ROW];      // [high, low]
    extern __shared__ int32_t scores[];                      // [TQ][stride]
    const AttnParams& p = sp.a;
    grid_launch_dependents();
    int64_t b = blockIdx.x;
    const int head = static_cast<int>(b % p.hkv);
    b /= p.hkv;
    const int tile = static_cast<int>(b % sp.token_tiles), seq = static_cast<int>(b / sp.token_tiles);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int32_t* table = p.page_table + static_cast<int64_t>(seq) * p.table_width;
    int64_t first;
    int count;
    attn_tokens(p, seq, first, count);
    const int n = min(TQ, count - tile * TQ);
    if (p.q_start != nullptr && seq == 0 && tile == 0) {  // tokens of no sequence read no page (the attention reports them)
        int64_t from, to;
        if (!attn_covered(p, from, to)) {
            for (int64_t t = 0; t < p.T; ++t) {
                if (t == from) t = to;
                if (t >= p.T) break;
                for (int e = tid; e < p.select; e += kSelectThreads) sp.pages[(t * p.hkv + head) * p.select + e] = -1;
            }
        }
    }
    if (n <= 0) return;
    const int64_t t0 = first + tile * TQ;
    const int64_t place0 = static_cast<int64_t>(attn_length(p, seq)) - count + tile * TQ;
    const int64_t last = place0 + n - 1;
    const int most = last < 0 ? 0 : static_cast<int>(last >> p.page_shift);  // candidates of the last token
    const int k = p.select - 1;
    auto physical = [&](int page) {
        int phys = __ldg(table + page);
        if (phys < 0 || phys >= p.num_pages) {
            attn_report(kAttnErrIndex);
            phys = 0;
        }
        return sp.summary + (static_cast<int64_t>(phys) * p.hkv + head) * 2 * D;
    };
    const bool scoring = most > k && k > 0;
    // Single tokens: four threads per page, a quarter of its summary each, two pages of a thread on their way at a time and
    // the table's entries a round ahead of that.
    constexpr int V = 2 * D / 64, PAGES = kSelectThreads / 4;
    uint4 part[2][V];
    const int8_t* next_row = nullptr;
    auto locate = [&](int page) {
        if (page < most) next_row = physical(page) + (tid & 3) * (D / 2);
    };
    auto fetch = [&](int page, uint4 (&to)[V]) {
        if (page < most) {
#pragma unroll
            for (int v = 0; v < V; ++v) to[v] = __ldg(reinterpret_cast<const uint4*>(next_row) + v);
        }
    };
    if (TQ == 1 && scoring) {  // started before the query is made whole numbers
        locate(tid >> 2);
        fetch(tid >> 2, part[0]);
        locate(PAGES + (tid >> 2));
    }
    if (scoring) {
        constexpr int C = D / 32;
        for (int i = warp; i < TQ; i += kSelectThreads / 32) {
            if (i >= n) {
                for (int c = lane; c < ROW; c += 32) digits[0][i][c] = digits[1][i][c] = 0;
                continue;
            }
            const T* q = static_cast<const T*>(p.q) + (t0 + i) * p.q_st + static_cast<int64_t>(head) * p.group * p.q_sh;
            // eight heads' values at a time, all loads in flight; groups of up to eight are read once
            constexpr int GB = 8;
            float x[GB][C];
            auto heads = [&](int g0) {
#pragma unroll
                for (int g = 0; g < GB; ++g)
#pragma unroll
                    for (int c = 0; c < C; ++c) x[g][c] = g0 + g < p.group ? load_f32(q + (g0 + g) * p.q_sh + lane + 32 * c) : 0.0f;
            };
            float top = 0.0f;
            for (int g0 = 0; g0 < p.group; g0 += GB) {
                heads(g0);
#pragma unroll
                for (int g = 0; g < GB; ++g)
#pragma unroll
                    for (int c = 0; c < C; ++c) top = fmaxf(top, fabsf(x[g][c]));
            }
#pragma unroll
            for (int s = 16; s; s >>= 1) top = fmaxf(top, __shfl_xor_sync(kFullMask, top, s));
            const float r = top > 1e-30f ? __fmul_rn(__frcp_rn(top), 127.0f) : 0.0f;
            int up[C], down[C];
#pragma unroll
            for (int c = 0; c < C; ++c) up[c] = down[c] = 0;
            for (int g0 = 0; g0 < p.group; g0 += GB) {
                if (p.group > GB) heads(g0);
#pragma unroll
                for (int g = 0; g < GB; ++g)
#pragma unroll
                    for (int c = 0; c < C; ++c) {
                        // (an infinite or NaN query gives no number: 0)
                        const int v = max(-127, min(127, __float2int_rn(__fmul_rn(x[g][c], r))));
                        up[c] += max(v, 0);
                        down[c] += min(v, 0);
                    }
            }
#pragma unroll
            for (int c = 0; c < C; ++c) {
                // base-64 digits; a summary is least | most, so that the digits of `down` come first
                const int at = lane + 32 * c, uh = (up[c] + 32) >> 6, dh = (down[c] + 32) >> 6;
                digits[0][i][at] = static_cast<int8_t>(dh);
                digits[1][i][at] = static_cast<int8_t>(down[c] - dh * 64);
                digits[0][i][D + at] = static_cast<int8_t>(uh);
                digits[1][i][D + at] = static_cast<int8_t>(up[c] - uh * 64);
            }
        }
        __syncthreads();
        if constexpr (TQ == 1) {
            const int8_t* high = &digits[0][0][(tid & 3) * (D / 2)];
            const int8_t* low = &digits[1][0][(tid & 3) * (D / 2)];
            auto dot = [](const uint4& x, const uint4& y, int acc) {
                acc = __dp4a(static_cast<int>(x.x), static_cast<int>(y.x), acc);
                acc = __dp4a(static_cast<int>(x.y), static_cast<int>(y.y), acc);
                acc = __dp4a(static_cast<int>(x.z), static_cast<int>(y.z), acc);
                return __dp4a(static_cast<int>(x.w), static_cast<int>(y.w), acc);
            };
            auto round = [&](int p0, const uint4 (&now)[V], uint4 (&next)[V]) {  // (all threads: a page's four exchange their sums)
                const int page = p0 + (tid >> 2);
                fetch(page + PAGES, next);
                locate(page + 2 * PAGES);
                int hi = 0, lo = 0;
                if (page < most) {
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        hi = dot(*reinterpret_cast<const uint4*>(high + v * 16), now[v], hi);
                        lo = dot(*reinterpret_cast<const uint4*>(low + v * 16), now[v], lo);
                    }
                }
                int sum = hi * 64 + lo;
                sum += __shfl_xor_sync(kFullMask, sum, 1);
                sum += __shfl_xor_sync(kFullMask, sum, 2);
                if (page < most && !(tid & 3)) scores[page] = sum;
            };
            for (int p0 = 0; p0 < most; p0 += 2 * PAGES) {
                round(p0, part[0], part[1]);
                if (p0 + PAGES < most) round(p0 + PAGES, part[1], part[0]);
            }
        } else {
            const int r4 = lane >> 2, c4 = lane & 3;
            constexpr int NG = 2;                            // 8-page groups at a time
            for (int p0 = warp * 8 * NG; p0 < most; p0 += kSelectThreads / 32 * 8 * NG) {
                const int8_t* row[NG];
#pragma unroll
                for (int g = 0; g < NG; ++g) row[g] = physical(min(p0 + 8 * g + r4, most - 1)) + 16 * c4;
                int hi[NG][4], lo[NG][4];
#pragma unroll
                for (int g = 0; g < NG; ++g)
#pragma unroll
                    for (int i = 0; i < 4; ++i) hi[g][i] = lo[g][i] = 0;
                uint4 s[2 * D / 64][NG];
#pragma unroll
                for (int x = 0; x < 2 * D / 64; ++x)
#pragma unroll
                    for (int g = 0; g < NG; ++g) s[x][g] = __ldg(reinterpret_cast<const uint4*>(row[g] + 64 * x));
#pragma unroll
                for (int x = 0; x < 2 * D / 64; ++x) {
                    const uint4 h0 = *reinterpret_cast<const uint4*>(&digits[0][r4][64 * x + 16 * c4]);
                    const uint4 h1 = *reinterpret_cast<const uint4*>(&digits[0][r4 + 8][64 * x + 16 * c4]);
                    const uint4 l0 = *reinterpret_cast<const uint4*>(&digits[1][r4][64 * x + 16 * c4]);
                    const uint4 l1 = *reinterpret_cast<const uint4*>(&digits[1][r4 + 8][64 * x + 16 * c4]);
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        mma_s8_16832(hi[g], h0.x, h1.x, h0.y, h1.y, s[x][g].x, s[x][g].y);
                        mma_s8_16832(hi[g], h0.z, h1.z, h0.w, h1.w, s[x][g].z, s[x][g].w);
                        mma_s8_16832(lo[g], l0.x, l1.x, l0.y, l1.y, s[x][g].x, s[x][g].y);
                        mma_s8_16832(lo[g], l0.z, l1.z, l0.w, l1.w, s[x][g].z, s[x][g].w);
                    }
                }
#pragma unroll
                for (int g = 0; g < NG; ++g)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int page = p0 + 8 * g + 2 * c4 + (i & 1);
                        if (page < most) scores[(r4 + 8 * (i >> 1)) * sp.stride + page] = hi[g][i] * 64 + lo[g][i];
                    }
            }
        }
        __syncthreads();
    }
    for (int i = warp; i < n; i += kSelectThreads / 32) {
        const int64_t place = place0 + i;
        const int own = place < 0 ? -1 : static_cast<int>(place >> p.page_shift);
        int32_t* out = sp.pages + ((t0 + i) * p.hkv + head) * p.select;
        if (own <= k) {
            for (int e = lane; e < p.select; e += 32) out[e] = e <= own ? e : -1;
        } else if (k == 0) {
            if (lane == 0) out[0] = own;
        } else {
            if (own <= 8 * 32) warp_pick<8>(scores + i * sp.stride, own, k, out);
            else if (TQ == 1 && own <= 16 * 32) warp_pick<16>(scores + i * sp.stride, own, k, out);
            else warp_pick<0>(scores + i * sp.stride, own, k, out);
        }
    }
}

// Sum of `v` over the block, the same for every thread.  `slot` alternates between calls.
template <int THREADS>
__device__ __forceinline__ int block_sum(int v, int* buf) {
    const int w = __reduce_add_sync(kFullMask, v);
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = w;
    __syncthreads();
    int s = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) s += buf[i];
    return s;
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS)
attn_pick_kernel(const SelectParams sp) {
    extern __shared__ uint32_t keys[];
    __shared__ int buf[3][2 * (THREADS / 32)];
    const AttnParams& p = sp.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t row = blockIdx.x;  // token * Hkv + head
    const int64_t t = row / p.hkv;
    int32_t* out = sp.pages + row * p.select;
    grid_dependency_wait();
    grid_launch_dependents();
    const int seq = attn_sequence_of(p, t);
    int64_t first;
    int count;
    attn_tokens(p, seq, first, count);
    const int64_t place = attn_place(p, seq, t, first, count);
    const int n = place < 0 ? -1 : static_cast<int>(place >> p.page_shift);  // candidates, and the token's own page
    const int k = p.select - 1;
    if (n <= k) {
        for (int i = tid; i < p.select; i += THREADS) out[i] = i <= n ? i : -1;
        return;
    }
    if (k == 0) {
        if (tid == 0) out[0] = n;
        return;
    }
    const int32_t* src = sp.scores + row * sp.stride;
    uint32_t least = 0xffffffffu, most = 0;
    for (int i = tid; i < n; i += THREADS) {
        const uint32_t v = static_cast<uint32_t>(src[i]) ^ 0x80000000u;
        keys[i] = v;
        least = min(least, v);
        most = max(most, v);
    }
    least = __reduce_min_sync(kFullMask, least);
    most = __reduce_max_sync(kFullMask, most);
    if (lane == 0) {
        buf[0][warp] = static_cast<int>(least);
        buf[0][THREADS / 32 + warp] = static_cast<int>(most);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) {
        least = min(least, static_cast<uint32_t>(buf[0][i]));
        most = max(most, static_cast<uint32_t>(buf[0][THREADS / 32 + i]));
    }
    // the largest threshold that at least k keys reach
    uint32_t cut = 0;
    bool exact = false;  // exactly k keys reach it
    for (int bit = 31 - __clz(static_cast<int>((most - least) | 1u)), turn = 1; bit >= 0 && !exact; --bit) {
        const uint32_t want = cut | (1u << bit);
        int c = 0;
        for (int i = tid; i < n; i += THREADS) c += keys[i] - least >= want;
        c = block_sum<THREADS>(c, buf[turn]);
        turn = turn == 2 ? 0 : turn + 1;
        if (c >= k) {
            cut |= 1u << bit;
            exact = c == k;
        }
    }
    // ordered pass: thread i has the i-th run of consecutive pages
    const int per = (n + THREADS - 1) / THREADS;
    const int i0 = min(n, tid * per), i1 = min(n, i0 + per);
    int above = 0, equal = 0;
    for (int i = i0; i < i1; ++i) {
        const uint32_t v = keys[i] - least;
        above += exact ? v >= cut : v > cut;
        equal += !exact && v == cut;
    }
    int sa = above, se = equal;  // inclusive scans
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
        const int xa = __shfl_up_sync(kFullMask, sa, s), xe = __shfl_up_sync(kFullMask, se, s);
        if (lane >= s) {
            sa += xa;
            se += xe;
        }
    }
    __syncthreads();
    if (lane == 31) {
        buf[0][warp] = sa;
        buf[0][THREADS / 32 + warp] = se;
    }
    __syncthreads();
    int total = 0, before_a = 0, before_e = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) {
        if (i < warp) {
            before_a += buf[0][i];
            before_e += buf[0][THREADS / 32 + i];
        }
        total += buf[0][i];
    }
    const int wanted = k - total;  // of those that equal the threshold
    int a = before_a + sa - above, e = before_e + se - equal;
    for (int i = i0; i < i1; ++i) {
        const uint32_t v = keys[i] - least;
        const bool is_above = exact ? v >= cut : v > cut, is_equal = !exact && v == cut;
        if (is_above || (is_equal && e < wanted)) out[a + min(e, wanted)] = i;
        a += is_above;
        e += is_equal;
    }
    if (tid == 0) out[k] = n;
}

}  // namespace wht
