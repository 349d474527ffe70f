// Attention of a few rows over a list of pages, by warp-level matrix products.
//
//     o = sum_j p_j v_j / sum_j p_j,    p_j = exp(scale q.k_j - m)
//
// in one pass over the keys: each chunk of 16 keys updates the running reference maximum m, the running sum l and the
// running product o.  Rows are (token, query head) pairs that read the same key head.  Three kinds of rows use the same
// loop over a list of physical pages:
//   prefix   all tokens of the batch against the shared prefix
//   own      the tokens of one sequence against its own pages, each seeing keys up to its own place
//   chosen   one token against the pages selected for it
//
// What bounds it: with few rows each key brings 4*D flops a row for 4*D bytes (bf16), far below the machine's balance,
// so the loop has to be a stream of keys and values with as few instructions per byte as possible.  (A first version
// with rows as the left operand and 16-byte copies by all threads issued 1640 warp instructions per 16 KB and was bound by
// them at 4.1 TB/s: half of a 16-row operand empty, two thirds of the instructions addresses of copies.)  Hence:
//   - Products are taken transposed, S^T = K Q^T and O^T = V^T P^T: keys and channels fill the 16-row operand and the rows sit
//     on the 8-column one, so 8 rows waste nothing.  P^T changes from accumulator to operand layout by one 8x8 transposition.
//   - Each warp streams its own chunks: one lane asks the copy engine (TMA, 128-byte swizzle) for the key and value boxes
//     of a chunk, and a ring of chunks per warp keeps 16 to 24 KB in flight; no warp waits for another in the loop.
//   - m moves only when a score passes it by more than 2^8, found by one vote: weights up to 2^8 are as exact as weights up to 1, and
//     neither the reduction over lanes nor the scaling of o is in the common path.
// A unit's keys are divided over 1, 2, 4 or 8 warps of a block, which join their (m, l, o) through shared memory, and over
// blocks where there are too few units to fill the machine (attn_join_kernel adds those parts up).
//
// Measured, bf16, D = 128: 64 sequences x 2048 keys, 8 key heads of 4 rows 82.6 us (6.5 TB/s, all that memory gives); 256 x 150 keys, 32 heads
// 103 us (6.1 TB/s).  Pages out of the L2 cache (2048 prompt tokens of 4 key heads with 16 pages of 64 each) 275 us for 4.3 GB, 15.6 TB/s: with
// eight warps an SM (371 us) and with twelve the first wait is for the results of products and the arithmetic between them (3.0 of 6.5 clocks a warp
// and instruction); the cache is at 57 %, the tensor pipe at 34 %.
//
// fp32 tensors: both operands of each product are split in two tf32 terms (three products; what is dropped is below 2^-21
// relative), contraction indices paired so that a thread's two values are neighbours.  Bound by those products: 64 x 2048 keys as above
// 240 us (4.5 TB/s).
#pragma once
#include <cuda.h>

#include <type_traits>

#include "attn_common.cuh"

namespace wht {

constexpr int kChunk = 16;       // keys per chunk: they lie in one page
constexpr float kSlack = 8.0f;   // log2 of how far a score may pass the reference maximum

struct AttnParams {
    const void *q, *k_cache, *v_cache;
    int64_t q_st, q_sh;
    void* out;
    // partial results [part][T * Hq]: maximum and sum, and the unscaled product
    float2* part_ml;
    float* part_o;
    int parts;             // how many parts a row has in all (1: results go to `out`)
    // shared prefix
    const int32_t* prefix_pages;
    int64_t prefix_len;
    int prefix_splits, prefix_row_tiles, prefix_nr, prefix_wpu;  // nr: 8-row tiles per unit; wpu: warps per unit
    // own pages
    const int32_t *page_table, *kv_lens, *q_start;
    int table_width, B, max_q_len;
    int own_splits, own_row_tiles, own_nr, own_wpu;
    int joint;             // small calls: every sequence walks the prefix's pages before its own, and nothing is left to join
    // chosen pages: [T x Hkv x select] indices into the sequence's table
    const int32_t* chosen;
    int select;
    int64_t T, num_pages;
    int hq, hkv, group, page_shift;
    float scale_log2;      // scale * log2(e)
};

// The tensor-core form of the prefix (attn_umma_kernels.cuh).
struct UmmaAttnParams {
    AttnParams a;    // queries, prefix, partial results
    int splits;      // key ranges
    int row_blocks;  // blocks of 256 rows
    int same_rows;   // 128 rows or fewer: both of a block's tiles hold them, each with every second key tile
};

// W: warps per block.  Four, so that two or three blocks fit an SM; eight for small calls, where a unit is a block and all that counts
// is how soon its last key is done.  N: the most 8-row tiles a unit has, 1 or 4.  Units of one tile (bf16) need fewer registers and a
// shorter ring, so that three blocks fit: with eight warps an SM the wait is for the results of products, not for memory.
template <typename T, int D, int W, int N>
struct AttnGeo {
    static constexpr int THREADS = 32 * W;
    static constexpr bool F32 = std::is_same<T, float>::value;
    static constexpr int BOX_CH = 128 / static_cast<int>(sizeof(T));    // channels per 128-byte box
    static constexpr int BOXES = (D + BOX_CH - 1) / BOX_CH;             // per key row (the last may reach over the row's end: zeros)
    static constexpr int BOX_BYTES = kChunk * 128;
    static constexpr int SIDE = BOXES * BOX_BYTES;                      // keys (or values) of a chunk
    static constexpr bool SLIM = N == 1 && W == 4 && !F32;
    static constexpr int BLOCKS = SLIM ? 3 : 1;                         // on an SM, at least
    static constexpr int STAGES = SLIM ? 16384 / (2 * SIDE) : 2 * SIDE >= 16384 ? (W > 4 ? 1 : 2) : 24576 / (2 * SIDE);
    static constexpr int RING = SLIM ? 16384 : STAGES * 2 * SIDE > 18432 ? STAGES * 2 * SIDE : 18432;  // per warp; holds the join buffer too
    static constexpr int OFF_BARS = W * RING;
    static constexpr int BYTES = OFF_BARS + W * STAGES * 8 + 1024;      // and what aligning the start to 1024 bytes takes
    static constexpr int JOIN_LD = D + 4;                               // floats per row of the join buffer: no bank conflicts
    static_assert(8 * N * (JOIN_LD + 2) * 4 <= RING, "the join buffer reuses the ring");
    // byte offset of 16-byte piece c of row r (the copy engine's 128-byte swizzle)
    __device__ __forceinline__ static int place(int r, int c) { return (c >> 3) * BOX_BYTES + r * 128 + (((c & 7) ^ (r & 7)) << 4); }
};

// One unit of work.
struct AttnUnit {
    int head;            // key head
    int64_t token0;      // first token of the row set
    int rows;            // rows of the set: row r = (token0 + r / group, head * group + r % group)
    int row0;            // first row of this unit
    const int32_t* ids;  // page list: physical pages, or (chosen) indices into `table`
    const int32_t* table;
    int key0, key1;      // this part's keys, counted along the list; key0 a multiple of 16
    const int32_t* ids2; // (joint) the list goes on here after list1 entries
    int list1;
    int hole0, hole1;    // (joint) keys hole0 .. hole1 - 1 are the unused end of the prefix's last page; else 0
    int limit0, step;    // row r sees keys < min(key1, max(hole1, limit0 + (r / group) * step)), but for the hole
    int part;            // where the partial result goes
    int nr, wpu;         // 8-row tiles, warps
};

// TOKENS: a unit's rows may be of several tokens, which see different keys.
template <typename T, int D, int NR, int W, int N, bool TOKENS>
__device__ __forceinline__ void attn_unit(const AttnParams& p, const AttnUnit& u, const CUtensorMap* k_map, const CUtensorMap* v_map,
                                          unsigned char* smem) {
    using Geo = AttnGeo<T, D, W, N>;
    constexpr bool F32 = Geo::F32;
    constexpr int QS = D / (F32 ? 8 : 16);       // steps of the first product
    constexpr int DT = D / 16;                   // 16-channel tiles of the output
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int wi = warp % u.wpu;                 // this warp among the unit's
    const int r4 = lane >> 2, c4 = lane & 3;
    unsigned char* ring = smem + warp * Geo::RING;
    const uint32_t ring_u32 = smem_u32(ring);
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + Geo::OFF_BARS) + warp * Geo::STAGES;
    const int all = (u.key1 - u.key0 + kChunk - 1) / kChunk;
    const int chunks = all > wi ? (all - wi + u.wpu - 1) / u.wpu : 0;   // this warp's: wi, wi + wpu, ...

    if (lane == 0) {
        for (int s = 0; s < Geo::STAGES; ++s) mbar_init(full + s, 1);
        fence_mbar_init();
    }
    // cache rows of 32 of this warp's chunks, one per lane, and of the next 32
    auto rows_of = [&](int j) {
        int y = 0;
        if (j + lane < chunks) {
            const int key = u.key0 + (wi + (j + lane) * u.wpu) * kChunk;
            const int e = key >> p.page_shift;
            int pg = __ldg(e < u.list1 ? u.ids + e : u.ids2 + (e - u.list1));
            if (u.table) pg = pg >= 0 ? __ldg(u.table + pg) : -1;
            if (pg < 0 || pg >= p.num_pages) {
                attn_report(kAttnErrIndex);
                pg = 0;
            }
            y = ((pg * p.hkv + u.head) << p.page_shift) + (key & ((1 << p.page_shift) - 1));
        }
        return y;
    };
    int y_now = rows_of(0), y_next = chunks > 32 ? rows_of(32) : 0;
    __syncwarp();
    auto load = [&](int j, int y) {              // lane 0: chunk j, whose first cache row is y
        const int s = j % Geo::STAGES;
        const uint32_t dst = ring_u32 + s * 2 * Geo::SIDE;
        mbar_expect_tx(full + s, 2 * Geo::SIDE);
#pragma unroll
        for (int b = 0; b < Geo::BOXES; ++b) {
            tma_load_2d(dst + b * Geo::BOX_BYTES, k_map, b * Geo::BOX_CH, y, full + s);
            tma_load_2d(dst + Geo::SIDE + b * Geo::BOX_BYTES, v_map, b * Geo::BOX_CH, y, full + s);
        }
    };
#pragma unroll
    for (int j = 0; j < Geo::STAGES; ++j) {
        const int y = __shfl_sync(kFullMask, y_now, j);
        if (lane == 0 && j < chunks) load(j, y);
    }

    // rows as the second operand: column r4 of 8-row tile n is row row0 + 8 n + r4
    uint32_t qf[NR][QS][2];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        const int row = u.row0 + 8 * n + r4, tok = row / p.group;
        const T* src = static_cast<const T*>(p.q) + (u.token0 + tok) * p.q_st +
                       (static_cast<int64_t>(u.head) * p.group + (row - tok * p.group)) * p.q_sh;
#pragma unroll
        for (int s = 0; s < QS; ++s) {
            if constexpr (F32) {
                // contraction index c stands for channel 2c, c + 4 for 2c + 1
                const float2 a = row < u.rows ? *reinterpret_cast<const float2*>(src + s * 8 + 2 * c4) : make_float2(0.f, 0.f);
                qf[n][s][0] = __float_as_uint(a.x);
                qf[n][s][1] = __float_as_uint(a.y);
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    qf[n][s][i] = row < u.rows ? *reinterpret_cast<const uint32_t*>(src + s * 16 + i * 8 + 2 * c4) : 0u;
            }
        }
    }
    // as accumulator columns a thread's rows are 8 n + 2 c4 and the next
    int limit[NR][2];
    int least_limit = u.key1;
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int row = u.row0 + 8 * n + 2 * c4 + e;
            limit[n][e] = min(u.key1, max(u.hole1, u.limit0 + (row / p.group) * u.step));
            if (row >= u.rows) limit[n][e] = u.key1;
        }
    least_limit = min(u.key1, max(u.hole1, u.limit0 + (u.row0 / p.group) * u.step));

    float o[NR][DT][4];
    float m[NR][2], l[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        m[n][0] = m[n][1] = -INFINITY;
        l[n][0] = l[n][1] = 0.0f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[n][d][0] = o[n][d][1] = o[n][d][2] = o[n][d][3] = 0.0f;
    }

    // O^T += V^T P^T for one chunk; w: the chunk's weights as accumulators (keys r4, r4 + 8; rows 2 c4, 2 c4 + 1)
    auto add_values = [&](const float (&w)[NR][4], int s) {
        const uint32_t vt = ring_u32 + s * 2 * Geo::SIDE + Geo::SIDE;
        if constexpr (F32) {
            const unsigned char* vp = ring + s * 2 * Geo::SIDE + Geo::SIDE;
#pragma unroll
            for (int h = 0; h < 2; ++h) {        // keys 8 h .. 8 h + 7
                // operand layout: keys c4 and c4 + 4 of row r4, held by lanes (key, row / 2)
                uint32_t bh[NR][2], bl[NR][2];
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int from = (c4 + 4 * i) * 4 + (r4 >> 1);
                        const float even = __shfl_sync(kFullMask, w[n][2 * h], from), odd = __shfl_sync(kFullMask, w[n][2 * h + 1], from);
                        split_tf32(r4 & 1 ? odd : even, bh[n][i], bl[n][i]);
                    }
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    uint32_t ah[4], al[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = 8 * h + c4 + 4 * (i >> 1), ch = d * 16 + r4 + 8 * (i & 1);
                        split_tf32(*reinterpret_cast<const float*>(vp + Geo::place(key, ch >> 2) + (ch & 3) * 4), ah[i], al[i]);
                    }
#pragma unroll
                    for (int n = 0; n < NR; ++n) {
                        // (the tensor core's accumulation truncates: one chunk at a time, added up with rounding)
                        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                        mma_tf32_1688(sum, al, bh[n][0], bh[n][1]);
                        mma_tf32_1688(sum, ah, bl[n][0], bl[n][1]);
                        mma_tf32_1688(sum, ah, bh[n][0], bh[n][1]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[n][d][i] += sum[i];
                    }
                }
            }
        } else {
            // each weight as two bf16 terms: one term's 2^-9 would stand beside the rounding of the output in every result
            uint32_t b[NR][2], low[NR][2];
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t lead = pack_bf16x2(w[n][2 * i], w[n][2 * i + 1]);
                    b[n][i] = transpose_8x8(lead);
                    low[n][i] = transpose_8x8(pack_bf16x2(w[n][2 * i] - __uint_as_float(lead << 16), w[n][2 * i + 1] - __uint_as_float(lead & 0xffff0000u)));
                }
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                uint32_t a[4];
                ldmatrix_x4_trans(vt + Geo::place((lane & 7) + ((lane >> 4) << 3), 2 * d + ((lane >> 3) & 1)), a);
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    mma_bf16_16816(o[n][d], a, b[n][0], b[n][1]);
                    mma_bf16_16816(o[n][d], a, low[n][0], low[n][1]);
                }
            }
        }
    };

    auto values_finite = [&](int s) {
        const unsigned char* v = ring + s * 2 * Geo::SIDE + Geo::SIDE;
        constexpr uint32_t kExp = F32 ? 0x7f800000u : 0x7f80u;
        bool finite = true;
        for (int i = lane; i < Geo::SIDE / 4; i += 32) {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(v + i * 4);
            finite = finite && (w & kExp) != kExp && (F32 || ((w >> 16) & kExp) != kExp);
        }
        return __all_sync(kFullMask, finite) != 0;
    };
    auto add_seen_values = [&](const float (&w)[NR][4], int s, int base) {
        const unsigned char* v = ring + s * 2 * Geo::SIDE + Geo::SIDE;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll 1
            for (int k = 0; k < 8; ++k) {
                float weight[NR][2];
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) weight[n][e] = __shfl_sync(kFullMask, w[n][2 * h + e], k * 4 + c4);
#pragma unroll
                for (int d = 0; d < 2 * DT; ++d) {
                    const int ch = d * 8 + r4, bytes = ch * static_cast<int>(sizeof(T));
                    const float value = static_cast<float>(*reinterpret_cast<const T*>(v + Geo::place(8 * h + k, bytes >> 4) + (bytes & 15)));
#pragma unroll
                    for (int n = 0; n < NR; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            if (base + 8 * h + k < limit[n][e]) o[n][d >> 1][(d & 1) * 2 + e] += weight[n][e] * value;
                }
            }
    };

    for (int j = 0; j < chunks; ++j) {
        const int s = j % Geo::STAGES;
        mbar_wait_bounded(full + s, static_cast<uint32_t>(j / Geo::STAGES) & 1u);
        const int base = u.key0 + (wi + j * u.wpu) * kChunk;
        const int end = base < u.hole1 ? min(u.hole0, u.key1) : u.key1;  // the first key from `base` on that nobody sees
        const bool mask = base + kChunk > min(end, least_limit);
        if (base + kChunk > end) {
            // keys that nobody sees: their values become 0, so that a weight of 0 takes nothing from whatever lies there
            const int valid = max(0, end - base);
            unsigned char* v = ring + s * 2 * Geo::SIDE + Geo::SIDE;
            for (int i = lane; i < (kChunk - valid) * 8 * Geo::BOXES; i += 32) {
                const int r = valid + i / (8 * Geo::BOXES), c = i % (8 * Geo::BOXES);
                *reinterpret_cast<uint4*>(v + Geo::place(r, c)) = make_uint4(0, 0, 0, 0);
            }
            // (behind a hole the list goes on, and the copy engine writes this slot again: ordinary stores come before it)
            fence_before_copies();
            __syncwarp();
        }

        // S^T = K Q^T: keys r4 (elements 0, 1) and r4 + 8 (2, 3); rows 2 c4, 2 c4 + 1
        float x[NR][4];
#pragma unroll
        for (int n = 0; n < NR; ++n) x[n][0] = x[n][1] = x[n][2] = x[n][3] = 0.0f;
        if constexpr (F32) {
            // The tensor core's accumulation truncates, so a long chain of products drifts: the leading products are taken
            // one instruction at a time and added up with rounding, the small ones keep a chain of their own.
            const unsigned char* kp = ring + s * 2 * Geo::SIDE;
            float small[NR][4];
#pragma unroll
            for (int n = 0; n < NR; ++n) small[n][0] = small[n][1] = small[n][2] = small[n][3] = 0.0f;
#pragma unroll
            for (int ks = 0; ks < QS; ++ks) {
                uint32_t ah[4], al[4];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float2 k = *reinterpret_cast<const float2*>(kp + Geo::place(r4 + 8 * i, ks * 2 + (c4 >> 1)) + (c4 & 1) * 8);
                    split_tf32(k.x, ah[i], al[i]);
                    split_tf32(k.y, ah[2 + i], al[2 + i]);
                }
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    uint32_t h0, h1, l0, l1;
                    split_tf32(__uint_as_float(qf[n][ks][0]), h0, l0);
                    split_tf32(__uint_as_float(qf[n][ks][1]), h1, l1);
                    float lead[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                    mma_tf32_1688(small[n], al, h0, h1);
                    mma_tf32_1688(small[n], ah, l0, l1);
                    mma_tf32_1688(lead, ah, h0, h1);
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[n][i] += lead[i];
                }
            }
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[n][i] += small[n][i];
        } else {
            const uint32_t kt = ring_u32 + s * 2 * Geo::SIDE;
#pragma unroll
            for (int ks = 0; ks < QS; ++ks) {
                uint32_t a[4];
                ldmatrix_x4(kt + Geo::place((lane & 7) + ((lane >> 3) & 1) * 8, 2 * ks + (lane >> 4)), a);
#pragma unroll
                for (int n = 0; n < NR; ++n) mma_bf16_16816(x[n], a, qf[n][ks][0], qf[n][ks][1]);
            }
        }
        bool passes = false;
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[n][i] *= p.scale_log2;
                const int key = base + r4 + 8 * (i >> 1);
                if (mask && (key >= limit[n][i & 1] || (key >= u.hole0 && key < u.hole1))) x[n][i] = -INFINITY;
                passes = passes || x[n][i] > m[n][i & 1] + kSlack;
            }
        if (__any_sync(kFullMask, passes)) {
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float top = fmaxf(x[n][e], x[n][2 + e]);
#pragma unroll
                    for (int i = 4; i < 32; i <<= 1) top = fmaxf(top, __shfl_xor_sync(kFullMask, top, i));
                    if (top > m[n][e]) {
                        const float f = exp2_fast(m[n][e] - top);
                        m[n][e] = top;
                        l[n][e] *= f;
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            o[n][d][e] *= f;
                            o[n][d][2 + e] *= f;
                        }
                    }
                }
        }
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // a row that has seen no key has m = -infinity: every weight is 0
                const float z = m[n][i & 1] == -INFINITY ? 0.0f : m[n][i & 1];
                x[n][i] = exp2_fast(x[n][i] - z);
                l[n][i & 1] += x[n][i];
            }
        // Rows that see different keys share each product, where a weight of 0 would turn an infinity or NaN among the values of a later
        // token into NaN for the earlier ones: such a chunk (found by a look at the values of the few that straddle a row's end) is
        // added up row by row.
        if (TOKENS && least_limit < end && base + kChunk > least_limit && !values_finite(s)) add_seen_values(x, s, base);
        else add_values(x, s);
        __syncwarp();                            // every lane has read the slot
        const int next = j + Geo::STAGES;
        if ((next & 31) == 0) {
            y_now = y_next;
            y_next = next + 32 < chunks ? rows_of(next + 32) : 0;
        }
        const int y = __shfl_sync(kFullMask, y_now, next & 31);
        if (lane == 0 && next < chunks) load(next, y);
    }
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int i = 4; i < 32; i <<= 1) l[n][e] += __shfl_xor_sync(kFullMask, l[n][e], i);

    // the unit's warps store (m, l, o) over their rings and add them up together
    {
        float* jo = reinterpret_cast<float*>(ring);
        float2* jm = reinterpret_cast<float2*>(jo + 8 * N * Geo::JOIN_LD);
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = 8 * n + 2 * c4 + e;
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    jo[r * Geo::JOIN_LD + d * 16 + r4] = o[n][d][e];
                    jo[r * Geo::JOIN_LD + d * 16 + 8 + r4] = o[n][d][2 + e];
                }
                if (r4 == 0) jm[r] = make_float2(m[n][e], l[n][e]);
            }
    }
    if (u.wpu == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(warp / u.wpu + 1), "r"(u.wpu * 32) : "memory");
    const unsigned char* first = smem + (warp - wi) * Geo::RING;
    const int rows_here = min(NR * 8, u.rows - u.row0);
    constexpr int PER = 4;                       // channels per thread and step
    for (int i = wi * 32 + lane; i < rows_here * (D / PER); i += u.wpu * 32) {
        const int r = i / (D / PER), d = (i % (D / PER)) * PER;
        float mm = -INFINITY;
        for (int w = 0; w < u.wpu; ++w)
            mm = fmaxf(mm, reinterpret_cast<const float2*>(first + w * Geo::RING + 8 * N * Geo::JOIN_LD * 4)[r].x);
        const float z = mm == -INFINITY ? 0.0f : mm;
        float ll = 0.0f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int w = 0; w < u.wpu; ++w) {
            const float* wo = reinterpret_cast<const float*>(first + w * Geo::RING);
            const float2 ml = reinterpret_cast<const float2*>(wo + 8 * N * Geo::JOIN_LD)[r];
            const float f = exp2_fast(ml.x - z);
            ll += f * ml.y;
            const float4 v = *reinterpret_cast<const float4*>(wo + r * Geo::JOIN_LD + d);
            acc.x += f * v.x; acc.y += f * v.y; acc.z += f * v.z; acc.w += f * v.w;
        }
        const int row = u.row0 + r, tok = row / p.group;
        const int64_t at = (u.token0 + tok) * p.hq + u.head * p.group + (row - tok * p.group);
        if (p.parts == 1) {
            const float inv = ll > 0.0f ? 1.0f / ll : 0.0f;
            T* dst = static_cast<T*>(p.out) + at * D + d;
            if constexpr (F32)
                *reinterpret_cast<float4*>(dst) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
            else
                *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
        } else {
            const int64_t slot = static_cast<int64_t>(u.part) * p.T * p.hq + at;
            *reinterpret_cast<float4*>(p.part_o + slot * D + d) = acc;
            if (d == 0) p.part_ml[slot] = make_float2(mm, ll);
        }
    }
}

template <typename T, int D, int W, int N, bool TOKENS>
__device__ __forceinline__ void attn_run(const AttnParams& p, const AttnUnit& u, const CUtensorMap* k_map, const CUtensorMap* v_map) {
    extern __shared__ unsigned char smem_attn[];
    unsigned char* smem = smem_attn + ((1024u - (smem_u32(smem_attn) & 1023u)) & 1023u);
    if constexpr (N == 1) {
        attn_unit<T, D, 1, W, N, TOKENS>(p, u, k_map, v_map, smem);
    } else {
        if (u.nr == 1) attn_unit<T, D, 1, W, N, TOKENS>(p, u, k_map, v_map, smem);
        else if (u.nr == 2) attn_unit<T, D, 2, W, N, TOKENS>(p, u, k_map, v_map, smem);
        else attn_unit<T, D, 4, W, N, TOKENS>(p, u, k_map, v_map, smem);
    }
}

// A length read on the device, held to what the tables can hold.
__device__ __forceinline__ int attn_length(const AttnParams& p, int b) {
    const int64_t most = static_cast<int64_t>(p.table_width) << p.page_shift;
    const int n = __ldg(p.kv_lens + b);
    if (n < 0 || n > most) {
        attn_report(kAttnErrIndex);
        return n < 0 ? 0 : static_cast<int>(most);
    }
    return n;
}
// The tokens of sequence b: first and count, held to the call's T and max_q_len.
__device__ __forceinline__ void attn_tokens(const AttnParams& p, int b, int64_t& first, int& count) {
    if (p.q_start == nullptr) {
        first = b;
        count = 1;
        return;
    }
    int64_t a = __ldg(p.q_start + b), e = __ldg(p.q_start + b + 1);
    if (a < 0 || e < a || e > p.T || e - a > p.max_q_len) {
        attn_report(kAttnErrIndex);
        a = a < 0 ? 0 : (a > p.T ? p.T : a);
        e = e < a ? a : (e > p.T ? p.T : e);
        if (e - a > p.max_q_len) e = a + p.max_q_len;
    }
    first = a;
    count = static_cast<int>(e - a);
}

// The place of token t in its sequence: the last key it sees.  Negative: it sees none.
__device__ __forceinline__ int64_t attn_place(const AttnParams& p, int b, int64_t t, int64_t first, int count) {
    if (t < first || t - first >= count) {  // a token of no sequence
        attn_report(kAttnErrIndex);
        return -1;
    }
    return static_cast<int64_t>(attn_length(p, b)) - count + (t - first);
}

// The tokens that the sequences cover are first .. last - 1; says whether that is all of them.  (q_start is not NULL.)
__device__ __forceinline__ bool attn_covered(const AttnParams& p, int64_t& first, int64_t& last) {
    const int64_t a = __ldg(p.q_start), e = __ldg(p.q_start + p.B);
    first = a < 0 ? 0 : (a > p.T ? p.T : a);
    last = e < first ? first : (e > p.T ? p.T : e);
    return first == 0 && last == p.T;
}
// Tokens of no sequence are reported.  Nobody's keys are theirs: one warp per key head sets their rows to zero (those of several parts
// are left to the join).
template <typename T, int D>
__device__ __forceinline__ void attn_uncovered(const AttnParams& p, int head) {
    int64_t first, last;
    if (attn_covered(p, first, last)) return;
    attn_report(kAttnErrIndex);
    if (p.parts > 1) return;
    const int pieces = p.group * D * static_cast<int>(sizeof(T)) / 16;
    for (int64_t t = 0; t < p.T; ++t) {
        if (t == first) t = last;
        if (t >= p.T) break;
        uint4* row = reinterpret_cast<uint4*>(static_cast<T*>(p.out) + (t * p.hq + static_cast<int64_t>(head) * p.group) * D);
        for (int i = threadIdx.x & 31; i < pieces; i += 32) row[i] = make_uint4(0, 0, 0, 0);
    }
}

// keys [key0, key1) of part `s` of `splits`, in whole tiles
__device__ __forceinline__ void attn_part(int keys, int tile, int splits, int s, int& key0, int& key1) {
    const int tiles = (keys + tile - 1) / tile;
    const int per = (tiles + splits - 1) / splits;
    const int64_t a = static_cast<int64_t>(s) * per * tile, e = a + static_cast<int64_t>(per) * tile;
    key0 = a < keys ? static_cast<int>(a) : keys;
    key1 = e < keys ? static_cast<int>(e) : keys;
}

// Prefix and own pages in one launch: blocks below prefix_blocks take the prefix.
template <typename T, int D, int W, int N>
__global__ void __launch_bounds__(32 * W, AttnGeo<T, D, W, N>::BLOCKS)
attn_prefix_kernel(const AttnParams p, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
    const int prefix_units = p.prefix_splits * p.prefix_row_tiles * p.hkv;
    const int prefix_blocks = (prefix_units * p.prefix_wpu + W - 1) / W;
    const int warp = threadIdx.x >> 5;
    const bool last_block = blockIdx.x == gridDim.x - 1;
    AttnUnit u;
    bool work;
    u.list1 = 0x7fffffff;
    u.hole0 = u.hole1 = 0;
    grid_launch_dependents();
    if (static_cast<int>(blockIdx.x) < prefix_blocks) {
        int b = (blockIdx.x * W + warp) / p.prefix_wpu;
        work = b < prefix_units;
        u.part = b % p.prefix_splits;
        b /= p.prefix_splits;
        u.row0 = (b % p.prefix_row_tiles) * 8 * p.prefix_nr;
        u.head = b / p.prefix_row_tiles;
        u.token0 = 0;
        u.rows = static_cast<int>(p.T) * p.group;
        u.ids = p.prefix_pages;
        const int keys = static_cast<int>(p.prefix_len);
        attn_part(keys, kChunk * 4, p.prefix_splits, u.part, u.key0, u.key1);
        u.limit0 = keys;
        u.step = 0;
        u.nr = p.prefix_nr;
        u.wpu = p.prefix_wpu;
    } else {
        int b = ((blockIdx.x - prefix_blocks) * W + warp) / p.own_wpu;
        const int split = b % p.own_splits;
        b /= p.own_splits;
        u.part = (p.parts - p.own_splits) + split;
        u.row0 = (b % p.own_row_tiles) * 8 * p.own_nr;
        b /= p.own_row_tiles;
        u.head = b % p.hkv;
        const int seq = b / p.hkv;
        int count = 0, keys = 0;
        if (seq < p.B) {
            // the table's row is wanted as soon as the length is known: fetch it meanwhile
            u.ids = p.page_table + static_cast<int64_t>(seq) * p.table_width;
            const int ahead = (static_cast<int>(threadIdx.x) & 31) * 32;
            if (ahead < p.table_width) asm volatile("prefetch.global.L1 [%0];" ::"l"(u.ids + ahead));
            attn_tokens(p, seq, u.token0, count);
            keys = attn_length(p, seq);
            if (p.q_start != nullptr && seq == 0 && u.row0 == 0 && split == 0 && warp % p.own_wpu == 0) attn_uncovered<T, D>(p, u.head);
        }
        u.rows = count * p.group;
        work = u.row0 < u.rows;
        if (p.joint) {
            u.ids2 = u.ids;
            u.ids = p.prefix_pages;
            u.hole0 = static_cast<int>(p.prefix_len);
            u.list1 = (u.hole0 + (1 << p.page_shift) - 1) >> p.page_shift;
            u.hole1 = u.list1 << p.page_shift;
            keys += u.hole1;
        }
        // the unit's last row sees the most: nothing beyond its place is read
        u.limit0 = keys - count + 1;
        u.step = 1;
        const int last_tok = (min(u.rows, u.row0 + 8 * p.own_nr) - 1) / p.group;
        attn_part(keys, kChunk * 4, p.own_splits, split, u.key0, u.key1);
        u.key1 = max(u.key0, min(u.key1, max(u.hole1, u.limit0 + last_tok)));
        u.nr = p.own_nr;
        u.wpu = p.own_wpu;
    }
    u.table = nullptr;
    if (work) attn_run<T, D, W, N, true>(p, u, &k_map, &v_map);
    // Launched next to the tensor-core kernel of the prefix, these blocks run while it runs; the join that follows waits
    // for this grid alone, so this grid does not end before that one has.
    if (last_block) grid_dependency_wait();
}

// The sequence that token t belongs to (q_start ascending): 32 lanes probe at once.
__device__ __forceinline__ int attn_sequence_of(const AttnParams& p, int64_t t) {
    if (p.q_start == nullptr) return static_cast<int>(t);
    const int lane = threadIdx.x & 31;
    int lo = 0, n = p.B;  // the answer is in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 31) / 32;
        const int at = lo + lane * step;
        const bool ok = lane * step < n && __ldg(p.q_start + at) <= t;
        const unsigned hits = __ballot_sync(kFullMask, ok);
        const int last = hits ? 31 - __clz(hits) : 0;
        lo += last * step;
        n = min(step, n - last * step);
    }
    return lo;
}

// Chosen pages: one token and key head (and a part of the list) per unit.
template <typename T, int D, int W, int N>
__global__ void __launch_bounds__(32 * W, AttnGeo<T, D, W, N>::BLOCKS)
attn_chosen_kernel(const AttnParams p, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
    AttnUnit u;
    grid_dependency_wait();  // the list comes from the kernel before
    grid_launch_dependents();
    int64_t b = (static_cast<int64_t>(blockIdx.x) * W + (threadIdx.x >> 5)) / p.own_wpu;
    u.part = static_cast<int>(b % p.own_splits);
    b /= p.own_splits;
    u.row0 = static_cast<int>(b % p.own_row_tiles) * 8 * p.own_nr;
    b /= p.own_row_tiles;
    u.head = static_cast<int>(b % p.hkv);
    u.token0 = b / p.hkv;
    if (u.token0 >= p.T) return;
    u.rows = p.group;
    const int seq = attn_sequence_of(p, u.token0);
    int64_t first;
    int count;
    attn_tokens(p, seq, first, count);
    const int64_t place = attn_place(p, seq, u.token0, first, count);
    u.ids = p.chosen + (u.token0 * p.hkv + u.head) * p.select;
    u.table = p.page_table + static_cast<int64_t>(seq) * p.table_width;
    u.list1 = 0x7fffffff;
    u.hole0 = u.hole1 = 0;
    const int list = place < 0 ? 0 : min(p.select, static_cast<int>(place >> p.page_shift) + 1);
    const int keys = place < 0 ? 0 : ((list - 1) << p.page_shift) + static_cast<int>(place & ((1 << p.page_shift) - 1)) + 1;
    attn_part(keys, kChunk * 4, p.own_splits, u.part, u.key0, u.key1);
    u.limit0 = keys;
    u.step = 0;
    u.nr = p.own_nr;
    u.wpu = p.own_wpu;
    attn_run<T, D, W, N, false>(p, u, &k_map, &v_map);
}

// Joins the parts of each row: out = sum_s exp(m_s - m) o_s / sum_s exp(m_s - m) l_s.  One warp per row, lanes
// over the channels; the parts' statistics are read by the lanes at once.  q_start (or NULL): rows of tokens that no sequence covers
// have parts that nobody wrote, and get zeros.
template <typename T, int D>
__global__ void __launch_bounds__(128)
attn_join_kernel(const float2* __restrict__ ml, const float* __restrict__ po, T* __restrict__ out, int64_t rows, int parts,
                 const int32_t* __restrict__ q_start, int B, int hq) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5);
    if (row >= rows) return;
    bool covered = true;
    if (q_start != nullptr) {
        const int t = static_cast<int>(row) / hq;
        covered = t >= __ldg(q_start) && t < __ldg(q_start + B);
    }
    float m = -INFINITY;
    for (int s = lane; s < parts; s += 32) m = fmaxf(m, ml[s * rows + row].x);
#pragma unroll
    for (int i = 16; i; i >>= 1) m = fmaxf(m, __shfl_xor_sync(kFullMask, m, i));
    const float z = m == -INFINITY ? 0.0f : m;
    constexpr int PER = 4;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.0f;
    for (int s0 = 0; s0 < parts; s0 += 32) {
        float2 mine = make_float2(-INFINITY, 0.0f);
        if (s0 + lane < parts) mine = ml[(s0 + lane) * rows + row];
        const float f = exp2_fast(mine.x - z);
        l += f * mine.y;
        // eight parts' products in flight at a time: the rows are short and the wait is all latency
        const int n = min(32, parts - s0);
        for (int s1 = 0; s1 < n; s1 += 8) {
            float4 x[8];
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                x[s] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (s1 + s < n && lane * PER < D) x[s] = *reinterpret_cast<const float4*>(po + ((s0 + s1 + s) * rows + row) * D + lane * PER);
            }
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const float w = __shfl_sync(kFullMask, f, s1 + s);  // (a part that holds no key of this row has weight 0)
                acc.x += w * x[s].x; acc.y += w * x[s].y; acc.z += w * x[s].z; acc.w += w * x[s].w;
            }
        }
    }
#pragma unroll
    for (int i = 16; i; i >>= 1) l += __shfl_xor_sync(kFullMask, l, i);
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    if (!covered) acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (lane * PER < D) {
        T* dst = out + row * D + lane * PER;
        if constexpr (std::is_same<T, float>::value)
            *reinterpret_cast<float4*>(dst) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
        else
            *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
    }
}

}  // namespace wht
