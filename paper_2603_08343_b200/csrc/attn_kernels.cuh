// Attention of a few rows over a list of pages, by warp-level matrix products.
//
//     o = sum_j p_j v_j / sum_j p_j,    p_j = exp(scale q.k_j - m),   m = max_j scale q.k_j
//
// in one pass over the keys: each tile of keys updates the running maximum m, the running sum l and the running
// product o, which is scaled by exp(m_old - m_new) when the maximum moves.  Rows are (token, query head) pairs that
// read the same key head; a group of 2 or 4 warps takes up to 64 rows and one part of their keys, so each key and value is
// read once for all of the block's rows.  Three kinds of rows use the same loop over a list of physical pages:
//   prefix   all tokens of the batch against the shared prefix
//   own      the tokens of one sequence against its own pages, each seeing keys up to its own place
//   chosen   one token against the pages selected for it
//
// What bounds it: with few rows each key brings 4*D flops a row for 4*D bytes (bf16), far below the machine's
// balance, so the loop is a stream of keys and values: a ring of kStages tiles filled by 16-byte async copies keeps
// 64 KB a block in flight.  Warps that share a row tile take their own keys of each tile and join their (m, l, o)
// through shared memory at the end; with 4 row tiles every warp takes all keys for its rows.
// Keys are split over blocks where there are too few rows to fill the machine; the parts are joined by attn_join_kernel.
//
// Operands: rows of a tile are stored with their 16-byte chunks permuted by the row number (swizzle), so that matrix
// loads touch all banks.  The score accumulators' layout is the layout of the next product's left operand, so the
// weights never leave registers.  fp32 tensors: both operands of each product are split in two tf32 terms
// (three products, what is dropped is below 2^-21 relative), contraction indices paired so that a thread's two values are neighbours.
#pragma once
#include <type_traits>

#include "attn_common.cuh"

namespace wht {

constexpr int kAttnThreads = 128;
constexpr int kAttnIds = 512;  // pages of a block's list that are held at a time

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
    int prefix_splits, prefix_row_tiles, prefix_rw;  // rw: row tiles of 16 per block
    // own pages
    const int32_t *page_table, *kv_lens, *q_start;
    int table_width, B, max_q_len;
    int own_splits, own_row_tiles, own_rw;
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

// Bytes per row, and where a 16-byte chunk of a row lies.
template <typename T, int D>
struct AttnRow {
    static constexpr bool F32 = std::is_same<T, float>::value;
    static constexpr int ROW_BYTES = D * sizeof(T);
    static constexpr int CHUNKS = ROW_BYTES / 16;         // 16-byte chunks per key
    static constexpr int BLOCK_KEYS = F32 ? 32 : 64;      // keys per tile, all groups of a block together
    static constexpr int STAGES = D == 128 ? 3 : D == 96 ? 4 : 6;
    static constexpr int RING_BYTES = STAGES * 2 * BLOCK_KEYS * ROW_BYTES;  // 96 KB: two blocks per SM
    static constexpr int SMEM = RING_BYTES + kAttnIds * 4;
    // place of chunk c of row r: the permutation makes 8 consecutive rows' same chunk (bf16), or 4 rows' pairs of
    // chunks (fp32), fall into different banks
    __device__ __forceinline__ static int place(int r, int c) {
        int x;
        if constexpr (F32) x = ((r & 3) ^ ((r >> 2) & 1)) << 1;
        else if constexpr (D == 96) x = (r >> 1) & 3;
        else x = r & 7;
        return r * ROW_BYTES + ((c ^ x) << 4);
    }
};

// A group of warps works on one unit.  Up to 16 rows: two warps share the rows and halve the keys, and a block holds two
// such groups with a unit each (short sequences are all latency: four units in flight per SM instead of two took the own
// pages of 256 sequences at 32 x 128 heads from OWN_BEFORE to OWN_AFTER).  Up to 32 rows: two row tiles and two key halves.  Up to 64: four row tiles.
template <typename T, int D, int RW>
struct AttnGeo : AttnRow<T, D> {
    static constexpr int KW = RW == 4 ? 1 : 2;            // warps that share a row tile, each with its own keys of a tile
    static constexpr int THREADS = 32 * RW * KW;
    static constexpr int GROUPS = kAttnThreads / THREADS;
    static constexpr int KEYS = AttnRow<T, D>::BLOCK_KEYS / GROUPS;   // keys per tile
    static constexpr int TILE_BYTES = KEYS * AttnRow<T, D>::ROW_BYTES;  // keys (or values) of one tile
    static constexpr int GROUP_RING = AttnRow<T, D>::RING_BYTES / GROUPS;
    static constexpr int IDS = kAttnIds / GROUPS;
    // the join of the warps' results reuses the ring: 16 rows of D sums per warp, and their maxima and sums
    static_assert(RW * KW * 16 * (D + 4) * 4 <= GROUP_RING, "join buffer");
};
__host__ __device__ constexpr int attn_groups(int rw) { return rw == 1 ? 2 : 1; }
__device__ __forceinline__ void attn_group_sync(int group, int threads) {
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(threads) : "memory");
}

// One block's work.
struct AttnUnit {
    int head;            // key head
    int64_t token0;      // first token of the row set
    int rows;            // rows of the set: row r = (token0 + r / group, head * group + r % group)
    int row0;            // first row of this block
    const int32_t* ids;  // page list: physical pages, or (chosen) indices into `table`
    const int32_t* table;
    int list;            // entries of the list
    int key0, key1;      // this part's keys, counted along the list
    int limit0, step;    // row r sees keys < min(key1, limit0 + (r / group) * step)
    int part;            // where the partial result goes
};

template <typename T, int D, int RW>
__device__ __forceinline__ void attn_block(const AttnParams& p, const AttnUnit& u, unsigned char* block_smem) {
    using Geo = AttnGeo<T, D, RW>;
    constexpr bool F32 = Geo::F32;
    constexpr int KW = Geo::KW, THREADS = Geo::THREADS;
    constexpr int WKEYS = Geo::KEYS / KW;        // keys of a tile per warp
    constexpr int NT = WKEYS / 8;                // score tiles of 8 keys
    constexpr int DT = D / 8;                    // output tiles of 8 channels
    constexpr int KSTEP = F32 ? 8 : 16;          // contraction length of one instruction
    constexpr int QS = D / KSTEP;
    const int group = threadIdx.x / THREADS, tid = threadIdx.x % THREADS, lane = tid & 31, warp = tid >> 5;
    const int rt = warp / KW, kw = warp % KW;
    const int r4 = lane >> 2, c4 = lane & 3;
    unsigned char* smem = block_smem + group * Geo::GROUP_RING;
    int32_t* ids = reinterpret_cast<int32_t*>(block_smem + Geo::RING_BYTES) + group * Geo::IDS;
    const uint32_t ring = attn_smem_u32(smem);
    const T* kc = static_cast<const T*>(p.k_cache);
    const T* vc = static_cast<const T*>(p.v_cache);
    const int tiles = (u.key1 - u.key0 + Geo::KEYS - 1) / Geo::KEYS;

    // this thread's two rows (r4 and r4 + 8 of the warp's tile)
    int row[2], limit[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        row[i] = u.row0 + rt * 16 + r4 + 8 * i;
        const int tok = row[i] / p.group;
        limit[i] = row[i] < u.rows ? min(u.key1, u.limit0 + tok * u.step) : 0;
    }
    // the least limit of the block's rows: tiles that end before it need no mask
    const int free_keys = min(u.key1, u.limit0 + (u.row0 / p.group) * u.step);

    uint32_t qf[QS][4];
    {
        const T* q = static_cast<const T*>(p.q);
        const T* src[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int tok = row[i] / p.group;
            src[i] = q + (u.token0 + tok) * p.q_st + (static_cast<int64_t>(u.head) * p.group + (row[i] - tok * p.group)) * p.q_sh;
        }
#pragma unroll
        for (int s = 0; s < QS; ++s) {
            if constexpr (F32) {
                // contraction index c stands for channel 2c, c + 4 for 2c + 1
                const float2 a = row[0] < u.rows ? *reinterpret_cast<const float2*>(src[0] + s * 8 + 2 * c4) : make_float2(0.f, 0.f);
                const float2 b = row[1] < u.rows ? *reinterpret_cast<const float2*>(src[1] + s * 8 + 2 * c4) : make_float2(0.f, 0.f);
                qf[s][0] = __float_as_uint(a.x); qf[s][1] = __float_as_uint(b.x);
                qf[s][2] = __float_as_uint(a.y); qf[s][3] = __float_as_uint(b.y);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    qf[s][i] = row[i & 1] < u.rows
                                   ? *reinterpret_cast<const uint32_t*>(src[i & 1] + s * 16 + 2 * c4 + (i >> 1) * 8)
                                   : 0u;
            }
        }
    }

    float o[DT][4];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};

    const int ids0 = u.key0 >> p.page_shift;     // list entry of ids[0]
    int ids_base = ids0;
    auto load_ids = [&](int base) {              // all threads; the caller synchronises around it
        for (int i = tid; i < Geo::IDS; i += THREADS) {
            const int e = base + i;
            int32_t pg = -1;
            if (e < u.list) {
                pg = __ldg(u.ids + e);
                if (u.table) pg = pg >= 0 ? __ldg(u.table + pg) : -1;
                if (pg < 0 || pg >= p.num_pages) {
                    attn_report(kAttnErrIndex);
                    pg = -1;
                }
            }
            ids[i] = pg;
        }
    };
    auto load_tile = [&](int t) {                // keys and values of tile t into ring slot t % STAGES
        const uint32_t kd = ring + (t % Geo::STAGES) * 2 * Geo::TILE_BYTES, vd = kd + Geo::TILE_BYTES;
#pragma unroll
        for (int i = 0; i < Geo::KEYS * Geo::CHUNKS / THREADS; ++i) {
            const int j = tid + i * THREADS;
            const int r = j / Geo::CHUNKS, c = j % Geo::CHUNKS;
            const int key = u.key0 + t * Geo::KEYS + r;
            int64_t off = 0;
            int bytes = 0;
            if (key < u.key1) {
                const int pg = ids[(key >> p.page_shift) - ids_base];
                if (pg >= 0) {
                    bytes = 16;
                    off = (((static_cast<int64_t>(pg) * p.hkv + u.head) << p.page_shift) + (key & ((1 << p.page_shift) - 1))) * D +
                          c * (16 / static_cast<int>(sizeof(T)));
                }
            }
            const int at = Geo::place(r, c);
            cp_async16(kd + at, kc + off, bytes);
            cp_async16(vd + at, vc + off, bytes);
        }
    };

    load_ids(ids0);
    attn_group_sync(group, THREADS);
#pragma unroll
    for (int s = 0; s < Geo::STAGES - 1; ++s) {
        if (s < tiles) load_tile(s);
        cp_async_commit();
    }
    for (int t = 0; t < tiles; ++t) {
        cp_async_wait<Geo::STAGES - 2>();
        attn_group_sync(group, THREADS);                         // tile t has arrived, and everyone is done with tile t - 1
        const int next = t + Geo::STAGES - 1;
        if (next < tiles) {
            // the list moves on when the next tile's last key leaves the entries that are held
            const int last = min(u.key1 - 1, u.key0 + (next + 1) * Geo::KEYS - 1) >> p.page_shift;
            if (last >= ids_base + Geo::IDS) {
                ids_base = (u.key0 + next * Geo::KEYS) >> p.page_shift;
                load_ids(ids_base);
                attn_group_sync(group, THREADS);
            }
            load_tile(next);
        }
        cp_async_commit();

        const uint32_t kt = ring + (t % Geo::STAGES) * 2 * Geo::TILE_BYTES, vt = kt + Geo::TILE_BYTES;
        const unsigned char* kp = smem + (t % Geo::STAGES) * 2 * Geo::TILE_BYTES;
        const unsigned char* vp = kp + Geo::TILE_BYTES;
        const int k0 = kw * WKEYS;               // this warp's keys within the tile
        float s[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.0f;
        if constexpr (F32) {
            // The tensor core's accumulation truncates, so a long chain of products drifts: the leading products are taken
            // one instruction at a time and added up with rounding, the small ones keep a chain of their own.
            float small[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n) small[n][0] = small[n][1] = small[n][2] = small[n][3] = 0.0f;
#pragma unroll
            for (int ks = 0; ks < QS; ++ks) {
                uint32_t ah[4], al[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) split_tf32(__uint_as_float(qf[ks][i]), ah[i], al[i]);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int r = k0 + n * 8 + r4;
                    const float2 b = *reinterpret_cast<const float2*>(kp + Geo::place(r, ks * 2 + (c4 >> 1)) + (c4 & 1) * 8);
                    uint32_t h0, h1, l0, l1;
                    split_tf32(b.x, h0, l0);
                    split_tf32(b.y, h1, l1);
                    float lead[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                    mma_tf32_1688(small[n], al, h0, h1);
                    mma_tf32_1688(small[n], ah, l0, l1);
                    mma_tf32_1688(lead, ah, h0, h1);
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[n][i] += lead[i];
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[n][i] += small[n][i];
        } else {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int r = k0 + n * 8 + (lane & 7);
#pragma unroll
                for (int kk = 0; kk < D / 32; ++kk) {
                    uint32_t b[4];
                    ldmatrix_x4(kt + Geo::place(r, kk * 4 + (lane >> 3)), b);
                    mma_bf16_16816(s[n], qf[2 * kk], b[0], b[1]);
                    mma_bf16_16816(s[n], qf[2 * kk + 1], b[2], b[3]);
                }
            }
        }
        // scores in units of log2, masked; the running maximum
        const int base = u.key0 + t * Geo::KEYS + k0;
        const bool mask = u.key0 + (t + 1) * Geo::KEYS > free_keys;
        float top[2] = {m[0], m[1]};
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x = s[n][i] * p.scale_log2;
                if (mask && base + n * 8 + 2 * c4 + (i & 1) >= limit[i >> 1]) x = -INFINITY;
                s[n][i] = x;
                top[i >> 1] = fmaxf(top[i >> 1], x);
            }
        }
        float turn[2], zero[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            top[i] = fmaxf(top[i], __shfl_xor_sync(kFullMask, top[i], 1));
            top[i] = fmaxf(top[i], __shfl_xor_sync(kFullMask, top[i], 2));
            zero[i] = top[i] == -INFINITY ? 0.0f : top[i];  // a row that has seen no key: every weight is 0
            turn[i] = exp2_fast(m[i] - zero[i]);
        }
        if (__any_sync(kFullMask, top[0] != m[0] || top[1] != m[1])) {
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                o[i][0] *= turn[0]; o[i][1] *= turn[0];
                o[i][2] *= turn[1]; o[i][3] *= turn[1];
            }
            l[0] *= turn[0];
            l[1] *= turn[1];
            m[0] = top[0];
            m[1] = top[1];
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[n][i] = exp2_fast(s[n][i] - zero[i >> 1]);
                l[i >> 1] += s[n][i];
            }
        }
        if constexpr (F32) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                // contraction index c stands for key 2c, c + 4 for 2c + 1
                uint32_t ah[4], al[4];
                split_tf32(s[n][0], ah[0], al[0]);
                split_tf32(s[n][2], ah[1], al[1]);
                split_tf32(s[n][1], ah[2], al[2]);
                split_tf32(s[n][3], ah[3], al[3]);
                const int r = k0 + n * 8 + 2 * c4;
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                    const float b0 = *reinterpret_cast<const float*>(vp + Geo::place(r, d * 2 + (r4 >> 2)) + (r4 & 3) * 4);
                    const float b1 = *reinterpret_cast<const float*>(vp + Geo::place(r + 1, d * 2 + (r4 >> 2)) + (r4 & 3) * 4);
                    uint32_t h0, h1, l0, l1;
                    split_tf32(b0, h0, l0);
                    split_tf32(b1, h1, l1);
                    mma_tf32_1688(sum, al, h0, h1);
                    mma_tf32_1688(sum, ah, l0, l1);
                    mma_tf32_1688(sum, ah, h0, h1);
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[d][i] += sum[i];
                }
            }
        } else {
#pragma unroll
            for (int n = 0; n < NT; n += 2) {
                const uint32_t a[4] = {pack_bf16x2(s[n][0], s[n][1]), pack_bf16x2(s[n][2], s[n][3]),
                                       pack_bf16x2(s[n + 1][0], s[n + 1][1]), pack_bf16x2(s[n + 1][2], s[n + 1][3])};
                const int r = k0 + n * 8 + (lane & 15);
#pragma unroll
                for (int d = 0; d < DT; d += 2) {
                    uint32_t b[4];
                    ldmatrix_x4_trans(vt + Geo::place(r, d + (lane >> 4)), b);
                    mma_bf16_16816(o[d], a, b[0], b[1]);
                    mma_bf16_16816(o[d + 1], a, b[2], b[3]);
                }
            }
        }
    }
    cp_async_wait<0>();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        l[i] += __shfl_xor_sync(kFullMask, l[i], 1);
        l[i] += __shfl_xor_sync(kFullMask, l[i], 2);
    }

    if constexpr (KW > 1) {
        // join the warps that share rows: everyone stores (m, l, o), then the block's threads add them up
        attn_group_sync(group, THREADS);
        float* jo = reinterpret_cast<float*>(smem);           // [warp][16][D]
        float2* jm = reinterpret_cast<float2*>(jo + RW * KW * 16 * D);  // [warp][16]
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = r4 + 8 * i;
#pragma unroll
            for (int d = 0; d < DT; ++d)
                *reinterpret_cast<float2*>(jo + (warp * 16 + r) * D + d * 8 + 2 * c4) = make_float2(o[d][2 * i], o[d][2 * i + 1]);
            if (c4 == 0) jm[warp * 16 + r] = make_float2(m[i], l[i]);
        }
        attn_group_sync(group, THREADS);
        constexpr int PER = 4;                                 // channels per thread and step
        for (int j = tid; j < RW * 16 * (D / PER); j += THREADS) {
            const int r = j / (D / PER), d = (j % (D / PER)) * PER;
            const int rr = u.row0 + r;
            if (rr >= u.rows) continue;
            const int w0 = (r >> 4) * KW;
            float2 ml[KW];
            float mm = -INFINITY;
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                ml[w] = jm[(w0 + w) * 16 + (r & 15)];
                mm = fmaxf(mm, ml[w].x);
            }
            const float z = mm == -INFINITY ? 0.0f : mm;
            float ll = 0.0f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                const float f = exp2_fast(ml[w].x - z);
                ll += f * ml[w].y;
                const float4 x = *reinterpret_cast<const float4*>(jo + ((w0 + w) * 16 + (r & 15)) * D + d);
                acc.x += f * x.x; acc.y += f * x.y; acc.z += f * x.z; acc.w += f * x.w;
            }
            const int tok = rr / p.group;
            const int64_t at = (u.token0 + tok) * p.hq + u.head * p.group + (rr - tok * p.group);
            if (p.parts == 1) {
                const float inv = ll > 0.0f ? 1.0f / ll : 0.0f;
                T* dst = static_cast<T*>(p.out) + at * D + d;
                if constexpr (F32) {
                    *reinterpret_cast<float4*>(dst) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
                } else {
                    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
                }
            } else {
                const int64_t slot = static_cast<int64_t>(u.part) * p.T * p.hq + at;
                *reinterpret_cast<float4*>(p.part_o + slot * D + d) = acc;
                if (d == 0) p.part_ml[slot] = make_float2(mm, ll);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (row[i] >= u.rows) continue;
            const int tok = row[i] / p.group;
            const int64_t at = (u.token0 + tok) * p.hq + u.head * p.group + (row[i] - tok * p.group);
            if (p.parts == 1) {
                const float inv = l[i] > 0.0f ? 1.0f / l[i] : 0.0f;
                T* dst = static_cast<T*>(p.out) + at * D + 2 * c4;
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    if constexpr (F32)
                        *reinterpret_cast<float2*>(dst + d * 8) = make_float2(o[d][2 * i] * inv, o[d][2 * i + 1] * inv);
                    else
                        *reinterpret_cast<uint32_t*>(dst + d * 8) = pack_bf16x2(o[d][2 * i] * inv, o[d][2 * i + 1] * inv);
                }
            } else {
                const int64_t slot = static_cast<int64_t>(u.part) * p.T * p.hq + at;
#pragma unroll
                for (int d = 0; d < DT; ++d)
                    *reinterpret_cast<float2*>(p.part_o + slot * D + d * 8 + 2 * c4) = make_float2(o[d][2 * i], o[d][2 * i + 1]);
                if (c4 == 0) p.part_ml[slot] = make_float2(m[i], l[i]);
            }
        }
    }
}

template <typename T, int D>
__device__ __forceinline__ void attn_block_rw(int rw, const AttnParams& p, const AttnUnit& u, unsigned char* smem) {
    if (rw == 1) attn_block<T, D, 1>(p, u, smem);
    else if (rw == 2) attn_block<T, D, 2>(p, u, smem);
    else attn_block<T, D, 4>(p, u, smem);
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

// keys [key0, key1) of part `s` of `splits`, in whole tiles
__device__ __forceinline__ void attn_part(int keys, int tile, int splits, int s, int& key0, int& key1) {
    const int tiles = (keys + tile - 1) / tile;
    const int per = (tiles + splits - 1) / splits;
    const int64_t a = static_cast<int64_t>(s) * per * tile, e = a + static_cast<int64_t>(per) * tile;
    key0 = a < keys ? static_cast<int>(a) : keys;
    key1 = e < keys ? static_cast<int>(e) : keys;
}

// Prefix and own pages in one launch: blocks below prefix_blocks take the prefix.
template <typename T, int D>
__global__ void __launch_bounds__(kAttnThreads)
attn_prefix_kernel(const AttnParams p) {
    extern __shared__ __align__(128) unsigned char smem_attn[];
    constexpr int KEYS = AttnRow<T, D>::BLOCK_KEYS;
    const int prefix_units = p.prefix_splits * p.prefix_row_tiles * p.hkv;
    const int prefix_groups = attn_groups(p.prefix_rw);
    const int prefix_blocks = (prefix_units + prefix_groups - 1) / prefix_groups;
    AttnUnit u;
    int b = blockIdx.x;
    grid_launch_dependents();
    if (b < prefix_blocks) {
        b = b * prefix_groups + static_cast<int>(threadIdx.x) / (kAttnThreads / prefix_groups);
        if (b >= prefix_units) return;
        u.part = b % p.prefix_splits;
        b /= p.prefix_splits;
        u.row0 = (b % p.prefix_row_tiles) * 16 * p.prefix_rw;
        u.head = b / p.prefix_row_tiles;
        u.token0 = 0;
        u.rows = static_cast<int>(p.T) * p.group;
        u.ids = p.prefix_pages;
        u.table = nullptr;
        const int keys = static_cast<int>(p.prefix_len);
        u.list = (keys + (1 << p.page_shift) - 1) >> p.page_shift;
        attn_part(keys, KEYS, p.prefix_splits, u.part, u.key0, u.key1);
        u.limit0 = keys;
        u.step = 0;
        attn_block_rw<T, D>(p.prefix_rw, p, u, smem_attn);
        return;
    }
    const bool last_block = blockIdx.x == gridDim.x - 1;
    const int own_groups = attn_groups(p.own_rw);
    b = (b - prefix_blocks) * own_groups + static_cast<int>(threadIdx.x) / (kAttnThreads / own_groups);
    const int split = b % p.own_splits;
    b /= p.own_splits;
    u.part = (p.parts - p.own_splits) + split;
    u.row0 = (b % p.own_row_tiles) * 16 * p.own_rw;
    b /= p.own_row_tiles;
    u.head = b % p.hkv;
    const int seq = b / p.hkv;
    if (seq < p.B) {
        // the table's row is wanted as soon as the length is known: fetch it meanwhile
        u.ids = p.page_table + static_cast<int64_t>(seq) * p.table_width;
        const int ahead = (static_cast<int>(threadIdx.x) & 31) * 32;
        if (ahead < p.table_width) asm volatile("prefetch.global.L1 [%0];" ::"l"(u.ids + ahead));
    }
    int count = 0;
    if (seq < p.B) attn_tokens(p, seq, u.token0, count);
    u.rows = count * p.group;
    if (u.row0 >= u.rows) {
        if (last_block) grid_dependency_wait();
        return;
    }
    const int keys = attn_length(p, seq);
    u.table = nullptr;
    u.list = (keys + (1 << p.page_shift) - 1) >> p.page_shift;
    // the block's last row sees the most: nothing beyond its place is read
    u.limit0 = keys - count + 1;
    u.step = 1;
    const int last_tok = (min(u.rows, u.row0 + 16 * p.own_rw) - 1) / p.group;
    attn_part(keys, KEYS, p.own_splits, split, u.key0, u.key1);
    u.key1 = max(u.key0, min(u.key1, u.limit0 + last_tok));
    attn_block_rw<T, D>(p.own_rw, p, u, smem_attn);
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

// Chosen pages: one token and key head (and a part of the list) per block.
template <typename T, int D>
__global__ void __launch_bounds__(kAttnThreads)
attn_chosen_kernel(const AttnParams p) {
    extern __shared__ __align__(128) unsigned char smem_attn[];
    constexpr int KEYS = AttnRow<T, D>::BLOCK_KEYS;
    AttnUnit u;
    grid_dependency_wait();  // the list comes from the kernel before
    grid_launch_dependents();
    const int groups = attn_groups(p.own_rw);
    int64_t b = static_cast<int64_t>(blockIdx.x) * groups + static_cast<int>(threadIdx.x) / (kAttnThreads / groups);
    u.part = static_cast<int>(b % p.own_splits);
    b /= p.own_splits;
    u.row0 = static_cast<int>(b % p.own_row_tiles) * 16 * p.own_rw;
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
    const int page = static_cast<int>(place >> p.page_shift);
    u.list = place < 0 ? 0 : min(p.select, page + 1);
    const int keys = place < 0 ? 0 : ((u.list - 1) << p.page_shift) + static_cast<int>(place & ((1 << p.page_shift) - 1)) + 1;
    attn_part(keys, KEYS, p.own_splits, u.part, u.key0, u.key1);
    u.limit0 = keys;
    u.step = 0;
    attn_block_rw<T, D>(p.own_rw, p, u, smem_attn);
}

// Joins the parts of each row: out = sum_s exp(m_s - m) o_s / sum_s exp(m_s - m) l_s.  One warp per row, lanes
// over the channels; the parts' statistics are read by the lanes at once.
template <typename T, int D>
__global__ void __launch_bounds__(128)
attn_join_kernel(const float2* __restrict__ ml, const float* __restrict__ po, T* __restrict__ out, int64_t rows, int parts) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5);
    if (row >= rows) return;
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
        const int n = min(32, parts - s0);
#pragma unroll 4
        for (int s = 0; s < n; ++s) {
            const float w = __shfl_sync(kFullMask, f, s);
            // a part that holds no key of this row has weight 0 and its product is 0
            if (lane * PER < D) {
                const float4 x = *reinterpret_cast<const float4*>(po + ((s0 + s) * rows + row) * D + lane * PER);
                acc.x += w * x.x; acc.y += w * x.y; acc.z += w * x.z; acc.w += w * x.w;
            }
        }
    }
#pragma unroll
    for (int i = 16; i; i >>= 1) l += __shfl_xor_sync(kFullMask, l, i);
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    if (lane * PER < D) {
        T* dst = out + row * D + lane * PER;
        if constexpr (std::is_same<T, float>::value)
            *reinterpret_cast<float4*>(dst) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
        else
            *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
    }
}

}  // namespace wht
