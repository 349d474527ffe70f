// C ABI of the 4-bit cache (see include/wht_cache4.h): argument checks and launches.
#include "../../include/wht_cache4.h"

#include "attn_checks.h"
#include "cache4_append_kernels.cuh"
#include "cache4_attend_kernels.cuh"
#include "cache4_evict_kernels.cuh"
#include "cache4_host.h"

namespace {
using namespace wht_host;
using namespace wht_plan;
constexpr int64_t kMostEvictKeys = 1ll << 30;
}  // namespace

extern "C" {

int wht_kv_append4(const void* k, int64_t k_stride_t, int64_t k_stride_h, const void* v, int64_t v_stride_t, int64_t v_stride_h,
                   const void* q, int64_t q_stride_t, int64_t q_stride_h, void* q_out, const int64_t* slots,
                   const int32_t* positions, const float* cos_table, const float* sin_table, void* cache, int64_t T, int32_t Hq,
                   int32_t Hkv, int32_t D, int32_t rot, int32_t interleaved, int64_t max_pos, int64_t num_pages, int32_t page,
                   int dtype, void* stream) {
    int rc = check_shape(T, q ? Hq : Hkv, Hkv, D, num_pages, page, dtype);
    if (rc != WHT_OK) return rc;
    if (rot < 0 || rot > D || rot % 16 != 0 || (rot > 0 && max_pos < 1)) return WHT_ERR_BAD_DIM;
    if ((q == nullptr) != (q_out == nullptr)) return WHT_ERR_NULL;
    if (T == 0) return WHT_OK;
    if (!k || !v || !slots || !cache || (rot > 0 && (!positions || !cos_table || !sin_table))) return WHT_ERR_NULL;
    if (!strides_ok(k, k_stride_t, k_stride_h, T, Hkv, dtype) || !strides_ok(v, v_stride_t, v_stride_h, T, Hkv, dtype) ||
        (q && !strides_ok(q, q_stride_t, q_stride_h, T, Hq, dtype)) || !aligned16(q_out) || !aligned16(cache) || !aligned16(cos_table) ||
        !aligned16(sin_table))
        return WHT_ERR_MISALIGNED;
    wht::Append4Params p{};
    wht::AppendParams& a = p.a;
    a.k = k; a.v = v; a.q = q;
    a.k_st = k_stride_t; a.k_sh = k_stride_h;
    a.v_st = v_stride_t; a.v_sh = v_stride_h;
    a.q_st = q_stride_t; a.q_sh = q_stride_h;
    a.q_out = q_out;
    a.slots = slots; a.positions = positions; a.cos_t = cos_table; a.sin_t = sin_table;
    a.T = T; a.max_pos = max_pos; a.num_slots = num_pages * page;
    a.hq = q ? Hq : 0; a.hkv = Hkv; a.d = D; a.rot = rot; a.page_shift = page_shift_of(page);
    p.cache = static_cast<unsigned char*>(cache);
    return launch_append4(p, dtype, interleaved != 0, D, static_cast<cudaStream_t>(stream));
}

int wht_kv_read4(const void* cache, const int64_t* slots, void* k_out, void* v_out, int64_t n, int32_t Hkv, int32_t D,
                 int64_t num_pages, int32_t page, int dtype, void* stream) {
    const int rc = check_shape(n, Hkv, Hkv, D, num_pages, page, dtype);
    if (rc != WHT_OK) return rc;
    if (n == 0) return WHT_OK;
    if (!cache || !slots || !k_out || !v_out) return WHT_ERR_NULL;
    if (!aligned16(cache) || !aligned16(k_out) || !aligned16(v_out)) return WHT_ERR_MISALIGNED;
    const wht::Read4Params p{static_cast<const unsigned char*>(cache), slots, k_out, v_out, n, num_pages * page, Hkv, page_shift_of(page)};
    return launch_read4(p, dtype, D, static_cast<cudaStream_t>(stream));
}

size_t wht_attn_paged4_workspace_bytes(int32_t table_width, int64_t T, int32_t B, int32_t max_q_len, int32_t Hq, int32_t Hkv,
                                       int32_t D, int32_t page, int dtype, int32_t weigh) {
    int dev = 0, sms = 0;
    if (check_shape(T, Hq, Hkv, D, 0, page, dtype) != WHT_OK || check_batch(T, B, max_q_len, table_width, page, true) != WHT_OK ||
        device_info(&dev, &sms) != WHT_OK)
        return 0;
    return plan_attend4(table_width, T, B, max_q_len, Hq, Hkv, D, page, dtype, weigh != 0, sms).bytes;
}

int wht_attn_paged4(const void* q, int64_t q_stride_t, int64_t q_stride_h, const void* cache, const int32_t* page_table,
                    int32_t table_width, const int32_t* kv_lens, const int32_t* q_start, void* out, const float* weights,
                    float* weights_out, int64_t T, int32_t B, int32_t max_q_len, int32_t Hq, int32_t Hkv, int32_t D,
                    int64_t num_pages, int32_t page, float scale, int dtype, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_shape(T, Hq, Hkv, D, num_pages, page, dtype);
    if (rc == WHT_OK) rc = check_batch(T, B, max_q_len, table_width, page, q_start != nullptr);
    if (rc != WHT_OK) return rc;
    if (weights && !weights_out) return WHT_ERR_NULL;
    if (T == 0 && (!weights_out || B == 0 || table_width == 0)) return WHT_OK;
    if (!kv_lens || (table_width > 0 && !page_table) || (T > 0 && (!q || !cache || !out))) return WHT_ERR_NULL;
    if (!strides_ok(q, q_stride_t, q_stride_h, T, Hq, dtype) || !aligned16(cache) || !aligned16(out) || !aligned16(workspace) ||
        !aligned16(weights) || !aligned16(weights_out))
        return WHT_ERR_MISALIGNED;
    int dev = 0, sms = 0;
    rc = device_info(&dev, &sms);
    if (rc != WHT_OK) return rc;
    if (num_pages < 1) return WHT_ERR_BAD_DIM;
    const Attend4Plan f = plan_attend4(table_width, T, B, max_q_len, Hq, Hkv, D, page, dtype, weights_out != nullptr, sms);
    if (f.bytes > 0 && (!workspace || workspace_bytes < f.bytes)) return WHT_ERR_WORKSPACE;
    wht::Attn4Params p{};
    wht::AttnParams& a = p.a;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    a.q = q;
    a.q_st = q_stride_t; a.q_sh = q_stride_h;
    a.out = out;
    a.parts = 1;
    a.part_ml = reinterpret_cast<float2*>(ws);
    a.part_o = reinterpret_cast<float*>(ws + f.ml_bytes);
    a.page_table = page_table; a.kv_lens = kv_lens; a.q_start = q_start;
    a.table_width = table_width; a.B = B; a.max_q_len = max_q_len;
    a.T = T; a.num_pages = num_pages;
    a.hq = Hq; a.hkv = Hkv; a.group = Hq / Hkv; a.page_shift = page_shift_of(page);
    a.scale_log2 = scale * wht::kLog2e;
    p.cache = static_cast<const unsigned char*>(cache);
    p.warps = f.warps;
    p.least = f.least;
    p.grain = f.grain;
    p.part_rows = f.part_rows;
    p.lse = weights_out ? reinterpret_cast<float*>(ws + f.ml_bytes + up256(f.o_bytes)) : nullptr;
    p.scores = f.scores_bytes ? reinterpret_cast<float*>(ws + f.ml_bytes + up256(f.o_bytes) + f.lse_bytes) : nullptr;
    p.weights = weights;
    p.weights_out = weights_out;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (T > 0) {
        rc = f.umma ? launch_attend4_umma(p, D, dev, s)
             : dtype == WHT_F32 ? launch_attend4<float>(p, f.row_tiles, D, dev, s) : launch_attend4<__nv_bfloat16>(p, f.row_tiles, D, dev, s);
        if (rc != WHT_OK) return rc;
    }
    if (!weights_out) return WHT_OK;
    const bool few = static_cast<int64_t>(max_q_len) * a.group <= 8;
    return dtype == WHT_F32 ? launch_weigh4<float>(p, few, T > 0, D, dev, s) : launch_weigh4<__nv_bfloat16>(p, few, T > 0, D, dev, s);
}

int wht_kv_evict4(void* cache, const int32_t* page_table, int32_t table_width, const int32_t* kv_lens, const float* weights,
                  const int32_t* out_table, int32_t out_width, int32_t* lens_out, float* weights_out, int32_t* kept, int32_t B,
                  int32_t Hkv, int32_t D, int64_t num_pages, int32_t page, int32_t budget, int32_t keep_first, int32_t keep_last,
                  void* stream) {
    const int rc = check_shape(B, Hkv, Hkv, D, num_pages, page, WHT_BF16);
    if (rc != WHT_OK) return rc;
    if (table_width < 0 || static_cast<int64_t>(table_width) * page > kMostEvictKeys || out_width < 0 ||
        static_cast<int64_t>(out_width) * page > kMostEvictKeys || budget < 1 || budget > static_cast<int64_t>(out_width) * page ||
        keep_first < 0 || keep_last < 0 || static_cast<int64_t>(keep_first) + keep_last > budget)
        return WHT_ERR_BAD_DIM;
    if (B == 0) return WHT_OK;
    if (!cache || !kv_lens || !out_table || !lens_out || !weights_out || !kept || (table_width > 0 && (!page_table || !weights))) return WHT_ERR_NULL;
    if (!aligned16(cache) || !aligned16(weights) || !aligned16(weights_out)) return WHT_ERR_MISALIGNED;
    // (blocks read lengths and weights while others write theirs)
    if (lens_out == kv_lens || weights_out == weights || out_table == page_table) return WHT_ERR_BAD_DIM;
    wht::Evict4Params p{};
    wht::AttnParams& a = p.a;
    a.page_table = page_table; a.kv_lens = kv_lens;
    a.table_width = table_width; a.B = B;
    a.num_pages = num_pages;
    a.hkv = Hkv; a.page_shift = page_shift_of(page);
    p.cache = static_cast<unsigned char*>(cache);
    p.out_table = out_table; p.out_width = out_width;
    p.weights = weights; p.weights_out = weights_out;
    p.lens_out = lens_out; p.kept = kept;
    p.budget = budget; p.first = keep_first; p.last = keep_last;
    return launch_evict4(p, D, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
