// C ABI of the serving attention (see include/wht_attention.h): argument checks and launches.
#include <algorithm>

#include "attn_checks.h"
#include "attn_plan.h"
#include "cache4_host.h"
#include "kv_append_kernels.cuh"
#include "select_kernels.cuh"

namespace {

using namespace wht_host;
using namespace wht_plan;
using wht::AppendParams;
using wht::AttnParams;
using wht::SelectParams;
using wht::UmmaAttnParams;

void set_parts(AttnParams& p, unsigned char* at, int64_t rows) {
    if (p.parts <= 1) return;
    p.part_ml = reinterpret_cast<float2*>(at);
    p.part_o = reinterpret_cast<float*>(at + up256(static_cast<size_t>(rows) * p.parts * sizeof(float2)));
}

int join(const AttnParams& p, int dtype, int32_t D, cudaStream_t s) {
    if (p.parts <= 1) return WHT_OK;
    return dtype == WHT_F32 ? launch_attn_join<float>(p, D, s) : launch_attn_join<__nv_bfloat16>(p, D, s);
}

}  // namespace

extern "C" {

int wht_kv_append(const void* k, int64_t k_stride_t, int64_t k_stride_h, const void* v, int64_t v_stride_t, int64_t v_stride_h,
                  const void* q, int64_t q_stride_t, int64_t q_stride_h, void* q_out, const int64_t* slots,
                  const int32_t* positions, const float* cos_table, const float* sin_table, void* k_cache, void* v_cache,
                  int8_t* summary, const float* summary_scale, int64_t T, int32_t Hq, int32_t Hkv, int32_t D, int32_t rot,
                  int32_t interleaved, int64_t max_pos, int64_t num_pages, int32_t page, int dtype, void* stream) {
    int rc = check_shape(T, q ? Hq : Hkv, Hkv, D, num_pages, page, dtype);
    if (rc != WHT_OK) return rc;
    if (rot < 0 || rot > D || rot % 16 != 0 || (rot > 0 && max_pos < 1)) return WHT_ERR_BAD_DIM;
    if ((q == nullptr) != (q_out == nullptr)) return WHT_ERR_NULL;
    if (T == 0) return WHT_OK;
    if (!k || !v || !slots || !k_cache || !v_cache) return WHT_ERR_NULL;
    if (rot > 0 && (!positions || !cos_table || !sin_table)) return WHT_ERR_NULL;
    if (summary && !summary_scale) return WHT_ERR_NULL;
    if (!strides_ok(k, k_stride_t, k_stride_h, T, Hkv, dtype) || !strides_ok(v, v_stride_t, v_stride_h, T, Hkv, dtype) ||
        (q && !strides_ok(q, q_stride_t, q_stride_h, T, Hq, dtype)) || !aligned16(q_out) || !aligned16(k_cache) || !aligned16(v_cache) ||
        !aligned16(summary) || !aligned16(cos_table) || !aligned16(sin_table))
        return WHT_ERR_MISALIGNED;
    int dev = 0, sms = 0;
    rc = device_info(&dev, &sms);
    if (rc != WHT_OK) return rc;
    AppendParams p{};
    p.k = k; p.v = v; p.q = q;
    p.k_st = k_stride_t; p.k_sh = k_stride_h;
    p.v_st = v_stride_t; p.v_sh = v_stride_h;
    p.q_st = q_stride_t; p.q_sh = q_stride_h;
    p.q_out = q_out; p.k_cache = k_cache; p.v_cache = v_cache;
    p.slots = slots; p.positions = positions; p.cos_t = cos_table; p.sin_t = sin_table;
    p.summary = summary; p.summary_scale = summary_scale;
    p.T = T; p.max_pos = max_pos; p.num_slots = num_pages * page;
    p.hq = q ? Hq : 0; p.hkv = Hkv; p.d = D; p.rot = rot; p.page_shift = page_shift_of(page);
    return launch_append(p, dtype, interleaved != 0, static_cast<cudaStream_t>(stream));
}

size_t wht_attn_prefix_workspace_bytes(int64_t prefix_len, int32_t table_width, int64_t T, int32_t B, int32_t max_q_len, int32_t Hq,
                                       int32_t Hkv, int32_t D, int32_t page, int dtype) {
    int dev = 0, sms = 0;
    if (check_shape(T, Hq, Hkv, D, 0, page, dtype) != WHT_OK || check_batch(T, B, max_q_len, table_width, page, true) != WHT_OK ||
        prefix_len < 0 || prefix_len > kMostKeys || device_info(&dev, &sms) != WHT_OK)
        return 0;
    // either form of the prefix may be taken (the tcgen05 one has conditions that are not known here)
    return std::max(plan_prefix(prefix_len, table_width, T, B, max_q_len, Hq, Hkv, D, page, dtype, true, sms).bytes,
                    plan_prefix(prefix_len, table_width, T, B, max_q_len, Hq, Hkv, D, page, dtype, false, sms).bytes);
}

int wht_attn_prefix(const void* q, int64_t q_stride_t, int64_t q_stride_h, const void* k_cache, const void* v_cache,
                    const int32_t* prefix_pages, int64_t prefix_len, const int32_t* page_table, int32_t table_width,
                    const int32_t* kv_lens, const int32_t* q_start, void* out, int64_t T, int32_t B, int32_t max_q_len,
                    int32_t Hq, int32_t Hkv, int32_t D, int64_t num_pages, int32_t page, float scale, int dtype,
                    void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_shape(T, Hq, Hkv, D, num_pages, page, dtype);
    if (rc == WHT_OK) rc = check_batch(T, B, max_q_len, table_width, page, q_start != nullptr);
    if (rc != WHT_OK) return rc;
    if (prefix_len < 0 || prefix_len > kMostKeys) return WHT_ERR_BAD_T;
    if (T == 0) return WHT_OK;
    if (!q || !k_cache || !v_cache || !out || !kv_lens || (table_width > 0 && !page_table) || (prefix_len > 0 && !prefix_pages))
        return WHT_ERR_NULL;
    if (!strides_ok(q, q_stride_t, q_stride_h, T, Hq, dtype) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out) || !aligned16(workspace))
        return WHT_ERR_MISALIGNED;
    int dev = 0, sms = 0;
    rc = device_info(&dev, &sms);
    if (rc != WHT_OK) return rc;
    if (num_pages < 1) return WHT_ERR_BAD_DIM;
    const bool umma_allowed = scale > 0.0f;  // the tcgen05 kernel finds a row's maximum before it scales
    const PrefixPlan f = plan_prefix(prefix_len, table_width, T, B, max_q_len, Hq, Hkv, D, page, dtype, umma_allowed, sms);
    if (f.bytes > 0 && (!workspace || workspace_bytes < f.bytes)) return WHT_ERR_WORKSPACE;
    AttnParams p{};
    p.q = q; p.k_cache = k_cache; p.v_cache = v_cache;
    p.q_st = q_stride_t; p.q_sh = q_stride_h;
    p.out = out;
    p.parts = f.parts;
    set_parts(p, static_cast<unsigned char*>(workspace), T * Hq);
    p.prefix_pages = prefix_pages; p.prefix_len = prefix_len;
    p.prefix_splits = f.prefix_splits; p.prefix_row_tiles = f.prefix_row_tiles; p.prefix_nr = f.prefix_nr; p.prefix_wpu = f.prefix_wpu;
    p.page_table = page_table; p.kv_lens = kv_lens; p.q_start = q_start;
    p.table_width = table_width; p.B = B; p.max_q_len = max_q_len;
    p.own_splits = f.own_splits; p.own_row_tiles = f.own_row_tiles; p.own_nr = f.own_nr; p.own_wpu = f.own_wpu;
    p.joint = f.joint;
    p.T = T; p.num_pages = num_pages;
    p.hq = Hq; p.hkv = Hkv; p.group = Hq / Hkv; p.page_shift = page_shift_of(page);
    p.scale_log2 = scale * wht::kLog2e;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (f.umma) {
        const UmmaAttnParams up{p, f.umma_splits, f.umma_row_blocks, f.same_rows};
        rc = launch_attn_umma_prefix(up, D, dev, s);
        if (rc != WHT_OK) return rc;
    }
    rc = dtype == WHT_F32 ? launch_attn_prefix<float>(p, D, dev, f.umma, s) : launch_attn_prefix<__nv_bfloat16>(p, D, dev, f.umma, s);
    return rc != WHT_OK ? rc : join(p, dtype, D, s);
}

size_t wht_attn_select_workspace_bytes(int32_t table_width, int32_t select, int64_t T, int32_t B, int32_t max_q_len, int32_t Hq,
                                       int32_t Hkv, int32_t D, int32_t page, int dtype) {
    int dev = 0, sms = 0;
    if (check_shape(T, Hq, Hkv, D, 0, page, dtype) != WHT_OK || check_batch(T, B, max_q_len, table_width, page, true) != WHT_OK ||
        select < 1 || select > 1024 || device_info(&dev, &sms) != WHT_OK)
        return 0;
    return plan_select(table_width, select, T, B, max_q_len, Hq, Hkv, D, page, dtype, sms).bytes;
}

int wht_attn_select(const void* q, int64_t q_stride_t, int64_t q_stride_h, const void* k_cache, const void* v_cache,
                    const int8_t* summary, const int32_t* page_table, int32_t table_width, const int32_t* kv_lens,
                    const int32_t* q_start, int32_t select, void* out, int32_t* pages_out, int64_t T, int32_t B,
                    int32_t max_q_len, int32_t Hq, int32_t Hkv, int32_t D, int64_t num_pages, int32_t page, float scale,
                    int dtype, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_shape(T, Hq, Hkv, D, num_pages, page, dtype);
    if (rc == WHT_OK) rc = check_batch(T, B, max_q_len, table_width, page, q_start != nullptr);
    if (rc != WHT_OK) return rc;
    if (select < 1 || select > 1024 || table_width > 49152) return WHT_ERR_BAD_DIM;
    if (T == 0) return WHT_OK;
    if (num_pages < 1) return WHT_ERR_BAD_DIM;
    if (!q || !k_cache || !v_cache || !summary || !out || !pages_out || !kv_lens || (table_width > 0 && !page_table)) return WHT_ERR_NULL;
    if (!strides_ok(q, q_stride_t, q_stride_h, T, Hq, dtype) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(summary) ||
        !aligned16(out) || !aligned16(workspace))
        return WHT_ERR_MISALIGNED;
    int dev = 0, sms = 0;
    rc = device_info(&dev, &sms);
    if (rc != WHT_OK) return rc;
    const SelectPlan f = plan_select(table_width, select, T, B, max_q_len, Hq, Hkv, D, page, dtype, sms);
    if (f.bytes > 0 && (!workspace || workspace_bytes < f.bytes)) return WHT_ERR_WORKSPACE;
    SelectParams sp{};
    AttnParams& p = sp.a;
    p.q = q; p.k_cache = k_cache; p.v_cache = v_cache;
    p.q_st = q_stride_t; p.q_sh = q_stride_h;
    p.out = out;
    p.parts = f.splits;
    set_parts(p, static_cast<unsigned char*>(workspace) + f.scores_bytes, T * Hq);
    p.page_table = page_table; p.kv_lens = kv_lens; p.q_start = q_start;
    p.table_width = table_width; p.B = B; p.max_q_len = max_q_len;
    p.own_splits = f.splits; p.own_row_tiles = f.row_tiles; p.own_nr = f.nr; p.own_wpu = f.wpu;
    p.chosen = pages_out; p.select = select;
    p.T = T; p.num_pages = num_pages;
    p.hq = Hq; p.hkv = Hkv; p.group = Hq / Hkv; p.page_shift = page_shift_of(page);
    p.scale_log2 = scale * wht::kLog2e;
    sp.summary = summary;
    sp.scores = f.one_kernel ? nullptr : static_cast<int32_t*>(workspace);
    sp.pages = pages_out;
    sp.stride = table_width;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    rc = launch_select(sp, f.one_kernel, dtype, D, s);
    if (rc == WHT_OK) rc = dtype == WHT_F32 ? launch_attn_chosen<float>(p, D, dev, s) : launch_attn_chosen<__nv_bfloat16>(p, D, dev, s);
    return rc != WHT_OK ? rc : join(p, dtype, D, s);
}

int wht_attn_device_status(void) {
    // the words are copied on the default stream, which other streams need not wait for, nor it for them
    WHT_CUDA_TRY(cudaDeviceSynchronize());
    unsigned any = 0;
    for (auto take : {take_attn_error_append, take_attn_error_paged_bf16, take_attn_error_paged_f32, take_attn_error_select,
                      take_attn_error_umma, take_attn_error_append4, take_attn_error_attend4_bf16, take_attn_error_attend4_f32,
                      take_attn_error_umma4, take_attn_error_evict4}) {
        unsigned flag = 0;
        const int rc = take(&flag);
        if (rc != WHT_OK) return rc;
        any |= flag;
    }
    for (auto take : {take_device_error_attn_umma, take_device_error_attn_paged_bf16, take_device_error_attn_paged_f32,
                      take_device_error_attend4_bf16, take_device_error_attend4_f32, take_device_error_umma4}) {
        unsigned waits = 0;
        const int rc = take(&waits);
        if (rc != WHT_OK) return rc;
        if (waits) any |= wht::kAttnErrWait;
    }
    return any & wht::kAttnErrIndex ? WHT_ERR_DEVICE_INDEX : any ? WHT_ERR_DEVICE_WAIT : WHT_OK;
}

}  // extern "C"
