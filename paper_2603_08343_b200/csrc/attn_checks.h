// Argument checks shared by the C entry points of the serving attention.
#pragma once
#include "attn_host.h"

namespace wht_host {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t elem(int dtype) { return dtype == WHT_F32 ? 4 : 2; }

inline int page_shift_of(int32_t page) { return page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : page == 128 ? 7 : -1; }

// Rows of a strided [T x H x D] tensor start on 16-byte boundaries.  (The stride of a dimension of one may be anything.)
inline bool strides_ok(const void* p, int64_t st, int64_t sh, int64_t T, int32_t H, int dtype) {
    const int64_t unit = 16 / static_cast<int64_t>(elem(dtype));
    return aligned16(p) && (T == 1 || st % unit == 0) && (H == 1 || sh % unit == 0);
}

inline int check_shape(int64_t T, int32_t Hq, int32_t Hkv, int32_t D, int64_t num_pages, int32_t page, int dtype) {
    if (dtype != WHT_F32 && dtype != WHT_BF16) return WHT_ERR_BAD_DTYPE;
    if (D != 64 && D != 96 && D != 128) return WHT_ERR_BAD_DIM;
    if (Hkv < 1 || Hq < Hkv || Hq % Hkv != 0 || Hq / Hkv > 64 || Hq > 65536) return WHT_ERR_BAD_DIM;
    // (tiled copies count a cache's rows in 31 bits; one of more rows would not fit the device's memory)
    if (page_shift_of(page) < 0 || num_pages < 0 || num_pages > 0x7fffffff / page / Hkv) return WHT_ERR_BAD_DIM;
    if (T < 0 || T * Hq > 0x7fffffff) return WHT_ERR_BAD_T;
    return WHT_OK;
}

// Keys of a list are counted in 31 bits, and the kernels round counts up to whole tiles: some room is left above the longest list.
constexpr int64_t kMostKeys = 0x7fffff00;

inline int check_batch(int64_t T, int32_t B, int32_t max_q_len, int32_t table_width, int32_t page, bool ragged) {
    if (B < 0 || max_q_len < 1 || table_width < 0 || static_cast<int64_t>(table_width) * page > kMostKeys) return WHT_ERR_BAD_DIM;
    if (max_q_len > (1 << 20) || (!ragged && (T != B || max_q_len != 1)) || (T > 0 && B == 0)) return WHT_ERR_BAD_T;
    return WHT_OK;
}

}  // namespace wht_host
