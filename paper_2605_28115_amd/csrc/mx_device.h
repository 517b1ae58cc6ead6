// Elements and scales of the microscaled caches (OCP microscaling: e2m1 or e4m3 numbers, one power of two for 32 of them).
#pragma once

#include <utility>

#include "civic_internal.h"

namespace civic {

constexpr int kMxBlock = 32;                                  // channels of one scale
constexpr int64_t kMxMaxRows = int64_t{1} << 22;              // rows of a head: 32-bit offsets inside it, 256 bytes a row at most

typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 mx_bf16x8 __attribute__((ext_vector_type(8)));
typedef float mx_f32x2 __attribute__((ext_vector_type(2)));
typedef float mx_f32x4 __attribute__((ext_vector_type(4)));
typedef short mx_i16x2 __attribute__((ext_vector_type(2)));

// Whether the rows of head_dim elements of a written tensor [n0, n1, n2, head_dim] lie apart: from the smallest stride to the largest, each
// passes over all that the smaller ones span.  (Rows that share memory would be written by several threads at once.)
static inline bool mx_rows_apart(const int64_t* strides, int64_t n0, int64_t n1, int64_t n2, int32_t head_dim)
{
    int64_t stride[3] = {strides[0], strides[1], strides[2]}, n[3] = {n0, n1, n2};
    if (stride[0] > stride[1]) { std::swap(stride[0], stride[1]); std::swap(n[0], n[1]); }
    if (stride[1] > stride[2]) { std::swap(stride[1], stride[2]); std::swap(n[1], n[2]); }
    if (stride[0] > stride[1]) { std::swap(stride[0], stride[1]); std::swap(n[0], n[1]); }
    int64_t span = head_dim;
    for (int i = 0; i < 3; ++i) {
        if (n[i] <= 1) continue;
        if (stride[i] < span) return false;
        if (stride[i] > (INT64_MAX - span) / (n[i] - 1)) return false;
        span += stride[i] * (n[i] - 1);
    }
    return true;
}

static inline bool mx_format_ok(int format) { return format == CIVIC_MXFP4 || format == CIVIC_MXFP8; }

// Channels 2 i and 2 i + 1 of the words of a row as bf16, times the scale.  Exact: an element has at most four significant bits,
// and the scale is a power of two (the instruction takes the exponent field of `scale` alone; 255 there gives NaN).
template <int FMT>
__device__ __forceinline__ uint32_t mx_pair_bf16(const uint32_t* w, int i, float scale)
{
    mx_bf16x2 p;
    if constexpr (FMT == 4) {
        const uint32_t x = w[i >> 2];
        switch (i & 3) {
        case 0: p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 0); break;
        case 1: p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 1); break;
        case 2: p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 2); break;
        default: p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 3); break;
        }
    } else {
        const uint32_t x = w[i >> 1];
        p = (i & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, false);
    }
    return __builtin_bit_cast(uint32_t, p);
}

}  // namespace civic
