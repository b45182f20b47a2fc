// Device helpers of the paged-cache kernels: where a cached row lies, and the
// types that it is held in.
#pragma once

#include "common.hpp"
#include "kernels.hpp"

namespace mmskv {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float floatx2_t __attribute__((ext_vector_type(2)));

constexpr int kCacheBf16 = 1, kCacheE4m3 = 2, kCacheI8 = 3;   // mmskv_dtype

template <int TYPE>
struct CacheType {
    static constexpr int value = TYPE;
};

template <int TYPE>
constexpr int kCacheBytes = TYPE == kCacheBf16 ? 2 : 1;

// Page of row t (>= 0) of sequence b, or -1: t behind the table, or an entry
// that names no page.
__device__ __forceinline__ int page_of(const Pages& p, int b, int t) {
    const int j = t >> p.shift;
    if (j >= p.max_pages) return -1;
    const int id = p.table[static_cast<int64_t>(b) * p.max_pages + j];
    return static_cast<uint32_t>(id) < static_cast<uint32_t>(p.n_pages) ? id : -1;
}

// Row number, in the pool seen as [n_pages * Hkv * page, d], of row t of head c
// on page id (in 64 bits: a pool may hold more than 2^31 rows).
__device__ __forceinline__ int64_t pool_row(const Pages& p, int Hkv, int c, int id, int t) {
    return ((static_cast<int64_t>(id) * Hkv + c) << p.shift) + (t & ((1 << p.shift) - 1));
}

// Four e4m3 / int8 values (one register) in fp32; exact.
template <int TYPE>
__device__ __forceinline__ void unpack4(uint32_t w, float (&x)[4]) {
    if constexpr (TYPE == kCacheE4m3) {
        const floatx2_t a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
        x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1];
    } else {
        // bytes + 128 are unsigned: one conversion instruction each
        w ^= 0x80808080u;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = static_cast<float>((w >> (8 * j)) & 255u) - 128.f;
    }
}

// The same four as bf16 (both types fit it exactly).
template <int TYPE>
__device__ __forceinline__ u32x2 widen4(uint32_t w) {
    if constexpr (TYPE == kCacheE4m3) {
        return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true))};
    } else {
        float x[4];
        unpack4<TYPE>(w, x);
        return u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    }
}

}  // namespace mmskv
