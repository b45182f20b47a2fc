// Paged cache on gfx950: rows written into pages, quantised on the way
// (mmshiftkv_cache_write), and read back (mmshiftkv_cache_read).  Both are
// bound by HBM: a row is read and written once, its scale is formed from the
// registers that hold it.  A group of d / 8 lanes has one row of K and of V,
// eight values each, so that a row's largest value is a maximum over the group.
#include "pages.hpp"

namespace mmskv {
namespace {

constexpr int kCacheThreads = 256;

// Eight values of a source row in fp32.
template <bool F32>
__device__ __forceinline__ void load8(const void* base, int64_t elem, float (&x)[8]) {
    if constexpr (F32) {
        const float4 a = *reinterpret_cast<const float4*>(static_cast<const float*>(base) + elem);
        const float4 b = *reinterpret_cast<const float4*>(static_cast<const float*>(base) + elem + 4);
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
        const u32x4 r = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(base) + elem);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[2 * j] = __uint_as_float(r[j] << 16);
            x[2 * j + 1] = __uint_as_float(r[j] & 0xFFFF0000u);
        }
    }
}

// Scale of a row with largest value a, and what its values are multiplied by.
template <int TYPE>
__device__ __forceinline__ float row_scale(float a, float* mul) {
    if constexpr (TYPE == kCacheE4m3) {
        // a = 1.m * 2^(x - 127); 448 = 1.75 * 2^8: exponent x - 8, one more where 1.m > 1.75.
        // At least 2^-126, so that its inverse is in range too (biased exponents 1..254).
        const uint32_t bits = __float_as_uint(a);
        const int x = static_cast<int>(bits >> 23);
        const int e = max(x - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0), 1);
        *mul = __uint_as_float(static_cast<uint32_t>(254 - e) << 23);
        return __uint_as_float(static_cast<uint32_t>(e) << 23);
    } else {
        a = fmaxf(a, 0x1p-100f);                 // (the inverse stays finite, a row of zeros is zero)
        *mul = 127.f / a;
        return a / 127.f;
    }
}

// Eight values as the cache holds them, to element e of the pool; the row's
// scale by its first lane.
template <int TYPE, int LANES>
__device__ __forceinline__ void store_row(void* pool, float* scales, int64_t row, int lane, const float (&x)[8]) {
    if constexpr (TYPE == kCacheBf16) {
        u32x4 y;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = pack_bf16(x[2 * j], x[2 * j + 1]);
        *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(pool) + (row * LANES + lane) * 8) = y;
    } else {
        float a = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) a = fmaxf(a, fabsf(x[j]));
#pragma unroll
        for (int m = 1; m < LANES; m *= 2) a = fmaxf(a, __shfl_xor(a, m, LANES));
        float mul;
        const float scale = row_scale<TYPE>(a, &mul);
        u32x2 y;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            if constexpr (TYPE == kCacheE4m3) {
                int v = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * w] * mul, x[4 * w + 1] * mul, 0, false);
                y[w] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * w + 2] * mul, x[4 * w + 3] * mul, v, true);
            } else {
                // |x * mul| <= 127 (1 + 2^-22): rounds to 127 at most
                uint32_t v = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    v |= (static_cast<uint32_t>(static_cast<int>(rintf(x[4 * w + j] * mul))) & 255u) << (8 * j);
                y[w] = v;
            }
        }
        *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(pool) + (row * LANES + lane) * 8) = y;
        if (lane == 0) scales[row] = scale;
    }
}

template <int D, int TYPE, bool F32>
__global__ void __launch_bounds__(kCacheThreads) cache_write_kernel(CacheWriteArgs a) {
    constexpr int LANES = D / 8;
    const int lane = threadIdx.x % LANES;
    const int64_t j = static_cast<int64_t>(blockIdx.x) * (kCacheThreads / LANES) + threadIdx.x / LANES;
    const int c = blockIdx.y, b = blockIdx.z;
    const int64_t hc = static_cast<int64_t>(b) * a.Hkv + c;
    if (j >= (a.counts ? min(a.counts[hc], a.n) : a.n)) return;
    const int64_t t = j + (a.start ? a.start[hc] : 0);
    if (t < 0 || t >= a.pages.cap) return;
    const int id = page_of(a.pages, b, static_cast<int>(t));
    if (id < 0) return;
    const int64_t row = pool_row(a.pages, a.Hkv, c, id, static_cast<int>(t));
    const int src = a.idx ? a.idx[hc * a.n + j] : static_cast<int>(j);
    float k[8] = {}, v[8] = {};
    if (src >= 0 && src < a.T) {
        load8<F32>(a.k, b * a.ksb + c * a.ksh + src * a.kst + 8 * lane, k);
        load8<F32>(a.v, b * a.vsb + c * a.vsh + src * a.vst + 8 * lane, v);
    }
    store_row<TYPE, LANES>(a.pages.k, a.pages.k_scale, row, lane, k);
    store_row<TYPE, LANES>(a.pages.v, a.pages.v_scale, row, lane, v);
}

// Eight cached values times their scale, rounded once, to dst.
template <int TYPE, bool F32>
__device__ __forceinline__ void load_row(const void* pool, const float* scales, int64_t row, int lanes, int lane,
                                         float (&x)[8]) {
    const int64_t e = (row * lanes + lane) * 8;
    if constexpr (TYPE == kCacheBf16) {
        load8<false>(pool, e, x);
    } else {
        const u32x2 w = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(pool) + e);
        const float s = scales[row];
        float y[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            unpack4<TYPE>(w[h], y);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[4 * h + j] = y[j] * s;
        }
    }
}

template <bool F32>
__device__ __forceinline__ void store8(void* base, int64_t elem, const float (&x)[8]) {
    if constexpr (F32) {
        float* p = static_cast<float*>(base) + elem;
        *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        u32x4 y;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = pack_bf16(x[2 * j], x[2 * j + 1]);
        *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(base) + elem) = y;
    }
}

template <int D, int TYPE, bool F32>
__global__ void __launch_bounds__(kCacheThreads) cache_read_kernel(CacheReadArgs a) {
    constexpr int LANES = D / 8;
    const int lane = threadIdx.x % LANES;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * (kCacheThreads / LANES) + threadIdx.x / LANES;
    const int c = blockIdx.y, b = blockIdx.z;
    const int64_t hc = static_cast<int64_t>(b) * a.Hkv + c;
    if (t >= a.T) return;
    float k[8] = {}, v[8] = {};
    if (t < min(a.lens[hc], a.pages.cap)) {
        const int id = page_of(a.pages, b, static_cast<int>(t));
        if (id >= 0) {
            const int64_t row = pool_row(a.pages, a.Hkv, c, id, static_cast<int>(t));
            load_row<TYPE, F32>(a.pages.k, a.pages.k_scale, row, LANES, lane, k);
            load_row<TYPE, F32>(a.pages.v, a.pages.v_scale, row, LANES, lane, v);
        }
    }
    store8<F32>(a.k, b * a.ksb + c * a.ksh + t * a.kst + 8 * lane, k);
    store8<F32>(a.v, b * a.vsb + c * a.vsh + t * a.vst + 8 * lane, v);
}

template <int D, int TYPE>
void write_rows(const CacheWriteArgs& a, dim3 grid, hipStream_t s) {
    if (a.dtype == 0) hipLaunchKernelGGL((cache_write_kernel<D, TYPE, true>), grid, dim3(kCacheThreads), 0, s, a);
    else hipLaunchKernelGGL((cache_write_kernel<D, TYPE, false>), grid, dim3(kCacheThreads), 0, s, a);
}

template <int D, int TYPE>
void read_rows(const CacheReadArgs& a, dim3 grid, hipStream_t s) {
    if (a.dtype == 0) hipLaunchKernelGGL((cache_read_kernel<D, TYPE, true>), grid, dim3(kCacheThreads), 0, s, a);
    else hipLaunchKernelGGL((cache_read_kernel<D, TYPE, false>), grid, dim3(kCacheThreads), 0, s, a);
}

dim3 row_grid(int rows, int d, int Hkv, int B) {
    const int per = kCacheThreads / (d / 8);
    return dim3(static_cast<unsigned>((static_cast<int64_t>(rows) + per - 1) / per), Hkv, B);
}

}  // namespace

hipError_t launch_cache_write(const CacheWriteArgs& a, hipStream_t s) {
    const dim3 grid = row_grid(a.n, a.d, a.Hkv, a.B);
    const auto at = [&](auto type) {
        if (a.d == 64) write_rows<64, decltype(type)::value>(a, grid, s);
        else write_rows<128, decltype(type)::value>(a, grid, s);
    };
    if (a.pages.dtype == kCacheBf16) at(CacheType<kCacheBf16>{});
    else if (a.pages.dtype == kCacheE4m3) at(CacheType<kCacheE4m3>{});
    else at(CacheType<kCacheI8>{});
    return hipGetLastError();
}

hipError_t launch_cache_read(const CacheReadArgs& a, hipStream_t s) {
    const dim3 grid = row_grid(a.T, a.d, a.Hkv, a.B);
    const auto at = [&](auto type) {
        if (a.d == 64) read_rows<64, decltype(type)::value>(a, grid, s);
        else read_rows<128, decltype(type)::value>(a, grid, s);
    };
    if (a.pages.dtype == kCacheBf16) at(CacheType<kCacheBf16>{});
    else if (a.pages.dtype == kCacheE4m3) at(CacheType<kCacheE4m3>{});
    else at(CacheType<kCacheI8>{});
    return hipGetLastError();
}

}  // namespace mmskv
