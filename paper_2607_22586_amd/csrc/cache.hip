// Paged cache on gfx950: rows written into pages, quantised on the way
// (mmshiftkv_cache_write), and read back (mmshiftkv_cache_read).  Both are
// bound by HBM: a row is read and written once, its scale is formed from the
// registers that hold it.  A group of d / 8 lanes has one row of K and of V,
// eight values each, so that a row's largest value is a maximum over the group,
// by lane moves without LDS.  What is written is stored past the caches (two
// prompts of 32768 rows of 8 heads, 407 MB: 82 -> 78 us; 65536 rows of 4 heads
// read back, 194 MB: 41 -> 29 us with the pages still in the memory-side cache);
// several rows per group, and loads past the caches, were no faster.
#include "pages.hpp"

namespace mmskv {
namespace {

constexpr int kCacheThreads = 256;

typedef float f32x4 __attribute__((ext_vector_type(4)));
template <typename V>
__device__ __forceinline__ void put(void* p, V x) {
    __builtin_nontemporal_store(x, static_cast<V*>(p));
}

// Eight values of a source row in fp32.
template <bool F32>
__device__ __forceinline__ void load8(const void* base, int64_t elem, float (&x)[8]) {
    if constexpr (F32) {
        const f32x4 a = *reinterpret_cast<const f32x4*>(static_cast<const float*>(base) + elem);
        const f32x4 b = *reinterpret_cast<const f32x4*>(static_cast<const float*>(base) + elem + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = a[j], x[4 + j] = b[j];
    } else {
        const u32x4 r = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(base) + elem);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[2 * j] = __uint_as_float(r[j] << 16);
            x[2 * j + 1] = __uint_as_float(r[j] & 0xFFFF0000u);
        }
    }
}

// The larger of two magnitudes.  An e4m3 row holds its NaN in their places and the
// scale is of the others; int8 has no place for one, so that its scale is to be NaN:
// as whole numbers NaN is above infinity.
template <int TYPE>
__device__ __forceinline__ float larger(float x, float y) {
    if constexpr (TYPE == kCacheI8) return __uint_as_float(max(__float_as_uint(x), __float_as_uint(y)));
    else return fmaxf(x, y);
}

// Largest of groups of 8 or 16 lanes: neighbours, pairs, then mirrored quads and
// octets.
template <int TYPE, int LANES>
__device__ __forceinline__ float group_max(float x) {
    const auto moved = [](float v, auto ctrl) {
        const int b = static_cast<int>(__float_as_uint(v));
        return __uint_as_float(static_cast<uint32_t>(__builtin_amdgcn_update_dpp(b, b, decltype(ctrl)::value, 0xF, 0xF, false)));
    };
    x = larger<TYPE>(x, moved(x, Constant<0xB1>{}));     // quad_perm [1, 0, 3, 2]
    x = larger<TYPE>(x, moved(x, Constant<0x4E>{}));     // quad_perm [2, 3, 0, 1]
    x = larger<TYPE>(x, moved(x, Constant<0x141>{}));    // row_half_mirror
    if constexpr (LANES == 16) x = larger<TYPE>(x, moved(x, Constant<0x140>{}));     // row_mirror
    return x;
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
        a = a < 0x1p-100f ? 0x1p-100f : a;       // (the inverse stays finite, a row of zeros is zero; NaN stays)
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
        put(static_cast<uint16_t*>(pool) + (row * LANES + lane) * 8, y);
    } else {
        float a = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) a = larger<TYPE>(a, fabsf(x[j]));
        a = group_max<TYPE, LANES>(a);
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
        put(static_cast<uint8_t*>(pool) + (row * LANES + lane) * 8, y);
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

// The two groups of four values that a lane reads back start kApart values apart:
// next to each other for bf16, which stores them as 16 bytes, half a row for fp32,
// so that the lanes' 16 bytes of each store lie side by side (32 adjacent bytes a
// lane leave every store with gaps: 4 x 8 heads of 16384 keys of 128, e4m3, 145 us
// against 124, 5.4 TB/s; 8 x 8 heads of 8192 keys of 64, 106 us against 51).
template <int D, bool F32>
constexpr int kApart = F32 ? D / 2 : 4;

// Eight cached values times their scale.
template <int D, int TYPE, bool F32>
__device__ __forceinline__ void load_row(const void* pool, const float* scales, int64_t row, int lane, float (&x)[8]) {
    const int64_t e = row * D + (F32 ? 4 : 8) * lane;
    if constexpr (TYPE == kCacheBf16) {
        if constexpr (F32) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint16_t* p = static_cast<const uint16_t*>(pool) + e + h * kApart<D, F32>;
                const u32x2 r = *reinterpret_cast<const u32x2*>(p);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    x[4 * h + 2 * j] = __uint_as_float(r[j] << 16);
                    x[4 * h + 2 * j + 1] = __uint_as_float(r[j] & 0xFFFF0000u);
                }
            }
        } else {
            load8<false>(pool, e, x);
        }
    } else {
        uint32_t w[2];
        const uint8_t* p = static_cast<const uint8_t*>(pool) + e;
        if constexpr (F32) {
            w[0] = *reinterpret_cast<const uint32_t*>(p);
            w[1] = *reinterpret_cast<const uint32_t*>(p + kApart<D, F32>);
        } else {
            const u32x2 r = *reinterpret_cast<const u32x2*>(p);
            w[0] = r[0], w[1] = r[1];
        }
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

template <int D, bool F32>
__device__ __forceinline__ void store8(void* base, int64_t row, int lane, const float (&x)[8]) {
    if constexpr (F32) {
        float* p = static_cast<float*>(base) + row + 4 * lane;
        put(p, f32x4{x[0], x[1], x[2], x[3]});
        put(p + kApart<D, F32>, f32x4{x[4], x[5], x[6], x[7]});
    } else {
        u32x4 y;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = pack_bf16(x[2 * j], x[2 * j + 1]);
        put(static_cast<uint16_t*>(base) + row + 8 * lane, y);
    }
}

template <int D, int TYPE, bool F32>
__global__ void __launch_bounds__(kCacheThreads) cache_read_kernel(CacheReadArgs a) {
    constexpr int LANES = D / 8;
    const int lane = threadIdx.x % LANES;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * (kCacheThreads / LANES) + threadIdx.x / LANES;
    const int c = blockIdx.y, b = blockIdx.z;
    if (t >= a.T) return;
    float k[8] = {}, v[8] = {};
    if (t < min(a.lens[static_cast<int64_t>(b) * a.Hkv + c], a.pages.cap)) {
        const int id = page_of(a.pages, b, static_cast<int>(t));
        if (id >= 0) {
            const int64_t row = pool_row(a.pages, a.Hkv, c, id, static_cast<int>(t));
            load_row<D, TYPE, F32>(a.pages.k, a.pages.k_scale, row, lane, k);
            load_row<D, TYPE, F32>(a.pages.v, a.pages.v_scale, row, lane, v);
        }
    }
    store8<D, F32>(a.k, b * a.ksb + c * a.ksh + t * a.kst, lane, k);
    store8<D, F32>(a.v, b * a.vsb + c * a.vsh + t * a.vst, lane, v);
}

// A group of lanes for each row of each head.
dim3 row_grid(int rows, int d, int Hkv, int B) {
    const int per = kCacheThreads / (d / 8);
    return dim3(static_cast<unsigned>((static_cast<int64_t>(rows) + per - 1) / per), Hkv, B);
}

// The kernel's type and row size as constants.
template <typename F>
void with_type(int d, int type, F&& run) {
    const auto at = [&](auto t) {
        if (d == 64) run(Constant<64>{}, t);
        else run(Constant<128>{}, t);
    };
    if (type == kCacheBf16) at(Constant<kCacheBf16>{});
    else if (type == kCacheE4m3) at(Constant<kCacheE4m3>{});
    else at(Constant<kCacheI8>{});
}

}  // namespace

hipError_t launch_cache_write(const CacheWriteArgs& a, hipStream_t s) {
    with_type(a.d, a.pages.dtype, [&](auto d, auto type) {
        constexpr int D = decltype(d)::value, TYPE = decltype(type)::value;
        const dim3 grid = row_grid(a.n, a.d, a.Hkv, a.B);
        if (a.dtype == 0) hipLaunchKernelGGL((cache_write_kernel<D, TYPE, true>), grid, dim3(kCacheThreads), 0, s, a);
        else hipLaunchKernelGGL((cache_write_kernel<D, TYPE, false>), grid, dim3(kCacheThreads), 0, s, a);
    });
    return hipGetLastError();
}

hipError_t launch_cache_read(const CacheReadArgs& a, hipStream_t s) {
    with_type(a.d, a.pages.dtype, [&](auto d, auto type) {
        constexpr int D = decltype(d)::value, TYPE = decltype(type)::value;
        const dim3 grid = row_grid(a.T, a.d, a.Hkv, a.B);
        if (a.dtype == 0) hipLaunchKernelGGL((cache_read_kernel<D, TYPE, true>), grid, dim3(kCacheThreads), 0, s, a);
        else hipLaunchKernelGGL((cache_read_kernel<D, TYPE, false>), grid, dim3(kCacheThreads), 0, s, a);
    });
    return hipGetLastError();
}

}  // namespace mmskv
