// Device helpers of the paged-cache kernels: where a cached row lies, and the
// types that it is held in.
#pragma once

#include "common.hpp"
#include "kernels.hpp"

namespace mmskv {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float floatx2_t __attribute__((ext_vector_type(2)));

constexpr int kCacheBf16 = 1, kCacheE4m3 = 2, kCacheI8 = 3;   // mmskv_dtype

template <int N>
struct Constant {                          // a number as a type, for generic lambdas
    static constexpr int value = N;
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

// Memory that stands for the rows of a page that is not there: 1 KB, what one
// load instruction of a wave fetches.
__device__ __attribute__((aligned(16))) const unsigned char kNoRows[1024] = {};

// 16 / 4 bytes per lane from memory to LDS (dst + 16 / 4 * lane); OFF is added
// to both addresses.  The 16 bytes are fetched as not to be used again (cached
// rows that one workgroup alone reads: 16 x 8 heads of 32768 rows 304 -> 272 us).
template <int OFF = 0>
__device__ __forceinline__ void load16_to_lds(const char* src, char* dst) {
    __builtin_amdgcn_global_load_lds(src, (__attribute__((address_space(3))) void*)dst, 16, OFF, 2);
}
__device__ __forceinline__ void load4_to_lds(const char* src, char* dst) {
    __builtin_amdgcn_global_load_lds(src, (__attribute__((address_space(3))) void*)dst, 4, 0, 0);
}

// s_waitcnt with vmcnt = N and the other counters not waited on
template <int N>
__device__ __forceinline__ void wait_vm() {
    static_assert(N < 64, "vmcnt field");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
}

// LDS address of a generic pointer into LDS, for the reads below.
__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)p));
}

// LDS reads of a wave's staged tiles, several at a time with their wait, from
// LDS address at[i] + OFF::at(i).  As plain reads or builtins they would wait for every
// load to LDS that is under way, the later stages' among them: the compiler does
// not see which bytes those write.  What they read has been waited for before.
template <class OFF>
__device__ __forceinline__ void read128(const uint32_t (&at)[8], u32x4 (&x)[8]) {
    asm volatile("ds_read_b128 %0, %8 offset:%16\n\tds_read_b128 %1, %9 offset:%17\n\t"
                 "ds_read_b128 %2, %10 offset:%18\n\tds_read_b128 %3, %11 offset:%19\n\t"
                 "ds_read_b128 %4, %12 offset:%20\n\tds_read_b128 %5, %13 offset:%21\n\t"
                 "ds_read_b128 %6, %14 offset:%22\n\tds_read_b128 %7, %15 offset:%23\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]),
                   "=&v"(x[7])
                 : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "v"(at[4]), "v"(at[5]), "v"(at[6]),
                   "v"(at[7]), "n"(OFF::at(0)), "n"(OFF::at(1)), "n"(OFF::at(2)), "n"(OFF::at(3)), "n"(OFF::at(4)),
                   "n"(OFF::at(5)), "n"(OFF::at(6)), "n"(OFF::at(7))
                 : "memory");
}
template <class OFF>
__device__ __forceinline__ void read64(const uint32_t (&at)[8], u32x2 (&x)[8]) {
    asm volatile("ds_read_b64 %0, %8 offset:%16\n\tds_read_b64 %1, %9 offset:%17\n\t"
                 "ds_read_b64 %2, %10 offset:%18\n\tds_read_b64 %3, %11 offset:%19\n\t"
                 "ds_read_b64 %4, %12 offset:%20\n\tds_read_b64 %5, %13 offset:%21\n\t"
                 "ds_read_b64 %6, %14 offset:%22\n\tds_read_b64 %7, %15 offset:%23\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]),
                   "=&v"(x[7])
                 : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "v"(at[4]), "v"(at[5]), "v"(at[6]),
                   "v"(at[7]), "n"(OFF::at(0)), "n"(OFF::at(1)), "n"(OFF::at(2)), "n"(OFF::at(3)), "n"(OFF::at(4)),
                   "n"(OFF::at(5)), "n"(OFF::at(6)), "n"(OFF::at(7))
                 : "memory");
}
// (two or four, at offset 0)
__device__ __forceinline__ void read128(const uint32_t (&at)[2], u32x4 (&x)[2]) {
    asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %3\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(x[0]), "=&v"(x[1])
                 : "v"(at[0]), "v"(at[1])
                 : "memory");
}
__device__ __forceinline__ void read128(const uint32_t (&at)[4], u32x4 (&x)[4]) {
    asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\t"
                 "ds_read_b128 %3, %7\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3])
                 : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3])
                 : "memory");
}
// Transposing reads.  16-bit: the 16 lanes of a group name four rows of 16
// columns (lane: row lane / 4, columns 4 (lane % 4) ..) and get column lane % 16
// of them; 8-bit: eight rows of 16 columns (row lane / 2, columns 8 (lane % 2) ..).
template <class OFF>
__device__ __forceinline__ void read_transposed16(const uint32_t (&at)[8], u32x2 (&x)[8]) {
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%16\n\tds_read_b64_tr_b16 %1, %9 offset:%17\n\t"
                 "ds_read_b64_tr_b16 %2, %10 offset:%18\n\tds_read_b64_tr_b16 %3, %11 offset:%19\n\t"
                 "ds_read_b64_tr_b16 %4, %12 offset:%20\n\tds_read_b64_tr_b16 %5, %13 offset:%21\n\t"
                 "ds_read_b64_tr_b16 %6, %14 offset:%22\n\tds_read_b64_tr_b16 %7, %15 offset:%23\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]),
                   "=&v"(x[7])
                 : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "v"(at[4]), "v"(at[5]), "v"(at[6]),
                   "v"(at[7]), "n"(OFF::at(0)), "n"(OFF::at(1)), "n"(OFF::at(2)), "n"(OFF::at(3)), "n"(OFF::at(4)),
                   "n"(OFF::at(5)), "n"(OFF::at(6)), "n"(OFF::at(7))
                 : "memory");
}
template <class OFF>
__device__ __forceinline__ void read_transposed8(const uint32_t (&at)[8], u32x2 (&x)[8]) {
    asm volatile("ds_read_b64_tr_b8 %0, %8 offset:%16\n\tds_read_b64_tr_b8 %1, %9 offset:%17\n\t"
                 "ds_read_b64_tr_b8 %2, %10 offset:%18\n\tds_read_b64_tr_b8 %3, %11 offset:%19\n\t"
                 "ds_read_b64_tr_b8 %4, %12 offset:%20\n\tds_read_b64_tr_b8 %5, %13 offset:%21\n\t"
                 "ds_read_b64_tr_b8 %6, %14 offset:%22\n\tds_read_b64_tr_b8 %7, %15 offset:%23\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]),
                   "=&v"(x[7])
                 : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "v"(at[4]), "v"(at[5]), "v"(at[6]),
                   "v"(at[7]), "n"(OFF::at(0)), "n"(OFF::at(1)), "n"(OFF::at(2)), "n"(OFF::at(3)), "n"(OFF::at(4)),
                   "n"(OFF::at(5)), "n"(OFF::at(6)), "n"(OFF::at(7))
                 : "memory");
}

// Page of row t of sequence b for a whole wave, by a scalar load (its wait is not
// that of the vector loads); -1 as page_of.
__device__ __forceinline__ int uniform_page(const Pages& p, int b, int t) {
    typedef const int __attribute__((address_space(4))) * ctable;
    const ctable row = (ctable)(p.table) + static_cast<int64_t>(b) * p.max_pages;
    const int j = t >> p.shift;
    const int id = row[min(j, p.max_pages - 1)];
    return j < p.max_pages && static_cast<uint32_t>(id) < static_cast<uint32_t>(p.n_pages) ? id : -1;
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
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = static_cast<float>(static_cast<int8_t>(w >> (8 * j)));
    }
}

// The same four as bf16 (both types fit it exactly); e4m3: times a power of two.
template <int TYPE>
__device__ __forceinline__ u32x2 widen4(uint32_t w, float scale = 1.f) {
    if constexpr (TYPE == kCacheE4m3) {
        return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true))};
    } else {
        float x[4];
        unpack4<TYPE>(w, x);
        return u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    }
}

}  // namespace mmskv
