// Attention of a chunk of new tokens over a paged cache on gfx950.
//
// The Gh heads that share a KV head are rows of one problem: row r = i * Gh + g
// is query i of head g, so that a decoding step has Gh rows and a chunk Gh * n,
// and the cached rows are read once for all of them.  A workgroup of 4 waves
// has 128 rows of one (b, c), 32 per wave, and walks the keys in tiles of 64
// that are staged in LDS for all waves (8-bit values widened to bf16 there,
// which is exact).  One pass over the keys with the running maximum m and sum l
// of the softmax, base 2:
//   S^T = K Q^T   (v_mfma_f32_32x32x16_bf16: lane = query row, its values = keys,
//                  so the softmax runs within a lane and its other half-wave)
//   O^T = O^T 2^(m_old - m) + V^T P^T
// P^T is the second product's B operand as it stands in the registers of S^T
// (both products run over the keys in the order of the accumulator's rows); V^T
// comes from the staged rows by transposing LDS reads.
#include "pages.hpp"

namespace mmskv {
namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kRows = 32 * kWaves;         // query rows of a workgroup
constexpr int kKeys = 64;                  // keys of a tile
constexpr float kNone = -3e38f;            // running maximum before the first visible key

__device__ __forceinline__ floatx16 mfma32(bf16x8 a, bf16x8 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ float half_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float half_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Bytes from the start of a staged tile to 16-byte chunk ch of row r.  Rows
// without padding; the chunks of a row are permuted by its index, so that 16
// consecutive rows of one chunk (the reads of K) and four rows of 64 bytes (the
// transposing reads of V) both spread over all banks.
template <int D>
__device__ __forceinline__ int staged(int r, int ch) {
    const int swz = D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    return r * (2 * D) + 16 * (ch ^ swz);
}

template <int D, int TYPE>
__global__ void __launch_bounds__(kThreads, 2) chunk_kernel(ChunkArgs a) {
    constexpr int KC = D / 16;             // 16-dim steps of S
    constexpr int NT = D / 32;             // 32-dim tiles of O
    constexpr int CH = D / 8;              // 16-byte chunks (8 values) of a staged row
    constexpr int LD = kKeys * CH / kThreads;   // chunks of K (and of V) that a thread stages
    constexpr bool SCALED = TYPE != kCacheBf16;
    __shared__ __align__(16) char kt[kKeys * 2 * D];
    __shared__ __align__(16) char vt[kKeys * 2 * D];
    __shared__ __align__(16) float ksc[kKeys], vsc[kKeys];

    const int bc = blockIdx.x, b = bc / a.Hkv, c = bc - b * a.Hkv;
    const int r0 = static_cast<int>(gridDim.y - 1 - blockIdx.y) * kRows;
    const int split = blockIdx.z;
    const int tid = threadIdx.x, lane = lane_id();
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int half = lane >> 5;

    const int nq = a.q_counts ? min(max(a.q_counts[b], 0), a.n) : a.n;
    const int len = min(max(a.lens[bc], 0), a.max_len);
    // this lane's query row, and the last key that it sees (below 0: none)
    const int r = r0 + 32 * wave + (lane & 31);
    const int i = r / a.Gh, h = c * a.Gh + (r - i * a.Gh);
    const bool there = r < a.rows && i < nq;
    const int last = !there ? -1 : (a.causal ? len - nq + i : len - 1);
    // keys that the workgroup's rows see together, and this split's part of them
    const int i_end = min((min(r0 + kRows, a.rows) - 1) / a.Gh, nq - 1);
    const int end = i_end < r0 / a.Gh ? 0 : max(a.causal ? len - nq + i_end + 1 : len, 0);
    const int tiles = (end + kKeys - 1) / kKeys, per = (tiles + a.splits - 1) / a.splits;
    const int tile0 = split * per, tile1 = min(tile0 + per, tiles);

    bf16x8 qf[KC];
    {
        const uint16_t* q = a.q + b * a.qsb + h * a.qsh + i * a.qst + 8 * half;
#pragma unroll
        for (int kc = 0; kc < KC; ++kc) qf[kc] = there ? load_bf16x8(q + 16 * kc) : zero_bf16x8();
    }
    floatx16 o[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[t][j] = 0.f;
    float m = kNone, l = 0.f;

    for (int tile = tile0; tile < tile1; ++tile) {
        const int key0 = tile * kKeys;
        __syncthreads();                   // the previous tile has been read
#pragma unroll
        for (int j = 0; j < LD; ++j) {
            const int row = (tid + j * kThreads) / CH, ch = tid % CH, t = key0 + row;
            u32x4 kv = {0u, 0u, 0u, 0u}, vv = kv;
            float ks = 0.f, vs = 0.f;
            const int id = t < end ? page_of(a.pages, b, t) : -1;
            if (id >= 0) {
                const int64_t pr = pool_row(a.pages, a.Hkv, c, id, t);
                const int64_t e = (pr * CH + ch) * 8;
                if constexpr (SCALED) {
                    const u32x2 kr = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(a.pages.k) + e);
                    const u32x2 vr = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(a.pages.v) + e);
                    const u32x2 k0 = widen4<TYPE>(kr[0]), k1 = widen4<TYPE>(kr[1]);
                    const u32x2 v0 = widen4<TYPE>(vr[0]), v1 = widen4<TYPE>(vr[1]);
                    kv = u32x4{k0[0], k0[1], k1[0], k1[1]};
                    vv = u32x4{v0[0], v0[1], v1[0], v1[1]};
                    ks = a.pages.k_scale[pr];
                    vs = a.pages.v_scale[pr];
                } else {
                    kv = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.pages.k) + e);
                    vv = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.pages.v) + e);
                }
            }
            *reinterpret_cast<u32x4*>(kt + staged<D>(row, ch)) = kv;
            *reinterpret_cast<u32x4*>(vt + staged<D>(row, ch)) = vv;
            if (SCALED && ch == 0) ksc[row] = ks * a.scale, vsc[row] = vs;
        }
        __syncthreads();

        // value e of s[u] is key key0 + 32 u + 8 (e / 4) + 4 half + e % 4
        floatx16 s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[u][e] = 0.f;
#pragma unroll
            for (int kc = 0; kc < KC; ++kc) {
                const bf16x8 k = load_bf16x8(reinterpret_cast<const uint16_t*>(
                    kt + staged<D>(32 * u + (lane & 31), 2 * kc + half)));
                s[u] = mfma32(k, qf[kc], s[u]);
            }
        }
        float mx = kNone;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int row = 32 * u + 8 * (e >> 2) + 4 * half + (e & 3);
                float x = s[u][e] * (SCALED ? ksc[row] : a.scale);
                x = key0 + row <= last ? x : -INFINITY;
                s[u][e] = x;
                mx = fmaxf(mx, x);
            }
        mx = fmaxf(half_max(mx), m);
        const float f = fast_exp2(m - mx);
        m = mx;
        l *= f;
        bf16x8 p[4];                       // p[2 u + w]: values 8 w .. 8 w + 7 of s[u]
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                u32x4 y;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float x[2];
#pragma unroll
                    for (int z = 0; z < 2; ++z) {
                        const int e = 8 * w + 2 * j + z, row = 32 * u + 8 * (e >> 2) + 4 * half + (e & 3);
                        x[z] = fast_exp2(s[u][e] - m);
                        l += x[z];
                        if (SCALED) x[z] *= vsc[row];
                    }
                    y[j] = pack_bf16(x[0], x[1]);
                }
                p[2 * u + w] = __builtin_bit_cast(bf16x8, y);
            }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int j = 0; j < 16; ++j) o[t][j] *= f;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                // V^T: dims 32 t + lane % 32, keys 16 u + 4 half + {0..3, 8..11}
                typedef s16x4 __attribute__((address_space(3))) * lds4;
                u32x4 v;
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const int row = 16 * u + 8 * w + 4 * half + ((lane & 15) >> 2);
                    const int dim = 32 * t + (lane & 16) + 4 * (lane & 3);
                    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (lds4)(vt + staged<D>(row, dim >> 3) + 2 * (dim & 7)));
                    const u32x2 y = __builtin_bit_cast(u32x2, x);
                    v[2 * w] = y[0];
                    v[2 * w + 1] = y[1];
                }
                o[t] = mfma32(__builtin_bit_cast(bf16x8, v), p[u], o[t]);
            }
        }
    }
    l = half_sum(l);
    if (r >= a.rows) return;
    // value 4 w + j of o[t] is dim 32 t + 8 w + 4 half + j
    if (a.splits > 1) {
        const int64_t pr = (static_cast<int64_t>(split) * gridDim.x + bc) * a.rows + r;
        float* po = a.part_o + pr * D + 4 * half;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int w = 0; w < 4; ++w)
                *reinterpret_cast<float4*>(po + 32 * t + 8 * w) =
                    make_float4(o[t][4 * w], o[t][4 * w + 1], o[t][4 * w + 2], o[t][4 * w + 3]);
        if (half == 0) a.part_ml[pr] = make_float2(m, l);
        return;
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    uint16_t* out = a.out + b * a.osb + h * a.osh + i * a.ost + 4 * half;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int w = 0; w < 4; ++w)
            *reinterpret_cast<u32x2*>(out + 32 * t + 8 * w) =
                u32x2{pack_bf16(o[t][4 * w] * inv, o[t][4 * w + 1] * inv),
                      pack_bf16(o[t][4 * w + 2] * inv, o[t][4 * w + 3] * inv)};
}

// Joins the splits of a row: the largest m as reference, every sum rescaled to
// it.  A group of D / 8 lanes per row, 8 dims each.
template <int D>
__global__ void __launch_bounds__(256) chunk_join_kernel(ChunkArgs a) {
    constexpr int LANES = D / 8;
    const int lane = threadIdx.x % LANES;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (256 / LANES) + threadIdx.x / LANES;
    const int64_t heads = static_cast<int64_t>(a.B) * a.Hkv, rows = heads * a.rows;
    if (row >= rows) return;
    const int bc = static_cast<int>(row / a.rows), r = static_cast<int>(row - static_cast<int64_t>(bc) * a.rows);
    float m = kNone;
    for (int s = 0; s < a.splits; ++s) m = fmaxf(m, a.part_ml[s * rows + row].x);
    float l = 0.f, o[8] = {};
    for (int s = 0; s < a.splits; ++s) {
        const float2 ml = a.part_ml[s * rows + row];
        if (!(ml.y > 0.f)) continue;       // saw no key
        const float f = fast_exp2(ml.x - m);
        const float* po = a.part_o + (s * rows + row) * D + 8 * lane;
        const float4 x = *reinterpret_cast<const float4*>(po), y = *reinterpret_cast<const float4*>(po + 4);
        l = fmaf(ml.y, f, l);
        o[0] = fmaf(x.x, f, o[0]), o[1] = fmaf(x.y, f, o[1]), o[2] = fmaf(x.z, f, o[2]), o[3] = fmaf(x.w, f, o[3]);
        o[4] = fmaf(y.x, f, o[4]), o[5] = fmaf(y.y, f, o[5]), o[6] = fmaf(y.z, f, o[6]), o[7] = fmaf(y.w, f, o[7]);
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    const int b = bc / a.Hkv, c = bc - b * a.Hkv, i = r / a.Gh, h = c * a.Gh + (r - i * a.Gh);
    u32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = pack_bf16(o[2 * j] * inv, o[2 * j + 1] * inv);
    *reinterpret_cast<u32x4*>(a.out + b * a.osb + h * a.osh + i * a.ost + 8 * lane) = v;
}

constexpr int64_t kTarget = 2 * kPlanCus;  // workgroups that fill the chip
constexpr int kMaxSplits = 128;

template <int D>
hipError_t launch(const ChunkArgs& a, hipStream_t s) {
    const int tiles = (a.rows + kRows - 1) / kRows;
    const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(a.B) * a.Hkv), tiles, a.splits);
    if (a.pages.dtype == kCacheBf16) hipLaunchKernelGGL((chunk_kernel<D, kCacheBf16>), grid, dim3(kThreads), 0, s, a);
    else if (a.pages.dtype == kCacheE4m3)
        hipLaunchKernelGGL((chunk_kernel<D, kCacheE4m3>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((chunk_kernel<D, kCacheI8>), grid, dim3(kThreads), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    const int64_t rows = static_cast<int64_t>(a.B) * a.Hkv * a.rows;
    const int per = 256 / (D / 8);
    hipLaunchKernelGGL((chunk_join_kernel<D>), dim3(static_cast<unsigned>((rows + per - 1) / per)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

int chunk_splits(int64_t heads, int rows, int T) {
    const int64_t base = heads * ((rows + kRows - 1) / kRows);
    const int64_t want = (kTarget + base - 1) / base, most = (T + 255) / 256;
    const int64_t s = want < most ? want : most;
    return static_cast<int>(s < kMaxSplits ? s : kMaxSplits);
}

size_t chunk_workspace_bound(int64_t heads, int rows, int T, int d) {
    // splits * heads * rows: fewer than 2 kTarget workgroups have splits
    const int64_t most = static_cast<int64_t>(T) / 256 + 1 < kMaxSplits ? static_cast<int64_t>(T) / 256 + 1 : kMaxSplits;
    int64_t part = heads * rows;
    part = part > (2 * kTarget * kRows) / most ? 2 * kTarget * kRows : part * most;
    return static_cast<size_t>(part) * (d * sizeof(float) + sizeof(float2)) + 256;
}

hipError_t launch_chunk_attention(const ChunkArgs& a, hipStream_t s) {
    return a.d == 64 ? launch<64>(a, s) : launch<128>(a, s);
}

}  // namespace mmskv
