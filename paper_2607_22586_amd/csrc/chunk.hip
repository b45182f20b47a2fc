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
// What bounds it: the matrix pipe and the exponentials by turns, two waves a SIMD
// (d = 128: 238 registers for bf16 rows, 229 for e4m3, all 256 for int8, which keeps
// 48 bytes a lane in scratch; 64 KB of LDS a workgroup, int8 65).  2048 queries of 64
// heads of 128 on 8 over 32768 rows reach 1050 to 1070 TFLOP/s from e4m3, 1010 to 1030
// from bf16 and 900 from int8 rows (96 conversions and packs and 32 products with V's
// scales a lane and tile, where e4m3 has 32 conversions); a bf16 product of 8192 x 8192
// x 8192 reaches 1230 on this card.  1024 queries of 28 heads on 4 over 16384 rows,
// batch 4, reach 970, 945 and 820: 896 workgroups on 512 places.
#include "pages.hpp"

namespace mmskv {
namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kRows = 32 * kWaves;         // query rows of a workgroup
constexpr int kKeys = 64;                  // keys of a tile
constexpr float kNone = -3e38f;            // running maximum before the first visible key
// The reference m of a row's sums need not be its maximum, only near it: it moves,
// to kLead above the largest logit so far, where a lane's 16 (few rows: 8 or 16)
// weights 2^(x - m) add up to kBehind, so that no maximum is formed in most tiles
// and the output is seldom rescaled.  The lead is what the largest logit may gain
// before that: no weight is above 1, and the sums are in range wherever those
// relative to the maximum itself are (without it they were up to 2^8 times larger).
constexpr float kLead = 8.f, kBehind = 1.f;

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

// sum + the two bf16 values of y, by one instruction (DOT) or two additions.  The
// sum of a row's weights is of the weights as the product with V takes them, rounded
// to bf16, so that the quotient does not hold what their roundings have in common,
// nearly all of a heavy weight's: 1111 bf16 rows, queries of standard deviation 4,
// results off by 0.0018 of their 2-norm (their own rounding: 0.0017), with the sum of
// the unrounded weights by 0.0020.  (int8 weights are rounded with the scale of V,
// which the sum has no part in: 0.0023 to 0.0025; rounding a value to int8 costs more.)
template <bool DOT = true>
__device__ __forceinline__ float add_pair(uint32_t y, float sum) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    if constexpr (!DOT) return sum + (__uint_as_float(y << 16) + __uint_as_float(y & 0xFFFF0000u));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, y), __builtin_bit_cast(bf16x2, 0x3F803F80u), sum,
                                           false);
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
    constexpr int kRow = D * kCacheBytes<TYPE>;      // bytes of a cached row
    constexpr int kCh = kRow / 16;                   // its 16-byte chunks
    constexpr int kWaveRows = kKeys / kWaves;         // rows of a tile that a wave stages
    constexpr int kLoads = kWaveRows * kRow / 1024;  // its 16-byte loads of a lane of K (and of V)
    static_assert(kLoads >= 1, "whole load instructions");
    constexpr bool kScaled = TYPE == kCacheI8;       // scales applied to the logits and to p
    __shared__ __align__(16) char kt[2][kKeys * 2 * D];
    __shared__ __align__(16) char vt[2][kKeys * 2 * D];
    __shared__ __align__(16) float ksc[2][kScaled ? kKeys : 4], vsc[2][kScaled ? kKeys : 4];

    const int bc = blockIdx.x, b = bc / a.Hkv, c = bc - b * a.Hkv;
    // the last rows, which see most keys, first, with all their splits
    const int r0 = static_cast<int>((gridDim.y - 1 - blockIdx.y) / a.splits) * kRows;
    const int split = blockIdx.y % a.splits;
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
    // keys that all rows of the workgroup see (those that are not there aside)
    const int all_see = a.causal ? len - nq + r0 / a.Gh + 1 : len;
    // keys that the workgroup's rows see together, and this split's part of them
    const int i_end = min((min(r0 + kRows, a.rows) - 1) / a.Gh, nq - 1);
    const int end = i_end < r0 / a.Gh ? 0 : max(a.causal ? len - nq + i_end + 1 : len, 0);
    const int tiles = (end + kKeys - 1) / kKeys, per = (tiles + a.splits - 1) / a.splits;
    const int tile0 = split * per, tile1 = min(tile0 + per, tiles);

    // A wave stages rows kWaveRows * wave .. of a tile, which are on one page:
    // consecutive bytes of K and of V, by way of registers, so that the next
    // tile's are on their way while this one is worked on.
    u32x4 kr[kLoads], vr[kLoads];
    float ksr[kLoads], vsr[kLoads];
    auto load = [&](int tile) {
        const int t = tile * kKeys + kWaveRows * wave;
        const int id = uniform_page(a.pages, b, t);
        const int64_t pr = pool_row(a.pages, a.Hkv, c, id, t);
        typedef const char __attribute__((address_space(1))) * gchar;
        typedef const u32x4 __attribute__((address_space(1))) * gvec;
        typedef const float __attribute__((address_space(1))) * gfloat;
        const gchar none = (gchar)(kNoRows);
        const gchar ks = id >= 0 ? (gchar)(a.pages.k) + pr * kRow : none;
        const gchar vs = id >= 0 ? (gchar)(a.pages.v) + pr * kRow : none;
        const int step = id >= 0 ? 1024 : 0;         // (1 KB stands for a page that is not there)
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            kr[j] = *(gvec)(ks + j * step + 16 * lane);
            vr[j] = *(gvec)(vs + j * step + 16 * lane);
        }
        if constexpr (TYPE != kCacheBf16) {
            const gfloat kss = id >= 0 ? (gfloat)(a.pages.k_scale) + pr : (gfloat)(none);
            const gfloat vss = id >= 0 ? (gfloat)(a.pages.v_scale) + pr : (gfloat)(none);
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                ksr[j] = kss[j * (64 / kCh) + lane / kCh];
                vsr[j] = vss[j * (64 / kCh) + lane / kCh];
            }
        }
    };
    // Piece z (of kPieces) of what a lane stages: 16 bytes of a staged row of K (z
    // even) or V.
    constexpr int kPieces = 2 * kLoads * (TYPE == kCacheBf16 ? 1 : 2);
    auto store_piece = [&](int buf, int z) {
        const int j = TYPE == kCacheBf16 ? z / 2 : z / 4, w = z / 2 % 2;
        const int row = kWaveRows * wave + j * (64 / kCh) + lane / kCh, ch = lane % kCh;
        const bool v = z % 2 != 0;
        char* const to = (v ? vt : kt)[buf];
        const u32x4 x = v ? vr[j] : kr[j];
        if constexpr (TYPE == kCacheBf16) {
            *reinterpret_cast<u32x4*>(to + staged<D>(row, ch)) = x;
        } else {
            const float by = v ? vsr[j] : ksr[j];
            const u32x2 y0 = widen4<TYPE>(w ? x[2] : x[0], by), y1 = widen4<TYPE>(w ? x[3] : x[1], by);
            *reinterpret_cast<u32x4*>(to + (staged<D>(row, 2 * ch) ^ (16 * w))) = u32x4{y0[0], y0[1], y1[0], y1[1]};
            if (kScaled && w == 0 && ch == 0) (v ? vsc : ksc)[buf][row] = v ? by : by * a.scale;
        }
    };
    // store_piece widens e4m3 values by the exponent of their scale, which is all of it
    // in rows that cache_write made.  Where a wave's rows have another scale (a branch
    // that the tiles of such rows do not take) its part of the tile is staged again:
    // values times scales, rounded to bf16.  The look at them runs beside the matrix
    // instructions: 2048 queries over 32768 rows 2013 us, without it 2001, behind the
    // tile 2026; scales on the logits and on p, as int8 has them, would cost every tile.
    auto other_scales = [&] {
        if constexpr (TYPE != kCacheE4m3) return false;
        uint32_t rest = 0;                 // sign and mantissa bits
#pragma unroll
        for (int j = 0; j < kLoads; ++j) rest |= __float_as_uint(ksr[j]) | __float_as_uint(vsr[j]);
        return __any((rest & 0x807FFFFFu) != 0u) != 0;
    };
    auto stage_again = [&](int buf) {
        if constexpr (TYPE == kCacheE4m3) {
#pragma unroll
            for (int z = 0; z < 2 * kLoads; ++z) {
                const int j = z / 2, row = kWaveRows * wave + j * (64 / kCh) + lane / kCh, ch = lane % kCh;
                char* const to = (z % 2 ? vt : kt)[buf];
                const float by = z % 2 ? vsr[j] : ksr[j];
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    u32x4 y;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float x[4];
                        unpack4<TYPE>(z % 2 ? vr[j][2 * w + e] : kr[j][2 * w + e], x);
                        y[2 * e] = pack_bf16(x[0] * by, x[1] * by);
                        y[2 * e + 1] = pack_bf16(x[2] * by, x[3] * by);
                    }
                    *reinterpret_cast<u32x4*>(to + (staged<D>(row, 2 * ch) ^ (16 * w))) = y;
                }
            }
        }
    };
    // Rows of V behind the last key may hold anything: zeros, for p = 0 to meet
    // (their logits are masked).  By the wave that staged them.
    auto clear_tail = [&](int tile, int buf) {
        if ((tile + 1) * kKeys <= end) return;
        constexpr int kOut = 2 * D / 16;
        for (int x = lane; x < kWaveRows * kOut; x += kWave) {
            const int row = kWaveRows * wave + x / kOut;
            if (tile * kKeys + row < end) continue;
            *reinterpret_cast<u32x4*>(vt[buf] + row * 2 * D + 16 * (x % kOut)) = u32x4{0u, 0u, 0u, 0u};
            if (kScaled) vsc[buf][row] = 0.f;
        }
    };

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

    // value e of s[u] is key key0 + 32 u + 8 (e / 4) + 4 half + e % 4
    const float scale = kScaled ? 1.f : a.scale;
    // One tile, in two 32-key halves u, as a sequence of steps of one matrix
    // instruction with vector instructions to run beside it: the exponentials of
    // half 0 with the second half's S, those of half 1 with the first half's part
    // of O, the staging of the next tile with the second's.  (Left to itself the
    // compiler puts all matrix instructions of a phase first, and a SIMD's two
    // waves do not fill the gaps: 960 TFLOP/s.)  MASKED: some row does not see all.
    auto attend = [&](int key0, int buf, auto masked, auto staging) {
        constexpr bool MASKED = decltype(masked)::value != 0;
        constexpr int N = KC;              // steps of a phase: KC = 2 NT
        constexpr int PAIRS = 8 / N;       // pairs of exponentials of a step
        constexpr int AHEAD = 4;           // steps from a read of LDS to its use
        static_assert(N == 2 * NT, "as many steps in S as in O");
        // staged() of this lane's rows of K (chunk 2 kc + half: a permuted chunk is
        // one exclusive or away) and of V; opaque, so that they are formed where
        // they are used instead of being kept in 24 registers
        int ka = staged<D>(lane & 31, half), va = staged<D>(4 * half + ((lane & 15) >> 2), (lane & 16) / 8 + ((lane & 3) >> 1));
        va += 8 * (lane & 1);
        asm volatile("" : "+v"(ka), "+v"(va));
        const int rel = last - key0 - 4 * half;
        floatx16 s[2];
        floatx4 kw[4], vw[4];              // scales of a half's keys
        auto scales = [&](int u) {
            if constexpr (kScaled) {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    kw[g] = *reinterpret_cast<const floatx4*>(ksc[buf] + 32 * u + 8 * g + 4 * half);
                    vw[g] = *reinterpret_cast<const floatx4*>(vsc[buf] + 32 * u + 8 * g + 4 * half);
                }
            }
        };
        auto k_frag = [&](int j) {         // step j % N of half j / N
            return load_bf16x8(reinterpret_cast<const uint16_t*>(kt[buf] + j / N * 32 * 2 * D + (ka ^ (32 * (j % N)))));
        };
        auto v_frag = [&](int j) {         // half j / N, step j % N: keys 16 w .., dims 32 t ..
            typedef s16x4 __attribute__((address_space(3))) * lds4;
            const int u = j / N, w = j % N / NT, t = j % NT;
            u32x4 v;
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                // V^T: dims 32 t + lane % 32, keys 32 u + 16 w + 4 half + {0..3, 8..11}; eight
                // rows further the permutation differs by two chunks (d = 128 and 64)
                const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds4)(vt[buf] + (32 * u + 16 * w + 8 * z) * 2 * D + (va ^ (64 * t + 32 * z))));
                const u32x2 y = __builtin_bit_cast(u32x2, x);
                v[2 * z] = y[0];
                v[2 * z + 1] = y[1];
            }
            return __builtin_bit_cast(bf16x8, v);
        };
        // logit e of half u, scaled; a masked one is -inf whatever its row's scale
        auto logit = [&](int u, int e, float less) {
            float x = fmaf(s[u][e], kScaled ? kw[e >> 2][e & 3] : scale, -less);
            if (MASKED) x = 32 * u + 8 * (e >> 2) + (e & 3) <= rel ? x : -INFINITY;
            return x;
        };
        // p of values 2 j, 2 j + 1 of half u relative to m, as bf16; their sum
        auto pair = [&](int u, int j, float& sum) {
            float x[2];
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                const int e = 2 * j + z;
                x[z] = fast_exp2(logit(u, e, m));
                if (kScaled) {             // (rounded with the scale of V: the sum has the weights before)
                    sum += x[z];
                    x[z] *= vw[e >> 2][e & 3];
                }
            }
            const uint32_t y = pack_bf16(x[0], x[1]);
            // (2048 queries over 32768 rows, additions / one instruction: bf16 2080 / 2150 us,
            // e4m3 2012 / 1993)
            if (!kScaled) sum = add_pair<TYPE != kCacheBf16>(y, sum);
            return y;
        };
        // m moved where half u leaves it behind
        auto settle = [&](int u, uint32_t (&p)[8], float sum) {
            if (__any(!(sum < kBehind))) {
                float mx = kNone;
#pragma unroll
                for (int e = 0; e < 16; ++e) mx = fmaxf(mx, logit(u, e, 0.f));
                mx = fmaxf(half_max(mx) + kLead, m);
                const float f = fast_exp2(m - mx);
                m = mx;
                l *= f;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[t][j] *= f;
                sum = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) p[j] = pair(u, j, sum);
            }
            l += sum;
        };
        auto p_frag = [](const uint32_t (&p)[8], int w) {
            return __builtin_bit_cast(bf16x8, (u32x4{p[4 * w], p[4 * w + 1], p[4 * w + 2], p[4 * w + 3]}));
        };
        const auto fence = [] { __builtin_amdgcn_sched_barrier(0); };

        bf16x8 f[2 * N];
        uint32_t p0[8], p1[8];
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) f[j] = k_frag(j);
        scales(0);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[u][e] = 0.f;
#pragma unroll
        for (int j = 0; j < 2 * N; ++j) {
            fence();
            if (j + AHEAD < 2 * N) f[j + AHEAD] = k_frag(j + AHEAD);
            s[j / N] = mfma32(f[j], qf[j % N], s[j / N]);
            if (j >= N) {
#pragma unroll
                for (int z = 0; z < PAIRS; ++z) p0[(j - N) * PAIRS + z] = pair(0, (j - N) * PAIRS + z, sum);
            }
        }
        fence();
        settle(0, p0, sum);
        sum = 0.f;
        scales(1);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) f[j] = v_frag(j);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            fence();
            f[j + AHEAD] = v_frag(j + AHEAD);
            o[j % NT] = mfma32(f[j], p_frag(p0, j / NT), o[j % NT]);
#pragma unroll
            for (int z = 0; z < PAIRS; ++z) p1[j * PAIRS + z] = pair(1, j * PAIRS + z, sum);
        }
        fence();
        settle(1, p1, sum);
#pragma unroll
        for (int j = N; j < 2 * N; ++j) {
            fence();
            if (j + AHEAD < 2 * N) f[j + AHEAD] = v_frag(j + AHEAD);
            o[j % NT] = mfma32(f[j], p_frag(p1, (j - N) / NT), o[j % NT]);
            staging(j - N);
        }
        fence();
    };

    if (tile0 < tile1) {
        load(tile0);
#pragma unroll
        for (int z = 0; z < kPieces; ++z) store_piece(0, z);
        if (other_scales()) stage_again(0);
        clear_tail(tile0, 0);
    }
    __syncthreads();
    int buf = 0, tile = tile0;
    auto step = [&](auto masked) {
        if (tile + 1 < tile1) load(tile + 1);
        // (behind the last tile the registers' old values, which nobody reads)
        bool other = false;
        attend(tile * kKeys, buf, masked, [&](int j) {
            if (j == 0) other = other_scales();
#pragma unroll
            for (int z = j * kPieces / KC; z < (j + 1) * kPieces / KC; ++z) store_piece(buf ^ 1, z);
        });
        if (tile + 1 < tile1) {
            if (other) stage_again(buf ^ 1);
            clear_tail(tile + 1, buf ^ 1);
        }
        __syncthreads();
        ++tile, buf ^= 1;
    };
    const int whole = min(max(all_see, 0) / kKeys, tile1);
    while (tile < whole) step(Constant<0>{});
    while (tile < tile1) step(Constant<1>{});
    l = half_sum(l);
    if (r >= a.rows) return;
    if (!there) l = 0.f;                   // (took part where nothing is masked)
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
    // (by selects: the sums of a row without weight may hold NaN, of 0 or 1 times an infinite V of its tiles)
    const bool none = l == 0.f;
    const float inv = 1.f / l;
    uint16_t* out = a.out + b * a.osb + h * a.osh + i * a.ost + 4 * half;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const u32x2 y{pack_bf16(o[t][4 * w] * inv, o[t][4 * w + 1] * inv),
                          pack_bf16(o[t][4 * w + 2] * inv, o[t][4 * w + 3] * inv)};
            *reinterpret_cast<u32x2*>(out + 32 * t + 8 * w) = none ? u32x2{0u, 0u} : y;
        }
}

// ---- few rows -----------------------------------------------------------
// Up to 64 rows of a (b, c): the keys are read from HBM once and little is
// computed on them, so what counts is how many bytes are in flight.  Each wave
// of a workgroup (four, or eight with half as large stages) has key tiles of its
// own, one of every four or eight, and all rows, in NR tiles of 16; it loads its
// tiles straight to LDS of its own, in two stages of up to 8 KB of K and 8 KB of
// V, so that no wave waits for another before the end and a CU has 64 KB on their
// way while it works on as many.  (16 sequences of 8 heads of up to 32768 bf16
// rows of 128, 1.63 GB: 272 us, 6.0 TB/s, where reading alone reaches 7.0 and a
// copy 5.7; the lengths differ, so that some CUs end early.)
// The rows stay as the cache holds them; 8-bit values are widened in registers.
//   S^T = K Q^T  (v_mfma_f32_16x16x32_bf16, lane = query row lane % 16)
//   O^T += V^T P^T
// Row m of the s-th of two 16-key tiles of S^T is key 8 (m / 4) + 4 s + m % 4 of
// their 32: with that order a lane's eight p are those of eight consecutive
// keys, the ones that its transposing reads of V fetch.
constexpr int kFewRows = 64;

__device__ __forceinline__ floatx4 mfma16(bf16x8 a, bf16x8 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Largest value / sum over the four lanes that hold a query row (lane % 16).
__device__ __forceinline__ float quarter_max(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return half_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quarter_sum(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return half_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// Waves of a workgroup: widening 8-bit values takes longer than their loads, and
// two waves of a SIMD do it in turn where their sums fit LDS, up to 32 rows (7 rows
// over 300 e4m3 rows 7.6 -> 6.2 us; 32 sequences of 4 heads of up to 1100, 13.9 -> 11.3).
constexpr int few_waves(int d, int type, int nr) { return d == 128 && type != kCacheBf16 && nr <= 2 ? 8 : 4; }

template <int D, int TYPE, int WAVES>
struct FewTile {
    static constexpr int kRow = D * kCacheBytes<TYPE>;          // bytes of a cached row: 64, 128 or 256
    static constexpr int kCh = kRow / 16;                       // its 16-byte chunks
    static constexpr int kKeys = kRow == 256 || WAVES == 8 ? 32 : 64;   // keys of a stage
    static constexpr int kTile = kKeys * kRow;                  // bytes of its K (and of its V)
    static constexpr int kPer = 1024 / kRow;                    // rows of one load instruction: 4 to 16, on one page
    static constexpr int kLoads = kKeys / kPer;                 // load instructions of K (and of V)
    static constexpr bool kScaled = TYPE != kCacheBf16;
    static constexpr int kGroups = kKeys / 16;                  // 16-row groups, each on one page
    static constexpr int kAll = 2 * kLoads + (kScaled ? kKeys / 32 : 0);
    static constexpr int kStage = 2 * kTile + (kScaled ? 2 * kKeys * 4 : 0);
    // Byte of 16-byte chunk ch of row r.  The chunks of a row are permuted by those
    // bits of r that differ between the lanes of a read (0, 1, 3 and 4), so that the
    // reads spread over all banks and rows 4 or 32 apart are a constant apart.
    static __device__ __forceinline__ int swz(int r) {
        return kCh == 16 ? ((r & 3) << 2) | ((r >> 3) & 3)
                         : kCh == 8 ? ((r >> 1) & 1) | (((r >> 3) & 3) << 1) : (r >> 3) & 3;
    }
    static __device__ __forceinline__ int at(int r, int ch) { return r * kRow + 16 * (ch ^ swz(r)); }
};

// Offsets of eight reads of a stage's K, V and scales.
template <class T, int STAGE, int U0, int KC>
struct KOffsets {                          // 16-key tiles U0 + z / KC
    static constexpr int at(int z) {
        const int u = U0 + z / KC;
        return STAGE * T::kStage + (32 * (u >> 1) + 4 * (u & 1)) * T::kRow;
    }
};
template <class T, int STAGE>
struct ScaleOffsets {                      // half of K, half of V: keys 32 (u / 2) + 4 (u % 2)
    static constexpr int at(int z) {
        constexpr int kTiles = T::kKeys / 16;
        const int u = z % kTiles;
        return STAGE * T::kStage + 2 * T::kTile + z / kTiles * T::kKeys * 4 + 4 * (32 * (u / 2) + 4 * (u % 2));
    }
};
template <class T, int STAGE, int U0>
struct VOffsets {                          // 8-bit: 32-key steps z % (NS / 2); bf16: step U0, keys 4 (z % 2) ..
    static constexpr int at(int z) {
        const int row = T::kScaled ? 32 * (z % (T::kKeys / 32)) : 32 * U0 + 4 * (z & 1);
        return STAGE * T::kStage + T::kTile + row * T::kRow;
    }
};

// The load instructions J .. LOADS - 1 of a 16-row group from src (its first row;
// 1 KB of zeros where `any` is not set) to dst; row0: its first row in the tile.
template <class T, int J, int LOADS>
__device__ __forceinline__ void load_group(const char* src, char* dst, int row0, int ld_row, int lane, bool any) {
    const int r = row0 + J * T::kPer + ld_row;
    const int off = ld_row * T::kRow + 16 * ((lane % T::kCh) ^ T::swz(r));
    // (the offset of an instruction is added to both of its addresses)
    load16_to_lds<1024 * J>(src + off - (any ? 0 : 1024 * J), dst);
    if constexpr (J + 1 < LOADS) load_group<T, J + 1, LOADS>(src, dst, row0, ld_row, lane, any);
}

// Workgroup: WAVES waves; (b, c) and a split of its keys.
template <int D, int TYPE, int NR, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, 1) chunk_few_kernel(ChunkArgs a) {
    using T = FewTile<D, TYPE, WAVES>;
    constexpr int kWaves = WAVES, kThreads = 64 * WAVES;
    constexpr int KC = D / 32;             // 32-dim steps of S
    constexpr int NT = D / 16;             // 16-dim tiles of O
    constexpr int NS = T::kKeys / 16;      // 16-key tiles of S
    constexpr int kLd = D + 4;             // floats of a row in the merge
    constexpr int kMerge = NR * 16 * kLd * 4;
    constexpr int kWaveLds = 2 * T::kStage > kMerge ? 2 * T::kStage : kMerge;
    __shared__ __align__(16) char lds[kWaves][kWaveLds];
    __shared__ __align__(16) char qs[NR * 16 * 2 * D];
    __shared__ float2 ml[kWaves][NR * 16];

    const int bc = blockIdx.x, b = bc / a.Hkv, c = bc - b * a.Hkv, split = blockIdx.y;
    const int tid = threadIdx.x, lane = lane_id();
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int quarter = lane >> 4;
    char* const base = lds[wave];

    const int nq = a.q_counts ? min(max(a.q_counts[b], 0), a.n) : a.n;
    const int len = min(max(a.lens[bc], 0), a.max_len);
    const int end = nq > 0 ? len : 0;      // keys that the rows see together
    const int tiles = (end + T::kKeys - 1) / T::kKeys, per = (tiles + a.splits - 1) / a.splits;
    const int tile0 = split * per + wave, tile1 = min(split * per + per, tiles);

    // pages of the 16-row groups of a tile (-1: none)
    struct Ids {
        int id[T::kGroups];
    };
    auto pages_of = [&](int tile) {
        Ids ids;
#pragma unroll
        for (int g = 0; g < T::kGroups; ++g) ids.id[g] = uniform_page(a.pages, b, tile * T::kKeys + 16 * g);
        return ids;
    };
    // A load instruction fetches 1 KB, kPer rows of a group; a lane's bytes of it are
    // those of the chunk that its place in the staged order stands for.
    constexpr int kGroupLoads = 16 / T::kPer;
    const int ld_row = lane / T::kCh;
    auto load_stage = [&](int tile, int stage, const Ids& ids) {
        char* dst = base + stage * T::kStage;
        const int t0 = tile * T::kKeys;
        const char* none = reinterpret_cast<const char*>(kNoRows);
#pragma unroll
        for (int g = 0; g < T::kGroups; ++g) {
            const bool any = ids.id[g] >= 0;
            const int64_t e = pool_row(a.pages, a.Hkv, c, ids.id[g], t0 + 16 * g) * T::kRow;
            const char* ks = any ? static_cast<const char*>(a.pages.k) + e : none;
            const char* vs = any ? static_cast<const char*>(a.pages.v) + e : none;
            load_group<T, 0, kGroupLoads>(ks, dst + g * 16 * T::kRow, 16 * g, ld_row, lane, any);
            load_group<T, 0, kGroupLoads>(vs, dst + T::kTile + g * 16 * T::kRow, 16 * g, ld_row, lane, any);
        }
        if constexpr (T::kScaled) {
            // a lane has the scales of one row; of 32 rows, those of K or those of V
            const int t = lane & (T::kKeys - 1);
            int id = ids.id[0];
#pragma unroll
            for (int g = 1; g < T::kGroups; ++g) id = t / 16 == g ? ids.id[g] : id;
            const int64_t pr = pool_row(a.pages, a.Hkv, c, id, t0 + t);
            const float* one = T::kKeys == 32 && lane >= 32 ? a.pages.v_scale : a.pages.k_scale;
            load4_to_lds(id >= 0 ? reinterpret_cast<const char*>(one + pr) : none, dst + 2 * T::kTile);
            if constexpr (T::kKeys == 64)
                load4_to_lds(id >= 0 ? reinterpret_cast<const char*>(a.pages.v_scale + pr) : none,
                             dst + 2 * T::kTile + 256);
        }
    };

    // the rows of all waves to LDS, 1 KB per instruction (missing ones as zeros), then two stages
    constexpr int QC = D / 8;              // 16-byte chunks of a query row
    const auto q_at = [](int r, int ch) { return r * 2 * D + 16 * (ch ^ ((QC == 16 ? r : r >> 1) & (QC - 1))); };
#pragma unroll
    for (int j = 0; j < NR * 16 * QC / kWave; j += kWaves) {
        if (j + wave >= NR * 16 * QC / kWave) break;
        const int r = (j + wave) * (kWave / QC) + lane / QC, i = r / a.Gh, h = c * a.Gh + (r - i * a.Gh);
        const int ch = (lane % QC) ^ ((QC == 16 ? r : r >> 1) & (QC - 1));
        const bool there = r < a.rows && i < nq;
        const char* src = there ? reinterpret_cast<const char*>(a.q + b * a.qsb + h * a.qsh + i * a.qst + 8 * ch)
                                : reinterpret_cast<const char*>(kNoRows);
        load16_to_lds(src, qs + (j + wave) * 1024);
    }
    // (the waits below count on this order)
    __builtin_amdgcn_sched_barrier(0);
    Ids ids = pages_of(tile0);
    if (tile0 < tile1) load_stage(tile0, 0, ids);
    __builtin_amdgcn_sched_barrier(0);
    ids = pages_of(tile0 + kWaves);
    if (tile0 + kWaves < tile1) load_stage(tile0 + kWaves, 1, ids);
    __builtin_amdgcn_sched_barrier(0);

    // the last key that each of this lane's rows sees (below 0: none)
    int last[NR];
#pragma unroll
    for (int x = 0; x < NR; ++x) {
        const int r = 16 * x + (lane & 15), i = r / a.Gh;
        last[x] = r < a.rows && i < nq ? (a.causal ? len - nq + i : len - 1) : -1;
    }
    // keys that every row sees
    const int all_see = a.causal ? max(len - nq + 1, 0) : len;

    floatx4 o[NR][NT];
    float m[NR], l[NR];
#pragma unroll
    for (int x = 0; x < NR; ++x) {
        m[x] = kNone;
        l[x] = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t) o[x][t] = floatx4{0.f, 0.f, 0.f, 0.f};
    }

    if (tile0 + kWaves < tile1) wait_vm<2 * T::kAll>();
    else if (tile0 < tile1) wait_vm<T::kAll>();
    else wait_vm<0>();
    asm volatile("s_barrier" ::: "memory");
    bf16x8 qf[NR][KC];
#pragma unroll
    for (int x = 0; x < NR; ++x) {
        uint32_t at[KC];
        u32x4 w[KC];
#pragma unroll
        for (int kc = 0; kc < KC; ++kc) at[kc] = lds_address(qs) + q_at(16 * x + (lane & 15), 4 * kc + quarter);
        read128(at, w);
#pragma unroll
        for (int kc = 0; kc < KC; ++kc) qf[x][kc] = __builtin_bit_cast(bf16x8, w[kc]);
    }

    // a lane's places in a stage: of K, one for each 32-dim step; of V, for each
    // 16-dim tile; of the scales
    uint32_t k_at[KC], v_at[NT];
    const uint32_t s_at = lds_address(base) + 32 * quarter;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
        const int row = 8 * ((lane & 15) >> 2) + (lane & 3);
        k_at[kc] = lds_address(base) + (T::kScaled ? T::at(row, 2 * kc + (quarter >> 1)) + 8 * (quarter & 1)
                                                   : T::at(row, 4 * kc + quarter));
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
        v_at[t] = lds_address(base) + 8 * (lane & 1) +
                  (T::kScaled ? T::at(8 * quarter + ((lane & 15) >> 1), t)
                              : T::at(8 * quarter + ((lane & 15) >> 2), 2 * t + ((lane >> 1) & 1)));

    auto step = [&](int tile, auto which, bool first) {
        constexpr int STAGE = decltype(which)::value;
        if (tile + kWaves < tile1) wait_vm<T::kAll>();     // all but the next stage
        else wait_vm<0>();
        __builtin_amdgcn_sched_barrier(0);
        ids = pages_of(tile + 2 * kWaves);
        const int key0 = tile * T::kKeys;
        if (key0 + T::kKeys > end) {
            // rows behind the last key may hold anything: zeros, with zero scales
            char* const vt = base + STAGE * T::kStage + T::kTile;
            float* const sc = reinterpret_cast<float*>(vt + T::kTile);
            for (int i = lane; i < T::kKeys * T::kCh; i += kWave)
                if (key0 + i / T::kCh >= end) *reinterpret_cast<u32x4*>(vt + i * 16) = u32x4{0u, 0u, 0u, 0u};
            if (T::kScaled && lane < T::kKeys && key0 + lane >= end) sc[lane] = 0.f, sc[T::kKeys + lane] = 0.f;
        }
        // value e of s[x][u] is key key0 + 32 (u / 2) + 8 quarter + 4 (u % 2) + e
        floatx4 s[NR][NS];
#pragma unroll
        for (int u = 0; u < NS; ++u)
#pragma unroll
            for (int x = 0; x < NR; ++x) s[x][u] = floatx4{0.f, 0.f, 0.f, 0.f};
        constexpr int UB = 8 / KC;         // 16-key tiles of eight reads
        auto logits = [&](auto first_tile) {
            constexpr int U0 = decltype(first_tile)::value;
            uint32_t at[8];
            bf16x8 k[8];
#pragma unroll
            for (int z = 0; z < 8; ++z) at[z] = k_at[z % KC];
            if constexpr (T::kScaled) {
                u32x2 w[8];
                read64<KOffsets<T, STAGE, U0, KC>>(at, w);
#pragma unroll
                for (int z = 0; z < 8; ++z) {
                    const u32x2 y0 = widen4<TYPE>(w[z][0]), y1 = widen4<TYPE>(w[z][1]);
                    k[z] = __builtin_bit_cast(bf16x8, (u32x4{y0[0], y0[1], y1[0], y1[1]}));
                }
            } else {
                u32x4 w[8];
                read128<KOffsets<T, STAGE, U0, KC>>(at, w);
#pragma unroll
                for (int z = 0; z < 8; ++z) k[z] = __builtin_bit_cast(bf16x8, w[z]);
            }
#pragma unroll
            for (int z = 0; z < 8; ++z)
#pragma unroll
                for (int x = 0; x < NR; ++x) s[x][U0 + z / KC] = mfma16(k[z], qf[x][z % KC], s[x][U0 + z / KC]);
        };
        logits(Constant<0>{});
        if constexpr (UB < NS) logits(Constant<UB < NS ? UB : 0>{});
        static_assert(2 * UB >= NS, "two blocks of reads");
        floatx4 vw[NS];                    // scales of the keys' V
        if constexpr (T::kScaled) {
            u32x4 w[2 * NS];               // of K, then of V
            if constexpr (NS == 4) {
                uint32_t at[8];
#pragma unroll
                for (int z = 0; z < 8; ++z) at[z] = s_at;
                read128<ScaleOffsets<T, STAGE>>(at, w);
            } else {
                static_assert(NS == 2, "four or eight reads of four scales");
                uint32_t at[4];
#pragma unroll
                for (int z = 0; z < 4; ++z) at[z] = s_at + ScaleOffsets<T, STAGE>::at(z);
                read128(at, w);
            }
#pragma unroll
            for (int u = 0; u < NS; ++u) {
                vw[u] = __builtin_bit_cast(floatx4, w[NS + u]);
#pragma unroll
                for (int x = 0; x < NR; ++x) s[x][u] *= __builtin_bit_cast(floatx4, w[u]);
            }
        }
        if (key0 + T::kKeys > all_see) {
            asm volatile("");              // (a branch: few tiles come here)
#pragma unroll
            for (int x = 0; x < NR; ++x) {
                const int rel = last[x] - key0 - 8 * quarter;
#pragma unroll
                for (int u = 0; u < NS; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        s[x][u][e] = 32 * (u >> 1) + 4 * (u & 1) + e <= rel ? s[x][u][e] : -INFINITY;
            }
        }
        bf16x8 p[NR][NS / 2];
        float sum[NR];
        auto weights = [&]() {
#pragma unroll
            for (int x = 0; x < NR; ++x) {
                sum[x] = 0.f;
#pragma unroll
                for (int u = 0; u < NS; u += 2) {
                    u32x4 y;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int z = u + (j >> 1), e = 2 * (j & 1);
                        const float p0 = fast_exp2(fmaf(s[x][z][e], a.scale, -m[x]));
                        const float p1 = fast_exp2(fmaf(s[x][z][e + 1], a.scale, -m[x]));
                        // (e4m3: times a power of two, which commutes with the rounding; int8 weights
                        // are rounded with the scale of V, their sum has them before)
                        if (TYPE != kCacheI8) sum[x] = add_pair(y[j] = pack_bf16(p0, p1), sum[x]);
                        else sum[x] += p0 + p1;
                        if (T::kScaled) y[j] = pack_bf16(p0 * vw[z][e], p1 * vw[z][e + 1]);
                    }
                    p[x][u / 2] = __builtin_bit_cast(bf16x8, y);
                }
            }
        };
        // m moves where the tile leaves it behind; in the first tile there is none yet
        bool behind = first;
        if (!first) {
            weights();
            float most = sum[0];
#pragma unroll
            for (int x = 1; x < NR; ++x) most = sum[x] < kBehind ? most : sum[x];
            behind = __any(!(most < kBehind));
        }
        if (behind) {
#pragma unroll
            for (int x = 0; x < NR; ++x) {
                float mx = s[x][0][0];
#pragma unroll
                for (int u = 0; u < NS; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[x][u][e]);
                mx = fmaxf(quarter_max(mx) * a.scale + kLead, m[x]);
                const float f = fast_exp2(m[x] - mx);
                m[x] = mx;
                l[x] *= f;
#pragma unroll
                for (int t = 0; t < NT; ++t) o[x][t] *= f;
            }
            weights();
        }
#pragma unroll
        for (int x = 0; x < NR; ++x) l[x] += sum[x];
        // V^T: dims 16 t + lane % 16, keys 32 u + 8 quarter + 0 .. 7; eight reads: four
        // tiles t of one 32-key step (bf16: two reads each), or of both
        constexpr int TB = T::kScaled ? 8 / (NS / 2) : 4;
        auto output = [&](auto first_tile, auto key_step) {
            constexpr int T0 = decltype(first_tile)::value, U0 = decltype(key_step)::value;
            uint32_t at[8];
            u32x2 w[8];
#pragma unroll
            for (int z = 0; z < 8; ++z) at[z] = v_at[T0 + z * TB / 8];
            if constexpr (T::kScaled) {
                read_transposed8<VOffsets<T, STAGE, U0>>(at, w);
#pragma unroll
                for (int z = 0; z < 8; ++z) {
                    const u32x2 y0 = widen4<TYPE>(w[z][0]), y1 = widen4<TYPE>(w[z][1]);
                    const bf16x8 v = __builtin_bit_cast(bf16x8, (u32x4{y0[0], y0[1], y1[0], y1[1]}));
                    const int t = T0 + z * TB / 8, u = z % (NS / 2);
#pragma unroll
                    for (int x = 0; x < NR; ++x) o[x][t] = mfma16(v, p[x][u], o[x][t]);
                }
            } else {
                read_transposed16<VOffsets<T, STAGE, U0>>(at, w);
#pragma unroll
                for (int z = 0; z < 4; ++z) {
                    const bf16x8 v = __builtin_bit_cast(bf16x8, (u32x4{w[2 * z][0], w[2 * z][1], w[2 * z + 1][0],
                                                                      w[2 * z + 1][1]}));
#pragma unroll
                    for (int x = 0; x < NR; ++x) o[x][T0 + z] = mfma16(v, p[x][U0], o[x][T0 + z]);
                }
            }
        };
        constexpr int US = T::kScaled ? 1 : NS / 2;        // blocks of reads per TB tiles
        static_assert(NT <= 2 * TB && US <= 2, "two by two blocks of reads");
        output(Constant<0>{}, Constant<0>{});
        if constexpr (US > 1) output(Constant<0>{}, Constant<1>{});
        if constexpr (NT > TB) output(Constant<NT - TB>{}, Constant<0>{});
        if constexpr (NT > TB && US > 1) output(Constant<NT - TB>{}, Constant<1>{});
        __builtin_amdgcn_sched_barrier(0);
        // this stage has been read: the one after the next into its place
        if (tile + 2 * kWaves < tile1) load_stage(tile + 2 * kWaves, STAGE, ids);
        __builtin_amdgcn_sched_barrier(0);
    };
    for (int tile = tile0; tile < tile1; tile += 2 * kWaves) {
        step(tile, Constant<0>{}, tile == tile0);
        if (tile + kWaves < tile1) step(tile + kWaves, Constant<1>{}, false);
    }

    // join the waves: value e of o[x][t] is dim 16 t + 4 quarter + e of row 16 x + lane % 16
    float* const ob = reinterpret_cast<float*>(base);
#pragma unroll
    for (int x = 0; x < NR; ++x) {
        const float sum = quarter_sum(l[x]);
        if (quarter == 0) ml[wave][16 * x + lane] = make_float2(m[x], sum);
#pragma unroll
        for (int t = 0; t < NT; ++t)
            *reinterpret_cast<floatx4*>(ob + (16 * x + (lane & 15)) * kLd + 16 * t + 4 * quarter) = o[x][t];
    }
    __syncthreads();
    constexpr int G = D / 8;               // lanes of a row, 8 dims each
    for (int it = tid; it < a.rows * G; it += kThreads) {
        const int r = it / G, d0 = 8 * (it - r * G), i = r / a.Gh;
        float M = kNone, L = 0.f, x[8] = {};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) M = fmaxf(M, ml[w][r].x);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float2 v = ml[w][r];
            const float f = fast_exp2(v.x - M);
            L = fmaf(v.y, f, L);
            const float* src = reinterpret_cast<const float*>(lds[w]) + r * kLd + d0;
            const floatx4 y0 = *reinterpret_cast<const floatx4*>(src), y1 = *reinterpret_cast<const floatx4*>(src + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = fmaf(y0[e], f, x[e]), x[4 + e] = fmaf(y1[e], f, x[4 + e]);
        }
        if (i >= nq) L = 0.f;              // (a row that is not there took part where nothing is masked)
        if (a.splits > 1) {
            const int64_t pr = (static_cast<int64_t>(split) * gridDim.x + bc) * a.rows + r;
            float* po = a.part_o + pr * D + d0;
            *reinterpret_cast<float4*>(po) = make_float4(x[0], x[1], x[2], x[3]);
            *reinterpret_cast<float4*>(po + 4) = make_float4(x[4], x[5], x[6], x[7]);
            if (d0 == 0) a.part_ml[pr] = make_float2(M, L);
        } else {
            const float inv = 1.f / L;
            const int h = c * a.Gh + (r - i * a.Gh);
            u32x4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = pack_bf16(x[2 * j] * inv, x[2 * j + 1] * inv);
            if (L == 0.f) v = u32x4{0u, 0u, 0u, 0u};       // (x may hold NaN, as in chunk_kernel)
            *reinterpret_cast<u32x4*>(a.out + b * a.osb + h * a.osh + i * a.ost + d0) = v;
        }
    }
}

// Joins the splits of a row: the largest m as reference, every sum rescaled to
// it.  D / 8 lanes per row and group of splits, 8 dims each; SG groups share a
// row's splits and add their sums through LDS.  All loads of a thread (kJoinPer
// splits at a time, no branch between them) are on their way before the first
// is needed: a loop that waited for each split took 0.8 us a split.
constexpr int kJoinThreads = 256;
constexpr int kJoinPer = 8;

template <int D, int SG>
__global__ void __launch_bounds__(kJoinThreads) chunk_join_kernel(ChunkArgs a) {
    constexpr int LANES = D / 8, kRowThreads = LANES * SG, kPerBlock = kJoinThreads / kRowThreads;
    __shared__ __align__(16) float sums[SG > 1 ? kJoinThreads : 1][8];
    __shared__ float2 ml[SG > 1 ? kJoinThreads : 1];
    const int lane = threadIdx.x % LANES, g = threadIdx.x / LANES % SG;
    const int64_t rows = static_cast<int64_t>(a.B) * a.Hkv * a.rows;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * kPerBlock + threadIdx.x / kRowThreads;
    const int64_t rd = min(row, rows - 1);             // (rows behind the last one read it and write nothing)
    float m = kNone, l = 0.f, o[8] = {};
    for (int s0 = g; s0 < a.splits; s0 += SG * kJoinPer) {
        float2 v[kJoinPer];
        float4 x[kJoinPer], y[kJoinPer];
#pragma unroll
        for (int j = 0; j < kJoinPer; ++j) {
            const int64_t at = min(s0 + j * SG, a.splits - 1) * rows + rd;
            const float* po = a.part_o + at * D + 8 * lane;
            v[j] = a.part_ml[at];
            x[j] = *reinterpret_cast<const float4*>(po);
            y[j] = *reinterpret_cast<const float4*>(po + 4);
        }
        float mx = m;
#pragma unroll
        for (int j = 0; j < kJoinPer; ++j) {
            if (s0 + j * SG >= a.splits) v[j] = make_float2(kNone, 0.f);
            mx = fmaxf(mx, v[j].x);
        }
        const float f0 = fast_exp2(m - mx);
        m = mx;
        l *= f0;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] *= f0;
#pragma unroll
        for (int j = 0; j < kJoinPer; ++j) {
            const bool any = v[j].y != 0.f;            // a split that saw no key leaves m only (a NaN sum is kept)
            const float f = any ? fast_exp2(v[j].x - m) : 0.f;
            const float z[8] = {x[j].x, x[j].y, x[j].z, x[j].w, y[j].x, y[j].y, y[j].z, y[j].w};
            l = fmaf(v[j].y, f, l);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = fmaf(any ? z[e] : 0.f, f, o[e]);
        }
    }
    if constexpr (SG > 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[threadIdx.x][e] = o[e];
        ml[threadIdx.x] = make_float2(m, l);
        __syncthreads();
        if (g != 0) return;
        float mx = kNone;
#pragma unroll
        for (int j = 0; j < SG; ++j) mx = fmaxf(mx, ml[threadIdx.x + j * LANES].x);
        l = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = 0.f;
#pragma unroll
        for (int j = 0; j < SG; ++j) {
            const float2 v = ml[threadIdx.x + j * LANES];
            const float f = fast_exp2(v.x - mx);
            l = fmaf(v.y, f, l);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = fmaf(sums[threadIdx.x + j * LANES][e], f, o[e]);
        }
    }
    if (row >= rows) return;
    const float inv = l != 0.f ? 1.f / l : 0.f;        // (no split saw a key: o is 0 too)
    const int bc = static_cast<int>(row / a.rows), r = static_cast<int>(row - static_cast<int64_t>(bc) * a.rows);
    const int b = bc / a.Hkv, c = bc - b * a.Hkv, i = r / a.Gh, h = c * a.Gh + (r - i * a.Gh);
    u32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = pack_bf16(o[2 * j] * inv, o[2 * j + 1] * inv);
    *reinterpret_cast<u32x4*>(a.out + b * a.osb + h * a.osh + i * a.ost + 8 * lane) = v;
}

constexpr int kMaxSplits = 64;             // splits of a head's rows
constexpr int64_t kTileBlocks = 4 * kPlanCus;   // workgroups of many rows, where there are splits

template <int D, int TYPE>
void attend(const ChunkArgs& a, hipStream_t s) {
    const unsigned heads = static_cast<unsigned>(static_cast<int64_t>(a.B) * a.Hkv);
    if (a.rows > kFewRows) {
        const int tiles = (a.rows + kRows - 1) / kRows;
        hipLaunchKernelGGL((chunk_kernel<D, TYPE>), dim3(heads, tiles * a.splits), dim3(kThreads), 0, s, a);
        return;
    }
    const dim3 grid(heads, a.splits);
    constexpr int W = few_waves(D, TYPE, 1);
    if (a.rows <= 16) hipLaunchKernelGGL((chunk_few_kernel<D, TYPE, 1, W>), grid, dim3(64 * W), 0, s, a);
    else if (a.rows <= 32) hipLaunchKernelGGL((chunk_few_kernel<D, TYPE, 2, W>), grid, dim3(64 * W), 0, s, a);
    else hipLaunchKernelGGL((chunk_few_kernel<D, TYPE, 4, 4>), grid, dim3(kThreads), 0, s, a);
}

template <int D>
hipError_t launch(const ChunkArgs& a, hipStream_t s) {
    if (a.pages.dtype == kCacheBf16) attend<D, kCacheBf16>(a, s);
    else if (a.pages.dtype == kCacheE4m3) attend<D, kCacheE4m3>(a, s);
    else attend<D, kCacheI8>(a, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    // a row's splits in one round of loads (kMaxSplits: four of the eight places of 16
    // groups; eight groups took the same time)
    const auto join = [&](auto groups) {
        constexpr int SG = decltype(groups)::value, kPer = kJoinThreads / (D / 8 * SG);
        const int64_t rows = static_cast<int64_t>(a.B) * a.Hkv * a.rows;
        hipLaunchKernelGGL((chunk_join_kernel<D, SG>), dim3(static_cast<unsigned>((rows + kPer - 1) / kPer)),
                           dim3(kJoinThreads), 0, s, a);
    };
    if (a.splits <= kJoinPer) join(Constant<1>{});
    else if (a.splits <= 4 * kJoinPer) join(Constant<4>{});
    else join(Constant<16>{});
    return hipGetLastError();
}

}  // namespace

namespace {

constexpr int kFewBlocks = 4 * kPlanCus;   // workgroups of few rows, where there are splits

// Splits for few rows.  A workgroup has a CU for itself (its LDS; for d = 64 in 8 bits
// and up to 32 rows two fit, which is not priced), so that the launch takes
// as many turns as there are workgroups per CU, each of them 2 us and the rounds
// of its split (a tile for each of its waves); a join reads and writes what the
// splits left beside 3 us for its launch.  (What memory takes for the keys is the
// same for any number.)  A round takes one workgroup, at d = 128 and 16 rows, 0.75
// us for 128 bf16 rows, 1.2 for 256 e4m3 and 1.6 for 256 int8 ones, and more with
// more tiles of 16 rows.  (28 heads on 4, d = 128, bf16, 1 / 6 / 12 / 64 splits: one
// is best at 321 rows, 6.6 us, twelve at 1100, 8.2 against 11.3, 48 or more at
// 16384, 13.8 against 101; for 16 sequences of 16384 rows four, 97 against 105 with
// 2 and 166 with 1; for 32 of 1100 e4m3 rows one, 11.9 against 13.8 with 2.)
int few_splits(int64_t heads, int rows, int T, int d, int dtype) {
    const int keys = d == 128 && dtype == kCacheBf16 ? 32 : 64;
    const int nr = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    int64_t round;
    if (d == 64) round = (dtype == kCacheBf16 ? 340 : dtype == kCacheE4m3 ? 460 : 590) + 140 * nr;
    else if (dtype == kCacheBf16) round = 550 + 200 * nr;
    else if (nr <= 2) round = dtype == kCacheE4m3 ? 1000 + 200 * nr : 1300 + 300 * nr;
    else round = dtype == kCacheE4m3 ? 3000 : 3500;
    const int64_t rounds = (T + 4 * keys - 1) / (4 * keys);
    int64_t best = 0;
    int best_s = 1;
    for (int s = 1; s <= kMaxSplits && s <= rounds && (s == 1 || s * heads <= kFewBlocks); ++s) {
        const int64_t turns = (heads * s + kPlanCus - 1) / kPlanCus;
        const int64_t work = turns * ((rounds + s - 1) / s * round + 2000);
        const int64_t cost = work + (s > 1 ? 3000 + heads * rows * s * d * 2 / 1000 : 0);
        if (s == 1 || cost < best) best = cost, best_s = s;
    }
    return best_s;
}

// Splits for more rows.  In ns, as measured at d = 128 (64): a tile takes a
// workgroup 1500 (950) with a CU to itself, 2000 (1250) beside another, which is
// how they run from one per CU up to two (of d = 64, but for int8, three fit, which
// is not priced); it begins within two tiles' time.  A join reads and writes what the
// splits left (4 TB/s) beside 3000 for its launch.
// (1024 queries of 28 heads on 4 over 8191 rows, 224 row tiles: 197 us with 1 split,
// 142 with 2, 154 with 3; 512 of 32 on 8 over 4096, 128: 98 / 67 / 60 / 56 / 60 us
// with 1 / 2 / 3 / 4 / 6; 1024 of 32 on 8 over 1024, 256: 31 with 1, 40 with 2.)
int tile_splits(int64_t heads, int rows, int T, int d) {
    const int64_t alone = d == 64 ? 950 : 1500, paired = d == 64 ? 1250 : 2000;
    const int64_t base = heads * ((rows + kRows - 1) / kRows), tiles = (T + kKeys - 1) / kKeys;
    int64_t best = 0;
    int best_s = 1;
    for (int s = 1; s <= kMaxSplits && s <= tiles && (s == 1 || base * s <= kTileBlocks); ++s) {
        const int64_t n = base * s, rest = n % (2 * kPlanCus);
        const int64_t turns = n / (2 * kPlanCus) * paired + (rest == 0 ? 0 : rest <= kPlanCus ? alone : paired);
        const int64_t join = s > 1 ? 3000 + heads * rows * s * d * 3 / 1000 : 0;
        const int64_t cost = turns * ((tiles + s - 1) / s + 2) + join;
        if (s == 1 || cost < best) best = cost, best_s = s;
    }
    return best_s;
}

}  // namespace

int chunk_splits(int64_t heads, int rows, int T, int d, int dtype) {
    if (rows <= kFewRows) return few_splits(heads, rows, T, d, dtype);
    return tile_splits(heads, rows, T, d);
}

size_t chunk_workspace_bound(int64_t heads, int rows, int T, int d) {
    // rows of partial sums: splits * heads * rows.  Few rows: kFewBlocks
    // workgroups at most, a split for every 128 keys at most ...
    const int64_t few_s = T / 128 + 1 < kMaxSplits ? T / 128 + 1 : kMaxSplits;
    const int64_t few_b = heads > kFewBlocks / few_s ? kFewBlocks : heads * few_s;
    int64_t part = few_b * (rows < kFewRows ? rows : kFewRows);
    // ... more rows: kTileBlocks workgroups of kRows at most
    if (rows > kFewRows) {
        const int64_t most = T / kKeys + 1 < kMaxSplits ? T / kKeys + 1 : kMaxSplits;
        int64_t tile = heads * rows;
        tile = tile > kTileBlocks * kRows / most ? kTileBlocks * kRows : tile * most;
        if (tile > part) part = tile;
    }
    return static_cast<size_t>(part) * (d * sizeof(float) + sizeof(float2)) + 256;
}

hipError_t launch_chunk_attention(const ChunkArgs& a, hipStream_t s) {
    return a.d == 64 ? launch<64>(a, s) : launch<128>(a, s);
}

}  // namespace mmskv
