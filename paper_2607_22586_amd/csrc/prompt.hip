// Attention of whole prompts over themselves on gfx950 (mmshiftkv_prompt_attention).
//
// The Gh heads that share a KV head are rows of one problem: row r = i * Gh + g is
// token i of head g, so that a workgroup's 128 rows (4 waves of 32) span few tokens
// and its keys end soon behind its own.  It walks the keys from the start of its
// first token's sequence in tiles of 64, staged in LDS for all waves by
// loads straight to it (the next tile's are on their way while one is worked on).  One
// pass with the running reference m and sum l of the softmax, base 2:
//   S^T = K Q^T   (v_mfma_f32_32x32x16_bf16: lane = query row, its values = keys,
//                  so the softmax runs within a lane and its other half-wave)
//   O^T = O^T 2^(m_old - m) + V^T P^T
// P^T is the second product's B operand as it stands in the registers of S^T; V^T
// comes from the staged rows by transposing LDS reads.
// Packed sequences need no plan: a row tile that spans several of them walks the
// keys of all, each row masked to [its sequence's start, its end), both found by
// counting the starts at or before a token.
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
constexpr float kNone = -3e38f;            // reference before the first visible key
// The reference moves, to kLead above the largest logit so far, where a lane's 16
// weights 2^(x - m) add up to kBehind: no weight is above 1 and most tiles form no
// maximum.
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

// Byte of 16-byte chunk ch of row r of a staged tile; the chunks of a row are
// permuted so that the reads of K (16 rows of one chunk) and of V (four rows of 64
// bytes) spread over all banks.
template <int D>
__device__ __forceinline__ int staged(int r, int ch) {
    const int swz = D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    return r * (2 * D) + 16 * (ch ^ swz);
}

// 16 bytes a lane from memory to LDS at dst + 16 * lane.
__device__ __forceinline__ void load_tile16(const char* src, char* dst) {
    __builtin_amdgcn_global_load_lds(src, (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
}

// Whether one of a register's two bf16 values is an infinity or NaN.
__device__ __forceinline__ bool not_finite(uint32_t x) {
    return (x & 0x7F80u) == 0x7F80u || (x & 0x7F800000u) == 0x7F800000u;
}

// The last start at or before a token, and the first behind it.
struct Span {
    int lo, hi;
};

template <int D, bool LSE>
__global__ void __launch_bounds__(kThreads, 2) prompt_kernel(PromptArgs a) {
    constexpr int KC = D / 16;             // 16-dim steps of S
    constexpr int NT = D / 32;             // 32-dim tiles of O
    constexpr int kCh = D / 8;             // 16-byte chunks of a row
    constexpr int kWaveRows = kKeys / kWaves;
    constexpr int kLoads = kWaveRows * 2 * D / 1024;   // 16-byte loads of a lane of K (and of V)
    // (a variable for each stage: the compiler then sees which reads of LDS need not
    // wait for the loads to it that are under way)
    __shared__ __align__(16) char kt0[kKeys * 2 * D], kt1[kKeys * 2 * D], vt0[kKeys * 2 * D], vt1[kKeys * 2 * D];
    __shared__ unsigned long long begins[2];           // tokens of the row tile that begin a sequence
    __shared__ int edge[3];                // last start at or before the tile, first behind it, end of the last sequence
    __shared__ int poisoned[2];            // by buffer: the last tile staged there with values of V that are not finite

    const int bc = blockIdx.x, b = bc / a.Hkv, c = bc - b * a.Hkv;
    const int r0 = static_cast<int>(gridDim.y - 1 - blockIdx.y) * kRows;   // the last rows, which see most keys, first
    const int tid = threadIdx.x, lane = lane_id();
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int half = lane >> 5;
    const int i0 = r0 / a.Gh, i1 = min((r0 + kRows - 1) / a.Gh, a.T - 1);  // tokens of the row tile: at most 128

    // this lane's row and the keys [lo, hi) that it sees; `first`, `last`: tokens of the
    // tile that are in some sequence
    const int r = r0 + 32 * wave + (lane & 31);
    const int i = r / a.Gh, h = c * a.Gh + (r - i * a.Gh);
    int lo = 0, hi = a.T, first = i0, last = i1, lo_first = 0, lo_last = 0, hi_first = a.T, hi_last = a.T;
    if (a.starts) {
        if (tid < 2) begins[tid] = 0;
        if (tid < 3) edge[tid] = tid == 1 ? a.T : tid == 0 ? -1 : 0;
        __syncthreads();
        for (int s = tid; s <= a.n_seq; s += kThreads) {
            const int t = min(max(a.starts[s], 0), a.T);
            if (t <= i0) atomicMax(&edge[0], t);
            else if (t > i1) atomicMin(&edge[1], t);
            else atomicOr(&begins[(t - i0) >> 6], 1ull << ((t - i0) & 63));
            if (s == a.n_seq) edge[2] = t;
        }
        __syncthreads();
        const unsigned long long w0 = begins[0], w1 = begins[1];
        const int before = edge[0], behind = edge[1], end = edge[2];
        const auto span = [&](int t) {     // of token t of the tile
            const int x = t - i0;
            const unsigned long long below0 = x >= 63 ? ~0ull : (2ull << x) - 1;       // bits up to x
            const unsigned long long below1 = x < 64 ? 0ull : x >= 127 ? ~0ull : (2ull << (x - 64)) - 1;
            const unsigned long long p0 = w0 & below0, p1 = w1 & below1, n0 = w0 & ~below0, n1 = w1 & ~below1;
            Span y;
            y.lo = p1 ? i0 + 127 - __builtin_clzll(p1) : p0 ? i0 + 63 - __builtin_clzll(p0) : before;
            y.hi = n0 ? i0 + __builtin_ctzll(n0) : n1 ? i0 + 64 + __builtin_ctzll(n1) : behind;
            return y;
        };
        // tokens before the first start (no start at or before them) are in no sequence
        first = before >= 0 ? i0 : w0 ? i0 + __builtin_ctzll(w0) : w1 ? i0 + 64 + __builtin_ctzll(w1) : i1 + 1;
        last = min(i1, end - 1);
        if (first > last) return;
        const Span y = span(min(max(i, i0), i1)), f = span(first), g = span(last);
        lo = y.lo, hi = y.hi, lo_first = f.lo, hi_first = f.hi, lo_last = g.lo, hi_last = g.hi;
    }
    const bool there = r < a.rows && i >= first && i <= last;
    if (a.causal) hi = i + 1, hi_first = first + 1, hi_last = last + 1;
    const uint32_t sees = there ? hi - lo : 0;
    const int key00 = lo_first;            // the first tile's first key
    const int tiles = (hi_last - key00 + kKeys - 1) / kKeys;
    // tiles [clear0, clear1): every row that is there sees all keys
    const int clear0 = (lo_last - key00 + kKeys - 1) / kKeys, clear1 = (hi_first - key00) / kKeys;

    const uint16_t* const kb = a.k + b * a.ksb + c * a.ksh;
    const uint16_t* const vb = a.v + b * a.vsb + c * a.vsh;
    // A wave stages rows kWaveRows * wave .. of a tile by loads straight to LDS, 1 KB (4
    // rows at d = 128) an instruction; a lane fetches the chunk that its place in the
    // staged order stands for.
    const auto k_tile = [&](auto which) { return decltype(which)::value ? kt1 : kt0; };
    const auto v_tile = [&](auto which) { return decltype(which)::value ? vt1 : vt0; };
    // In-tile offsets of 32 bits beside addresses that the whole wave has in common.
    const int ld_row = lane / kCh;
    uint32_t k_off[kLoads], v_off[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
        const int r = kWaveRows * wave + j * (64 / kCh) + ld_row, ch = staged<D>(r, lane % kCh) - r * 2 * D;
        k_off[j] = 2 * static_cast<uint32_t>(ld_row * a.kst) + ch;
        v_off[j] = 2 * static_cast<uint32_t>(ld_row * a.vst) + ch;
    }
    auto load = [&](int key0, auto which) {
        char* const kd = k_tile(which) + kWaveRows * wave * 2 * D;
        char* const vd = v_tile(which) + kWaveRows * wave * 2 * D;
        const int t0 = key0 + kWaveRows * wave;
        if (t0 + kWaveRows <= a.T) {
            const char* const ks = reinterpret_cast<const char*>(kb + t0 * a.kst);
            const char* const vs = reinterpret_cast<const char*>(vb + t0 * a.vst);
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                load_tile16(ks + j * (64 / kCh) * 2 * a.kst + k_off[j], kd + 1024 * j);
                load_tile16(vs + j * (64 / kCh) * 2 * a.vst + v_off[j], vd + 1024 * j);
            }
        } else {                           // (rows behind the last token: the last, which their mask keeps out)
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int r = j * (64 / kCh) + ld_row;
                const int64_t t = min(t0 + r, a.T - 1), over = t - ld_row;
                load_tile16(reinterpret_cast<const char*>(kb + over * a.kst) + k_off[j], kd + 1024 * j);
                load_tile16(reinterpret_cast<const char*>(vb + over * a.vst) + v_off[j], vd + 1024 * j);
            }
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
    float m = kNone, l = 0.f, l_all = 0.f;             // (l_all: of the weights before their rounding)

    // One tile in two 32-key halves u, as a sequence of steps of one matrix instruction
    // with vector instructions to run beside it: the exponentials of half 0 with the
    // second half's S, those of half 1 with the first half's part of O.  Value e of s[u] is key key0 + 32 u + 8 (e / 4) +
    // 4 half + e % 4.  MASKED: some row does not see all.
    auto attend = [&](int key0, auto which, auto masked) {
        const char* const kt = k_tile(which);
        char* const vt = v_tile(which);
        constexpr bool MASKED = decltype(masked)::value != 0;
        constexpr int N = KC;              // steps of a phase: KC = 2 NT
        constexpr int PAIRS = 8 / N;       // pairs of exponentials of a step
        constexpr int AHEAD = 4;           // steps from a read of LDS to its use
        static_assert(N == 2 * NT, "as many steps in S as in O");
        int ka = staged<D>(lane & 31, half), va = staged<D>(4 * half + ((lane & 15) >> 2), (lane & 16) / 8 + ((lane & 3) >> 1));
        va += 8 * (lane & 1);
        asm volatile("" : "+v"(ka), "+v"(va));         // (formed where they are used, not kept)
        const uint32_t rel = key0 + 4 * half - lo;
        floatx16 s[2];
        auto k_frag = [&](int j) {         // step j % N of half j / N
            return load_bf16x8(reinterpret_cast<const uint16_t*>(kt + j / N * 32 * 2 * D + (ka ^ (32 * (j % N)))));
        };
        auto v_frag = [&](int j) {         // half j / N, step j % N: keys 16 w .., dims 32 t ..
            typedef s16x4 __attribute__((address_space(3))) * lds4;
            const int u = j / N, w = j % N / NT, t = j % NT;
            u32x4 v;
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds4)(vt + (32 * u + 16 * w + 8 * z) * 2 * D + (va ^ (64 * t + 32 * z))));
                const u32x2 y = __builtin_bit_cast(u32x2, x);
                v[2 * z] = y[0];
                v[2 * z + 1] = y[1];
            }
            return __builtin_bit_cast(bf16x8, v);
        };
        auto logit = [&](int u, int e, float less) {
            float x = fmaf(s[u][e], a.scale, -less);
            if (MASKED) x = rel + (32 * u + 8 * (e >> 2) + (e & 3)) < sees ? x : -INFINITY;
            return x;
        };
        // p of values 2 j, 2 j + 1 of half u relative to m, as bf16.  The quotient's sum is
        // of the weights as the product with V takes them, so that what their roundings
        // have in common leaves it; the log-sum-exp's is of the weights before.
        struct Sums {
            float rounded = 0.f, all = 0.f;
        };
        auto pair = [&](int u, int j, Sums& sum) {
            const float x0 = fast_exp2(logit(u, 2 * j, m)), x1 = fast_exp2(logit(u, 2 * j + 1, m));
            const uint32_t y = pack_bf16(x0, x1);
            sum.rounded += __uint_as_float(y << 16) + __uint_as_float(y & 0xFFFF0000u);
            if (LSE) sum.all += x0 + x1;
            return y;
        };
        auto settle = [&](int u, uint32_t (&p)[8], Sums sum) {
            if (__any(!(sum.rounded < kBehind))) {
                float mx = kNone;
#pragma unroll
                for (int e = 0; e < 16; ++e) mx = fmaxf(mx, logit(u, e, 0.f));
                mx = fmaxf(half_max(mx) + kLead, m);
                const float f = fast_exp2(m - mx);
                m = mx;
                l *= f;
                l_all *= f;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[t][j] *= f;
                sum = Sums{};
#pragma unroll
                for (int j = 0; j < 8; ++j) p[j] = pair(u, j, sum);
            }
            l += sum.rounded;
            l_all += sum.all;
        };
        auto p_frag = [](const uint32_t (&p)[8], int w) {
            return __builtin_bit_cast(bf16x8, (u32x4{p[4 * w], p[4 * w + 1], p[4 * w + 2], p[4 * w + 3]}));
        };
        const auto fence = [] { __builtin_amdgcn_sched_barrier(0); };

        bf16x8 f[2 * N];
        uint32_t p0[8], p1[8];
        Sums sum;
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) f[j] = k_frag(j);
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
        sum = Sums{};
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
        }
        fence();
    };

    // A key that a row does not see must not reach it, but 0 times an infinity or NaN
    // in its V would.  Tiles that some row sees in part are looked over as they are
    // staged; values that are not finite become zeros there, and are added by hand to
    // the rows that see them (whose results are then not finite whatever the weight).
    auto clean = [&](int tile, auto which) {           // (a wave: of what it has staged itself)
        char* const at = v_tile(which) + kWaveRows * wave * 2 * D + 16 * lane;
        u32x4 x[kLoads];
        bool bad = false;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            x[j] = *reinterpret_cast<const u32x4*>(at + 1024 * j);
#pragma unroll
            for (int e = 0; e < 4; ++e) bad |= not_finite(x[j][e]);
        }
        if (!__any(bad)) return;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if ((x[j][e] & 0x7F80u) == 0x7F80u) x[j][e] &= 0xFFFF0000u;
                if ((x[j][e] & 0x7F800000u) == 0x7F800000u) x[j][e] &= 0xFFFFu;
            }
            *reinterpret_cast<u32x4*>(at + 1024 * j) = x[j];
        }
        poisoned[decltype(which)::value] = tile;
    };
    auto add_poison = [&](int key0) {
        for (int x = 0; x < kKeys; ++x) {
            const int64_t t = min(key0 + x, a.T - 1);
            const bool seen = static_cast<uint32_t>(key0 + x - lo) < sees;
            const uint16_t* const row = vb + t * a.vst + 4 * half;
            u32x2 v[4 * NT];
#pragma unroll
            for (int d = 0; d < 4 * NT; ++d) v[d] = *reinterpret_cast<const u32x2*>(row + 8 * d);
#pragma unroll
            for (int d = 0; d < NT; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const uint32_t w = v[4 * d + (e >> 2)][(e & 3) >> 1], y = e & 1 ? w & 0xFFFF0000u : w << 16;
                    if (seen && (y & 0x7F800000u) == 0x7F800000u) o[d][e] += __uint_as_float(y);
                }
        }
    };

    // The tiles that some row sees in part first (those before the clear ones, then those
    // behind: the rows' own keys, whose logits are likely large), each half of them in a
    // loop of its own.  The stages take turns so that the clear ones begin with stage 0.
    const int masked = tiles - max(clear1 - clear0, 0), ahead = min(clear0, masked);
    const auto key_of = [&](int n) {       // first key of the n-th tile worked on
        const int tile = n < ahead ? n : n < masked ? n + (tiles - masked) : n - masked + ahead;
        return key00 + tile * kKeys;
    };
    auto step = [&](int n, auto which, auto part) {
        constexpr int W = decltype(which)::value;
        if (n + 1 < tiles) load(key_of(n + 1), Constant<1 - W>{});
        attend(key_of(n), which, part);
        if (decltype(part)::value && poisoned[W] == n) add_poison(key_of(n));
        wait_vm<0>();
        if (decltype(part)::value && n + 1 < masked) clean(n + 1, Constant<1 - W>{});
        __syncthreads();
    };
    if (tid < 2) poisoned[tid] = -1;
    __syncthreads();
    if (masked & 1) {
        load(key_of(0), Constant<1>{});
        wait_vm<0>();
        clean(0, Constant<1>{});
    } else {
        load(key_of(0), Constant<0>{});
        wait_vm<0>();
        if (masked) clean(0, Constant<0>{});
    }
    __syncthreads();
    int n = 0;
    if (masked & 1) step(n++, Constant<1>{}, Constant<1>{});
    while (n < masked) {
        step(n++, Constant<0>{}, Constant<1>{});
        step(n++, Constant<1>{}, Constant<1>{});
    }
    while (n < tiles) {
        step(n++, Constant<0>{}, Constant<0>{});
        if (n < tiles) step(n++, Constant<1>{}, Constant<0>{});
    }
    l = half_sum(l);
    if (LSE) l_all = half_sum(l_all);
    if (!there) return;
    const float inv = 1.f / l;
    uint16_t* out = a.out + b * a.osb + h * a.osh + i * a.ost + 4 * half;
    // value 4 w + j of o[t] is dim 32 t + 8 w + 4 half + j
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int w = 0; w < 4; ++w)
            *reinterpret_cast<u32x2*>(out + 32 * t + 8 * w) =
                u32x2{pack_bf16(o[t][4 * w] * inv, o[t][4 * w + 1] * inv),
                      pack_bf16(o[t][4 * w + 2] * inv, o[t][4 * w + 3] * inv)};
    if (LSE && half == 0)
        a.lse[(static_cast<int64_t>(b) * a.Hq + h) * a.T + i] = (m + __builtin_amdgcn_logf(l_all)) * 0.6931471805599453f;
}

}  // namespace

hipError_t launch_prompt_attention(const PromptArgs& a, hipStream_t s) {
    const dim3 grid(static_cast<unsigned>(a.B * a.Hkv), (a.rows + kRows - 1) / kRows);
    if (a.d == 64 && a.lse) hipLaunchKernelGGL((prompt_kernel<64, true>), grid, dim3(kThreads), 0, s, a);
    else if (a.d == 64) hipLaunchKernelGGL((prompt_kernel<64, false>), grid, dim3(kThreads), 0, s, a);
    else if (a.lse) hipLaunchKernelGGL((prompt_kernel<128, true>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((prompt_kernel<128, false>), grid, dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace mmskv
