// Attention of whole prompts over themselves on gfx950 (mmshiftkv_prompt_attention).
//
// The Gh heads that share a KV head are rows of one problem: row r = i * Gh + g is
// token i of head g, so that a workgroup's 128 rows (4 waves of 32; 256 where sequences
// are long) span few tokens and its keys end soon behind its own.  It walks the keys
// from the start of its first token's sequence in tiles of 64, staged in LDS for all
// waves by loads straight to it (the next tile's are on their way while one is worked
// on).  One pass with the running reference m and sum l of the softmax, base 2:
//   S^T = K Q^T   (v_mfma_f32_32x32x16_bf16: lane = query row, its values = keys,
//                  so the softmax runs within a lane and its other half-wave)
//   O^T = O^T 2^(m_old - m) + V^T P^T
// P^T is the second product's B operand as it stands in the registers of S^T; V^T
// comes from the staged rows by transposing LDS reads.
// Packed sequences need no plan: a row tile that spans several of them walks the
// keys of all, each row masked to [its sequence's start, its end), both found by
// counting the starts at or before a token.
// What bounds it: at d = 128 no pipe alone.  Counters show the matrix pipe busy for 53 to
// 56% of the cycles, the vector one for 57%, 30% of a wave's cycles spent waiting, with two
// waves a SIMD, and a clock of 1.77 to 1.9 GHz (4 x 28 heads of 16384 tokens on 4, causal:
// 6.9 to 7.4 ms, 1040 to 1119 TFLOP/s, card to card; a bf16 product of 8192^3 reaches 1219
// to 1389).  That fits latencies (of LDS, and from product to exponential to product) that two
// waves do not cover, and a clock set by power: fewer vector instructions alone change
// nothing, fewer reads of the tiles do.  At d = 64 the vector pipe: as many exponentials
// for half the products (4 x 16 heads of 8192 tokens 890 to 910 TFLOP/s).  Short
// sequences: a chain of latencies, 5 us for one token, 1.2 us more for every tile of 64
// keys at d = 128 and 0.9 at 64.
#include "pages.hpp"

namespace mmskv {
namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// (lambdas of a kernel's registers that are called in several places)
#define kInline __attribute__((always_inline))

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

// sum + the two bf16 values of y, by one instruction (DOT) or two additions: the vector
// pipe bounds d = 64 (images of 16 heads 203 -> 195 us by the instruction), at d = 128 the
// additions let the clock be higher (7.26 against 7.36 ms).
template <bool DOT>
__device__ __forceinline__ float add_pair(uint32_t y, float sum) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    if constexpr (!DOT) return sum + (__uint_as_float(y << 16) + __uint_as_float(y & 0xFFFF0000u));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, y), __builtin_bit_cast(bf16x2, 0x3F803F80u), sum,
                                           false);
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

// Workgroup: WAVES waves, GROUPS of them with the same 32 rows, each with 64 keys of a
// tile of its own; their sums are joined at the end.
template <int D, bool LSE, int WAVES, int GROUPS>
__global__ void __launch_bounds__(64 * WAVES, 2) prompt_kernel(PromptArgs a) {
    constexpr int kWaves = WAVES, kThreads = 64 * WAVES;
    constexpr int kRows = 32 * WAVES / GROUPS;         // query rows of a workgroup
    constexpr int kTile = kKeys * GROUPS;              // keys of a tile
    constexpr int kWords = kRows / 64;
    constexpr int KC = D / 16;             // 16-dim steps of S
    constexpr int NT = D / 32;             // 32-dim tiles of O
    constexpr int kCh = D / 8;             // 16-byte chunks of a row
    constexpr int kWaveRows = kTile / kWaves;
    constexpr int kLoads = kWaveRows * 2 * D / 1024;   // 16-byte loads of a lane of K (and of V)
    // (a variable for each stage: the compiler then sees which reads of LDS need not
    // wait for the loads to it that are under way)
    __shared__ __align__(16) char kt0[kTile * 2 * D], kt1[kTile * 2 * D], vt0[kTile * 2 * D], vt1[kTile * 2 * D];
    __shared__ unsigned long long begins[kWords];      // tokens of the row tile that begin a sequence
    __shared__ int edge[3];                // last start at or before the tile, first behind it, end of the last sequence
    __shared__ int poisoned[2];            // by buffer: the last tile staged there with values of V that are not finite

    // Consecutive workgroups are on different XCDs.  Of long sequences each XCD has a KV
    // head of its own with all row tiles, as long as there are eight heads, so that its
    // cache serves them the same keys (4 x 32 heads of 8192 tokens on 32: 2.47 -> 2.19
    // ms); the heads that are left are shared by all.  Of shorter ones all heads' long
    // rows come first (32 heads of 4096 on 32: 164 us, by head 184).
    const uint32_t heads = a.B * a.Hkv, row_tiles = (a.rows + kRows - 1) / kRows;
    const uint32_t alone = a.by_head ? heads / 8 * 8 : 0, shared = heads - alone;
    const uint32_t own = alone / 8 * row_tiles;        // workgroups of an XCD with heads of its own
    const bool behind_cut = a.cut && blockIdx.x < heads * row_tiles;
    const uint32_t x = a.cut && !behind_cut ? blockIdx.x - heads * row_tiles : blockIdx.x;
    const uint32_t turn = x / 8, rest = x - 8 * own;
    const uint32_t bc = turn < own ? x % 8 + turn / row_tiles * 8 : alone + rest % shared;
    const int b = bc / a.Hkv, c = bc - b * a.Hkv;
    // the last rows, which see most keys, first
    const int r0 = (row_tiles - 1 - (turn < own ? turn % row_tiles : rest / shared)) * kRows;
    const int tid = threadIdx.x, lane = lane_id();
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int half = lane >> 5;
    const int rows32 = wave % (kWaves / GROUPS), group = wave / (kWaves / GROUPS);
    const int i0 = r0 / a.Gh, i1 = min((r0 + kRows - 1) / a.Gh, a.T - 1);  // tokens of the row tile

    // this lane's row and the keys [lo, hi) that it sees; `first`, `last`: tokens of the
    // tile that are in some sequence
    const int r = r0 + 32 * rows32 + (lane & 31);
    const int i = r / a.Gh, h = c * a.Gh + (r - i * a.Gh);
    int lo = 0, hi = a.T, first = i0, last = i1, lo_first = 0, lo_last = 0, hi_first = a.T, hi_last = a.T;
    if (a.starts) {
        if (tid < kWords) begins[tid] = 0;
        if (tid < 3) edge[tid] = tid == 1 ? a.T : tid == 0 ? -1 : 0;
        const auto start = [&](int s) { return min(max(a.starts[s], 0), a.T); };
        // of many starts those between the last of kThreads samples at or before the tile
        // and the first behind it (they ascend)
        int s0 = 0, s1 = a.n_seq;
        if (a.n_seq >= 4 * kThreads) {
            const int step = a.n_seq / kThreads + 1, t = start(min(tid * step, a.n_seq));
            const int before = __syncthreads_count(t <= i0), upto = __syncthreads_count(t <= i1);
            s0 = max(before - 1, 0) * step;
            if (upto < kThreads) s1 = min(upto * step, a.n_seq);
        } else {
            __syncthreads();
        }
        for (int s = s0 + tid; s <= s1; s += kThreads) {
            const int t = start(s);
            if (t <= i0) atomicMax(&edge[0], t);
            else if (t > i1) atomicMin(&edge[1], t);
            else atomicOr(&begins[(t - i0) >> 6], 1ull << ((t - i0) & 63));
        }
        if (tid == 0) edge[2] = start(a.n_seq);
        __syncthreads();
        unsigned long long word[kWords];
#pragma unroll
        for (int w = 0; w < kWords; ++w) word[w] = begins[w];
        const int before = edge[0], behind = edge[1], end = edge[2];
        const auto span = [&](int t) {     // of token t of the tile
            Span y{before, behind};
#pragma unroll
            for (int w = 0; w < kWords; ++w) {         // the bits up to t, and those behind
                const int x = t - i0 - 64 * w;
                const unsigned long long upto = x < 0 ? 0ull : x >= 63 ? ~0ull : (2ull << x) - 1;
                if (word[w] & upto) y.lo = i0 + 64 * w + 63 - __builtin_clzll(word[w] & upto);
            }
#pragma unroll
            for (int w = kWords - 1; w >= 0; --w) {
                const int x = t - i0 - 64 * w;
                const unsigned long long upto = x < 0 ? 0ull : x >= 63 ? ~0ull : (2ull << x) - 1;
                if (word[w] & ~upto) y.hi = i0 + 64 * w + __builtin_ctzll(word[w] & ~upto);
            }
            return y;
        };
        // tokens before the first start (no start at or before them) are in no sequence
        if (before < 0) first = i1 + 1;
#pragma unroll
        for (int w = kWords - 1; w >= 0; --w)
            if (before < 0 && word[w]) first = i0 + 64 * w + __builtin_ctzll(word[w]);
        last = min(i1, end - 1);
        if (first > last) return;
        Span f = span(first), g = span(last);
        // The rows of one tile walk the keys of all its sequences, none of which all rows
        // see.  Without causality, where the first has many keys before the tile or the last
        // behind it, two workgroups have the rows before and behind that cut: the longest
        // walk is no longer that of two sequences (images of 4041 patches and six smaller
        // ones, 16 heads of 64: 198 -> 154 us; causal rows gain nothing by it).
        constexpr int kApart = 256;
        if (a.cut) {
            const int cut = f.hi <= last && i0 - f.lo >= kApart ? f.hi
                            : g.lo > first && g.hi - i1 > kApart ? g.lo : last + 1;
            if (behind_cut) first = cut;
            else last = cut - 1;
            if (first > last) return;
            f = span(first), g = span(last);
        }
        const Span y = span(min(max(i, i0), i1));
        lo = y.lo, hi = y.hi, lo_first = f.lo, hi_first = f.hi, lo_last = g.lo, hi_last = g.hi;
    }
    const bool there = r < a.rows && i >= first && i <= last;
    if (a.causal) hi = i + 1, hi_first = first + 1, hi_last = last + 1;
    const uint32_t sees = there ? hi - lo : 0;
    const int key00 = lo_first;            // the first tile's first key
    const int tiles = (hi_last - key00 + kTile - 1) / kTile;
    // tiles [clear0, clear1): every row that is there sees all keys
    const int clear0 = (lo_last - key00 + kTile - 1) / kTile, clear1 = (hi_first - key00) / kTile;

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
    auto load = [&](const uint16_t* base, int64_t stride, const uint32_t (&off)[kLoads], int key0, char* tile) kInline {
        char* const to = tile + kWaveRows * wave * 2 * D;
        const int t0 = key0 + kWaveRows * wave;
        if (t0 + kWaveRows <= a.T) {
            const char* const src = reinterpret_cast<const char*>(base + t0 * stride);
#pragma unroll
            for (int j = 0; j < kLoads; ++j) load_tile16(src + j * (64 / kCh) * 2 * stride + off[j], to + 1024 * j);
        } else {                           // (rows behind the last token: the last, which their mask keeps out)
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int64_t t = min(t0 + j * (64 / kCh) + ld_row, a.T - 1) - ld_row;
                load_tile16(reinterpret_cast<const char*>(base + t * stride) + off[j], to + 1024 * j);
            }
        }
    };
    const auto load_k = [&](int key0, auto which) kInline { load(kb, a.kst, k_off, key0, k_tile(which)); };
    const auto load_v = [&](int key0, auto which) kInline { load(vb, a.vst, v_off, key0, v_tile(which)); };

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

    // The keys are worked on in halves of a tile, 32 at a time, as a sequence of steps,
    // each with a matrix instruction of the next half's S, one of the part that the half
    // before has in O, and this half's exponentials beside them: the matrix pipe and the
    // vector one have about the same to do in every step.  (Left to itself the compiler
    // puts the matrix instructions of a phase first, and a SIMD's two waves do not fill
    // the gaps.)  Value e of a lane's s is key key0 + 8 (e / 4) + 4 half + e % 4.
    // MASKED: some row does not see all keys.
    floatx16 s[2];                         // of this half and the next, in turn
    uint32_t p[2][8];                      // weights of this half and the one before, pairs of bf16
#pragma unroll
    for (int j = 0; j < 8; ++j) p[1][j] = 0;
    const int ka0 = staged<D>(lane & 31, half);
    const int va0 = staged<D>(4 * half + ((lane & 15) >> 2), (lane & 16) / 8 + ((lane & 3) >> 1)) + 8 * (lane & 1);
    auto k_frag = [&](const char* kt, int ka, int j) kInline {             // dims 16 j ..
        return load_bf16x8(reinterpret_cast<const uint16_t*>(kt + (ka ^ (32 * j))));
    };
    auto v_frag = [&](char* vt, int va, int j) kInline {                   // keys 16 w .., dims 32 t ..
        typedef s16x4 __attribute__((address_space(3))) * lds4;
        const int w = j / NT, t = j % NT;
        u32x4 v;
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            const s16x4 x =
                __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(vt + (16 * w + 8 * z) * 2 * D + (va ^ (64 * t + 32 * z))));
            const u32x2 y = __builtin_bit_cast(u32x2, x);
            v[2 * z] = y[0];
            v[2 * z + 1] = y[1];
        }
        return __builtin_bit_cast(bf16x8, v);
    };
    auto p_frag = [](const uint32_t (&x)[8], int w) kInline {
        return __builtin_bit_cast(bf16x8, (u32x4{x[4 * w], x[4 * w + 1], x[4 * w + 2], x[4 * w + 3]}));
    };
    const auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
    // which: this half's place in s and p; kt, vt: the next half's K, the V of the one before
    auto attend = [&](int key0, auto which, auto masked, const char* kt, char* vt) kInline {
        constexpr int U = decltype(which)::value;
        constexpr bool MASKED = decltype(masked)::value != 0;
        constexpr int N = KC;              // steps: KC of S, 2 NT of O
        constexpr int PAIRS = 8 / N;       // pairs of exponentials of a step
        constexpr int AHEAD = 2;           // steps from a read of LDS to its use
        static_assert(N == 2 * NT, "as many steps in S as in O");
        int ka = ka0, va = va0;
        asm volatile("" : "+v"(ka), "+v"(va));         // (permuted addresses are formed where they are used, not kept)
        const uint32_t rel = key0 + 4 * half - lo;
        auto logit = [&](int e, float less) kInline {
            float x = fmaf(s[U][e], a.scale, -less);
            if (MASKED) x = rel + (8 * (e >> 2) + (e & 3)) < sees ? x : -INFINITY;
            return x;
        };
        // Weights of values 2 j, 2 j + 1 relative to m, as bf16.  The quotient's sum is of
        // the weights as the product with V takes them, so that what their roundings have
        // in common leaves it; the log-sum-exp's is of the weights before.
        float sum = 0.f, sum_all = 0.f;
        auto pair = [&](int j) kInline {
            const float x0 = fast_exp2(logit(2 * j, m)), x1 = fast_exp2(logit(2 * j + 1, m));
            const uint32_t y = pack_bf16(x0, x1);
            sum = add_pair<D == 64>(y, sum);
            if (LSE) sum_all += x0 + x1;
            p[U][j] = y;
        };
        bf16x8 fk[N], fv[N];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) fk[j] = k_frag(kt, ka, j), fv[j] = v_frag(vt, va, j);
#pragma unroll
        for (int e = 0; e < 16; ++e) s[1 - U][e] = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            fence();
            if (j + AHEAD < N) fk[j + AHEAD] = k_frag(kt, ka, j + AHEAD), fv[j + AHEAD] = v_frag(vt, va, j + AHEAD);
            s[1 - U] = mfma32(fk[j], qf[j], s[1 - U]);
            o[j % NT] = mfma32(fv[j], p_frag(p[1 - U], j / NT), o[j % NT]);
#pragma unroll
            for (int z = 0; z < PAIRS; ++z) pair(j * PAIRS + z);
        }
        fence();
        if (__any(!(sum < kBehind))) {     // the reference moves
            float mx = kNone;
#pragma unroll
            for (int e = 0; e < 16; ++e) mx = fmaxf(mx, logit(e, 0.f));
            mx = fmaxf(half_max(mx) + kLead, m);
            const float f = fast_exp2(m - mx);
            m = mx;
            l *= f;
            l_all *= f;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int j = 0; j < 16; ++j) o[t][j] *= f;
            sum = sum_all = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) pair(j);
        }
        l += sum;
        l_all += sum_all;
        fence();
    };

    // A key that a row does not see must not reach it, but 0 times an infinity or NaN
    // in its V would.  Tiles that some row sees in part are looked over as they are
    // staged; values that are not finite become zeros there, and are added by hand to
    // the rows that see them (whose results are then not finite whatever the weight).
    auto clean = [&](int tile, auto which) kInline {           // (a wave: of what it has staged itself)
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
    auto add_poison = [&](int key0) kInline {
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
        return key00 + tile * kTile;
    };
    // Tile n, in stage W: K of the next tile and V of this one have landed by the middle
    // of it, where the stages of K of this tile and V of the one before are free again.
    constexpr int kHalf = kKeys / 2 * 2 * D;
    const int mine = group * kKeys;        // this wave's keys of a tile
    auto step = [&](int n, auto which, auto part) kInline {
        constexpr int W = decltype(which)::value;
        const int key0 = key_of(n) + mine, at = mine * 2 * D;
        attend(key0, Constant<0>{}, part, k_tile(which) + at + kHalf, v_tile(Constant<1 - W>{}) + at + kHalf);
        wait_vm<0>();
        if (decltype(part)::value) clean(n, which);
        __syncthreads();
        if (n + 2 < tiles) load_k(key_of(n + 2), which);
        if (n + 1 < tiles) load_v(key_of(n + 1), Constant<1 - W>{});
        attend(key0 + kKeys / 2, Constant<1>{}, part, k_tile(Constant<1 - W>{}) + at, v_tile(which) + at);
        if (decltype(part)::value && poisoned[W] == n) add_poison(key0);
    };
    // before the first tile, in stage W: its first half's S, and no weights for the half
    // before, whose V are zeros
    auto begin = [&](auto which) kInline {
        constexpr int W = decltype(which)::value;
        load_k(key_of(0), which);
        char* const vt = v_tile(Constant<1 - W>{});
        for (int x = 16 * tid; x < kTile * 2 * D; x += 16 * kThreads) *reinterpret_cast<u32x4*>(vt + x) = u32x4{0u, 0u, 0u, 0u};
        wait_vm<0>();
        __syncthreads();
        if (tiles > 1) load_k(key_of(1), Constant<1 - W>{});
        load_v(key_of(0), which);
#pragma unroll
        for (int e = 0; e < 16; ++e) s[0][e] = 0.f;
#pragma unroll
        for (int j = 0; j < KC; ++j) s[0] = mfma32(k_frag(k_tile(which) + mine * 2 * D, ka0, j), qf[j], s[0]);
    };
    auto end = [&](auto which) kInline {           // the last half's part of O, of the tile in stage W
#pragma unroll
        for (int j = 0; j < KC; ++j)
            o[j % NT] = mfma32(v_frag(v_tile(which) + mine * 2 * D + kHalf, va0, j), p_frag(p[1], j / NT), o[j % NT]);
    };
    if (tid < 2) poisoned[tid] = -1;       // (seen by all behind the barriers of begin)
    int n = 0;
    if (masked & 1) {
        begin(Constant<1>{});
        step(n++, Constant<1>{}, Constant<1>{});
    } else {
        begin(Constant<0>{});
    }
    while (n < masked) {
        step(n++, Constant<0>{}, Constant<1>{});
        step(n++, Constant<1>{}, Constant<1>{});
    }
    while (n + 1 < tiles) {
        step(n++, Constant<0>{}, Constant<0>{});
        step(n++, Constant<1>{}, Constant<0>{});
    }
    if (n < tiles) {
        step(n++, Constant<0>{}, Constant<0>{});
        end(Constant<0>{});
    } else {
        end(Constant<1>{});
    }
    l = half_sum(l);
    if (LSE) l_all = half_sum(l_all);
    if constexpr (GROUPS > 1) {
        // the groups' sums to the first one, a float of every lane side by side, by way of
        // the stages
        __syncthreads();                   // (the last tile has been read)
        constexpr int kOne = (16 * NT + 4) * 256, kAll = (GROUPS - 1) * (kWaves / GROUPS), kPer = kTile * 2 * D / kOne;
        static_assert(kPer >= 1 && kAll <= 4 * kPer, "the sums of the other groups fit the stages");
        const auto place = [&](int g) kInline {
            const int x = (g - 1) * (kWaves / GROUPS) + rows32;
            char* const stage = x < kPer ? kt0 : x < 2 * kPer ? kt1 : x < 3 * kPer ? vt0 : vt1;
            return reinterpret_cast<float*>(stage + x % kPer * kOne) + lane;
        };
        if (group > 0) {
            float* const to = place(group);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int j = 0; j < 16; ++j) to[64 * (16 * t + j)] = o[t][j];
            to[64 * 16 * NT] = m, to[64 * (16 * NT + 1)] = l, to[64 * (16 * NT + 2)] = l_all;
        }
        __syncthreads();
        if (group == 0) {
#pragma unroll
            for (int g = 1; g < GROUPS; ++g) {
                const float* const from = place(g);
                const float m1 = from[64 * 16 * NT], most = fmaxf(m, m1);
                const float f0 = fast_exp2(m - most), f1 = fast_exp2(m1 - most);
                m = most;
                l = l * f0 + from[64 * (16 * NT + 1)] * f1;
                l_all = l_all * f0 + from[64 * (16 * NT + 2)] * f1;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[t][j] = o[t][j] * f0 + from[64 * (16 * t + j)] * f1;
            }
        }
    }
    if (LSE && there && group == 0 && half == 0)
        a.lse[(static_cast<int64_t>(b) * a.Hq + h) * a.T + i] = (m + __builtin_amdgcn_logf(l_all)) * 0.6931471805599453f;
    // Results by way of LDS, so that a store writes whole rows: a wave's 32 rows, their
    // chunks permuted by the row.  Value 4 w + j of o[t] is dim 32 t + 8 w + 4 half + j.
    const float inv = 1.f / l;
    const int64_t to = there ? b * a.osb + h * a.osh + i * a.ost : -1;     // this lane's row
    __syncthreads();                       // (the last tile, or the sums, have been read)
    if (group > 0) return;
    static_assert(kRows <= 4 * kTile, "the rows fit the stages");
    const int place = 32 * rows32 / kTile;
    char* const rows = (place == 0 ? kt0 : place == 1 ? kt1 : place == 2 ? vt0 : vt1) + 32 * rows32 % kTile * 2 * D;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int w = 0; w < 4; ++w)
            *reinterpret_cast<u32x2*>(rows + (lane & 31) * 2 * D + 16 * ((4 * t + w) ^ (lane & (kCh - 1))) + 8 * half) =
                u32x2{pack_bf16(o[t][4 * w] * inv, o[t][4 * w + 1] * inv),
                      pack_bf16(o[t][4 * w + 2] * inv, o[t][4 * w + 3] * inv)};
#pragma unroll
    for (int j = 0; j < 32; j += kWave / kCh) {
        const int row = j + lane / kCh, ch = lane % kCh;
        const u32x4 y = *reinterpret_cast<const u32x4*>(rows + row * 2 * D + 16 * (ch ^ (row & (kCh - 1))));
        const int64_t at = __shfl(to, row);
        if (at >= 0) *reinterpret_cast<u32x4*>(a.out + at + 8 * ch) = y;
    }
}

}  // namespace

hipError_t launch_prompt_attention(const PromptArgs& args, hipStream_t s) {
    PromptArgs a = args;
    const int mean = a.T / (a.starts ? a.n_seq : 1);   // tokens of a sequence
    a.by_head = mean >= 8192;
    a.cut = a.starts && !a.causal && mean >= 512;
    const auto workgroups = [&](int rows) { return static_cast<int64_t>(a.B) * a.Hkv * ((a.rows + rows - 1) / rows); };
    const auto run = [&](auto d, auto waves, auto groups) {
        constexpr int D = decltype(d)::value, W = decltype(waves)::value, G = decltype(groups)::value;
        const dim3 grid(static_cast<unsigned>(workgroups(32 * W / G) * (a.cut ? 2 : 1)));
        if (a.lse) hipLaunchKernelGGL((prompt_kernel<D, true, W, G>), grid, dim3(64 * W), 0, s, a);
        else hipLaunchKernelGGL((prompt_kernel<D, false, W, G>), grid, dim3(64 * W), 0, s, a);
    };
    // Eight waves fetch a tile for twice the rows, which at d = 128 lets the matrix pipe
    // run at a higher clock (4 x 28 heads of 16384 tokens 7.3 -> 7.1 ms); four have twice
    // the workgroups, and less beside the diagonal (of 2048 tokens 149 us against 157).
    // At d = 64 and with few workgroups, waves with keys of their own shorten what each
    // does in turn by more than the join takes (16 heads on 2, four groups / none: 512
    // tokens 9.9 / 11.4 us, 1024 13.2 / 19.9; two groups of eight waves, 2048 28 / 34; of
    // four, 256 7.2 / 8.1, 64 6.0 / 5.5; 8 heads, 23 sequences in 3001 tokens 13.3 / 15.4;
    // at d = 128 28 heads on 4 of 1024 24.7 / 26, of 512 16.1 / 15.9).
    if (a.d == 64) {
        const int64_t wide = workgroups(128), narrow = workgroups(64);
        if (mean >= 512 && narrow <= kPlanCus) run(Constant<64>{}, Constant<8>{}, Constant<4>{});
        else if (mean >= 512 && wide <= kPlanCus) run(Constant<64>{}, Constant<8>{}, Constant<2>{});
        else if (mean >= 96 && narrow <= 2 * kPlanCus) run(Constant<64>{}, Constant<4>{}, Constant<2>{});
        else run(Constant<64>{}, Constant<4>{}, Constant<1>{});
    } else {
        if (a.by_head) run(Constant<128>{}, Constant<8>{}, Constant<1>{});
        else run(Constant<128>{}, Constant<4>{}, Constant<1>{});
    }
    return hipGetLastError();
}

}  // namespace mmskv
