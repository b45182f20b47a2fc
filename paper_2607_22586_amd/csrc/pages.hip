// Pages of a paged cache given, taken and copied on gfx950
// (mmshiftkv_cache_hold, _fork, _compact and mmshiftkv_shared_table).  The numbers of rows are the
// device's (a selection leaves them there), so the pages are assigned there too,
// without a wait of the host:
//   count  what each sequence wants, the free pages of the pool as bits and by chunk, a
//          copy of the table and the lengths as they were;
//   plan   each sequence's new row of the table, and the counters by the difference of
//          the two.  The pages wanted are ranked by sequence and entry, the free ones by
//          number, and rank r gets the r-th free page: the outcome does not depend on the
//          order of workgroups;
//   copy   the rows that a fork or a compaction copies: a unit of work is one head of one
//          new page.
// For small pools and tables one workgroup does the first two (a launch less: 3 us of the
// host's time and of the GPU's; 4 to 5 us for 768 entries, 12 for 5000, which the two
// kernels take 8 for).  They are bound by latency, the copies by HBM: 56 forks' tails of
// 8 heads of e4m3 rows, 132 MB, 18.5 us; a quarter of 8 x 8 heads of up to 32768 bf16
// rows, 345 MB, 66 us.
#include "pages.hpp"

namespace mmskv {
namespace {

constexpr int kBookThreads = 256;
constexpr int kChunk = kBookChunk;

__device__ __forceinline__ bool named(const Pages& p, int id) {
    return static_cast<uint32_t>(id) < static_cast<uint32_t>(p.n_pages);
}

// Inclusive prefix sum over a workgroup of kBookThreads, and its total.
__device__ __forceinline__ int block_scan(int x, int* lds, int* total) {
    const int wave = threadIdx.x / kWave;
    x = wave_incl_scan(x);
    __syncthreads();                       // (lds may still be read)
    if (lane_id() == kWave - 1) lds[wave] = x;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kBookThreads / kWave; ++w) {
        before += w < wave ? lds[w] : 0;
        all += lds[w];
    }
    *total = all;
    return x + before;
}

struct Extent {
    int most, least;
};

// Largest and smallest of a sequence's numbers of rows, over a wave.
__device__ __forceinline__ Extent wave_extent(const int32_t* rows, int Hkv, int first, int step) {
    int most = INT32_MIN, least = INT32_MAX;
    for (int c = first; c < Hkv; c += step) {
        const int n = rows[c];
        most = max(most, n);
        least = min(least, n);
    }
#pragma unroll
    for (int s = kWave / 2; s > 0; s /= 2) {
        most = max(most, __shfl_xor(most, s));
        least = min(least, __shfl_xor(least, s));
    }
    return {most, least};
}
// The same over a workgroup (every thread gets them).
__device__ __forceinline__ Extent extent(const int32_t* rows, int Hkv, int* lds) {
    Extent e = wave_extent(rows, Hkv, threadIdx.x, kBookThreads);
    __syncthreads();
    if (lane_id() == 0) lds[2 * (threadIdx.x / kWave)] = e.most, lds[2 * (threadIdx.x / kWave) + 1] = e.least;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kBookThreads / kWave; ++w) e = {max(e.most, lds[2 * w]), min(e.least, lds[2 * w + 1])};
    return e;
}

// What a call makes of a sequence's row of the table: entries j < keep as those of
// sequence `from`, new pages for the entries keep <= j < end (hold: for those j < end
// that name none; fork: for those that name one), none behind.
struct Change {
    int from, keep, end;
    bool moves;
};

// (extent_of: the extent of a sequence's numbers of rows)
template <int OP, class EXTENT>
__device__ __forceinline__ Change change_of(const BookArgs& a, int b, const int32_t* lens, EXTENT&& extent_of) {
    const auto pages_of = [&](int rows) { return (min(max(rows, 0), a.pages.cap) + (1 << a.pages.shift) - 1) >> a.pages.shift; };
    if constexpr (OP == kBookHold) {
        return {b, 0, pages_of(extent_of(a.rows + static_cast<int64_t>(b) * a.Hkv).most), true};
    } else if constexpr (OP == kBookFork) {
        const int from = a.src[b];
        const bool moves = static_cast<uint32_t>(from) < static_cast<uint32_t>(a.B) && from != b;
        const Extent e = extent_of(lens + static_cast<int64_t>(moves ? from : b) * a.Hkv);
        return {from, min(max(e.least, 0), a.pages.cap) >> a.pages.shift, pages_of(e.most), moves};
    } else {
        const Extent e = extent_of(a.rows + static_cast<int64_t>(b) * a.Hkv);
        return {b, 0, pages_of(min(e.most, a.n)), e.most >= 0};
    }
}

// Whether entry j, which named `id` before, gets a new page.
template <int OP>
__device__ __forceinline__ bool wants(const BookArgs& a, const Change& c, int j, int id) {
    if (!c.moves || j >= c.end) return false;
    return OP == kBookHold ? !named(a.pages, id) : OP == kBookFork ? j >= c.keep && named(a.pages, id) : true;
}

// What entry j, which named `id` before, names after the call if it gets no new page.
template <int OP>
__device__ __forceinline__ int stays(const BookArgs& a, const Change& c, int j, int id) {
    return j < c.end && (OP == kBookHold || (OP == kBookFork && j < c.keep)) && named(a.pages, id) ? id : -1;
}

// The rows of head h of sequence b after a fork or a compaction.
template <int OP>
__device__ __forceinline__ int new_len(const BookArgs& a, const Change& c, int b, int h) {
    return OP == kBookFork ? a.old_lens[static_cast<int64_t>(c.from) * a.Hkv + h]
                           : min(max(a.rows[static_cast<int64_t>(b) * a.Hkv + h], 0), a.n);
}

// An entry of the table and the counters of the pages that it named and names.  (Nobody
// else writes the entry; the counters are sums, in any order.)
__device__ __forceinline__ void change_entry(const BookArgs& a, int64_t e, int old, int now) {
    if (now == old) return;
    a.table[e] = now;
    if (named(a.pages, old)) atomicSub(a.refs + old, 1);
    if (named(a.pages, now)) atomicAdd(a.refs + now, 1);
}

template <int OP>
__global__ void __launch_bounds__(kBookThreads) book_count_kernel(BookArgs a) {
    __shared__ int lds[2 * kBookThreads / kWave];
    const int b = blockIdx.x, tid = threadIdx.x;
    int total;
    if (b >= a.B) {
        const int64_t p0 = static_cast<int64_t>(b - a.B) * kChunk;
        int n[kChunk / kBookThreads], x = 0;
#pragma unroll
        for (int j = 0; j < kChunk / kBookThreads; ++j) n[j] = a.refs[min(p0 + j * kBookThreads + tid, static_cast<int64_t>(a.pages.n_pages) - 1)];
#pragma unroll
        for (int j = 0; j < kChunk / kBookThreads; ++j) {
            const int64_t p = p0 + j * kBookThreads + tid;
            const bool is_free = p < a.pages.n_pages && n[j] == 0;
            const uint64_t word = __ballot(is_free);
            if (lane_id() == 0) a.free_bits[p / kWave] = word;
            x += is_free;
        }
        block_scan(x, lds, &total);
        if (tid == 0) a.free[b - a.B] = total;
        return;
    }
    if (b == 0 && tid == 0) *a.taken = 0;
    const Change c = change_of<OP>(a, b, a.lens, [&](const int32_t* rows) { return extent(rows, a.Hkv, lds); });
    const int64_t row = static_cast<int64_t>(b) * a.pages.max_pages;
    const int64_t theirs = static_cast<int64_t>(c.moves ? c.from : b) * a.pages.max_pages;
    int x = 0;
    for (int j = tid; j < a.pages.max_pages; j += kBookThreads) {
        a.old_table[row + j] = a.table[row + j];
        x += wants<OP>(a, c, j, a.table[theirs + j]);
    }
    if (OP != kBookHold)
        for (int h = tid; h < a.Hkv; h += kBookThreads) {
            const int64_t at = static_cast<int64_t>(b) * a.Hkv + h;
            a.old_lens[at] = a.lens[at];
        }
    block_scan(x, lds, &total);
    if (tid == 0) a.want[b] = total;
}

template <int OP>
__global__ void __launch_bounds__(kBookThreads) book_plan_kernel(BookArgs a) {
    __shared__ int lds[2 * kBookThreads / kWave], upto[kBookThreads];
    const int b = blockIdx.x, tid = threadIdx.x;
    const Change c = change_of<OP>(a, b, a.old_lens, [&](const int32_t* rows) { return extent(rows, a.Hkv, lds); });
    // this sequence's ranks [lo, hi) (sums of at most B * max_pages entries)
    int x = 0, lo, total;
    for (int i = tid; i < b; i += kBookThreads) x += a.want[i];
    block_scan(x, lds, &lo);
    const int want = a.want[b], hi = lo + want;
    // the free pages of these ranks, to ids[lo ..]
    int run = 0;                           // free pages before the chunks looked at
    for (int64_t x0 = 0; x0 < a.chunks && want > 0 && run < hi; x0 += kBookThreads) {
        const int n = x0 + tid < a.chunks ? a.free[x0 + tid] : 0;
        const int mine = run + block_scan(n, lds, &total);
        upto[tid] = mine;
        // the chunks that hold free pages of ranks in [lo, hi)
        const int i0 = __syncthreads_count(mine <= lo), i1 = min(__syncthreads_count(mine < hi), kBookThreads - 1);
        for (int i = i0; i <= i1; ++i) {
            const int before = i ? upto[i - 1] : run;
            if (before == upto[i]) continue;
            static_assert(kChunk == 8 * kBookThreads, "a byte of the chunk's bits for each thread");
            const int64_t byte = (x0 + i) * kBookThreads + tid;
            uint32_t bits = reinterpret_cast<const uint8_t*>(a.free_bits)[byte];
            int all, rank = before + block_scan(__popc(bits), lds, &all) - __popc(bits);
            for (; bits != 0; bits &= bits - 1, ++rank)
                if (rank >= lo && rank < hi) a.ids[rank] = static_cast<int>(8 * byte + __ffs(bits) - 1);
        }
        run += total;
        __syncthreads();
    }
    const bool ok = want == 0 || run >= hi;
    __syncthreads();                       // (ids)
    if (tid == 0) {
        a.missing[b] = ok ? 0 : want;
        if (ok && want > 0) atomicMax(a.taken, hi);
    }
    if (!c.moves || (OP != kBookHold && !ok)) return;
    const int64_t row = static_cast<int64_t>(b) * a.pages.max_pages;
    const int32_t* const theirs = a.old_table + static_cast<int64_t>(c.from) * a.pages.max_pages;
    int rank = lo;
    for (int j0 = 0; j0 < a.pages.max_pages; j0 += kBookThreads) {
        const int j = j0 + tid;
        const int id = j < a.pages.max_pages ? theirs[j] : -1;
        const bool take = j < a.pages.max_pages && wants<OP>(a, c, j, id);
        const int at = rank + block_scan(take, lds, &total) - 1;
        rank += total;
        if (j >= a.pages.max_pages) continue;
        const int old = a.old_table[row + j], now = take ? (ok ? a.ids[at] : -1) : stays<OP>(a, c, j, id);
        if (OP != kBookHold && take) a.items[at] = make_int2(b, j);
        change_entry(a, row + j, old, now);
    }
    if (OP == kBookHold) return;
    for (int h = tid; h < a.Hkv; h += kBookThreads) a.lens[static_cast<int64_t>(b) * a.Hkv + h] = new_len<OP>(a, c, b, h);
}

// All of it but the copies for small pools and tables, in one workgroup: the free pages
// as a list in LDS, a thread for what each sequence asks for, and then for a few
// consecutive entries of the table, all of whose loads are on their way at once: the rank
// of a wanted page is the number of those before it, whatever the sequence.
constexpr int kSmallThreads = 1024, kSmallWaves = kSmallThreads / kWave;
constexpr int kSmallSeqs = 1024, kSmallHeads = 64;
constexpr int kSmallEach = 4, kSmallFree = 8;      // entries, and pages, of a thread
constexpr int kSmallPages = kSmallFree * kSmallThreads, kSmallEntries = kSmallEach * kSmallThreads;

template <int OP>
__global__ void __launch_bounds__(kSmallThreads) book_small_kernel(BookArgs a) {
    __shared__ int free_ids[kSmallPages], part[2][kSmallWaves];
    __shared__ int from[kSmallSeqs], keep[kSmallSeqs], end[kSmallSeqs], upto[kSmallSeqs + 1];
    const int tid = threadIdx.x, lane = lane_id(), wave = tid / kWave, most = a.pages.max_pages;
    // Inclusive prefix sum over the workgroup, and its total.
    const auto scan = [&](int x, int which, int* total) {
        x = wave_incl_scan(x);
        if (lane == kWave - 1) part[which][wave] = x;
        __syncthreads();
        int before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < kSmallWaves; ++w) {
            const int n = part[which][w];
            before += w < wave ? n : 0;
            all += n;
        }
        *total = all;
        return x + before;
    };
    // the free pages, a thread's consecutive ones
    const int per = (a.pages.n_pages + kSmallThreads - 1) / kSmallThreads, p0 = tid * per;
    uint32_t is_free = 0;
    int count[kSmallFree];
#pragma unroll
    for (int j = 0; j < kSmallFree; ++j) count[j] = a.refs[min(p0 + j, a.pages.n_pages - 1)];
#pragma unroll
    for (int j = 0; j < kSmallFree; ++j)
        is_free |= static_cast<uint32_t>(j < per && p0 + j < a.pages.n_pages && count[j] == 0) << j;
    if (tid < a.B) {
        const Change c = change_of<OP>(a, tid, a.lens, [&](const int32_t* rows) {
            Extent e{INT32_MIN, INT32_MAX};
            for (int h0 = 0; h0 < a.Hkv; h0 += 8) {
                int n[8];
#pragma unroll
                for (int h = 0; h < 8; ++h) n[h] = rows[min(h0 + h, a.Hkv - 1)];
#pragma unroll
                for (int h = 0; h < 8; ++h) e = {max(e.most, n[h]), min(e.least, n[h])};
            }
            return e;
        });
        from[tid] = c.moves ? c.from : -1;
        keep[tid] = c.keep;
        end[tid] = c.end;
    }
    if (OP != kBookHold)
        for (int x = tid; x < a.B * a.Hkv; x += kSmallThreads) a.old_lens[x] = a.lens[x];
    if (tid == 0) upto[0] = 0, *a.taken = 0;
    int n_free, wanted;
    int rank = scan(__popc(is_free), 0, &n_free) - __popc(is_free);
    for (uint32_t x = is_free; x != 0; x &= x - 1) free_ids[rank++] = p0 + __ffs(x) - 1;
    // a thread's consecutive entries: their sequence (-1: none), place in its row, what they
    // and the entries that they become copies of name
    const int entries = a.B * most, each = (entries + kSmallThreads - 1) / kSmallThreads;
    int seq[kSmallEach], own[kSmallEach], theirs[kSmallEach];
    const auto change = [&](int b) {
        const int x = from[b];
        return Change{x < 0 ? b : x, keep[b], end[b], x >= 0};
    };
#pragma unroll
    for (int x = 0; x < kSmallEach; ++x) {
        const int e = tid * each + x;
        seq[x] = x < each && e < entries ? e / most : -1;
        own[x] = theirs[x] = -1;
        if (seq[x] >= 0) {
            own[x] = a.table[e];
            theirs[x] = a.table[change(seq[x]).from * most + e - seq[x] * most];
        }
    }
    uint32_t take = 0;
#pragma unroll
    for (int x = 0; x < kSmallEach; ++x) {
        if (seq[x] < 0) continue;
        const int e = tid * each + x;
        a.old_table[e] = own[x];
        take |= static_cast<uint32_t>(wants<OP>(a, change(seq[x]), e - seq[x] * most, theirs[x])) << x;
    }
    const int first = scan(__popc(take), 1, &wanted) - __popc(take);
#pragma unroll
    for (int x = 0; x < kSmallEach; ++x) {
        const int e = tid * each + x;
        if (seq[x] >= 0 && e + 1 == (seq[x] + 1) * most) upto[seq[x] + 1] = first + __popc(take & ((2u << x) - 1));
    }
    __syncthreads();                       // (and the table has been read)
    if (tid < a.B) {
        const int want = upto[tid + 1] - upto[tid];
        const bool fits = want == 0 || upto[tid + 1] <= n_free;
        a.missing[tid] = fits ? 0 : want;
        if (want > 0 && fits) atomicMax(a.taken, upto[tid + 1]);
    }
    if (OP != kBookHold)
        for (int x = tid; x < a.B * a.Hkv; x += kSmallThreads) {
            const int b = x / a.Hkv;
            if (from[b] >= 0 && (upto[b + 1] == upto[b] || upto[b + 1] <= n_free))
                a.lens[x] = new_len<OP>(a, Change{from[b], 0, 0, true}, b, x - b * a.Hkv);
        }
#pragma unroll
    for (int x = 0; x < kSmallEach; ++x) {
        if (seq[x] < 0) continue;
        const int b = seq[x], e = tid * each + x, j = e - b * most, at = first + __popc(take & ((1u << x) - 1));
        const Change c = change(b);
        const bool new_page = take >> x & 1, fits = upto[b + 1] == upto[b] || upto[b + 1] <= n_free;
        if (!c.moves || (OP != kBookHold && !fits)) continue;
        const int now = new_page ? (fits ? free_ids[at] : -1) : stays<OP>(a, c, j, theirs[x]);
        if (OP != kBookHold && new_page) a.items[at] = make_int2(b, j), a.ids[at] = now;
        change_entry(a, e, own[x], now);
    }
}

// Rows of one head of one new page, 16 bytes a lane: a group of lanes has a row of K
// and of V.  Fork: the rows of the page that the source has there; compact: the rows
// that idx names, zeros (scale 1) where it names none.
template <int OP, int ROW>                 // bytes of a row
__global__ void __launch_bounds__(kBookThreads) book_copy_kernel(BookArgs a) {
    constexpr int kCh = ROW / 16, kPer = kBookThreads / kCh;
    const int page = 1 << a.pages.shift, ch = threadIdx.x % kCh;
    const int64_t units = static_cast<int64_t>(*a.taken) * a.Hkv;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int64_t item = u / a.Hkv;
        const int c = static_cast<int>(u - item * a.Hkv);
        const int2 at = a.items[item];
        const int b = at.x, t0 = at.y << a.pages.shift;
        const int64_t hc = static_cast<int64_t>(b) * a.Hkv + c;
        const int n = min(a.lens[hc] - t0, page);      // rows of this head on the page
        const int64_t to = (static_cast<int64_t>(a.ids[item]) * a.Hkv + c) << a.pages.shift;
        const int from = OP == kBookFork ? a.src[b] : b;
        const int32_t* const theirs = a.old_table + static_cast<int64_t>(from) * a.pages.max_pages;
        const int known = OP == kBookFork ? 0 : min(max(a.old_lens[hc], 0), a.pages.cap);
        for (int r = threadIdx.x / kCh; r < n; r += kPer) {
            int t = t0 + r;
            bool any = true;
            if (OP == kBookCompact) {
                t = a.idx[hc * a.n + t];
                any = t >= 0 && t < known;
            }
            const int id = any ? theirs[t >> a.pages.shift] : -1;
            any = named(a.pages, id);
            u32x4 k{0u, 0u, 0u, 0u}, v = k;
            float ks = 1.f, vs = 1.f;
            if (any) {
                const int64_t row = pool_row(a.pages, a.Hkv, c, id, t);
                k = *reinterpret_cast<const u32x4*>(static_cast<const char*>(a.pages.k) + row * ROW + 16 * ch);
                v = *reinterpret_cast<const u32x4*>(static_cast<const char*>(a.pages.v) + row * ROW + 16 * ch);
                if (a.pages.dtype != kCacheBf16 && ch == 0) ks = a.pages.k_scale[row], vs = a.pages.v_scale[row];
            }
            *reinterpret_cast<u32x4*>(static_cast<char*>(a.pages.k) + (to + r) * ROW + 16 * ch) = k;
            *reinterpret_cast<u32x4*>(static_cast<char*>(a.pages.v) + (to + r) * ROW + 16 * ch) = v;
            if (a.pages.dtype != kCacheBf16 && ch == 0) a.pages.k_scale[to + r] = ks, a.pages.v_scale[to + r] = vs;
        }
    }
}

// The table of a group's shared rows (mmshiftkv_shared_table).  A thread has an entry and
// looks through the group's sequences in order, kBookThreads of them at a time, with a
// thread to see what each has of the shared rows; sequences that have ended are passed over
// by their bits.  As a rule the first one left ends the search, a chain of three loads:
// 3.3 us for 8 entries of 8 sequences, 4.2 for 520 of 32, 4.7 where 500 of 512 have ended.
__global__ void __launch_bounds__(kBookThreads) shared_table_kernel(SharedTableArgs a) {
    constexpr int kWords = kBookThreads / kWave;
    __shared__ int rows[kBookThreads], lds[2 * kWords];
    __shared__ uint64_t whole[kWords], some[kWords];   // sequences with all shared rows, and with any row
    const int tid = threadIdx.x, g = blockIdx.x, entries = a.pages.max_pages;
    const int32_t* const shared = a.shared + static_cast<int64_t>(g) * a.Hkv;
    const int most = min(extent(shared, a.Hkv, lds).most, a.pages.cap);
    for (int64_t j0 = static_cast<int64_t>(blockIdx.y) * kBookThreads; j0 < entries; j0 += gridDim.y * kBookThreads) {
        const int64_t j = j0 + tid, row = j << a.pages.shift;          // the entry, its first row
        const bool wanted = j < entries && row < most;
        int id = -1, part = -1;            // of a sequence with all shared rows, of one with some of this page
        for (int s0 = 0; s0 < a.each; s0 += kBookThreads) {
            int longest = 0;
            bool has = s0 + tid < a.each;
            if (has) {
                const int32_t* const lens = a.lens + (static_cast<int64_t>(g) * a.each + s0 + tid) * a.Hkv;
                for (int c = 0; c < a.Hkv; ++c) {
                    const int n = min(max(lens[c], 0), a.pages.cap);
                    longest = max(longest, n);
                    has = has && n >= min(shared[c], a.pages.cap);
                }
            }
            const uint64_t has_all = __ballot(has), has_some = __ballot(longest > 0);
            __syncthreads();               // (those of the last round have been read)
            rows[tid] = longest;
            if (lane_id() == 0) whole[tid / kWave] = has_all, some[tid / kWave] = has_some;
            if (!__syncthreads_or(wanted && id < 0)) break;
            if (!wanted) continue;
            // the first page that one of these sequences names, of those with a row behind `from`
            const auto first = [&](const uint64_t* of, int from) {
                for (int w = 0; w < kWords; ++w)
                    for (uint64_t bits = of[w]; bits != 0; bits &= bits - 1) {
                        const int x = w * kWave + __ffsll(static_cast<unsigned long long>(bits)) - 1;
                        if (rows[x] <= from) continue;
                        const int p = a.pages.table[(static_cast<int64_t>(g) * a.each + s0 + x) * entries + j];
                        if (named(a.pages, p)) return p;
                    }
                return -1;
            };
            if (id < 0) id = first(whole, -1);
            if (id < 0 && part < 0) part = first(some, static_cast<int>(row));
        }
        if (j < entries) a.out[static_cast<int64_t>(g) * entries + j] = id >= 0 ? id : part;
    }
}

template <int OP>
hipError_t launch(const BookArgs& a, hipStream_t s) {
    const int64_t entries = static_cast<int64_t>(a.B) * a.pages.max_pages;
    const bool small = a.pages.n_pages <= kSmallPages && a.B <= kSmallSeqs && a.Hkv <= kSmallHeads && entries <= kSmallEntries;
    if (small) {
        hipLaunchKernelGGL((book_small_kernel<OP>), dim3(1), dim3(kSmallThreads), 0, s, a);
    } else {
        hipLaunchKernelGGL((book_count_kernel<OP>), dim3(static_cast<unsigned>(a.B + a.chunks)), dim3(kBookThreads), 0, s, a);
        hipLaunchKernelGGL((book_plan_kernel<OP>), dim3(a.B), dim3(kBookThreads), 0, s, a);
    }
    if constexpr (OP != kBookHold) {
        const int64_t units = entries * a.Hkv;         // (as many new pages as there are entries, at most)
        const dim3 grid(static_cast<unsigned>(units < 8 * kPlanCus ? units : 8 * kPlanCus));
        const auto copy = [&](auto row) {
            hipLaunchKernelGGL((book_copy_kernel<OP, decltype(row)::value>), grid, dim3(kBookThreads), 0, s, a);
        };
        const int row = a.d * (a.pages.dtype == kCacheBf16 ? 2 : 1);
        if (row == 256) copy(Constant<256>{});
        else if (row == 128) copy(Constant<128>{});
        else copy(Constant<64>{});
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_book(const BookArgs& a, int op, hipStream_t s) {
    return op == kBookHold ? launch<kBookHold>(a, s) : op == kBookFork ? launch<kBookFork>(a, s) : launch<kBookCompact>(a, s);
}

hipError_t launch_shared_table(const SharedTableArgs& a, hipStream_t s) {
    const int blocks = (a.pages.max_pages + kBookThreads - 1) / kBookThreads;
    const dim3 grid(a.groups, blocks < 65535 ? blocks : 65535);
    hipLaunchKernelGGL(shared_table_kernel, grid, dim3(kBookThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace mmskv
