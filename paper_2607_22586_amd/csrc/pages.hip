// Pages of a paged cache given, taken and copied on gfx950
// (mmshiftkv_cache_hold, _fork and _compact).  The numbers of rows are the
// device's (a selection leaves them there), so the pages are assigned there too,
// without a wait of the host.  Three kernels:
//   count  what each sequence wants, the free pages of each chunk of the pool,
//          a copy of the table and the lengths as they were;
//   plan   each sequence's new row of the table.  The pages wanted are ranked by
//          sequence and entry, the free ones by number, and rank r gets the r-th
//          free page: the outcome does not depend on the order of workgroups;
//   apply  the counters, by the difference of the two tables, and the rows that a
//          fork or a compaction copies: a unit of work is one head of one new page.
// The first two are bound by latency, the copies by HBM.
#include "pages.hpp"

namespace mmskv {
namespace {

constexpr int kBookThreads = 256;
constexpr int kChunk = 8 * kBookThreads;   // pages of a chunk

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

// Largest and smallest of a sequence's numbers of rows (every thread gets them).
__device__ __forceinline__ Extent extent(const int32_t* rows, int Hkv, int* lds) {
    int most = INT32_MIN, least = INT32_MAX;
    for (int c = threadIdx.x; c < Hkv; c += kBookThreads) {
        most = max(most, rows[c]);
        least = min(least, rows[c]);
    }
#pragma unroll
    for (int s = kWave / 2; s > 0; s /= 2) {
        most = max(most, __shfl_xor(most, s));
        least = min(least, __shfl_xor(least, s));
    }
    __syncthreads();
    if (lane_id() == 0) lds[2 * (threadIdx.x / kWave)] = most, lds[2 * (threadIdx.x / kWave) + 1] = least;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kBookThreads / kWave; ++w) most = max(most, lds[2 * w]), least = min(least, lds[2 * w + 1]);
    return {most, least};
}

// What a call makes of a sequence's row of the table: entries j < keep as those of
// sequence `from`, new pages for the entries keep <= j < end (hold: for those j < end
// that name none; fork: for those that name one), none behind.
struct Change {
    int from, keep, end;
    bool moves;
};

template <int OP>
__device__ __forceinline__ Change change_of(const BookArgs& a, int b, const int32_t* lens, int* lds) {
    const auto pages_of = [&](int rows) { return (min(max(rows, 0), a.pages.cap) + (1 << a.pages.shift) - 1) >> a.pages.shift; };
    if constexpr (OP == kBookHold) {
        return {b, 0, pages_of(extent(a.rows + static_cast<int64_t>(b) * a.Hkv, a.Hkv, lds).most), true};
    } else if constexpr (OP == kBookFork) {
        const int from = a.src[b];
        const bool moves = static_cast<uint32_t>(from) < static_cast<uint32_t>(a.B) && from != b;
        const Extent e = extent(lens + static_cast<int64_t>(moves ? from : b) * a.Hkv, a.Hkv, lds);
        return {from, min(max(e.least, 0), a.pages.cap) >> a.pages.shift, pages_of(e.most), moves};
    } else {
        const Extent e = extent(a.rows + static_cast<int64_t>(b) * a.Hkv, a.Hkv, lds);
        return {b, 0, pages_of(min(e.most, a.n)), e.most >= 0};
    }
}

// Whether entry j, which named `id` before, gets a new page.
template <int OP>
__device__ __forceinline__ bool wants(const BookArgs& a, const Change& c, int j, int id) {
    if (!c.moves || j >= c.end) return false;
    return OP == kBookHold ? !named(a.pages, id) : OP == kBookFork ? j >= c.keep && named(a.pages, id) : true;
}

template <int OP>
__global__ void __launch_bounds__(kBookThreads) book_count_kernel(BookArgs a) {
    __shared__ int lds[2 * kBookThreads / kWave];
    const int b = blockIdx.x, tid = threadIdx.x;
    int total;
    if (b >= a.B) {
        const int64_t p0 = static_cast<int64_t>(b - a.B) * kChunk;
        int x = 0;
#pragma unroll
        for (int j = 0; j < kChunk / kBookThreads; ++j) {
            const int64_t p = p0 + j * kBookThreads + tid;
            x += p < a.pages.n_pages && a.refs[p] == 0;
        }
        block_scan(x, lds, &total);
        if (tid == 0) a.free[b - a.B] = total;
        return;
    }
    if (b == 0 && tid == 0) *a.taken = 0;
    const Change c = change_of<OP>(a, b, a.lens, lds);
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
    const Change c = change_of<OP>(a, b, a.old_lens, lds);
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
            const int64_t p0 = (x0 + i) * kChunk + tid * (kChunk / kBookThreads);
            int here = 0, all;
#pragma unroll
            for (int j = 0; j < kChunk / kBookThreads; ++j) here += p0 + j < a.pages.n_pages && a.refs[p0 + j] == 0;
            int rank = before + block_scan(here, lds, &all) - here;
#pragma unroll
            for (int j = 0; j < kChunk / kBookThreads; ++j) {
                if (p0 + j >= a.pages.n_pages || a.refs[p0 + j] != 0) continue;
                if (rank >= lo && rank < hi) a.ids[rank] = static_cast<int>(p0 + j);
                ++rank;
            }
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
        int now = -1;
        if (take) {
            if (ok) {
                now = a.ids[at];
                if (OP != kBookHold) a.items[at] = make_int2(b, j);
            }
        } else if (j < c.end && (OP == kBookHold || (OP == kBookFork && j < c.keep)) && named(a.pages, id)) {
            now = id;
        }
        a.table[row + j] = now;
    }
    if (OP == kBookHold) return;
    for (int h = tid; h < a.Hkv; h += kBookThreads) {
        const int64_t at = static_cast<int64_t>(b) * a.Hkv + h;
        a.lens[at] = OP == kBookFork ? a.old_lens[static_cast<int64_t>(c.from) * a.Hkv + h] : min(max(a.rows[at], 0), a.n);
    }
}

// Every entry that changed: one naming less of its old page, one more of its new.
__device__ __forceinline__ void count_changes(const BookArgs& a) {
    const int64_t entries = static_cast<int64_t>(a.B) * a.pages.max_pages;
    const int64_t step = static_cast<int64_t>(gridDim.x) * kBookThreads;
    for (int64_t e = static_cast<int64_t>(blockIdx.x) * kBookThreads + threadIdx.x; e < entries; e += step) {
        const int before = a.old_table[e], after = a.table[e];
        if (before == after) continue;
        if (named(a.pages, before)) atomicSub(a.refs + before, 1);
        if (named(a.pages, after)) atomicAdd(a.refs + after, 1);
    }
}

__global__ void __launch_bounds__(kBookThreads) book_hold_kernel(BookArgs a) { count_changes(a); }

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
    count_changes(a);
}

template <int OP>
hipError_t launch(const BookArgs& a, hipStream_t s) {
    const int64_t entries = static_cast<int64_t>(a.B) * a.pages.max_pages;
    hipLaunchKernelGGL((book_count_kernel<OP>), dim3(static_cast<unsigned>(a.B + a.chunks)), dim3(kBookThreads), 0, s, a);
    hipLaunchKernelGGL((book_plan_kernel<OP>), dim3(a.B), dim3(kBookThreads), 0, s, a);
    const int64_t blocks = (entries + kBookThreads - 1) / kBookThreads;
    if constexpr (OP == kBookHold) {
        hipLaunchKernelGGL(book_hold_kernel, dim3(static_cast<unsigned>(blocks < 1024 ? blocks : 1024)), dim3(kBookThreads), 0, s, a);
    } else {
        const int64_t units = entries * a.Hkv;         // (as many new pages as there are entries, at most)
        const dim3 grid(static_cast<unsigned>(units < 8 * kPlanCus ? units : 8 * kPlanCus)), threads(kBookThreads);
        const int row = a.d * (a.pages.dtype == kCacheBf16 ? 2 : 1);
        if (row == 256) hipLaunchKernelGGL((book_copy_kernel<OP, 256>), grid, threads, 0, s, a);
        else if (row == 128) hipLaunchKernelGGL((book_copy_kernel<OP, 128>), grid, threads, 0, s, a);
        else hipLaunchKernelGGL((book_copy_kernel<OP, 64>), grid, threads, 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace

int64_t book_chunks(int n_pages) { return (static_cast<int64_t>(n_pages) + kChunk - 1) / kChunk; }

hipError_t launch_book(const BookArgs& a, int op, hipStream_t s) {
    return op == kBookHold ? launch<kBookHold>(a, s) : op == kBookFork ? launch<kBookFork>(a, s) : launch<kBookCompact>(a, s);
}

}  // namespace mmskv
