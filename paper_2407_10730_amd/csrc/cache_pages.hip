// cache_pages.hip -- pages of the cache for the next tokens of a batch of requests, and where each token goes.
//
// What is to be done is a few running sums over the sequences (pages that go back, pages that are taken) and a
// copy of page numbers each way; it moves some kilobytes, so a call is bound by its launch and by the chain of
// dependent loads (slot -> length -> table -> list of pages).  One workgroup does it all in one launch, up to kOneLaunch
// rows; more rows get their places from a second launch.
#include <algorithm>

#include "seqmix_device.h"

namespace cv {

constexpr int64_t kOneLaunch = 4096;

// Of two values each, sums over the threads before this one, and over all.
struct Two {
    uint32_t a, b;
};
template <int THREADS>
__device__ __forceinline__ Two scan_before(Two v, Two* sums, Two* total) {
    constexpr int WAVES = THREADS / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Two up{scan_lanes(v.a), scan_lanes(v.b)};
    Two before{0, 0}, all{0, 0};
    if constexpr (WAVES == 1) {
        all = {(uint32_t)__builtin_amdgcn_readlane((int)up.a, 63), (uint32_t)__builtin_amdgcn_readlane((int)up.b, 63)};
    } else {
        __syncthreads();  // former readers of sums
        if (lane == 63) sums[wave] = up;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const Two s = sums[w];
            before.a += w < wave ? s.a : 0, before.b += w < wave ? s.b : 0;
            all.a += s.a, all.b += s.b;
        }
    }
    *total = all;
    return Two{before.a + up.a - v.a, before.b + up.b - v.b};
}

// The last of n + 1 ascending values (first 0) that is at most x, among the first n.
__device__ __forceinline__ int last_at_most(const uint32_t* v, int n, uint32_t x) {
    int lo = 0;
    while (n > 1) {
        const int half = n / 2;
        if (v[lo + half] <= x) lo += half, n -= half;
        else n = half;
    }
    return lo;
}

// f(i, x) for the pages x < n of all sequences, sequence i (of this step) having `mine` of them from `first` on, which starts[]
// holds too: each thread its own sequence's where no sequence has many, else page by page over all threads.  Waits first.
template <int THREADS, typename F>
__device__ __forceinline__ void each_page(const uint32_t* starts, uint32_t first, uint32_t mine, uint32_t n, F f) {
    constexpr uint32_t kFew = 4;
    if (!__syncthreads_or(mine > kFew)) {
        for (uint32_t k = 0; k < mine; ++k)
            if (first + k < n) f(threadIdx.x, first + k);
    } else {
        for (uint32_t x = threadIdx.x; x < n; x += THREADS) f(last_at_most(starts, THREADS, x), x);
    }
}

struct PageSeq {
    int slot;  // -1: skipped
    uint32_t first, rows, keep, have_pages, keep_pages, want_pages;
    bool room;
};
__device__ __forceinline__ PageSeq page_seq(const PagesArgs& A, int i) {
    PageSeq s{-1, 0, 0, 0, 0, 0, 0, true};
    if (i >= A.sq.seqs) return s;
    const SeqRange r = seq_range(A.sq, i);
    s.first = (uint32_t)r.first;
    s.rows = (uint32_t)r.len;
    s.slot = (int)seq_slot(A.sq, i);
    if (s.slot < 0) return s;
    const uint32_t page = 1u << A.shift;
    const int64_t most = (int64_t)A.max_pages << A.shift;
    const int64_t have = min(max((int64_t)A.lens[s.slot], (int64_t)0), most);
    const int64_t keep = A.kept ? min(max((int64_t)A.kept[i], (int64_t)0), have) : have;
    s.keep = (uint32_t)keep;
    s.have_pages = (uint32_t)((have + page - 1) >> A.shift);
    s.keep_pages = (uint32_t)((keep + page - 1) >> A.shift);
    const int64_t want = (keep + s.rows + page - 1) >> A.shift;
    s.room = want <= A.max_pages;
    s.want_pages = s.room ? (uint32_t)want : s.keep_pages;
    return s;
}

__device__ __forceinline__ void put_row(const PagesArgs& A, uint32_t t, bool on, int32_t page, uint32_t position) {
    on = on && (uint32_t)page < (uint32_t)A.pages;
    A.place[t] = on ? (page << A.shift) + (int32_t)(position & ((1u << A.shift) - 1)) : -1;
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void pages_kernel(PagesArgs A, int rows_too) {
    __shared__ Two sums[THREADS / 64];
    __shared__ uint32_t s_back[THREADS], s_take[THREADS], s_page[THREADS], s_first[THREADS], s_rows[THREADS], s_keep[THREADS];
    __shared__ int32_t s_slot[THREADS], s_admitted[THREADS];
    __shared__ uint32_t s_granted;
    const int tid = threadIdx.x;
    const uint32_t pages = (uint32_t)A.pages;
    uint32_t taken = (uint32_t)min(max(A.taken[0], 0), A.pages);
    const bool once = A.sq.seqs <= THREADS;

    // Pages that go back, of all sequences; and, in steps of THREADS sequences, which: the last `back` of those in use.
    Two both{0, 0}, all{0, 0};
    uint32_t back = 0;
    PageSeq s = page_seq(A, tid);
    if (!once) {
        for (int i = tid; i < A.sq.seqs; i += THREADS) {
            const PageSeq x = page_seq(A, i);
            both.a += x.have_pages - x.keep_pages;
        }
        (void)scan_before<THREADS>(both, sums, &all);
        back = all.a;
    }
    uint32_t done = 0;
    for (int c = 0; c < A.sq.seqs; c += THREADS) {
        if (!once) s = page_seq(A, c + tid);
        both = scan_before<THREADS>(Two{s.have_pages - s.keep_pages, s.want_pages - s.keep_pages}, sums, &all);
        if (once) back = all.a;
        if (all.a) {
            const uint32_t base = taken - min(back, taken) + done;
            s_back[tid] = both.a;
            s_slot[tid] = s.slot;
            s_page[tid] = s.keep_pages;
            each_page<THREADS>(s_back, both.a, s.have_pages - s.keep_pages, min(all.a, pages), [&](int i, uint32_t x) {
                const uint32_t j = s_page[i] + (x - s_back[i]);  // (sums may wrap where lengths or offsets lie)
                if (s_slot[i] >= 0 && j < (uint32_t)A.max_pages && base + x < pages)
                    A.free_pages[base + x] = A.table[(int64_t)s_slot[i] * A.max_pages + j];
            });
            done += all.a;
            __syncthreads();
        }
    }
    taken -= min(back, taken);

    // Pages that are taken.
    uint32_t used = 0;          // of those granted,
    uint32_t want_before = 0;   // of those that were wanted, by the sequences before these
    for (int c = 0; c < A.sq.seqs; c += THREADS) {
        if (!once) {
            s = page_seq(A, c + tid);
            both = scan_before<THREADS>(Two{0, s.want_pages - s.keep_pages}, sums, &all);
        }
        const uint32_t want = s.want_pages - s.keep_pages;
        const bool fits = s.room && (want == 0 || (uint64_t)want_before + both.b + want + taken <= pages);
        const bool on = s.slot >= 0 && fits;
        // those that get pages are the first that want any, so the sums before them are those of what is granted
        s_take[tid] = both.b;
        s_slot[tid] = s.slot;
        s_admitted[tid] = on ? s.slot : -1;
        s_page[tid] = s.keep_pages;
        s_first[tid] = s.first;
        s_rows[tid] = s.rows;
        s_keep[tid] = s.keep;
        if (tid == 0) s_granted = 0;
        if (c + tid < A.sq.seqs) A.admitted[c + tid] = on ? s.slot : -1;
        if (s.slot >= 0) A.lens[s.slot] = (int32_t)(on ? s.keep + s.rows : s.keep);
        __syncthreads();
        if (all.b) {
            if (on && want) atomicMax(&s_granted, both.b + want);
            __syncthreads();
            const uint32_t granted = min(s_granted, pages), base = taken + min(want_before, pages);
            each_page<THREADS>(s_take, both.b, on ? want : 0, granted, [&](int i, uint32_t x) {
                const uint32_t j = s_page[i] + (x - s_take[i]);
                if (s_slot[i] >= 0 && j < (uint32_t)A.max_pages && base + x < pages)
                    A.table[(int64_t)s_slot[i] * A.max_pages + j] = A.free_pages[base + x];
            });
            used += granted;
            want_before += all.b;
            if (!once) __syncthreads();
        }
    }
    if (tid == 0) A.taken[0] = (int32_t)min(taken + used, pages);
    if (!rows_too) return;
    // The rows' pages: from the table, or where they are new from the list, so that no row waits for the table's update.
    const uint32_t tokens = (uint32_t)A.sq.tokens;
    constexpr int AT_ONCE = THREADS == 1024 ? 4 : 1;  // rows of a thread whose loads are under way together
    for (uint32_t t0 = tid; t0 < tokens; t0 += AT_ONCE * THREADS) {
        int32_t page[AT_ONCE];
        uint32_t position[AT_ONCE];
        bool on[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const uint32_t t = min(t0 + u * THREADS, tokens - 1);
            const int i = A.sq.off ? last_at_most(s_first, A.sq.seqs, t) : (int)fdiv(t, A.by_len);
            const uint32_t at = t - s_first[i];
            on[u] = t >= s_first[i] && at < s_rows[i] && s_admitted[i] >= 0;
            position[u] = on[u] ? s_keep[i] + at : 0;
            const uint32_t j = position[u] >> A.shift, fresh = taken + s_take[i] + (j - s_page[i]);
            page[u] = -1;
            if (on[u]) {
                if (j < s_page[i]) page[u] = A.table[(int64_t)s_admitted[i] * A.max_pages + j];
                else if (fresh < pages) page[u] = A.free_pages[fresh];
            }
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const uint32_t t = t0 + u * THREADS;
            if (t >= tokens) break;
            put_row(A, t, on[u], page[u], position[u]);
            A.position[t] = (int32_t)position[u];
        }
    }
}

__global__ __launch_bounds__(256) void page_rows_kernel(PagesArgs A) {
    const uint32_t t = blockIdx.x * 256 + threadIdx.x;
    if (t >= A.sq.tokens) return;
    int i = 0;
    if (A.sq.off) {
        for (int n = A.sq.seqs; n > 1;) {
            const int half = n / 2;
            if (clamp_row(A.sq.off[i + half], A.sq.tokens) <= t) i += half, n -= half;
            else n = half;
        }
    } else {
        i = (int)fdiv(t, A.by_len);
    }
    const SeqRange r = seq_range(A.sq, i);
    const int64_t at = (int64_t)t - r.first;
    int slot = at >= 0 && at < r.len ? A.admitted[i] : -1;
    const int64_t position = slot >= 0 ? (int64_t)A.lens[slot] - r.len + at : 0;
    if (position < 0 || position >> A.shift >= A.max_pages) slot = -1;
    put_row(A, t, slot >= 0, slot >= 0 ? A.table[(int64_t)slot * A.max_pages + (position >> A.shift)] : -1, (uint32_t)position);
    A.position[t] = slot >= 0 ? (int32_t)position : 0;
}

hipError_t launch_pages(const PagesArgs& a, hipStream_t s) {
    const int64_t most = std::max<int64_t>(a.sq.seqs, a.sq.tokens);
    const bool one = a.sq.tokens <= kOneLaunch && a.sq.seqs <= 1024;
    // as few waves as the rows need
    if (one && most <= 64)
        hipLaunchKernelGGL(pages_kernel<64>, dim3(1), dim3(64), 0, s, a, 1);
    else if (one && most <= 256)
        hipLaunchKernelGGL(pages_kernel<256>, dim3(1), dim3(256), 0, s, a, 1);
    else
        hipLaunchKernelGGL(pages_kernel<1024>, dim3(1), dim3(1024), 0, s, a, one ? 1 : 0);
    if (!one && a.sq.tokens > 0)
        hipLaunchKernelGGL(page_rows_kernel, dim3((unsigned)((a.sq.tokens + 255) / 256)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace cv
