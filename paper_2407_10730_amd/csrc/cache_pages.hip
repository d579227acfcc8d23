// cache_pages.hip -- pages of the cache for the next tokens of a batch of requests, and where each token goes.
//
// What is to be done is a few running sums over the sequences (pages that go back, pages that are taken) and a
// copy of page numbers each way; it moves some kilobytes, so a call is bound by its launch and by the chain of
// dependent loads (slot -> length -> table -> list of pages).  One workgroup does it all in one launch, up to kOneLaunch
// rows; more rows get their places from a second launch.
#include "seqmix_device.h"

namespace cv {

constexpr int kPagesThreads = 1024;
constexpr int64_t kOneLaunch = 4096;

// Sum over the threads before this one (the first kPagesThreads / 64 of sums are scratch); total: over all.
__device__ __forceinline__ uint64_t scan_before(uint64_t v, uint64_t* sums, uint64_t* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint64_t up = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint64_t w = __shfl_up(up, d);
        if (lane >= d) up += w;
    }
    __syncthreads();  // former readers of sums
    if (lane == 63) sums[wave] = up;
    __syncthreads();
    uint64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kPagesThreads / 64; ++w) {
        const uint64_t s = sums[w];
        before += w < wave ? s : 0;
        all += s;
    }
    *total = all;
    return before + up - v;
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

__device__ __forceinline__ void place_row(const PagesArgs& A, uint32_t t, int slot, uint32_t position) {
    int32_t place = -1;
    if (slot >= 0) {
        const int32_t page = A.table[(int64_t)slot * A.max_pages + (position >> A.shift)];
        if ((uint32_t)page < (uint32_t)A.pages) place = (page << A.shift) + (int32_t)(position & ((1u << A.shift) - 1));
    }
    A.place[t] = place;
    A.position[t] = slot >= 0 ? (int32_t)position : 0;
}

__global__ __launch_bounds__(kPagesThreads) void pages_kernel(PagesArgs A, int rows_too) {
    __shared__ uint64_t sums[kPagesThreads / 64];
    __shared__ uint32_t s_back[kPagesThreads], s_take[kPagesThreads];
    __shared__ int32_t s_slot[kPagesThreads], s_admitted[kPagesThreads];
    __shared__ uint32_t s_page[kPagesThreads], s_first[kPagesThreads], s_rows[kPagesThreads], s_keep[kPagesThreads];
    const int tid = threadIdx.x;
    const uint32_t pages = (uint32_t)A.pages;
    uint32_t taken = (uint32_t)min(max(A.taken[0], 0), A.pages);
    const bool once = A.sq.seqs <= kPagesThreads;

    // pages that go back: how many
    uint64_t total = 0;
    PageSeq s = page_seq(A, tid);
    uint64_t back = 0;
    if (!once) {
        for (int i = tid; i < A.sq.seqs; i += kPagesThreads) {
            const PageSeq x = page_seq(A, i);
            back += x.have_pages - x.keep_pages;
        }
        (void)scan_before(back, sums, &total);
        back = total;
    }
    // ... and which: the last `back` of those in use
    uint64_t done = 0, want_before = 0;
    uint64_t both = 0, all = 0;
    for (int c = 0; c < A.sq.seqs; c += kPagesThreads) {
        if (!once) s = page_seq(A, c + tid);
        both = (uint64_t)(s.have_pages - s.keep_pages) << 32 | (s.want_pages - s.keep_pages);
        both = scan_before(both, sums, &all);
        const uint32_t n = (uint32_t)(all >> 32);
        if (once) back = n;
        const uint32_t base = taken - (uint32_t)min<uint64_t>(back, taken) + (uint32_t)done;
        s_back[tid] = (uint32_t)(both >> 32);
        s_slot[tid] = s.slot;
        s_page[tid] = s.keep_pages;
        __syncthreads();
        for (uint32_t x = tid; x < min(n, pages); x += kPagesThreads) {
            const int i = last_at_most(s_back, kPagesThreads, x);
            const uint32_t j = s_page[i] + (x - s_back[i]);  // (sums may wrap where lengths or offsets lie)
            if (s_slot[i] >= 0 && j < (uint32_t)A.max_pages && base + x < pages)
                A.free_pages[base + x] = A.table[(int64_t)s_slot[i] * A.max_pages + j];
        }
        done += n;
        __syncthreads();
    }
    taken -= (uint32_t)min<uint64_t>(back, taken);

    // pages that are taken
    uint32_t used = 0;  // the most of the granted running sums
    for (int c = 0; c < A.sq.seqs; c += kPagesThreads) {
        if (!once) {
            s = page_seq(A, c + tid);
            both = scan_before((uint64_t)(s.want_pages - s.keep_pages), sums, &all);
        }
        const uint32_t want = s.want_pages - s.keep_pages;
        const uint64_t before = want_before + (uint32_t)both;
        const bool fits = s.room && (want == 0 || before + want + taken <= pages);
        const bool on = s.slot >= 0 && fits;
        // those that get pages are the first that want any, so their sums before them are those of what is granted
        s_take[tid] = (uint32_t)min<uint64_t>(before - want_before, 0xffffffffu);
        s_slot[tid] = s.slot;
        s_admitted[tid] = on ? s.slot : -1;
        s_page[tid] = s.keep_pages;
        s_first[tid] = s.first;
        s_rows[tid] = s.rows;
        s_keep[tid] = s.keep;
        if (c + tid < A.sq.seqs) A.admitted[c + tid] = on ? s.slot : -1;
        if (s.slot >= 0) A.lens[s.slot] = (int32_t)(on ? s.keep + s.rows : s.keep);
        uint64_t granted = 0;
        const uint64_t mine = on ? want : 0;
        (void)scan_before(mine, sums, &granted);  // (also waits)
        const uint32_t base = taken + (uint32_t)min<uint64_t>(want_before, pages);
        for (uint32_t x = tid; x < min((uint32_t)granted, pages); x += kPagesThreads) {
            const int i = last_at_most(s_take, kPagesThreads, x);
            const uint32_t j = s_page[i] + (x - s_take[i]);
            if (s_slot[i] >= 0 && j < (uint32_t)A.max_pages && base + x < pages)
                A.table[(int64_t)s_slot[i] * A.max_pages + j] = A.free_pages[base + x];
        }
        used += (uint32_t)granted;
        want_before += (uint32_t)all;
        __syncthreads();
    }
    if (tid == 0) A.taken[0] = (int32_t)min(taken + used, pages);
    if (!rows_too) return;
    const uint32_t tokens = (uint32_t)A.sq.tokens;
    for (uint32_t t = tid; t < tokens; t += kPagesThreads) {
        int i;
        if (A.sq.off) i = last_at_most(s_first, A.sq.seqs, t);
        else i = (int)(t / (uint32_t)A.sq.seq_len);
        const uint32_t at = t - s_first[i];
        const bool in = t >= s_first[i] && at < s_rows[i];
        place_row(A, t, in ? s_admitted[i] : -1, in ? s_keep[i] + at : 0);
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
        i = (int)(t / (uint32_t)A.sq.seq_len);
    }
    const SeqRange r = seq_range(A.sq, i);
    const int64_t at = (int64_t)t - r.first;
    int slot = at >= 0 && at < r.len ? A.admitted[i] : -1;
    const int64_t position = slot >= 0 ? (int64_t)A.lens[slot] - r.len + at : 0;
    if (position < 0 || position >> A.shift >= A.max_pages) slot = -1;
    place_row(A, t, slot, (uint32_t)position);
}

hipError_t launch_pages(const PagesArgs& a, hipStream_t s) {
    const bool one = a.sq.tokens <= kOneLaunch && a.sq.seqs <= kPagesThreads;
    hipLaunchKernelGGL(pages_kernel, dim3(1), dim3(kPagesThreads), 0, s, a, one ? 1 : 0);
    if (!one && a.sq.tokens > 0)
        hipLaunchKernelGGL(page_rows_kernel, dim3((unsigned)((a.sq.tokens + 255) / 256)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace cv
