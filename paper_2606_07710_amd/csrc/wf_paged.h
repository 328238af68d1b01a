// wf_paged.h -- what the paged-cache kernels share (gfx950): the ragged batch
// as a kernel sees it.  Internal header; not part of the C ABI.
#pragma once

#include "wf_api_internal.h"
#include "wf_device.h"

namespace wf {

// A batch and its pool as kernel arguments.
struct PagedView {
    const int32_t *table;      // [n_seqs][max_pages]
    const int32_t *row_start;  // [n_seqs + 1]
    const int32_t *ctx_len;    // [n_seqs]
    int n_seqs, max_pages, max_rows, n_rows;
    int n_pages, page_shift, n_kv_heads;
};

inline PagedView paged_view(const wf_paged_cache_t &c, const wf_paged_batch_t &b, int n_rows) {
    return PagedView{b.page_table, b.row_start, b.ctx_len, b.n_seqs,
                     b.max_pages,  b.max_rows,  n_rows,    c.n_pages,
                     __builtin_ctz((unsigned)c.page_size), c.n_kv_heads};
}

// Sequence b's rows [r0, r0 + rows) of the call and its context.  The lists are
// device memory that the host cannot check: a sequence whose numbers break the
// limits has no rows, so nothing of it is read or written.
struct Seq {
    int r0, rows, ctx;
};

__device__ __forceinline__ Seq paged_seq(const PagedView &a, int b, int max_rows) {
    const int r0 = a.row_start[b], r1 = a.row_start[b + 1], ctx = a.ctx_len[b];
    const long long end = (long long)ctx + ((long long)r1 - r0);
    const bool ok = r0 >= 0 && r1 >= r0 && r1 <= a.n_rows && r1 - r0 <= max_rows && ctx >= 0 &&
                    end <= ((long long)a.max_pages << a.page_shift);
    return Seq{r0, ok ? r1 - r0 : 0, ctx};
}

// The pool's page that holds logical page p of sequence b, or -1.
__device__ __forceinline__ int paged_page(const PagedView &a, int b, int p) {
    const int id = a.table[(size_t)b * a.max_pages + p];
    return (unsigned)id < (unsigned)a.n_pages ? id : -1;
}

// A value that all lanes hold alike, as a scalar.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ long long uniform64(long long x) {
    const unsigned lo = uniform((int)(unsigned)x), hi = uniform((int)(x >> 32));
    return (long long)(((unsigned long long)hi << 32) | lo);
}

// Where unit at(total) of a ragged list lies: sequence b owns count(its Seq)
// units, in order, `total` of them in all (also *total).  All threads of the
// workgroup call this alike, once or again after a barrier; the result is the owning
// sequence (-1 if there is no such unit), with *first its first unit and *seq its rows.
template <int THREADS, typename F, typename At>
__device__ __forceinline__ int paged_find(const PagedView &a, int max_rows, At &&at_of, F &&count,
                                          long long *first, long long *total, Seq *seq) {
    constexpr int WAVES = THREADS / kWave;
    __shared__ long long wave_sums[WAVES];
    __shared__ long long found_first;
    __shared__ int found;
    __shared__ Seq found_seq;
    const int per = (a.n_seqs + THREADS - 1) / THREADS;
    const int b0 = threadIdx.x * per;
    long long mine = 0;
    Seq s{0, 0, 0};
    for (int i = 0; i < per; ++i)
        if (b0 + i < a.n_seqs) {
            s = paged_seq(a, b0 + i, max_rows);
            mine += count(s);
        }
    const int lane = threadIdx.x % kWave;
    const long long incl = wave_scan_add(mine);
    if (threadIdx.x == 0)
        found = -1;
    if (lane == kWave - 1)
        wave_sums[threadIdx.x / kWave] = incl;
    __syncthreads();
    long long before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        before += w < (int)(threadIdx.x / kWave) ? wave_sums[w] : 0;
        all += wave_sums[w];
    }
    const long long at = at_of(uniform64(all));
    long long lo = before + incl - mine;
    if (at >= lo && at < lo + mine) {
        int b = b0;
        if (per > 1)
            for (;; ++b) {
                s = paged_seq(a, b, max_rows);
                const long long n = count(s);
                if (at < lo + n)
                    break;
                lo += n;
            }
        found = b;
        found_first = lo;
        found_seq = s;
    }
    __syncthreads();
    *first = uniform64(found_first);
    *total = uniform64(all);
    *seq = Seq{uniform(found_seq.r0), uniform(found_seq.rows), uniform(found_seq.ctx)};
    return uniform(found);
}

}  // namespace wf
