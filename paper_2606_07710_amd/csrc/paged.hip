// paged.hip -- the paged cache of a batch of requests: the append, which
// rotates K and q on the way and keeps the pages' bounds, and the selection of
// the pages that a row's attention is worth reading.
#include <cmath>

#include "wf_paged.h"

namespace wf {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxHalfDim = 64;

template <typename T>
struct Elem;
template <>
struct Elem<uint16_t> {
    static constexpr int kVec = 8;                   // elements of 16 bytes
    static __device__ __forceinline__ void unpack(u32x4 w, float (&f)[8]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ u32x4 pack(const float (&f)[8]) {
        return u32x4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]),
                     pack_bf16x2(f[6], f[7])};
    }
};
template <>
struct Elem<float> {
    static constexpr int kVec = 4;
    static __device__ __forceinline__ void unpack(u32x4 w, float (&f)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            f[i] = __uint_as_float(w[i]);
    }
    static __device__ __forceinline__ u32x4 pack(const float (&f)[4]) {
        return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                     __float_as_uint(f[3])};
    }
};

// Smaller and larger of two values, NaN if either is one (one instruction each).
__device__ __forceinline__ float nan_min(float a, float b) {
    return __builtin_elementwise_minimum(a, b);
}
__device__ __forceinline__ float nan_max(float a, float b) {
    return __builtin_elementwise_maximum(a, b);
}

// ---------------------------------------------------------------------------
// Append.  A workgroup takes one page that the batch writes and a run of KV
// heads with the query heads that read them.  It forms the sines and cosines of
// the page's new rows once, in LDS; then each of its waves takes one head's rows
// after the other, in 16-byte pieces, a thread holding both halves of its
// rotation pairs:
//   k' = R(pos) k: (lo, hi) -> (lo cos - hi sin, hi cos + lo sin), the angle
//   pos * theta_i in turns, reduced to half a turn in fp64 (an fp32 product
//   would be off by a part in a hundred of a radian at 64K positions), sine and
//   cosine in fp32.
// The bounds are taken anew from all of the page's valid rows, older ones
// included, so they never depend on what the page held before.  Prompts are
// bound by memory: 11000 rows of 32 + 8 + 8 heads, 277 MB, take 63 us, 4.4 TB/s, in
// pages of 16 (on inputs that the last-level cache still holds 54; there, with the
// angles formed anew by every head's workgroup, 92).  In pages of 128 they take 88:
// the sines and cosines of a page are 70 KB of LDS, two workgroups a CU.  64 rows of
// 64 sequences take 7 us in pages of 64 and of 128, the latency of a table entry,
// then a page's rows and the stores.
// ---------------------------------------------------------------------------
struct AppendParams {
    PagedView v;
    double turns[kMaxHalfDim];     // theta_i / 2 pi
    const void *k_in, *v_in, *q_in;
    void *k, *vc, *bounds, *q_out;
    const int32_t *positions;
    size_t kv_stride, q_stride;    // elements
    int group, n_q_heads;          // 0 without q
    int run;                       // KV heads of a workgroup
};

// The unit-th page that the batch writes; returns how many there are.
template <typename T, int DH>
__device__ __forceinline__ long long append_page(const AppendParams &a, long long unit) {
    using E = Elem<T>;
    constexpr int V = E::kVec, H = DH / 2;
    constexpr int LPR = H / V;                       // lanes per row
    constexpr int ROWS = kWave / LPR;                // rows of a wave at a time
    constexpr int WAVES = kThreads / kWave;
    // cosines and sines of the page's rows, [page_size][H + 4] each (padded, so
    // that the rows of a wave start in different banks)
    extern __shared__ __attribute__((aligned(16))) float trig[];
    constexpr int TST = H + 4;
    const int page = 1 << a.v.page_shift;
    const int any_rows = a.v.n_rows;
    long long first, total;
    Seq s;
    const int b = paged_find<kThreads>(
        a.v, any_rows, [&](long long) { return unit; },
        [&](const Seq &q) {
            return q.rows ? ((q.ctx + q.rows - 1) >> a.v.page_shift) - (q.ctx >> a.v.page_shift) + 1
                          : 0;
        },
        &first, &total, &s);
    if (b < 0)
        return total;
    const int lp = (s.ctx >> a.v.page_shift) + (int)(unit - first);
    const int p0 = lp << a.v.page_shift;
    // page rows [from, to) are new, [0, from) older
    const int from = max(s.ctx - p0, 0), to = min(s.ctx + s.rows - p0, page);
    const int row0 = s.r0 + p0 - s.ctx;              // the call's row of page row 0
    const int id = paged_page(a.v, b, lp);
    const int wave = wave_id(), lane = threadIdx.x % kWave;
    const int c = lane % LPR, rt = lane / LPR;
    const int g0 = blockIdx.y * a.run, n_kv = min(a.run, a.v.n_kv_heads - g0);
    const int n_heads = n_kv * (1 + a.group);        // KV heads, then query heads

    float *cs = trig, *sn = trig + page * TST;

    // smallest and largest of what the lane has seen of a head's keys
    float mn[2 * V], mx[2 * V];
    auto count = [&](const u32x4 &lo, const u32x4 &hi) {
        float x[V], y[V];
        E::unpack(lo, x);
        E::unpack(hi, y);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            mn[e] = nan_min(mn[e], x[e]);
            mx[e] = nan_max(mx[e], x[e]);
            mn[V + e] = nan_min(mn[V + e], y[e]);
            mx[V + e] = nan_max(mx[V + e], y[e]);
        }
    };
    // the older rows of KV head h
    auto older = [&](int h) {
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) {
            mn[e] = INFINITY;
            mx[e] = -INFINITY;
        }
        const T *kp = static_cast<const T *>(a.k) +
                      (((size_t)id * a.v.n_kv_heads + h) << a.v.page_shift) * DH;
        constexpr int U = 8;                         // rows of a lane in flight
        for (int r0 = rt; r0 < from; r0 += U * ROWS) {
            u32x4 w[U][2];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                // (past the last row: that one again)
                const T *src = kp + (size_t)min(r0 + u * ROWS, from - 1) * DH;
                w[u][0] = *reinterpret_cast<const u32x4 *>(src + c * V);
                w[u][1] = *reinterpret_cast<const u32x4 *>(src + H + c * V);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                count(w[u][0], w[u][1]);
        }
    };
    const bool bounds = a.bounds && id >= 0;
    if (bounds && wave < n_kv)
        older(g0 + wave);

    for (int at = threadIdx.x; at < (to - from) * H; at += kThreads) {
        const int r = at / H, i = at % H;
        const int pos = a.positions ? a.positions[row0 + from + r] : p0 + from + r;
        const double x = (double)pos * a.turns[i];
        sincospif(2.f * (float)(x - rint(x)), &sn[r * TST + i], &cs[r * TST + i]);
    }
    __syncthreads();
    // (a single KV head, with its older rows, is work enough for the first wave)
    const bool apart = n_kv == 1 && a.group > 0;
    for (int head = wave; head < (apart && wave == 0 ? 1 : n_heads);
         head += apart ? WAVES - 1 : WAVES) {
        const bool is_q = head >= n_kv;
        if (!is_q && id < 0)
            continue;
        const int h = is_q ? g0 * a.group + head - n_kv : g0 + head;
        const size_t unit = (size_t)max(id, 0) * a.v.n_kv_heads + h;
        const size_t head_row = unit << a.v.page_shift;
        if (!is_q && bounds && head != wave)
            older(h);
        for (int r = from + rt; r < to; r += ROWS) {
            const size_t in_row = row0 + r;
            const T *src = is_q ? static_cast<const T *>(a.q_in) + in_row * a.q_stride +
                                      (size_t)h * DH
                                : static_cast<const T *>(a.k_in) + in_row * a.kv_stride +
                                      (size_t)h * DH;
            T *dst = is_q ? static_cast<T *>(a.q_out) + (in_row * a.n_q_heads + h) * DH
                          : static_cast<T *>(a.k) + (head_row + r) * DH;
            float x[V], y[V], lo[V], hi[V];
            E::unpack(*reinterpret_cast<const u32x4 *>(src + c * V), x);
            E::unpack(*reinterpret_cast<const u32x4 *>(src + H + c * V), y);
            if (!is_q) {
                const T *vs = static_cast<const T *>(a.v_in) + in_row * a.kv_stride +
                              (size_t)h * DH;
                T *vd = static_cast<T *>(a.vc) + (head_row + r) * DH;
                const u32x4 v0 = *reinterpret_cast<const u32x4 *>(vs + c * V);
                const u32x4 v1 = *reinterpret_cast<const u32x4 *>(vs + H + c * V);
                *reinterpret_cast<u32x4 *>(vd + c * V) = v0;
                *reinterpret_cast<u32x4 *>(vd + H + c * V) = v1;
            }
#pragma unroll
            for (int e = 0; e < V; e += 4) {
                const int at = (r - from) * TST + c * V + e;
                const f32x4 co = *reinterpret_cast<const f32x4 *>(cs + at);
                const f32x4 si = *reinterpret_cast<const f32x4 *>(sn + at);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    lo[e + i] = x[e + i] * co[i] - y[e + i] * si[i];
                    hi[e + i] = y[e + i] * co[i] + x[e + i] * si[i];
                }
            }
            const u32x4 wlo = E::pack(lo), whi = E::pack(hi);
            *reinterpret_cast<u32x4 *>(dst + c * V) = wlo;
            *reinterpret_cast<u32x4 *>(dst + H + c * V) = whi;
            if (!is_q && bounds)
                count(wlo, whi);                     // as stored
        }
        if (is_q || !bounds)
            continue;
        // over the wave's ROWS rows
        float keep[2 * V];
        const bool up = lane & 32;
        auto pick = [&](float x, float y) { return up ? nan_max(x, y) : nan_min(x, y); };
        typedef unsigned u32pair __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) {
            // the halves' minima side by side in the lower lanes, their maxima in
            // the upper ones
            u32pair w = __builtin_bit_cast(
                u32pair, __builtin_amdgcn_permlane32_swap(__float_as_uint(mn[e]),
                                                          __float_as_uint(mx[e]), false, false));
            keep[e] = pick(__uint_as_float(w[0]), __uint_as_float(w[1]));
            // rows of 16 lanes: each with its neighbour
            w = __builtin_bit_cast(
                u32pair, __builtin_amdgcn_permlane16_swap(__float_as_uint(keep[e]),
                                                          __float_as_uint(keep[e]), false, false));
            keep[e] = pick(__uint_as_float(w[0]), __uint_as_float(w[1]));
            if constexpr (LPR <= 8)
                keep[e] = pick(keep[e], __int_as_float(dpp<kRowRor8, 0xf>(
                                            0, __float_as_int(keep[e]))));
            if constexpr (LPR <= 4)
                keep[e] = pick(keep[e], __int_as_float(dpp<kRowRor4, 0xf>(
                                            0, __float_as_int(keep[e]))));
        }
        static_assert(LPR == 4 || LPR == 8 || LPR == 16, "the lanes of a row");
        if ((lane & 31) < LPR) {
            T *dst = static_cast<T *>(a.bounds) + (unit * 2 + (up ? 1 : 0)) * DH;
            float x[V], y[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                x[e] = keep[e];
                y[e] = keep[V + e];
            }
            // (exact: they are stored values)
            *reinterpret_cast<u32x4 *>(dst + c * V) = E::pack(x);
            *reinterpret_cast<u32x4 *>(dst + H + c * V) = E::pack(y);
        }
    }
    return total;
}

// A workgroup has one page, unless a decreasing row_start gives rows to several
// sequences: then there may be more pages than the host counts.
template <typename T, int DH>
__global__ __launch_bounds__(kThreads) void paged_append(AppendParams a) {
    for (long long unit = blockIdx.x; append_page<T, DH>(a, unit) > unit + gridDim.x;
         unit += gridDim.x)
        __syncthreads();
}

// ---------------------------------------------------------------------------
// Selection, in two launches.
//
// Scores:  s = max_h sum_d q_d (q_d >= 0 ? hi_d : lo_d)
//            = max_h sum_d max(q_d, 0) hi_d + min(q_d, 0) lo_d,
// in fp64 (bf16 products are exact there and their sums all but exact, so the
// order of the pages does not hang on the order of the sums), as products of the
// fp64 matrix instruction: 16 query rows -- the heads of a group, and as many of
// the sequence's rows as fit -- with the bounds of 16 pages.  A lane holds a
// quarter of the dims of one query row and of one page, 64 bytes of them next to
// its neighbours' at a time; which dims meet in a step is the same for both.
// Bound by the matrix unit, 64 cycles for each of DH / 2 steps a tile, and by the
// vector work, which does not go on beside fp64 products, whichever wave's they
// are: a product with two conversions takes 87 cycles.  So there is little of it
// (two instructions split q, nothing is masked that is not looked at), and none
// between products.  45 rows of 16 sequences of up to 32K tokens take 24 us (89
// with each lane summing by itself and sums over lanes at the end, 29 with the
// conversions between the products; the next tile's operands loaded ahead, 48
// registers to move, 10 more; q kept converted for a pack's tiles, 128 registers, 6
// more).  The tiles are dealt out evenly to 512 workgroups (256 or 1024: 8 more).
//
// Choice:  a workgroup per (row, KV head) finds the n_top-th largest key digit
// by digit and lists the pages at or above it in page order.
// ---------------------------------------------------------------------------
typedef double f64x4 __attribute__((ext_vector_type(4)));

struct SelectParams {
    PagedView v;
    const void *q, *bounds;
    int32_t *sel;
    uint64_t *keys;                // [n_rows * n_kv_heads][max_pages]
    int n_sel, n_recent, group, n_q_heads;
    int pack;                      // rows of a sequence that share a tile
};

// A key of a score: larger scores have larger keys; a score that is not finite
// (something not finite went into it) has the largest; 0 is kept for pages
// without an entry.
__device__ __forceinline__ uint64_t score_key(double s) {
    if (!(fabs(s) < INFINITY))
        return ~0ull;
    const uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);
    return (u >> 63) ? ~u : u | (1ull << 63);
}

// The first recent page of a sequence's row, that is, the number of its old ones.
__device__ __forceinline__ int old_pages(const SelectParams &a, const Seq &s, int row) {
    return max(((s.ctx + row) >> a.v.page_shift) + 1 - a.n_recent, 0);
}

// The score tiles, [sequence][KV head][pack of rows][16 pages], laid end to end,
// go out in equal runs to the workgroups, in turn to a run's waves.
template <typename T, int DH>
__global__ __launch_bounds__(kThreads) void paged_scores(SelectParams a) {
    using E = Elem<T>;
    constexpr int V = E::kVec, PIECES = DH / 4 / V, WAVES = kThreads / kWave;
    __shared__ double sc[WAVES][16][17];
    const int n_top = a.n_sel - a.n_recent;
    // a sequence's tiles of a pack, none where all old pages are selected
    auto tiles_of = [&](const Seq &q) {
        const int n_old = q.rows ? old_pages(a, q, q.rows - 1) : 0;
        return n_old > n_top ? (n_old + 15) / 16 : 0;
    };
    auto count = [&](const Seq &q) {
        return (long long)tiles_of(q) * a.v.n_kv_heads * ((q.rows + a.pack - 1) / a.pack);
    };
    long long first, total;
    Seq s;
    int b = paged_find<kThreads>(
        a.v, a.v.max_rows, [&](long long n) { return n * blockIdx.x / gridDim.x; }, count, &first,
        &total, &s);
    const long long end = total * (blockIdx.x + 1) / gridDim.x;
    const int wave = wave_id(), lane = threadIdx.x % kWave;
    long long at = total * blockIdx.x / gridDim.x + wave;
    if (b < 0 || at >= end)
        return;
    const int m16 = lane & 15, c4 = lane >> 4;
    const int heads = min(a.group, 16);              // of a row in a tile
    int tiles = tiles_of(s), packs = (s.rows + a.pack - 1) / a.pack;
    // A tile: rows [row, row + rows) of the call, KV head g, 16 pages from p0 on, of
    // which the lane has one; n_old of the sequence's are old to the last row.
    struct Tile {
        int row, rows, g, n_old, p0, id;
    };
    auto locate = [&](long long to) {
        while (to >= first + (long long)tiles * packs * a.v.n_kv_heads) {
            first += (long long)tiles * packs * a.v.n_kv_heads;
            s = paged_seq(a.v, ++b, a.v.max_rows);
            tiles = tiles_of(s);
            packs = (s.rows + a.pack - 1) / a.pack;
        }
        const int unit = (int)(to - first);          // < 2^31: see the limits
        const int tile = unit % tiles, pack = unit / tiles % packs;
        const int row0 = pack * a.pack;
        Tile w;
        w.g = unit / tiles / packs;
        w.row = s.r0 + row0;
        w.rows = min(s.rows - row0, a.pack);
        w.n_old = old_pages(a, s, row0 + w.rows - 1);
        w.p0 = tile * 16;
        w.id = w.p0 + m16 < w.n_old ? paged_page(a.v, b, w.p0 + m16) : -1;
        return w;
    };
    // (a page that is not there has another's bounds, a row that is not there
    // another's q: what comes of them is not looked at)
    auto load_bounds = [&](const Tile &w, u32x4 (&lo)[PIECES], u32x4 (&hi)[PIECES]) {
        const T *src = static_cast<const T *>(a.bounds) +
                       ((size_t)max(w.id, 0) * a.v.n_kv_heads + w.g) * 2 * DH + c4 * V;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            lo[i] = *reinterpret_cast<const u32x4 *>(src + i * 4 * V);
            hi[i] = *reinterpret_cast<const u32x4 *>(src + DH + i * 4 * V);
        }
    };
    auto load_q = [&](const Tile &w, int h0, u32x4 (&q)[PIECES]) {
        const int row = min(m16 / heads, w.rows - 1), h = min(h0 + m16 % heads, a.group - 1);
        const T *src = static_cast<const T *>(a.q) +
                       ((size_t)(w.row + row) * a.n_q_heads + w.g * a.group + h) * DH +
                       c4 * V;
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
            q[i] = *reinterpret_cast<const u32x4 *>(src + i * 4 * V);
    };
    for (; at < end; at += WAVES) {
        const Tile now = locate(at);
        u32x4 lo[PIECES], hi[PIECES], qw[PIECES];
        load_bounds(now, lo, hi);
        load_q(now, 0, qw);
        double best = -INFINITY;
        bool odd = false;
        for (int h0 = 0; h0 < a.group; h0 += 16) {
            if (h0)
                load_q(now, h0, qw);
            f64x4 sum = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                float q[V], l[V], u[V];
                E::unpack(qw[i], q);
                E::unpack(lo[i], l);
                E::unpack(hi[i], u);
                double up[V], dn[V], ud[V], ld[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    // (not finite: one of the two is NaN or infinite, the score odd)
                    const float x = __builtin_amdgcn_fmed3f(q[e], 0.f, INFINITY);
                    up[e] = (double)x;
                    dn[e] = (double)(q[e] - x);
                    ud[e] = (double)u[e];
                    ld[e] = (double)l[e];
                }
                // (a conversion between two products would wait for the first of them
                // and hold up the second)
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    sum = __builtin_amdgcn_mfma_f64_16x16x4f64(up[e], ud[e], sum, 0, 0, 0);
                    sum = __builtin_amdgcn_mfma_f64_16x16x4f64(dn[e], ld[e], sum, 0, 0, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            // lane (m16, c4) has rows 4 i + c4 of column m16
            wave_sync();
#pragma unroll
            for (int i = 0; i < 4; ++i)
                sc[wave][4 * i + c4][m16] = sum[i];
            wave_sync();
            const int live = min(heads, a.group - h0);
            // four rows at a time (there is one where the group has several parts)
#pragma unroll 1
            for (int r0 = 0; r0 < now.rows; r0 += 4) {
                const int r = r0 + c4, page = now.p0 + m16;
                if (h0 == 0) {
                    best = -INFINITY;
                    odd = false;
                }
                if (r >= now.rows)
                    continue;
                // (four heads at a time, the last one again past the last)
#pragma unroll 1
                for (int h2 = 0; h2 < live; h2 += 4) {
                    double x[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        x[k] = sc[wave][r * heads + min(h2 + k, live - 1)][m16];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        odd |= !(fabs(x[k]) < INFINITY);
                        best = x[k] > best ? x[k] : best;
                    }
                }
                if (h0 + 16 >= a.group && page < now.n_old)
                    a.keys[((size_t)(now.row + r) * a.v.n_kv_heads + now.g) * a.v.max_pages +
                           page] = now.id < 0 ? 0ull : score_key(odd ? (double)NAN : best);
            }
        }
    }
}

constexpr int kLdsKeys = 2048;

template <int THREADS>
__global__ __launch_bounds__(THREADS) void paged_choose(SelectParams a) {
    constexpr int WAVES = THREADS / kWave;
    __shared__ int seq_of_row;
    const int unit = blockIdx.x;
    const int r = unit / a.v.n_kv_heads;
    if (threadIdx.x == 0)
        seq_of_row = -1;
    __syncthreads();
    for (int i = threadIdx.x; i < a.v.n_seqs; i += THREADS) {
        const Seq q = paged_seq(a.v, i, a.v.max_rows);
        if (r >= q.r0 && r < q.r0 + q.rows)
            seq_of_row = i;
    }
    __syncthreads();
    const int b = uniform(seq_of_row);
    if (b < 0)
        return;
    const Seq s = paged_seq(a.v, b, a.v.max_rows);
    const int newest = (s.ctx + r - s.r0) >> a.v.page_shift;
    const int n_old = old_pages(a, s, r - s.r0);
    const int n_top = a.n_sel - a.n_recent;
    const int wave = wave_id(), lane = threadIdx.x % kWave;
    const uint64_t *keys = a.keys + (size_t)unit * a.v.max_pages;
    const bool choose = n_old > n_top && n_top > 0;

    // ---- the smallest selected key ----
    __shared__ uint64_t lds_keys[kLdsKeys];
    __shared__ int hist[256];
    __shared__ int wave_count[2][WAVES];
    __shared__ int digit, above;
    __shared__ uint64_t same[2][WAVES];
    uint64_t least = 1;                              // all pages with an entry
    int equal_quota = n_old;                         // of the pages at `least`
    const bool in_lds = n_old <= kLdsKeys;
    if (in_lds) {
        // (all of a thread's loads at once)
        constexpr int N = kLdsKeys / THREADS;
        uint64_t got[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = j * THREADS + threadIdx.x;
            got[j] = i >= n_old ? 0ull
                     : choose   ? keys[i]
                                : (n_top > 0 && paged_page(a.v, b, i) >= 0 ? 1ull : 0ull);
        }
#pragma unroll
        for (int j = 0; j < N; ++j)
            lds_keys[j * THREADS + threadIdx.x] = got[j];
    }
    auto key = [&](int i) -> uint64_t {
        if (in_lds)
            return lds_keys[i];
        return choose ? keys[i] : n_top > 0 && paged_page(a.v, b, i) >= 0 ? 1ull : 0ull;
    };
    if (choose) {
        // (the keys' common leading digits need no counting)
        uint64_t ones = ~0ull, zeros = ~0ull;
        for (int i = threadIdx.x; i < n_old; i += THREADS) {
            ones &= key(i);
            zeros &= ~key(i);
        }
        auto all_of = [](uint64_t x) -> uint64_t {
            auto both = [](int u, int v) { return u & v; };
            return ((uint64_t)(uint32_t)wave_reduce((int)(x >> 32), -1, both) << 32) |
                   (uint32_t)wave_reduce((int)(uint32_t)x, -1, both);
        };
        ones = all_of(ones);
        zeros = all_of(zeros);
        if (lane == 0) {
            same[0][wave] = ones;
            same[1][wave] = zeros;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            ones &= same[0][w];
            zeros &= same[1][w];
        }
        const uint64_t differ = uniform64((long long)~(ones | zeros));
        int shift = differ ? (63 - __builtin_clzll(differ)) / 8 * 8 : 0;
        uint64_t prefix = shift < 56 ? uniform64((long long)ones) >> (shift + 8) << (shift + 8) : 0;
        const int top_shift = shift;
        int need = n_top;
        for (;; shift -= 8) {
            for (int i = threadIdx.x; i < 256; i += THREADS)
                hist[i] = 0;
            __syncthreads();
            for (int i0 = wave * kWave; i0 < n_old; i0 += THREADS) {
                const int i = i0 + lane;
                const uint64_t k = i < n_old ? key(i) : 0ull;
                const bool in = i < n_old &&
                                (shift == top_shift ||
                                 (k >> (shift + 8)) == (prefix >> (shift + 8)));
                const int d = (int)(k >> shift) & 255;
                // many keys share their first digits: those of the wave's first
                // such key go in as one
                const uint64_t live = __ballot(in);
                if (!live)
                    continue;
                const int lead = __builtin_ctzll(live);
                const int d0 = __builtin_amdgcn_readlane(d, lead);
                const uint64_t same = __ballot(in && d == d0);
                if (lane == lead)
                    atomicAdd(&hist[d0], __popcll(same));
                else if (in && d != d0)
                    atomicAdd(&hist[d], 1);
            }
            __syncthreads();
            // the digit of the need-th largest key: bins from the top on
            if (wave == 0) {
                int mine[4], sum = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    mine[j] = hist[255 - (4 * lane + j)];
                    sum += mine[j];
                }
                const int incl = (int)wave_scan_add(sum);
                int before = incl - sum;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (before < need && need <= before + mine[j]) {
                        digit = 255 - (4 * lane + j);
                        above = before;
                    }
                    before += mine[j];
                }
            }
            __syncthreads();
            need -= above;
            prefix |= (uint64_t)digit << shift;
            const bool whole = hist[digit] == need;
            if (shift == 0 || whole)
                break;
            __syncthreads();
        }
        // every key from `prefix` on: all of them where the last bin was taken
        // whole, else the first `need` of those equal to it
        least = prefix;
        equal_quota = shift == 0 ? need : n_old;
        if (least == 0)                              // fewer pages than n_top have entries
            least = 1, equal_quota = n_old;
    } else {
        __syncthreads();
    }

    // ---- list them in page order: a run of pages per wave ----
    const int run = (n_old + WAVES * kWave - 1) / (WAVES * kWave) * kWave;
    const int i0 = wave * run, i1 = min(i0 + run, n_old);
    auto tally = [&](int i, bool &gt, bool &eq) {
        const uint64_t k = i < i1 ? key(i) : 0ull;
        gt = k > least;
        eq = k == least;
    };
    int n_gt = 0, n_eq = 0;
    for (int i = i0; i < i1; i += kWave) {
        bool gt, eq;
        tally(i + lane, gt, eq);
        n_gt += __popcll(__ballot(gt));
        n_eq += __popcll(__ballot(eq));
    }
    if (lane == 0) {
        wave_count[0][wave] = n_gt;
        wave_count[1][wave] = n_eq;
    }
    __syncthreads();
    int at = 0, eq_seen = 0, all_gt = 0, all_eq = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const int gt = wave_count[0][w], eq = wave_count[1][w];
        if (w < wave) {
            at += gt + min(eq, max(equal_quota - eq_seen, 0));
            eq_seen += eq;
        }
        all_gt += gt;
        all_eq += eq;
    }
    const int listed = all_gt + min(all_eq, equal_quota);
    int32_t *out = a.sel + (size_t)unit * a.n_sel;
    const uint64_t below = (1ull << lane) - 1ull;
    for (int i = i0; i < i1; i += kWave) {
        bool gt, eq;
        tally(i + lane, gt, eq);
        const uint64_t em = __ballot(eq);
        const bool take = gt || (eq && eq_seen + __popcll(em & below) < equal_quota);
        const uint64_t tm = __ballot(take);
        if (take)
            out[at + __popcll(tm & below)] = i + lane;
        at += __popcll(tm);
        eq_seen += __popcll(em);
    }
    // the recent pages, and -1 behind them
    const int recent = newest + 1 - n_old;
    for (int i = listed + threadIdx.x; i < a.n_sel; i += THREADS)
        out[i] = i - listed < recent ? n_old + i - listed : -1;
}

}  // namespace

wf_status_t launch_paged_append(wf_dtype_t dt, const wf_paged_cache_t &c,
                                const wf_paged_batch_t &b, const void *k, const void *v,
                                size_t kv_stride, const void *q, size_t q_stride, void *q_out,
                                int n_q_heads, const int32_t *positions, double rope_base,
                                int n_rows, hipStream_t stream) {
    AppendParams a{};
    a.v = paged_view(c, b, n_rows);
    // base^(-2 i / D) = base^(-2 (i - i % 8) / D) base^(-2 (i % 8) / D): two roundings
    // more than a power each, a quarter of its time on the host
    double fine[8];
    for (int i = 0; i < 8; ++i)
        fine[i] = std::pow(rope_base, -2.0 * i / c.head_dim) / 6.283185307179586;
    for (int i = 0; i < c.head_dim / 2; i += 8) {
        const double coarse = std::pow(rope_base, -2.0 * i / c.head_dim);
        for (int j = 0; j < 8; ++j)
            a.turns[i + j] = coarse * fine[j];
    }
    a.k_in = k;
    a.v_in = v;
    a.q_in = q;
    a.k = c.k;
    a.vc = c.v;
    a.bounds = c.bounds;
    a.q_out = q_out;
    a.positions = positions;
    a.kv_stride = kv_stride;
    a.q_stride = q_stride;
    a.n_q_heads = n_q_heads;
    a.group = q ? n_q_heads / c.n_kv_heads : 0;
    // at most this many pages receive rows, each row of one sequence: a sequence's
    // rows reach one page more than they fill
    const int pages = (int)std::min<long long>(
        n_rows, n_rows / c.page_size + 2ll * std::min(b.n_seqs, n_rows));
    // as many workgroups as fill the chip four times over, no more than heads
    a.run = std::max(1, c.n_kv_heads / std::max(1, 1024 / pages));
    const dim3 grid(pages, (c.n_kv_heads + a.run - 1) / a.run);
    const dim3 block(kThreads);
    const size_t lds = (size_t)2 * c.page_size * (c.head_dim / 2 + 4) * sizeof(float);
    if (dt == WF_BF16) {
        if (c.head_dim == 128)
            hipLaunchKernelGGL((paged_append<uint16_t, 128>), grid, block, lds, stream, a);
        else
            hipLaunchKernelGGL((paged_append<uint16_t, 64>), grid, block, lds, stream, a);
    } else if (c.head_dim == 128)
        hipLaunchKernelGGL((paged_append<float, 128>), grid, block, lds, stream, a);
    else
        hipLaunchKernelGGL((paged_append<float, 64>), grid, block, lds, stream, a);
    return hipGetLastError() == hipSuccess ? WF_OK : WF_ERR_HIP;
}

size_t paged_select_workspace_bytes(int n_rows, int n_kv_heads, int max_pages) {
    const size_t units = std::max<size_t>((size_t)n_rows * n_kv_heads, 1);
    return kCounterBytes + units * max_pages * sizeof(uint64_t);
}

wf_status_t launch_paged_select(wf_dtype_t dt, const void *q, const wf_paged_cache_t &c,
                                const wf_paged_batch_t &b, int32_t *sel, int n_sel, int n_recent,
                                int n_rows, int n_q_heads, void *workspace, hipStream_t stream) {
    SelectParams a{};
    a.v = paged_view(c, b, n_rows);
    a.q = q;
    a.bounds = c.bounds;
    a.sel = sel;
    a.keys = reinterpret_cast<uint64_t *>(static_cast<char *>(workspace) + kCounterBytes);
    a.n_sel = n_sel;
    a.n_recent = n_recent;
    a.group = n_q_heads / c.n_kv_heads;
    a.n_q_heads = n_q_heads;
    a.pack = std::min(std::max(16 / a.group, 1), b.max_rows);
    // two workgroups a CU share the tiles evenly; there are at most this many
    const long long tiles = (long long)std::min(n_rows, n_rows / a.pack + b.n_seqs) *
                            c.n_kv_heads * ((b.max_pages + 15) / 16);
    const dim3 grid((unsigned)std::min<long long>(512, (tiles + 3) / 4));
    const dim3 block(kThreads);
    if (n_sel > n_recent) {
        if (dt == WF_BF16) {
            if (c.head_dim == 128)
                hipLaunchKernelGGL((paged_scores<uint16_t, 128>), grid, block, 0, stream, a);
            else
                hipLaunchKernelGGL((paged_scores<uint16_t, 64>), grid, block, 0, stream, a);
        } else if (c.head_dim == 128)
            hipLaunchKernelGGL((paged_scores<float, 128>), grid, block, 0, stream, a);
        else
            hipLaunchKernelGGL((paged_scores<float, 64>), grid, block, 0, stream, a);
    }
    hipLaunchKernelGGL((paged_choose<512>), dim3(n_rows * c.n_kv_heads), dim3(512), 0, stream, a);
    return hipGetLastError() == hipSuccess ? WF_OK : WF_ERR_HIP;
}

}  // namespace wf
