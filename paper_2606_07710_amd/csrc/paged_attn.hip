// paged_attn.hip -- verification attention of a batch of requests over a paged
// KV cache (the parallel verification of Sec. 3.2 of the WhiFlash paper, for
// many requests at once), over all of a sequence's pages or over a selection.
//
// The work is a list of items, each up to ROWS query rows that read one KV
// head's keys: dense, (sequence, KV head, row group); sparse, (row, KV head,
// group of query heads).  An item's keys are cut into chunks of kChunk, and all
// items' chunks, laid end to end, are dealt out in equal runs to a fixed number
// of workgroups: however ragged the batch, every workgroup has the same number
// of chunks, and the lengths may live on the device.  An item that lies within
// one run is finished there; the others leave one partial per run (the
// unnormalised rows, running maximum and sum in fp32), which a second launch
// joins in run order.
//
// bf16, per 32-key tile and wave, as in the dense kernel (attn.hip):
//   S^T = K Q^T    A = 16 keys x 32 dims from the LDS copy of the K tile
//   P   = exp2((S - m) * scale * log2 e), online maximum and sum per row
//   O^T += V^T P^T   A from transposing reads of the LDS copy of the V tile
// P goes into the second product in bf16, the type that the matrix instruction
// takes beside V, as in the dense kernel; its sum is of the unrounded weights, and
// all else is fp32 up to the output.  So a weight is off by half a step, 2^-8, at
// most, and the output by 0.0022 of itself in the mean square, where its own
// rounding alone is 0.0017.  (The rest of each weight as a second bf16 operand gives
// 0.0017: decoding takes 0.3 % longer, blocks 2 %, trees 45 -> 48 us, and an infinite
// V beside a weight without a rest becomes NaN.)
// fp32: the same with the fp32 matrix instruction, operands from memory.
//
// What bounds it (32 heads over 8 of 128, attention and join): decoding 128
// requests of up to 16K keys moves 3.0 GB in 462 us, 6.5 TB/s; 45 rows' selections
// of 122 pages of 32 keys 0.68 GB in 110 us, 6.2 TB/s.  Blocks of 16 rows (16 requests
// of up to 8K, 183 MB, 46 us) and draft trees (4 of 61 nodes, 55 MB and 11.5 GFLOP,
// 43 us) are bound by the issue of the loads and of exp2 and by the partials, one
// request of 1K keys (9.5 us) by launch and dependent trips.
#include "wf_lds_dma.h"
#include "wf_paged.h"

namespace wf {

namespace {

constexpr int kChunk = 128;        // keys
constexpr int kTile = 32;
constexpr int kWorkgroups = 256;
constexpr int kMetaInts = 8;

struct PagedAttnParams {
    PagedView v;
    const void *q, *k, *vc;
    void *out;
    const int32_t *sel;            // null: dense
    const uint64_t *tree_mask;
    int n_sel, group, n_q_heads;
    float sl2;                     // softmax scale * log2 e
    const char *zeros;             // kPagedZeroBytes of zeros
    float *part_o;                 // [2 * workgroups][ROWS][DH]
    float *part_ml;                // [2 * workgroups][ROWS][2]
    int32_t *meta;                 // [workgroups][kMetaInts]: the split item that
                                   // begins in the workgroup
};

// One item: rows [r0, r0 + rows) of the call, query row q of it = (row r0 + q /
// heads, head h0 + q % heads), `first` the item's first query row.
struct Item {
    int b, r0, rows, ctx, g, h0, heads, first, n_q, chunks, n_keys;
};

// Units are chunks; sequence b's are [KV head][row group][chunk] (dense).
template <int ROWS>
__device__ __forceinline__ long long dense_units(const PagedAttnParams &a, const Seq &s) {
    if (!s.rows)
        return 0;
    const int groups = (s.rows * a.group + ROWS - 1) / ROWS;
    const int chunks = (s.ctx + s.rows + kChunk - 1) / kChunk;
    return (long long)a.v.n_kv_heads * groups * chunks;
}

// Runs of `total` units for W workgroups: the first `more` of them have len + 1.
// (Units count in 32 bits: 2^31 chunks are more than a day's work of 2^47 bytes;
// a batch with more of them is not run at all.)
struct Runs {
    int len, more;
    __device__ __forceinline__ Runs(int total, int W) : len(total / W) { more = total - len * W; }
    __device__ __forceinline__ int begin(int w) const { return len * w + min(w, more); }
    __device__ __forceinline__ int owner(int u) const {
        const int split = more * (len + 1);
        return u < split ? u / (len + 1) : more + (u - split) / len;
    }
};

// ---------------------------------------------------------------------------
// Pages of a key list: 64 of them at a time in the lanes of a wave.
// ROW_BYTES: of a key.
template <bool SPARSE, int ROW_BYTES>
struct Pages {
    // of list page base + lane: where its KV head's keys start in the pool, in
    // bytes (hi < 0: no such page), and the position of its first key
    int lo, hi, pos;
    int base;

    __device__ __forceinline__ void load(const PagedAttnParams &a, const Item &it, int at) {
        base = at;
        const int i = at + (int)(threadIdx.x % kWave);
        int p = i;
        if constexpr (SPARSE) {
            p = i < a.n_sel
                    ? a.sel[((size_t)it.r0 * a.v.n_kv_heads + it.g) * a.n_sel + i] : -1;
            if (p > (it.n_keys - 1) >> a.v.page_shift)
                p = -1;
        } else if (i > (it.n_keys - 1) >> a.v.page_shift) {
            p = -1;
        }
        const int id = p >= 0 ? paged_page(a.v, it.b, p) : -1;
        const size_t off = (((size_t)max(id, 0) * a.v.n_kv_heads + it.g) << a.v.page_shift) *
                           ROW_BYTES;
        lo = (int)(unsigned)off;
        hi = id < 0 ? -1 : (int)(off >> 32);
        pos = p << a.v.page_shift;
    }
    // 16 keys from list key k on (k % 16 == 0, wave-uniform, its page among the
    // 64): their position, how many of them there are, where in the pool
    __device__ __forceinline__ void find(const PagedAttnParams &a, const Item &it, int k, int &at,
                                         int &n, size_t &off) const {
        const int lane = (k >> a.v.page_shift) - base;
        const int in = k & ((1 << a.v.page_shift) - 1);
        const int h = __builtin_amdgcn_readlane(hi, lane);
        at = SPARSE ? __builtin_amdgcn_readlane(pos, lane) + in : k;
        n = h < 0 ? 0 : min(max(it.n_keys - at, 0), 16);
        off = (((size_t)(unsigned)h << 32) | (unsigned)__builtin_amdgcn_readlane(lo, lane)) +
              (unsigned)(in * ROW_BYTES);
    }
};

// ---------------------------------------------------------------------------
// What a wave's 16 * NB rows know of themselves.
template <int NB>
struct Rows {
    int i[NB], h[NB];              // row of the sequence (clamped), head
    uint64_t mask[NB];

    __device__ __forceinline__ void set(const PagedAttnParams &a, const Item &it, int row0) {
        const int m16 = threadIdx.x & 15;
        // (q < 2^14 and at most 256 heads: (q + 1/2) / heads is at least 2^-9 away
        // from a whole number, the product off by less than 2^-15)
        const float per_row = __builtin_amdgcn_rcpf((float)it.heads);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            // rows past the item's repeat its last one and are not stored
            const int q = min(it.first + row0 + nb * 16 + m16, it.n_q - 1);
            i[nb] = (int)(((float)q + 0.5f) * per_row);
            h[nb] = it.h0 + q - i[nb] * it.heads;
        }
    }
    __device__ __forceinline__ void load_mask(const PagedAttnParams &a, const Item &it, int seq_i) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
            mask[nb] = a.tree_mask
                           ? a.tree_mask[it.r0 + i[nb]] | (1ull << (seq_i + i[nb]))
                           : 0ull;
    }
};

// Item -> output rows or a partial.  lds_o holds the KS streams' unnormalised
// rows [KS][ROWS][DH + 4], lds_ml their (maximum, sum).
template <typename T, int DH, int ROWS, int KS, int THREADS>
__device__ __forceinline__ void store_item(const PagedAttnParams &a, const Item &it, bool whole,
                                           int slot, const float *lds_o,
                                           const float (*lds_ml)[ROWS][2]) {
    constexpr int OST = DH + 4, PIECES = DH / 8;
    for (int pc = threadIdx.x; pc < ROWS * PIECES; pc += THREADS) {
        const int row = pc / PIECES, d = pc % PIECES * 8;
        const int q = it.first + row;
        if (q >= it.n_q)
            continue;
        float m = -INFINITY;
#pragma unroll
        for (int s = 0; s < KS; ++s)
            m = fmaxf(m, lds_ml[s][row][0]);
        const float muse = m == -INFINITY ? 0.f : m;
        float l = 0.f;
        f32x4 o0 = {0.f, 0.f, 0.f, 0.f}, o1 = o0;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const float f = KS == 1 ? 1.f : fast_exp2((lds_ml[s][row][0] - muse) * a.sl2);
            l += lds_ml[s][row][1] * f;
            const float *src = lds_o + (s * ROWS + row) * OST + d;
            o0 += *reinterpret_cast<const f32x4 *>(src) * f;
            o1 += *reinterpret_cast<const f32x4 *>(src + 4) * f;
        }
        if (whole) {
            // (a row that saw nothing has l = 0 and o = 0; NaN stays NaN)
            const float inv = l == 0.f ? 0.f : 1.f / l;
            o0 *= inv;
            o1 *= inv;
            T *dst = static_cast<T *>(a.out) +
                     ((size_t)(it.r0 + q / it.heads) * a.n_q_heads + it.h0 + q % it.heads) * DH + d;
            if constexpr (sizeof(T) == 2) {
                *reinterpret_cast<u32x4 *>(dst) =
                    u32x4{pack_bf16x2(o0[0], o0[1]), pack_bf16x2(o0[2], o0[3]),
                          pack_bf16x2(o1[0], o1[1]), pack_bf16x2(o1[2], o1[3])};
            } else {
                *reinterpret_cast<f32x4 *>(dst) = o0;
                *reinterpret_cast<f32x4 *>(dst + 4) = o1;
            }
        } else {
            float *dst = a.part_o + ((size_t)slot * ROWS + row) * DH + d;
            *reinterpret_cast<f32x4 *>(dst) = o0;
            *reinterpret_cast<f32x4 *>(dst + 4) = o1;
            if (d == 0) {
                a.part_ml[((size_t)slot * ROWS + row) * 2] = m;
                a.part_ml[((size_t)slot * ROWS + row) * 2 + 1] = l;
            }
        }
    }
}

// ---------------------------------------------------------------------------
// The walk over a workgroup's run: calls segment(item, chunk0, n) for each
// piece of an item in it, and store(item, whole, slot) after it.
template <bool SPARSE, int ROWS, int THREADS, typename Segment, typename Store>
__device__ __forceinline__ void walk(const PagedAttnParams &a, Segment &&segment, Store &&store) {
    const int w = blockIdx.x;
    Item it;
    int item0 = 0;                 // the item's first unit
    int item = 0;                  // dense: item of the sequence; sparse: of all
    int b = 0, total = 0;
    Seq s{0, 0, 0};
    const int sparse_groups = (a.group + ROWS - 1) / ROWS;
    const int sparse_chunks =
        SPARSE ? (int)((((long long)a.n_sel << a.v.page_shift) + kChunk - 1) / kChunk) : 0;
    // ---- where the run begins ----
    auto workgroups = [&](int n) { return min((int)gridDim.x, max(n, 1)); };
    if constexpr (SPARSE) {
        total = a.v.n_rows * a.v.n_kv_heads * sparse_groups * sparse_chunks;
    } else {
        long long first, all;
        Seq q;
        b = paged_find<THREADS>(
            a.v, a.v.max_rows,
            [&](long long n) -> long long {
                if (n > 0x7fffffff)
                    return n;
                const int of = workgroups((int)n);
                return w < of ? Runs((int)n, of).begin(w) : n;
            },
            [&](const Seq &o) { return dense_units<ROWS>(a, o); }, &first, &all, &q);
        if (b >= 0) {
            s = q;
            item0 = (int)first;
            total = (int)all;
        }
    }
    const int active = workgroups(total);
    const Runs runs(total, active);
    int tail_owner = -1;           // last workgroup of the split item that begins here
    Item tail{};
    if (w < active && total > 0) {
        int at = runs.begin(w);
        const int end = runs.begin(w + 1);
        if constexpr (SPARSE) {
            item = at / sparse_chunks;
            item0 = item * sparse_chunks;
        } else {
            const int chunks = (s.ctx + s.rows + kChunk - 1) / kChunk;
            item = (at - item0) / chunks;
            item0 += item * chunks;
        }
        int row_now = -1;
        while (at < end) {
            if constexpr (SPARSE) {
                const int grp = item % sparse_groups;
                const int rg = item / sparse_groups;
                const int row = rg / a.v.n_kv_heads;
                it.g = rg % a.v.n_kv_heads;
                if (row != row_now) {
                    row_now = row;
                    __shared__ int owner;
                    __syncthreads();
                    if (threadIdx.x == 0)
                        owner = -1;
                    __syncthreads();
                    for (int i = threadIdx.x; i < a.v.n_seqs; i += THREADS) {
                        const Seq o = paged_seq(a.v, i, a.v.max_rows);
                        if (row >= o.r0 && row < o.r0 + o.rows)
                            owner = i;
                    }
                    __syncthreads();
                    b = uniform(owner);
                    if (b >= 0)
                        s = paged_seq(a.v, b, a.v.max_rows);
                }
                it.b = b;
                it.r0 = row;
                it.rows = 1;
                it.ctx = s.ctx;
                it.h0 = it.g * a.group;
                it.heads = a.group;
                it.first = grp * ROWS;
                it.n_q = a.group;
                it.chunks = sparse_chunks;
                it.n_keys = s.ctx + (row - s.r0) + 1;
            } else {
                const int groups = (s.rows * a.group + ROWS - 1) / ROWS;
                it.b = b;
                it.r0 = s.r0;
                it.rows = s.rows;
                it.ctx = s.ctx;
                it.g = item / groups;
                it.h0 = it.g * a.group;
                it.heads = a.group;
                it.first = item % groups * ROWS;
                it.n_q = s.rows * a.group;
                it.n_keys = s.ctx + s.rows;
                it.chunks = (it.n_keys + kChunk - 1) / kChunk;
            }
            const int chunk0 = at - item0;
            const int n = min(it.chunks - chunk0, end - at);
            const bool whole = n == it.chunks;
            const bool tail_piece = chunk0 == 0 && !whole;
            if (!SPARSE || it.b >= 0) {
                segment(it, SPARSE ? it.r0 - s.r0 : 0, chunk0, n);
                // a run's pieces of split items: the one that it begins with
                // and the one that it ends with
                store(it, whole, 2 * w + (tail_piece ? 1 : 0));
            }
            if (tail_piece && it.b >= 0) {
                tail_owner = runs.owner(item0 + it.chunks - 1);
                tail = it;
            }
            at += n;
            item0 += it.chunks;
            ++item;
            if constexpr (!SPARSE) {
                // the next item of this sequence, or the next sequence's first
                const int groups = (s.rows * a.group + ROWS - 1) / ROWS;
                if (at < end && item == a.v.n_kv_heads * groups) {
                    item = 0;
                    do
                        s = paged_seq(a.v, ++b, a.v.max_rows);
                    while (!s.rows);
                }
            }
        }
    }
    if (threadIdx.x == 0) {
        int32_t *m = a.meta + w * kMetaInts;
        m[0] = tail_owner;
        m[1] = tail.r0;
        m[2] = tail.h0;
        m[3] = tail.heads;
        m[4] = tail.first;
        m[5] = tail.n_q;
    }
}

// ---------------------------------------------------------------------------
// bf16.  A workgroup is KS key streams x RG row groups of waves; a tile of 32
// keys travels memory -> LDS in 1 KB wave loads, split over the RG waves that
// share it, into a ring of NBUF stages.  With RG == 1 every wave has a ring of
// its own and no barrier but the one at an item's end.
//
// LDS tile = K rows, then V rows, swizzled so that the operand reads are free
// of bank conflicts: K's 16-byte granule g of key k at g ^ (k mod GRAN), V's
// 32-byte segment j at j ^ (k mod SEGS).
template <int DH, int NB, int RG, int KS, int NBUF, bool SPARSE>
__global__ __launch_bounds__(64 * KS * RG) void paged_attn_bf16(PagedAttnParams a) {
    constexpr int THREADS = 64 * KS * RG;
    constexpr int ROWS = 16 * NB * RG;
    // Up to 64 rows an item's keys are read by this workgroup alone and only
    // once: with the non-temporal hint they pass the caches by (128 rows of up to
    // 16K keys: 520 -> 465 us, 16 blocks of 16: 53 -> 47).  Several row groups,
    // and the rows of a sequence that select the same pages, share them there.
    constexpr bool NT = !SPARSE && NB == 1;
    constexpr int RB = DH * 2;                        // row bytes
    constexpr int HALF = kTile * RB;
    constexpr int TILE = 2 * HALF;
    constexpr int GRAN = RB / 16, SEGS = RB / 32;
    constexpr int KC = DH / 32, MD = DH / 16;
    constexpr int LPH = 16 * RB / 1024;               // wave loads for 16 keys of K or V
    constexpr int NLOAD = 4 * LPH;
    constexpr int LPW = NLOAD / RG;
    static_assert(NLOAD % RG == 0, "tile loads must split evenly over row groups");
    constexpr int RING = NBUF * KS * TILE;
    constexpr int OST = DH + 4;
    constexpr int MERGE = KS * ROWS * OST * 4;
    constexpr int SMEM = RING > MERGE ? RING : MERGE;
    static_assert(SMEM + KS * ROWS * 8 + 2048 <= 160 * 1024, "LDS budget");
    __shared__ __attribute__((aligned(1024))) char smem[SMEM];
    __shared__ float ml[KS][ROWS][2];

    const int wave = wave_id();
    const int lane = threadIdx.x % kWave;
    const int m16 = lane & 15, c4 = lane >> 4;
    const int stream = wave % KS, rgi = wave / KS;
    const float sl2 = a.sl2;

    // This wave's loads of a tile: RG waves share the LPH loads that 16 keys of K
    // (or V) take, or (LPH < RG) a half's go to some waves and the other's to the
    // others.  A lane's byte offset in the 16 keys, swizzled (the swizzles repeat
    // after 16 keys):
    constexpr int NJ = LPH >= RG ? LPH / RG : 1;
    constexpr int RPL = 1024 / RB;                    // keys per load
    unsigned koff[NJ], voff[NJ], row_of[NJ];
#pragma unroll
    for (int ji = 0; ji < NJ; ++ji) {
        const int j = LPH >= RG ? rgi + ji * RG : rgi % LPH;
        const int kl = j * RPL + lane / GRAN, pg = lane % GRAN;
        const int seg = (pg >> 1) ^ (kl & (SEGS - 1));
        row_of[ji] = kl;
        koff[ji] = (unsigned)(kl * RB + (pg ^ (kl & (GRAN - 1))) * 16);
        voff[ji] = (unsigned)(kl * RB + (2 * seg + (pg & 1)) * 16);
    }
    // Where a lane's operands lie in its stream's tile: K's granules (16 keys
    // further on by an immediate offset), V's segments.
    const WF_LDS(char) *const tile0 = (const WF_LDS(char) *)smem + stream * TILE;
    int kread[KC], vread[MD];
    const int q4 = m16 & 3, qk = m16 >> 2;
#pragma unroll
    for (int kk = 0; kk < KC; ++kk)
        kread[kk] = m16 * RB + ((4 * kk + c4) ^ (m16 & (GRAN - 1))) * 16;
#pragma unroll
    for (int md = 0; md < MD; ++md)
        vread[md] = (4 * c4 + qk) * RB + (md ^ ((4 * c4 + qk) & (SEGS - 1))) * 32 + q4 * 8;

    bf16x8 qf[NB][KC];
    f32x4 o[MD][NB];
    float mref[NB], lrow_sum[NB];

    auto segment = [&](const Item &it, int seq_i, int chunk0, int n) __attribute__((always_inline)) {
        const int list_end = SPARSE ? a.n_sel << a.v.page_shift : it.n_keys;
        const int k_begin = chunk0 * kChunk;
        const int k_end = min(k_begin + n * kChunk, list_end);
        const int n_tiles = (k_end - k_begin + kTile - 1) / kTile;
        // waves that share barriers take the same number of steps
        const int n_steps = RG > 1 ? (n_tiles + KS - 1) / KS
                                   : (n_tiles - stream + KS - 1) / KS;
        Rows<NB> rows;
        rows.set(a, it, rgi * 16 * NB);
        rows.load_mask(a, it, seq_i);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const uint16_t *qp = static_cast<const uint16_t *>(a.q) +
                                 ((size_t)(it.r0 + rows.i[nb]) * a.n_q_heads + rows.h[nb]) * DH +
                                 c4 * 8;
#pragma unroll
            for (int kk = 0; kk < KC; ++kk)
                qf[nb][kk] = load_bf16x8(qp + kk * 32);
            mref[nb] = -INFINITY;
            lrow_sum[nb] = 0.f;
#pragma unroll
            for (int md = 0; md < MD; ++md)
                o[md][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        Pages<SPARSE, RB> pages;
        pages.load(a, it, (k_begin + stream * kTile) >> a.v.page_shift);

        // position and number of the keys in the two halves of a stage's tile
        struct Where {
            int pos[2], n[2];
        };
        Where ring_where[NBUF - 1];

        // (the ring's buffer is known where a step is compiled, so that addresses
        // in it are immediates)
        auto issue = [&](auto bi, int st) __attribute__((always_inline)) -> Where {
            const int kb = k_begin + (KS * st + stream) * kTile;
            const unsigned slot =
                lds_addr(smem) + stream * TILE + decltype(bi)::value * (KS * TILE);
            if ((kb + 16) >> a.v.page_shift >= pages.base + kWave)
                pages.load(a, it, kb >> a.v.page_shift);
            Where wh;
            size_t off[2];
            pages.find(a, it, kb, wh.pos[0], wh.n[0], off[0]);
            if (a.v.page_shift > 4) {                // the same page
                wh.pos[1] = wh.pos[0] + 16;
                wh.n[1] = wh.n[0] < 16 ? 0 : min(max(it.n_keys - wh.pos[1], 0), 16);
                off[1] = off[0] + 16 * RB;
            } else {
                pages.find(a, it, kb + 16, wh.pos[1], wh.n[1], off[1]);
            }
            auto copy = [&](auto whole_tag) __attribute__((always_inline)) {
                constexpr bool WHOLE = decltype(whole_tag)::value;
#pragma unroll
                for (int jr = 0; jr < LPW; ++jr) {
                    const bool is_v = jr >= LPW / 2;
                    const int hf = LPH >= RG ? jr / NJ % 2 : rgi / LPH;
                    const int ji = LPH >= RG ? jr % NJ : 0;
                    const int j = LPH >= RG ? rgi + ji * RG : rgi % LPH;
                    const char *src =
                        static_cast<const char *>(is_v ? a.vc : a.k) + (hf ? off[1] : off[0]);
                    unsigned at = is_v ? voff[ji] : koff[ji];
                    if constexpr (!WHOLE) {
                        // keys that are not there repeat the half's last one, or
                        // are zeros
                        const int n = hf ? wh.n[1] : wh.n[0];
                        src = n ? src : a.zeros;
                        at -= (row_of[ji] - min(row_of[ji], (unsigned)max(n - 1, 0))) * RB;
                    }
                    // (the copy takes scalars; these are, but the compiler may hold
                    // them in vector registers)
                    lds_dma16_so<NT>(
                        reinterpret_cast<const char *>(uniform64(reinterpret_cast<intptr_t>(src))),
                        at, uniform((int)(slot + (is_v ? HALF : 0) + (hf * LPH + j) * 1024)));
                }
            };
            if (wh.n[0] + wh.n[1] == 32)
                copy(std::true_type{});
            else
                copy(std::false_type{});
            return wh;
        };

        auto compute = [&](auto bi, const Where &wh) __attribute__((always_inline)) {
            const WF_LDS(char) *kt = tile0 + decltype(bi)::value * (KS * TILE);
            const WF_LDS(char) *vt = kt + HALF;
            f32x4 s[2][NB];
#pragma unroll
            for (int mb = 0; mb < 2; ++mb) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
                    s[mb][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < KC; ++kk) {
                    const bf16x8 kop = __builtin_bit_cast(
                        bf16x8, *(const WF_LDS(u32x4) *)(kt + kread[kk] + 16 * mb * RB));
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
                        s[mb][nb] = mfma16x16x32(kop, qf[nb][kk], s[mb][nb]);
                }
            }
            // V^T, while the scores are formed: two transposing reads per 16 dims
            typedef short v4i16 __attribute__((ext_vector_type(4)));
            typedef short v8i16 __attribute__((ext_vector_type(8)));
            bf16x8 vop[MD];
#pragma unroll
            for (int md = 0; md < MD; ++md) {
                v4i16 half[2];
#pragma unroll
                for (int hh = 0; hh < 2; ++hh)
                    half[hh] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (WF_LDS(v4i16) *)(vt + vread[md] + 16 * hh * RB));
                const v8i16 both = __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7);
                vop[md] = __builtin_bit_cast(bf16x8, both);
            }
            // masks, where a half is short or reaches into the block
            if (wh.n[0] + wh.n[1] < 32 || max(wh.pos[0], wh.pos[1]) + 15 >= it.ctx) {
#pragma unroll
                for (int mb = 0; mb < 2; ++mb)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int j = wh.pos[mb] + 4 * c4 + i - it.ctx;
                            const int me = seq_i + rows.i[nb];
                            const bool seen =
                                a.tree_mask ? ((rows.mask[nb] >> (j & 63)) & 1ull) != 0 : j <= me;
                            const bool vis = (4 * c4 + i < wh.n[mb]) & ((j < 0) | seen);
                            s[mb][nb][i] = vis ? s[mb][nb][i] : -INFINITY;
                        }
            }
            // The reference maximum of a row moves only when a score outgrows it
            // by 8 log2 units: weights stay below 2^8, exact either way.  Only
            // then (and at the first keys) do the row's four lanes compare notes.
            float mx[NB];
            bool grow = false;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                mx[nb] = fmaxf(fmaxf(fmaxf(s[0][nb][0], s[0][nb][1]), fmaxf(s[0][nb][2], s[0][nb][3])),
                               fmaxf(fmaxf(s[1][nb][0], s[1][nb][1]), fmaxf(s[1][nb][2], s[1][nb][3])));
                grow |= (mx[nb] - mref[nb]) * sl2 > 8.f;
            }
            if (__ballot(grow)) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    float m = fmaxf(mx[nb], __shfl_xor(mx[nb], 16, kWave));
                    m = fmaxf(m, __shfl_xor(m, 32, kWave));
                    const bool up = (m - mref[nb]) * sl2 > 8.f;
                    const float alpha = up ? fast_exp2((mref[nb] - m) * sl2) : 1.f;
                    mref[nb] = up ? m : mref[nb];
                    lrow_sum[nb] *= alpha;
#pragma unroll
                    for (int md = 0; md < MD; ++md)
                        o[md][nb] *= alpha;
                }
            }
            bf16x8 pb[NB];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const float mu = mref[nb] == -INFINITY ? 0.f : mref[nb];
                float p[8];
                float sum = 0.f;
#pragma unroll
                for (int mb = 0; mb < 2; ++mb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        // the difference first: scores may be far larger than
                        // their differences
                        p[4 * mb + i] = fast_exp2((s[mb][nb][i] - mu) * sl2);
                        sum += p[4 * mb + i];
                    }
                lrow_sum[nb] += sum;
                const u32x4 pv = {pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]),
                                  pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])};
                pb[nb] = __builtin_bit_cast(bf16x8, pv);
            }
#pragma unroll
            for (int md = 0; md < MD; ++md)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
                    o[md][nb] = mfma16x16x32(vop[md], pb[nb], o[md][nb]);
        };

        // q is in before the first copy goes out, so that the compiler waits
        // for none of the copies on its account
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int kk = 0; kk < KC; ++kk)
                asm volatile("" : "+v"(qf[nb][kk]));
        asm volatile("" : "+v"(pages.lo), "+v"(pages.hi), "+v"(pages.pos));
        if (0 < n_steps)
            ring_where[0] = issue(ic<0>{}, 0);
        if constexpr (NBUF > 2)
            if (1 < n_steps)
                ring_where[1] = issue(ic<1>{}, 1);
        auto step = [&](auto bi, int st) __attribute__((always_inline)) {
            constexpr int B = decltype(bi)::value;
            // stage st is in LDS once only the later stages' copies are out
            if (NBUF > 2 && st + 1 < n_steps)
                wait_vmcnt<LPW>();
            else
                wait_vmcnt<0>();
            // ... for every wave that copied a part of it, and every wave is
            // done with stage st - 1, whose buffer takes the next copies
            if constexpr (RG > 1)
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            else
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            const Where now = ring_where[0];
            if constexpr (NBUF > 2)
                ring_where[0] = ring_where[1];
            if (st + NBUF - 1 < n_steps)
                ring_where[NBUF - 2] = issue(ic<(B + NBUF - 1) % NBUF>{}, st + NBUF - 1);
            if (RG == 1 || KS * st + stream < n_tiles)
                compute(bi, now);
        };
        static_assert(NBUF == 2 || NBUF == 3, "the steps of a turn of the ring");
        for (int st = 0; st < n_steps; st += NBUF) {
            step(ic<0>{}, st);
            if (st + 1 < n_steps)
                step(ic<1>{}, st + 1);
            if constexpr (NBUF > 2)
                if (st + 2 < n_steps)
                    step(ic<2>{}, st + 2);
        }
        // ---- the streams' rows meet in LDS ----
        __syncthreads();
        float *so = reinterpret_cast<float *>(smem);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            float l = lrow_sum[nb];
            l += __shfl_xor(l, 16, kWave);
            l += __shfl_xor(l, 32, kWave);
            const int r = (rgi * NB + nb) * 16 + m16;
            if (c4 == 0) {
                ml[stream][r][0] = mref[nb];
                ml[stream][r][1] = l;
            }
#pragma unroll
            for (int md = 0; md < MD; ++md)
                *reinterpret_cast<f32x4 *>(so + (stream * ROWS + r) * OST + md * 16 + 4 * c4) =
                    o[md][nb];
        }
        __syncthreads();
    };
    auto store = [&](const Item &it, bool whole, int slot) {
        store_item<uint16_t, DH, ROWS, KS, THREADS>(a, it, whole, slot,
                                                    reinterpret_cast<const float *>(smem), ml);
        __syncthreads();
    };
    walk<SPARSE, ROWS, THREADS>(a, segment, store);
}

// ---------------------------------------------------------------------------
// fp32: four key streams of 16 rows, tiles of 16 keys straight from memory.
// The fp32 matrix instruction multiplies and adds in full fp32; lane (m16, c4)
// takes dims 16 j + 4 c4 + e of key m16 for its e-th step, the same for q.
template <int DH, bool SPARSE>
__global__ __launch_bounds__(256) void paged_attn_f32(PagedAttnParams a) {
    constexpr int KS = 4, THREADS = 256, ROWS = 16, MD = DH / 16, OST = DH + 4;
    __shared__ __attribute__((aligned(16))) float so[KS * ROWS * OST];
    __shared__ float ml[KS][ROWS][2];
    const int stream = wave_id();
    const int lane = threadIdx.x % kWave;
    const int m16 = lane & 15, c4 = lane >> 4;
    const float sl2 = a.sl2;

    auto segment = [&](const Item &it, int seq_i, int chunk0, int n) __attribute__((always_inline)) {
        const int list_end = SPARSE ? a.n_sel << a.v.page_shift : it.n_keys;
        const int k_begin = chunk0 * kChunk;
        const int k_end = min(k_begin + n * kChunk, list_end);
        Rows<1> rows;
        rows.set(a, it, 0);
        rows.load_mask(a, it, seq_i);
        const float *qp = static_cast<const float *>(a.q) +
                          ((size_t)(it.r0 + rows.i[0]) * a.n_q_heads + rows.h[0]) * DH;
        f32x4 qv[MD], o[MD];
#pragma unroll
        for (int j = 0; j < MD; ++j) {
            qv[j] = *reinterpret_cast<const f32x4 *>(qp + 16 * j + 4 * c4);
            o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        float mref = -INFINITY, lsum = 0.f;
        Pages<SPARSE, DH * 4> pages;
        pages.load(a, it, (k_begin + 16 * stream) >> a.v.page_shift);
        for (int k = k_begin + 16 * stream; k < k_end; k += 16 * KS) {
            if (k >> a.v.page_shift >= pages.base + kWave)
                pages.load(a, it, k >> a.v.page_shift);
            int pos, nk;
            size_t off;
            pages.find(a, it, k, pos, nk, off);
            if (nk == 0)
                continue;
            const size_t row = off / (DH * 4);
            const float *kp = static_cast<const float *>(a.k) + (row + min(m16, nk - 1)) * DH;
            f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < MD; ++j) {
                const f32x4 kv = *reinterpret_cast<const f32x4 *>(kp + 16 * j + 4 * c4);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    s = __builtin_amdgcn_mfma_f32_16x16x4f32(kv[e], qv[j][e], s, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = pos + 4 * c4 + i - it.ctx;
                const int me = seq_i + rows.i[0];
                const bool seen =
                    a.tree_mask ? ((rows.mask[0] >> (j & 63)) & 1ull) != 0 : j <= me;
                s[i] = (4 * c4 + i < nk) & ((j < 0) | seen) ? s[i] : -INFINITY;
            }
            float m = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
            m = fmaxf(m, __shfl_xor(m, 16, kWave));
            m = fmaxf(m, __shfl_xor(m, 32, kWave));
            if (m > mref) {                          // per row: uniform over its lanes
                const float alpha = fast_exp2((mref - m) * sl2);
                mref = m;
                lsum *= alpha;
#pragma unroll
                for (int md = 0; md < MD; ++md)
                    o[md] *= alpha;
            }
            const float mu = mref == -INFINITY ? 0.f : mref;
            float p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[i] = fast_exp2((s[i] - mu) * sl2);
                lsum += p[i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float *vp = static_cast<const float *>(a.vc) +
                                  (row + min(4 * c4 + i, nk - 1)) * DH + m16;
#pragma unroll
                for (int md = 0; md < MD; ++md)
                    o[md] = __builtin_amdgcn_mfma_f32_16x16x4f32(vp[md * 16], p[i], o[md], 0, 0, 0);
            }
        }
        lsum += __shfl_xor(lsum, 16, kWave);
        lsum += __shfl_xor(lsum, 32, kWave);
        if (c4 == 0) {
            ml[stream][m16][0] = mref;
            ml[stream][m16][1] = lsum;
        }
#pragma unroll
        for (int md = 0; md < MD; ++md)
            *reinterpret_cast<f32x4 *>(so + (stream * ROWS + m16) * OST + md * 16 + 4 * c4) = o[md];
        __syncthreads();
    };
    auto store = [&](const Item &it, bool whole, int slot) {
        store_item<float, DH, ROWS, KS, THREADS>(a, it, whole, slot, so, ml);
        __syncthreads();
    };
    walk<SPARSE, ROWS, THREADS>(a, segment, store);
}

// ---------------------------------------------------------------------------
// Joins the partials of the split item that begins in workgroup blockIdx.x, in
// run order: 16 lanes to a row, a sixteenth of its dims each, 16 rows to a
// workgroup.  Bound by the latency of its three trips to memory: 2.5 us for the parts
// of one request's heads, 12 for 32 MB of draft trees' partials (with one part's
// row in flight instead of eight 12 us for 32 parts, longer than the
// attention; with a wave to a row, four times the workgroups, 10 us for 128
// items of 64 rows; sixteen rows in flight gain nothing).
template <typename T, int DH, int ROWS>
__global__ __launch_bounds__(256) void paged_attn_join(PagedAttnParams a) {
    const int w0 = blockIdx.x;
    const int32_t *m = a.meta + w0 * kMetaInts;
    const int w1 = m[0];
    if (w1 < 0)
        return;
    const int row = blockIdx.y * 16 + threadIdx.x / 16;
    const int q = m[4] + row;
    if (q >= m[5])
        return;
    const int sub = threadIdx.x % 16, lane0 = threadIdx.x % kWave & ~15;
    constexpr int E = DH / 16;
    const int parts = w1 - w0 + 1;
    auto slot = [&](int p) { return (size_t)(p == 0 ? 2 * w0 + 1 : 2 * (w0 + p)); };
    auto over16 = [&](float x, auto op) {
#pragma unroll
        for (int off = 1; off < 16; off <<= 1)
            x = op(x, __shfl_xor(x, off, kWave));
        return x;
    };
    // eight parts' rows at a time (past the last part: the last again, with
    // factor 0), the first eight before their factors are known
    f32x4 x[8][E / 4];
    auto fetch = [&](int p0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float *src = a.part_o + (slot(min(p0 + i, parts - 1)) * ROWS + row) * DH + sub * E;
#pragma unroll
            for (int e = 0; e < E / 4; ++e)
                x[i][e] = *reinterpret_cast<const f32x4 *>(src + 4 * e);
        }
    };
    fetch(0);
    float mm = -INFINITY;
    for (int p = sub; p < parts; p += 16)
        mm = fmaxf(mm, a.part_ml[(slot(p) * ROWS + row) * 2]);
    mm = over16(mm, [](float x, float y) { return fmaxf(x, y); });
    const float muse = mm == -INFINITY ? 0.f : mm;
    float l = 0.f, o[E];
#pragma unroll
    for (int e = 0; e < E; ++e)
        o[e] = 0.f;
    for (int p0 = 0; p0 < parts; p0 += 16) {
        float f = 0.f, lp = 0.f;
        if (p0 + sub < parts) {
            const float *src = a.part_ml + (slot(p0 + sub) * ROWS + row) * 2;
            f = fast_exp2((src[0] - muse) * a.sl2);
            lp = src[1] * f;
        }
        l += over16(lp, [](float x, float y) { return x + y; });
        for (int p = 0; p < min(parts - p0, 16); p += 8) {
            if (p0 + p)
                fetch(p0 + p);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float fp = __shfl(f, lane0 + p + i, kWave);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    o[e] = p0 + p + i < parts ? fmaf(x[i][e / 4][e % 4], fp, o[e]) : o[e];
            }
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int e = 0; e < E; ++e)
        o[e] *= inv;
    T *dst = static_cast<T *>(a.out) +
             ((size_t)(m[1] + q / m[3]) * a.n_q_heads + m[2] + q % m[3]) * DH + sub * E;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < E; e += 4)
            *reinterpret_cast<f32x4 *>(dst + e) = f32x4{o[e], o[e + 1], o[e + 2], o[e + 3]};
    } else {
#pragma unroll
        for (int e = 0; e < E; e += 4)
            *reinterpret_cast<u32x2 *>(dst + e) =
                u32x2{pack_bf16x2(o[e], o[e + 1]), pack_bf16x2(o[e + 2], o[e + 3])};
    }
}

template <typename T, int DH, int ROWS>
void join(const PagedAttnParams &a, int workgroups, hipStream_t stream) {
    hipLaunchKernelGGL((paged_attn_join<T, DH, ROWS>), dim3(workgroups, ROWS / 16), dim3(256), 0,
                       stream, a);
}

template <int DH, int NB, int RG, int KS, int NBUF, bool SPARSE>
void launch_bf16(const PagedAttnParams &a, int workgroups, hipStream_t stream) {
    hipLaunchKernelGGL((paged_attn_bf16<DH, NB, RG, KS, NBUF, SPARSE>), dim3(workgroups),
                       dim3(64 * KS * RG), 0, stream, a);
    join<uint16_t, DH, 16 * NB * RG>(a, workgroups, stream);
}

template <int DH>
wf_status_t launch(wf_dtype_t dt, const PagedAttnParams &a, const PagedPlan &p,
                   hipStream_t stream) {
    const int W = p.workgroups;
    if (dt == WF_F32) {
        if (a.sel)
            hipLaunchKernelGGL((paged_attn_f32<DH, true>), dim3(W), dim3(256), 0, stream, a);
        else
            hipLaunchKernelGGL((paged_attn_f32<DH, false>), dim3(W), dim3(256), 0, stream, a);
        join<float, DH, 16>(a, W, stream);
    } else if (a.sel) {
        launch_bf16<DH, 1, 1, 4, 2, true>(a, W, stream);
    } else if (p.rg == 1) {
        launch_bf16<DH, 1, 1, 4, 2, false>(a, W, stream);
    } else if (p.rg == 2) {
        launch_bf16<DH, 1, 2, 2, 2, false>(a, W, stream);
    } else if (p.nb == 1) {
        launch_bf16<DH, 1, 4, 1, 3, false>(a, W, stream);
    } else {
        launch_bf16<DH, 2, 4, 1, 3, false>(a, W, stream);
    }
    return hipGetLastError() == hipSuccess ? WF_OK : WF_ERR_HIP;
}

size_t meta_bytes(const PagedPlan &p) {
    return ((size_t)p.workgroups * kMetaInts * sizeof(int32_t) + 255) & ~(size_t)255;
}
size_t ml_bytes(const PagedPlan &p) {
    return (size_t)2 * p.workgroups * p.rows() * 2 * sizeof(float);
}

}  // namespace

// Rows that share each key's bytes: the query heads of a group and, dense, the
// sequence's rows.  Up to 16 rows and fp32: four key streams, four waves with
// rings of their own, one workgroup a CU (two streams and two workgroups a CU:
// one request of 1K 9.98 us instead of 9.5, selected pages 12.7 instead of 12.3,
// 128 requests of up to 16K the same).  More rows: a tile serves all waves, so two
// workgroups a CU hide each other's barriers (one: draft trees of 4 requests 54.6
// us instead of 47.8), and 768 workgroups write more partials than they balance
// (blocks of 16 of 16 requests 47 us instead of 43.5).  Items of 256 rows, which
// read keys half as often, leave too little work in flight (trees 53 us instead
// of 45).
PagedPlan plan_paged(wf_dtype_t dt, int max_rows, int n_q_heads, int n_kv_heads, bool sparse) {
    const int rows = n_q_heads / n_kv_heads * (sparse ? 1 : max_rows);
    if (dt == WF_F32 || sparse || rows <= 16)
        return PagedPlan{1, 1, 4, kWorkgroups};
    if (rows <= 32)
        return PagedPlan{1, 2, 2, 2 * kWorkgroups};
    return PagedPlan{rows <= 64 ? 1 : 2, 4, 1, 2 * kWorkgroups};
}

size_t paged_attn_workspace_bytes(const PagedPlan &p, int head_dim) {
    return kCounterBytes + meta_bytes(p) + ml_bytes(p) +
           (size_t)2 * p.workgroups * p.rows() * head_dim * sizeof(float);
}

wf_status_t launch_paged_attn(wf_dtype_t dt, const void *q, const wf_paged_cache_t &c,
                              const wf_paged_batch_t &b, const int32_t *sel, int n_sel, void *out,
                              const uint64_t *tree_mask, int n_rows, int n_q_heads,
                              float softmax_scale, const PagedPlan &p, void *workspace,
                              hipStream_t stream) {
    PagedAttnParams a{};
    a.v = paged_view(c, b, n_rows);
    a.q = q;
    a.k = c.k;
    a.vc = c.v;
    a.out = out;
    a.sel = sel;
    a.tree_mask = tree_mask;
    a.n_sel = n_sel;
    a.group = n_q_heads / c.n_kv_heads;
    a.n_q_heads = n_q_heads;
    a.sl2 = softmax_scale * kLog2e;
    char *ws = static_cast<char *>(workspace);
    a.zeros = ws + kCounterBytes - kPagedZeroBytes;
    a.meta = reinterpret_cast<int32_t *>(ws + kCounterBytes);
    a.part_ml = reinterpret_cast<float *>(ws + kCounterBytes + meta_bytes(p));
    a.part_o = reinterpret_cast<float *>(ws + kCounterBytes + meta_bytes(p) + ml_bytes(p));
    return c.head_dim == 128 ? launch<128>(dt, a, p, stream) : launch<64>(dt, a, p, stream);
}

}  // namespace wf
