// logprob.hip -- log probabilities of given tokens, their rank, the entropy and
// the best alternatives, from rows of logits read once.
//
// A row is cut into `parts`, one workgroup each, and a part into one run per
// wave.  A wave reads its run front to back in 16-byte pieces; each lane keeps
// the running maximum m of its values, l = sum e^(z-m) and t = sum e^(z-m)(z-m),
// so that
//   log p(z) = z - m - log l,   entropy = log l - t / l,
// and the wave keeps the run's n best values in LDS: a value enters the list if
// it beats the n-th best of those before it (the first ones always do), and a
// full list is cut down to its n best.  Lists hold 64-bit keys, the value's
// order in the high half and the index's complement in the low one, so that the
// order of equal values is that of their indexes and no result hangs on which
// lane came first.  The waves' states and lists meet in LDS, the parts' in
// memory, where the row's last workgroup joins them in part order.
#include <type_traits>

#include "wf_api_internal.h"
#include "wf_device.h"

namespace wf {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kCap = 512;                  // keys a wave's list holds
constexpr int kMaxParts = 64;

struct LogprobParams {
    const void *logits;
    size_t stride;
    const int32_t *tokens;
    float *logprob, *entropy;
    int32_t *rank, *top_ids;
    float *top_lp;
    int vocab, n_top, parts, part_len;     // part_len: elements, a multiple of kThreads * 8
    unsigned *arrived;                     // [n_rows], in the zero block
    float *part_state;                     // [rows][parts][4]: m, l, t, rank
    uint64_t *part_keys;                   // [rows][parts][n_top]
};

// The order of fp32 values as unsigned integers: NaN above +inf, -0 as 0.
__device__ __forceinline__ uint32_t value_order(float x) {
    if (x != x)
        return ~0u;
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u >> 31) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float order_value(uint32_t o) {
    return __uint_as_float((o >> 31) ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint64_t make_key(float x, int idx) {
    return ((uint64_t)value_order(x) << 32) | (uint32_t)~(uint32_t)idx;
}

// Orders a wave's LDS stores before its lanes' later loads of them.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

template <int N>
__device__ __forceinline__ bool has_nan(const float (&x)[N]) {
    bool any = false;
#pragma unroll
    for (int e = 0; e < N; ++e)
        any |= x[e] != x[e];
    return any;
}

// Running state of a set of logits.
struct SumState {
    float m, l, t;
};
__device__ __forceinline__ SumState join(SumState x, SumState y) {
    const float m = fmaxf(x.m, y.m);
    const float dx = x.m - m, dy = y.m - m;
    // (an empty side: l = t = 0 and m = -inf, which must not become NaN)
    const float ex = x.m == -INFINITY ? 0.f : expf(dx), ey = y.m == -INFINITY ? 0.f : expf(dy);
    const float fx = x.m == -INFINITY ? 0.f : dx, fy = y.m == -INFINITY ? 0.f : dy;
    SumState r;
    r.m = m;
    r.l = x.l * ex + y.l * ey;
    r.t = (x.t + x.l * fx) * ex + (y.t + y.l * fy) * ey;
    return r;
}

// Cuts a list of n keys (n <= kCap, all different) down to its `top` best, in
// no particular order; returns the least of them.  Called by one wave.
__device__ __forceinline__ uint64_t keep_best(uint64_t *list, int n, int top) {
    const int lane = threadIdx.x % kWave;
    uint64_t k[kCap / kWave];
#pragma unroll
    for (int j = 0; j < kCap / kWave; ++j)
        k[j] = j * kWave + lane < n ? list[j * kWave + lane] : 0ull;
    // the largest number that at least `top` keys reach, bit by bit from the
    // top; it is found early where exactly `top` keys reach it
    uint64_t least = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const uint64_t cand = least | (1ull << bit);
        int count = 0;
#pragma unroll
        for (int j = 0; j < kCap / kWave; ++j)
            count += __popcll(__ballot(k[j] >= cand));
        if (count >= top) {
            least = cand;
            if (count == top)
                break;
        }
    }
    const uint64_t below = (1ull << lane) - 1ull;
    int at = 0;
    uint64_t min_kept = ~0ull;
    wave_sync();
#pragma unroll
    for (int j = 0; j < kCap / kWave; ++j) {
        const bool take = k[j] >= least && k[j] != 0;
        const uint64_t mask = __ballot(take);
        if (take) {
            list[at + __popcll(mask & below)] = k[j];
            min_kept = min(min_kept, k[j]);
        }
        at += __popcll(mask);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
        min_kept = min(min_kept, (uint64_t)__shfl_xor((unsigned long long)min_kept, off, kWave));
    wave_sync();
    return min_kept;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void token_logprobs(LogprobParams a) {
    constexpr int V = 16 / sizeof(T);
    __shared__ uint64_t lists[kWaves][kCap];
    __shared__ SumState states[kWaves];
    __shared__ int ranks[kWaves], counts[kWaves];
    const int row = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const int wave = wave_id(), lane = threadIdx.x % kWave;
    const T *z = static_cast<const T *>(a.logits) + (size_t)row * a.stride;
    auto at = [&](int i) -> float {
        if constexpr (sizeof(T) == 2)
            return bf16_to_f32(z[i]);
        else
            return z[i];
    };
    const int token = a.tokens ? a.tokens[row] : -1;
    const bool has_token = token >= 0 && token < a.vocab;
    const float zt = has_token ? at(token) : INFINITY;
    const bool zt_nan = zt != zt;

    // ---- this wave's run ----
    // Elements before `head` and behind the last whole piece are taken one by
    // one, so that a row may begin at any element.
    const int run = a.part_len / kWaves;
    const int i0 = min(part * a.part_len + wave * run, a.vocab);
    const int i1 = min(i0 + run, a.vocab);
    uint64_t *list = lists[wave];
    int n_list = 0;                        // uniform
    float enter = -INFINITY;               // a value enters if it is larger, or while
    bool filled = false;                   // the list has not held n_top yet
    float m = -INFINITY, l = 0.f, t = 0.f;
    int ahead = 0;
    // V values of every lane, a lane's from index base on, the wave's from
    // `tile` on; full: all of them are there, else the lane's first `valid`.
    auto take = [&](const float (&x)[V], int tile, int base, int valid, auto full_tag)
        __attribute__((always_inline)) {
        constexpr bool FULL = decltype(full_tag)::value;
        auto there = [&](int e) { return FULL || e < valid; };
        float mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < V; ++e)
            mx = there(e) ? fmaxf(mx, x[e]) : mx;
        if (mx > m) {
            const float f = m == -INFINITY ? 0.f : m - mx;
            const float s = m == -INFINITY ? 0.f : fast_exp2(f * kLog2e);
            t = (t + l * f) * s;
            l *= s;
            m = mx;
        }
        const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float d = there(e) ? x[e] - mu : -INFINITY;
            const float w = fast_exp2(d * kLog2e);
            l += w;
            t = fmaf(w, fmaxf(d, -1e30f), t);        // (0 * -inf would be NaN)
        }
        // ---- the token's rank: whole tiles lie before it or behind it ----
        if (FULL && !zt_nan && tile + kWave * V <= token) {
#pragma unroll
            for (int e = 0; e < V; ++e)
                ahead += !(x[e] < zt) ? 1 : 0;
        } else if (FULL && !zt_nan && tile > token) {
#pragma unroll
            for (int e = 0; e < V; ++e)
                ahead += !(x[e] <= zt) ? 1 : 0;
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const bool before = base + e < token;
                const bool a_nan = x[e] != x[e];
                const bool first = zt_nan ? a_nan && before
                                          : a_nan || x[e] > zt || (x[e] == zt && before);
                ahead += there(e) && first ? 1 : 0;
            }
        }
        if (a.n_top == 0)
            return;
        // ---- the list: what beats the n-th best of the tiles before (values
        // equal to it have higher indexes here), or, until a list was full, all
        if (filled && !__ballot(!(mx <= enter)) && !__ballot(has_nan(x)))
            return;
        bool in[V];
#pragma unroll
        for (int e = 0; e < V; ++e)
            in[e] = there(e) && (!filled || !(x[e] <= enter));
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const uint64_t mask = __ballot(in[e]);
            if (!mask)
                continue;
            const int more = __popcll(mask);
            if (n_list + more > kCap) {
                const uint64_t least = keep_best(list, n_list, a.n_top);
                n_list = a.n_top;
                filled = true;
                enter = order_value((uint32_t)(least >> 32));
            }
            if (in[e])
                list[n_list + __popcll(mask & ((1ull << lane) - 1ull))] = make_key(x[e], base + e);
            n_list += more;
        }
        wave_sync();
    };
    auto unpack = [&](u32x4 w, float (&x)[V]) {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[2 * e] = __uint_as_float(w[e] << 16);
                x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[e] = __uint_as_float(w[e]);
        }
    };
    auto singles = [&](int from, int to) {           // fewer than V elements
        if (from < to) {
            float x[V] = {};
            const int i = from + lane;
            if (i < to)
                x[0] = at(i);
            take(x, from, i, i < to ? 1 : 0, std::false_type{});
        }
    };
    const int head =
        min(i1, i0 + (int)(((16 - (reinterpret_cast<uintptr_t>(z + i0) & 15)) & 15) / sizeof(T)));
    const int body = head + (i1 - head) / V * V;
    constexpr int TILE = kWave * V, U = 4;
    singles(i0, head);
    int base = head;
    for (; base + U * TILE <= body; base += U * TILE) {
        u32x4 w[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            w[u] = *reinterpret_cast<const u32x4 *>(z + base + u * TILE + lane * V);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float x[V];
            unpack(w[u], x);
            take(x, base + u * TILE, base + u * TILE + lane * V, V, std::true_type{});
        }
    }
    for (; base < body; base += TILE) {
        const int i = base + lane * V;
        u32x4 w = {0u, 0u, 0u, 0u};
        if (i < body)
            w = *reinterpret_cast<const u32x4 *>(z + i);
        float x[V];
        unpack(w, x);
        take(x, base, i, i < body ? V : 0, std::false_type{});
    }
    singles(body, i1);

    // ---- the waves meet ----
    SumState s{m, l, t};
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        SumState o{__shfl_xor(s.m, off, kWave), __shfl_xor(s.l, off, kWave),
                   __shfl_xor(s.t, off, kWave)};
        // the lower lane first, so that both sides add alike
        s = (lane & off) ? join(o, s) : join(s, o);
        ahead += __shfl_xor(ahead, off, kWave);
    }
    if (n_list > a.n_top) {
        keep_best(list, n_list, a.n_top);
        n_list = a.n_top;
    }
    if (lane == 0) {
        states[wave] = s;
        ranks[wave] = ahead;
        counts[wave] = n_list;
    }
    __syncthreads();
    // Joins the keys of `sets` sets (set i: n(i) keys, key(i, j)) into the first
    // list, cut to n_top; called by wave 0.
    int held = 0;
    auto add = [&](uint64_t k, bool in) {
        const uint64_t mask = __ballot(in);
        const int more = __popcll(mask);
        if (held + more > kCap) {
            keep_best(lists[0], held, a.n_top);
            held = a.n_top;
        }
        if (in)
            lists[0][held + __popcll(mask & ((1ull << lane) - 1ull))] = k;
        held += more;
        wave_sync();
    };
    int all_ahead = 0;
    if (wave == 0) {
        held = counts[0];
        s = states[0];
        all_ahead = ranks[0];
        for (int w = 1; w < kWaves; ++w) {
            s = join(s, states[w]);
            all_ahead += ranks[w];
            add(lane < counts[w] ? lists[w][lane] : 0ull, lane < counts[w]);
        }
        if (held > a.n_top) {
            keep_best(lists[0], held, a.n_top);
            held = a.n_top;
        }
    }
    if (a.parts > 1) {
        const size_t slot = (size_t)row * a.parts + part;
        if (wave == 0) {
            if (lane == 0) {
                float *ps = a.part_state + slot * 4;
                ps[0] = s.m;
                ps[1] = s.l;
                ps[2] = s.t;
                ps[3] = __int_as_float(all_ahead);
            }
            if (lane < a.n_top)
                a.part_keys[slot * a.n_top + lane] = lane < held ? lists[0][lane] : 0ull;
        }
        if (!arrive_last(a.arrived + row, a.parts))
            return;
        if (threadIdx.x == 0)
            a.arrived[row] = 0;
        if (wave != 0)
            return;
        held = 0;
        all_ahead = 0;
        s = SumState{-INFINITY, 0.f, 0.f};
        for (int p = 0; p < a.parts; ++p) {
            const size_t from = (size_t)row * a.parts + p;
            const float *ps = a.part_state + from * 4;
            s = join(s, SumState{ps[0], ps[1], ps[2]});
            all_ahead += __float_as_int(ps[3]);
            const uint64_t k = lane < a.n_top ? a.part_keys[from * a.n_top + lane] : 0ull;
            add(k, k != 0ull);
        }
        if (held > a.n_top)
            keep_best(lists[0], held, a.n_top);
    }
    if (wave != 0)
        return;
    // ---- results: one wave ----
    // (a row of nothing but -inf has l = 0; +inf or NaN leave NaN in l)
    const float logl = s.l > 0.f ? logf(s.l) : NAN;
    auto lp = [&](float x) { return (x - s.m) - logl; };
    if (lane == 0) {
        if (a.logprob)
            a.logprob[row] = has_token ? lp(zt) : 0.f;
        if (a.rank)
            a.rank[row] = has_token ? all_ahead : -1;
        if (a.entropy)
            a.entropy[row] = logl - s.t / s.l;
    }
    if (lane < a.n_top) {
        const uint64_t mine = lists[0][lane];
        int place = 0;
        for (int j = 0; j < a.n_top; ++j)
            place += lists[0][j] > mine ? 1 : 0;
        const uint32_t o = (uint32_t)(mine >> 32);
        const size_t dst = (size_t)row * a.n_top + place;
        a.top_ids[dst] = (int32_t)~(uint32_t)mine;
        a.top_lp[dst] = lp(o == ~0u ? NAN : order_value(o));
    }
}

struct LogprobPlan {
    int parts, part_len;
};

// Rows are cut where they are too few to fill the chip (about four workgroups a
// CU), down to two 16-byte pieces of each lane.
LogprobPlan plan_logprobs(wf_dtype_t dt, int n_rows, int vocab) {
    const int unit = kThreads * (dt == WF_F32 ? 4 : 8);
    const int most = std::max(1, std::min(kMaxParts, (vocab + 2 * unit - 1) / (2 * unit)));
    const int want = std::max(1, 1024 / std::max(n_rows, 1));
    const int parts = std::min(most, want);
    const int len = ((vocab + parts - 1) / parts + unit - 1) / unit * unit;
    return LogprobPlan{(vocab + len - 1) / len, len};
}

size_t state_bytes(int n_rows, const LogprobPlan &p) {
    return ((size_t)n_rows * p.parts * 16 + 255) & ~(size_t)255;
}

}  // namespace

size_t token_logprobs_workspace_bytes(wf_dtype_t dt, int n_rows, int vocab, int n_top) {
    const LogprobPlan p = plan_logprobs(dt, n_rows, vocab);
    return kCounterBytes +
           (p.parts > 1 ? state_bytes(n_rows, p) + (size_t)n_rows * p.parts * n_top * 8 : 0);
}

wf_status_t launch_token_logprobs(wf_dtype_t dt, const void *logits, size_t row_stride,
                                  const int32_t *tokens, int n_rows, int vocab, int n_top,
                                  float *logprob, float *entropy, int32_t *rank,
                                  int32_t *top_ids, float *top_lp, void *workspace,
                                  hipStream_t stream) {
    const LogprobPlan p = plan_logprobs(dt, n_rows, vocab);
    LogprobParams a{};
    a.logits = logits;
    a.stride = row_stride;
    a.tokens = tokens;
    a.logprob = logprob;
    a.entropy = entropy;
    a.rank = rank;
    a.top_ids = top_ids;
    a.top_lp = top_lp;
    a.vocab = vocab;
    a.n_top = n_top;
    a.parts = p.parts;
    a.part_len = p.part_len;
    char *ws = static_cast<char *>(workspace);
    a.arrived = reinterpret_cast<unsigned *>(ws);
    a.part_state = reinterpret_cast<float *>(ws + kCounterBytes);
    a.part_keys = reinterpret_cast<uint64_t *>(ws + kCounterBytes + state_bytes(n_rows, p));
    const dim3 grid(n_rows * p.parts), block(kThreads);
    if (dt == WF_BF16)
        hipLaunchKernelGGL(token_logprobs<uint16_t>, grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL(token_logprobs<float>, grid, block, 0, stream, a);
    return hipGetLastError() == hipSuccess ? WF_OK : WF_ERR_HIP;
}

}  // namespace wf
