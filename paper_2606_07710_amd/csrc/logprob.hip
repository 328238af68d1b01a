// logprob.hip -- log probabilities of given tokens, their rank, the entropy and
// the best alternatives, from rows of logits read once.
//
// A row is cut into `parts`, one workgroup each, and a part into one run per
// wave.  A wave reads its run front to back in 16-byte pieces; each lane keeps
// a reference m, which moves up to a value that is larger by more than 8 (so the
// weights stay below 2^12), l = sum e^(z-m) and t = sum e^(z-m)(z-m), so that
//   log p(z) = z - m - log l,   entropy = log l - t / l.
// The wave's best values lie sorted in its lanes, lane i the i-th, as 64-bit
// keys: the value's order in the high half, the index's complement in the low
// one, so that the order of equal values is that of their indexes and no result
// hangs on which lane came first.  The values of a group that beat the n-th best
// that any wave of the workgroup has, and reach what n of the lanes' maxima in
// the group reach, are gathered in LDS and enter together: all are compared with
// all.  The sorted lists of the waves, and then,
// in the row's last workgroup, of the parts, join by the same means: of P lists
// the (n / r)-th largest of their r-th keys, r = n / P, is reached by n keys, and
// what reaches it is few more than n.
//
// Short rows and few of them are bound by latency, in which the fetching of the
// code counts: loops that are not hot are kept rolled.  16 fp32 rows of 151936
// with 20 alternatives take 16 us (7 without: the rest are the lists, from a
// group's values to their two meetings); 2000 bf16 rows with 5 (608 MB) take 147
// us, 4.1 TB/s, bound by the vector unit (0.74 busy: 14 instructions a value, an
// exponential among them), 125 without.
#include <type_traits>

#include "wf_api_internal.h"
#include "wf_device.h"

namespace wf {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kMaxParts = 64;
constexpr int kLoads = 4;                  // 16-byte loads of a lane in a group
// Groups after which a lane's sums go into a second pair, so that rows of millions
// of values are no chain of as many roundings: kLoads * kFold pieces in one sum and,
// in the longest run there can be, 2^28 values in 2^18 groups, 2^10 such sums.
constexpr int kFold = 256;
// Up to so many values of a tile enter a full list one by one, a compare and
// seven moves each, more of them together (2000 bf16 rows with 5 alternatives: 157 ->
// 149 us in a graph; into an empty list one by one, 16 rows with 20 take 1.5 longer).
constexpr int kInserts = 8;
constexpr int kPartKeys = 1280;            // parts * n_top at most
// A row's arrival counter has a cache line to itself: counters side by side
// queue up at one place of the memory (16 rows without alternatives: 13.1 us in a
// graph, apart 7.6).
constexpr int kCounterStride = 32;
constexpr int kMaxSplitRows = 512;
static_assert(kMaxSplitRows * kCounterStride <= kCounterSlots, "the counters fit the zero block");

struct LogprobParams {
    const void *logits;
    size_t stride;
    const int32_t *tokens;
    float *logprob, *entropy;
    int32_t *rank, *top_ids;
    float *top_lp;
    int wave_r, wave_want, part_r, part_want;  // bounds of the lists that join
    int vocab, n_top, parts, part_len;     // part_len: elements, whole groups of the waves
    unsigned *arrived;                     // [n_rows][kCounterStride], in the zero block
    float *part_state;                     // [rows][parts][4]: m, l, t, rank
    uint64_t *part_keys;                   // [rows][parts][n_top], sorted
};

// The order of fp32 values as unsigned integers: NaN above +inf, -0 as 0.  No
// value has order 0.
__device__ __forceinline__ uint32_t value_order(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    const uint32_t o = (u >> 31) ? ~u : u | 0x80000000u;
    return x != x ? ~0u : o;
}
__device__ __forceinline__ float order_value(uint32_t o) {
    return __uint_as_float((o >> 31) ? o & 0x7fffffffu : ~o);
}

__device__ __forceinline__ uint64_t make_key(float x, int idx) {
    return ((uint64_t)value_order(x) << 32) | (uint32_t)~(uint32_t)idx;
}

// Over the lanes of a wave.
__device__ __forceinline__ float lanes_max(float x) {
    return __int_as_float(wave_reduce(__float_as_int(x), __float_as_int(-INFINITY), [](int a, int b) {
        return __float_as_int(fmaxf(__int_as_float(a), __int_as_float(b)));
    }));
}
__device__ __forceinline__ float lanes_sum(float x) {
    return __int_as_float(wave_reduce(__float_as_int(x), 0, [](int a, int b) {
        return __float_as_int(__int_as_float(a) + __int_as_float(b));
    }));
}

// Running state of a set of logits, and that of the lanes' sets together.
struct SumState {
    float m, l, t;
};
// From reference m to a larger one, as far as it matters: at -1e20 every weight
// is 0 already, and l, below 2^43, times it is finite, where the difference itself
// may be -inf or, from an empty set's, NaN (the lowest number as a mask).
__device__ __forceinline__ float shift(float m, float to) { return fmaxf(m - to, -1e20f); }
__device__ __forceinline__ SumState lanes_join(SumState x) {
    const float m = lanes_max(x.m);
    const float d = shift(x.m, m), e = fast_exp2(d * kLog2e);
    return SumState{m, lanes_sum(x.l * e), lanes_sum((x.t + x.l * d) * e)};
}
// The sums l and t from reference m into `all`, whose reference is no larger; they
// begin anew.
__device__ __forceinline__ void fold(SumState &all, float m, float &l, float &t) {
    const float d = shift(all.m, m), e = fast_exp2(d * kLog2e);
    all = SumState{m, fmaf(all.l, e, l), fmaf(all.t + all.l * d, e, t)};
    l = t = 0.f;
}

__device__ __forceinline__ uint64_t volatile_load(const uint64_t *p) {
    return *(const volatile uint64_t *)p;
}
__device__ __forceinline__ uint64_t uniform64(uint64_t v) {
    return ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(v >> 32)) << 32) |
           (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v);
}
__device__ __forceinline__ uint64_t readlane64(uint64_t v, int lane) {
    return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane) << 32) |
           (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}

// Number of the n keys at `list` (LDS; zeros behind them up to a multiple of
// 8) above each of x and y.  The reads are the same for all lanes.
__device__ __forceinline__ void count_above(const uint64_t *list, int n, uint64_t x, uint64_t y,
                                            int &nx, int &ny) {
#pragma unroll 1
    for (int j = 0; j < n; j += 8) {
        uint64_t k[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            k[i] = list[j + i];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            nx += k[i] > x ? 1 : 0;
            ny += k[i] > y ? 1 : 0;
        }
    }
}

// A wave's n best values: lane i < n holds the i-th key, 0 where there is none.
struct BestList {
    uint64_t best, bar;                    // bar: the n-th key (uniform)
    int n;

    __device__ __forceinline__ void clear() { best = bar = 0; }
    // Takes in one key (uniform), no key of the list.
    __device__ __forceinline__ void insert(uint64_t key) {
        const int lane = threadIdx.x % kWave, place = __popcll(__ballot(best > key));
        const uint64_t before =
            ((uint64_t)(uint32_t)dpp<kWaveShr1, 0xf>(0, (int)(uint32_t)(best >> 32)) << 32) |
            (uint32_t)dpp<kWaveShr1, 0xf>(0, (int)(uint32_t)best);
        best = lane >= n || lane < place ? best : lane == place ? key : before;
        bar = readlane64(best, n - 1);
    }
    // Takes in the m <= 64 keys at `from` (LDS, zeros behind them up to a
    // multiple of 8; all different).  scratch: 64 keys of LDS, the wave's own.
    __device__ __forceinline__ void take(const uint64_t *from, int m, uint64_t *scratch) {
        const int lane = threadIdx.x % kWave;
        const uint64_t key = lane < m ? from[lane] : 0ull;
        int old_place = lane, new_place = 0, none = 0;
        count_above(from, m, best, key, old_place, new_place);
        if (bar | readlane64(best, 0)) {             // (an empty list has none above)
            scratch[lane] = best;
            wave_sync();
            count_above(scratch, n, key, ~0ull, new_place, none);
            wave_sync();
        }
        if (lane < n && old_place < n)
            scratch[old_place] = best;
        if (key && new_place < n)
            scratch[new_place] = key;
        wave_sync();
        best = lane < n ? scratch[lane] : 0ull;
        bar = readlane64(best, n - 1);
        wave_sync();
    }
};

template <typename T>
__global__ __launch_bounds__(kThreads) void token_logprobs(LogprobParams a) {
    constexpr int V = 16 / sizeof(T);
    constexpr int TILE = kWave * V, U = kLoads;
    // what enters a wave's list, at most a tile's values at a time; later the
    // lists of the waves and of the parts
    constexpr int kGather = TILE;
    __shared__ __attribute__((aligned(16))) uint64_t keys[2 * kPartKeys + 8];
    static_assert(kWaves * (kGather + 8) <= 2 * kPartKeys, "the waves' values");
    uint64_t *joined = keys + kPartKeys;   // what is left of the lists
    __shared__ int n_joined;
    __shared__ uint64_t bars[kWaves];
    __shared__ __attribute__((aligned(16))) uint64_t places[kWaves][kWave];
    __shared__ SumState states[kWaves];
    __shared__ int ranks[kWaves];
    const int row = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const int wave = wave_id(), lane = threadIdx.x % kWave;
    const T *z = static_cast<const T *>(a.logits) + (size_t)row * a.stride;
    auto value = [&](T raw) -> float {
        if constexpr (sizeof(T) == 2)
            return bf16_to_f32(raw);
        else
            return raw;
    };
    const int token = a.tokens ? a.tokens[row] : -1;
    const bool has_token = token >= 0 && token < a.vocab;
    const float zt = has_token ? value(z[token]) : INFINITY;
    // What comes before the token: behind it, the values above its own; before
    // it also the equal ones, which are those above the next lower number (all,
    // where its logit is -inf: !(x <= NaN)).  NaN counts as above.
    float zt_below;
    {
        const uint32_t u = __float_as_uint(zt + 0.f);
        zt_below = __uint_as_float(u == 0 ? 0x80000001u : (u >> 31) ? u + 1 : u - 1);
    }

    // ---- this wave's run ----
    const int run = a.part_len / kWaves;
    const int i0 = min(part * a.part_len + wave * run, a.vocab);
    const int i1 = min(i0 + run, a.vocab);
    BestList list;
    list.n = a.n_top;
    list.clear();
    uint64_t *buf = keys + wave * (kGather + 8);
    uint64_t *scratch = places[wave];
    if (threadIdx.x < kWaves)
        bars[threadIdx.x] = 0;
    __syncthreads();
    uint64_t bar = 0;                      // the highest of the waves' (uniform)
    float m = -INFINITY, l = 0.f, t = 0.f;
    SumState all{-INFINITY, 0.f, 0.f};     // of the groups before the last kFold
    int ahead = 0;                         // uniform

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
    // The sums over V values of every lane; the largest, or, where NaN or +inf is
    // among them, NaN.
    auto add = [&](const float (&x)[V]) __attribute__((always_inline)) -> float {
        float mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < V; ++e)
            mx = fmaxf(mx, x[e]);
        if (mx > m + 8.f) {
            const float f = shift(m, mx), s = fast_exp2(f * kLog2e);
            t = (t + l * f) * s;
            l *= s;
            m = mx;
        }
        const float mu = m == -INFINITY ? 0.f : m;
        // (sums of a piece first: the chains are V times shorter)
        float pl = 0.f, pt = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            // (0 * -inf would be NaN; a NaN stays one)
            const float d = __builtin_elementwise_maximum(x[e] - mu, -1e30f);
            const float p = fast_exp2(d * kLog2e);
            pl += p;
            pt = fmaf(p, d, pt);
        }
        l += pl;
        t += pt;
        return fmaf(pl, 0.f, mx);
    };
    // Elements before the first 16-byte boundary and behind the last whole piece
    // go one to a lane, whole groups of U tiles with their loads ahead, what is
    // left (and the group that has the token) tile by tile.
    const int head =
        min(i1, i0 + (int)(((16 - (reinterpret_cast<uintptr_t>(z + i0) & 15)) & 15) / sizeof(T)));
    const int body = head + (i1 - head) / V * V;
    // A piece of V lies before the token or not; the values before it in its own
    // piece are counted here where they equal it.
    if (token >= head && token < body) {
        const int i = token - (token - head) % V + lane;
        ahead = __popcll(__ballot(i < token && value(z[min(i, token)]) == zt));
    }
    if (zt != zt) {
        // a NaN's rank: the number of those before it
        for (int i = i0 + lane; i - lane < min(i1, token); i += kWave) {
            const float x = value(z[min(i, token)]);
            ahead += __popcll(__ballot(i < token && i < i1 && x != x));
        }
    }
    int next_fold = i0 + kFold * U * TILE;
#pragma unroll 1
    for (int pos = i0; pos < i1;) {
        if (pos >= next_fold) {
            fold(all, m, l, t);
            next_fold = pos + kFold * U * TILE;
        }
        const bool single = pos < head || pos >= body;
        const int group = pos + U * TILE;
        const bool whole = !single && group <= body;
        const int next = whole ? group : pos < head ? head : single ? i1 : min(body, pos + TILE);
        // a lane's elements in tile u: from index base + u * TILE on, n of them
        const int base = pos + (single ? lane : lane * V);
        const int n = base >= next ? 0 : single ? 1 : V;
        u32x4 w[U];
        float tops[U], top = -INFINITY;
#pragma unroll
        for (int u = 0; u < U; ++u)
            tops[u] = -INFINITY;
        if (whole) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                w[u] = *reinterpret_cast<const u32x4 *>(z + pos + u * TILE + lane * V);
        } else {
            w[0] = u32x4{0u, 0u, 0u, 0u};
            if (n == V) {
                w[0] = *reinterpret_cast<const u32x4 *>(z + base);
            } else if (n == 1) {
                if constexpr (sizeof(T) == 2)
                    w[0][0] = z[base];
                else
                    w[0][0] = __float_as_uint(z[base]);
            }
        }
        auto tile = [&](int u, auto full_tag) __attribute__((always_inline)) {
            constexpr bool FULL = decltype(full_tag)::value;
            float x[V];
            unpack(w[u], x);
#pragma unroll
            for (int e = 0; e < V; ++e)
                x[e] = FULL || e < n ? x[e] : -INFINITY;
            tops[u] = add(x);
            top = __builtin_elementwise_maximum(top, tops[u]);
            const bool before = base + u * TILE + (FULL ? V : n) <= token;
            const float above = before ? zt_below : zt;
            if (__ballot(!(tops[u] <= above)) && zt == zt)
#pragma unroll
                for (int e = 0; e < V; ++e)
                    ahead += __popcll(__ballot((FULL || e < n) && !(x[e] <= above)));
        };
        if (whole) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                tile(u, std::true_type{});
        } else {
            tile(0, std::false_type{});
        }
        // ---- the list (a value equal to its n-th best is behind it) ----
        const uint32_t top_order = n > 0 ? value_order(top) : 0u;
        if (a.n_top && __ballot(top_order >= max((uint32_t)(bar >> 32), 1u))) {
            // (the waves' bars rise; which one is seen changes no result)
            const uint64_t b = max(max(volatile_load(bars), volatile_load(bars + 1)),
                                   max(volatile_load(bars + 2), volatile_load(bars + 3)));
            bar = uniform64(b);
            uint32_t need = max((uint32_t)(bar >> 32), 1u);
            // A number that n values reach and few more.  (A lane whose maximum is NaN
            // may hold less: it counts as 0.)
            if (a.n_top <= kWave / 2) {
                // the n-th largest of the lanes' maxima: the least of those that
                // fewer than n are above
                const uint32_t o = top == top ? top_order : 0u;
                if (__popcll(__ballot(o > need)) >= a.n_top) {
                    uint32_t *tops_lds = reinterpret_cast<uint32_t *>(scratch);
                    tops_lds[lane] = o;
                    wave_sync();
                    int above = 0;
#pragma unroll 1
                    for (int j = 0; j < kWave; j += 16) {
                        uint32_t k[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            k[i] = tops_lds[j + i];
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            above += k[i] > o ? 1 : 0;
                    }
                    wave_sync();
                    const int reach = wave_reduce(
                        above < a.n_top ? (int)o : -1, -1,
                        [](int x, int y) { return (int)min((uint32_t)x, (uint32_t)y); });
                    need = max(need, (uint32_t)reach);
                }
            } else {
                // by halving, one that n of the lanes' maxima in the tiles reach and
                // at most a quarter more: the least of 64 lanes' maxima is reached by
                // a quarter of all values (16 rows of 151936 with 64 alternatives: 41
                // -> 31 us; with 20 the same, with 5 half a us more than the above)
                uint32_t o[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    o[u] = n > 0 && (u == 0 || whole) && tops[u] == tops[u] ? value_order(tops[u])
                                                                            : 0u;
                auto reach = [&](uint32_t x) {
                    int c = 0;
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        c += __popcll(__ballot(o[u] >= x));
                    return c;
                };
                if (reach(need + 1u) >= a.n_top) {
                    uint32_t most = o[0];
#pragma unroll
                    for (int u = 1; u < U; ++u)
                        most = max(most, o[u]);
                    // (every lane reaches the least of the lanes', 64 of them)
                    const uint32_t least = (uint32_t)wave_reduce((int)most, -1, [](int x, int y) {
                        return (int)min((uint32_t)x, (uint32_t)y);
                    });
                    uint32_t past = 1u + (uint32_t)wave_reduce((int)most, 0, [](int x, int y) {
                        return (int)max((uint32_t)x, (uint32_t)y);
                    });
                    need = max(need, least);
#pragma unroll 1
                    while (past - need > 1u) {
                        const uint32_t mid = need + (past - need) / 2u;
                        const int c = reach(mid);
                        if (c < a.n_top) {
                            past = mid;
                            continue;
                        }
                        need = mid;
                        if (c <= a.n_top + a.n_top / 4)
                            break;
                    }
                }
            }
            const float need_value = need > 1u ? order_value(need) : -INFINITY;
            int held = 0;
            const int tiles = whole ? U : 1;
#pragma unroll 1
            for (int u = 0; u <= tiles; ++u) {
                uint64_t in[V];
                float x[V];
                int more = 0;
                if (u < tiles) {
                    u32x4 wu = w[0];
                    float tu = tops[0];
#pragma unroll
                    for (int i = 1; i < U; ++i) {
                        wu = u == i ? w[i] : wu;
                        tu = u == i ? tops[i] : tu;
                    }
                    uint64_t lanes = __ballot(n > 0 && value_order(tu) >= need);
                    if (!lanes)
                        continue;
                    unpack(wu, x);
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        in[e] = __ballot(e < n && !(x[e] < need_value));
                        more += __popcll(in[e]);
                    }
                    // a few for a list that is full, each the largest of its lane's
                    if (list.bar && more <= kInserts && more == __popcll(lanes) && !__ballot(tu != tu)) {
                        int at = 0;                  // (behind the n-th lie no values)
#pragma unroll
                        for (int e = 1; e < V; ++e)
                            at = e < n && x[e] == tu ? e : at;
                        at += base + u * TILE;
#pragma unroll 1
                        for (; lanes; lanes &= lanes - 1) {
                            const int from = __builtin_ctzll(lanes);
                            list.insert(make_key(
                                __int_as_float(__builtin_amdgcn_readlane(__float_as_int(tu), from)),
                                __builtin_amdgcn_readlane(at, from)));
                        }
                        continue;
                    }
                }
                if (u == tiles || held + more > kGather) {
                    if (lane < 8)
                        buf[held + lane] = 0;
                    wave_sync();
#pragma unroll 1
                    for (int i = 0; i < held; i += kWave)
                        list.take(buf + i, min(held - i, kWave), scratch);
                    held = 0;
                }
                if (more) {
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        if (!in[e])
                            continue;
                        if ((in[e] >> lane) & 1ull)
                            buf[held + __popcll(in[e] & ((1ull << lane) - 1ull))] =
                                make_key(x[e], base + u * TILE + e);
                        held += __popcll(in[e]);
                    }
                }
            }
            if (lane == 0)
                *(volatile uint64_t *)(bars + wave) = list.bar;
            bar = max(bar, list.bar);
        }
        pos = next;
    }

    // ---- the waves meet, then, by the row's last workgroup, the parts ----
    const size_t first = (size_t)row * a.parts;
    fold(all, m, l, t);
    SumState s = all;
    bool last_round = a.parts == 1;
    int lists = 0;
#pragma unroll 1
    for (;;) {
        s = lanes_join(s);
        if (lane == 0) {
            states[wave] = s;
            ranks[wave] = ahead;
        }
        __syncthreads();                   // (the waves' buffers lie in `keys`)
        if (a.parts == 1 || !last_round) {
            if (lane < a.n_top)
                keys[wave * a.n_top + lane] = list.best;
            lists = kWaves;
        }
        if (threadIdx.x == 0)
            n_joined = 0;
        __syncthreads();
        if (a.n_top) {
            const int r = lists == kWaves ? a.wave_r : a.part_r;
            const int want = lists == kWaves ? a.wave_want : a.part_want;
            const uint64_t rth = lane < lists ? keys[lane * a.n_top + r - 1] : 0ull;
            int above = 0;
#pragma unroll 4
            for (int p = 0; p < lists; ++p)
                above += keys[p * a.n_top + r - 1] > rth ? 1 : 0;
            // (keys of no value, 0, may be equal: then there is no bound)
            const uint64_t at = __ballot(lane < lists && above == want - 1);
            const uint64_t least = at ? readlane64(rth, __builtin_ctzll(at)) : 0ull;
#pragma unroll 1
            for (int i = threadIdx.x; i - lane < lists * a.n_top; i += kThreads) {
                const uint64_t k = i < lists * a.n_top ? keys[i] : 0ull;
                const uint64_t in = __ballot(k && k >= least);
                int at = 0;
                if (in && lane == 0)
                    at = atomicAdd(&n_joined, __popcll(in));
                at = __builtin_amdgcn_readfirstlane(at);
                if (k && k >= least)
                    joined[at + __popcll(in & ((1ull << lane) - 1ull))] = k;
            }
            __syncthreads();
            list.clear();
            if (wave == 0) {
                const int m = n_joined;
                if (lane < 8)
                    joined[m + lane] = 0;
                wave_sync();
#pragma unroll 1
                for (int i = 0; i < m; i += kWave)
                    list.take(joined + i, min(m - i, kWave), scratch);
            }
        }
        if (wave == 0) {
            s = SumState{lane < kWaves ? states[lane].m : -INFINITY,
                         lane < kWaves ? states[lane].l : 0.f,
                         lane < kWaves ? states[lane].t : 0.f};
            s = lanes_join(s);
            ahead = ranks[0] + ranks[1] + ranks[2] + ranks[3];
        }
        if (last_round)
            break;
        if (wave == 0) {
            float *ps = a.part_state + (first + part) * 4;
            if (lane == 0) {
                store_agent(ps, s.m);
                store_agent(ps + 1, s.l);
                store_agent(ps + 2, s.t);
                store_agent(ps + 3, __int_as_float(ahead));
            }
            if (lane < a.n_top)
                store_agent(a.part_keys + (first + part) * a.n_top + lane, list.best);
        }
        if (!arrive_last_direct(a.arrived + row * kCounterStride, a.parts))
            return;
        if (threadIdx.x == 0)
            a.arrived[row * kCounterStride] = 0;
        // the parts' states, one to a lane of the first wave, and their lists
        s = SumState{-INFINITY, 0.f, 0.f};
        ahead = 0;
        if (wave == 0) {
            if (lane < a.parts) {
                const float *ps = a.part_state + (first + lane) * 4;
                s = SumState{load_agent(ps), load_agent(ps + 1), load_agent(ps + 2)};
                ahead = __float_as_int(load_agent(ps + 3));
            }
            ahead = wave_reduce(ahead, 0, [](int x, int y) { return x + y; });
        }
        if (a.n_top) {
            const int n = a.parts * a.n_top;
            constexpr int N = kPartKeys / kThreads;
            uint64_t got[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int at = i * kThreads + threadIdx.x;
                got[i] = at < n ? load_agent(a.part_keys + first * a.n_top + at) : 0ull;
            }
#pragma unroll
            for (int i = 0; i < N; ++i)
                keys[i * kThreads + threadIdx.x] = got[i];
            lists = a.parts;
        }
        last_round = true;
    }
    if (wave != 0)
        return;
    // ---- results: one wave ----
    // (a row of nothing but -inf has l = 0; +inf or NaN leave NaN in l)
    const float logl = s.l > 0.f ? logf(s.l) : NAN;
    if (lane == 0) {
        if (a.logprob)
            a.logprob[row] = has_token ? (zt - s.m) - logl : 0.f;
        if (a.rank)
            a.rank[row] = has_token ? ahead : -1;
        if (a.entropy)
            a.entropy[row] = logl - s.t / s.l;
    }
    if (lane < a.n_top) {
        const uint32_t o = (uint32_t)(list.best >> 32);
        const size_t dst = (size_t)row * a.n_top + lane;
        a.top_ids[dst] = (int32_t)~(uint32_t)list.best;
        a.top_lp[dst] = ((o == ~0u ? NAN : order_value(o)) - s.m) - logl;
    }
}

struct LogprobPlan {
    int parts, part_len;
};

// Rows are cut where they are too few to fill the chip (about four workgroups a
// CU), down to one group of a wave's loads a lane.  (2000 rows in four parts each
// take 201 us, whole 148: every part begins its lists anew.)
LogprobPlan plan_logprobs(wf_dtype_t dt, int n_rows, int vocab, int n_top) {
    const int unit = kThreads * (dt == WF_F32 ? 4 : 8) * kLoads;
    const int most = std::min({kMaxParts, (vocab + unit - 1) / unit, kPartKeys / std::max(n_top, 1)});
    const int want = std::max(1, 2 * kMaxSplitRows / std::max(n_rows, 1));
    const int parts = std::min(most, want);
    const int len = ((vocab + parts - 1) / parts + unit - 1) / unit * unit;
    return LogprobPlan{(vocab + len - 1) / len, len};
}

size_t state_bytes(int n_rows, const LogprobPlan &p) {
    return ((size_t)n_rows * p.parts * 16 + 255) & ~(size_t)255;
}

}  // namespace

size_t token_logprobs_workspace_bytes(wf_dtype_t dt, int n_rows, int vocab, int n_top) {
    const LogprobPlan p = plan_logprobs(dt, n_rows, vocab, n_top);
    return kCounterBytes +
           (p.parts > 1 ? state_bytes(n_rows, p) + (size_t)n_rows * p.parts * n_top * 8 : 0);
}

wf_status_t launch_token_logprobs(wf_dtype_t dt, const void *logits, size_t row_stride,
                                  const int32_t *tokens, int n_rows, int vocab, int n_top,
                                  float *logprob, float *entropy, int32_t *rank,
                                  int32_t *top_ids, float *top_lp, void *workspace,
                                  hipStream_t stream) {
    const LogprobPlan p = plan_logprobs(dt, n_rows, vocab, n_top);
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
    // of P lists of n keys, the want-th largest of the r-th keys is reached by
    // r * want >= n keys
    auto bound = [&](int lists, int &r, int &want) {
        r = (std::max(n_top, 1) + lists - 1) / lists;
        want = (std::max(n_top, 1) + r - 1) / r;
    };
    bound(kWaves, a.wave_r, a.wave_want);
    bound(p.parts, a.part_r, a.part_want);
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
