// kv8.hip -- writing the 8-bit KV cache: append (quantise new rows) and the
// compaction of an accepted tree path.  Both end in the same step: the valid
// rows of a 32-token block are encoded under the power of two that their
// largest magnitude asks for.
//
// A workgroup owns one block of one head, K or V (append), or the up to three
// blocks that a path can touch (compaction), so a block's scale needs no
// exchange between workgroups.  K blocks are [32][D], V blocks [D][32].
//
// Bound by: few tokens, the launch and one trip to memory (16 tokens, 8 heads:
// 3.8 us, 1.7 of it what an empty launch takes); many, the bytes (8190 tokens, 50
// MB: 11.6 us, 4.4 TB/s, where a large copy reaches 5.0).  Compaction: the
// launch and two dependent trips, the path before the rows it picks from LDS
// (one layer 4.7 us, 36 layers 6.0).
#include "wf_api_internal.h"
#include "wf_lowbit.h"

namespace wf {

namespace {

constexpr int kThreads = 256;            // of a compaction workgroup

// Largest of the values of a workgroup of N threads, in every thread.
template <int N>
__device__ __forceinline__ float group_max(float v, float *part) {
    v = wave_max(v);
    if (threadIdx.x % kWave == 0)
        part[threadIdx.x / kWave] = v;
    __syncthreads();
    float m = part[0];
#pragma unroll
    for (int w = 1; w < N / kWave; ++w)
        m = fmaxf(m, part[w]);
    return m;
}

// 16 values times `inv` as 16 code bytes.
__device__ __forceinline__ u32x4 encode16(const float (&f)[16], float inv) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] = f32x4_to_e4m3(f[4 * i] * inv, f[4 * i + 1] * inv, f[4 * i + 2] * inv,
                             f[4 * i + 3] * inv);
    return w;
}

struct AppendParams {
    const void *src[2];      // K rows, V rows
    char *codes[2];
    uint8_t *scale[2];
    size_t tok_stride, head_stride;      // source strides in elements
    int start, end, n_blocks, first_block;
    const char *zero_end;    // CLEAR: source rows before it are zeroed once read
};

// One block of one head, K or V.  A thread owns 4 rows x 4 dims: it takes new
// rows from the source and rows below `start` from their codes, and encodes
// its 16 values as the four words that they are in the block (4 dims of a row
// in K, 4 rows of a dim in V).  Everything is loaded before anything is used,
// one trip to memory; V's words are put in order in LDS and leave as 16 bytes.
// The codes go past the L2, where no later call of another XCD would look for
// them (8190 tokens: 12.8 -> 11.6 us, out of HBM 14.4 -> 12.6; an attention right
// behind takes as long as before).  (Rows staged as fp32 in LDS, new ones, old ones and the scale loaded one
// after the other: 4.15 us for 16 tokens, 13.4 for 8190.)  CLEAR: the source is a
// workspace whose zero block has to be zero again; each element is read by one
// thread, which stores the zero.
template <int D, bool BF16, bool CLEAR>
__global__ __launch_bounds__(2 * D) void kv8_append(AppendParams a) {
    __shared__ float part[2 * D / kWave];
    // a V block in pieces of 16 rows of a dim, one more after every four dims:
    // the words of a wave fall into 32 banks, not one
    __shared__ u32x4 turned[D / 4 * 9];
    const int b = a.first_block + blockIdx.x;
    const int g = blockIdx.y, kind = blockIdx.z;
    const int r0 = b * kKv8Block;
    const int first = max(a.start - r0, 0);              // first new row of the block
    const int last = min(a.end - r0, kKv8Block);         // end of its valid rows
    const size_t at = (size_t)g * a.n_blocks + b;
    uint32_t *codes = reinterpret_cast<uint32_t *>(a.codes[kind] + at * (kKv8Block * D));
    uint8_t *scale = a.scale[kind] + at;
    const int j = threadIdx.x % (D / 4), i0 = threadIdx.x / (D / 4) * 4;
    auto word = [&](int u) {             // where the thread's word u lies in the block
        return kind ? (4 * j + u) * (kKv8Block / 4) + i0 / 4 : (i0 + u) * (D / 4) + j;
    };
    const bool partly = first > 0 || last < kKv8Block;
    uint32_t old[4] = {};
    unsigned sb = 127;
    if (partly) {
        sb = *scale;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            old[u] = codes[word(u)];
    }
    float f[4][4];                       // [row][dim]
    using Raw = std::conditional_t<BF16, u32x2, f32x4>;
    Raw raw[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        raw[u] = Raw{};
        if (i0 + u >= first && i0 + u < last) {
            const size_t off = (size_t)(r0 + i0 + u - a.start) * a.tok_stride +
                               g * a.head_stride + 4 * j;
            const char *from = static_cast<const char *>(a.src[kind]) + off * (BF16 ? 2 : 4);
            raw[u] = *reinterpret_cast<const Raw *>(from);
            if (CLEAR && from < a.zero_end)
                *reinterpret_cast<Raw *>(const_cast<char *>(from)) = Raw{};
        }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        if constexpr (BF16) {
            f[u][0] = __uint_as_float(raw[u][0] << 16);
            f[u][1] = __uint_as_float(raw[u][0] & 0xffff0000u);
            f[u][2] = __uint_as_float(raw[u][1] << 16);
            f[u][3] = __uint_as_float(raw[u][1] & 0xffff0000u);
        } else {
#pragma unroll
            for (int d = 0; d < 4; ++d)
                f[u][d] = raw[u][d];
        }
    }
    if (first > 0) {
        const float s = scale_value((uint8_t)sb);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float x[4];
            e4m3x4_to_f32(old[u], x);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                if (kind && i0 + w < first)
                    f[w][u] = x[w] * s;
                if (!kind && i0 + u < first)
                    f[u][w] = x[w] * s;
            }
        }
    }
    float m = 0.f;
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int d = 0; d < 4; ++d)
            m = fmaxf(m, finite_abs(f[u][d]));
    m = group_max<2 * D>(m, part);
    const int e = e4m3_exponent(m);
    const float inv = __uint_as_float((unsigned)(127 - e) << 23);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        if (kind == 0) {
            if (i0 + u < last)
                __builtin_nontemporal_store(f32x4_to_e4m3(f[u][0] * inv, f[u][1] * inv,
                                                          f[u][2] * inv, f[u][3] * inv),
                                            codes + word(u));
        } else {
            uint32_t w = f32x4_to_e4m3(f[0][u] * inv, f[1][u] * inv, f[2][u] * inv,
                                       f[3][u] * inv);
            // rows behind the last valid one keep their codes
            const int n = min(max(last - i0, 0), 4);
            const uint32_t mask = n == 4 ? ~0u : (1u << (8 * n)) - 1u;
            reinterpret_cast<uint32_t *>(turned)[word(u) + 4 * j] =
                (w & mask) | (old[u] & ~mask);
        }
    }
    if (kind) {
        __syncthreads();
        const int c = threadIdx.x;
        if (c % 2 * 16 < last)
            __builtin_nontemporal_store(turned[c + c / 8], reinterpret_cast<u32x4 *>(codes) + c);
    }
    if (threadIdx.x == 0)
        *scale = (uint8_t)(e + 127);
}

// Compaction: the blocks from row ctx on that hold the draft tree (at most
// 31 + 64 rows, three blocks) are staged as they are; destination row r takes
// the value of its source row, and each destination block is encoded anew.
constexpr int kMaxPathRows = 64;
constexpr int kPathBlocks = (kKv8Block - 1 + kMaxPathRows + kKv8Block - 1) / kKv8Block;

template <int D>
__global__ __launch_bounds__(kThreads) void kv8_compact(char *k, char *v, uint8_t *k_scale,
                                                        uint8_t *v_scale, const int32_t *accept,
                                                        const int32_t *path, int gamma,
                                                        int ctx_len, int n_blocks,
                                                        size_t code_stride, size_t scale_stride) {
    constexpr int BB = kKv8Block * D;    // bytes of a block
    __shared__ u32x4 raw[kPathBlocks * BB / 16];
    __shared__ float sval[kPathBlocks];
    __shared__ int src[kPathBlocks * kKv8Block];         // staged row of each valid row
    __shared__ float part[kThreads / kWave];
    const int g = blockIdx.x, kind = blockIdx.y;
    const int b0 = ctx_len / kKv8Block;
    const int held = ctx_len % kKv8Block;                // valid rows before the path
    const int staged = (held + gamma - 1) / kKv8Block + 1;
    const size_t at = (size_t)g * n_blocks + b0;
    char *codes = (kind ? v : k) + blockIdx.z * code_stride + at * BB;
    uint8_t *scale = (kind ? v_scale : k_scale) + blockIdx.z * scale_stride + at;
    const int n = min(max(accept[0], 0), gamma - 1);
    const int valid = held + n + 1;
    for (int c = threadIdx.x; c < staged * BB / 16; c += kThreads)
        raw[c] = reinterpret_cast<const u32x4 *>(codes)[c];
    if ((int)threadIdx.x < staged)
        sval[threadIdx.x] = scale_value(scale[threadIdx.x]);
    if ((int)threadIdx.x < valid) {
        const int t = (int)threadIdx.x - held;
        int p = t;
        if (t >= 0) {
            const int q = path[t];
            // the node at depth t has index >= t; anything else stays in place
            p = q >= t && q < gamma ? q : t;
        }
        src[threadIdx.x] = held + p;
    }
    __syncthreads();
    const uint8_t *bytes = reinterpret_cast<const uint8_t *>(raw);
    auto value = [&](int r, int d) {
        const int s = src[r], sb = s / kKv8Block, sr = s % kKv8Block;
        const unsigned code = bytes[sb * BB + (kind ? d * kKv8Block + sr : sr * D + d)];
        return __builtin_amdgcn_cvt_f32_fp8((int)code, 0) * sval[sb];
    };
    for (int b = 0; b * kKv8Block < valid; ++b) {
        const int r0 = b * kKv8Block, last = min(valid - r0, kKv8Block);
        // 16-byte pieces of the block: 16 dims of a row (K), 16 rows of a dim (V)
        constexpr int P = BB / 16 / kThreads > 0 ? BB / 16 / kThreads : 1;
        float f[P][16];
        float m = 0.f;
#pragma unroll
        for (int u = 0; u < P; ++u) {
            const int c = threadIdx.x + u * kThreads;
            if (c >= BB / 16)
                continue;
            const int hi = kind ? c / 2 : c / (D / 16);
            const int lo = kind ? c % 2 * 16 : c % (D / 16) * 16;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = kind ? lo + i : hi, d = kind ? hi : lo + i;
                f[u][i] = r < last ? value(r0 + r, d) : 0.f;
                m = fmaxf(m, finite_abs(f[u][i]));
            }
        }
        m = group_max<kThreads>(m, part);
        const int e = e4m3_exponent(m);
        const float inv = __uint_as_float((unsigned)(127 - e) << 23);
#pragma unroll
        for (int u = 0; u < P; ++u) {
            const int c = threadIdx.x + u * kThreads;
            if (c >= BB / 16)
                continue;
            const int lo = kind ? c % 2 * 16 : 0, hi = kind ? 0 : c / (D / 16);
            if ((kind ? lo : hi) >= last)
                continue;
            u32x4 w = encode16(f[u], inv);
            if (kind && lo + 16 > last) {
                const u32x4 old = raw[b * (BB / 16) + c];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int keep = min(max(last - (lo + 4 * i), 0), 4);
                    const uint32_t mask = keep == 4 ? ~0u : (1u << (8 * keep)) - 1u;
                    w[i] = (w[i] & mask) | (old[i] & ~mask);
                }
            }
            reinterpret_cast<u32x4 *>(codes)[b * (BB / 16) + c] = w;
        }
        if (threadIdx.x == 0)
            scale[b] = (uint8_t)(e + 127);
        __syncthreads();                 // `part` is used again
    }
}

}  // namespace

wf_status_t launch_kv8_append(wf_dtype_t dt, const wf_kv8_cache_t &c, const void *k,
                              const void *v, int n_tok, int start, size_t tok_stride,
                              size_t head_stride, const void *zero_end, hipStream_t stream) {
    AppendParams a{};
    a.src[0] = k;
    a.src[1] = v;
    a.codes[0] = static_cast<char *>(c.k);
    a.codes[1] = static_cast<char *>(c.v);
    a.scale[0] = c.k_scale;
    a.scale[1] = c.v_scale;
    a.tok_stride = tok_stride;
    a.head_stride = head_stride;
    a.start = start;
    a.end = start + n_tok;
    a.n_blocks = kv8_blocks(c.cap);
    a.first_block = start / kKv8Block;
    const int blocks = (start + n_tok - 1) / kKv8Block - a.first_block + 1;
    a.zero_end = static_cast<const char *>(zero_end);
    const dim3 grid(blocks, c.n_kv_heads, 2);
#define WF_APPEND(DV, BV, CV)                                                          \
    if (c.head_dim == DV && (dt == WF_BF16) == BV && (zero_end != nullptr) == CV)      \
        kv8_append<DV, BV, CV><<<grid, 2 * DV, 0, stream>>>(a);                        \
    else
    WF_APPEND(128, true, false) WF_APPEND(64, true, false)
    WF_APPEND(128, false, false) WF_APPEND(64, false, false)
    WF_APPEND(128, false, true) WF_APPEND(64, false, true)
    return WF_ERR_UNSUPPORTED;
#undef WF_APPEND
    return hipGetLastError() == hipSuccess ? WF_OK : WF_ERR_HIP;
}

wf_status_t launch_kv8_compact(const wf_kv8_cache_t &c, const int32_t *accept,
                               const int32_t *path, int gamma, int ctx_len, int n_layers,
                               size_t code_stride, size_t scale_stride, hipStream_t stream) {
    const dim3 grid(c.n_kv_heads, 2, n_layers);
    char *k = static_cast<char *>(c.k), *v = static_cast<char *>(c.v);
    const int nb = kv8_blocks(c.cap);
    if (c.head_dim == 128)
        kv8_compact<128><<<grid, kThreads, 0, stream>>>(k, v, c.k_scale, c.v_scale, accept, path,
                                                        gamma, ctx_len, nb, code_stride,
                                                        scale_stride);
    else
        kv8_compact<64><<<grid, kThreads, 0, stream>>>(k, v, c.k_scale, c.v_scale, accept, path,
                                                       gamma, ctx_len, nb, code_stride,
                                                       scale_stride);
    return hipGetLastError() == hipSuccess ? WF_OK : WF_ERR_HIP;
}

}  // namespace wf
