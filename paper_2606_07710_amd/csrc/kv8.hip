// kv8.hip -- writing the 8-bit KV cache: append (quantise new rows) and the
// compaction of an accepted tree path.  Both end in the same step: the valid
// rows of a 32-token block are encoded under the power of two that their
// largest magnitude asks for.
//
// A workgroup owns one block of one head, K or V (append), or the up to three
// blocks that a path can touch (compaction), so a block's scale needs no
// exchange between workgroups.  K blocks are [32][D], V blocks [D][32]: the
// rows are staged in LDS and leave in 16-byte pieces of either order.
#include "wf_api_internal.h"
#include "wf_lowbit.h"

namespace wf {

namespace {

constexpr int kThreads = 256;

// Largest of the workgroup's values, in every thread.
__device__ __forceinline__ float group_max(float v, float *part) {
    v = wave_max(v);
    if (threadIdx.x % kWave == 0)
        part[threadIdx.x / kWave] = v;
    __syncthreads();
    float m = part[0];
#pragma unroll
    for (int w = 1; w < kThreads / kWave; ++w)
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
};

// One block of one head, K or V.  The block's valid rows are staged as fp32:
// new rows from the source, rows below `start` decoded from their codes.
template <int D, bool BF16>
__global__ __launch_bounds__(kThreads) void kv8_append(AppendParams a) {
    constexpr int LD = D + 1;            // columns of 32 rows in distinct banks
    __shared__ float val[kKv8Block * LD];
    __shared__ float part[kThreads / kWave];
    const int b = a.first_block + blockIdx.x;
    const int g = blockIdx.y, kind = blockIdx.z;
    const int r0 = b * kKv8Block;
    const int first = max(a.start - r0, 0);              // first new row of the block
    const int last = min(a.end - r0, kKv8Block);         // end of its valid rows
    const size_t at = (size_t)g * a.n_blocks + b;
    char *codes = a.codes[kind] + at * (kKv8Block * D);
    uint8_t *scale = a.scale[kind] + at;

    float m = 0.f;
    // new rows, 8 elements per thread
    for (int c = threadIdx.x; c < (last - first) * (D / 8); c += kThreads) {
        const int r = first + c / (D / 8), d = c % (D / 8) * 8;
        const size_t off = (size_t)(r0 + r - a.start) * a.tok_stride + g * a.head_stride + d;
        float f[8];
        if constexpr (BF16) {
            const u32x4 v = *reinterpret_cast<const u32x4 *>(
                static_cast<const uint16_t *>(a.src[kind]) + off);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f[2 * i] = __uint_as_float(v[i] << 16);
                f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
            }
        } else {
            const f32x4 *p = reinterpret_cast<const f32x4 *>(
                static_cast<const float *>(a.src[kind]) + off);
            const f32x4 lo = p[0], hi = p[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f[i] = lo[i];
                f[4 + i] = hi[i];
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m = fmaxf(m, finite_abs(f[i]));
            val[r * LD + d + i] = f[i];
        }
    }
    // the open block's earlier rows, 4 codes per thread: 4 dims of a row (K),
    // 4 rows of a dim (V)
    if (first > 0) {
        const float s = scale_value(*scale);
        for (int c = threadIdx.x; c < kKv8Block * D / 4; c += kThreads) {
            const int hi = c / (kind ? kKv8Block / 4 : D / 4);
            const int lo = c % (kind ? kKv8Block / 4 : D / 4) * 4;
            if ((kind ? lo : hi) >= first)
                continue;
            float f[4];
            e4m3x4_to_f32(reinterpret_cast<const uint32_t *>(codes)[c], f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = kind ? lo + i : hi, d = kind ? hi : lo + i;
                if (r < first) {
                    const float x = f[i] * s;
                    m = fmaxf(m, finite_abs(x));
                    val[r * LD + d] = x;
                }
            }
        }
    }
    m = group_max(m, part);              // (its barrier publishes the rows too)
    const int e = e4m3_exponent(m);
    const float inv = __uint_as_float((unsigned)(127 - e) << 23);
    for (int c = threadIdx.x; c < kKv8Block * D / 16; c += kThreads) {
        float f[16];
        u32x4 *dst = reinterpret_cast<u32x4 *>(codes) + c;
        if (kind == 0) {
            const int r = c / (D / 16), d = c % (D / 16) * 16;
            if (r >= last)
                continue;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                f[i] = val[r * LD + d + i];
            *dst = encode16(f, inv);
        } else {
            const int d = c / 2, r = c % 2 * 16;
            if (r >= last)
                continue;
            const bool whole = r + 16 <= last;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                f[i] = whole || r + i < last ? val[(r + i) * LD + d] : 0.f;
            u32x4 w = encode16(f, inv);
            if (!whole) {
                const u32x4 old = *dst;              // rows behind the last valid one
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int n = min(max(last - (r + 4 * i), 0), 4);
                    const uint32_t mask = n == 4 ? ~0u : (1u << (8 * n)) - 1u;
                    w[i] = (w[i] & mask) | (old[i] & ~mask);
                }
            }
            *dst = w;
        }
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
        m = group_max(m, part);
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
                              size_t head_stride, hipStream_t stream) {
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
    const dim3 grid(blocks, c.n_kv_heads, 2);
    if (c.head_dim == 128 && dt == WF_BF16)
        kv8_append<128, true><<<grid, kThreads, 0, stream>>>(a);
    else if (c.head_dim == 128)
        kv8_append<128, false><<<grid, kThreads, 0, stream>>>(a);
    else if (dt == WF_BF16)
        kv8_append<64, true><<<grid, kThreads, 0, stream>>>(a);
    else
        kv8_append<64, false><<<grid, kThreads, 0, stream>>>(a);
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
