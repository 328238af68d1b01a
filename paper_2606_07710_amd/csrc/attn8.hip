// attn8.hip -- verification attention over the 8-bit KV cache (the definition
// of attn.hip with K and V held as e4m3 codes under one power-of-two scale per
// 32-token block and head).
#include "wf_api_internal.h"
#include "wf_lowbit.h"

namespace wf {

namespace {

struct Attn8Params {
    const void *q;
    const char *k, *v;
    const uint8_t *k_scale, *v_scale;
    void *ws_o;               // [splits][gamma*n_q_heads][head_dim], unnormalised
    float *ws_ml;             // [splits][gamma*n_q_heads][2]: reference, sum
    const uint64_t *tree_mask;
    int gamma, ctx_len, n_blocks, n_q_heads, group, n_keys, splits, keys_per_split;
    float sl2;                // softmax_scale * log2(e)
};

// ---------------------------------------------------------------------------
// Plain kernel: one wave per (split, row, head), fp32 throughout.  64 keys at
// a time, two scale blocks: lane t forms key t's score from its code row, then
// lane d adds the weighted values of dim d (one or two per lane), whose codes
// lie together in the transposed V blocks.
// ---------------------------------------------------------------------------
template <int D, bool BF16>
__global__ __launch_bounds__(64) void attn8_rows(Attn8Params a) {
    constexpr int E = D / kWave;
    __shared__ float qs[D];
    __shared__ float ps[kWave];
    const int split = blockIdx.x;
    const int pr = blockIdx.y;           // i * n_q_heads + h
    const int i = pr / a.n_q_heads, h = pr % a.n_q_heads;
    const int g = h / a.group;
    const int lane = threadIdx.x;
    for (int d = lane; d < D; d += kWave) {
        if constexpr (BF16)
            qs[d] = bf16_to_f32(static_cast<const uint16_t *>(a.q)[(size_t)pr * D + d]);
        else
            qs[d] = static_cast<const float *>(a.q)[(size_t)pr * D + d];
    }
    __syncthreads();

    const int k_begin = split * a.keys_per_split;
    const bool tree = a.tree_mask != nullptr;
    const uint64_t gbits = a.gamma >= 64 ? ~0ull : (1ull << a.gamma) - 1ull;
    const uint64_t tm = tree ? ((a.tree_mask[i] | (1ull << i)) & gbits) : 0ull;
    const int k_end = min(min(a.n_keys, k_begin + a.keys_per_split),
                          tree ? a.n_keys : a.ctx_len + i + 1);
    const size_t head = (size_t)g * a.n_blocks;

    float m = -INFINITY, l = 0.f, acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e)
        acc[e] = 0.f;
    for (int kb = k_begin; kb < k_end; kb += kWave) {
        const int j = kb + lane;
        const int jb = j - a.ctx_len;
        const bool vis = j < k_end && (!tree || jb < 0 || ((tm >> jb) & 1ull));
        const uint64_t seen = __ballot(vis);
        float sc = -INFINITY;
        if (vis) {
            const size_t blk = head + j / kKv8Block;
            const u32x4 *kr = reinterpret_cast<const u32x4 *>(
                a.k + (blk * kKv8Block + j % kKv8Block) * D);
            float dot = 0.f;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                const u32x4 w = kr[c];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    float f[4];
                    e4m3x4_to_f32(w[u], f);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        dot = fmaf(qs[16 * c + 4 * u + e], f[e], dot);
                }
            }
            sc = dot * scale_value(a.k_scale[blk]);
        }
        if (seen == 0)                   // uniform: nothing of this step counts
            continue;
        const float mnew = fmaxf(m, wave_max(sc));
        const float alpha = (m == -INFINITY) ? 0.f : exp2f((m - mnew) * a.sl2);
        const float p = vis ? exp2f((sc - mnew) * a.sl2) : 0.f;
        l = fmaf(l, alpha, wave_sum(p));
        m = mnew;
        ps[lane] = p;
#pragma unroll
        for (int e = 0; e < E; ++e)
            acc[e] *= alpha;
        __syncthreads();
        for (int b = 0; b < 2; ++b) {
            const unsigned live = (unsigned)(seen >> (32 * b));
            if (live == 0)
                continue;
            const size_t blk = head + kb / kKv8Block + b;
            const float s = scale_value(a.v_scale[blk]);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const u32x4 *vr = reinterpret_cast<const u32x4 *>(
                    a.v + (blk * D + lane + e * kWave) * kKv8Block);
                const u32x4 w[2] = {vr[0], vr[1]};
                float sum = 0.f;
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    float f[4];
                    e4m3x4_to_f32(w[u / 4][u % 4], f);
#pragma unroll
                    for (int t = 0; t < 4; ++t)      // (a code no row sees may be a NaN)
                        if ((live >> (4 * u + t)) & 1u)
                            sum = fmaf(ps[32 * b + 4 * u + t], f[t], sum);
                }
                acc[e] = fmaf(sum, s, acc[e]);
            }
        }
        __syncthreads();
    }
    const size_t prs = (size_t)split * a.gamma * a.n_q_heads + pr;
#pragma unroll
    for (int e = 0; e < E; ++e)
        if constexpr (BF16)
            static_cast<uint16_t *>(a.ws_o)[prs * D + lane + e * kWave] = f32_to_bf16(acc[e]);
        else
            static_cast<float *>(a.ws_o)[prs * D + lane + e * kWave] = acc[e];
    if (lane == 0) {
        a.ws_ml[prs * 2] = m * a.sl2;
        a.ws_ml[prs * 2 + 1] = l;
    }
}

}  // namespace

AttnPlan plan_attn8(wf_dtype_t dt, int gamma, int ctx_len, int n_q_heads, int n_kv_heads,
                    int head_dim, int num_splits) {
    AttnPlan p = plan_attn(WF_F32, gamma, ctx_len, n_q_heads, n_kv_heads, head_dim, num_splits);
    p.part_bytes = dt == WF_BF16 ? 2 : 4;
    return p;
}

wf_status_t launch_attn8(wf_dtype_t dt, const void *q, const wf_kv8_cache_t &c, void *out,
                         int gamma, int ctx_len, int n_q_heads, float softmax_scale,
                         const uint64_t *tree_mask, const AttnPlan &p, void *workspace,
                         hipStream_t stream) {
    Attn8Params a{};
    const size_t pairs = (size_t)gamma * n_q_heads;
    a.q = q;
    a.k = static_cast<const char *>(c.k);
    a.v = static_cast<const char *>(c.v);
    a.k_scale = c.k_scale;
    a.v_scale = c.v_scale;
    a.ws_ml = reinterpret_cast<float *>(static_cast<char *>(workspace) + kCounterBytes);
    a.ws_o = a.ws_ml + (size_t)p.splits * pairs * 2;
    a.tree_mask = tree_mask;
    a.gamma = gamma;
    a.ctx_len = ctx_len;
    a.n_blocks = kv8_blocks(c.cap);
    a.n_q_heads = n_q_heads;
    a.group = n_q_heads / c.n_kv_heads;
    a.n_keys = ctx_len + gamma;
    a.splits = p.splits;
    a.keys_per_split = p.keys_per_split;
    a.sl2 = softmax_scale * kLog2e;
    const dim3 grid(p.splits, (unsigned)pairs);
    if (c.head_dim == 128 && dt == WF_BF16)
        attn8_rows<128, true><<<grid, 64, 0, stream>>>(a);
    else if (c.head_dim == 128)
        attn8_rows<128, false><<<grid, 64, 0, stream>>>(a);
    else if (dt == WF_BF16)
        attn8_rows<64, true><<<grid, 64, 0, stream>>>(a);
    else
        attn8_rows<64, false><<<grid, 64, 0, stream>>>(a);
    if (hipGetLastError() != hipSuccess)
        return WF_ERR_HIP;
    // (the references are held in log2 units, so the merge's factor is 1)
    return launch_attn_merge(c.head_dim, dt == WF_BF16, a.ws_o, a.ws_ml, out, (int)pairs,
                             p.splits, 1.f, stream);
}

}  // namespace wf
