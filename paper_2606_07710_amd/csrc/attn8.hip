// attn8.hip -- verification attention over the 8-bit KV cache (the definition
// of attn.hip with K and V held as e4m3 codes under one power-of-two scale per
// 32-token block and head).
//
// bf16 queries: split-KV over the key range as in attn.hip, on the block-scaled
// matrix instruction (16x16x128, e4m3 by e4m3, one power-of-two scale per 32
// elements of the inner dimension on either side).  The cache feeds it as it
// lies in memory, its block scales as the instruction's scale operands, so
// nothing is dequantised; what is not e4m3, q and the softmax weights, goes in
// as two e4m3 parts.  fp32 queries: a plain kernel.
#include "wf_api_internal.h"
#include "wf_lds_dma.h"
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
    int gamma, ctx_len, n_blocks, n_q_heads, n_kv_heads, group, rows, n_keys;
    int splits, keys_per_split, n_row_groups;
    float sl2;                // softmax_scale * log2(e)
};

// ---------------------------------------------------------------------------
// bf16 queries.  A workgroup owns one KV head, a run of 128-key tiles (four
// scale blocks) and 16 * RG of the head's query rows, 16 per wave; the waves
// share the tiles, which travel HBM -> LDS by DMA through a ring of NBUF
// stages.  Per tile and wave:
//   S^T = K Q^T    eight 16-key blocks, each one or two instructions: A = the
//                  codes of 16 keys, all dims, with the scales of their token
//                  blocks; B = q^T as e4m3 parts hi + lo (head_dim 64: both
//                  parts in one instruction, against the keys twice)
//   P = 2^(S sl2 - E + 8), E = ceil of the row's largest S sl2 in the tile
//   O^T += V^T P^T  per 16 dims two instructions over all 128 keys: A = the
//                  transposed V codes with the token blocks' scales, B = P^T as
//                  hi + lo with the scale 2^(E - R)
// The running softmax keeps one integer reference R per row, and a tile's
// weights are put under it by the scale operand, not by rescaling O: only a
// tile more than 2^64 above R moves it.
//
// Two parts of e4m3 hold 8 significant bits, as bf16 does, the second one 16
// times as large as it counts so that small values keep theirs: values of at
// most 256 are held to 2^-9 of themselves or 2^-14, whichever is more.  (With
// the second part as it is that floor is 2^-10, and the many small weights of
// a row with one large one come out up to 6 times further off.)  q is scaled
// to a largest element in [128, 256).
//
// Which key is which row of A is free, and chosen so that the S^T accumulators
// of a lane are, in order, the bytes of its P^T operand: instruction mb takes
// row m = 4 c + i from key 64 (mb / 4) + 16 c + 4 (mb % 4) + i, so lane (m16,
// c4) ends with the keys 16 c4 .. +15 of each half of the tile -- the 16 + 16
// inner indices that the instruction reads from lane group c4, against which
// a transposed V block lies as it is.
//
// LDS tiles are swizzled in 16-byte granules so that the eight lanes of a
// quarter of a ds_read_b128 meet distinct banks: K granule g of key k at
// g ^ ((k & 3) | (k >> 4 & 1) << 2) (head_dim 64: two keys share 128 bytes, g ^
// ((k >> 1 & 1) | (k >> 4 & 1) << 1)), V half h of dim d at
// h ^ (d >> 2 & 1) ^ (d >> 3 & 1).
// ---------------------------------------------------------------------------
constexpr int kTileKeys8 = 128;
constexpr int kTileBlocks = kTileKeys8 / kKv8Block;
constexpr float kRefGrow = 64.f;         // log2 growth that moves a row's reference

typedef int i32x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ i32x8 join(u32x4 lo, u32x4 hi) {
    return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3],
                 (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// Byte OA / OB of sa / sb is the lane's scale of A / B.
template <int OA, int OB>
__device__ __forceinline__ f32x4 mfma_e4m3(i32x8 a, i32x8 b, f32x4 c, unsigned sa, unsigned sb) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, OA, (int)sa, OB,
                                                            (int)sb);
}

// Four values of at most 256 as two e4m3 parts hi + lo / 16.
constexpr int kLoShift = 4;
__device__ __forceinline__ void two_parts(const float (&p)[4], uint32_t &hi, uint32_t &lo) {
    typedef short i16x2 __attribute__((ext_vector_type(2)));
    constexpr float kLo = 1.f / (1 << kLoShift);     // (the conversion divides by it)
    int h = __builtin_amdgcn_cvt_pk_fp8_f32(p[0], p[1], 0, false);
    h = __builtin_amdgcn_cvt_pk_fp8_f32(p[2], p[3], h, true);
    float f[4];
    e4m3x4_to_f32((uint32_t)h, f);
    i16x2 l = {0, 0};
    l = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(l, p[0] - f[0], p[1] - f[1], kLo, false);
    l = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(l, p[2] - f[2], p[3] - f[3], kLo, true);
    hi = (uint32_t)h;
    lo = __builtin_bit_cast(uint32_t, l);
}

// The scale bytes of a tile's four blocks, in one dword: two aligned scalar
// loads, neither of them past the dword that holds the head's last used byte.
// Blocks past it read as scale 1 (their codes are masked).
__device__ __forceinline__ unsigned tile_scales(const uint8_t *s, int block, int last_block) {
    typedef const __attribute__((address_space(4))) uint32_t *scalar_ptr;
    const uintptr_t at = reinterpret_cast<uintptr_t>(s + block);
    const uintptr_t end = reinterpret_cast<uintptr_t>(s + last_block);
    const uintptr_t a0 = at & ~(uintptr_t)3, e0 = end & ~(uintptr_t)3;
    const uint32_t w0 = *(scalar_ptr)a0;
    const uint32_t w1 = *(scalar_ptr)(a0 + 4 < e0 ? a0 + 4 : e0);
    uint32_t w = (uint32_t)(((uint64_t)w1 << 32 | w0) >> (8 * (at & 3)));
    const int live = last_block - block + 1;
    if (live < kTileBlocks) {
        const uint32_t keep = (1u << (8 * live)) - 1u;
        w = (w & keep) | (0x7f7f7f7fu & ~keep);
    }
    return w;
}

template <int D, int RG, int NBUF>
__global__ __launch_bounds__(64 * RG) void attn8_tiles(Attn8Params a) {
    constexpr int HALF = kTileKeys8 * D;             // bytes of a K or V tile
    constexpr int STAGE = 2 * HALF;
    constexpr int LOADS = STAGE / 1024;              // wave loads per stage
    constexpr int LPW = LOADS / RG;
    constexpr int MD = D / 16;
    constexpr int GRAN = D / 16;                     // 16-byte granules of a key
    constexpr int BLOCK = kKv8Block * D;             // bytes of a scale block
    static_assert(LOADS % (2 * RG) == 0 && (NBUF - 2) * LPW < 64, "ring");
    static_assert(NBUF * STAGE <= 160 * 1024, "LDS");
    __shared__ __attribute__((aligned(1024))) char ring[NBUF * STAGE];

    // ---- which (kv head, split, row group) this workgroup owns ----------------
    int unit, rgw;
    if (a.n_row_groups == 1) {
        unit = blockIdx.x;
        rgw = 0;
    } else {
        // the row groups of one (head, split) on one XCD, adjacent in its
        // dispatch order: all but the first find the tiles in its L2
        const int xcd = blockIdx.x & 7, w = blockIdx.x >> 3;
        rgw = w % a.n_row_groups;
        unit = (w / a.n_row_groups) * 8 + xcd;
    }
    if (unit >= a.n_kv_heads * a.splits)
        return;
    const int g = unit % a.n_kv_heads;
    const int split = unit / a.n_kv_heads;
    const int wave = wave_id();
    const int lane = threadIdx.x % kWave;
    const int m16 = lane & 15;
    const int c4 = lane >> 4;

    const int tiles = (a.n_keys + kTileKeys8 - 1) / kTileKeys8;
    const int t_first = (int)((long long)split * tiles / a.splits);
    const int n_steps = (int)((long long)(split + 1) * tiles / a.splits) - t_first;
    const int last_block = (a.n_keys - 1) / kKv8Block;
    const float sl2 = a.sl2;
    const size_t head = (size_t)g * a.n_blocks;
    const char *kg = a.k + head * BLOCK;
    const char *vg = a.v + head * BLOCK;

    // Copies stage st: load j < LOADS / 2 of K, the rest of V, 1 KB each, dealt
    // out to the waves.  A scale block past the last one repeats that block.
    auto issue = [&](int st) __attribute__((always_inline)) {
        const int b0 = (t_first + st) * kTileBlocks;
        const unsigned slot = lds_addr(ring) + (st % NBUF) * STAGE;
        const int most = last_block - b0;                // last block of the tile
#pragma unroll
        for (int jr = 0; jr < LPW; ++jr) {
            const bool is_v = jr >= LPW / 2;
            const int j = wave + (jr - (is_v ? LPW / 2 : 0)) * RG;
            unsigned off;
            if (is_v) {
                const int d = 32 * j + (lane >> 1);
                off = 1024u * j + 32u * (lane >> 1) + 16u * ((lane ^ (d >> 2) ^ (d >> 3)) & 1);
            } else {
                const int k = j * (1024 / D) + lane / GRAN;
                const int f = D == 128 ? (k & 3) | (k >> 2 & 4) : (k >> 1 & 1) | (k >> 3 & 2);
                off = (unsigned)(k * D + ((lane % GRAN) ^ f) * 16);
            }
            const int b = j * 1024 / BLOCK;
            const size_t src = (size_t)(b0 + min(b, most)) * BLOCK;
            lds_dma16_so((is_v ? vg : kg) + src, off - (unsigned)(b * BLOCK),
                         slot + (is_v ? HALF : 0) + j * 1024);
        }
    };

    // ---- the wave's 16 rows: q in two parts -------------------------------------
    const int row = rgw * 16 * RG + wave * 16 + m16;
    const int rc = min(row, a.rows - 1);             // (padding rows repeat the last one)
    const int qi = rc / a.group;
    const int qh = g * a.group + rc % a.group;
    constexpr int QW = D / 64;                       // 16-dim pieces of q per lane
    i32x8 qop[2];
    unsigned qscale, qlo;
    {
        const uint16_t *qp = static_cast<const uint16_t *>(a.q) +
                             ((size_t)qi * a.n_q_heads + qh) * D + c4 * 16;
        float f[16 * QW];
        float m = 0.f;
#pragma unroll
        for (int w = 0; w < 2 * QW; ++w) {
            const u32x4 v = *reinterpret_cast<const u32x4 *>(qp + (w / 2) * 64 + (w % 2) * 8);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[8 * w + 2 * e] = __uint_as_float(v[e] << 16);
                f[8 * w + 2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
            }
        }
#pragma unroll
        for (int e = 0; e < 16 * QW; ++e)
            m = fmaxf(m, fabsf(f[e]));
        m = fmaxf(m, __shfl_xor(m, 16, kWave));
        m = fmaxf(m, __shfl_xor(m, 32, kWave));
        const int e = max((int)(__float_as_uint(m) >> 23) - 127 - 7, -120);
        const float inv = __uint_as_float((unsigned)(127 - e) << 23);
        qscale = (unsigned)(e + 127);
        uint32_t hi[4 * QW], lo[4 * QW];
#pragma unroll
        for (int w = 0; w < 4 * QW; ++w) {
            const float p[4] = {f[4 * w] * inv, f[4 * w + 1] * inv, f[4 * w + 2] * inv,
                                f[4 * w + 3] * inv};
            two_parts(p, hi[w], lo[w]);
        }
        qlo = qscale - kLoShift;
        if constexpr (D == 128) {
            qop[0] = join(u32x4{hi[0], hi[1], hi[2], hi[3]}, u32x4{hi[4], hi[5], hi[6], hi[7]});
            qop[1] = join(u32x4{lo[0], lo[1], lo[2], lo[3]}, u32x4{lo[4], lo[5], lo[6], lo[7]});
        } else {
            qop[0] = join(u32x4{hi[0], hi[1], hi[2], hi[3]}, u32x4{lo[0], lo[1], lo[2], lo[3]});
            qop[1] = qop[0];
            if (c4 >= 2)                 // (lane groups 2 and 3 scale the second halves)
                qscale = qlo;
        }
    }
    const bool tree = a.tree_mask != nullptr;        // kernel argument: uniform
    const uint64_t gbits = a.gamma >= 64 ? ~0ull : (1ull << a.gamma) - 1ull;
    const uint64_t tm = tree ? ((a.tree_mask[qi] | (1ull << qi)) & gbits) : 0ull;
    const int lim = a.ctx_len + qi;
    // the loads above are in before the first copy is issued, so no wait for
    // them is left inside the loop
    asm volatile("s_waitcnt vmcnt(0)" : "+v"(qop[0]), "+v"(qop[1]), "+v"(qscale), "+v"(qlo));

    f32x4 o[MD];
#pragma unroll
    for (int md = 0; md < MD; ++md)
        o[md] = f32x4{0.f, 0.f, 0.f, 0.f};
    float ref = -INFINITY, lsum = 0.f;

    auto compute = [&](int st) __attribute__((always_inline)) {
        const WF_LDS(char) *kt = (const WF_LDS(char) *)ring + (st % NBUF) * STAGE;
        const WF_LDS(char) *vt = kt + HALF;
        const int b0 = (t_first + st) * kTileBlocks;
        const int kb = b0 * kKv8Block;
        // lane's scale of row m16 (token block m16 / 8 of either half) in bytes
        // 0 and 2; lane's scale of token block c4
        const unsigned ks = tile_scales(a.k_scale + head, b0, last_block) >> (8 * (m16 >> 3));
        const unsigned vs = tile_scales(a.v_scale + head, b0, last_block) >> (8 * c4);

        // S^T = K Q^T
        f32x4 s[8];
#pragma unroll
        for (int mb = 0; mb < 8; ++mb) {
            const int k = 64 * (mb >> 2) + 16 * (m16 >> 2) + 4 * (mb & 3) + (m16 & 3);
            const WF_LDS(char) *kr = kt + k * D;
            i32x8 kop;
            if constexpr (D == 128) {
                const int f = (k & 3) | (k >> 2 & 4);
                kop = join(*(const WF_LDS(u32x4) *)(kr + (c4 ^ f) * 16),
                           *(const WF_LDS(u32x4) *)(kr + ((c4 + 4) ^ f) * 16));
            } else {
                const int f = (k >> 1 & 1) | (k >> 3 & 2);
                const u32x4 w = *(const WF_LDS(u32x4) *)(kr + (c4 ^ f) * 16);
                kop = join(w, w);
            }
            const f32x4 z = {0.f, 0.f, 0.f, 0.f};
            s[mb] = mb < 4 ? mfma_e4m3<0, 0>(kop, qop[0], z, ks, qscale)
                           : mfma_e4m3<2, 0>(kop, qop[0], z, ks, qscale);
            if constexpr (D == 128)
                s[mb] = mb < 4 ? mfma_e4m3<0, 0>(kop, qop[1], s[mb], ks, qlo)
                               : mfma_e4m3<2, 0>(kop, qop[1], s[mb], ks, qlo);
        }
        // mask: only tiles that reach into the block
        if (kb + kTileKeys8 > a.ctx_len) {
#pragma unroll
            for (int mb = 0; mb < 8; ++mb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = kb + 64 * (mb >> 2) + 16 * c4 + 4 * (mb & 3) + i;
                    const int j = key - a.ctx_len;
                    const bool bit = ((tm >> (j & 63)) & 1ull) != 0;
                    const bool vis = tree ? (j < 0) | ((j < a.gamma) & bit) : key <= lim;
                    s[mb][i] = vis ? s[mb][i] : -INFINITY;
                }
        }
        float m = s[0][0];
#pragma unroll
        for (int mb = 0; mb < 8; ++mb)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                m = fmaxf(m, s[mb][i]);
        m = fmaxf(m, __shfl_xor(m, 16, kWave));
        m = fmaxf(m, __shfl_xor(m, 32, kWave));
        // the row's exponent in this tile, and against its reference
        const bool any = m > -INFINITY;
        const float e = any ? ceilf(m * sl2) : 0.f;
        if (__ballot(any && !(e - ref <= kRefGrow))) {
            // (also a row's first visible tile: ref is -inf, o and lsum zero)
            if (any && !(e - ref <= kRefGrow)) {
                const float back = fast_exp2(ref - e);
                lsum *= back;
#pragma unroll
                for (int md = 0; md < MD; ++md)
                    o[md] *= back;
                ref = e;
            }
        }
        const int shift = any ? (int)fmaxf(e - ref, -120.f) : 0;
        const unsigned ps = (unsigned)(127 + shift);
        // P, its sum and its two parts
        const float add = 8.f - e;
        float psum = 0.f;
        uint32_t hi[8], lo[8];
#pragma unroll
        for (int mb = 0; mb < 8; ++mb) {
            float p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[i] = fast_exp2(fmaf(s[mb][i], sl2, add));
                psum += p[i];
            }
            two_parts(p, hi[mb], lo[mb]);
        }
        lsum += ldexpf(psum, shift);
        const i32x8 ph = join(u32x4{hi[0], hi[1], hi[2], hi[3]}, u32x4{hi[4], hi[5], hi[6], hi[7]});
        const i32x8 pl = join(u32x4{lo[0], lo[1], lo[2], lo[3]}, u32x4{lo[4], lo[5], lo[6], lo[7]});
        // O^T += V^T P^T
        const bool ragged = kb + kTileKeys8 > a.n_keys;
#pragma unroll
        for (int md = 0; md < MD; ++md) {
            const int d = 16 * md + m16;
            const WF_LDS(char) *vr = vt + (c4 >> 1) * BLOCK + d * kKv8Block +
                                     ((c4 ^ (d >> 2) ^ (d >> 3)) & 1) * 16;
            u32x4 v0 = *(const WF_LDS(u32x4) *)vr;
            u32x4 v1 = *(const WF_LDS(u32x4) *)(vr + 2 * BLOCK);
            if (ragged) {
                // codes behind the last key may be NaN, and 0 * NaN is no zero
                const int n0 = a.n_keys - kb - 16 * c4, n1 = n0 - 64;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int x0 = min(max(n0 - 4 * w, 0), 4), x1 = min(max(n1 - 4 * w, 0), 4);
                    v0[w] &= (uint32_t)((1ull << (8 * x0)) - 1ull);
                    v1[w] &= (uint32_t)((1ull << (8 * x1)) - 1ull);
                }
            }
            const i32x8 vop = join(v0, v1);
            o[md] = mfma_e4m3<0, 0>(vop, ph, o[md], vs, ps);
            o[md] = mfma_e4m3<0, 0>(vop, pl, o[md], vs, ps - kLoShift);
        }
    };

    // ---- the ring: up to NBUF - 1 stages in flight -------------------------------
#pragma unroll
    for (int st = 0; st < NBUF - 1; ++st)
        if (st < n_steps)
            issue(st);
    for (int st = 0; st < n_steps; ++st) {
        // (loads complete in order; the stages issued after st stay in flight)
        const int later = min(NBUF - 2, n_steps - 1 - st);
        if (NBUF > 3 && later >= 2)
            wait_vmcnt<(NBUF > 3 ? 2 : 0) * LPW>();
        else if (later >= 1)
            wait_vmcnt<LPW>();
        else
            wait_vmcnt<0>();
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (st + NBUF - 1 < n_steps)
            issue(st + NBUF - 1);
        compute(st);
    }

    // ---- the split's partial ---------------------------------------------------------
    lsum += __shfl_xor(lsum, 16, kWave);
    lsum += __shfl_xor(lsum, 32, kWave);
    if (row >= a.rows)
        return;
    const size_t pr = ((size_t)split * a.gamma + qi) * a.n_q_heads + qh;
    uint2 *dst = reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.ws_o) + pr * D);
#pragma unroll
    for (int md = 0; md < MD; ++md)
        dst[md * 4 + c4] = uint2{pack_bf16x2(o[md][0], o[md][1]), pack_bf16x2(o[md][2], o[md][3])};
    if (c4 == 0) {
        a.ws_ml[pr * 2] = ref;
        a.ws_ml[pr * 2 + 1] = lsum;
    }
}

// ---------------------------------------------------------------------------
// fp32 queries: one wave per (split, row, head), fp32 throughout.  64 keys at
// a time, two scale blocks: lane t forms key t's score from its code row, then
// lane d adds the weighted values of dim d (one or two per lane), whose codes
// lie together in the transposed V blocks.
// ---------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(64) void attn8_rows(Attn8Params a) {
    constexpr int E = D / kWave;
    __shared__ float qs[D];
    __shared__ float ps[kWave];
    const int split = blockIdx.x;
    const int pr = blockIdx.y;           // i * n_q_heads + h
    const int i = pr / a.n_q_heads, h = pr % a.n_q_heads;
    const int g = h / a.group;
    const int lane = threadIdx.x;
    for (int d = lane; d < D; d += kWave)
        qs[d] = static_cast<const float *>(a.q)[(size_t)pr * D + d];
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
        static_cast<float *>(a.ws_o)[prs * D + lane + e * kWave] = acc[e];
    if (lane == 0) {
        a.ws_ml[prs * 2] = m * a.sl2;
        a.ws_ml[prs * 2 + 1] = l;
    }
}

}  // namespace

// Split plan of a call.  bf16: 16 rows per wave and up to 8 waves, so that up
// to 128 rows share a tile; one workgroup per CU, none without a tile.
AttnPlan plan_attn8(wf_dtype_t dt, int gamma, int ctx_len, int n_q_heads, int n_kv_heads,
                    int head_dim, int num_splits) {
    if (dt == WF_F32)
        return plan_attn(WF_F32, gamma, ctx_len, n_q_heads, n_kv_heads, head_dim, num_splits);
    AttnPlan p{};
    p.part_bytes = 2;
    p.rows = n_q_heads / n_kv_heads * gamma;
    p.nb = p.ks = 1;
    p.rg = p.rows <= 16 ? 1 : p.rows <= 32 ? 2 : p.rows <= 64 ? 4 : 8;
    p.n_row_groups = (p.rows + 16 * p.rg - 1) / (16 * p.rg);
    const int tiles = (ctx_len + gamma + kTileKeys8 - 1) / kTileKeys8;
    const int want = num_splits > 0 ? num_splits
                                    : std::max(1, 256 / (n_kv_heads * p.n_row_groups));
    p.splits = std::min(want, tiles);
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
    a.n_kv_heads = c.n_kv_heads;
    a.group = n_q_heads / c.n_kv_heads;
    a.rows = p.rows;
    a.n_keys = ctx_len + gamma;
    a.splits = p.splits;
    a.keys_per_split = p.keys_per_split;
    a.n_row_groups = p.n_row_groups;
    a.sl2 = softmax_scale * kLog2e;
    if (dt == WF_BF16) {
        const int units = c.n_kv_heads * p.splits;
        const dim3 grid(p.n_row_groups > 1 ? (units + 7) / 8 * 8 * p.n_row_groups : units);
#define WF_ATTN8(DV, RGV, NBUFV)                                                           \
    if (c.head_dim == DV && p.rg == RGV)                                                   \
        attn8_tiles<DV, RGV, NBUFV><<<grid, 64 * RGV, 0, stream>>>(a);                     \
    else
        WF_ATTN8(128, 1, 3) WF_ATTN8(128, 2, 4) WF_ATTN8(128, 4, 4) WF_ATTN8(128, 8, 4)
        WF_ATTN8(64, 1, 4) WF_ATTN8(64, 2, 4) WF_ATTN8(64, 4, 4) WF_ATTN8(64, 8, 4)
        return WF_ERR_UNSUPPORTED;
#undef WF_ATTN8
    } else {
        const dim3 grid(p.splits, (unsigned)pairs);
        if (c.head_dim == 128)
            attn8_rows<128><<<grid, 64, 0, stream>>>(a);
        else
            attn8_rows<64><<<grid, 64, 0, stream>>>(a);
    }
    if (hipGetLastError() != hipSuccess)
        return WF_ERR_HIP;
    // (the references are held in log2 units, so the merge's factor is 1)
    return launch_attn_merge(c.head_dim, dt == WF_BF16, a.ws_o, a.ws_ml, out, (int)pairs,
                             p.splits, 1.f, stream);
}

}  // namespace wf
