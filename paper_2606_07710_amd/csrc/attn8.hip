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
    void *ws_o;               // [splits][gamma*n_q_heads][head_dim] fp32, unnormalised;
                              // of one split: the output itself
    float *ws_ml;             // [splits][gamma*n_q_heads][2]: reference, sum
    const uint64_t *tree_mask;
    int gamma, ctx_len, n_blocks, n_q_heads, n_kv_heads, group, rows, n_keys;
    int splits, n_row_groups;
    int tiles_per_split, extra_tiles;    // a split's tiles (fp32: steps); the first ones' extra
    unsigned group_magic;     // floor(2^32 / group) + 1: row / group as a high product
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
//                  hi + lo with the scale 2^(E - R - 8)
// The running softmax keeps one integer reference R per row, and a tile's
// weights are put under it by the scale operand, not by rescaling O: only a
// tile more than 2^16 above R moves it.  So no sum passes n_keys 2^16 max|v|: values
// up to 2^111 / n_keys cannot overflow (with 2^64, and weights of 256, it was 2^56 /
// n_keys; the times are the same).
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
//
// Bound, up to 64 rows, by the cache's bytes, the first tile and the merge (16
// rows, 32K keys of 8 heads, 67 MB: 17 us and the merge's 5; out of HBM 24.6 in
// all); above by the two waves per SIMD that its registers allow: products, vector
// work and LDS reads of a tile take about half of its time (1024 rows and heads, 64K
// keys: 54 us out of HBM, 15 of products and 16 of vector work).
// ---------------------------------------------------------------------------
constexpr int kTileKeys8 = 128;
constexpr int kTileBlocks = kTileKeys8 / kKv8Block;
constexpr float kRefGrow = 16.f;         // log2 growth that moves a row's reference
constexpr float kFarScore = 0x1p22f;     // |S sl2| whose fp32 spacing a weight would feel

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

// Four values of at most 256 (279 where S sl2 is near kFarScore and rounded by 1/8) as
// two e4m3 parts hi + lo / 16.
constexpr int kLoShift = 4;
__device__ __forceinline__ void two_parts(const float (&p)[4], uint32_t dead, uint32_t &hi,
                                          uint32_t &lo) {
    typedef short i16x2 __attribute__((ext_vector_type(2)));
    constexpr float kLo = 1.f / (1 << kLoShift);     // (the conversion divides by it)
    // (the old value of a conversion's result, half of which it keeps, is any
    // register that is free by then: a zero would have to be written first)
    int h = __builtin_amdgcn_cvt_pk_fp8_f32(p[0], p[1], (int)dead, false);
    h = __builtin_amdgcn_cvt_pk_fp8_f32(p[2], p[3], h, true);
    float f[4];
    e4m3x4_to_f32((uint32_t)h, f);
    const float r0 = p[0] - f[0];
    i16x2 l = __builtin_bit_cast(i16x2, f[0]);
    l = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(l, r0, p[1] - f[1], kLo, false);
    l = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(l, p[2] - f[2], p[3] - f[3], kLo, true);
    hi = (uint32_t)h;
    lo = __builtin_bit_cast(uint32_t, l);
}

// Largest of the values that the four lane groups hold for a row, in all of
// them.
__device__ __forceinline__ float row_max(float m) {
    typedef unsigned u32pair __attribute__((ext_vector_type(2)));
    u32pair r = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false,
                                                 false);
    m = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Waves: KS key streams x RG row groups of 16 rows; a stage of the ring holds
// one tile of each stream.  MANY: several workgroups for the rows of a split.
template <int D, int RG, int KS, int NBUF, bool MANY>
__global__ __launch_bounds__(64 * RG * KS) void attn8_tiles(Attn8Params a) {
    constexpr int HALF = kTileKeys8 * D;             // bytes of a K or V tile
    constexpr int TILE = 2 * HALF + 1024;            // codes, then 16 bytes around the scales
    constexpr int STAGE = KS * TILE;
    constexpr int LPH = HALF / 1024 / RG;            // a wave's loads of K, and of V, per tile
    constexpr int LPW = 2 * LPH + 1;                 // ... and of a stage, scales included
    constexpr int MD = D / 16;
    constexpr int VAHEAD = MD / 2;                   // values read before the softmax, in 16 dims
    constexpr int GRAN = D / 16;                     // 16-byte granules of a key
    constexpr int BLOCK = kKv8Block * D;             // bytes of a scale block
    constexpr int QBYTES = 16 * D * 2;               // a wave's rows of q
    constexpr int OST = D + 4;                       // padded fp32 row of the stream merge
    static_assert((NBUF - 1) * LPW < 64 && RG * KS * QBYTES <= STAGE, "ring");
    static_assert(NBUF * STAGE + 64 <= 160 * 1024, "LDS");
    static_assert(KS <= 2 && (KS == 1 || RG * 16 * OST * 4 + RG * 128 <= NBUF * STAGE), "merge");
    __shared__ __attribute__((aligned(1024))) char ring[NBUF * STAGE];

    // ---- which (kv head, split, row group) this workgroup owns ----------------
    int g = blockIdx.x, split = blockIdx.y, rgw = 0;
    if constexpr (MANY) {
        // the row groups of one (head, split) on one XCD, adjacent in its
        // dispatch order: all but the first find the tiles in its L2
        const int xcd = blockIdx.x & 7, w = blockIdx.x >> 3;
        rgw = w % a.n_row_groups;
        const int unit = (w / a.n_row_groups) * 8 + xcd;
        if (unit >= a.n_kv_heads * a.splits)
            return;
        g = unit % a.n_kv_heads;
        split = unit / a.n_kv_heads;
    }
    const int wave = wave_id();
    const int stream = wave % KS, rg = wave / KS;
    const int lane = threadIdx.x % kWave;
    const int m16 = lane & 15;
    const int c4 = lane >> 4;

    // the first splits take one tile more where they do not divide evenly
    const int t_first = split * a.tiles_per_split + min(split, a.extra_tiles);
    const int n_tiles = a.tiles_per_split + (split < a.extra_tiles ? 1 : 0);
    const int n_steps = (n_tiles + KS - 1) / KS;
    const int last_block = (a.n_keys - 1) / kKv8Block;
    const float sl2 = a.sl2;
    const size_t head = (size_t)g * a.n_blocks;
    const char *kg = a.k + head * BLOCK;
    const char *vg = a.v + head * BLOCK;
    const uintptr_t ksat = reinterpret_cast<uintptr_t>(a.k_scale + head);
    const uintptr_t vsat = reinterpret_cast<uintptr_t>(a.v_scale + head);
    const uintptr_t ksend = (ksat + last_block) & ~(uintptr_t)3;
    const uintptr_t vsend = (vsat + last_block) & ~(uintptr_t)3;

    // ---- the wave's 16 rows of q, by DMA into the stage that is filled last ------
    const int row = (rgw * RG + rg) * 16 + m16;
    auto token = [&](int r) { return a.group == 1 ? r : (int)__umulhi(r, a.group_magic); };
    {
        constexpr int LPR = D / 8;                   // lanes (16 bytes) per row
#pragma unroll
        for (int w = 0; w < QBYTES / 1024; ++w) {
            const int r = min((rgw * RG + rg) * 16 + (w * kWave + lane) / LPR, a.rows - 1);
            const int i = token(r);
            const int h = g * a.group + (r - i * a.group);
            lds_dma16(static_cast<const char *>(a.q) + ((size_t)i * a.n_q_heads + h) * (D * 2) +
                          lane % LPR * 16,
                      lds_addr(ring) + (NBUF - 1) * STAGE + wave * QBYTES + w * 1024);
        }
    }

    // Copies the stream's tile of stage st to buffer `buf`: 1 KB loads j of K and
    // of V, dealt out to the stream's waves.  A stream without a tile in the last
    // stage copies the one before again (never used), so that every wave counts
    // the same loads; a scale block past the last one repeats that block.
    unsigned koff, voff;
    {
        const int k = lane / GRAN;
        koff = (unsigned)(k * D + ((lane % GRAN) ^ (D == 128 ? k & 3 : k >> 1 & 1)) * 16);
        voff = (unsigned)(32 * (lane >> 1) + 16 * ((lane ^ (lane >> 3) ^ (lane >> 4)) & 1));
    }
    auto issue_tile = [&](int t, int slot_at) __attribute__((always_inline)) {
        const int b0 = (t_first + min(t, n_tiles - 1)) * kTileBlocks;
        const unsigned slot = lds_addr(ring) + slot_at + rg * 1024;
        const int most = last_block - b0;                // last block of the tile
        const char *kt = kg + (size_t)b0 * BLOCK, *vt = vg + (size_t)b0 * BLOCK;
        auto go = [&](auto ragged) __attribute__((always_inline)) {
#pragma unroll
            for (int jr = 0; jr < 2 * LPH; ++jr) {
                const bool is_v = jr >= LPH;
                const int j = rg + (jr % LPH) * RG;
                // (key bit 4 in a K granule's place: bit 1 of j, or 0 at head_dim 64)
                unsigned off = is_v ? voff
                                    : koff ^ (D == 128 ? (unsigned)(j & 2) << 5
                                                       : (unsigned)(j & 1) << 5);
                off += (unsigned)j * 1024u;
                if constexpr (decltype(ragged)::value) {
                    const int b = j * 1024 / BLOCK;
                    off -= (unsigned)(max(b - most, 0) * BLOCK);
                }
                lds_dma16_so(is_v ? vt : kt, off, slot + (is_v ? HALF : 0) + jr % LPH * RG * 1024);
            }
        };
        if (most >= kTileBlocks - 1)
            go(std::false_type{});
        else
            go(std::true_type{});
        // The scale bytes lie anywhere: lanes 0, 1 copy the two aligned dwords
        // that hold the tile's four K scales, lanes 2, 3 those of V, neither
        // past the dword of the last used byte (the other lanes repeat them).
        const uintptr_t at = (lane & 2 ? vsat : ksat) + b0;
        const uintptr_t from = min((at & ~(uintptr_t)3) + (lane & 1) * 4, lane & 2 ? vsend : ksend);
        lds_dma4(reinterpret_cast<const char *>(from), lds_addr(ring) + slot_at + 2 * HALF);
    };
    auto issue = [&](int st, int buf) __attribute__((always_inline)) {
        issue_tile(KS * st + stream, buf * STAGE + stream * TILE);
    };
#pragma unroll
    for (int st = 0; st < NBUF - 1; ++st)
        if (st < n_steps)
            issue(st, st);
    // Waits until all but the `later` stages issued last have landed.
    auto landed = [&](int later) __attribute__((always_inline)) {
        if (NBUF > 3 && later >= 3)
            wait_vmcnt<(NBUF > 3 ? 3 : 0) * LPW>();
        else if (NBUF > 2 && later >= 2)
            wait_vmcnt<(NBUF > 2 ? 2 : 0) * LPW>();
        else if (later >= 1)
            wait_vmcnt<LPW>();
        else
            wait_vmcnt<0>();
    };
    const int qi = token(min(row, a.rows - 1));
    const bool tree = a.tree_mask != nullptr;        // kernel argument: uniform
    constexpr int QW = D / 64;                       // 16-dim pieces of q per lane
    i32x8 qop[2];
    unsigned qscale, qlo;
    landed(min(NBUF - 1, n_steps));
    {
        const WF_LDS(char) *qp = (const WF_LDS(char) *)ring + (NBUF - 1) * STAGE + wave * QBYTES +
                                 m16 * (D * 2) + c4 * 32;
        float f[16 * QW];
        float m = 0.f;
#pragma unroll
        for (int w = 0; w < 2 * QW; ++w) {
            const u32x4 v = *(const WF_LDS(u32x4) *)(qp + (w / 2) * 128 + (w % 2) * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[8 * w + 2 * e] = __uint_as_float(v[e] << 16);
                f[8 * w + 2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
            }
        }
#pragma unroll
        for (int e = 0; e < 16 * QW; ++e)
            m = fmaxf(m, fabsf(f[e]));
        m = row_max(m);
        const int e = max((int)(__float_as_uint(m) >> 23) - 127 - 7, -120);
        const float inv = __uint_as_float((unsigned)(127 - e) << 23);
        qscale = (unsigned)(e + 127);
        qlo = qscale - kLoShift;
        uint32_t hi[4 * QW], lo[4 * QW];
#pragma unroll
        for (int w = 0; w < 4 * QW; ++w) {
            const float p[4] = {f[4 * w] * inv, f[4 * w + 1] * inv, f[4 * w + 2] * inv,
                                f[4 * w + 3] * inv};
            two_parts(p, __float_as_uint(f[4 * w]), hi[w], lo[w]);
        }
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

    // o[MD] collects the sum of the weights: one more 16-row block, of ones
    f32x4 o[MD + 1];
#pragma unroll
    for (int md = 0; md <= MD; ++md)
        o[md] = f32x4{0.f, 0.f, 0.f, 0.f};
    float ref = -INFINITY;

    const int kk0 = 16 * (m16 >> 2) + (m16 & 3);     // key of row m16 in block 0 of a half
    const int kf = D == 128 ? (kk0 & 3) | (kk0 >> 2 & 4) : (kk0 >> 1 & 1) | (kk0 >> 3 & 2);
    const int klane = kk0 * D + (c4 ^ kf) * 16;
    const int vlane = HALF + (c4 >> 1) * BLOCK + m16 * kKv8Block +
                      ((c4 ^ (m16 >> 2) ^ (m16 >> 3)) & 1) * 16;

    auto compute = [&](int t, int at) __attribute__((always_inline)) {
        const WF_LDS(char) *base = (const WF_LDS(char) *)ring + at;
        const int kb = (t_first + t) * kTileKeys8;
        // the scales of the tile's four token blocks in a dword each
        const WF_LDS(u32x4) *sp = (const WF_LDS(u32x4) *)(base + 2 * HALF);
        const u32x4 sw = *sp;
        // S^T = K Q^T, all operands asked for before the first is used
        i32x8 kop[8];
#pragma unroll
        for (int mb = 0; mb < 8; ++mb) {
            const int off = (64 * (mb >> 2) + 4 * (mb & 3)) * D;
            const u32x4 k0 = *(const WF_LDS(u32x4) *)(base + klane + off);
            if constexpr (D == 128)
                kop[mb] = join(k0, *(const WF_LDS(u32x4) *)(base + (klane ^ 64) + off));
            else
                kop[mb] = join(k0, k0);
        }
        __builtin_amdgcn_sched_barrier(0);
        const int b0 = kb / kKv8Block;
        unsigned ks4 = __builtin_amdgcn_alignbyte(sw[1], sw[0], (unsigned)(ksat + b0) & 3u);
        unsigned vs4 = __builtin_amdgcn_alignbyte(sw[3], sw[2], (unsigned)(vsat + b0) & 3u);
        // lane's scale of row m16 (token block m16 / 8 of either half) in bytes
        // 0 and 2; lane's scale of token block c4 (past the last one: 1)
        const unsigned ks = ks4 >> (8 * (m16 >> 3));
        const unsigned vs = b0 + c4 <= last_block ? vs4 >> (8 * c4) : 127u;
        f32x4 s[8];
        const f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int mb = 0; mb < 8; ++mb)
            s[mb] = mb < 4 ? mfma_e4m3<0, 0>(kop[mb], qop[0], z, ks, qscale)
                           : mfma_e4m3<2, 0>(kop[mb], qop[0], z, ks, qscale);
        if constexpr (D == 128) {
#pragma unroll
            for (int mb = 0; mb < 8; ++mb)
                s[mb] = mb < 4 ? mfma_e4m3<0, 0>(kop[mb], qop[1], s[mb], ks, qlo)
                               : mfma_e4m3<2, 0>(kop[mb], qop[1], s[mb], ks, qlo);
        }
        // the values of the first dims, on their way during the softmax
        u32x4 vop[MD][2];
        auto read_v = [&](int md) {
            const WF_LDS(char) *vr = base + vlane + md * 16 * kKv8Block;
            vop[md][0] = *(const WF_LDS(u32x4) *)vr;
            vop[md][1] = *(const WF_LDS(u32x4) *)(vr + 2 * BLOCK);
        };
#pragma unroll
        for (int md = 0; md < VAHEAD; ++md)
            read_v(md);
        __builtin_amdgcn_sched_barrier(0);
        // mask: only tiles that reach into the block.  Bit 16 h + b of `seen`:
        // the row sees key 64 h + 16 c4 + b of the tile.
        if (kb + kTileKeys8 > a.ctx_len) {
            uint64_t tm = 0;
            if (tree) {
                const uint64_t gbits = a.gamma >= 64 ? ~0ull : (1ull << a.gamma) - 1ull;
                tm = (a.tree_mask[qi] | (1ull << qi)) & gbits;
            }
            unsigned seen = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int j = kb + 64 * h + 16 * c4 - a.ctx_len;     // block row of bit 0
                unsigned bits;
                if (tree)                // keys before the block are seen by every row
                    bits = j >= 64 ? 0u : j >= 0 ? (unsigned)(tm >> j)
                           : j <= -16 ? ~0u : (unsigned)(tm << -j) | ((1u << -j) - 1u);
                else
                    bits = (1u << min(max(qi + 1 - j, 0), 16)) - 1u;
                seen |= (bits & 0xffffu) << (16 * h);
            }
#pragma unroll
            for (int mb = 0; mb < 8; ++mb)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    s[mb][i] = seen >> (4 * mb + i) & 1u ? s[mb][i] : -INFINITY;
        }
        float m = s[0][0];
#pragma unroll
        for (int mb = 0; mb < 8; ++mb)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                m = fmaxf(m, s[mb][i]);
        m = row_max(m);
        // the row's exponent in this tile, and against its reference
        const bool any = m > -INFINITY;
        const float e = any ? ceilf(m * sl2) : 0.f;
        const bool far = fabsf(e) >= kFarScore;
        float add = 8.f - e;
        if (__ballot(far || (any && !(e - ref <= kRefGrow)))) {
            // (also a row's first visible tile: ref is -inf, o zero)
            if (any && !(e - ref <= kRefGrow)) {
                const float back = fast_exp2(ref - e);
#pragma unroll
                for (int md = 0; md <= MD; ++md)
                    o[md] *= back;
                ref = e;
            }
            // m sl2 is rounded, a score's product below is not: from 2^24 on that
            // could put a weight at 2^9, past e4m3.  Such scores are taken from
            // their largest first, whose weight is then 2^8 exactly.
            if (far) {
#pragma unroll
                for (int mb = 0; mb < 8; ++mb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        s[mb][i] -= m;
                add = 8.f;
            }
        }
        const int shift = any ? (int)fmaxf(e - ref, -114.f) : 0;
        const unsigned ps = (unsigned)(127 - 8 + shift), pslo = ps - kLoShift;
        // P in two parts
        uint32_t hi[8], lo[8];
#pragma unroll
        for (int mb = 0; mb < 8; ++mb) {
            float p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                p[i] = fast_exp2(fmaf(s[mb][i], sl2, add));
            two_parts(p, __float_as_uint(s[mb][0]), hi[mb], lo[mb]);
        }
        const i32x8 ph = join(u32x4{hi[0], hi[1], hi[2], hi[3]}, u32x4{hi[4], hi[5], hi[6], hi[7]});
        const i32x8 pl = join(u32x4{lo[0], lo[1], lo[2], lo[3]}, u32x4{lo[4], lo[5], lo[6], lo[7]});
        // O^T += V^T P^T
        auto pv = [&](auto ragged) __attribute__((always_inline)) {
            constexpr int kOnes = 0x38383838;
            const i32x8 ones = {kOnes, kOnes, kOnes, kOnes, kOnes, kOnes, kOnes, kOnes};
            o[MD] = mfma_e4m3<0, 0>(ones, ph, o[MD], 127u, ps);
#pragma unroll
            for (int md = VAHEAD; md < MD; ++md)
                read_v(md);
#pragma unroll
            for (int md = 0; md < MD; ++md) {
                if constexpr (decltype(ragged)::value) {
                    // codes behind the last key may be NaN, and 0 * NaN is no zero
                    const int n0 = a.n_keys - kb - 16 * c4, n1 = n0 - 64;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const int x0 = min(max(n0 - 4 * w, 0), 4), x1 = min(max(n1 - 4 * w, 0), 4);
                        vop[md][0][w] &= (uint32_t)((1ull << (8 * x0)) - 1ull);
                        vop[md][1][w] &= (uint32_t)((1ull << (8 * x1)) - 1ull);
                    }
                }
                o[md] = mfma_e4m3<0, 0>(join(vop[md][0], vop[md][1]), ph, o[md], vs, ps);
            }
#pragma unroll
            for (int md = 0; md < MD; ++md)
                o[md] = mfma_e4m3<0, 0>(join(vop[md][0], vop[md][1]), pl, o[md], vs, pslo);
            o[MD] = mfma_e4m3<0, 0>(ones, pl, o[MD], 127u, pslo);
        };
        if (kb + kTileKeys8 > a.n_keys)
            pv(std::true_type{});
        else
            pv(std::false_type{});
    };

    // ---- the ring: up to NBUF - 1 stages in flight ----------------------------------
    int buf = 0;
#pragma unroll 1
    for (int st = 0; st < n_steps; ++st) {
        landed(min(NBUF - 2, n_steps - 1 - st));
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (st + NBUF - 1 < n_steps)
            issue(st + NBUF - 1, buf == 0 ? NBUF - 1 : buf - 1);
        const int t = KS * st + stream;
        if (t < n_tiles)
            compute(t, buf * STAGE + stream * TILE);
        buf = buf + 1 == NBUF ? 0 : buf + 1;
    }

    // ---- the two streams of a row, in stream 0's registers -------------------------
    float l = o[MD][0];                              // (all 16 rows of the block are alike)
    if constexpr (KS == 2) {
        __syncthreads();                 // the ring is free
        WF_LDS(float) *part = (WF_LDS(float) *)ring + rg * 16 * OST;
        WF_LDS(float) *ml = (WF_LDS(float) *)ring + RG * 16 * OST + rg * 32;
        if (stream == 1) {
#pragma unroll
            for (int md = 0; md < MD; ++md)
                *(WF_LDS(f32x4) *)(part + m16 * OST + md * 16 + 4 * c4) = o[md];
            if (c4 == 0) {
                ml[m16] = ref;
                ml[16 + m16] = l;
            }
        }
        __syncthreads();
        if (stream == 1)
            return;
        const float ref1 = ml[m16], top = fmaxf(ref, ref1);
        const float use = top == -INFINITY ? 0.f : top;
        const float f0 = fast_exp2(ref - use), f1 = fast_exp2(ref1 - use);
        l = l * f0 + ml[16 + m16] * f1;
#pragma unroll
        for (int md = 0; md < MD; ++md)
            o[md] = o[md] * f0 + *(WF_LDS(f32x4) *)(part + m16 * OST + md * 16 + 4 * c4) * f1;
        ref = top;
    }

    // ---- the split's partial ---------------------------------------------------------
    if (row >= a.rows)
        return;
    const size_t pr = ((size_t)split * a.gamma + qi) * a.n_q_heads + g * a.group +
                      (row - qi * a.group);
    // Partial rows stay fp32: rounded to bf16 they would bring the merged row as
    // large an error again as its own rounding (from 64 bits 0.0024 of the output,
    // 0.0017 as it is; 16 rows, 8K keys: 13.7 us, 13.9 as it is).  More than 32 rows'
    // go past the L2, from which the merge, on another XCD, would have to fetch them
    // while the next call's are written in their place (one workspace: 64 rows, 8K
    // keys 15.1 us, 13.9 past it; 244 rows 26.3 and 22.2; 32 rows, 1K keys 8.5 and 8.7,
    // so not for those).
    if (a.splits > 1) {
        f32x4 *dst = reinterpret_cast<f32x4 *>(static_cast<float *>(a.ws_o) + pr * D) + c4;
#pragma unroll
        for (int md = 0; md < MD; ++md) {
            if constexpr (RG == 4)
                __builtin_nontemporal_store(o[md], dst + 4 * md);
            else
                dst[4 * md] = o[md];
        }
        if (c4 == 0) {
            a.ws_ml[pr * 2] = ref;
            a.ws_ml[pr * 2 + 1] = l;
        }
        return;
    }
    // One split: the output (every row sees itself: l > 0).  Lane groups 2i and
    // 2i + 1 hold 4 dims each of every 16; they trade, so that the first has 8 of the
    // even 16s and the second 8 of the odd ones: 16-byte stores, 64 bytes of a row
    // together.
    const float inv = 1.f / l;
    u32x4 *dst = reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.ws_o) + pr * D);
#pragma unroll
    for (int md = 0; md < MD; md += 2) {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const auto r = __builtin_amdgcn_permlane16_swap(
                pack_bf16x2(o[md][2 * i] * inv, o[md][2 * i + 1] * inv),
                pack_bf16x2(o[md + 1][2 * i] * inv, o[md + 1][2 * i + 1] * inv), false, false);
            v[i] = r[0];
            v[2 + i] = r[1];
        }
        dst[(md + (c4 & 1)) * 2 + (c4 >> 1)] = v;
    }
}

// ---------------------------------------------------------------------------
// fp32 queries: a workgroup per (split, row, head), fp32 throughout.  Its eight
// waves take 64 keys, two scale blocks, at a time, each with a softmax of its
// own: lane t forms key t's score from its code row, then lane d adds the
// weighted values of dim d (one or two per lane), whose codes lie together in
// the transposed V blocks.  The waves meet once, in LDS.  A step is one trip to
// memory: both blocks' codes and scales are asked for before any is used (one
// wave of 64 keys, each operand loaded where it is needed: 8 rows, 8 heads,
// 264 keys 6.8 us; now 3.7).  Bound by its launch at such sizes, by the
// conversions and products in fp32 at 4K keys (8 rows, 32 heads: 25.5 us).
// ---------------------------------------------------------------------------
// Orders a wave's LDS accesses before and after it.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

constexpr int kRowWaves = 8;
constexpr int kRowKeys = kRowWaves * kWave;          // keys of a workgroup's step

template <int D>
__global__ __launch_bounds__(64 * kRowWaves) void attn8_rows(Attn8Params a) {
    constexpr int E = D / kWave;
    __shared__ float qs[D];
    __shared__ float ps_all[kRowWaves][kWave];
    __shared__ float acc_all[kRowWaves][D], ml[kRowWaves][2];
    const int split = blockIdx.x;
    const int pr = blockIdx.y;           // i * n_q_heads + h
    const int i = pr / a.n_q_heads, h = pr % a.n_q_heads;
    const int g = h / a.group;
    const int wave = wave_id(), lane = threadIdx.x % kWave;
    float *ps = ps_all[wave];
    if (threadIdx.x < D)
        qs[threadIdx.x] = static_cast<const float *>(a.q)[(size_t)pr * D + threadIdx.x];
    __syncthreads();

    const int first = split * a.tiles_per_split + min(split, a.extra_tiles);
    const int steps = a.tiles_per_split + (split < a.extra_tiles ? 1 : 0);
    const int k_begin = first * kRowKeys;
    const bool tree = a.tree_mask != nullptr;
    const uint64_t gbits = a.gamma >= 64 ? ~0ull : (1ull << a.gamma) - 1ull;
    const uint64_t tm = tree ? ((a.tree_mask[i] | (1ull << i)) & gbits) : 0ull;
    const int k_end = min(min(a.n_keys, k_begin + steps * kRowKeys),
                          tree ? a.n_keys : a.ctx_len + i + 1);
    const size_t head = (size_t)g * a.n_blocks;

    float m = -INFINITY, l = 0.f, acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e)
        acc[e] = 0.f;
    for (int kb = k_begin + wave * kWave; kb < k_end; kb += kRowKeys) {
        const int j = kb + lane;
        const int jb = j - a.ctx_len;
        const bool vis = j < k_end && (!tree || jb < 0 || ((tm >> jb) & 1ull));
        const uint64_t seen = __ballot(vis);
        // the step's codes and scales at once (past the last key: that key's)
        const int jr = min(j, k_end - 1);
        const size_t kblk = head + jr / kKv8Block;
        const u32x4 *kr = reinterpret_cast<const u32x4 *>(
            a.k + (kblk * kKv8Block + jr % kKv8Block) * D);
        u32x4 kw[D / 16], vw[2][E][2];
        unsigned vs[2];
        const unsigned ks = a.k_scale[kblk];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const size_t blk = head + min(kb / kKv8Block + b, (k_end - 1) / kKv8Block);
            vs[b] = a.v_scale[blk];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const u32x4 *vr = reinterpret_cast<const u32x4 *>(
                    a.v + (blk * D + lane + e * kWave) * kKv8Block);
                vw[b][e][0] = vr[0];
                vw[b][e][1] = vr[1];
            }
        }
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
            kw[c] = kr[c];
        float dot = 0.f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                float f[4];
                e4m3x4_to_f32(kw[c][u], f);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    dot = fmaf(qs[16 * c + 4 * u + e], f[e], dot);
            }
        if (seen == 0)                   // uniform: nothing of this step counts
            continue;
        const float sc = vis ? dot * scale_value((uint8_t)ks) : -INFINITY;
        const float mnew = fmaxf(m, wave_max(sc));
        const float alpha = (m == -INFINITY) ? 0.f : exp2f((m - mnew) * a.sl2);
        const float p = vis ? exp2f((sc - mnew) * a.sl2) : 0.f;
        l = fmaf(l, alpha, wave_sum(p));
        m = mnew;
        ps[lane] = p;
#pragma unroll
        for (int e = 0; e < E; ++e)
            acc[e] *= alpha;
        wave_sync();
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const unsigned live = (unsigned)(seen >> (32 * b));
            float sum[E] = {};
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                // codes that the row does not see may be NaN: zeros instead
                const unsigned bytes =
                    ((live >> (4 * u) & 15u) * 0x00204081u & 0x01010101u) * 255u;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    float f[4];
                    e4m3x4_to_f32(vw[b][e][u / 4][u % 4] & bytes, f);
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        sum[e] = fmaf(ps[32 * b + 4 * u + t], f[t], sum[e]);
                }
            }
            const float s = live ? scale_value((uint8_t)vs[b]) : 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e)
                acc[e] = fmaf(sum[e], s, acc[e]);
        }
        wave_sync();
    }
    // the waves' parts under the largest reference; a wave without a key adds 0
#pragma unroll
    for (int e = 0; e < E; ++e)
        acc_all[wave][lane + e * kWave] = acc[e];
    if (lane == 0) {
        ml[wave][0] = m;
        ml[wave][1] = l;
    }
    __syncthreads();
    if (threadIdx.x >= D)
        return;
    float top = ml[0][0];
#pragma unroll
    for (int w = 1; w < kRowWaves; ++w)
        top = fmaxf(top, ml[w][0]);
    float sum = 0.f, out = 0.f;
#pragma unroll
    for (int w = 0; w < kRowWaves; ++w) {
        const float f = ml[w][0] == -INFINITY ? 0.f : exp2f((ml[w][0] - top) * a.sl2);
        sum = fmaf(ml[w][1], f, sum);
        out = fmaf(acc_all[w][threadIdx.x], f, out);
    }
    const size_t prs = (size_t)split * a.gamma * a.n_q_heads + pr;
    // (of one split: every row sees itself, sum > 0)
    static_cast<float *>(a.ws_o)[prs * D + threadIdx.x] = a.splits == 1 ? out / sum : out;
    if (threadIdx.x == 0 && a.splits > 1) {
        a.ws_ml[prs * 2] = top * a.sl2;
        a.ws_ml[prs * 2 + 1] = sum;
    }
}

}  // namespace

// Split plan of a call (figures: three caches in turn, one workspace, in a graph).
// bf16: up to 64 rows share a workgroup's tiles, two key streams of up to four 16-row
// waves, one workgroup per CU; of more rows each 64 take a workgroup of one stream, two
// per CU, which do not wait for each other's barriers (244 rows, 8K keys: 21.7 us, 23.8
// with 128 rows to a workgroup of eight waves; 128 rows, 8K 16.9 and 18.0, 64K 59 both
// ways).  No workgroup is without a tile.  Where each has few, one stream, whose first
// stage is there sooner and which has nothing to join at its end (one stream and two,
// us: 32 rows, 1K keys 8.4 and 9.3, 8K 12.8 and 13.2, 32K 21.1 and 19.7; 64 rows, 1K 9.5
// and 11.4, 8K 13.8 and 15.6, 32K 22.9 and 23.4, 64K 39.9 and 39.7, 128K 69.2 and 64.7).
// The fewest stay one split, whose workgroup writes the output and spares the merge: up
// to two steps (32 rows, 500 keys: 7.6 us, 8.2 as four splits), or one of 64 rows,
// whose steps take twice as long (256 keys: 6.9 us, 8.8 as two; 516 keys: 12.1 as one,
// 9.4 as five).  fp32: splits only where the rows leave CUs idle (256 rows and heads,
// 2K keys: 16.9 us, 18.6 as four; 32, 4K keys: 27.9 and 9.6 as eight).
AttnPlan plan_attn8(wf_dtype_t dt, int gamma, int ctx_len, int n_q_heads, int n_kv_heads,
                    int head_dim, int num_splits) {
    AttnPlan p{};
    p.part_bytes = 4;
    if (dt == WF_F32) {
        const int steps = (ctx_len + gamma + kRowKeys - 1) / kRowKeys;
        const int want = num_splits > 0 ? num_splits
                         : steps <= 2   ? 1
                                        : std::max(1, 256 / (gamma * n_q_heads));
        p.splits = std::min(want, steps);
        return p;
    }
    p.rows = n_q_heads / n_kv_heads * gamma;
    p.nb = 1;
    p.rg = p.rows <= 16 ? 1 : p.rows <= 32 ? 2 : 4;
    p.ks = p.rows <= 64 ? 2 : 1;
    p.n_row_groups = (p.rows + 16 * p.rg - 1) / (16 * p.rg);
    const int tiles = (ctx_len + gamma + kTileKeys8 - 1) / kTileKeys8;
    const int fill = p.ks == 2 ? 256 : 512;
    const int want = num_splits > 0 ? num_splits
                                    : std::max(1, fill / (n_kv_heads * p.n_row_groups));
    p.splits = std::min(want, tiles);
    if (num_splits == 0 && tiles <= (p.rg == 4 ? 1 : 2) * p.ks)
        p.splits = 1;
    const int each = (tiles + p.splits - 1) / p.splits;
    if (p.splits == 1 ? each == 1 : each <= (p.rg == 4 ? 12 : 3))
        p.ks = 1;
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
    if (p.splits == 1)
        a.ws_o = out;
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
    a.n_row_groups = p.n_row_groups;
    a.sl2 = softmax_scale * kLog2e;
    const int unit = dt == WF_BF16 ? kTileKeys8 : kRowKeys;
    const int tiles = (a.n_keys + unit - 1) / unit;
    a.tiles_per_split = tiles / p.splits;
    a.extra_tiles = tiles % p.splits;
    if (dt == WF_BF16) {
        // (exact for rows below 2^14 in groups of 2 to 2^8)
        a.group_magic = (unsigned)((1ull << 32) / a.group + 1);
        const int units = c.n_kv_heads * p.splits;
        const bool many = p.n_row_groups > 1;
        const dim3 grid = many ? dim3((units + 7) / 8 * 8 * p.n_row_groups)
                                             : dim3(c.n_kv_heads, p.splits);
#define WF_ATTN8(DV, RGV, KSV, NBUFV, MANYV)                                               \
    if (c.head_dim == DV && p.rg == RGV && p.ks == KSV && many == MANYV)                   \
        attn8_tiles<DV, RGV, KSV, NBUFV, MANYV><<<grid, 64 * RGV * KSV, 0, stream>>>(a);   \
    else
        WF_ATTN8(128, 1, 2, 2, false) WF_ATTN8(128, 2, 2, 2, false) WF_ATTN8(128, 4, 2, 2, false)
        WF_ATTN8(128, 1, 1, 2, false) WF_ATTN8(128, 2, 1, 2, false) WF_ATTN8(128, 4, 1, 2, false)
        WF_ATTN8(128, 4, 1, 2, true)
        WF_ATTN8(64, 1, 2, 2, false) WF_ATTN8(64, 2, 2, 4, false) WF_ATTN8(64, 4, 2, 4, false)
        WF_ATTN8(64, 1, 1, 2, false) WF_ATTN8(64, 2, 1, 2, false) WF_ATTN8(64, 4, 1, 4, false)
        WF_ATTN8(64, 4, 1, 4, true)
        return WF_ERR_UNSUPPORTED;
#undef WF_ATTN8
    } else {
        const dim3 grid(p.splits, (unsigned)pairs);
        if (c.head_dim == 128)
            attn8_rows<128><<<grid, 64 * kRowWaves, 0, stream>>>(a);
        else
            attn8_rows<64><<<grid, 64 * kRowWaves, 0, stream>>>(a);
    }
    if (hipGetLastError() != hipSuccess)
        return WF_ERR_HIP;
    if (p.splits == 1)
        return WF_OK;
    // (the references are held in log2 units, so the merge's factor is 1)
    return launch_attn_merge(c.head_dim, false, dt == WF_BF16, a.ws_o, a.ws_ml, out, (int)pairs,
                             p.splits, 1.f, stream);
}

}  // namespace wf
