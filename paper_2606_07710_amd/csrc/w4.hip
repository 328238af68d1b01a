// w4.hip -- products with 4-bit weights (e2m1 codes, one power-of-two scale
// byte per 32 inputs of a row) for a few rows x, the quantiser that makes such a
// weight, and the packing into the tiles that the products stream.
//
// y = W x streams 17/32 of a byte per weight.  The codes become bf16 in
// registers, scale included, in one conversion per two weights (exact: at most
// two mantissa bits), and meet x in 16x16x32 bf16 MFMAs, so the products are
// exact and the sums fp32, in a fixed order.  Two kernels: one splits the input
// over a workgroup's waves (few features: every CU gets some, all loads at once),
// one the features (many: x is read from memory once per workgroup and from LDS
// after that).
#include "wf_api_internal.h"
#include "wf_lowbit.h"

namespace wf {

namespace {

#ifdef NT
#define LOADW(p) __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p))
#else
#define LOADW(p) (*reinterpret_cast<const u32x4 *>(p))
#endif
#ifndef WIDE_FROM
#define WIDE_FROM 6
#endif
constexpr int kW4Waves = 8;
constexpr int kW4Group = 32;             // inputs per scale
constexpr int kW4Chunk = 128;            // inputs per tile: 16 bytes of codes per lane
constexpr int kW4Tile = 1024 + 64;       // 16 features x 128 inputs: codes, then scales

// Scale byte -> the float that the conversion multiplies by (255: NaN).
__device__ __forceinline__ float w4_scale(unsigned s) {
    return s == 255u ? __uint_as_float(0x7fc00000u) : scale_value(s);
}

// Eight codes (one dword, low nibble first) times their scale as an MFMA
// operand's eight bf16.
__device__ __forceinline__ bf16x8 w4_expand(uint32_t w, float s) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3);
    return bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// The sum of `n` waves' partial blocks, the residual, and the store.
template <bool F32OUT>
__device__ __forceinline__ void store_y(void *y, const uint16_t *res, size_t at, float z) {
    if (res)
        z += bf16_to_f32(res[at]);
    if constexpr (F32OUT)
        static_cast<float *>(y)[at] = z;
    else
        static_cast<uint16_t *>(y)[at] = f32_to_bf16(z);
}

// Input split: workgroup b owns FB blocks of 16 features and the whole input,
// its 8 waves take interleaved 128-input chunks, U of them loaded at once, and
// their sums meet in LDS in wave order.  NB 16-row blocks of x.  Lane (m16, c4)
// holds, for chunk c, the 32 inputs 128c + 32*c4 .. +31 (one scale group) of
// feature m16 of each block and of x row m16; MFMA kk takes the kk-th eight of
// them on both sides.
template <int NB, int FB, bool F32OUT>
__global__ __launch_bounds__(kW4Waves * kWave) void linear_w4(
    const uint16_t *__restrict__ x, const uint8_t *__restrict__ w, const uint16_t *res, void *y,
    int rows, int n_out, int k_in) {
    constexpr int U = FB * NB == 1 ? 4 : FB * NB <= 4 ? 2 : 1;
    __shared__ float zs[kW4Waves][16][16 * NB + 1];
    const int f0 = 16 * FB * blockIdx.x;
    const int wave = wave_id();
    const int lane = threadIdx.x % kWave;
    const int m16 = lane & 15;
    const int c4 = lane >> 4;
    const int n_c = (k_in + kW4Chunk - 1) / kW4Chunk;
    const int last_g = k_in / kW4Group - 1;
    // (a workgroup of the last blocks reads the last one again for those past it)
    const uint8_t *wp[FB];
#pragma unroll
    for (int fb = 0; fb < FB; ++fb)
        wp[fb] = w + (size_t)min(FB * (int)blockIdx.x + fb, (n_out + 15) / 16 - 1) * n_c * kW4Tile;
    // rows past the end read the last one; they are not stored
    const uint16_t *xp[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
        xp[nb] = x + (size_t)min(16 * nb + m16, rows - 1) * k_in;
    f32x4 acc[FB][NB];
#pragma unroll
    for (int fb = 0; fb < FB; ++fb)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
            acc[fb][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
    struct Batch {
        u32x4 w[U][FB];
        unsigned s[U][FB];
        bf16x8 x[U][NB][4];
    };
    auto load = [&](Batch &q, int cb) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = min(cb + kW4Waves * u, n_c - 1);
#pragma unroll
            for (int fb = 0; fb < FB; ++fb) {
                const uint8_t *t = wp[fb] + (size_t)c * kW4Tile;
                q.w[u][fb] = LOADW(t + lane * 16);
                q.s[u][fb] = t[1024 + lane];
            }
            // (inputs past the end: the row's last ones, against zero codes)
            const int g = min(4 * c + c4, last_g);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                    q.x[u][nb][kk] = load_bf16x8(xp[nb] + g * kW4Group + 8 * kk);
        }
    };
    auto multiply = [&](const Batch &q, int cb) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (cb + kW4Waves * u >= n_c)            // uniform
                break;
#pragma unroll
            for (int fb = 0; fb < FB; ++fb) {
                const float sf = w4_scale(q.s[u][fb]);
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) {
                    const bf16x8 wo = w4_expand(q.w[u][fb][kk], sf);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
                        acc[fb][nb] = mfma16x16x32(wo, q.x[u][nb][kk], acc[fb][nb]);
                }
            }
        }
    };
    // the next batch is on its way while one is multiplied
    constexpr int STEP = kW4Waves * U;
    Batch even, odd;
    load(even, wave);
    for (int cb = wave; cb < n_c; cb += 2 * STEP) {
        if (cb + STEP < n_c)
            load(odd, cb + STEP);
        multiply(even, cb);
        if (cb + 2 * STEP < n_c)
            load(even, cb + 2 * STEP);
        if (cb + STEP < n_c)
            multiply(odd, cb + STEP);
    }
#pragma unroll
    for (int fb = 0; fb < FB; ++fb) {
        if (fb)
            __syncthreads();
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                zs[wave][4 * c4 + i][16 * nb + m16] = acc[fb][nb][i];
        __syncthreads();
        for (int idx = threadIdx.x; idx < 16 * rows; idx += kW4Waves * kWave) {
            const int u = idx % 16, r = idx / 16, f = f0 + 16 * fb + u;
            if (f >= n_out)
                continue;
            float z = zs[0][u][r];
#pragma unroll
            for (int w = 1; w < kW4Waves; ++w)
                z += zs[w][u][r];
            store_y<F32OUT>(y, res, (size_t)r * n_out + f, z);
        }
    }
}

// Feature split: a workgroup's 8 waves own up to FB blocks of 16 features each,
// all rows, and walk the input together in chunks of 256, whose x is staged in
// LDS (a wave reads it once for all its blocks) while the next chunk's codes and
// x are on their way to registers.  Lanes and tiles as above.  The staged x is swizzled in 16-byte granules, g ^ (row & 7), so eight
// rows' reads meet distinct banks.
constexpr int kW4Wide = 256;

template <int NB, int FB, bool F32OUT>
__global__ __launch_bounds__(kW4Waves * kWave) void linear_w4_wide(
    const uint16_t *__restrict__ x, const uint8_t *__restrict__ w, const uint16_t *res, void *y,
    int rows, int n_out, int k_in) {
    constexpr int GRAN = kW4Wide / 8;                // 16-byte granules of a row's chunk
    __shared__ u32x4 xs[2][16 * NB * GRAN];
    const int wave = wave_id();
    const int lane = threadIdx.x % kWave;
    const int m16 = lane & 15;
    const int c4 = lane >> 4;
    const int n_t = (k_in + kW4Chunk - 1) / kW4Chunk, n_c = (n_t + 1) / 2;
    // blocks dealt out evenly over all waves of the launch
    const int blocks = (n_out + 15) / 16;
    const int waves = gridDim.x * kW4Waves, id = blockIdx.x * kW4Waves + wave;
    const int b_first = (int)((long long)id * blocks / waves);
    const int n_b = (int)((long long)(id + 1) * blocks / waves) - b_first;

    const uint8_t *wp[FB];
#pragma unroll
    for (int fb = 0; fb < FB; ++fb)      // (without an fb-th block: its last one again)
        wp[fb] = w + (size_t)min(b_first + min(fb, max(n_b - 1, 0)), blocks - 1) * n_t * kW4Tile;
    f32x4 acc[FB][NB];
#pragma unroll
    for (int fb = 0; fb < FB; ++fb)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
            acc[fb][nb] = f32x4{0.f, 0.f, 0.f, 0.f};

    struct Codes {
        u32x4 w[FB][2];
        unsigned s[FB][2];
    };
    auto load_w = [&](Codes &c, int ch) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int fb = 0; fb < FB; ++fb) {
                const uint8_t *t = wp[fb] + (size_t)min(2 * ch + h, n_t - 1) * kW4Tile;
                c.w[fb][h] = LOADW(t + lane * 16);
                c.s[fb][h] = t[1024 + lane];
            }
    };
    // x of a chunk: NB granules per thread (row past the end: the last row; a
    // granule past the input's end: the row's last, which meets zero codes)
    u32x4 xr[NB];
    auto load_x = [&](int ch) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int idx = threadIdx.x + j * kW4Waves * kWave;
            const int r = idx / GRAN, g = idx % GRAN;
            const int k = min(ch * GRAN + g, k_in / 8 - 1) * 8;
            xr[j] = *reinterpret_cast<const u32x4 *>(x + (size_t)min(r, rows - 1) * k_in + k);
        }
    };
    auto stage_x = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int idx = threadIdx.x + j * kW4Waves * kWave;
            const int r = idx / GRAN, g = idx % GRAN;
            xs[buf][r * GRAN + (g ^ (r & 7))] = xr[j];
        }
    };
    // every wave's LDS writes are done; loads in flight stay so
    auto barrier = [] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

    // One chunk: its codes are in `now`; the next one's go to `next`.
    auto step = [&](const Codes &now, Codes &next, int ch) __attribute__((always_inline)) {
        const int chn = min(ch + 1, n_c - 1);        // (the last chunk again: not used)
        load_x(chn);
        load_w(next, chn);
        const u32x4 *xb = xs[ch & 1];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (2 * ch + h >= n_t)                   // uniform
                break;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                bf16x8 xo[NB];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const int r = 16 * nb + m16, g = 16 * h + 4 * c4 + kk;
                    xo[nb] = __builtin_bit_cast(bf16x8, xb[r * GRAN + (g ^ (r & 7))]);
                }
#pragma unroll
                for (int fb = 0; fb < FB; ++fb) {
                    const bf16x8 wo = w4_expand(now.w[fb][h][kk], w4_scale(now.s[fb][h]));
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
                        acc[fb][nb] = mfma16x16x32(wo, xo[nb], acc[fb][nb]);
                }
            }
        }
        stage_x((ch + 1) & 1);
        barrier();
    };
    Codes even, odd;
    load_x(0);
    load_w(even, 0);
    stage_x(0);
    barrier();
    for (int ch = 0; ch < n_c; ch += 2) {
        step(even, odd, ch);
        if (ch + 1 < n_c)
            step(odd, even, ch + 1);
    }
    // lane (m16, c4) holds features 4*c4 .. +3 of row m16
#pragma unroll
    for (int fb = 0; fb < FB; ++fb) {
        if (fb >= n_b)
            break;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int r = 16 * nb + m16, f = 16 * (b_first + fb) + 4 * c4;
            if (r >= rows)
                continue;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (f + i < n_out)
                    store_y<F32OUT>(y, res, (size_t)r * n_out + f + i, acc[fb][nb][i]);
        }
    }
}

// Nearest e2m1 code of |a| <= 6, ties to the even code.
__device__ __forceinline__ unsigned e2m1_code(float x) {
    const float a = fabsf(x);
    const unsigned c = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) +
                       (a >= 3.5f) + (a > 5.f);
    return c | (__float_as_uint(x) >> 31 << 3);
}

// One group of 32 per thread.
__global__ __launch_bounds__(256) void w4_quantize(const uint16_t *__restrict__ w,
                                                   uint8_t *__restrict__ codes,
                                                   uint8_t *__restrict__ scales, size_t n) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n)
        return;
    u32x4 v[4];
    float m = 0.f;
    bool fine = true;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        v[u] = reinterpret_cast<const u32x4 *>(w)[4 * i + u];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float lo = fabsf(__uint_as_float(v[u][j] << 16));
            const float hi = fabsf(__uint_as_float(v[u][j] & 0xffff0000u));
            fine = fine && lo < INFINITY && hi < INFINITY;
            m = fmaxf(m, fmaxf(lo, hi));
        }
    }
    const int e = scale_exponent<0x400000u, 2>(m);       // 6 = 1.5 * 2^2
    const float inv = __uint_as_float((unsigned)(127 - e) << 23);
    u32x4 o;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        unsigned d = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            d |= (e2m1_code(__uint_as_float(v[u][j] << 16) * inv) |
                  e2m1_code(__uint_as_float(v[u][j] & 0xffff0000u) * inv) << 4)
                 << (8 * j);
        o[u] = d;
    }
    reinterpret_cast<u32x4 *>(codes)[i] = o;
    scales[i] = fine ? (uint8_t)(e + 127) : (uint8_t)255;
}

// Tile (block b, chunk c) of the packed weight: lane m16 + 16 * c4 of a wave
// finds its 16 bytes of codes (feature 16b + m16, inputs 128c + 32*c4 .. +31) at
// 16 * lane and their scale at 1024 + lane.  One wave per tile; features and
// inputs past the end are zeros under scale 1.
__global__ __launch_bounds__(kWave) void w4_pack(const uint8_t *__restrict__ codes,
                                                 const uint8_t *__restrict__ scales, int rows,
                                                 int groups, uint8_t *__restrict__ packed) {
    const int lane = threadIdx.x, m16 = lane & 15, c4 = lane >> 4;
    const int n_c = (groups + 3) / 4;
    const size_t tile = blockIdx.x;
    const size_t f = tile / n_c * 16 + m16;
    const int g = (int)(tile % n_c) * 4 + c4;
    u32x4 v = {0u, 0u, 0u, 0u};
    uint8_t s = 127;
    if (f < (size_t)rows && g < groups) {
        v = reinterpret_cast<const u32x4 *>(codes)[f * groups + g];
        s = scales[f * groups + g];
    }
    uint8_t *t = packed + tile * kW4Tile;
    reinterpret_cast<u32x4 *>(t)[lane] = v;
    t[1024 + lane] = s;
}

}  // namespace

size_t w4_packed_bytes(int rows, int cols) {
    return (size_t)((rows + 15) / 16) * ((cols + kW4Chunk - 1) / kW4Chunk) * kW4Tile;
}

wf_status_t launch_w4_pack(const void *codes, const uint8_t *scales, int rows, int cols,
                           void *packed, hipStream_t stream) {
    const size_t tiles = w4_packed_bytes(rows, cols) / kW4Tile;
    w4_pack<<<(unsigned)tiles, kWave, 0, stream>>>(static_cast<const uint8_t *>(codes), scales,
                                                   rows, cols / kW4Group,
                                                   static_cast<uint8_t *>(packed));
    return hipGetLastError() == hipSuccess ? WF_OK : WF_ERR_HIP;
}

size_t linear_w4_workspace_bytes(int rows, int n_out, int k_in) { return 0; }

wf_status_t launch_linear_w4(const uint16_t *x, const uint8_t *w, const uint16_t *res,
                             bool f32_out, void *y, int rows, int n_out, int k_in,
                             void *workspace, hipStream_t stream) {
    const int blocks = (n_out + 15) / 16;
    const dim3 block(kW4Waves * kWave);
    const int nb = (rows + 15) / 16;
    if (blocks > WIDE_FROM * 256) {
        const int per = kW4Waves * 256;              // waves of one workgroup per CU
        const int rounds = (blocks + 5 * per - 1) / (5 * per);
        const int fb = (blocks + rounds * per - 1) / (rounds * per);
        const dim3 grid(rounds * 256);
#define WF_W4(NBV, FBV)                                                                      \
    if (nb == NBV && fb == FBV) {                                                            \
        if (f32_out)                                                                         \
            linear_w4_wide<NBV, FBV, true><<<grid, block, 0, stream>>>(                      \
                x, w, res, y, rows, n_out, k_in);                                \
        else                                                                                 \
            linear_w4_wide<NBV, FBV, false><<<grid, block, 0, stream>>>(                     \
                x, w, res, y, rows, n_out, k_in);                                \
    } else
#define WF_W4_ROW(NBV) WF_W4(NBV, 1) WF_W4(NBV, 2) WF_W4(NBV, 3) WF_W4(NBV, 4) WF_W4(NBV, 5)
        WF_W4_ROW(1) WF_W4_ROW(2) WF_W4_ROW(3) WF_W4_ROW(4)
        { return WF_ERR_UNSUPPORTED; }
#undef WF_W4_ROW
#undef WF_W4
        return hipGetLastError() == hipSuccess ? WF_OK : WF_ERR_HIP;
    }
    // rounds of one workgroup per CU, and as few blocks each as that takes
    const int fb = (blocks + 255) / 256 <= 4 ? (blocks + 255) / 256 : 6;
    const dim3 grid((blocks + fb - 1) / fb);
#define WF_W4(NBV, FBV)                                                                      \
    if (nb == NBV && fb == FBV) {                                                            \
        if (f32_out)                                                                         \
            linear_w4<NBV, FBV, true><<<grid, block, 0, stream>>>(x, w, res, y, rows, n_out, k_in); \
        else                                                                                 \
            linear_w4<NBV, FBV, false><<<grid, block, 0, stream>>>(x, w, res, y, rows, n_out, k_in); \
    } else
#define WF_W4_ROW(NBV) WF_W4(NBV, 1) WF_W4(NBV, 2) WF_W4(NBV, 3) WF_W4(NBV, 4) WF_W4(NBV, 6)
    WF_W4_ROW(1) WF_W4_ROW(2) WF_W4_ROW(3) WF_W4_ROW(4)
    { return WF_ERR_UNSUPPORTED; }
#undef WF_W4_ROW
#undef WF_W4
    return hipGetLastError() == hipSuccess ? WF_OK : WF_ERR_HIP;
}

wf_status_t launch_w4_quantize(const void *w, int rows, int cols, void *codes, uint8_t *scales,
                               hipStream_t stream) {
    const size_t n = (size_t)rows * (cols / kW4Group);
    w4_quantize<<<(unsigned)((n + 255) / 256), 256, 0, stream>>>(
        static_cast<const uint16_t *>(w), static_cast<uint8_t *>(codes), scales, n);
    return hipGetLastError() == hipSuccess ? WF_OK : WF_ERR_HIP;
}

}  // namespace wf
