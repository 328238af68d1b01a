// w4.hip -- products with 4-bit weights (e2m1 codes, one power-of-two scale
// byte per 32 inputs of a row) for a few rows x, and the quantiser that makes
// such a weight.
//
// y = W x streams 17/32 of a byte per weight.  The codes become bf16 in
// registers, scale included, in one conversion per two weights (exact: at most
// two mantissa bits), and meet x in 16x16x32 bf16 MFMAs, so the products are
// exact and the sums fp32.  A workgroup owns 16 output features and the whole
// input; its 8 waves take interleaved 128-input chunks and their sums meet in
// LDS in wave order.
#include "wf_api_internal.h"
#include "wf_lowbit.h"

namespace wf {

namespace {

constexpr int kW4Waves = 8;
constexpr int kW4Group = 32;             // inputs per scale
constexpr int kW4Chunk = 128;            // inputs per wave load: 16 bytes of codes per lane

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

// NB 16-row blocks of x.  Lane (m16, c4) of a wave holds, for chunk c, the 32
// inputs 128c + 32*c4 .. +31 of feature m16 (one scale group) and of x row
// m16; MFMA kk takes the kk-th eight of them on both sides.
template <int NB, bool F32OUT>
__global__ __launch_bounds__(kW4Waves * kWave) void linear_w4(
    const uint16_t *__restrict__ x, const uint8_t *__restrict__ codes,
    const uint8_t *__restrict__ scales, const uint16_t *res, void *y, int rows, int n_out,
    int k_in) {
    __shared__ float zs[kW4Waves][16][16 * NB + 1];
    const int f0 = 16 * blockIdx.x;
    const int wave = wave_id();
    const int lane = threadIdx.x % kWave;
    const int m16 = lane & 15;
    const int c4 = lane >> 4;
    const int groups = k_in / kW4Group;
    const int n_c = (groups + 3) / 4;
    // features and rows past the end read the last one; they are not stored
    const size_t f = min(f0 + m16, n_out - 1);
    const uint8_t *wp = codes + f * (size_t)(k_in / 2) + c4 * 16;
    const uint8_t *sp = scales + f * (size_t)groups + c4;
    const uint16_t *xp[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
        xp[nb] = x + (size_t)min(16 * nb + m16, rows - 1) * k_in + c4 * 32;
    f32x4 acc[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
        acc[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int c = wave; c < n_c; c += kW4Waves) {
        // (lanes past the input's end multiply zeros)
        const bool in = 4 * c + c4 < groups;
        u32x4 w = {0u, 0u, 0u, 0u};
        float s = 1.f;
        bf16x8 xo[NB][4];
        if (in) {
            w = *reinterpret_cast<const u32x4 *>(wp + (size_t)c * 64);
            s = w4_scale(sp[4 * c]);
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
                xo[nb][kk] = in ? load_bf16x8(xp[nb] + c * kW4Chunk + 8 * kk) : zero_bf16x8();
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            const bf16x8 wo = w4_expand(w[kk], s);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
                acc[nb] = mfma16x16x32(wo, xo[nb][kk], acc[nb]);
        }
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            zs[wave][4 * c4 + i][16 * nb + m16] = acc[nb][i];
    __syncthreads();
    for (int idx = threadIdx.x; idx < 16 * rows; idx += kW4Waves * kWave) {
        const int u = idx % 16, r = idx / 16;
        if (f0 + u >= n_out)
            continue;
        float z = zs[0][u][r];
#pragma unroll
        for (int w = 1; w < kW4Waves; ++w)
            z += zs[w][u][r];
        const size_t at = (size_t)r * n_out + f0 + u;
        if (res)
            z += bf16_to_f32(res[at]);
        if constexpr (F32OUT)
            static_cast<float *>(y)[at] = z;
        else
            static_cast<uint16_t *>(y)[at] = f32_to_bf16(z);
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

}  // namespace

size_t linear_w4_workspace_bytes(int rows, int n_out, int k_in) { return 0; }

wf_status_t launch_linear_w4(const uint16_t *x, const uint8_t *codes, const uint8_t *scales,
                             const uint16_t *res, bool f32_out, void *y, int rows, int n_out,
                             int k_in, void *workspace, hipStream_t stream) {
    const dim3 grid((n_out + 15) / 16), block(kW4Waves * kWave);
    const int nb = (rows + 15) / 16;
#define WF_W4(NBV)                                                                          \
    if (nb == NBV) {                                                                        \
        if (f32_out)                                                                        \
            linear_w4<NBV, true><<<grid, block, 0, stream>>>(x, codes, scales, res, y, rows, \
                                                             n_out, k_in);                  \
        else                                                                                \
            linear_w4<NBV, false><<<grid, block, 0, stream>>>(x, codes, scales, res, y, rows, \
                                                              n_out, k_in);                 \
    } else
    WF_W4(1) WF_W4(2) WF_W4(3) WF_W4(4)
    { return WF_ERR_UNSUPPORTED; }
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
