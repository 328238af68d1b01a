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
#include "wf_lds_dma.h"
#include "wf_lowbit.h"

namespace wf {

namespace {

constexpr int kW4Waves = 8;
constexpr int kW4Group = 32;             // inputs per scale
constexpr int kW4Chunk = 128;            // inputs per tile: 16 bytes of codes per lane
constexpr int kW4Tile = 1024 + 64;       // 16 features x 128 inputs: codes, then scales

// Scale byte kk of a lane's dword -> the float that the conversion multiplies
// by: its exponent field (255 is then an infinity, which the conversion, like the
// format, takes for NaN).
__device__ __forceinline__ float w4_scale(unsigned s, int kk) {
    return __uint_as_float((kk < 3 ? s << (23 - 8 * kk) : s >> 1) & 0x7f800000u);
}

// A raw buffer's last word (data format 32, without which loads return nothing),
// and the cache policy of bytes that are read once.
constexpr int kRawBuffer = 4 << 15;
constexpr int kNonTemporal = 2;

// y[at] = z (+ the residual), in y's type.
__device__ __forceinline__ void store_y(void *y, const uint16_t *res, size_t at, float z,
                                        bool f32_out) {
    if (res)
        z += bf16_to_f32(res[at]);
    if (f32_out)
        static_cast<float *>(y)[at] = z;
    else
        static_cast<uint16_t *>(y)[at] = f32_to_bf16(z);
}

// Four features f .. f+3 of row r: in one store where `quads` says that rows keep
// its alignment, a quarter of the requests (61 rows, 2560 to 151936: 68 -> 56 us).
__device__ __forceinline__ void store_y4(void *y, const uint16_t *res, int r, int f, int n_out,
                                         f32x4 z, bool f32_out, bool quads) {
    const size_t at = (size_t)r * n_out + f;
    if (quads) {                                     // uniform
        if (f >= n_out)
            return;
        if (res) {
            const u32x2 v = *reinterpret_cast<const u32x2 *>(res + at);
            z[0] += __uint_as_float(v[0] << 16);
            z[1] += __uint_as_float(v[0] & 0xffff0000u);
            z[2] += __uint_as_float(v[1] << 16);
            z[3] += __uint_as_float(v[1] & 0xffff0000u);
        }
        if (f32_out)
            *reinterpret_cast<f32x4 *>(static_cast<float *>(y) + at) = z;
        else
            *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(y) + at) =
                uint2{pack_bf16x2(z[0], z[1]), pack_bf16x2(z[2], z[3])};
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (f + i < n_out)
            store_y(y, res, at + i, z[i], f32_out);
}

// The rows of x as a buffer; the offset of 16 bytes of it, behind its end (so
// that zeros are loaded) if `in` is false.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t x_buffer(const uint16_t *x, int rows, int k_in) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(x), 0, rows * k_in * 2,
                                             kRawBuffer);
}
__device__ __forceinline__ u32x4 load_x16(__amdgpu_buffer_rsrc_t x, unsigned at, bool in) {
    return __builtin_amdgcn_raw_buffer_load_b128(x, in ? at : 0x7ffffff0u, 0, 0);
}

// A lane's 16 bytes of a tile, which no other workgroup reads.
__device__ __forceinline__ u32x4 load_codes(const uint8_t *p) {
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
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

// Up to 16 rows, input split: workgroup b owns FB blocks of 16 features and the
// whole input, its 8 waves take interleaved 128-input chunks, U of them loaded
// at once and the next U on their way meanwhile, and their sums meet in LDS in
// wave order.  MFMA kk of chunk c takes the scale group 128c + 32kk ..: lane (m16,
// c4) its inputs 8*c4 .. +7 of feature m16 of each block and of x row m16, so four
// lanes read 64 contiguous bytes of x.  Bound by its launch and one or two trips to
// memory (one row, 4096 to 4096: 4.5 us out of HBM, 3.7 out of the last-level cache, of
// which an empty launch takes 1.7), or by the bytes in flight (12288 to 4096: 9.8 us,
// 2.7 TB/s).
template <int FB>
__global__ __launch_bounds__(kW4Waves * kWave) void linear_w4(
    const uint16_t *__restrict__ x, const uint8_t *__restrict__ w, const uint16_t *res, void *y,
    int rows, int n_out, int k_in, bool f32_out) {
    constexpr int U = FB == 1 ? 4 : 2;
    __shared__ float zs[kW4Waves][16][17];
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
    // (rows and inputs past the end are zeros)
    const __amdgpu_buffer_rsrc_t xp = x_buffer(x, rows, k_in);
    const unsigned xo = (unsigned)(m16 * k_in + c4 * 8) * 2;
    f32x4 acc[FB];
#pragma unroll
    for (int fb = 0; fb < FB; ++fb)
        acc[fb] = f32x4{0.f, 0.f, 0.f, 0.f};
    struct Batch {
        u32x4 w[U][FB];
        unsigned s[U][FB];
        bf16x8 x[U][4];
    };
    auto load = [&](Batch &q, int cb) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = min(cb + kW4Waves * u, n_c - 1);
#pragma unroll
            for (int fb = 0; fb < FB; ++fb) {
                const uint8_t *t = wp[fb] + (size_t)c * kW4Tile;
                q.w[u][fb] = load_codes(t + lane * 16);
                q.s[u][fb] = reinterpret_cast<const uint32_t *>(t + 1024)[m16];
            }
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
                q.x[u][kk] = __builtin_bit_cast(
                    bf16x8, load_x16(xp, xo + (4 * c + kk) * (kW4Group * 2), 4 * c + kk <= last_g));
        }
    };
    auto multiply = [&](const Batch &q, int cb) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (cb + kW4Waves * u >= n_c)            // uniform
                break;
#pragma unroll
            for (int fb = 0; fb < FB; ++fb) {
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                    acc[fb] = mfma16x16x32(w4_expand(q.w[u][fb][kk], w4_scale(q.s[u][fb], kk)),
                                           q.x[u][kk], acc[fb]);
            }
        }
    };
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
        for (int i = 0; i < 4; ++i)
            zs[wave][4 * c4 + i][m16] = acc[fb][i];
        __syncthreads();
        const int u = threadIdx.x % 16, r = threadIdx.x / 16, f = f0 + 16 * fb + u;
        if (r < rows && f < n_out) {                 // 512 threads: r up to 31
            float z = zs[0][u][r];
#pragma unroll
            for (int ww = 1; ww < kW4Waves; ++ww)
                z += zs[ww][u][r];
            store_y(y, res, (size_t)r * n_out + f, z, f32_out);
        }
    }
}

// Feature split: the 8 waves of a workgroup are 8 / KW feature groups, each of
// up to FB blocks of 16 features, of KW waves that share the input among them.
// All walk the input (or slice blockIdx.y of it) together in chunks of KW tiles
// of 128 inputs, one per wave, whose x, all rows, is staged in LDS, so a wave
// reads it once for all its blocks; the next chunk's codes and x are on their way
// to registers meanwhile.  KW > 1 is for few blocks: a wave of one block reads 4 KB of x per 1
// KB of codes and 16 rows from LDS, so with 64 rows the waves ask it for more than
// the 128 bytes a cycle it has; a quarter of the input and four times the blocks
// ask for a quarter.  Lanes and tiles as above.  The staged x is swizzled in 16-
// byte granules, g ^ (row & 7), so eight rows' reads meet distinct banks.  With
// several slices each stores its fp32 sums, part[slice][row][16 * blocks], for
// w4_sum.  Bound by HBM up to 16 rows (16 rows, 4096 to 24576: 13.5 us, 4.0 TB/s; 4096
// to 128256, fp32 out: 50, 5.7) and with many features (61 rows, 2560 to 151936: 55 us,
// 37 MB of them logits stored at the end), else by x: LDS, and L2 once per workgroup.
template <int NB, int FB, int KW>
__global__ __launch_bounds__(kW4Waves * kWave) void linear_w4_wide(
    const uint16_t *__restrict__ x, const uint8_t *__restrict__ w, const uint16_t *res, void *y,
    int rows, int n_out, int k_in, bool f32_out, bool quads, float *part) {
    constexpr int GRAN = 16 * KW;                    // 16-byte granules of a row's chunk
    constexpr int XG = 16 * NB * GRAN;               // ... of the chunk, XT of them a thread's
    constexpr int XT = (XG + kW4Waves * kWave - 1) / (kW4Waves * kWave);
    constexpr int FG = kW4Waves / KW;
    // x two chunks ahead where the registers take it easily (16 rows, 12288 to 4096:
    // 12.55 -> 12.0 us; one row, 4096 to 24576: 12.85 -> 12.3; 64 rows, two blocks,
    // 5120 to 16384: 20.0 -> 20.4, so not there)
    constexpr bool X2 = NB * FB < 8;
    // (with room for all threads' granules: under a condition the loads would move
    // behind the codes' to the stores, 1 row, 4096 to 128256: 55 us, 47 without)
    __shared__ u32x4 xs[2][XT * kW4Waves * kWave];
    const int wave = wave_id();
    const int kw = wave % KW, fg = wave / KW;
    const int lane = threadIdx.x % kWave;
    const int m16 = lane & 15;
    const int c4 = lane >> 4;
    const int n_t = (k_in + kW4Chunk - 1) / kW4Chunk, n_c = (n_t + KW - 1) / KW;
    const int c_first = (int)blockIdx.y * n_c / (int)gridDim.y;
    const int c_end = ((int)blockIdx.y + 1) * n_c / (int)gridDim.y;
    // blocks dealt out evenly over all feature groups of the launch
    const int blocks = (n_out + 15) / 16;
    const int groups = gridDim.x * FG, id = blockIdx.x * FG + fg;
    const int b_first = (int)((long long)id * blocks / groups);
    const int n_b = (int)((long long)(id + 1) * blocks / groups) - b_first;

    // A block's tiles up to the slice's end, as a buffer: loads past them return
    // zeros and cost no traffic.
    __amdgpu_buffer_rsrc_t wp[FB];
    const int w_bytes = min(KW * c_end, n_t) * kW4Tile;
#pragma unroll
    for (int fb = 0; fb < FB; ++fb)      // (without an fb-th block: none)
        wp[fb] = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<uint8_t *>(w) + (size_t)min(b_first + fb, blocks - 1) * n_t * kW4Tile, 0,
            fb < n_b ? w_bytes : 0, kRawBuffer);
    f32x4 acc[FB][NB];
#pragma unroll
    for (int fb = 0; fb < FB; ++fb)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
            acc[fb][nb] = f32x4{0.f, 0.f, 0.f, 0.f};

    // No branch surrounds the loads: the compiler would lose count of those in
    // flight and wait for all (one row, 2560 to 151936: 42 us, 51 with a branch at
    // the end of the input).
    struct Codes {
        u32x4 w[FB];
        unsigned s[FB];
    };
    Codes ring[2];
    u32x4 xr[X2 ? 2 : 1][XT];
    auto load_w = [&](Codes &q, int ch) __attribute__((always_inline)) {
        const unsigned at = (unsigned)(KW * ch + kw) * kW4Tile;
#pragma unroll
        for (int fb = 0; fb < FB; ++fb) {
            q.w[fb] = __builtin_amdgcn_raw_buffer_load_b128(wp[fb], at + lane * 16, 0, kNonTemporal);
            q.s[fb] = __builtin_amdgcn_raw_buffer_load_b32(wp[fb], at + 1024 + m16 * 4, 0, 0);
        }
    };
    // (rows and inputs past the end are zeros)
    const __amdgpu_buffer_rsrc_t xp = x_buffer(x, rows, k_in);
    auto load_x = [&](u32x4 (&to)[XT], int ch) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < XT; ++j) {
            const int idx = threadIdx.x + j * kW4Waves * kWave;
            const int r = idx / GRAN, g = ch * GRAN + idx % GRAN;
            to[j] = load_x16(xp, (unsigned)(r * k_in * 2 + g * 16),
                             g < k_in / 8 && (!X2 || ch < c_end));
        }
    };
    auto stage_x = [&](const u32x4 (&from)[XT], int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < XT; ++j) {
            const int idx = threadIdx.x + j * kW4Waves * kWave;
            const int r = idx / GRAN, g = idx % GRAN;
            xs[buf][r * GRAN + (g ^ (r & 7))] = from[j];
        }
    };
    // every wave's LDS writes are done; loads in flight stay so
    auto barrier = [] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
    // One chunk, its codes in ring[I], its x in buffer I; `more`: another follows.
    auto step = [&](auto it, auto more, int ch) __attribute__((always_inline)) {
        constexpr int I = decltype(it)::value;
        if constexpr (decltype(more)::value) {
            load_x(xr[X2 ? I : 0], X2 ? ch + 2 : ch + 1);
            __builtin_amdgcn_sched_barrier(0);       // (x first: its wait leaves the codes be)
            load_w(ring[1 - I], ch + 1);
            __builtin_amdgcn_sched_barrier(0);
        }
        const Codes &now = ring[I];
        const u32x4 *xb = xs[I];
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            bf16x8 xo[NB];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const int r = 16 * nb + m16, g = 16 * kw + 4 * kk + c4;
                xo[nb] = __builtin_bit_cast(bf16x8, xb[r * GRAN + (g ^ (r & 7))]);
            }
#pragma unroll
            for (int fb = 0; fb < FB; ++fb) {
                const bf16x8 wo = w4_expand(now.w[fb][kk], w4_scale(now.s[fb], kk));
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
                    acc[fb][nb] = mfma16x16x32(wo, xo[nb], acc[fb][nb]);
            }
        }
        if constexpr (decltype(more)::value) {
            stage_x(xr[X2 ? 1 - I : 0], 1 - I);
            barrier();
        }
    };
    load_x(xr[0], c_first);
    __builtin_amdgcn_sched_barrier(0);
    load_w(ring[0], c_first);
    if constexpr (X2)
        load_x(xr[1], c_first + 1);
    __builtin_amdgcn_sched_barrier(0);
    stage_x(xr[0], 0);
    barrier();
    constexpr std::true_type more;
    constexpr std::false_type last;
    int ch = c_first;
    for (; ch + 2 < c_end; ch += 2) {
        step(ic<0>{}, more, ch);
        step(ic<1>{}, more, ch + 1);
    }
    if (ch + 1 < c_end) {
        step(ic<0>{}, more, ch);
        step(ic<1>{}, last, ch + 1);
    } else {
        step(ic<0>{}, last, ch);
    }
    // lane (m16, c4) holds features 4*c4 .. +3 of row m16
    auto put = [&](int fb, int nb, f32x4 z) __attribute__((always_inline)) {
        const int r = 16 * nb + m16, f = 16 * (b_first + fb) + 4 * c4;
        if (r >= rows || fb >= n_b)
            return;
        if (gridDim.y > 1)
            *reinterpret_cast<f32x4 *>(part + ((size_t)blockIdx.y * rows + r) * 16 * blocks + f) =
                z;
        else
            store_y4(y, res, r, f, n_out, z, f32_out, quads);
    };
    if constexpr (KW == 1) {
#pragma unroll
        for (int fb = 0; fb < FB; ++fb)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
                put(fb, nb, acc[fb][nb]);
    } else {
        // The sums of a feature group's waves meet in the chunks' place, P blocks
        // at a time; each wave adds up, in wave order, and stores every KW-th
        // piece of 16 rows.
        constexpr int P = KW < FB ? KW : FB;
        static_assert(sizeof(xs) >= kW4Waves * P * NB * 1024, "room");
        f32x4 *meet = reinterpret_cast<f32x4 *>(xs) + fg * (KW * P * NB * kWave);
#pragma unroll
        for (int f0 = 0; f0 < FB; f0 += P) {
            __syncthreads();             // (the chunks, or the sums before, are done with)
#pragma unroll
            for (int t = 0; t < P * NB; ++t)
                if (f0 + t / NB < FB)
                    meet[(kw * P * NB + t) * kWave + lane] = acc[f0 + t / NB][t % NB];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < (P * NB + KW - 1) / KW; ++i) {
                const int t = i * KW + kw;
                if (P * NB % KW && t >= P * NB)
                    continue;
                f32x4 z = meet[t * kWave + lane];
#pragma unroll
                for (int k = 1; k < KW; ++k)
                    z += meet[(k * P * NB + t) * kWave + lane];
                put(f0 + t / NB, t % NB, z);
            }
        }
    }
}

// y = the slices' sums in order (and the residual); 4 features per thread.
constexpr int kW4MaxSlices = 4;

__global__ __launch_bounds__(256) void w4_sum(const float *__restrict__ part, int slices,
                                              const uint16_t *res, void *y, int rows, int n_out,
                                              bool f32_out, bool quads) {
    const int row_quads = (n_out + 15) / 16 * 4;
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (size_t)rows * row_quads)
        return;
    const int r = (int)(i / row_quads), f = (int)(i % row_quads) * 4;
    f32x4 v[kW4MaxSlices];
#pragma unroll
    for (int k = 0; k < kW4MaxSlices; ++k)
        if (k < slices)
            v[k] = reinterpret_cast<const f32x4 *>(part)[((size_t)k * rows + r) * row_quads + f / 4];
    f32x4 z = v[0];
#pragma unroll
    for (int k = 1; k < kW4MaxSlices; ++k)
        if (k < slices)
            z += v[k];
    store_y4(y, res, r, f, n_out, z, f32_out, quads);
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

// Tile (block b, chunk c) of the packed weight: lane m + 16 q of a wave finds
// its four dwords of codes at 16 * lane, dword kk the eight inputs 128c + 32kk +
// 8q .. +7 of feature 16b + m, and the scales of the chunk's four groups, bytes
// kk, at 1024 + 4m.  One wave per tile; features and inputs past the end are
// zeros under scale 1.
__global__ __launch_bounds__(kWave) void w4_pack(const uint8_t *__restrict__ codes,
                                                 const uint8_t *__restrict__ scales, int rows,
                                                 int groups, uint8_t *__restrict__ packed) {
    const int lane = threadIdx.x, m = lane & 15, q = lane >> 4;
    const int n_c = (groups + 3) / 4;
    const size_t tile = blockIdx.x;
    const size_t f = tile / n_c * 16 + m;
    const int g0 = (int)(tile % n_c) * 4;
    u32x4 v = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
        if (f < (size_t)rows && g0 + kk < groups)
            v[kk] = reinterpret_cast<const uint32_t *>(codes)[(f * groups + g0 + kk) * 4 + q];
    uint8_t *t = packed + tile * kW4Tile;
    reinterpret_cast<u32x4 *>(t)[lane] = v;
    // (lane m + 16 q writes the scale of group q)
    t[1024 + 4 * m + q] = f < (size_t)rows && g0 + q < groups ? scales[f * groups + g0 + q] : 127;
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

namespace {

// How a product runs: fb blocks of 16 features per workgroup (input split) or
// feature group (feature split, kw waves each), the launch's workgroups, and
// slices of the input.
struct W4Plan {
    bool wide;
    int fb, kw, groups, slices;
};

W4Plan plan_linear_w4(int rows, int n_out, int k_in) {
    const int blocks = (n_out + 15) / 16;
    W4Plan p{};
    p.slices = 1;
    // Up to 16 rows and three blocks per CU: the input split, one workgroup per CU
    // (one row, 4096 to 8192: 6.5 us, the feature split 7.6; to 12288: 8.3 and 9.4; 8
    // rows, 8192 to 8192: 12.2 and 13.5; 16 rows, 4096 to 12288: 10.3 and 10.0, to
    // 8192: 8.4 and 7.8).  But each workgroup reads all of x, so where that is much and
    // the features few, slices of the feature split (16 rows, 12288 to 4096: 15.6 us,
    // 12.5 in four slices; 25600 to 5120: 33.8 and 20.8; 8192 to 4096: 11.1 and 11.2; 8
    // rows, 12288 to 4096: 12.0 and 12.4).
    const bool much_x = blocks < 2 * 256 && rows * k_in > 144 * 1024;
    if (rows <= 16 && blocks <= 3 * 256 && !much_x) {
        p.fb = (blocks + 255) / 256;
        p.groups = (blocks + p.fb - 1) / p.fb;
        return p;
    }
    // As many waves to a feature group as leave each up to five blocks, at most four:
    // more loads in flight (us with one, two, four waves.  To 24576, from 4096: one row
    // -, 14.0, 12.1; 64 rows 28.2, 23.2, 21.5.  To 40000: one row, from 4096, -, 19.4,
    // 19.2; 64 rows, from 2560, 24.3, 21.8, 21.8, from 4096 -, 31.7, 30.3.  16 rows, 4096
    // to 64000: 28.0, 28.1, 29.3; to 100000: 39.3, 42.5, -; 64 rows, 2560 to 60000: 28.3,
    // 28.1, -; to 90000: 37.0, 43.2, -).  Eight gain on four nowhere but for one row of
    // long input (16 rows, 4096 to 16384: 11.0 and 10.8; one row, 2560 to 19456: 9.1 and
    // 8.1, 12288 to 16384: 22.2 and 22.7).
    p.wide = true;
    p.kw = blocks <= 10 * 256 ? 4 : blocks <= 20 * 256 ? 2 : 1;
    const int fg = kW4Waves / p.kw;
    // fewer than two blocks per CU: slices of at least two chunks, so a workgroup
    // reads less of x, at most four (64 rows, 4096 to 4096: 13.3 us without, 12.5 with
    // two or four, 16.1 with eight; 12288 to 4096: 32.3, 22.3 with two, 19.0 with four,
    // 20.8 with eight).  (The last workgroup to arrive adding the slices up instead of
    // w4_sum took 16.8 us where the second launch took 13.)
    const int chunks = (k_in + 128 * p.kw - 1) / (128 * p.kw);
    if (blocks < 2 * 256)
        p.slices = std::max(1, std::min({kW4MaxSlices, chunks / 2, 5 * fg * 256 / blocks}));
    const int per = fg * (256 / p.slices);           // feature groups of one workgroup per CU
    const int rounds = (blocks + 5 * per - 1) / (5 * per);
    p.fb = (blocks + rounds * per - 1) / (rounds * per);
    p.groups = std::min(rounds * (256 / p.slices), (blocks + fg - 1) / fg);
    return p;
}

}  // namespace

static bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

size_t linear_w4_workspace_bytes(int rows, int n_out, int k_in) {
    const W4Plan p = plan_linear_w4(rows, n_out, k_in);
    return p.slices == 1 ? 0
                         : kCounterBytes + (size_t)p.slices * rows * ((n_out + 15) / 16 * 16) *
                                               sizeof(float);
}

wf_status_t launch_linear_w4(const uint16_t *x, const uint8_t *w, const uint16_t *res,
                             bool f32_out, void *y, int rows, int n_out, int k_in,
                             void *workspace, hipStream_t stream) {
    const W4Plan p = plan_linear_w4(rows, n_out, k_in);
    const dim3 block(kW4Waves * kWave);
    if (!p.wide) {
#define WF_W4(FBV)                                                                            \
    if (p.fb == FBV)                                                                          \
        linear_w4<FBV><<<p.groups, block, 0, stream>>>(x, w, res, y, rows, n_out, k_in,       \
                                                       f32_out);                              \
    else
        WF_W4(1) WF_W4(2) WF_W4(3)
        return WF_ERR_UNSUPPORTED;
#undef WF_W4
        return hipGetLastError() == hipSuccess ? WF_OK : WF_ERR_HIP;
    }
    float *part = p.slices > 1 ? reinterpret_cast<float *>(static_cast<char *>(workspace) +
                                                           kCounterBytes)
                               : nullptr;
    const int nb = (rows + 15) / 16;
    const bool quads = n_out % 4 == 0 && aligned(y, 16) && aligned(res, 8);
    const dim3 grid(p.groups, p.slices);
#define WF_W4(NBV, FBV, KWV)                                                                  \
    if (nb == NBV && p.fb == FBV && p.kw == KWV)                                              \
        linear_w4_wide<NBV, FBV, KWV><<<grid, block, 0, stream>>>(x, w, res, y, rows, n_out,  \
                                                                  k_in, f32_out, quads, part);\
    else
#define WF_W4_FEW(NBV, KWV) WF_W4(NBV, 1, KWV) WF_W4(NBV, 2, KWV)
#define WF_W4_MANY(NBV, KWV) WF_W4(NBV, 3, KWV) WF_W4(NBV, 4, KWV) WF_W4(NBV, 5, KWV)
    // (what the plan can ask for)
    WF_W4_MANY(1, 1) WF_W4_MANY(2, 1) WF_W4_MANY(3, 1) WF_W4_MANY(4, 1)
    WF_W4_MANY(1, 2) WF_W4_MANY(2, 2) WF_W4_MANY(3, 2) WF_W4_MANY(4, 2)
    WF_W4_FEW(1, 4) WF_W4_FEW(2, 4) WF_W4_FEW(3, 4) WF_W4_FEW(4, 4)
    WF_W4_MANY(1, 4) WF_W4_MANY(2, 4) WF_W4_MANY(3, 4) WF_W4_MANY(4, 4)
    return WF_ERR_UNSUPPORTED;
#undef WF_W4_FEW
#undef WF_W4_MANY
#undef WF_W4
    if (p.slices > 1) {
        const size_t n = (size_t)rows * ((n_out + 15) / 16 * 4);
        const unsigned wg = (unsigned)((n + 255) / 256);
        w4_sum<<<wg, 256, 0, stream>>>(part, p.slices, res, y, rows, n_out, f32_out, quads);
    }
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
