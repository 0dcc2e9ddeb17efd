// Microscaled 4-bit floating point: quantisation, its inverse, the linear layer on stored weights and its gradient into the
// input (declared in include/pac_mx4.h, where the stored form is described).
#include "../../include/pac_mx4.h"
#include "pac_mma.h"
#include "pac_span.h"
#include <mutex>

namespace pac {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

static inline bool m_aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// The conversions take a block's scale as the exponent field of a float, which is the scale byte itself (0: 2^-127, 255: NaN).
__device__ __forceinline__ float mx4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// ---------------------------------------------------------------------------
// quantise: four lanes a block, eight neighbouring values each (16-byte loads where the rows allow them: VEC).  The block's
// absmax goes round its four lanes; the scale's exponent is the absmax's own exponent less two, so no logarithm is taken;
// the conversion divides by the scale, rounds to nearest even and saturates at 6 in one instruction a pair.  Memory bounds it:
// 4096 x 4096 fp32 in 12.5 us (76 MB: 6.1 TB/s, part of it from the last-level cache), the way back in 15.4 us (4.8 TB/s).
// ---------------------------------------------------------------------------
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_mx4_quant(const T *__restrict__ x, uint32_t units, uint32_t upr, int cols, int64_t ldx,
                                                   uint32_t *__restrict__ codes, uint8_t *__restrict__ scales)
{
    // a unit is 256 columns of a row: 32 lanes
    const uint32_t u = blockIdx.x * 8u + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (u >= units) return; // whole groups of 32 lanes leave: the exchanges below stay within four
    const uint32_t row = u / upr, col = (u - row * upr) * 256u + lane * 8u;
    const T *src = x + (int64_t)row * ldx + col;
    float v[8];
    if (VEC && (int)col + 8 <= cols) {
        if constexpr (sizeof(T) == 2) {
            const bf16x8 r = *reinterpret_cast<const bf16x8 *>(src);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (float)r[e];
        } else {
            const f32x4 r0 = *reinterpret_cast<const f32x4 *>(src), r1 = *reinterpret_cast<const f32x4 *>(src + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = r0[e], v[4 + e] = r1[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (int)col + e < cols ? (float)src[e] : 0.f;
    }
    uint32_t top = 0; // bits of the absmax: for non-negative floats, infinities and NaN among them, bits order as values do
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
    const uint32_t ex = top >> 23; // floor(log2) + 127; 0 for what is below 2^-126, whose scale is the least anyhow
    const bool none = ex == 255;
    const uint32_t byte = none ? 255u : ex > 2 ? ex - 2 : 0u;
    uint32_t w = 0;
    if (!none) {
        const float s = mx4_scale(byte);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], s, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], s, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], s, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], s, 3);
    }
    codes[(int64_t)u * 32 + lane] = w;
    if ((lane & 3) == 0) scales[(int64_t)u * 8 + (lane >> 2)] = (uint8_t)byte;
}

__device__ __forceinline__ void mx4_values(uint32_t w, float s, float (&v)[8])
{
    bf16x2 p;
    p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0); v[0] = (float)p[0]; v[1] = (float)p[1];
    p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1); v[2] = (float)p[0]; v[3] = (float)p[1];
    p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2); v[4] = (float)p[0]; v[5] = (float)p[1];
    p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3); v[6] = (float)p[0]; v[7] = (float)p[1];
}

// eight codes as bf16, which holds every e2m1 value times a power of two exactly
__device__ __forceinline__ bf16x8 mx4_bf16(uint32_t w, float s)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_mx4_dequant(const uint32_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                                                     uint32_t units, uint32_t upr, int cols, T *__restrict__ out, int64_t ldo)
{
    const uint32_t u = blockIdx.x * 8u + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (u >= units) return;
    const uint32_t row = u / upr, col = (u - row * upr) * 256u + lane * 8u;
    if ((int)col >= cols) return;
    float v[8];
    mx4_values(codes[(int64_t)u * 32 + lane], mx4_scale(scales[(int64_t)u * 8 + (lane >> 2)]), v);
    T *dst = out + (int64_t)row * ldo + col;
    if (VEC && (int)col + 8 <= cols) {
        if constexpr (sizeof(T) == 2) {
            bf16x8 r;
#pragma unroll
            for (int e = 0; e < 8; ++e) r[e] = (bf16_t)v[e];
            *reinterpret_cast<bf16x8 *>(dst) = r;
        } else {
            *reinterpret_cast<f32x4 *>(dst) = f32x4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4 *>(dst + 4) = f32x4{v[4], v[5], v[6], v[7]};
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if ((int)col + e < cols) dst[e] = (T)v[e];
    }
}

// ---------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------
struct Mx4Args {
    const void *x;     // bf16 [M][ldx], or codes of the stored form
    const uint8_t *xs; // scales of the stored form
    int64_t ldx;
    const uint8_t *w, *ws; // W, stored form
    int M, K, N;
    int64_t wp, sp; // pitches of W's codes and scales
    const float *bias;
    int gelu;
    void *y;
    int y_f32;
    int64_t ldy;
};

// GELU in the erf form, u Phi(u) = max(u, 0) - |u| Phi(-|u|).  log2 of the normal distribution's tail is smooth: one polynomial of
// degree 9 and one exponential, 14 instructions (erff alone takes some forty).  Coefficients: the linear programme that makes the
// largest error of |u| Phi(-|u|) over 0 <= |u| <= 11 least, measured in the smaller of 1e-7 |u| and 1e-3 of the value.  In 32 bits the
// result is off by less than 2e-7 |u|, and where u is negative by less than 1.4e-3 of itself down to -11, where it is 2e-27; from
// there on the polynomial keeps falling, so that it goes to zero.  (Degree 7, fitted to 5.75 and constant past it, was 1 % off at
// -5 and never reached zero.)  NaN stays NaN.
__device__ __forceinline__ float mx4_gelu(float u)
{
    const float x = __builtin_elementwise_minimum(fabsf(u), 14.f); // 2^-143: zero
    float p = 1.4396019487605827e-08f;
    p = fmaf(p, x, -5.287711246637627e-07f);
    p = fmaf(p, x, 6.437743650167249e-06f);
    p = fmaf(p, x, -6.743613084836397e-06f);
    p = fmaf(p, x, -0.0006199441850185394f);
    p = fmaf(p, x, 0.00774502893909812f);
    p = fmaf(p, x, -0.05298928543925285f);
    p = fmaf(p, x, -0.459043025970459f);
    p = fmaf(p, x, -1.1511250734329224f);
    p = fmaf(p, x, -0.9999996423721313f);
    return fmaf(-x, __builtin_amdgcn_exp2f(p), fmaxf(u, 0.f));
}

__device__ __forceinline__ void mx4_put(const Mx4Args &a, int m, int n, float v)
{
    if (a.bias) v += a.bias[n];
    if (a.gelu) v = mx4_gelu(v);
    if (a.y_f32) reinterpret_cast<float *>(a.y)[(int64_t)m * a.ldy + n] = v;
    else reinterpret_cast<bf16_t *>(a.y)[(int64_t)m * a.ldy + n] = (bf16_t)v;
}

// The epilogue of a wavefront's WTM x WTN accumulators: rows mw + 32 x + (8 (v / 4) + 4 g + v % 4), this lane's WTN neighbouring
// columns from n on, `cols` in all.  Everything that does not change from value to value is decided once, outside: written plainly,
// with the type, the bounds and GELU asked for at each value, a tile of 256 x 256 spent 16 us here.
template <int WTM, int WTN>
__device__ __forceinline__ void mx4_write(const Mx4Args &a, const f32x16 (&acc)[WTM][WTN], int mw, int n, int g, int cols)
{
    float bias[WTN];
#pragma unroll
    for (int y = 0; y < WTN; ++y) bias[y] = a.bias ? a.bias[min(n + y, cols - 1)] : 0.f;
    auto put = [&](auto f32, auto gelu, auto full) __attribute__((always_inline)) {
        typedef typename std::conditional<decltype(f32)::value, float, bf16_t>::type T;
        typedef T vec __attribute__((ext_vector_type(WTN)));
        T *const y0 = reinterpret_cast<T *>(a.y) + (int64_t)mw * a.ldy; // the same for all lanes
        const bool wide = n + WTN <= cols && a.ldy % WTN == 0 && (reinterpret_cast<uintptr_t>(a.y) & (sizeof(vec) - 1)) == 0;
        const int64_t lane_at = 4 * g * a.ldy + n;
#pragma unroll
        for (int x = 0; x < WTM; ++x)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int r = x * 32 + 8 * (v >> 2) + (v & 3);
                if (!decltype(full)::value && mw + r + 4 * g >= a.M) continue;
                vec o;
#pragma unroll
                for (int y = 0; y < WTN; ++y) {
                    float f = acc[x][y][v] + bias[y];
                    if constexpr (decltype(gelu)::value) f = mx4_gelu(f);
                    o[y] = (T)f;
                }
                T *const p = y0 + r * a.ldy + lane_at;
                if (decltype(full)::value || wide) *reinterpret_cast<vec *>(p) = o;
                else
#pragma unroll
                    for (int y = 0; y < WTN; ++y)
                        if (n + y < cols) p[y] = o[y];
            }
    };
    using yes = std::integral_constant<bool, true>;
    using no = std::integral_constant<bool, false>;
    // a whole tile whose rows take whole stores (the column test is the same for all lanes: the last lane's)
    const int n_last = __builtin_amdgcn_readlane(n, 63) + WTN, size = a.y_f32 ? 4 : 2;
    const bool full = mw + 32 * WTM <= a.M && n_last <= cols && a.ldy % WTN == 0 && (reinterpret_cast<uintptr_t>(a.y) & (WTN * size - 1)) == 0;
    if (full) {
        if (a.y_f32) a.gelu ? put(yes(), yes(), yes()) : put(yes(), no(), yes());
        else a.gelu ? put(no(), yes(), yes()) : put(no(), no(), yes());
    } else {
        if (a.y_f32) a.gelu ? put(yes(), yes(), no()) : put(yes(), no(), no());
        else a.gelu ? put(no(), yes(), no()) : put(no(), no(), no());
    }
}

// eight bf16 of which those from `valid` on do not count
__device__ __forceinline__ u32x4 mx4_keep(u32x4 v, int valid)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = valid >= 2 * e + 2 ? v[e] : valid == 2 * e + 1 ? v[e] & 0xffffu : 0u;
    return v;
}

// A tile of 16 columns of y by 16 RM rows a workgroup, the contraction dealt over its NW wavefronts in steps of 128 and joined in
// LDS in a fixed order.  Operands go from memory straight into registers: lane (i, q) holds row i's block of 32 number q of the
// step, so that a lane has one scale, its 16 bytes of codes are one load, and four matrix instructions of 32 (one of 128 where x
// is stored too) take eight codes of every lane's block each: the order of the sum does not matter to it.  For few rows, where
// neither tiles nor matrix rate count: 1 x 4096 x 4096 in 5.7 us, of which a launch takes 2.5 and the 9 MB of W 1.8 at a copy's
// rate.  (With the next step's operands requested ahead by hand it is slower, 64 x 4096 x 4096 25 -> 30 us: fewer workgroups fit.)
// What x is to it: bf16 rows, the stored form, or bf16 rows that are to count as their mx4 values: a lane holds whole blocks, so it
// quantises them by itself, and the call needs no launch and no memory for x's stored form.
enum { MX4_X16, MX4_X4, MX4_XQ };

// 32 bf16 as e2m1 with one scale: what k_mx4_quant stores of them, bit for bit
__device__ __forceinline__ uint32_t mx4_block(const u32x4 (&x)[4], i32x8 &codes)
{
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 top = {0, 0}; // absolute values' bits order as the values do
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t b = x[j][e] & 0x7fff7fffu;
            top = __builtin_elementwise_max(top, *reinterpret_cast<const u16x2 *>(&b));
        }
    const uint32_t ex = (uint32_t)max(top[0], top[1]) >> 7;
    const bool none = ex == 255;
    const uint32_t byte = none ? 255u : ex > 2 ? ex - 2 : 0u;
    const float s = mx4_scale(byte);
    codes = i32x8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t w = 0;
        const bf16x2 *p = reinterpret_cast<const bf16x2 *>(&x[j]);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, p[0], s, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, p[1], s, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, p[2], s, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, p[3], s, 3);
        codes[j] = none ? 0 : (int)w;
    }
    return byte;
}

template <int X, int RM, int NW> __global__ __launch_bounds__(64 * NW) void k_mx4_rows(Mx4Args a)
{
    constexpr bool X4 = X == MX4_X4;
    constexpr int TM = 16 * RM, PITCH = 20;
    __shared__ __attribute__((aligned(16))) float red[NW * TM * PITCH];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
    const int nt = (a.N + 15) / 16, n0 = (int)(blockIdx.x % nt) * 16, m0 = (int)(blockIdx.x / nt) * TM;
    const int nrow = min(n0 + i, a.N - 1), steps = (a.K + 255) / 256 * 2;
    const uint8_t *wr = a.w + nrow * a.wp + 16 * q, *sr = a.ws + nrow * a.sp + q;
    f32x4 acc[RM];
    const char *xr[RM];
    const uint8_t *xsr[RM];
#pragma unroll
    for (int r = 0; r < RM; ++r) {
        acc[r] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int64_t m = min(m0 + 16 * r + i, a.M - 1);
        xr[r] = X4 ? reinterpret_cast<const char *>(a.x) + m * a.wp + 16 * q
                   : reinterpret_cast<const char *>(a.x) + m * a.ldx * 2;
        xsr[r] = X4 ? a.xs + m * a.sp + q : nullptr;
    }
    const int last = (a.K + 7) / 8 * 8 - 8; // the last chunk of x that is there
    for (int s = wave; s < steps; s += NW) {
        const u32x4 w = *reinterpret_cast<const u32x4 *>(wr + 64 * s);
        const uint32_t sc = sr[4 * s];
        if constexpr (X4) {
            const i32x8 wf = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
#pragma unroll
            for (int r = 0; r < RM; ++r) {
                const u32x4 x = *reinterpret_cast<const u32x4 *>(xr[r] + 64 * s);
                const i32x8 xf = {(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0};
                acc[r] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf, xf, acc[r], 4, 4, 0, (int)sc, 0, (int)xsr[r][4 * s]);
            }
        } else if constexpr (X == MX4_XQ) {
            const i32x8 wf = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
            const int k0 = 128 * s + 32 * q;
#pragma unroll
            for (int r = 0; r < RM; ++r) {
                u32x4 x[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = *reinterpret_cast<const u32x4 *>(xr[r] + 2 * min(k0 + 8 * j, last));
                if (128 * s + 128 > a.K)
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = mx4_keep(x[j], a.K - (k0 + 8 * j));
                i32x8 xf;
                const uint32_t xs = mx4_block(x, xf);
                acc[r] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf, xf, acc[r], 4, 4, 0, (int)sc, 0, (int)xs);
            }
        } else {
            bf16x8 wf[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) wf[j] = mx4_bf16(w[j], mx4_scale(sc));
            const int k0 = 128 * s + 32 * q;
#pragma unroll
            for (int r = 0; r < RM; ++r)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int k = k0 + 8 * j;
                    u32x4 x = *reinterpret_cast<const u32x4 *>(xr[r] + 2 * min(k, last));
                    if (128 * s + 128 > a.K) x = mx4_keep(x, a.K - k);
                    acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[j], *reinterpret_cast<bf16x8 *>(&x), acc[r], 0, 0, 0);
                }
        }
    }
    // lane (i, q) holds columns 4 q .. 4 q + 3 of row i
#pragma unroll
    for (int r = 0; r < RM; ++r) *reinterpret_cast<f32x4 *>(red + (wave * TM + 16 * r + i) * PITCH + 4 * q) = acc[r];
    __syncthreads();
    for (int e = threadIdx.x; e < TM * 16; e += 64 * NW) {
        const int m = e >> 4, n = e & 15;
        if (m0 + m >= a.M || n0 + n >= a.N) continue;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) v += red[(w * TM + m) * PITCH + n];
        mx4_put(a, m0 + m, n0 + n, v);
    }
}

// dx: a tile of 128 columns of dx by 16 RM rows, the rows of W dealt over NW wavefronts in steps of 32.  The contraction runs
// across W's rows, eight of which a lane needs for one column: a lane loads 4 bytes (eight columns) of eight rows, converts them
// with each row's scale and swaps halves of register pairs, which leaves it the eight rows of eight columns.  The matrix
// instruction number c takes column c of every lane, so lanes i = 0 .. 15 cover 128 neighbouring columns and an output lane holds
// eight neighbouring ones: no transposed copy of W anywhere.  517 x 1001 x 775 in 6.7 us, 1 x 4096 x 4096 in 11 to 13 us.  Where
// workgroups fill the chip the vector units bound it (64 instructions a step to convert and swap, beside eight matrix instructions);
// with few rows it is their number: one for 128 columns, 32 of them at K = 4096, each walking all of N.
__device__ __forceinline__ uint32_t pk_lo(bf16x2 a, bf16x2 b) // {a[0], b[0]}
{
    return __builtin_amdgcn_perm(*reinterpret_cast<uint32_t *>(&b), *reinterpret_cast<uint32_t *>(&a), 0x05040100u);
}
__device__ __forceinline__ uint32_t pk_hi(bf16x2 a, bf16x2 b) // {a[1], b[1]}
{
    return __builtin_amdgcn_perm(*reinterpret_cast<uint32_t *>(&b), *reinterpret_cast<uint32_t *>(&a), 0x07060302u);
}

// w[e], s[e]: eight columns' codes and the scale of row e; col[c]: the eight rows of column c
__device__ __forceinline__ void mx4_columns(const uint32_t (&w)[8], const float (&s)[8], u32x4 (&col)[8])
{
#pragma unroll
    for (int p = 0; p < 4; ++p) { // rows 2 p and 2 p + 1
#define PAC_MX4_PAIR(C)                                                                                                        \
    {                                                                                                                          \
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[2 * p], s[2 * p], C);                                     \
        const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[2 * p + 1], s[2 * p + 1], C);                             \
        col[2 * C][p] = pk_lo(a, b);                                                                                           \
        col[2 * C + 1][p] = pk_hi(a, b);                                                                                       \
    }
        PAC_MX4_PAIR(0) PAC_MX4_PAIR(1) PAC_MX4_PAIR(2) PAC_MX4_PAIR(3)
#undef PAC_MX4_PAIR
    }
}

template <int RM, int NW> __global__ __launch_bounds__(64 * NW) void k_mx4_dx_rows(Mx4Args a)
{
    constexpr int TM = 16 * RM, PITCH = 132;
    extern __shared__ __attribute__((aligned(16))) float red[]; // [NW][TM][PITCH]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, q = lane >> 4;
    const int kt = (a.K + 127) / 128, kc0 = (int)(blockIdx.x % kt) * 128, m0 = (int)(blockIdx.x / kt) * TM;
    const int64_t w_at = 8 * q * a.wp + kc0 / 2 + 4 * i, s_at = 8 * q * a.sp + kc0 / 32 + (i >> 2); // this lane's place in a step
    f32x4 acc[8][RM];
    const bf16_t *dyr[RM];
#pragma unroll
    for (int r = 0; r < RM; ++r) {
        dyr[r] = reinterpret_cast<const bf16_t *>(a.x) + min(m0 + 16 * r + i, a.M - 1) * a.ldx;
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[c][r] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int steps = (a.N + 31) / 32, last = (a.N + 7) / 8 * 8 - 8;
    // The coming step's operands are under way while the present one's are multiplied; past the end: the last step's, unused.  Rows'
    // addresses are a scalar's work (at an address a lane and row the vector units bound small M).
    uint32_t wn[8], sn[8];
    u32x4 dn[RM];
    auto fetch = [&](int s) {
        s = min(s, steps - 1);
        if (32 * s + 32 <= a.N) {
            const uint8_t *w0 = a.w + 32 * s * a.wp, *s0 = a.ws + 32 * s * a.sp;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                wn[e] = *reinterpret_cast<const uint32_t *>(w0 + e * a.wp + w_at);
                sn[e] = *(s0 + e * a.sp + s_at);
            }
#pragma unroll
            for (int r = 0; r < RM; ++r) dn[r] = *reinterpret_cast<const u32x4 *>(dyr[r] + 32 * s + 8 * q);
        } else {
            const int n0 = 32 * s + 8 * q;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int64_t n = min(n0 + e, a.N - 1); // past the end dy counts as zero
                wn[e] = *reinterpret_cast<const uint32_t *>(a.w + n * a.wp + kc0 / 2 + 4 * i);
                sn[e] = a.ws[n * a.sp + kc0 / 32 + (i >> 2)];
            }
#pragma unroll
            for (int r = 0; r < RM; ++r) dn[r] = mx4_keep(*reinterpret_cast<const u32x4 *>(dyr[r] + min(n0, last)), a.N - n0);
        }
    };
    fetch(wave);
    for (int s = wave; s < steps; s += NW) {
        uint32_t w[8];
        float f[8];
        u32x4 d[RM], col[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = wn[e], f[e] = mx4_scale(sn[e]);
#pragma unroll
        for (int r = 0; r < RM; ++r) d[r] = dn[r];
        fetch(s + NW);
        mx4_columns(w, f, col);
#pragma unroll
        for (int r = 0; r < RM; ++r)
#pragma unroll
            for (int c = 0; c < 8; ++c)
                acc[c][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<bf16x8 *>(&col[c]), *reinterpret_cast<bf16x8 *>(&d[r]),
                                                                    acc[c][r], 0, 0, 0);
    }
    // lane (i, q): row i, columns 8 (4 q + v) + c
#pragma unroll
    for (int r = 0; r < RM; ++r)
#pragma unroll
        for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int c = 0; c < 8; c += 4)
                *reinterpret_cast<f32x4 *>(red + (wave * TM + 16 * r + i) * PITCH + 8 * (4 * q + v) + c) =
                    f32x4{acc[c][r][v], acc[c + 1][r][v], acc[c + 2][r][v], acc[c + 3][r][v]};
    __syncthreads();
    for (int e = threadIdx.x; e < TM * 128; e += 64 * NW) {
        const int m = e >> 7, c = e & 127;
        if (m0 + m >= a.M || kc0 + c >= a.K) continue;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) v += red[(w * TM + m) * PITCH + c];
        mx4_put(a, m0 + m, kc0 + c, v);
    }
}


// ---------------------------------------------------------------------------
// products of many rows: a workgroup's tile of 32 WM WTM rows by 32 WN WTN columns, wavefronts of WTM x WTN accumulators of 32 x 32.
// Both operands stream into a ring of LDS stages as they are stored (pac_mma.h: 16-byte transfers, swizzled chunks, counted waits):
// the 4-bit codes take a quarter of the space and of the LDS reads that bf16 would, and become bf16 in registers, eight a
// conversion group, between the matrix instructions of the piece before.  With x stored too both sides go to the scaled matrix
// instructions as they lie.  A lane (i, g) owns row i and, of each step, the blocks of its half g: one 16-byte read is a block of
// codes, and a lane has one scale a block.  Scales, eight bytes a row and 256 columns, come the same way into a ring of their own:
// loaded into registers they make the compiler, which does not count the transfers, wait for all of these at every use.
// 4096^3: 106 us, 1300 TFLOP/s (a library's bf16 product without the conversion: 98 us); 8192^3: 790 us, 1390 TFLOP/s
// (740 us with no transfers in the loop, on whatever LDS held).
// Fragment i of subtile y stands for column WTN i + y of the wavefront's, so that a lane ends up with WTN neighbouring columns.
// The 256 x 256 tiles of stored x take steps of 256 columns through two stages, half the barriers of steps of 128 through four:
// 4096 x 4096 x 16384 166 -> 161 us.  A step of theirs takes 2.07 us on the whole chip; 1.52 with no transfers, on whatever LDS
// held, so that up to a quarter is theirs (other operands may draw less power); its matrix instructions would take 0.98 at the rate
// that they reach alone.  Busy by counters: matrix units 39 %, LDS reads 18 %; what fills the rest is not settled.
// ---------------------------------------------------------------------------
template <bool X4_, int WM_, int WN_, int WTM_, int WTN_, int STAGES_, int BK_> struct Mx4Tile {
    static constexpr bool X4 = X4_;
    static constexpr int WM = WM_, WN = WN_, WTM = WTM_, WTN = WTN_, STAGES = STAGES_, NW = WM * WN;
    static constexpr int TM = 32 * WM * WTM, TN = 32 * WN * WTN;
    static constexpr int BK = BK_, PER = 256 / BK;   // columns a step, steps a group of 256
    static constexpr int AB = X4 ? BK / 2 : BK * 2, BB = BK / 2; // bytes of a row a step
    static constexpr int AI = TM * AB / 1024, TOTAL = AI + TN * BB / 1024, NI = (TOTAL + NW - 1) / NW;
    static constexpr int STAGE_BYTES = TM * AB + TN * BB;
    // scales: rows of W, then of x; rings deep enough that no group of 256 columns in use is written over
    static constexpr int SR = TN + (X4 ? TM : 0), STOTAL = SR / 32, SI = (STOTAL + NW - 1) / NW, RING = (STAGES - 1) / PER + 2;
    static constexpr int LDS_BYTES = STAGES * STAGE_BYTES + RING * SR * 8;
    static_assert(STAGES >= 2 && (NI + SI) * STAGES < 60, "transfers in flight must fit the counter");
    static constexpr bool AHEAD = WTM * WTN <= 4; // the next step's fragments are all read during this one's matrix instructions
};
// 4 bytes a lane from global memory into LDS, as dma16_at
__device__ __forceinline__ void dma4_at(const void *g, uint32_t lds_wave_address)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
                 : : "s"(__builtin_amdgcn_readfirstlane(lds_wave_address)), "v"(g) : "memory", "m0");
}
// chunk swizzle of rows of 256, 128, 64 and 32 bytes: the 16 rows that one pass of a 16-byte read covers meet every bank once
template <int BYTES> __device__ __forceinline__ int mx4_swz(int row)
{
    return BYTES == 256 ? row & 15 : BYTES == 128 ? (row >> 1) & 7 : BYTES == 64 ? (row >> 2) & 3 : (row >> 3) & 1;
}

// bf16 rows of a step that ends past the contraction's length: what lies there is cleared in LDS, before anyone reads it.  All
// threads call this, with the step's stage in place and a barrier behind it.
template <int ROWS, int BYTES, int THREADS> __device__ __forceinline__ void mx4_clip(char *stage, int valid)
{
    constexpr int CH = BYTES / 16;
    for (int e = threadIdx.x; e < ROWS * CH; e += THREADS) {
        const int row = e / CH, c = e % CH;
        if (8 * c + 8 <= valid) continue;
        u32x4 *p = reinterpret_cast<u32x4 *>(stage + row * BYTES + ((c ^ mx4_swz<BYTES>(row)) << 4));
        *p = mx4_keep(*p, valid - 8 * c);
    }
    __syncthreads();
}

// A die (blocks go round the eight of them) takes a run of tiles eight high, whose operands stay in its L2
__device__ __forceinline__ void mx4_place(int mt, int nt, int &tm, int &tn)
{
    const int all = nt * mt, die = blockIdx.x & 7;
    const int v = die * (all >> 3) + min(die, all & 7) + (blockIdx.x >> 3), mg = v / (8 * nt) * 8, high = min(8, mt - mg);
    tm = mg + v % (8 * nt) % high;
    tn = v % (8 * nt) / high;
}

// (two wavefronts a SIMD: with the 512 registers that one may have the compiler moves accumulators in and out at every instruction)
template <class TL> __global__ __launch_bounds__(64 * TL::NW, 2) void k_mx4_tiles(Mx4Args a)
{
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    constexpr int WTM = TL::WTM, WTN = TL::WTN;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / TL::WN, wn = wave % TL::WN, i = lane & 31, g = lane >> 5;
    int m0, n0;
    mx4_place((a.M + TL::TM - 1) / TL::TM, (a.N + TL::TN - 1) / TL::TN, m0, n0);
    m0 *= TL::TM;
    n0 *= TL::TN;
    const int nsteps = (a.K + TL::BK - 1) / TL::BK, ngroups = (nsteps + TL::PER - 1) / TL::PER;
    const int64_t xpitch = TL::X4 ? a.wp : a.ldx * 2;

    // this lane's share of a stage's transfers
    const char *gp[TL::NI];
    uint32_t goff[TL::NI], glim[TL::NI];
#pragma unroll
    for (int q = 0; q < TL::NI; ++q) {
        const int ii = min(wave + TL::NW * q, TL::TOTAL - 1);
        if (ii < TL::AI) {
            const int row = ii * (1024 / TL::AB) + lane / (TL::AB / 16);
            goff[q] = 16 * ((lane % (TL::AB / 16)) ^ mx4_swz<TL::AB>(row));
            gp[q] = reinterpret_cast<const char *>(a.x) + min(m0 + row, a.M - 1) * xpitch;
            glim[q] = TL::X4 ? 0x7fffffffu : 2u * ((a.K + 7) / 8 * 8 - 8); // x has no chunk past this one
        } else {
            const int row = (ii - TL::AI) * (1024 / TL::BB) + lane / (TL::BB / 16), w = row / (32 * WTN), y = row / 32 % WTN;
            goff[q] = 16 * ((lane % (TL::BB / 16)) ^ mx4_swz<TL::BB>(row));
            gp[q] = reinterpret_cast<const char *>(a.w) + min(n0 + w * 32 * WTN + (row & 31) * WTN + y, a.N - 1) * a.wp;
            glim[q] = 0x7fffffffu;
        }
    }
    // ... and of a group's scales: two lanes a row
    const uint8_t *sp[TL::SI];
#pragma unroll
    for (int q = 0; q < TL::SI; ++q) {
        const int row = min(wave + TL::NW * q, TL::STOTAL - 1) * 32 + lane / 2;
        if (row < TL::TN) {
            const int w = row / (32 * WTN), y = row / 32 % WTN;
            sp[q] = a.ws + min(n0 + w * 32 * WTN + (row & 31) * WTN + y, a.N - 1) * a.sp + 4 * (lane & 1);
        } else sp[q] = a.xs + min(m0 + row - TL::TN, a.M - 1) * a.sp + 4 * (lane & 1);
    }
    const uint32_t lds0 = lds_address(lds), ring0 = lds0 + TL::STAGES * TL::STAGE_BYTES;
    auto issue_scales = [&](int q, int step) {
        if (step % TL::PER == 0)
            dma4_at(sp[q] + 8 * min(step / TL::PER, ngroups - 1),
                    ring0 + step / TL::PER % TL::RING * (TL::SR * 8) + min(wave + TL::NW * q, TL::STOTAL - 1) * 256);
    };
    auto issue_rows = [&](int q, int slot, int step) {
        const int ii = min(wave + TL::NW * q, TL::TOTAL - 1);
        const uint32_t by = min(step, nsteps - 1) * (ii < TL::AI ? TL::AB : TL::BB); // past the end: the last step again, never used
        dma16_at(gp[q] + min(by + goff[q], glim[q]), lds0 + slot * TL::STAGE_BYTES + ii * 1024);
    };
    auto issue = [&](int slot, int step) {
#pragma unroll
        for (int q = 0; q < TL::SI; ++q) issue_scales(q, step);
#pragma unroll
        for (int q = 0; q < TL::NI; ++q) issue_rows(q, slot, step);
    };
#pragma unroll
    for (int s = 0; s < TL::STAGES; ++s) issue(s, s);

    f32x16 acc[WTM][WTN];
#pragma unroll
    for (int x = 0; x < WTM; ++x)
#pragma unroll
        for (int y = 0; y < WTN; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[x][y][v] = 0.f;
    int arow[WTM], brow[WTN], asw[WTM], bsw[WTN];
#pragma unroll
    for (int x = 0; x < WTM; ++x) {
        const int row = (wm * WTM + x) * 32 + i;
        arow[x] = row * TL::AB;
        asw[x] = mx4_swz<TL::AB>(row);
    }
#pragma unroll
    for (int y = 0; y < WTN; ++y) {
        const int row = (wn * WTN + y) * 32 + i;
        brow[y] = TL::TM * TL::AB + row * TL::BB;
        bsw[y] = mx4_swz<TL::BB>(row);
    }
    constexpr int BL = TL::BK / 64, J = TL::X4 ? BL : 4 * BL, FB = TL::AHEAD ? 2 * J : 2; // a lane's blocks a step, sub-steps, fragments held
    constexpr int CB = TL::AHEAD && !TL::X4 ? 2 * BL : 2; // steps' codes held beside bf16 rows, a lane's block each
    uint64_t bsc[WTN], asc[TL::X4 ? WTM : 1]; // this lane's half of a group's scales, shifted to the bottom
    u32x4 af[FB][WTM], bf[TL::X4 ? FB : CB][WTN]; // fragments; beside bf16 rows bf holds codes
    auto read_scales = [&](int grp, uint64_t (&bs)[WTN], uint64_t (&as)[TL::X4 ? WTM : 1]) {
        const char *sc = lds + TL::STAGES * TL::STAGE_BYTES + grp % TL::RING * (TL::SR * 8);
        const int half = 8 * BL * g;
#pragma unroll
        for (int y = 0; y < WTN; ++y) bs[y] = *reinterpret_cast<const uint64_t *>(sc + ((wn * WTN + y) * 32 + i) * 8) >> half;
        if constexpr (TL::X4)
#pragma unroll
            for (int x = 0; x < WTM; ++x) as[x] = *reinterpret_cast<const uint64_t *>(sc + (TL::TN + (wm * WTM + x) * 32 + i) * 8) >> half;
    };
    auto read_a = [&](const char *sb, int j, u32x4 (&to)[WTM]) {
#pragma unroll
        for (int x = 0; x < WTM; ++x) to[x] = *reinterpret_cast<const u32x4 *>(sb + arow[x] + (((J * g + j) ^ asw[x]) << 4));
    };
    auto read_b = [&](const char *sb, int j, u32x4 (&to)[WTN]) {
#pragma unroll
        for (int y = 0; y < WTN; ++y) to[y] = *reinterpret_cast<const u32x4 *>(sb + brow[y] + (((BL * g + j) ^ bsw[y]) << 4));
    };
    // the matrix instructions of a sub-step, `after(k)` behind the k-th of them
    auto multiply = [&](int u, int j, u32x4 (&pa)[WTM], const u32x4 (&pb)[WTN], auto after) __attribute__((always_inline)) {
        if constexpr (TL::X4) {
#pragma unroll
            for (int x = 0; x < WTM; ++x)
#pragma unroll
                for (int y = 0; y < WTN; ++y) {
                    const i32x8 p = {(int)pa[x][0], (int)pa[x][1], (int)pa[x][2], (int)pa[x][3], 0, 0, 0, 0};
                    const i32x8 q = {(int)pb[y][0], (int)pb[y][1], (int)pb[y][2], (int)pb[y][3], 0, 0, 0, 0};
                    const int sa = (int)(asc[x] >> (32 * u)), sc = (int)(bsc[y] >> (32 * u));
                    if (j == 0) acc[x][y] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(p, q, acc[x][y], 4, 4, 0, sa, 0, sc);
                    else if (j == 1) acc[x][y] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(p, q, acc[x][y], 4, 4, 1, sa, 1, sc);
                    else if (j == 2) acc[x][y] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(p, q, acc[x][y], 4, 4, 2, sa, 2, sc);
                    else acc[x][y] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(p, q, acc[x][y], 4, 4, 3, sa, 3, sc);
                    after(x * WTN + y);
                }
        } else {
            bf16x8 w[WTN];
#pragma unroll
            for (int y = 0; y < WTN; ++y) w[y] = mx4_bf16(pb[y][j % 4], mx4_scale((uint32_t)(bsc[y] >> (16 * BL * u + 8 * (j / 4))) & 255u));
#pragma unroll
            for (int x = 0; x < WTM; ++x)
#pragma unroll
                for (int y = 0; y < WTN; ++y) {
                    acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<bf16x8 *>(&pa[x]), w[y], acc[x][y], 0, 0, 0);
                    after(x * WTN + y);
                }
        }
    };
    // The transfers of the stage that takes a used one's place go between matrix instructions (k of m): issued in a row they keep
    // both wavefronts of a SIMD from issuing anything else.
    auto transfers = [&](int k, int m, int slot, int step) __attribute__((always_inline)) {
        constexpr int N = TL::SI + TL::NI;
#pragma unroll
        for (int q = k * N / m; q < (k + 1) * N / m; ++q) {
            if (q < TL::SI) issue_scales(q, step);
            else issue_rows(q - TL::SI, slot, step);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // hands over stage `step`: this wavefront's share of it, and of its scales, has landed, then everybody else's
    auto arrive = [&](char *stage, int step, auto pending) __attribute__((always_inline)) {
        wait_vm<decltype(pending)::value>();
        __syncthreads();
        if constexpr (!TL::X4)
            if (step == nsteps - 1 && a.K % TL::BK) mx4_clip<TL::TM, TL::AB, 64 * TL::NW>(stage, a.K - step * TL::BK);
    };
    arrive(lds, 0, std::integral_constant<int, TL::NI * (TL::STAGES - 1)>());
    read_scales(0, bsc, asc);
    int slot = 0;
    if constexpr (TL::AHEAD) {
        // Few matrix instructions a step: fragments are read a whole step ahead, else the latency of LDS shows at every sub-step
        // (64 x 64 tiles at K = 4096: 27 us a tile with sub-steps as below).
#pragma unroll
        for (int j = 0; j < J; ++j) {
            read_a(lds, j, af[j]);
            if (j < BL) read_b(lds, j, bf[j]);
        }
        for (int grp = 0; grp < ngroups; ++grp) {
#pragma unroll
            for (int u = 0; u < TL::PER; ++u) {
                const int st = grp * TL::PER + u;
                if (st >= nsteps) break;
                char *nb = lds + (slot + 1 == TL::STAGES ? 0 : slot + 1) * TL::STAGE_BYTES;
                arrive(nb, st + 1, std::integral_constant<int, TL::NI * (TL::STAGES - 2)>()); // (this stage has been read)
                uint64_t bsn[WTN], asn[TL::X4 ? WTM : 1];
                const int now = (u & 1) * J, next = J - now, nowb = (u & 1) * BL, nextb = BL - nowb;
                if (u == TL::PER - 1) read_scales(grp + 1, bsn, asn);
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    read_a(nb, j, af[next + j]);
                    if (j < BL) read_b(nb, j, bf[nextb + j]);
                }
                __builtin_amdgcn_sched_barrier(0); // the reads stay ahead of the matrix instructions
#pragma unroll
                for (int j = 0; j < J; ++j)
                    multiply(u, j, af[now + j], bf[nowb + (TL::X4 ? j : j / 4)], [&](int k) __attribute__((always_inline)) {
                        transfers(j * WTM * WTN + k, J * WTM * WTN, slot, st + TL::STAGES);
                    });
                if (u == TL::PER - 1) {
#pragma unroll
                    for (int y = 0; y < WTN; ++y) bsc[y] = bsn[y];
                    if constexpr (TL::X4)
#pragma unroll
                        for (int x = 0; x < WTM; ++x) asc[x] = asn[x];
                }
                slot = slot + 1 == TL::STAGES ? 0 : slot + 1;
            }
        }
    } else {
        // A step is walked in its J sub-steps, each reading the next one's fragments before its own matrix instructions.  The last
        // sub-step's come after the barrier that hands over the next stage, so that they cover the latency of that stage's first reads.
        read_a(lds, 0, af[0]);
        read_b(lds, 0, bf[0]);
        for (int grp = 0; grp < ngroups; ++grp) {
#pragma unroll
            for (int u = 0; u < TL::PER; ++u) {
                const int st = grp * TL::PER + u;
                if (st >= nsteps) break;
                const char *sb = lds + slot * TL::STAGE_BYTES;
                uint64_t bsn[WTN], asn[TL::X4 ? WTM : 1];
                u32x4 bn[WTN];
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    if (j + 1 < J) {
                        read_a(sb, j + 1, af[(j + 1) & 1]);
                        if constexpr (TL::X4) read_b(sb, j + 1, bf[(j + 1) & 1]);
                    } else {
                        __builtin_amdgcn_sched_barrier(0); // the matrix instructions so far go before the wait
                        char *nb = lds + (slot + 1 == TL::STAGES ? 0 : slot + 1) * TL::STAGE_BYTES;
                        arrive(nb, st + 1, std::integral_constant<int, TL::NI * (TL::STAGES - 2)>()); // (this stage has been read)
                        read_a(nb, 0, af[0]);
                        read_b(nb, 0, bn);
                        if (u == TL::PER - 1) read_scales(grp + 1, bsn, asn);
                    }
                    __builtin_amdgcn_sched_barrier(0); // the reads stay ahead of the matrix instructions
                    multiply(u, j, af[j & 1], bf[TL::X4 ? j & 1 : 0], [&](int k) __attribute__((always_inline)) {
                        if (j + 1 == J) transfers(k, WTM * WTN, slot, st + TL::STAGES);
                    });
                }
                slot = slot + 1 == TL::STAGES ? 0 : slot + 1;
#pragma unroll
                for (int y = 0; y < WTN; ++y) bf[0][y] = bn[y];
                if (u == TL::PER - 1) {
#pragma unroll
                    for (int y = 0; y < WTN; ++y) bsc[y] = bsn[y];
                    if constexpr (TL::X4)
#pragma unroll
                        for (int x = 0; x < WTM; ++x) asc[x] = asn[x];
                }
            }
        }
    }
    wait_vm<0>(); // the repeated transfers of the last steps end before the workgroup's LDS does

    mx4_write<WTM, WTN>(a, acc, m0 + wm * WTM * 32, n0 + wn * 32 * WTN + i * WTN, g, a.N);
}

// dx for many rows: a workgroup's tile of 32 WM WTM rows by 256 columns, W's rows in steps of 64.  dy and W's codes and scales stream
// into LDS as above.  W's step is turned round there, one step ahead, a part after each of the first three sub-steps' matrix
// instructions: a thread takes eight columns of four rows, converts them with each row's scale, and writes the four rows of each
// column side by side, as the fragments want them.  Stage t of the ring holds dy's step t and W's step t + 1.
// LDS row c 32 + i holds column 8 i + c: the writes of 32 threads and the reads of a fragment then go to neighbouring rows, and
// subtile c of lane i is column 8 i + c of the tile, WTN neighbouring ones a lane.  4096^3: 119 us, 1150 TFLOP/s; matrix units busy
// 53 % of the time, LDS reads 38 % (fragments of both sides in bf16; W's turned rows are written beside them), wavefronts waiting
// 26 %: neither unit is full, and what holds the loop is not settled.  (W through registers instead of LDS, in the same loop: 125 us.)
template <int WM_, int WN_, int WTM_, int WTN_, int STAGES_> struct Mx4DxTile {
    static constexpr int WM = WM_, WN = WN_, WTM = WTM_, WTN = WTN_, STAGES = STAGES_, NW = WM * WN;
    static constexpr int TM = 32 * WM * WTM, TK = 256;
    static constexpr int AI = TM / 8, TOTAL = AI + 8, NI = TOTAL / NW; // transfers of 1 KB: dy, then W's codes
    static constexpr int W_AT = TM * 128, S_AT = W_AT + 8192, STAGE_BYTES = S_AT + 512, B_BYTES = TK * 128;
    static constexpr int LDS_BYTES = STAGES * STAGE_BYTES + 2 * B_BYTES;
    static_assert(WN * WTN == 8 && NW == 8 && TOTAL % NW == 0, "256 columns, 512 threads");
    static_assert(STAGES >= 2 && (NI + 1) * STAGES < 60, "transfers in flight must fit the counter");
};

template <class TL> __global__ __launch_bounds__(64 * TL::NW, 2) void k_mx4_dx_tiles(Mx4Args a)
{
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    constexpr int WTM = TL::WTM, WTN = TL::WTN;
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    char *const bbuf = lds + TL::STAGES * TL::STAGE_BYTES;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / TL::WN, wn = wave % TL::WN, i = lane & 31, g = lane >> 5;
    int m0, k0;
    mx4_place((a.M + TL::TM - 1) / TL::TM, (a.K + TL::TK - 1) / TL::TK, m0, k0);
    m0 *= TL::TM;
    k0 *= TL::TK;
    const int nsteps = (a.N + 63) / 64;

    // this lane's share of a stage's transfers: wavefronts take 1 KB pieces in turn, eight rows of 128 bytes each
    const char *gp[TL::NI];
    uint32_t goff[TL::NI];
    const uint32_t glim = 2u * ((a.N + 7) / 8 * 8 - 8); // dy has no chunk past this one
#pragma unroll
    for (int q = 0; q < TL::NI; ++q) {
        const int ii = wave + TL::NW * q, row = ii * 8 + lane / 8;
        goff[q] = 16 * ((lane & 7) ^ mx4_swz<128>(row));
        gp[q] = reinterpret_cast<const char *>(a.x) + min(m0 + row, a.M - 1) * (a.ldx * 2);
    }
    const uint32_t lds0 = lds_address(lds);
    auto issue_rows = [&](int q, int slot, int step) {
        const int ii = wave + TL::NW * q;
        const uint32_t to = lds0 + slot * TL::STAGE_BYTES + ii * 1024;
        const int s = min(step, nsteps - 1); // past the end: the last step again, never used
        if (ii < TL::AI) dma16_at(gp[q] + min(128u * s + goff[q], glim), to);
        else {
            const int64_t n = min(64 * min(step + 1, nsteps - 1) + (ii - TL::AI) * 8 + lane / 8, a.N - 1); // past the end dy counts as zero
            dma16_at(a.w + n * a.wp + k0 / 2 + 16 * (lane & 7), to);
        }
    };
    auto issue_scales = [&](int slot, int step) { // two lanes a row, 32 rows a piece; the other wavefronts repeat the second piece
        const int piece = min(wave, 1);
        const int64_t n = min(64 * min(step + 1, nsteps - 1) + piece * 32 + lane / 2, a.N - 1);
        dma4_at(a.ws + n * a.sp + k0 / 32 + 4 * (lane & 1), lds0 + slot * TL::STAGE_BYTES + TL::S_AT + piece * 256);
    };
    // this thread's part of turning W: columns 8 cg .. 8 cg + 7, rows 4 ng .. 4 ng + 3 of a step; 32 lanes are 16 cg and two ng, whose
    // 8-byte writes fill each other's 16 bytes
    const int cg = (lane & 15) + 16 * g, ng = 2 * wave + ((lane >> 4) & 1);
    const int wat = cg * 128 + (((ng >> 1) ^ mx4_swz<128>(cg)) << 4) + 8 * (ng & 1); // where column 8 cg goes; the next: 4096 bytes on
    uint32_t wr[4], sr[4];
    auto turn = [&](auto c, char *to) __attribute__((always_inline)) {
        constexpr int C = decltype(c)::value;
        bf16x2 p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(wr[e], mx4_scale(sr[e]), C);
        *reinterpret_cast<u32x2 *>(to + wat + 8192 * C) = u32x2{pk_lo(p[0], p[1]), pk_lo(p[2], p[3])};
        *reinterpret_cast<u32x2 *>(to + wat + 8192 * C + 4096) = u32x2{pk_hi(p[0], p[1]), pk_hi(p[2], p[3])};
    };
    using c0 = std::integral_constant<int, 0>;
    using c1 = std::integral_constant<int, 1>;
    using c2 = std::integral_constant<int, 2>;
    using c3 = std::integral_constant<int, 3>;
    // W's first step comes through registers
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int64_t n = min(4 * ng + e, a.N - 1);
        wr[e] = *reinterpret_cast<const uint32_t *>(a.w + n * a.wp + k0 / 2 + 4 * cg);
        sr[e] = a.ws[n * a.sp + k0 / 32 + (cg >> 2)];
    }
    turn(c0(), bbuf);
    turn(c1(), bbuf);
    turn(c2(), bbuf);
    turn(c3(), bbuf);
#pragma unroll
    for (int s = 0; s < TL::STAGES; ++s) {
        issue_scales(s, s);
#pragma unroll
        for (int q = 0; q < TL::NI; ++q) issue_rows(q, s, s);
    }

    f32x16 acc[WTM][WTN];
#pragma unroll
    for (int x = 0; x < WTM; ++x)
#pragma unroll
        for (int y = 0; y < WTN; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[x][y][v] = 0.f;
    int arow[WTM];
#pragma unroll
    for (int x = 0; x < WTM; ++x) arow[x] = ((wm * WTM + x) * 32 + i) * 128;
    const int brow = (wn * WTN * 32 + i) * 128, swz = mx4_swz<128>(i); // (the swizzle repeats every 16 rows)
    u32x4 af[2][WTM], bf[2][WTN];
    auto read = [&](const char *sa, const char *sb, int j) {
#pragma unroll
        for (int x = 0; x < WTM; ++x) af[j & 1][x] = *reinterpret_cast<const u32x4 *>(sa + arow[x] + (((4 * g + j) ^ swz) << 4));
#pragma unroll
        for (int y = 0; y < WTN; ++y) bf[j & 1][y] = *reinterpret_cast<const u32x4 *>(sb + brow + y * 4096 + (((4 * g + j) ^ swz) << 4));
    };
    auto read_w = [&](const char *sa) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            wr[e] = *reinterpret_cast<const uint32_t *>(sa + TL::W_AT + (4 * ng + e) * 128 + 4 * cg);
            sr[e] = *reinterpret_cast<const uint8_t *>(sa + TL::S_AT + (4 * ng + e) * 8 + (cg >> 2));
        }
    };
    // hands over stage `step`: this wavefront's share of it has landed, then everybody else's
    auto arrive = [&](char *stage, int step, auto pending) __attribute__((always_inline)) {
        wait_vm<decltype(pending)::value>();
        __syncthreads();
        if (step == nsteps - 1 && a.N % 64) mx4_clip<TL::TM, 128, 64 * TL::NW>(stage, a.N - step * 64);
    };
    arrive(lds, 0, std::integral_constant<int, (TL::NI + 1) * (TL::STAGES - 1)>());
    read(lds, bbuf, 0);
    read_w(lds);
    int slot = 0;
    for (int st = 0; st < nsteps; ++st) {
        const char *sa = lds + slot * TL::STAGE_BYTES, *sb = bbuf + (st & 1) * TL::B_BYTES;
        char *to = bbuf + ((st + 1) & 1) * TL::B_BYTES;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j < 3) read(sa, sb, j + 1);
            else {
                __builtin_amdgcn_sched_barrier(0); // the matrix instructions so far go before the wait
                char *na = lds + (slot + 1 == TL::STAGES ? 0 : slot + 1) * TL::STAGE_BYTES;
                arrive(na, st + 1, std::integral_constant<int, (TL::NI + 1) * (TL::STAGES - 2)>()); // (this stage has been read, W's next step turned)
                read(na, to, 0);
                read_w(na);
            }
            __builtin_amdgcn_sched_barrier(0); // the reads stay ahead of the matrix instructions
#pragma unroll
            for (int x = 0; x < WTM; ++x)
#pragma unroll
                for (int y = 0; y < WTN; ++y) {
                    acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<bf16x8 *>(&af[j & 1][x]), *reinterpret_cast<bf16x8 *>(&bf[j & 1][y]),
                                                                        acc[x][y], 0, 0, 0);
                    if (j == 3) { // transfers between matrix instructions, as above
                        constexpr int N = TL::NI + 1, M = WTM * WTN;
                        const int k = x * WTN + y;
#pragma unroll
                        for (int q = k * N / M; q < (k + 1) * N / M; ++q) {
                            if (q == 0) issue_scales(slot, st + TL::STAGES);
                            else issue_rows(q - 1, slot, st + TL::STAGES);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            if (j == 0) turn(c0(), to), turn(c1(), to);
            else if (j == 1) turn(c2(), to);
            else if (j == 2) turn(c3(), to);
        }
        slot = slot + 1 == TL::STAGES ? 0 : slot + 1;
    }
    wait_vm<0>(); // the repeated transfers of the last steps end before the workgroup's LDS does
    mx4_write<WTM, WTN>(a, acc, m0 + wm * WTM * 32, k0 + 8 * i + WTN * wn, g, a.K);
}

static inline int64_t code_pitch(int cols) { return ((int64_t)cols + 255) / 256 * 128; }
static inline int64_t scale_pitch(int cols) { return ((int64_t)cols + 255) / 256 * 8; }
static inline bool dtype_ok(int32_t t) { return t == PAC_BF16 || t == PAC_F32; }

constexpr int32_t kMx4Most = 1 << 28; // rows and columns: places past a tile's end still fit 32 bits
// A launch takes fewer than 2^32 threads, blocks of all sizes counted together: with 512 a block these many tiles
constexpr int64_t kMx4Tiles = (1ll << 32) / 512 - 1;

// do a matrix, its codes and its scales share memory?
static bool stored_shares(const uint8_t *codes, const uint8_t *scales, int64_t rows, int32_t cols, const Span &x)
{
    const Span c(codes, rows * code_pitch(cols)), s(scales, rows * scale_pitch(cols));
    return shares(x, {c, s}) || share(c, s);
}

static pac_status check_convert(const void *x, int32_t dtype, int64_t rows, int32_t cols, int64_t stride, const uint8_t *codes,
                                const uint8_t *scales)
{
    if (rows != 0 && (!x || !codes || !scales)) return PAC_ERR_NULL; // an empty tensor has no address
    if (cols < 1 || !dtype_ok(dtype)) return PAC_ERR_SHAPE;
    if (rows < 0 || stride < cols) return PAC_ERR_RANGE;
    if (!m_aligned(x, dtype == PAC_F32 ? 4 : 2) || !m_aligned(codes, 16) || !m_aligned(scales, 8)) return PAC_ERR_ALIGN;
    if (cols > kMx4Most) return PAC_ERR_UNSUPPORTED;
    const int64_t upr = ((int64_t)cols + 255) / 256;
    if (rows > 0x7fffffffll / upr) return PAC_ERR_UNSUPPORTED;
    const int size = dtype == PAC_F32 ? 4 : 2;
    if (stored_shares(codes, scales, rows, cols, Span(x, rows, stride * size, (int64_t)cols * size))) return PAC_ERR_RANGE;
    return PAC_OK;
}

static pac_status done() { return hipGetLastError() == hipSuccess ? PAC_OK : PAC_ERR_DEVICE; }

static pac_status check_product(const void *x, int32_t M, int32_t K, int32_t N, const uint8_t *codes, const uint8_t *scales, const void *y,
                                int32_t y_dtype)
{
    if (!codes || !scales || (M != 0 && (!x || !y))) return PAC_ERR_NULL; // an empty tensor has no address
    if (M < 0 || K < 1 || N < 1 || !dtype_ok(y_dtype)) return PAC_ERR_SHAPE;
    if (M > kMx4Most || K > kMx4Most || N > kMx4Most) return PAC_ERR_UNSUPPORTED;
    if (!m_aligned(codes, 16) || !m_aligned(scales, 8) || !m_aligned(x, 16) || !m_aligned(y, y_dtype == PAC_F32 ? 4 : 2))
        return PAC_ERR_ALIGN;
    return PAC_OK;
}

// asked for once a kernel; where it was refused every launch of that kernel is an error
template <auto Kern> static hipError_t allow_lds_once(int lds)
{
    static std::once_flag once;
    static hipError_t result = hipSuccess;
    std::call_once(once, [&] {
        result = hipFuncSetAttribute(reinterpret_cast<const void *>(Kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    });
    return result;
}

template <class TL> static pac_status launch_tiles(const Mx4Args &a, hipStream_t st)
{
    const int64_t tiles = ((int64_t)a.N + TL::TN - 1) / TL::TN * (((int64_t)a.M + TL::TM - 1) / TL::TM);
    if (allow_lds_once<&k_mx4_tiles<TL>>(TL::LDS_BYTES) != hipSuccess) return PAC_ERR_DEVICE;
    hipLaunchKernelGGL((k_mx4_tiles<TL>), dim3((unsigned)tiles), dim3(64 * TL::NW), TL::LDS_BYTES, st, a);
    return done();
}

template <class TL> static pac_status launch_dx_tiles(const Mx4Args &a, hipStream_t st)
{
    const int64_t tiles = ((int64_t)a.K + TL::TK - 1) / TL::TK * (((int64_t)a.M + TL::TM - 1) / TL::TM);
    if (allow_lds_once<&k_mx4_dx_tiles<TL>>(TL::LDS_BYTES) != hipSuccess) return PAC_ERR_DEVICE;
    hipLaunchKernelGGL((k_mx4_dx_tiles<TL>), dim3((unsigned)tiles), dim3(64 * TL::NW), TL::LDS_BYTES, st, a);
    return done();
}

template <int X, int RM> static pac_status launch_rows(const Mx4Args &a, hipStream_t st)
{
    const int64_t tiles = ((int64_t)a.N + 15) / 16 * (((int64_t)a.M + 16 * RM - 1) / (16 * RM));
    hipLaunchKernelGGL((k_mx4_rows<X, RM, 8>), dim3((unsigned)tiles), dim3(512), 0, st, a);
    return done();
}
template <int RM> static pac_status launch_dx_rows(const Mx4Args &a, hipStream_t st)
{
    const int64_t tiles = ((int64_t)a.K + 127) / 128 * (((int64_t)a.M + 16 * RM - 1) / (16 * RM));
    constexpr int NW = 8, LDS = NW * 16 * RM * 132 * 4;
    if (allow_lds_once<&k_mx4_dx_rows<RM, NW>>(LDS) != hipSuccess) return PAC_ERR_DEVICE;
    hipLaunchKernelGGL((k_mx4_dx_rows<RM, NW>), dim3((unsigned)tiles), dim3(64 * NW), LDS, st, a);
    return done();
}

// Which tiles a product runs on.  For each form the time in us is estimated as  start + tile n + steps max(least, share n)  with n
// its tiles over 256 compute units (whole rounds where one tile fills a unit): a step's latency where units have less than one tile,
// its throughput where they have more.  The constants are fitted to all forms' times at 594 shapes (446 for dx; M to 4096, K to 8192,
// a multiple of 8, N to 16384; profiles/mx4_forms_times.csv): over the best one the form taken costs 0.3 % (x in bf16), 0.5 % (x in mx4)
// and 0.1 % (dx) on the geometric mean, and 25 %, 33 % and 11 % at the worst shape (665 x 200 x 695, 336 x 816 x 1434, 961 x 1120 x 1427).
// Both sides, us: x in bf16, 64 x 4096 x 4096: 16 rows 25, 64 x 64 14; 1024 x 1024 x 4096: 64 x 64 17.1, 64 x 128 13.5, 128 x 128
// 13.1, 256 x 256 25; 4096^3: 123 on 128 x 128, 106 on 256 x 256.  In mx4, 64 x 4096 x 4096: 32 rows 13.3, 64 x 64 8.5.
// dx, 333 x 4096 x 4096: 16 rows 40, 32 rows 37, 64 rows 62.
struct Mx4Form {
    int rows, cols, step; // of a tile; of the contraction (with 16 and 32 rows all of a workgroup's wavefronts together)
    bool whole;
    float start, tile, least, share;
};
constexpr Mx4Form kMx4Linear[] = {{16, 16, 1024, false, 1.02f, 0.f, 0.607f, 0.693f},
                                  {64, 64, 128, false, 4.86f, 0.91f, 0.15f, 0.429f},
                                  {64, 128, 128, false, 5.55f, 1.41f, 0.692f, 0.609f},
                                  {128, 128, 64, false, 6.48f, 1.64f, 0.768f, 0.594f},
                                  {256, 256, 64, true, 0.46f, 32.22f, 0.434f, 0.937f}};
constexpr Mx4Form kMx4LinearX4[] = {{16, 16, 1024, false, 2.35f, 0.f, 0.055f, 0.522f},
                                    {32, 16, 1024, false, 2.57f, 0.f, 0.461f, 0.705f},
                                    {64, 64, 128, false, 5.15f, 0.63f, 0.064f, 0.166f},
                                    {128, 128, 128, false, 7.87f, 2.39f, 0.279f, 0.422f},
                                    {256, 256, 256, true, 0.26f, 23.01f, 0.806f, 1.223f}};
constexpr Mx4Form kMx4Dx[] = {{16, 128, 256, false, 4.06f, 0.58f, 0.035f, 0.801f},
                              {32, 128, 256, false, 3.55f, 3.64f, 0.876f, 0.993f},
                              {64, 256, 64, true, 2.04f, 5.51f, 0.285f, 0.75f},
                              {128, 256, 64, true, 0.04f, 8.42f, 0.101f, 0.897f},
                              {256, 256, 64, true, 1.19f, 6.65f, 0.763f, 1.608f}};

// the form for a product of M x `deep` by `deep` x `wide`: of those whose tiles one launch takes the one that is estimated fastest (of
// all of them where it takes none's, which the launch then refuses)
template <int F> static const Mx4Form &mx4_form(const Mx4Form (&forms)[F], int64_t M, int64_t deep, int64_t wide)
{
    const Mx4Form *best = nullptr;
    float least = 0.f;
    bool best_fits = false;
    for (const Mx4Form &q : forms) {
        const int64_t tiles = ((M + q.rows - 1) / q.rows) * ((wide + q.cols - 1) / q.cols);
        const bool fits = tiles <= kMx4Tiles;
        const float n = q.whole ? (float)((tiles + 255) / 256) : (float)tiles / 256.f, steps = (float)((deep + q.step - 1) / q.step);
        const float t = q.start + q.tile * n + steps * (q.least > q.share * n ? q.least : q.share * n);
        if (!best || (fits == best_fits ? t < least : fits)) best = &q, least = t, best_fits = fits;
    }
    return *best;
}
static bool fits_launch(const Mx4Form &q, int64_t M, int64_t wide)
{
    return ((M + q.rows - 1) / q.rows) * ((wide + q.cols - 1) / q.cols) <= kMx4Tiles;
}
// the results, and whether they lie over W or the bias
static Span results(const Mx4Args &a, int64_t wide) { return Span(a.y, a.M, a.ldy * (a.y_f32 ? 4 : 2), wide * (a.y_f32 ? 4 : 2)); }
static bool over_weights(const Mx4Args &a, const Span &out)
{
    return shares(out, {Span(a.w, a.N * a.wp), Span(a.ws, a.N * a.sp), Span(a.bias, (int64_t)a.N * 4)});
}
static const Mx4Form &linear_form(bool x4, int M, int K, int N) { return x4 ? mx4_form(kMx4LinearX4, M, K, N) : mx4_form(kMx4Linear, M, K, N); }
static const Mx4Form &dx_form(int M, int K, int N) { return mx4_form(kMx4Dx, M, N, K); }

template <bool X4> static pac_status launch_linear(const Mx4Args &a, hipStream_t st)
{
    (void)hipGetLastError();
    const Mx4Form &form = linear_form(X4, a.M, a.K, a.N);
    if (!fits_launch(form, a.M, a.N)) return PAC_ERR_UNSUPPORTED;
    const Span y = results(a, a.N);
    if (over_weights(a, y) || (X4 ? shares(y, {Span(a.x, a.M * a.wp), Span(a.xs, a.M * a.sp)}) : share(y, Span(a.x, a.M, a.ldx * 2, (int64_t)a.K * 2))))
        return PAC_ERR_RANGE;
    switch (form.rows + form.cols) {
    case 16 + 16: return launch_rows<X4 ? MX4_X4 : MX4_X16, 1>(a, st);
    case 32 + 16: if constexpr (X4) return launch_rows<MX4_X4, 2>(a, st); [[fallthrough]];
    case 64 + 64: return launch_tiles<Mx4Tile<X4, 2, 2, 1, 1, X4 ? 4 : 3, 128>>(a, st);
    case 64 + 128: if constexpr (!X4) return launch_tiles<Mx4Tile<X4, 2, 2, 1, 2, X4 ? 4 : 3, 128>>(a, st); [[fallthrough]];
    case 128 + 128: return launch_tiles<Mx4Tile<X4, 2, 2, 2, 2, X4 ? 4 : 3, X4 ? 128 : 64>>(a, st);
    default: return launch_tiles<Mx4Tile<X4, 2, 4, 4, 2, X4 ? 2 : 3, X4 ? 256 : 64>>(a, st);
    }
}

static pac_status launch_dx(const Mx4Args &a, hipStream_t st)
{
    (void)hipGetLastError();
    const Mx4Form &form = dx_form(a.M, a.K, a.N);
    if (!fits_launch(form, a.M, a.K)) return PAC_ERR_UNSUPPORTED;
    const Span dx = results(a, a.K);
    if (over_weights(a, dx) || share(dx, Span(a.x, a.M, a.ldx * 2, (int64_t)a.N * 2))) return PAC_ERR_RANGE;
    switch (form.rows) {
    case 16: return launch_dx_rows<1>(a, st);
    case 32: return launch_dx_rows<2>(a, st);
    case 64: return launch_dx_tiles<Mx4DxTile<2, 4, 1, 2, 5>>(a, st);
    case 128: return launch_dx_tiles<Mx4DxTile<2, 4, 2, 2, 3>>(a, st);
    default: return launch_dx_tiles<Mx4DxTile<4, 2, 2, 4, 2>>(a, st);
    }
}

// The conversions' kernels take 32 threads a group of 256 columns, so that one launch takes fewer than 2^27 groups: more rows go in
// several, of this many groups at most.  call(first row, groups of its rows)
constexpr int64_t kMx4Groups = 1 << 26;
template <class Call> static pac_status by_rows(int64_t rows, int32_t cols, Call call)
{
    const int64_t upr = ((int64_t)cols + 255) / 256, step = kMx4Groups / upr; // (a row has 2^20 groups at most)
    for (int64_t r = 0; r < rows; r += step) {
        call(r, (uint32_t)((rows - r < step ? rows - r : step) * upr));
        const pac_status s = done();
        if (s != PAC_OK) return s;
    }
    return PAC_OK;
}

static pac_status launch_quant(const void *x, int32_t x_dtype, int64_t rows, int32_t cols, int64_t x_stride, uint8_t *codes, uint8_t *scales,
                               hipStream_t st)
{
    const uint32_t upr = (uint32_t)(((int64_t)cols + 255) / 256);
    const bool vec = m_aligned(x, 16) && x_stride % (x_dtype == PAC_F32 ? 4 : 8) == 0;
    return by_rows(rows, cols, [&](int64_t row, uint32_t units) {
        const dim3 g((units + 7) / 8), b(256);
        uint32_t *c = reinterpret_cast<uint32_t *>(codes) + row * upr * 32;
        uint8_t *s = scales + row * upr * 8;
        if (x_dtype == PAC_F32) {
            const float *p = static_cast<const float *>(x) + row * x_stride;
            if (vec) hipLaunchKernelGGL((k_mx4_quant<float, true>), g, b, 0, st, p, units, upr, cols, x_stride, c, s);
            else hipLaunchKernelGGL((k_mx4_quant<float, false>), g, b, 0, st, p, units, upr, cols, x_stride, c, s);
        } else {
            const bf16_t *p = static_cast<const bf16_t *>(x) + row * x_stride;
            if (vec) hipLaunchKernelGGL((k_mx4_quant<bf16_t, true>), g, b, 0, st, p, units, upr, cols, x_stride, c, s);
            else hipLaunchKernelGGL((k_mx4_quant<bf16_t, false>), g, b, 0, st, p, units, upr, cols, x_stride, c, s);
        }
    });
}

static pac_status launch_dequant(const uint8_t *codes, const uint8_t *scales, int64_t rows, int32_t cols, void *out, int32_t out_dtype,
                                 int64_t out_stride, hipStream_t st)
{
    const uint32_t upr = (uint32_t)(((int64_t)cols + 255) / 256);
    const bool vec = m_aligned(out, 16) && out_stride % (out_dtype == PAC_F32 ? 4 : 8) == 0;
    return by_rows(rows, cols, [&](int64_t row, uint32_t units) {
        const dim3 g((units + 7) / 8), b(256);
        const uint32_t *c = reinterpret_cast<const uint32_t *>(codes) + row * upr * 32;
        const uint8_t *s = scales + row * upr * 8;
        if (out_dtype == PAC_F32) {
            float *p = static_cast<float *>(out) + row * out_stride;
            if (vec) hipLaunchKernelGGL((k_mx4_dequant<float, true>), g, b, 0, st, c, s, units, upr, cols, p, out_stride);
            else hipLaunchKernelGGL((k_mx4_dequant<float, false>), g, b, 0, st, c, s, units, upr, cols, p, out_stride);
        } else {
            bf16_t *p = static_cast<bf16_t *>(out) + row * out_stride;
            if (vec) hipLaunchKernelGGL((k_mx4_dequant<bf16_t, true>), g, b, 0, st, c, s, units, upr, cols, p, out_stride);
            else hipLaunchKernelGGL((k_mx4_dequant<bf16_t, false>), g, b, 0, st, c, s, units, upr, cols, p, out_stride);
        }
    });
}

} // namespace pac

using namespace pac;

extern "C" {

int64_t pac_mx4_code_pitch(int32_t cols) { return cols < 1 ? -1 : code_pitch(cols); }
int64_t pac_mx4_scale_pitch(int32_t cols) { return cols < 1 ? -1 : scale_pitch(cols); }

pac_status pac_mx4_quantize(const void *x, int32_t x_dtype, int64_t rows, int32_t cols, int64_t x_stride, uint8_t *codes,
                            uint8_t *scales, void *hip_stream)
{
    const pac_status s = check_convert(x, x_dtype, rows, cols, x_stride, codes, scales);
    if (s != PAC_OK || rows == 0) return s;
    (void)hipGetLastError();
    return launch_quant(x, x_dtype, rows, cols, x_stride, codes, scales, static_cast<hipStream_t>(hip_stream));
}

pac_status pac_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int32_t cols, void *out, int32_t out_dtype,
                              int64_t out_stride, void *hip_stream)
{
    const pac_status s = check_convert(out, out_dtype, rows, cols, out_stride, codes, scales);
    if (s != PAC_OK || rows == 0) return s;
    (void)hipGetLastError();
    return launch_dequant(codes, scales, rows, cols, out, out_dtype, out_stride, static_cast<hipStream_t>(hip_stream));
}

pac_status pac_mx4_linear(const void *x, int32_t M, int32_t K, int64_t x_stride, const uint8_t *codes, const uint8_t *scales, int32_t N,
                          const float *bias, int32_t act, void *y, int32_t y_dtype, int64_t y_stride, void *hip_stream)
{
    const pac_status s = check_product(x, M, K, N, codes, scales, y, y_dtype);
    if (s != PAC_OK) return s;
    if (act != PAC_MX4_ACT_NONE && act != PAC_MX4_ACT_GELU) return PAC_ERR_SHAPE;
    if (x_stride < K || y_stride < N) return PAC_ERR_RANGE;
    if (x_stride % 8 || !m_aligned(bias, 4)) return PAC_ERR_ALIGN;
    if (M == 0) return PAC_OK;
    return launch_linear<false>(Mx4Args{x, nullptr, x_stride, codes, scales, M, K, N, code_pitch(K), scale_pitch(K), bias, act, y,
                                        y_dtype == PAC_F32, y_stride}, static_cast<hipStream_t>(hip_stream));
}

pac_status pac_mx4_linear_x4(const uint8_t *x_codes, const uint8_t *x_scales, int32_t M, int32_t K, const uint8_t *codes,
                             const uint8_t *scales, int32_t N, const float *bias, int32_t act, void *y, int32_t y_dtype,
                             int64_t y_stride, void *hip_stream)
{
    if (M != 0 && !x_scales) return PAC_ERR_NULL;
    const pac_status s = check_product(x_codes, M, K, N, codes, scales, y, y_dtype);
    if (s != PAC_OK) return s;
    if (act != PAC_MX4_ACT_NONE && act != PAC_MX4_ACT_GELU) return PAC_ERR_SHAPE;
    if (y_stride < N) return PAC_ERR_RANGE;
    if (!m_aligned(x_scales, 8) || !m_aligned(bias, 4)) return PAC_ERR_ALIGN;
    if (M == 0) return PAC_OK;
    return launch_linear<true>(Mx4Args{x_codes, x_scales, 0, codes, scales, M, K, N, code_pitch(K), scale_pitch(K), bias, act, y,
                                       y_dtype == PAC_F32, y_stride}, static_cast<hipStream_t>(hip_stream));
}

int64_t pac_mx4_linear_qx_workspace_bytes(int32_t M, int32_t K)
{
    if (M < 0 || K < 1 || M > kMx4Most || K > kMx4Most) return -1;
    return (int64_t)M * (code_pitch(K) + scale_pitch(K));
}

pac_status pac_mx4_linear_qx(const void *x, int32_t x_dtype, int32_t M, int32_t K, int64_t x_stride, const uint8_t *codes,
                             const uint8_t *scales, int32_t N, const float *bias, int32_t act, void *y, int32_t y_dtype, int64_t y_stride,
                             void *workspace, int64_t workspace_bytes, void *hip_stream)
{
    if (!codes || !scales || (M != 0 && (!x || !y || !workspace))) return PAC_ERR_NULL;
    if (M < 0 || K < 1 || N < 1 || !dtype_ok(x_dtype) || !dtype_ok(y_dtype) || (act != PAC_MX4_ACT_NONE && act != PAC_MX4_ACT_GELU))
        return PAC_ERR_SHAPE;
    if (M > kMx4Most || K > kMx4Most || N > kMx4Most) return PAC_ERR_UNSUPPORTED;
    if (x_stride < K || y_stride < N) return PAC_ERR_RANGE;
    if (!m_aligned(x, x_dtype == PAC_F32 ? 4 : 2) || !m_aligned(codes, 16) || !m_aligned(scales, 8) || !m_aligned(bias, 4) ||
        !m_aligned(y, y_dtype == PAC_F32 ? 4 : 2) || !m_aligned(workspace, 16))
        return PAC_ERR_ALIGN;
    if (M == 0) return PAC_OK;
    if (workspace_bytes < pac_mx4_linear_qx_workspace_bytes(M, K)) return PAC_ERR_WORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    Mx4Args a{x, nullptr, x_stride, codes, scales, M, K, N, code_pitch(K), scale_pitch(K), bias, act, y, y_dtype == PAC_F32, y_stride};
    (void)hipGetLastError();
    const Mx4Form &form = linear_form(true, M, K, N);
    if (!fits_launch(form, M, N)) return PAC_ERR_UNSUPPORTED;
    const int size = x_dtype == PAC_F32 ? 4 : 2;
    const Span rows(x, M, x_stride * size, (int64_t)K * size), y_rows = results(a, N), ws(workspace, pac_mx4_linear_qx_workspace_bytes(M, K));
    if (over_weights(a, y_rows) || over_weights(a, ws) || share(y_rows, rows) || share(ws, rows) || share(ws, y_rows)) return PAC_ERR_RANGE;
    // few rows in whole 16-byte pieces: quantised where they are multiplied (one launch)
    if (form.rows <= 32 && x_dtype == PAC_BF16 && K % 8 == 0 && x_stride % 8 == 0 && m_aligned(x, 16))
        return form.rows == 16 ? launch_rows<MX4_XQ, 1>(a, st) : launch_rows<MX4_XQ, 2>(a, st);
    uint8_t *xc = static_cast<uint8_t *>(workspace), *xs = xc + (int64_t)M * a.wp; // rows of codes are whole multiples of 128 bytes
    if ((int64_t)M > 0x7fffffffll / (a.wp / 128)) return PAC_ERR_UNSUPPORTED;
    const pac_status s = launch_quant(x, x_dtype, M, K, x_stride, xc, xs, st);
    if (s != PAC_OK) return s;
    a.x = xc;
    a.xs = xs;
    return launch_linear<true>(a, st);
}

pac_status pac_mx4_tiles(int32_t product, int32_t M, int32_t K, int32_t N, int32_t out[2])
{
    if (!out) return PAC_ERR_NULL;
    if (product < PAC_MX4_LINEAR || product > PAC_MX4_LINEAR_DX || M < 1 || K < 1 || N < 1) return PAC_ERR_SHAPE;
    if (M > kMx4Most || K > kMx4Most || N > kMx4Most) return PAC_ERR_UNSUPPORTED;
    const Mx4Form &f = product == PAC_MX4_LINEAR_DX ? dx_form(M, K, N) : linear_form(product == PAC_MX4_LINEAR_X4, M, K, N);
    out[0] = f.rows;
    out[1] = f.cols;
    return PAC_OK;
}

pac_status pac_mx4_linear_dx(const void *dy, int32_t M, int32_t N, int64_t dy_stride, const uint8_t *codes, const uint8_t *scales,
                             int32_t K, void *dx, int32_t dx_dtype, int64_t dx_stride, void *hip_stream)
{
    const pac_status s = check_product(dy, M, K, N, codes, scales, dx, dx_dtype);
    if (s != PAC_OK) return s;
    if (dy_stride < N || dx_stride < K) return PAC_ERR_RANGE;
    if (dy_stride % 8) return PAC_ERR_ALIGN;
    if (M == 0) return PAC_OK;
    const Mx4Args a{dy, nullptr, dy_stride, codes, scales, M, K, N, code_pitch(K), scale_pitch(K), nullptr, 0, dx, dx_dtype == PAC_F32,
                    dx_stride};
    return launch_dx(a, static_cast<hipStream_t>(hip_stream));
}

} // extern "C"
