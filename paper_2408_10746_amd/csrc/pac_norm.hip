// Norms before and after a block, fused with the block's gate and the scale of the residual path, and their gradients (declared
// in include/pac_norm.h).
#include "../../include/pac_norm.h"
#include "pac_gemm.h"
#include "pac_span.h"

namespace pac {

struct NormArgs {
    const void *x, *o, *dy, *dn;
    void *y, *n;   // forward
    void *dx, *d_o; // backward
    const float *w_post, *b_post, *gate, *res, *w_pre, *b_pre;
    int64_t rows;
    int d, gate_len;
    float eps, inv_d;
    float *cols;   // backward: [G][nv][d] partial sums of the columns: N(o) g, g, N(y) dn, dn, those that are wanted
    double *scal;  // backward: [G][2] partial sums of g x and g p
    int nv, v_a, v_b, v_c, v_d; // vectors of cols, and which is which (-1: not wanted)
};

// Sum over a wavefront, the same bits on every lane: four rotations inside rows of 16 lanes, then the four rows' sums in order.
// (Lane exchanges through LDS take six round trips for it; a row needs up to four such sums one after the other.)
template <int R> __device__ __forceinline__ float add_ror(float v) // v + v of the lane R to the side, in rows of 16
{
    return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x120 + R, 0xf, 0xf, false));
}
__device__ __forceinline__ float wave_sum(float v)
{
    v = add_ror<1>(add_ror<2>(add_ror<4>(add_ror<8>(v))));
    auto at = [&](int l) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), l)); };
    return (at(0) + at(16)) + (at(32) + at(48));
}

// sums of a row's NS values over its TPR threads, on all of them; `red` belongs to the row, [2][TPR / 64][2], `turn` alternates
// so that one barrier a sum is enough
template <int TPR, int NS> __device__ __forceinline__ void row_sums(float (&s)[NS], float *red, int &turn)
{
#pragma unroll
    for (int k = 0; k < NS; ++k) s[k] = wave_sum(s[k]);
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        float *r = red + turn * W * 2;
        turn ^= 1;
        const int wave = (threadIdx.x % TPR) >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < NS; ++k) r[k * W + wave] = s[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NS; ++k) {
            s[k] = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) s[k] += r[k * W + w];
        }
    }
}

// E values of a row a thread, in chunks of VEC neighbours: chunk c holds columns (c TPR + t) VEC and the VEC - 1 after it
template <typename T, int VEC, int TPR, int E> struct RowIO {
    static constexpr int CH = E / VEC;
    typedef T vec __attribute__((ext_vector_type(VEC)));
    struct Raw { vec v[CH]; }; // as it comes from memory: the coming row waits in this form while the present one is worked on
    static __device__ __forceinline__ int col(int t, int c) { return (c * TPR + t) * VEC; }
    static __device__ __forceinline__ bool in(int t, int e, int d) { return col(t, e / VEC) + e % VEC < d; }
    static __device__ __forceinline__ void fetch(Raw &r, const void *p, int64_t row, int d, int t)
    {
        const T *src = reinterpret_cast<const T *>(p) + row * d;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int j = col(t, c);
            // past the row's end: its first values, which widen() leaves out (d is a multiple of VEC)
            r.v[c] = *reinterpret_cast<const vec *>(src + (j < d ? j : 0));
        }
    }
    static __device__ __forceinline__ void widen(const Raw &r, int d, int t, float (&v)[E])
    {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = in(t, e, d) ? (float)r.v[e / VEC][e % VEC] : 0.f;
    }
    static __device__ __forceinline__ void store(void *p, int64_t row, int d, int t, const float (&v)[E])
    {
        T *dst = reinterpret_cast<T *>(p) + row * d;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int j = col(t, c);
            if (j >= d) continue;
            vec r;
#pragma unroll
            for (int e = 0; e < VEC; ++e) r[e] = (T)v[c * VEC + e];
            *reinterpret_cast<vec *>(dst + j) = r;
        }
    }
    // a parameter's values at this thread's columns (`none` where there is no such parameter; anything where no such column)
    static __device__ __forceinline__ void param(const float *p, int d, int t, float none, float (&v)[E])
    {
        constexpr int PV = VEC >= 4 ? 4 : 1;
        typedef float pv __attribute__((ext_vector_type(PV)));
#pragma unroll
        for (int e = 0; e < E; e += PV) {
            const int j = col(t, e / VEC) + e % VEC;
            pv r;
            if (p) r = *reinterpret_cast<const pv *>(p + (j < d ? j : 0));
#pragma unroll
            for (int k = 0; k < PV; ++k) v[e + k] = p ? r[k] : none;
        }
    }
};

// N(v): v becomes the normalised row; returns 1 / its deviation.  Two passes over registers: the mean first, then the squares of
// what is left of it, so that a row far from zero loses nothing.
template <int TPR, int E, class IO, bool LAYER>
__device__ __forceinline__ float normalise(float (&v)[E], const NormArgs &a, int t, float *red, int &turn)
{
    float s[1];
    if constexpr (LAYER) {
        s[0] = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) s[0] += v[e];
        row_sums<TPR, 1>(s, red, turn);
        const float mean = s[0] * a.inv_d;
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = IO::in(t, e, a.d) ? v[e] - mean : 0.f;
    }
    s[0] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s[0] = fmaf(v[e], v[e], s[0]);
    row_sums<TPR, 1>(s, red, turn);
    const float r = 1.f / sqrtf(s[0] * a.inv_d + a.eps);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] *= r;
    return r;
}

// g becomes the gradient of N's input, given that of its output; h: N's output, r: 1 / deviation
template <int TPR, int E, class IO, bool LAYER>
__device__ __forceinline__ void norm_back(float (&g)[E], const float (&h)[E], float r, const NormArgs &a, float *red, int &turn)
{
    float along, mean = 0.f;
    if constexpr (LAYER) {
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < E; ++e) s[0] = fmaf(g[e], h[e], s[0]), s[1] += g[e];
        row_sums<TPR, 2>(s, red, turn);
        along = s[0] * a.inv_d;
        mean = s[1] * a.inv_d;
    } else {
        float s[1] = {0.f};
#pragma unroll
        for (int e = 0; e < E; ++e) s[0] = fmaf(g[e], h[e], s[0]);
        row_sums<TPR, 1>(s, red, turn);
        along = s[0] * a.inv_d;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) g[e] = r * (g[e] - mean - h[e] * along);
}

template <int TPR> constexpr int kRowsPerBlock = TPR < 512 ? 512 / TPR : 1;
template <int TPR> constexpr int kNormThreads = TPR < 512 ? 512 : TPR;

// Forward: a row is loaded once, lives in registers through both norms, and y and n are stored from there: two reads and two writes
// a value, the least there is.  Blocks go through rows with the next row's loads under way.  Memory bounds it: 16384 x 4096 bf16 in
// 104 us is 5.2 TB/s, what a copy reaches; one row of 4096 takes 2.9 us, a launch's time.  (16 values a thread and the parameters
// read at every row: 116 us.)
// HOLD: the parameters stay in registers from row to row, loaded along with the first row; else (rows past 8192, whose values fill
// the registers) they are loaded for every row.  The 16 values a thread of those rows do not fit beside it all the same: 280 to 408 bytes a
// lane go to scratch (some 1050 with single loads), and 4096 x 16384 bf16 takes 318 us, 1.7 TB/s; 4096 x 8192 46 us.
template <typename T, int VEC, int TPR, int E, bool LAYER, bool HOLD> __global__ __launch_bounds__(kNormThreads<TPR>) void k_norm_fwd(NormArgs a)
{
    constexpr int RPB = kRowsPerBlock<TPR>;
    using IO = RowIO<T, VEC, TPR, E>;
    __shared__ __attribute__((aligned(16))) float redm[RPB * 2 * (TPR / 64) * 2];
    const int t = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    float *red = redm + slot * 2 * (TPR / 64) * 2;
    int turn = 0;
    const int64_t stride = (int64_t)gridDim.x * RPB;
    // every thread of a block goes round as often (barriers): a slot whose row is past the end works on the last one, unstored
    int64_t row0 = (int64_t)blockIdx.x * RPB;
    auto clamp = [&](int64_t r) { return r < a.rows ? r : a.rows - 1; };
    const void *const po = a.o ? a.o : a.x; // what is not there is not used
    typename IO::Raw rx, ro;
    IO::fetch(rx, a.x, clamp(row0 + slot), a.d, t);
    IO::fetch(ro, po, clamp(row0 + slot), a.d, t);
    const float res = a.res ? a.res[0] : 1.f, g0 = a.gate_len == 1 ? a.gate[0] : 1.f;
    float wo[E], bo[E], gt[E], wn[E], bn[E];
    auto params = [&] {
        IO::param(a.w_post, a.d, t, 1.f, wo);
        IO::param(a.b_post, a.d, t, 0.f, bo);
        IO::param(a.gate_len > 1 ? a.gate : nullptr, a.d, t, g0, gt);
        IO::param(a.w_pre, a.d, t, 0.f, wn);
        IO::param(a.b_pre, a.d, t, 0.f, bn);
    };
    if constexpr (HOLD) params();
    for (; row0 < a.rows; row0 += stride) {
        const bool live = row0 + slot < a.rows;
        const int64_t row = clamp(row0 + slot);
        float y[E], o[E];
        IO::widen(rx, a.d, t, y);
        IO::widen(ro, a.d, t, o);
        if constexpr (!HOLD) params();
        if (row0 + stride < a.rows) {
            const int64_t next = clamp(row0 + stride + slot);
            IO::fetch(rx, a.x, next, a.d, t);
            IO::fetch(ro, po, next, a.d, t);
        }
        if (a.o) {
            if (a.w_post) {
                normalise<TPR, E, IO, LAYER>(o, a, t, red, turn);
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] = fmaf(o[e], wo[e], bo[e]);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = fmaf(res, y[e], gt[e] * o[e]);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] *= res;
        }
        if (a.y && live) IO::store(a.y, row, a.d, t, y);
        if (a.w_pre) {
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = IO::in(t, e, a.d) ? y[e] : 0.f; // (a parameter has any value past the row's end)
            normalise<TPR, E, IO, LAYER>(y, a, t, red, turn);
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = fmaf(y[e], wn[e], bn[e]);
            if (live) IO::store(a.n, row, a.d, t, y);
        }
    }
}

// Backward: y and both norms are made again from x and o (nothing is saved by the forward pass: a row in registers costs no memory
// traffic), then the gradients go back through them; four reads and two writes a value.  Sums over rows stay with the columns'
// threads, one partial sum a block and column, added by k_norm_sums: no atomics, the same bits each time.  4096 x 4096 bf16 in 50
// us is 4.0 TB/s, then 4.4 us of sums; what bounds it is a row's chain of four sums over 16 wavefronts, one block a compute unit.
// Four values a thread and the parameters held: 8 a thread with parameters read at every row 51 us at 4096 and 35 against 19 us at
// 2723 x 768 fp32, held at 8 a thread 66 us; 16 a thread 142 us; two rows under way 53 us.
// Rows past 4096 take 8 a thread and past 8192 16, and their values go to scratch in part, the parameters read at every row or not: 96 to
// 280 and 544 to 896 bytes a lane, up to 1724 with single loads.  bf16: 4096 x 5120 110 us (2.3 TB/s), 4096 x 8192 135 us (3.0),
// 4096 x 16384 895 us (0.9); with single loads 4096 x 8191 517 us, 4096 x 16383 1960 us.
// SHIFT: sums of g and of dn for the shifts' gradients (b_post, b_pre) are wanted too
template <typename T, int VEC, int TPR, int E, bool LAYER, bool SHIFT, bool HOLD>
__global__ __launch_bounds__(kNormThreads<TPR>, 4) void k_norm_bwd(NormArgs a)
{
    constexpr int RPB = kRowsPerBlock<TPR>, W = RPB * TPR / 64;
    using IO = RowIO<T, VEC, TPR, E>;
    __shared__ __attribute__((aligned(16))) float redm[RPB * 2 * (TPR / 64) * 2];
    __shared__ double sred[2 * W];
    __shared__ float join[RPB > 1 ? RPB * TPR * E : 1];
    const int t = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    float *red = redm + slot * 2 * (TPR / 64) * 2;
    int turn = 0;
    const int64_t stride = (int64_t)gridDim.x * RPB;
    int64_t row0 = (int64_t)blockIdx.x * RPB;
    auto clamp = [&](int64_t r) { return r < a.rows ? r : a.rows - 1; };
    const void *const po = a.o ? a.o : a.x, *const pn = a.dn ? a.dn : a.x, *const py = a.dy ? a.dy : a.x; // what is not there is not used
    typename IO::Raw rx, ro, ry, rn;
    auto fetch = [&](int64_t r) {
        IO::fetch(rx, a.x, r, a.d, t);
        IO::fetch(ro, po, r, a.d, t);
        IO::fetch(rn, pn, r, a.d, t);
        IO::fetch(ry, py, r, a.d, t);
    };
    fetch(clamp(row0 + slot));
    const float res = a.res ? a.res[0] : 1.f, g0 = a.gate_len == 1 ? a.gate[0] : 1.f;
    float wo[E], bo[E], gt[E], wn[E];
    if constexpr (HOLD) {
        IO::param(a.w_post, a.d, t, 1.f, wo);
        IO::param(a.b_post, a.d, t, 0.f, bo);
        IO::param(a.gate_len > 1 ? a.gate : nullptr, a.d, t, g0, gt);
        IO::param(a.w_pre, a.d, t, 0.f, wn);
    }
    float ca[E], cb[E], cc[E], cd[E];
#pragma unroll
    for (int e = 0; e < E; ++e) ca[e] = cb[e] = cc[e] = cd[e] = 0.f;
    double s_res = 0., s_gate = 0.;
    for (; row0 < a.rows; row0 += stride) {
        const bool live = row0 + slot < a.rows;
        const int64_t row = clamp(row0 + slot);
        float x[E], oh[E], p[E], g[E];
        IO::widen(rx, a.d, t, x);
        IO::widen(ro, a.d, t, oh);
        IO::widen(ry, a.d, t, g);
        float dn[E];
        IO::widen(rn, a.d, t, dn);
        if (row0 + stride < a.rows) fetch(clamp(row0 + stride + slot));
        if (!a.dy)
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] = 0.f;
        float r_o = 1.f;
        if (!a.o) {
#pragma unroll
            for (int e = 0; e < E; ++e) p[e] = oh[e] = 0.f;
        } else if (a.w_post) {
            r_o = normalise<TPR, E, IO, LAYER>(oh, a, t, red, turn);
            if constexpr (!HOLD) IO::param(a.w_post, a.d, t, 1.f, wo), IO::param(a.b_post, a.d, t, 0.f, bo);
#pragma unroll
            for (int e = 0; e < E; ++e) p[e] = IO::in(t, e, a.d) ? fmaf(oh[e], wo[e], bo[e]) : 0.f;
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) p[e] = oh[e];
        }
        if (a.w_pre) {
            float yh[E];
            if constexpr (!HOLD) IO::param(a.gate_len > 1 ? a.gate : nullptr, a.d, t, g0, gt), IO::param(a.w_pre, a.d, t, 0.f, wn);
#pragma unroll
            for (int e = 0; e < E; ++e) yh[e] = fmaf(res, x[e], gt[e] * p[e]);
            const float r_y = normalise<TPR, E, IO, LAYER>(yh, a, t, red, turn);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (live) {
                    cc[e] = fmaf(dn[e], yh[e], cc[e]);
                    if constexpr (SHIFT) cd[e] += dn[e];
                }
                dn[e] *= wn[e];
            }
            norm_back<TPR, E, IO, LAYER>(dn, yh, r_y, a, red, turn);
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] = IO::in(t, e, a.d) ? g[e] + dn[e] : 0.f;
        }
        float sr = 0.f, sg = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            sr = fmaf(g[e], x[e], sr);
            sg = fmaf(g[e], p[e], sg);
            if (live) {
                ca[e] = fmaf(g[e], oh[e], ca[e]);
                if constexpr (SHIFT) cb[e] += g[e];
            }
        }
        if (live) s_res += sr, s_gate += sg;
        if (a.dx && live) {
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = res * g[e];
            IO::store(a.dx, row, a.d, t, x);
        }
        if (a.d_o) {
            if constexpr (!HOLD) IO::param(a.gate_len > 1 ? a.gate : nullptr, a.d, t, g0, gt), IO::param(a.w_post, a.d, t, 1.f, wo);
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] *= gt[e] * wo[e];
            if (a.w_post) {
                norm_back<TPR, E, IO, LAYER>(g, oh, r_o, a, red, turn);
            }
            if (live) IO::store(a.d_o, row, a.d, t, g);
        }
    }
    // the block's partial sums, its slots' joined in their order
    auto put = [&](int v, const float (&c)[E]) {
        if (v < 0) return;
        float *dst = a.cols + ((int64_t)blockIdx.x * a.nv + v) * a.d;
        if constexpr (RPB > 1) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < E; ++e) join[(slot * E + e) * TPR + t] = c[e];
            __syncthreads();
            for (int k = threadIdx.x; k < TPR * E; k += kNormThreads<TPR>) {
                const int e = k / TPR, j = IO::col(k % TPR, e / VEC) + e % VEC;
                float s = 0.f;
#pragma unroll
                for (int q = 0; q < RPB; ++q) s += join[q * E * TPR + k];
                if (j < a.d) dst[j] = s;
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int j = IO::col(t, e / VEC) + e % VEC;
                if (j < a.d) dst[j] = c[e];
            }
        }
    };
    put(a.v_a, ca);
    put(a.v_c, cc);
    if constexpr (SHIFT) {
        put(a.v_b, cb);
        put(a.v_d, cd);
    }
    if (a.scal) {
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) s_res += __shfl_xor(s_res, o, 64), s_gate += __shfl_xor(s_gate, o, 64);
        if ((threadIdx.x & 63) == 0) sred[2 * (threadIdx.x >> 6)] = s_res, sred[2 * (threadIdx.x >> 6) + 1] = s_gate;
        __syncthreads();
        if (threadIdx.x < 2) {
            double s = 0.;
            for (int w = 0; w < W; ++w) s += sred[2 * w + threadIdx.x];
            a.scal[2 * blockIdx.x + threadIdx.x] = s;
        }
    }
}

struct NormSums {
    const float *cols;
    const double *scal;
    int parts, d, nv, v_a, v_b, v_c, v_d, gate_len;
    const float *w_post, *b_post, *gate;
    float *dw_post, *db_post, *dgate, *dres, *dw_pre, *db_pre;
};

__device__ __forceinline__ double add_lanes(double v, int o) { return v + __shfl_xor(v, o, 64); }

// The parameters' gradients from the blocks' partial sums, in a fixed order and in 64 bits.  A block takes 16 columns (64 bytes a
// row) of one vector, 32 threads a column, four loads under way each; a gate's gradient takes the first vector and the second.
__global__ __launch_bounds__(512) void k_norm_sums(NormSums a)
{
    __shared__ double red[2][8][16];
    const int cj = threadIdx.x & 15, part = threadIdx.x >> 4, j = blockIdx.x * 16 + cj, v = blockIdx.y, wave = threadIdx.x >> 6;
    if (v < a.nv) {
        const bool gates = v == a.v_a && a.dgate && a.gate_len > 1, two = gates && a.b_post;
        double s[2] = {0., 0.};
        const int64_t row = (int64_t)a.nv * a.d;
        const float *src = a.cols + (int64_t)v * a.d + min(j, a.d - 1), *src2 = a.cols + (int64_t)(two ? a.v_b : v) * a.d + min(j, a.d - 1);
        for (int p0 = part; p0 < a.parts; p0 += 4 * 32) {
            float f[4], g[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t at = min(p0 + 32 * u, a.parts - 1) * row;
                f[u] = src[at];
                if (two) g[u] = src2[at];
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (p0 + 32 * u < a.parts) {
                    s[0] += (double)f[u];
                    if (two) s[1] += (double)g[u];
                }
        }
        // a wavefront holds four threads a column
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            s[k] = add_lanes(add_lanes(s[k], 16), 32);
            if ((threadIdx.x & 63) < 16) red[k][wave][cj] = s[k];
        }
        __syncthreads();
        if (threadIdx.x < 16 && j < a.d) {
            double t = 0., t2 = 0.;
#pragma unroll
            for (int w = 0; w < 8; ++w) t += red[0][w][cj], t2 += red[1][w][cj];
            const double ga = a.gate ? (double)a.gate[a.gate_len > 1 ? j : 0] : 1.;
            if (v == a.v_a && a.dw_post) a.dw_post[j] = (float)(ga * t);
            if (v == a.v_b && a.db_post) a.db_post[j] = (float)(ga * t);
            if (gates) a.dgate[j] = (float)(a.w_post ? (double)a.w_post[j] * t + (two ? (double)a.b_post[j] * t2 : 0.) : t);
            if (v == a.v_c && a.dw_pre) a.dw_pre[j] = (float)t;
            if (v == a.v_d && a.db_pre) a.db_pre[j] = (float)t;
        }
    } else if (blockIdx.x == 0 && threadIdx.x < 64 && (a.dres || (a.dgate && a.gate_len == 1))) { // one block behind the vectors': the two scalars
        double u = 0., w = 0.;
        for (int p = threadIdx.x; p < a.parts; p += 64) u += a.scal[2 * p], w += a.scal[2 * p + 1];
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) u = add_lanes(u, o), w = add_lanes(w, o);
        if (threadIdx.x == 0) {
            if (a.dres) a.dres[0] = (float)u;
            if (a.dgate && a.gate_len == 1) a.dgate[0] = (float)w;
        }
    }
}

static inline bool n_aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

static pac_status check_norm(const pac_block_norm *b, int64_t rows)
{
    if (!b) return PAC_ERR_NULL;
    if (b->d < 1 || b->d > 16384 || (b->dtype != PAC_BF16 && b->dtype != PAC_F32) || (b->layer != 0 && b->layer != 1) ||
        !(b->eps > 0.f) || !(b->eps <= 3.4e38f))
        return PAC_ERR_SHAPE;
    if (b->gate ? b->gate_len != 1 && b->gate_len != b->d : b->gate_len != 0) return PAC_ERR_SHAPE;
    if ((b->b_post && !b->w_post) || (b->b_pre && !b->w_pre)) return PAC_ERR_NULL;
    if (rows < 0) return PAC_ERR_RANGE;
    if (!n_aligned(b->w_post, 4) || !n_aligned(b->b_post, 4) || !n_aligned(b->gate, 4) || !n_aligned(b->res, 4) ||
        !n_aligned(b->w_pre, 4) || !n_aligned(b->b_pre, 4))
        return PAC_ERR_ALIGN;
    return PAC_OK;
}

// Values a thread and threads a row: as few threads as hold it, so that short rows take one wavefront and no barrier.
struct NormForm { int e, tpr; };
static NormForm norm_form(int d, bool backward)
{
    const int e = d > 8192 ? 16 : d > 4096 || !backward ? 8 : 4;
    int tpr = 64;
    while (tpr * e < d) tpr *= 2;
    return {e, tpr};
}

// A block adds its columns over rows in 32 bits, this many one after the other at most: past that there are more blocks instead, whose
// sums are joined in 64 bits, so that the error does not grow with the batch (to the 2^30 rows that the last number is good for).
constexpr int64_t kNormRounds = 64, kNormBlocks = 1 << 21;

// Blocks that rows may take, which never falls as they grow: a workspace for many rows serves fewer ...
static int64_t norm_blocks_most(int d, int64_t rows, bool backward)
{
    const int tpr = norm_form(d, backward).tpr, rpb = tpr < 512 ? 512 / tpr : 1;
    const int64_t want = (rows + rpb - 1) / rpb, most = backward ? (tpr == 1024 ? 256 : 512) : 1024;
    const int64_t more = backward ? (want + kNormRounds - 1) / kNormRounds : 0;
    return want < most ? want : more < most ? most : more < kNormBlocks ? more : kNormBlocks;
}
// ... and those that a launch has: as many rows a block everywhere, as few blocks' sums as that leaves
static int64_t norm_blocks(int d, int64_t rows, bool backward)
{
    const int tpr = norm_form(d, backward).tpr, rpb = tpr < 512 ? 512 / tpr : 1;
    const int64_t want = (rows + rpb - 1) / rpb, most = norm_blocks_most(d, rows, backward), rounds = (want + most - 1) / most;
    return (want + rounds - 1) / rounds;
}

template <typename T, int VEC, int TPR, int E, bool LAYER> static void launch_fwd(const NormArgs &a, dim3 g, hipStream_t st)
{
    hipLaunchKernelGGL((k_norm_fwd<T, VEC, TPR, E, LAYER, (E < 16)>), g, dim3(kNormThreads<TPR>), 0, st, a);
}
template <typename T, int VEC, int TPR, int E, bool LAYER> static void launch_bwd(const NormArgs &a, dim3 g, hipStream_t st)
{
    if (a.v_b >= 0 || a.v_d >= 0) hipLaunchKernelGGL((k_norm_bwd<T, VEC, TPR, E, LAYER, true, (E < 8)>), g, dim3(kNormThreads<TPR>), 0, st, a);
    else hipLaunchKernelGGL((k_norm_bwd<T, VEC, TPR, E, LAYER, false, (E < 8)>), g, dim3(kNormThreads<TPR>), 0, st, a);
}

template <typename T, bool WIDE, bool LAYER> static void launch_norm(const NormArgs &a, bool backward, hipStream_t st)
{
    const NormForm f = norm_form(a.d, backward);
    const dim3 g((unsigned)norm_blocks(a.d, a.rows, backward));
    constexpr int V8 = WIDE ? 16 / (int)sizeof(T) : 1, V4 = WIDE ? 4 : 1;
    if (backward) {
        if (f.e == 4) {
            if (f.tpr == 64) launch_bwd<T, V4, 64, 4, LAYER>(a, g, st);
            else if (f.tpr == 128) launch_bwd<T, V4, 128, 4, LAYER>(a, g, st);
            else if (f.tpr == 256) launch_bwd<T, V4, 256, 4, LAYER>(a, g, st);
            else if (f.tpr == 512) launch_bwd<T, V4, 512, 4, LAYER>(a, g, st);
            else launch_bwd<T, V4, 1024, 4, LAYER>(a, g, st);
        } else if (f.e == 8) launch_bwd<T, V8, 1024, 8, LAYER>(a, g, st);
        else launch_bwd<T, V8, 1024, 16, LAYER>(a, g, st);
    } else if (f.e == 8) {
        if (f.tpr == 64) launch_fwd<T, V8, 64, 8, LAYER>(a, g, st);
        else if (f.tpr == 128) launch_fwd<T, V8, 128, 8, LAYER>(a, g, st);
        else if (f.tpr == 256) launch_fwd<T, V8, 256, 8, LAYER>(a, g, st);
        else if (f.tpr == 512) launch_fwd<T, V8, 512, 8, LAYER>(a, g, st);
        else launch_fwd<T, V8, 1024, 8, LAYER>(a, g, st);
    } else launch_fwd<T, V8, 1024, 16, LAYER>(a, g, st);
}

static pac_status run_norm(const pac_block_norm *b, const NormArgs &a, bool vec, bool backward, hipStream_t st)
{
    if (b->dtype == PAC_F32) {
        if (vec) b->layer ? launch_norm<float, true, true>(a, backward, st) : launch_norm<float, true, false>(a, backward, st);
        else b->layer ? launch_norm<float, false, true>(a, backward, st) : launch_norm<float, false, false>(a, backward, st);
    } else {
        if (vec) b->layer ? launch_norm<bf16_t, true, true>(a, backward, st) : launch_norm<bf16_t, true, false>(a, backward, st);
        else b->layer ? launch_norm<bf16_t, false, true>(a, backward, st) : launch_norm<bf16_t, false, false>(a, backward, st);
    }
    return hipGetLastError() == hipSuccess ? PAC_OK : PAC_ERR_DEVICE;
}

static NormArgs norm_args(const pac_block_norm *b, int64_t rows, const void *x, const void *o)
{
    NormArgs a = {};
    a.x = x; a.o = o; a.rows = rows; a.d = b->d; a.eps = b->eps; a.inv_d = 1.f / (float)b->d;
    a.v_a = a.v_b = a.v_c = a.v_d = -1;
    a.w_post = b->w_post; a.b_post = b->b_post; a.gate = b->gate; a.res = b->res; a.w_pre = b->w_pre; a.b_pre = b->b_pre;
    a.gate_len = b->gate ? (b->gate_len == 1 ? 1 : b->d) : 0;
    return a;
}

// 16-byte accesses need whole 16-byte pieces a row
static bool norm_vec(const pac_block_norm *b, std::initializer_list<const void *> ps)
{
    if (b->d % (b->dtype == PAC_F32 ? 4 : 8)) return false;
    for (const void *p : ps)
        if (!n_aligned(p, 16)) return false;
    for (const float *p : {b->w_post, b->b_post, b->gate_len > 1 ? b->gate : nullptr, b->w_pre, b->b_pre})
        if (!n_aligned(p, 16)) return false;
    return true;
}
static bool norm_typed(const pac_block_norm *b, std::initializer_list<const void *> ps)
{
    for (const void *p : ps)
        if (!n_aligned(p, b->dtype == PAC_F32 ? 4 : 2)) return false;
    return true;
}

// States that are written: in the place of one that is read (a row is read before it is written), or away from all of them, and away
// from the parameters
static bool state_misplaced(const pac_block_norm *b, int64_t rows, const void *out, std::initializer_list<const void *> in)
{
    const int64_t bytes = rows * b->d * (b->dtype == PAC_F32 ? 4 : 2), vec = (int64_t)b->d * 4;
    const Span o(out, bytes);
    for (const void *p : in)
        if (p != out && share(o, Span(p, bytes))) return true;
    return shares(o, {Span(b->w_post, vec), Span(b->b_post, vec), Span(b->gate, (int64_t)b->gate_len * 4), Span(b->res, 4), Span(b->w_pre, vec),
                      Span(b->b_pre, vec)});
}

} // namespace pac

using namespace pac;

extern "C" {

pac_status pac_block_norm_forward(const pac_block_norm *b, int64_t rows, const void *x, const void *o, void *y, void *n, void *hip_stream)
{
    const pac_status s = check_norm(b, rows);
    if (s != PAC_OK) return s;
    if (rows && (!x || (!o && (b->w_post || b->gate)) || (b->w_pre && !n) || (!b->w_pre && (n || !y)))) return PAC_ERR_NULL;
    if (!norm_typed(b, {x, o, y, n})) return PAC_ERR_ALIGN;
    if (rows == 0) return PAC_OK;
    if (state_misplaced(b, rows, y, {x, o}) || state_misplaced(b, rows, n, {x, o, y})) return PAC_ERR_RANGE;
    NormArgs a = norm_args(b, rows, x, o);
    a.y = y; a.n = n;
    (void)hipGetLastError();
    return run_norm(b, a, norm_vec(b, {x, o, y, n}), false, static_cast<hipStream_t>(hip_stream));
}

int64_t pac_block_norm_workspace_bytes(const pac_block_norm *b, int64_t rows)
{
    if (check_norm(b, rows) != PAC_OK) return -1;
    return (norm_blocks_most(b->d, rows < 1 ? 1 : rows, true) * (16 + 16 * (int64_t)b->d) + 255) / 256 * 256; // two doubles, four rows of floats
}

pac_status pac_block_norm_backward(const pac_block_norm *b, int64_t rows, const void *x, const void *o, const void *dy, const void *dn,
                                   void *dx, void *do_, float *dw_post, float *db_post, float *dgate, float *dres, float *dw_pre,
                                   float *db_pre, void *workspace, int64_t workspace_bytes, void *hip_stream)
{
    const pac_status s = check_norm(b, rows);
    if (s != PAC_OK) return s;
    if (rows && (!x || (!o && (b->w_post || b->gate || do_)) || (!b->w_pre) != (!dn) || (!dy && !dn))) return PAC_ERR_NULL;
    if ((dw_post && !b->w_post) || (db_post && !b->b_post) || (dgate && !b->gate) || (dres && !b->res) || (dw_pre && !b->w_pre) ||
        (db_pre && !b->b_pre))
        return PAC_ERR_NULL;
    const bool sums = dw_post || db_post || dgate || dres || dw_pre || db_pre;
    if (sums && !workspace) return PAC_ERR_NULL;
    if (!norm_typed(b, {x, o, dy, dn, dx, do_})) return PAC_ERR_ALIGN;
    for (const void *p : {(const void *)dw_post, (const void *)db_post, (const void *)dgate, (const void *)dres, (const void *)dw_pre, (const void *)db_pre})
        if (!n_aligned(p, 4)) return PAC_ERR_ALIGN;
    if (sums && !n_aligned(workspace, 16)) return PAC_ERR_ALIGN;
    if (sums && workspace_bytes < pac_block_norm_workspace_bytes(b, rows)) return PAC_ERR_WORKSPACE;
    if (state_misplaced(b, rows, dx, {x, o, dy, dn, do_}) || state_misplaced(b, rows, do_, {x, o, dy, dn, dx}) || (dx && dx == do_ && rows))
        return PAC_ERR_RANGE;
    if (sums) {
        // the sums' launch reads the parameters and the workspace while it writes the gradients
        const int64_t vec = (int64_t)b->d * 4, states = rows * b->d * (b->dtype == PAC_F32 ? 4 : 2);
        const Span outs[] = {Span(dw_post, vec), Span(db_post, vec), Span(dgate, (int64_t)b->gate_len * 4), Span(dres, 4), Span(dw_pre, vec),
                             Span(db_pre, vec), Span(workspace, pac_block_norm_workspace_bytes(b, rows))};
        for (const Span &u : outs) {
            if (shares(u, {Span(b->w_post, vec), Span(b->b_post, vec), Span(b->gate, (int64_t)b->gate_len * 4), Span(b->res, 4), Span(b->w_pre, vec),
                           Span(b->b_pre, vec), Span(x, states), Span(o, states), Span(dy, states), Span(dn, states), Span(dx, states), Span(do_, states)}))
                return PAC_ERR_RANGE;
            for (const Span &v : outs)
                if (&u != &v && share(u, v)) return PAC_ERR_RANGE;
        }
    }
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    NormArgs a = norm_args(b, rows, x, o);
    a.dy = dy; a.dn = dn; a.dx = dx; a.d_o = do_;
    // which column sums the wanted gradients are made of
    const bool gate_vec = dgate && b->gate_len > 1;
    // (a gate of one value is never a vector, also where d is 1)
    a.v_a = dw_post || gate_vec ? a.nv++ : -1;
    a.v_b = db_post || (gate_vec && b->b_post) ? a.nv++ : -1;
    a.v_c = dw_pre ? a.nv++ : -1;
    a.v_d = db_pre ? a.nv++ : -1;
    const bool scalars = dres || (dgate && b->gate_len == 1);
    const int64_t blocks = rows ? norm_blocks(b->d, rows, true) : 0;
    if (sums) {
        a.scal = scalars ? static_cast<double *>(workspace) : nullptr;
        a.cols = reinterpret_cast<float *>(static_cast<char *>(workspace) + 16 * blocks);
    }
    (void)hipGetLastError();
    if (rows) {
        const pac_status r = run_norm(b, a, norm_vec(b, {x, o, dy, dn, dx, do_}), true, st);
        if (r != PAC_OK) return r;
    }
    if (!sums) return PAC_OK;
    const NormSums u{a.cols, a.scal, (int)blocks, b->d, a.nv, a.v_a, a.v_b, a.v_c, a.v_d, a.gate_len,
                     b->w_post, b->b_post, b->gate, dw_post, db_post, dgate, dres, dw_pre, db_pre};
    // columns by vectors, and where scalars are wanted one more row of blocks, of which the first sums them
    const dim3 gs(a.nv ? (unsigned)((b->d + 15) / 16) : 1u, (unsigned)(a.nv + (scalars ? 1 : 0)));
    hipLaunchKernelGGL(k_norm_sums, gs, dim3(512), 0, st, u);
    return hipGetLastError() == hipSuccess ? PAC_OK : PAC_ERR_DEVICE;
}

} // extern "C"
