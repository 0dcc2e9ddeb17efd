// Norms before and after a block, fused with the block's gate and the scale of the residual path, and their gradients (declared
// in include/pac_norm.h).
#include "../../include/pac_norm.h"
#include "pac_gemm.h"

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

// sums of a row's NS values over its TPR threads, on all of them; `red` belongs to the row, [2][TPR / 64][4], `turn` alternates
// so that one barrier a sum is enough
template <int TPR, int NS> __device__ __forceinline__ void row_sums(float (&s)[NS], float *red, int &turn)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1)
#pragma unroll
        for (int k = 0; k < NS; ++k) s[k] += __shfl_xor(s[k], o, 64);
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        float *r = red + turn * W * 4;
        turn ^= 1;
        const int wave = (threadIdx.x % TPR) >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < NS; ++k) r[wave * 4 + k] = s[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NS; ++k) {
            s[k] = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) s[k] += r[w * 4 + k];
        }
    }
}

// E neighbouring-by-VEC values of a row a thread: chunk c holds columns (c TPR + t) VEC and the VEC - 1 after it
template <typename T, int VEC, int TPR, int E> struct RowIO {
    static constexpr int CH = E / VEC;
    typedef T vec __attribute__((ext_vector_type(VEC)));
    static __device__ __forceinline__ int col(int t, int c) { return (c * TPR + t) * VEC; }
    static __device__ __forceinline__ void load(const void *p, int64_t row, int d, int t, float (&v)[E])
    {
        const T *src = reinterpret_cast<const T *>(p) + row * d;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int j = col(t, c);
            if constexpr (VEC == 1) v[c] = j < d ? (float)src[j] : 0.f;
            else {
                const bool in = j < d; // d is a multiple of VEC
                const vec r = *reinterpret_cast<const vec *>(src + (in ? j : 0));
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[c * VEC + e] = in ? (float)r[e] : 0.f;
            }
        }
    }
    static __device__ __forceinline__ void store(void *p, int64_t row, int d, int t, const float (&v)[E])
    {
        T *dst = reinterpret_cast<T *>(p) + row * d;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int j = col(t, c);
            if (j >= d) continue;
            if constexpr (VEC == 1) dst[j] = (T)v[c];
            else {
                vec r;
#pragma unroll
                for (int e = 0; e < VEC; ++e) r[e] = (T)v[c * VEC + e];
                *reinterpret_cast<vec *>(dst + j) = r;
            }
        }
    }
    // a parameter's values at this thread's columns (`none` where there is no such parameter or no such column)
    static __device__ __forceinline__ void param(const float *p, int d, int t, float none, float (&v)[E])
    {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const int j = col(t, c) + e;
                v[c * VEC + e] = p && j < d ? p[j] : none;
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
        for (int e = 0; e < E; ++e) v[e] = IO::col(t, e / (E / IO::CH)) < a.d ? v[e] - mean : 0.f;
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
__device__ __forceinline__ void norm_back(float (&g)[E], const float (&h)[E], float r, const NormArgs &a, int t, float *red, int &turn)
{
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < E; ++e) s[0] = fmaf(g[e], h[e], s[0]), s[1] += g[e];
    if constexpr (LAYER) row_sums<TPR, 2>(s, red, turn);
    else {
        float s1[1] = {s[0]};
        row_sums<TPR, 1>(s1, red, turn);
        s[0] = s1[0];
    }
    const float along = s[0] * a.inv_d, mean = LAYER ? s[1] * a.inv_d : 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) g[e] = r * (g[e] - mean - h[e] * along);
}

template <typename T, int VEC, int TPR, int E, bool LAYER>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_norm_fwd(NormArgs a)
{
    constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
    using IO = RowIO<T, VEC, TPR, E>;
    __shared__ float redm[RPB * 2 * (TPR / 64) * 4];
    const int t = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    float *red = redm + slot * 2 * (TPR / 64) * 4;
    int turn = 0;
    const float res = a.res ? a.res[0] : 1.f;
    float wp[E], bp[E], gt[E], wn[E], bn[E];
    IO::param(a.w_post, a.d, t, 1.f, wp);
    IO::param(a.b_post, a.d, t, 0.f, bp);
    IO::param(a.w_pre, a.d, t, 0.f, wn);
    IO::param(a.b_pre, a.d, t, 0.f, bn);
    if (a.gate_len > 1) IO::param(a.gate, a.d, t, 0.f, gt);
    else {
        const float g = a.gate ? a.gate[0] : 1.f;
#pragma unroll
        for (int e = 0; e < E; ++e) gt[e] = g;
    }
    // every thread of a block goes round as often (barriers): a slot whose row is past the end works on the last one, unstored
    for (int64_t row0 = (int64_t)blockIdx.x * RPB; row0 < a.rows; row0 += (int64_t)gridDim.x * RPB) {
        const bool live = row0 + slot < a.rows;
        const int64_t row = live ? row0 + slot : a.rows - 1;
        float y[E];
        IO::load(a.x, row, a.d, t, y);
        if (a.o) {
            float o[E];
            IO::load(a.o, row, a.d, t, o);
            if (a.w_post) {
                normalise<TPR, E, IO, LAYER>(o, a, t, red, turn);
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] = fmaf(o[e], wp[e], bp[e]);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = fmaf(res, y[e], gt[e] * o[e]);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] *= res;
        }
        if (a.y && live) IO::store(a.y, row, a.d, t, y);
        if (a.w_pre) {
            normalise<TPR, E, IO, LAYER>(y, a, t, red, turn);
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = fmaf(y[e], wn[e], bn[e]);
            if (live) IO::store(a.n, row, a.d, t, y);
        }
    }
}

template <typename T, int VEC, int TPR, int E, bool LAYER>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_norm_bwd(NormArgs a)
{
    constexpr int RPB = TPR < 256 ? 256 / TPR : 1, W = RPB * TPR / 64;
    using IO = RowIO<T, VEC, TPR, E>;
    __shared__ float redm[RPB * 2 * (TPR / 64) * 4];
    __shared__ double sred[2 * W];
    const int t = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    float *red = redm + slot * 2 * (TPR / 64) * 4;
    int turn = 0;
    const float res = a.res ? a.res[0] : 1.f, g0 = a.gate_len == 1 ? a.gate[0] : 1.f;
    float ca[E], cb[E], cc[E], cd[E];
#pragma unroll
    for (int e = 0; e < E; ++e) ca[e] = cb[e] = cc[e] = cd[e] = 0.f;
    double s_res = 0., s_gate = 0.;
    for (int64_t row0 = (int64_t)blockIdx.x * RPB; row0 < a.rows; row0 += (int64_t)gridDim.x * RPB) {
        const bool live = row0 + slot < a.rows;
        const int64_t row = live ? row0 + slot : a.rows - 1;
        float x[E], oh[E], gt[E], wp[E], g[E];
        IO::load(a.x, row, a.d, t, x);
        if (a.gate_len > 1) IO::param(a.gate, a.d, t, 0.f, gt);
        else {
#pragma unroll
            for (int e = 0; e < E; ++e) gt[e] = g0;
        }
        IO::param(a.w_post, a.d, t, 1.f, wp);
        float ro = 1.f;
        float p[E];
        if (a.o) {
            IO::load(a.o, row, a.d, t, oh);
            if (a.w_post) {
                ro = normalise<TPR, E, IO, LAYER>(oh, a, t, red, turn);
                float bp[E];
                IO::param(a.b_post, a.d, t, 0.f, bp);
#pragma unroll
                for (int e = 0; e < E; ++e) p[e] = fmaf(oh[e], wp[e], bp[e]);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) p[e] = oh[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) p[e] = oh[e] = 0.f;
        }
        if (a.w_pre) {
            float yh[E], wn[E], dn[E];
#pragma unroll
            for (int e = 0; e < E; ++e) yh[e] = fmaf(res, x[e], gt[e] * p[e]);
            IO::load(a.dn, row, a.d, t, dn);
            IO::param(a.w_pre, a.d, t, 0.f, wn);
            const float ry = normalise<TPR, E, IO, LAYER>(yh, a, t, red, turn);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (live) cc[e] = fmaf(dn[e], yh[e], cc[e]), cd[e] += dn[e];
                g[e] = dn[e] * wn[e];
            }
            norm_back<TPR, E, IO, LAYER>(g, yh, ry, a, t, red, turn);
            if (a.dy) {
                float dy[E];
                IO::load(a.dy, row, a.d, t, dy);
#pragma unroll
                for (int e = 0; e < E; ++e) g[e] += dy[e];
            }
        } else if (a.dy) IO::load(a.dy, row, a.d, t, g);
        else {
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] = 0.f;
        }
        float sr = 0.f, sg = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const bool in = IO::col(t, e / VEC) + e % VEC < a.d;
            if (!in) g[e] = 0.f;
            sr = fmaf(g[e], x[e], sr);
            sg = fmaf(g[e], p[e], sg);
            if (live) ca[e] = fmaf(g[e], oh[e], ca[e]), cb[e] += g[e];
        }
        if (live) s_res += sr, s_gate += sg;
        if (a.dx && live) {
            float dx[E];
#pragma unroll
            for (int e = 0; e < E; ++e) dx[e] = res * g[e];
            IO::store(a.dx, row, a.d, t, dx);
        }
        if (a.o && a.d_o) {
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] *= gt[e] * wp[e];
            if (a.w_post) norm_back<TPR, E, IO, LAYER>(g, oh, ro, a, t, red, turn);
            if (live) IO::store(a.d_o, row, a.d, t, g);
        }
    }
    if (a.nv == 0 && !a.scal) return;
    // the block's sums: rows dealt over its slots are joined slot by slot
    auto put = [&](int v, const float (&c)[E]) {
        if (v < 0) return;
        float *dst = a.cols + ((int64_t)(blockIdx.x * RPB + slot) * a.nv + v) * a.d;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int j = IO::col(t, e / VEC) + e % VEC;
            if (j < a.d) dst[j] = c[e];
        }
    };
    put(a.v_a, ca);
    put(a.v_b, cb);
    put(a.v_c, cc);
    put(a.v_d, cd);
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
    int parts, blocks, d, nv, v_a, v_b, v_c, v_d, gate_len;
    const float *w_post, *b_post, *gate;
    float *dw_post, *db_post, *dgate, *dres, *dw_pre, *db_pre;
    int post;
};

// The parameters' gradients from the blocks' partial sums, in their order and in 64 bits.  16 columns a block, 16 threads a column.
__global__ __launch_bounds__(256) void k_norm_sums(NormSums a)
{
    __shared__ double red[4][16][17];
    const int cj = threadIdx.x & 15, part = threadIdx.x >> 4, j = blockIdx.x * 16 + cj;
    double s[4] = {0., 0., 0., 0.};
    if (j < a.d)
        for (int p = part; p < a.parts; p += 16)
            for (int v = 0; v < a.nv; ++v) s[v] += (double)a.cols[((int64_t)p * a.nv + v) * a.d + j];
#pragma unroll
    for (int v = 0; v < 4; ++v) red[v][part][cj] = s[v];
    __syncthreads();
    if (threadIdx.x < 16 && j < a.d) {
        double t[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            t[v] = 0.;
            for (int p = 0; p < 16; ++p) t[v] += red[v][p][cj];
        }
        auto pick = [&](int v) { return v == 0 ? t[0] : v == 1 ? t[1] : v == 2 ? t[2] : v == 3 ? t[3] : 0.; };
        const double ga = a.gate ? (double)a.gate[a.gate_len > 1 ? j : 0] : 1.;
        if (a.dw_post) a.dw_post[j] = (float)(ga * pick(a.v_a));
        if (a.db_post) a.db_post[j] = (float)(ga * pick(a.v_b));
        if (a.dgate && a.gate_len > 1)
            a.dgate[j] = (float)(a.post ? (double)a.w_post[j] * pick(a.v_a) + (a.b_post ? (double)a.b_post[j] * pick(a.v_b) : 0.) : pick(a.v_a));
        if (a.dw_pre) a.dw_pre[j] = (float)pick(a.v_c);
        if (a.db_pre) a.db_pre[j] = (float)pick(a.v_d);
    }
    if (blockIdx.x == 0 && (a.dres || (a.dgate && a.gate_len == 1))) {
        __syncthreads();
        double *r = &red[0][0][0];
        double u[2] = {0., 0.};
        for (int p = threadIdx.x; p < a.blocks; p += 256) u[0] += a.scal[2 * p], u[1] += a.scal[2 * p + 1];
        r[2 * threadIdx.x] = u[0];
        r[2 * threadIdx.x + 1] = u[1];
        __syncthreads();
        if (threadIdx.x < 2) {
            double t = 0.;
            for (int p = 0; p < 256; ++p) t += r[2 * p + threadIdx.x];
            if (threadIdx.x == 0 && a.dres) a.dres[0] = (float)t;
            if (threadIdx.x == 1 && a.dgate && a.gate_len == 1) a.dgate[0] = (float)t;
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

// Threads a row: as few as hold it at `E` values each, so that short rows take one wavefront and no barrier.
static int threads_for(int d, int e) { return d <= 64 * e ? 64 : d <= 256 * e ? 256 : 1024; }

constexpr int kNormE = 16; // values a thread

static int64_t norm_blocks(int d, int64_t rows, bool backward)
{
    const int tpr = threads_for(d, kNormE), rpb = tpr < 256 ? 256 / tpr : 1;
    const int64_t want = (rows + rpb - 1) / rpb, most = backward ? (tpr == 1024 ? 256 : 512) : (tpr == 1024 ? 512 : 2048);
    return want < most ? want : most;
}
static int64_t norm_parts(int d, int64_t rows)
{
    const int tpr = threads_for(d, kNormE);
    return norm_blocks(d, rows, true) * (tpr < 256 ? 256 / tpr : 1);
}

template <typename T, int VEC, bool LAYER> static void launch_norm(const NormArgs &a, bool backward, hipStream_t st)
{
    const int tpr = threads_for(a.d, kNormE);
    const dim3 g((unsigned)norm_blocks(a.d, a.rows, backward)), b(tpr < 256 ? 256 : tpr);
#define PAC_NORM_LAUNCH(TPR)                                                                                                   \
    if (backward) hipLaunchKernelGGL((k_norm_bwd<T, VEC, TPR, kNormE, LAYER>), g, b, 0, st, a);                                \
    else hipLaunchKernelGGL((k_norm_fwd<T, VEC, TPR, kNormE, LAYER>), g, b, 0, st, a);
    if (tpr == 64) { PAC_NORM_LAUNCH(64) }
    else if (tpr == 256) { PAC_NORM_LAUNCH(256) }
    else { PAC_NORM_LAUNCH(1024) }
#undef PAC_NORM_LAUNCH
}

static pac_status run_norm(const pac_block_norm *b, const NormArgs &a, bool vec, bool backward, hipStream_t st)
{
    if (b->dtype == PAC_F32) {
        if (vec) b->layer ? launch_norm<float, 4, true>(a, backward, st) : launch_norm<float, 4, false>(a, backward, st);
        else b->layer ? launch_norm<float, 1, true>(a, backward, st) : launch_norm<float, 1, false>(a, backward, st);
    } else {
        if (vec) b->layer ? launch_norm<bf16_t, 8, true>(a, backward, st) : launch_norm<bf16_t, 8, false>(a, backward, st);
        else b->layer ? launch_norm<bf16_t, 1, true>(a, backward, st) : launch_norm<bf16_t, 1, false>(a, backward, st);
    }
    return hipGetLastError() == hipSuccess ? PAC_OK : PAC_ERR_DEVICE;
}

static NormArgs norm_args(const pac_block_norm *b, int64_t rows, const void *x, const void *o)
{
    NormArgs a = {};
    a.x = x; a.o = o; a.rows = rows; a.d = b->d; a.eps = b->eps; a.inv_d = 1.f / (float)b->d;
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
    return true;
}
static bool norm_typed(const pac_block_norm *b, std::initializer_list<const void *> ps)
{
    for (const void *p : ps)
        if (!n_aligned(p, b->dtype == PAC_F32 ? 4 : 2)) return false;
    return true;
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
    NormArgs a = norm_args(b, rows, x, o);
    a.y = y; a.n = n;
    (void)hipGetLastError();
    return run_norm(b, a, norm_vec(b, {x, o, y, n}), false, static_cast<hipStream_t>(hip_stream));
}

int64_t pac_block_norm_workspace_bytes(const pac_block_norm *b, int64_t rows)
{
    if (check_norm(b, rows) != PAC_OK) return -1;
    const int64_t blocks = norm_blocks(b->d, rows < 1 ? 1 : rows, true), parts = norm_parts(b->d, rows < 1 ? 1 : rows);
    return (16 * blocks + 4 * parts * 4 * (int64_t)b->d + 255) / 256 * 256;
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
    const NormSums u{a.cols, a.scal, (int)(rows ? norm_parts(b->d, rows) : 0), (int)blocks, b->d, a.nv, a.v_a, a.v_b, a.v_c, a.v_d, a.gate_len,
                     b->w_post, b->b_post, b->gate, dw_post, db_post, dgate, dres, dw_pre, db_pre, b->w_post != nullptr};
    hipLaunchKernelGGL(k_norm_sums, dim3(a.nv ? (unsigned)((b->d + 15) / 16) : 1u), dim3(256), 0, st, u);
    return hipGetLastError() == hipSuccess ? PAC_OK : PAC_ERR_DEVICE;
}

} // extern "C"
