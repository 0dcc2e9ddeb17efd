// Attention over packed sequences and its gradients (declared in include/pac_attn.h).
#include "../../include/pac_attn.h"
#include "pac_attn_tile.h"
#include "pac_mma.h"
#include "pac_span.h"
#include <cfloat>
#include <cmath>

namespace pac {

struct AttnArgs {
    const int32_t *off; // [batch + 1]
    int batch, rows;
    int heads, kv_heads, group, d;
    float scale, c2; // scale, scale log2(e)
    const bf16_t *q, *k, *v, *o, *d_o;
    int64_t qs, ks, vs, os, dos;
    bf16_t *out; // forward: o
    float *lse;  // [heads][rows]
    bf16_t *dq, *dk, *dv;
    int64_t dqs, dks, dvs;
    float *nlse2, *delta; // [heads][rows] each: -lse log2(e), do . o
    int splits;     // of the queries that a tile of keys goes through, in dk and dv
    float *part;    // [splits][rows][2][kv_heads d]: dk / scale and dv of the splits, where there are several
};

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------------------
// Which rows a workgroup has.  A sequence that begins at row s may have the numbers s / BM + b and up to the next one's, of which there are
// never fewer than its tiles, so that the grid follows from rows and batch alone and a number's sequence is found by a search over the
// offsets, 64 places a time.  The search ends at up to 64 sequences, whose tiles have the first of the numbers that they have together: numbers
// without a tile come last, where no compute unit waits for its share behind them (numbers without one after every sequence / at the end, us:
// 4 x 1024 tokens of 8 heads of 64 there and back 146 / 108, 8 x 128 of 32 of 128 56 / 50; but 16 x 256 of 32 forward 34.5 / 35.7, whose tiles
// of one and of two steps then lie less evenly).  With causal a sequence's tiles begin with the one that takes longest.
// (Most work first across sequences, us: 16 x 256 35 / 44, 8 x 512 175 / 201, 8 x 256..1024 280 / 290: a sequence's keys are read while they
// are in the cache when its tiles follow each other.)
// ---------------------------------------------------------------------------
struct AttnSeq {
    int start, len, tile; // len < 1: nothing to do
};
// sums over the lanes up to each
__device__ __forceinline__ int wave_sums(int x)
{
#define PAC_ATTN_STEP(CTRL, ROWS) x += __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false)
    PAC_ATTN_STEP(0x111, 0xf); // from the lanes 1, 2, 4, 8 places before in a row of 16, then from the rows before
    PAC_ATTN_STEP(0x112, 0xf);
    PAC_ATTN_STEP(0x114, 0xf);
    PAC_ATTN_STEP(0x118, 0xf);
    PAC_ATTN_STEP(0x142, 0xa);
    PAC_ATTN_STEP(0x143, 0xc);
#undef PAC_ATTN_STEP
    return x;
}
template <int BM, bool CAUSAL, bool KEYS = false> __device__ __forceinline__ AttnSeq attn_seq(const AttnArgs &a, int number)
{
    const int lane = threadIdx.x & 63;
    auto at = [&](int b) { return min(max(a.off[b], 0), a.rows); };
    int lo = 0, n = a.batch;
    while (n > 64) {
        const int step = (n + 63) / 64, b = lane * step;
        const bool before = b < n && at(lo + b) / BM + lo + b <= number;
        const int cnt = __builtin_popcountll(__ballot(before));
        if (cnt == 0) return AttnSeq{0, 0, 0};
        lo += (cnt - 1) * step;
        n = min(step, n - (cnt - 1) * step);
    }
    const int start = lane < n ? at(lo + lane) : 0, len = lane < n ? at(lo + lane + 1) - start : 0, tiles = len > 0 ? (len - 1) / BM + 1 : 0;
    const int r = number - (__builtin_amdgcn_readfirstlane(start) / BM + lo);
    // (where offsets fall, the search may end anywhere: what is before the first number is none)
    const int sums = wave_sums(tiles);
    if (r < 0 || r >= __builtin_amdgcn_readlane(sums, 63)) return AttnSeq{0, 0, 0};
    const int mine = __builtin_popcountll(__ballot(sums <= r)); // sequences whose tiles come before
    const int its = __builtin_amdgcn_readlane(tiles, mine), i = __builtin_amdgcn_readlane(sums, mine) - 1 - r; // tiles from the last one
    return AttnSeq{__builtin_amdgcn_readlane(start, mine), __builtin_amdgcn_readlane(len, mine), CAUSAL && !KEYS ? i : its - 1 - i};
}

// A tile of ROWS rows on its way from memory straight to LDS (pac_attn_tile.h: which lane fetches what).  Rows past `have` repeat the last one,
// so that a wavefront always has N transfers under way; the kernels mask them.  Pieces past d are not fetched: their places keep the zeros of
// clear_tiles, or, where D is 96 and a row's place has four pieces more, are never read.  (Offsets stay under 2^32 bytes for strides up to 2^24.)
template <int D, int ROWS, int WAVES = 4> struct AttnDma { // WAVES: that share the tile
    using F = AttnFetch<D, ROWS, WAVES>;
    static_assert(F::steady(), "one decision for all transfers of a lane");
    static constexpr int N = F::N;
    uint32_t stride2, off[N];
    int row, to, dd; // dd: values of a row that are fetched
    __device__ __forceinline__ void plan(int64_t stride, int d)
    {
        const int lane = threadIdx.x & 63, first = F::first(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
        row = F::row(first, lane);
        to = first * 1024;
        stride2 = (uint32_t)(stride * 2);
        // (rows of a transfer begin at a multiple of RPI; the swizzle's period is 16 rows)
#pragma unroll
        for (int i = 0; i < N; ++i) off[i] = F::offset(row + i * F::RPI, piece(i), stride2);
        dd = d;
    }
    __device__ __forceinline__ int piece(int i) const { return F::piece(threadIdx.x & 63, row + i * F::RPI); }
    __device__ __forceinline__ static void one(const bf16_t *base, uint32_t off, uint32_t lds)
    {
        // one wait state between the write of M0 and the transfer that reads it; the compiler does not know of the transfer and so does
        // not wait for it at every LDS read: the kernels do, before the barrier that hands a tile over
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(off), "s"(base) : "memory", "m0");
    }
    // base: the tile's first row, the same for all lanes, as `lds` is
    __device__ __forceinline__ void issue(const bf16_t *base, uint32_t lds, int have) const
    {
        const uint32_t at = __builtin_amdgcn_readfirstlane(lds + to);
        if (F::whole(dd, have)) {
            if (F::part_of_whole(threadIdx.x & 63, row)) {
#pragma unroll
                for (int i = 0; i < N; ++i) one(base, off[i], at + i * 1024);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (F::part(piece(i), dd)) one(base, F::offset(min(row + i * F::RPI, have - 1), piece(i), stride2), at + i * 1024);
        }
    }
};
// Zeros in all of a workgroup's tiles, before the first transfer, where some pieces are never fetched
template <int BYTES> __device__ __forceinline__ void clear_tiles(char *lds)
{
    for (int i = threadIdx.x * 16; i < BYTES; i += blockDim.x * 16) *reinterpret_cast<u32x4 *>(lds + i) = u32x4{0, 0, 0, 0};
    __syncthreads();
}

// Operands of 32x32x16 products from a tile at LDS address `tile` (a multiple of 1024).
// "Along": lane (i = lane % 32, h = lane / 32) holds row row0 + i, values 16 ks + 8 h ..+7.
// "Turned": lane (i, h) holds value 32 t + i of the rows row0 + 16 j + {4 h ..+3, 8 + 4 h ..+3}, which are the rows of the registers
// 8 j ..+7 of a 32 x 32 result in the same lane: a result enters the next product as it is.
// What varies from read to read is an exclusive or with a constant (ks, t, the second four rows) and a constant distance, so that a lane
// keeps one address for each of the two ways.
typedef const __attribute__((address_space(3))) u32x4 *lds_u32x4;
template <int D> struct AttnLane {
    using T = AttnTile<D>;
    uint32_t a, t;
    __device__ __forceinline__ explicit AttnLane(uint32_t tile)
    {
        const int lane = threadIdx.x & 63, p = lane & 15, h = lane >> 5;
        a = tile + T::at(lane & 31, h);
        t = tile + T::at(4 * h + (p >> 2), 2 * (lane >> 4 & 1) + (p >> 1 & 1)) + 8 * (p & 1);
    }
    __device__ __forceinline__ bf16x8 along(int row0, int ks) const
    {
        return __builtin_bit_cast(bf16x8, *reinterpret_cast<lds_u32x4>((a ^ (uint32_t)(ks << 5)) + (uint32_t)(row0 * T::RB)));
    }
    __device__ __forceinline__ bf16x8 turned(int row0, int j, int t_) const
    {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        const uint32_t lo = (t ^ (uint32_t)(t_ << 6)) + (uint32_t)((row0 + 16 * j) * T::RB), hi = (t ^ (uint32_t)(t_ << 6 | 32)) + (uint32_t)((row0 + 16 * j + 8) * T::RB);
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) s16x4 *>(lo));
        const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) s16x4 *>(hi));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};
// The same of a matrix in memory: row i of 32 (zeros past `have`, and past d)
__device__ __forceinline__ bf16x8 along_mem(const bf16_t *base, int64_t stride, int have, int d, int ks)
{
    const int lane = threadIdx.x & 63, i = lane & 31, at = 16 * ks + 8 * (lane >> 5);
    bf16x8 r{};
    if (i < have && at < d) r = *reinterpret_cast<const bf16x8 *>(base + i * stride + at);
    return r;
}
__device__ __forceinline__ f32x16 zeros16()
{
    f32x16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
    return z;
}
// row of a 32 x 32 result in register i
__device__ __forceinline__ int row_of(int i) { return 8 * (i >> 2) + 4 * ((threadIdx.x & 63) >> 5) + (i & 3); }
// the value on the diagonal of a 32 x 32 result in the lane's column
__device__ __forceinline__ float diagonal_of(const f32x16 &s)
{
    const int lane = threadIdx.x & 63, me = lane & 31;
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) x = row_of(i) == me ? s[i] : x;
    const float other = __shfl_xor(x, 32, 64);
    return (me >> 2 & 1) == lane >> 5 ? x : other;
}
__device__ __forceinline__ bf16x8 rounded(const f32x16 &s, int j)
{
    bf16x8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (bf16_t)s[8 * j + e];
    return r;
}

// Reads run a few operands ahead of the products and no further, because a kernel's registers are spoken for.
#define PAC_ATTN_PACE __builtin_amdgcn_sched_barrier(0x6) /* only vector and scalar arithmetic moves across */

// s[x] = (rows row0 + 32 x ..+31 of the tile) q^T
template <int D, int NS> __device__ __forceinline__ void scores(f32x16 (&s)[NS], const AttnLane<D> &l, int row0, const bf16x8 (&q)[D / 16])
{
    constexpr int N = NS * D / 16, AHEAD = 4;
    bf16x8 f[AHEAD];
#pragma unroll
    for (int n = 0; n < AHEAD - 1; ++n) f[n] = l.along(row0 + 32 * (n % NS), n / NS);
#pragma unroll
    for (int x = 0; x < NS; ++x) s[x] = zeros16();
#pragma unroll
    for (int n = 0; n < N; ++n) {
        constexpr int K = AHEAD - 1;
        if (n + K < N) f[(n + K) % AHEAD] = l.along(row0 + 32 * ((n + K) % NS), (n + K) / NS);
        s[n % NS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[n % AHEAD], q[n / NS], s[n % NS], 0, 0, 0);
        PAC_ATTN_PACE;
    }
}
// acc[t] += (turned tile)^T p over 32 rows of the tile, p in the registers of a 32 x 32 result.
template <int D> __device__ __forceinline__ void add_turned(f32x16 (&acc)[D / 32], const AttnLane<D> &l, int row0, const bf16x8 (&p)[2])
{
    constexpr int N = 2 * D / 32, AHEAD = N < 4 ? N : 4;
    bf16x8 f[AHEAD];
#pragma unroll
    for (int n = 0; n < AHEAD - 1; ++n) f[n] = l.turned(row0, n / (D / 32), n % (D / 32));
#pragma unroll
    for (int n = 0; n < N; ++n) {
        constexpr int K = AHEAD - 1;
        if (n + K < N) f[(n + K) % AHEAD] = l.turned(row0, (n + K) / (D / 32), (n + K) % (D / 32));
        acc[n % (D / 32)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[n % AHEAD], p[n / (D / 32)], acc[n % (D / 32)], 0, 0, 0);
        PAC_ATTN_PACE;
    }
}
// Is one of eight values an infinity or NaN?
__device__ __forceinline__ uint32_t special(const bf16x8 &x)
{
    const u32x4 w = __builtin_bit_cast(u32x4, x);
    uint32_t bad = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) bad |= ((w[e] & 0x7f80u) == 0x7f80u) | ((w[e] & 0x7f800000u) == 0x7f800000u);
    return bad;
}
// Do 32 rows of a tile hold one?
template <int D> __device__ __forceinline__ bool any_special(const AttnLane<D> &l, int row0)
{
    uint32_t bad = 0;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) bad |= special(l.along(row0, ks));
    return __any(bad != 0);
}
// add_turned where row x of 32 takes part in column c of the result only if part(x, c): a matrix instruction would multiply an infinity or
// NaN of a row that is masked by 0.  Row by row in the vector units, with the rows from memory, for the tiles at a mask's border that hold
// such values; rows past `have` take no part.
template <int D, class Part>
__device__ __forceinline__ void add_turned_apart(f32x16 (&acc)[D / 32], const bf16_t *base, int64_t stride, int have, int d, const bf16x8 (&p)[2],
                                                 const Part &part)
{
    const int lane = threadIdx.x & 63, h = lane >> 5;
#pragma unroll 1
    for (int x = 0; x < min(have, 32); ++x) {
        const int reg = (x >> 3) * 4 + (x & 3); // row_of, the other way round
        float px = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) px = e == reg ? (float)p[e >> 3][e & 7] : px;
        px = __shfl(px, (lane & 31) | (x >> 2 & 1) << 5, 64);
        if (part(x, lane & 31)) {
#pragma unroll
            for (int t = 0; t < D / 32; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    if (32 * t + 8 * g >= d) continue;
                    __builtin_amdgcn_sched_barrier(0); // few registers at a time: the kernels need theirs
                    const bf16x4 w = *reinterpret_cast<const bf16x4 *>(base + x * stride + 32 * t + 8 * g + 4 * h);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[t][4 * g + e] = fmaf((float)w[e], px, acc[t][4 * g + e]);
                }
        }
    }
}

// A wavefront's 32 rows of results, turned round: lane's column is its row, register i of acc[t] the value 32 t + row_of(i).
template <int D> __device__ __forceinline__ void put_rows(bf16_t *base, int64_t stride, int have, int d, const f32x16 (&acc)[D / 32], float by)
{
    const int lane = threadIdx.x & 63, i = lane & 31, h = lane >> 5;
    if (i >= have) return;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int at = 32 * t + 8 * g + 4 * h;
            bf16x4 r;
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = (bf16_t)(acc[t][4 * g + e] * by);
            if (at < d) *reinterpret_cast<bf16x4 *>(base + i * stride + at) = r;
        }
}

// Adds up what four wavefronts have for the same 32 rows: x[t] and, of each wavefront, a factor for the lane's row.  Through LDS at `at`, 16
// bytes a lane side by side; wavefront w gets the sums of x[w] (all of them where D is 128, none past D / 32).
typedef __attribute__((address_space(3))) f32x4 *lds_f32x4;
template <int D> __device__ __forceinline__ void join_put(uint32_t at, const f32x16 (&x)[D / 32])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<lds_f32x4>(at + ((wave * (D / 32) + t) * 4 + g) * 1024 + lane * 16) = f32x4{x[t][4 * g], x[t][4 * g + 1], x[t][4 * g + 2], x[t][4 * g + 3]};
}
template <int D> __device__ __forceinline__ f32x16 join_get(uint32_t at, const float (&by)[4])
{
    const int lane = threadIdx.x & 63, t = threadIdx.x >> 6;
    f32x16 r = zeros16();
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 y = *reinterpret_cast<lds_f32x4>(at + ((w * (D / 32) + t) * 4 + g) * 1024 + lane * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) r[4 * g + e] = fmaf(by[w], y[e], r[4 * g + e]);
        }
    return r;
}

// Head and number of a workgroup.  Heads vary fastest; workgroups go to the eight dies in turn, so that where their number allows it a
// die has neighbouring heads, which share keys and values, in its L2.
struct AttnWork {
    int head, number;
};
__device__ __forceinline__ AttnWork attn_work(unsigned heads)
{
    const unsigned i = blockIdx.x % heads, number = blockIdx.x / heads;
    return AttnWork{(int)(heads % 8 == 0 ? (i % 8) * (heads / 8) + i / 8 : i), (int)number};
}

// ---------------------------------------------------------------------------
// forward: one pass over the keys with a running maximum m and sum,
//     o = (sum_j 2^(s_j c - m) v_j) / (sum_j 2^(s_j c - m)),     c = scale log2 e,     lse = (m + log2 of the sum) ln 2
// 128 rows a workgroup, 32 a wavefront, which holds its queries and o in registers; 64 keys and values at a time in LDS, the
// next ones on their way.  S^T = K q^T has a query's scores in one column, so that maximum, sum and rescaling stay in a lane, and p in
// place as the operand of o^T = V^T p^T.  p is rounded to bf16 because the matrix units take it so; the sum is of the values before.
// Long sequences: 8192 tokens of 32/8 heads of 128, causal, 510 us, 1.08 PFLOP/s (a product of 8192^3: 1.23 to 1.48).  Matrix units 60 % busy, LDS reads
// 30 %, waiting 18 %, at the 1.9 GHz that such a load is given: bound by the issue of matrix and vector instructions side by side.  Short ones
// by memory and the first loads' latency: 16 x 256 tokens of 32 heads 36 us (3.8 TB/s).  Two wavefronts a SIMD use all of the registers; without
// tiles on their way and with spilled registers the first took 2173 us.  Rescaling only where a row's maximum has grown by 2^8 leaves most
// steps without it, and p below 2^8, far from where sums of fp32 end.
// ---------------------------------------------------------------------------
template <int D> struct AttnRow { // a wavefront's 32 rows on their way
    f32x16 acc[D / 32];
    float top, sum; // scores are taken relative to `top`, which stays within 2^8 of the largest so far

    // `most` is the largest of the scores at hand, in units of log 2
    __device__ __forceinline__ void raise(float most)
    {
        if (__any(most > top + 8.f)) {
            // each row for itself: what its neighbours' scores are changes no bit of it
            most = fmaxf(most, __shfl_xor(most, 32, 64));
            const float next = most > top + 8.f ? most : top, by = __builtin_amdgcn_exp2f(top - next);
            top = next;
            sum *= by;
#pragma unroll
            for (int t = 0; t < D / 32; ++t) acc[t] *= by;
        }
    }
    __device__ __forceinline__ void weigh(f32x16 &s, float c2)
    {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c2, -top));
            sum += s[i];
        }
    }
};
__device__ __forceinline__ float largest(const f32x16 &s)
{
    float most = fmaxf(s[0], s[1]);
#pragma unroll
    for (int i = 2; i < 16; i += 2) most = fmaxf(fmaxf(most, s[i]), s[i + 1]);
    return most;
}

template <int D, bool CAUSAL> __global__ __launch_bounds__(256, 2) void k_attn_fwd(const AttnArgs a)
{
    using T = AttnTile<D>;
    constexpr int BM = 128, BK = 64, TILE = BK * T::RB;
    __shared__ __attribute__((aligned(1024))) char lds[4 * TILE]; // keys, values, keys, values
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const AttnWork w = attn_work(a.heads);
    const AttnSeq seq = attn_seq<BM, CAUSAL>(a, w.number);
    if (seq.len < 1) return;
    const int head = w.head, hk = head / a.group;
    const int q0 = seq.tile * BM + wave * 32, have = min(32, seq.len - q0);
    const bf16_t *kp = a.k + (int64_t)seq.start * a.ks + (int64_t)hk * a.d, *vp = a.v + (int64_t)seq.start * a.vs + (int64_t)hk * a.d;
    const int keys = CAUSAL ? min(seq.len, seq.tile * BM + BM) : seq.len;
    const uint32_t at = lds_address(lds);

    AttnDma<D, BK> fk, fv;
    fk.plan(a.ks, a.d);
    fv.plan(a.vs, a.d);
    if (a.d != D) clear_tiles<4 * TILE>(lds);
    fk.issue(kp, at, keys);
    fv.issue(vp, at + TILE, keys);
    bf16x8 q[D / 16];
    const bf16_t *qp = a.q + (int64_t)(seq.start + q0) * a.qs + (int64_t)head * a.d;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) q[ks] = along_mem(qp, a.qs, have, a.d, ks);
    AttnRow<D> r;
#pragma unroll
    for (int t = 0; t < D / 32; ++t) r.acc[t] = zeros16();
    r.top = -FLT_MAX;
    r.sum = 0.f;
    // keys from `border` on are masked in part; the last of 32 that a query sees; their p where it has to wait for the end
    const int border = CAUSAL ? q0 : seq.len & ~31, last = CAUSAL ? lane & 31 : seq.len - 1 - border;
    bf16x8 late[2];
    bool apart = false;

    const int tiles = (keys + BK - 1) / BK, full = have < 1 ? 0 : (CAUSAL ? q0 : seq.len) / BK; // of all wavefronts; unmasked ones of this one
    auto arrive = [&](int t) {
        wait_vm<0>();
        __syncthreads(); // everybody's share of this tile is there, and the other one is free
        if (t + 1 < tiles) {
            const uint32_t to = at + (uint32_t)((t + 1) & 1) * (2 * TILE);
            fk.issue(kp + (int64_t)(t + 1) * BK * a.ks, to, keys - (t + 1) * BK);
            fv.issue(vp + (int64_t)(t + 1) * BK * a.vs, to + TILE, keys - (t + 1) * BK);
        }
    };
    const AttnLane<D> lk0(at), lv0(at + TILE);
    // an unmasked tile; in which of the two places it lies is known at compile time, so that no address is made in the loop
    auto tile = [&](auto place, int t) {
        constexpr int ROW = decltype(place)::value * (2 * BK);
        arrive(t);
        f32x16 s[2];
        scores<D, 2>(s, lk0, ROW, q);
        r.raise(fmaxf(largest(s[0]), largest(s[1])) * a.c2);
        r.weigh(s[0], a.c2);
        const bf16x8 p0[2] = {rounded(s[0], 0), rounded(s[0], 1)};
        add_turned<D>(r.acc, lv0, ROW, p0);
        r.weigh(s[1], a.c2);
        const bf16x8 p1[2] = {rounded(s[1], 0), rounded(s[1], 1)};
        add_turned<D>(r.acc, lv0, ROW + 32, p1);
    };
    int t = 0;
    for (; t + 1 < full; t += 2) {
        tile(std::integral_constant<int, 0>(), t);
        tile(std::integral_constant<int, 1>(), t + 1);
    }
    if (t < full) tile(std::integral_constant<int, 0>(), t), ++t;
    if (t < tiles && have > 0) {
        arrive(t);
        const AttnLane<D> lk(at + (uint32_t)(t & 1) * (2 * TILE)), lv(at + (uint32_t)(t & 1) * (2 * TILE) + TILE);
#pragma unroll 1
        for (int sub = 0; sub < BK; sub += 32) {
            const int key0 = t * BK + sub;
            if (key0 >= keys || (CAUSAL && key0 > q0)) break;
            f32x16 s1[1];
            scores<D, 1>(s1, lk, sub, q);
            f32x16 &s = s1[0];
            const bool cut = key0 == border;
            if (cut) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = row_of(i) <= last ? s[i] : -INFINITY;
            }
            r.raise(largest(s) * a.c2);
            r.weigh(s, a.c2);
            const bf16x8 p[2] = {rounded(s, 0), rounded(s, 1)};
            if (cut && any_special<D>(lv, sub)) {
                apart = true;
                late[0] = p[0];
                late[1] = p[1];
            } else {
                add_turned<D>(r.acc, lv, sub, p);
            }
        }
        ++t;
    }
    for (; t < tiles; ++t) arrive(t); // what other wavefronts see
    if (have < 1) return;
    if (apart) add_turned_apart<D>(r.acc, vp + (int64_t)border * a.vs, a.vs, seq.len - border, a.d, late, [&](int key, int) { return key <= last; });
    const float sum = r.sum + __shfl_xor(r.sum, 32, 64);
    put_rows<D>(a.out + (int64_t)(seq.start + q0) * a.os + (int64_t)head * a.d, a.os, have, a.d, r.acc, 1.f / sum);
    if (a.lse && lane < have) a.lse[(int64_t)head * a.rows + seq.start + q0 + lane] = (r.top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}

// ---------------------------------------------------------------------------
// forward, few rows: 32 rows a workgroup, whose four wavefronts deal the keys among them, 32 at a time, each through two LDS places of its own
// and without a barrier, and join what they have at the end.  Four times the workgroups, a quarter of the way for each; every key is fetched for
// 32 rows instead of 128, so that it pays only where the card would be mostly idle (attn_few has both sides' times).  Bound by the longest
// workgroup's chain of steps: 1788 tokens of 6 heads of 128, causal, 20 us, 14 steps a wavefront.
// ---------------------------------------------------------------------------
template <int D, bool CAUSAL> __global__ __launch_bounds__(256, 1) void k_attn_fwd_few(const AttnArgs a)
{
    using T = AttnTile<D>;
    constexpr int TILE = 32 * T::RB > 1024 ? 32 * T::RB : 1024, OWN = 4 * TILE;
    extern __shared__ __attribute__((aligned(1024))) char lds[]; // keys and values of 32 rows, twice, of each wavefront; largest scores and sums
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), me = lane & 31;
    const AttnWork w = attn_work(a.heads);
    const AttnSeq seq = attn_seq<32, CAUSAL>(a, w.number);
    if (seq.len < 1) return;
    const int head = w.head, hk = head / a.group, q0 = seq.tile * 32, have = min(32, seq.len - q0);
    const bf16_t *kp = a.k + (int64_t)seq.start * a.ks + (int64_t)hk * a.d, *vp = a.v + (int64_t)seq.start * a.vs + (int64_t)hk * a.d;
    const int subs = CAUSAL ? seq.tile + 1 : (seq.len + 31) / 32; // of all wavefronts
    const uint32_t base = lds_address(lds), at = base + wave * OWN;

    AttnDma<D, 32, 1> fk, fv;
    fk.plan(a.ks, a.d);
    fv.plan(a.vs, a.d);
    if (a.d != D) clear_tiles<4 * OWN>(lds);
    auto issue = [&](int sub) {
        const uint32_t to = at + (uint32_t)(sub >> 2 & 1) * (2 * TILE);
        fk.issue(kp + (int64_t)sub * 32 * a.ks, to, seq.len - sub * 32);
        fv.issue(vp + (int64_t)sub * 32 * a.vs, to + TILE, seq.len - sub * 32);
    };
    if (wave < subs) issue(wave);
    bf16x8 q[D / 16];
    const bf16_t *qp = a.q + (int64_t)(seq.start + q0) * a.qs + (int64_t)head * a.d;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) q[ks] = along_mem(qp, a.qs, have, a.d, ks);
    AttnRow<D> r;
#pragma unroll
    for (int t = 0; t < D / 32; ++t) r.acc[t] = zeros16();
    r.top = -FLT_MAX;
    r.sum = 0.f;
    const int last = CAUSAL ? me : seq.len - 1 - 32 * (subs - 1); // key of the last subtile
    bf16x8 late[2];
    bool apart = false;
    for (int sub = wave; sub < subs; sub += 4) {
        if (sub + 4 < subs) {
            issue(sub + 4); // (this wavefront has all that it asked of that place)
            wait_vm<fk.N + fv.N>();
        } else {
            wait_vm<0>();
        }
        const uint32_t here = at + (uint32_t)(sub >> 2 & 1) * (2 * TILE);
        const AttnLane<D> lk(here), lv(here + TILE);
        f32x16 s[1];
        scores<D, 1>(s, lk, 0, q);
        const bool cut = sub == subs - 1; // where the mask ends
        if (cut) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[0][i] = row_of(i) <= last ? s[0][i] : -INFINITY;
        }
        r.raise(largest(s[0]) * a.c2);
        r.weigh(s[0], a.c2);
        const bf16x8 p[2] = {rounded(s[0], 0), rounded(s[0], 1)};
        apart = cut && any_special<D>(lv, 0);
        if (apart) late[0] = p[0], late[1] = p[1];
        else add_turned<D>(r.acc, lv, 0, p);
    }
    if (apart) add_turned_apart<D>(r.acc, vp + (int64_t)(subs - 1) * 32 * a.vs, a.vs, seq.len - (subs - 1) * 32, a.d, late, [&](int key, int) { return key <= last; });
    r.sum += __shfl_xor(r.sum, 32, 64);

    float *stat = reinterpret_cast<float *>(lds + 4 * OWN); // [2][4][32]
    __syncthreads();
    join_put<D>(base, r.acc);
    if (lane < 32) {
        stat[wave * 32 + me] = r.top;
        stat[128 + wave * 32 + me] = r.sum;
    }
    __syncthreads();
    float by[4], top = stat[me], sum = 0.f;
#pragma unroll
    for (int x = 1; x < 4; ++x) top = fmaxf(top, stat[x * 32 + me]);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        by[x] = __builtin_amdgcn_exp2f(stat[x * 32 + me] - top);
        sum = fmaf(by[x], stat[128 + x * 32 + me], sum);
    }
    if (a.lse && wave == 0 && lane < have) a.lse[(int64_t)head * a.rows + seq.start + q0 + lane] = (top + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
    if (wave >= D / 32) return;
    const f32x16 o[1] = {join_get<D>(base, by)};
    put_rows<32>(a.out + (int64_t)(seq.start + q0) * a.os + (int64_t)head * a.d + 32 * wave, a.os, have, a.d - 32 * wave, o, 1.f / sum);
}

// ---------------------------------------------------------------------------
// backward.  Both kernels walk over subtiles of 32 x 32 pairs, whose rows come through a ring of LDS slots: two products (scores, do . v),
// 16 values of p and ds a lane, and the products that p and ds enter.  Two wavefronts share a SIMD: alone on it, one issues a vector
// instruction in every second slot at best (measured: 6.5 cycles each against 4 with two).  At 128 values a head that takes one of the
// wavefront's own two operands out of the registers: do (of dq) or v (of dk and dv) is read from LDS again for every subtile, and leaves room
// for a ring of two slots.  (4001 + 6143 tokens of 32/8 heads there and back, us: one wavefront a SIMD and four slots 2397, two wavefronts
// and two slots 2238; with three or four slots for dk and dv, one workgroup a compute unit, 2479.)
// ---------------------------------------------------------------------------
template <int D> struct AttnBack {
    using T = AttnTile<D>;
    static constexpr bool OWN = D == 128;                  // the second operand lies in LDS
    static constexpr int TILE = 32 * T::RB > 1024 ? 32 * T::RB : 1024, SLOT = 2 * TILE, RING = OWN ? 2 : 3;
    static constexpr int HELD = OWN ? 128 * T::RB : 0;     // bytes of the second operand
    static constexpr int REGS = OWN ? 1 : D / 16;
};

// s = (rows of the first tile) b1^T, dn = (rows of the second) b2^T, b2 from registers or from `own`; operands are read ahead
template <int D>
__device__ __forceinline__ void pair_products(f32x16 &s, f32x16 &dn, const AttnLane<D> &l1, const AttnLane<D> &l2, const bf16x8 (&b1)[D / 16],
                                              const bf16x8 (&b2)[AttnBack<D>::REGS], const AttnLane<D> &own)
{
    constexpr bool OWN = AttnBack<D>::OWN;
    constexpr int N = D / 16, AHEAD = OWN ? 1 : 2; // (128 values a head: two sets ahead are spilled registers; 8 x 256..1024 tokens there and back 321 us, one 287)
    bf16x8 f1[AHEAD + 1], f2[AHEAD + 1], f3[AHEAD + 1];
    auto read = [&](int n) {
        f1[n % (AHEAD + 1)] = l1.along(0, n);
        f2[n % (AHEAD + 1)] = l2.along(0, n);
        if constexpr (OWN) f3[n % (AHEAD + 1)] = own.along(0, n);
    };
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) read(n);
    s = zeros16();
    dn = zeros16();
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (n + AHEAD < N) read(n + AHEAD);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f1[n % (AHEAD + 1)], b1[n], s, 0, 0, 0);
        dn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f2[n % (AHEAD + 1)], OWN ? f3[n % (AHEAD + 1)] : b2[OWN ? 0 : n], dn, 0, 0, 0);
        PAC_ATTN_PACE;
    }
}
// acc[t] += (first tile, turned)^T p,  more[t] += (second tile, turned)^T q.  SAME: both are one tile, whose operands serve both.
template <int D, bool SAME>
__device__ __forceinline__ void pair_sums(f32x16 (&acc)[D / 32], f32x16 (&more)[D / 32], const AttnLane<D> &l1, const AttnLane<D> &l2, const bf16x8 (&p)[2],
                                          const bf16x8 (&q)[2])
{
    // product n: tile n % 2, 16 rows j, 32 values t; operand m = n, or n / 2 where both tiles are one
    constexpr int T = D / 32, N = 4 * T, M = SAME ? N / 2 : N, K = 2;
    bf16x8 g[4];
    auto read = [&](int m) { g[m % 4] = SAME ? l1.turned(0, m / T, m % T) : (m % 2 ? l2 : l1).turned(0, m / 2 / T, m / 2 % T); };
#pragma unroll
    for (int m = 0; m < K; ++m)
        if (m < M) read(m);
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int m = SAME ? n / 2 : n;
        if ((!SAME || n % 2 == 0) && m + K < M) read(m + K);
        if (n % 2) more[n / 2 % T] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(g[m % 4], q[n / 2 / T], more[n / 2 % T], 0, 0, 0);
        else acc[n / 2 % T] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(g[m % 4], p[n / 2 / T], acc[n / 2 % T], 0, 0, 0);
        PAC_ATTN_PACE;
    }
}

// ---------------------------------------------------------------------------
// dq: 128 rows a workgroup, 32 a wavefront.
//     dq_i = scale sum_j p_ij (dp_ij - delta_i) k_j
// o is at hand in bf16 only, and delta' = do . bf16(o) would make dq twice as far off as all other roundings together.  With
// r_i = sum_j p_ij (dp_ij - delta'_i), which is delta_i - delta'_i because p sums to 1, and y_i = sum_j p_ij k_j,
//     dq_i = scale (sum_j p_ij (dp_ij - delta'_i) k_j - r_i y_i)
// has the exact delta; r is small, so that p in bf16 is more than enough for y, whose products share their operand from LDS with dq's.
// delta' + r goes to memory for the other kernel, with -lse log2(e).  delta' comes from the product that makes do . v too (the diagonal of
// do o^T), so that a row with one key has exactly no gradient in q and k.
// Four products instead of three: 4001 + 6143 tokens of 32/8 heads 757 us, 1.16 PFLOP/s, matrix units 66 % busy, LDS reads 33 %, waiting 22 %,
// at 1.84 GHz; dq's error 0.0024 of its size, 0.0037 with bf16(o)'s delta.  8 x 256..1024 tokens of 32 heads 112 us: 45 % waiting for first loads.
// ---------------------------------------------------------------------------
template <int D, bool CAUSAL> __global__ __launch_bounds__(256, 2) void k_attn_dq(const AttnArgs a)
{
    using B = AttnBack<D>;
    constexpr int BM = 128, RING = B::RING;
    __shared__ __attribute__((aligned(1024))) char lds[RING * B::SLOT + B::HELD]; // 32 keys and their values a slot; do
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const AttnWork w = attn_work(a.heads);
    const AttnSeq seq = attn_seq<BM, CAUSAL>(a, w.number);
    if (seq.len < 1) return;
    const int head = w.head, hk = head / a.group;
    const int q0 = seq.tile * BM + wave * 32, have = min(32, seq.len - q0), me = lane & 31;
    const bf16_t *kp = a.k + (int64_t)seq.start * a.ks + (int64_t)hk * a.d, *vp = a.v + (int64_t)seq.start * a.vs + (int64_t)hk * a.d;
    const int keys = CAUSAL ? min(seq.len, seq.tile * BM + BM) : seq.len, tiles = (keys + 31) / 32;
    const int subs = have < 1 ? 0 : CAUSAL ? q0 / 32 + 1 : tiles; // of this wavefront
    const uint32_t at = lds_address(lds);
    const AttnLane<D> own(at + RING * B::SLOT + wave * 32 * AttnTile<D>::RB); // this wavefront's rows

    AttnDma<D, 32> fk, fv;
    fk.plan(a.ks, a.d);
    fv.plan(a.vs, a.d);
    if (a.d != D) clear_tiles<RING * B::SLOT + B::HELD>(lds);
    auto slot = [&](int tile) { return at + (uint32_t)(tile % RING) * B::SLOT; };
    auto issue = [&](int tile) {
        fk.issue(kp + (int64_t)tile * 32 * a.ks, slot(tile), keys - tile * 32);
        fv.issue(vp + (int64_t)tile * 32 * a.vs, slot(tile) + B::TILE, keys - tile * 32);
    };
    bf16x8 q[D / 16], d_o[B::REGS];
    const int64_t row = seq.start + q0;
    if constexpr (B::OWN) {
        AttnDma<D, 128> fo; // a wavefront's transfers are its own 32 rows
        fo.plan(a.dos, a.d);
        fo.issue(a.d_o + (int64_t)(seq.start + seq.tile * BM) * a.dos + (int64_t)head * a.d, at + RING * B::SLOT, seq.len - seq.tile * BM);
    }
    issue(0);
    f32x16 s = zeros16(), dp;
    if constexpr (B::OWN) wait_vm<fk.N + fv.N>();
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        q[ks] = along_mem(a.q + row * a.qs + (int64_t)head * a.d, a.qs, have, a.d, ks);
        bf16x8 x;
        if constexpr (B::OWN) x = own.along(0, ks);
        else x = d_o[ks] = along_mem(a.d_o + row * a.dos + (int64_t)head * a.d, a.dos, have, a.d, ks);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(along_mem(a.o + row * a.os + (int64_t)head * a.d, a.os, have, a.d, ks), x, s, 0, 0, 0);
    }
    const float nlse2 = me < have ? a.lse[(int64_t)head * a.rows + row + me] * -1.4426950408889634f : 0.f;
    const float delta = diagonal_of(s);
    float rest = 0.f;
    f32x16 acc[D / 32], y[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t) acc[t] = y[t] = zeros16();
    bf16x8 p[2], ds[2];
    bool apart = false;

    if (RING > 2 && tiles > 1) issue(1);
    auto arrive = [&](int n) {
        // this tile is there; with three slots the next one's transfers may still be under way
        if (RING > 2 && n + 1 < tiles) wait_vm<fk.N + fv.N>();
        else wait_vm<0>();
        __syncthreads();
        if (n + RING - 1 < tiles) issue(n + RING - 1); // in the place of the one that everybody has left behind
    };
    int n = 0;
    for (; n < subs - 1; ++n) {
        arrive(n);
        const AttnLane<D> lk(slot(n)), lv(slot(n) + B::TILE);
        pair_products<D>(s, dp, lk, lv, q, d_o, own);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float e = __builtin_amdgcn_exp2f(fmaf(s[i], a.c2, nlse2)), z = e * (dp[i] - delta);
            rest += z;
            p[i >> 3][i & 7] = (bf16_t)e;
            ds[i >> 3][i & 7] = (bf16_t)z;
        }
        pair_sums<D, true>(acc, y, lk, lk, ds, p);
    }
    if (subs > 0) { // the last subtile, where the mask ends
        arrive(n);
        const AttnLane<D> lk(slot(n)), lv(slot(n) + B::TILE);
        pair_products<D>(s, dp, lk, lv, q, d_o, own);
        const int last = CAUSAL ? me : seq.len - 1 - 32 * n;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const bool in = row_of(i) <= last;
            const float e = __builtin_amdgcn_exp2f(fmaf(s[i], a.c2, nlse2)), z = in ? e * (dp[i] - delta) : 0.f;
            rest += z;
            p[i >> 3][i & 7] = (bf16_t)(in ? e : 0.f);
            ds[i >> 3][i & 7] = (bf16_t)z;
        }
        apart = any_special<D>(lk, 0);
        if (!apart) pair_sums<D, true>(acc, y, lk, lk, ds, p);
        ++n;
    }
    for (; n < tiles; ++n) arrive(n); // what other wavefronts see
    if (have < 1) return;
    if (apart) {
        const int key0 = 32 * (subs - 1);
        auto part = [&](int key, int query) { return !CAUSAL || key <= query; };
        add_turned_apart<D>(acc, kp + (int64_t)key0 * a.ks, a.ks, seq.len - key0, a.d, ds, part);
        add_turned_apart<D>(y, kp + (int64_t)key0 * a.ks, a.ks, seq.len - key0, a.d, p, part);
    }
    rest += __shfl_xor(rest, 32, 64);
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[t][i] = fmaf(-rest, y[t][i], acc[t][i]);
    put_rows<D>(a.dq + row * a.dqs + (int64_t)head * a.d, a.dqs, have, a.d, acc, a.scale);
    if (lane < have) {
        a.nlse2[(int64_t)head * a.rows + row + lane] = nlse2;
        a.delta[(int64_t)head * a.rows + row + lane] = delta + rest;
    }
}

// dq, few rows: as the forward kernel for few rows (4096 tokens of one head of 64 there and back 168 us with 128 rows a workgroup, 98 with this)
template <int D, bool CAUSAL> __global__ __launch_bounds__(256, 1) void k_attn_dq_few(const AttnArgs a)
{
    using B = AttnBack<D>;
    constexpr int PLACE = 2 * B::SLOT, RB = AttnTile<D>::RB;
    // keys and values of 32 rows, twice, of each wavefront; do; r
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), me = lane & 31;
    const AttnWork w = attn_work(a.heads);
    const AttnSeq seq = attn_seq<32, CAUSAL>(a, w.number);
    if (seq.len < 1) return;
    const int head = w.head, hk = head / a.group, q0 = seq.tile * 32, have = min(32, seq.len - q0);
    const int64_t row = seq.start + q0;
    const bf16_t *kp = a.k + (int64_t)seq.start * a.ks + (int64_t)hk * a.d, *vp = a.v + (int64_t)seq.start * a.vs + (int64_t)hk * a.d;
    const int subs = CAUSAL ? seq.tile + 1 : (seq.len + 31) / 32; // of all wavefronts
    const uint32_t base = lds_address(lds), at = base + wave * PLACE;
    const AttnLane<D> own(base + 4 * PLACE);

    AttnDma<D, 32, 1> fk, fv;
    fk.plan(a.ks, a.d);
    fv.plan(a.vs, a.d);
    if (a.d != D) clear_tiles<4 * PLACE + (B::OWN ? 32 * RB : 0)>(lds);
    bf16x8 q[D / 16], d_o[B::REGS];
    if constexpr (B::OWN) {
        AttnDma<D, 32> fo;
        fo.plan(a.dos, a.d);
        fo.issue(a.d_o + row * a.dos + (int64_t)head * a.d, base + 4 * PLACE, have);
        wait_vm<0>();
        __syncthreads();
    }
    auto issue = [&](int sub) {
        const uint32_t to = at + (uint32_t)(sub >> 2 & 1) * B::SLOT;
        fk.issue(kp + (int64_t)sub * 32 * a.ks, to, seq.len - sub * 32);
        fv.issue(vp + (int64_t)sub * 32 * a.vs, to + B::TILE, seq.len - sub * 32);
    };
    if (wave < subs) issue(wave);
    f32x16 s = zeros16(), dp;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        q[ks] = along_mem(a.q + row * a.qs + (int64_t)head * a.d, a.qs, have, a.d, ks);
        bf16x8 x;
        if constexpr (B::OWN) x = own.along(0, ks);
        else x = d_o[ks] = along_mem(a.d_o + row * a.dos + (int64_t)head * a.d, a.dos, have, a.d, ks);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(along_mem(a.o + row * a.os + (int64_t)head * a.d, a.os, have, a.d, ks), x, s, 0, 0, 0);
    }
    const float nlse2 = me < have ? a.lse[(int64_t)head * a.rows + row + me] * -1.4426950408889634f : 0.f;
    const float delta = diagonal_of(s);
    float rest = 0.f;
    f32x16 acc[D / 32], y[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t) acc[t] = y[t] = zeros16();
    const int last = CAUSAL ? me : seq.len - 1 - 32 * (subs - 1);
    bf16x8 p[2], ds[2];
    bool apart = false;
    for (int sub = wave; sub < subs; sub += 4) {
        if (sub + 4 < subs) {
            issue(sub + 4); // (this wavefront has all that it asked of that place)
            wait_vm<fk.N + fv.N>();
        } else {
            wait_vm<0>();
        }
        const uint32_t here = at + (uint32_t)(sub >> 2 & 1) * B::SLOT;
        const AttnLane<D> lk(here), lv(here + B::TILE);
        pair_products<D>(s, dp, lk, lv, q, d_o, own);
        const bool cut = sub == subs - 1; // where the mask ends
        const int to = cut ? last : 31;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const bool in = row_of(i) <= to;
            const float e = __builtin_amdgcn_exp2f(fmaf(s[i], a.c2, nlse2)), z = in ? e * (dp[i] - delta) : 0.f;
            rest += z;
            p[i >> 3][i & 7] = (bf16_t)(in ? e : 0.f);
            ds[i >> 3][i & 7] = (bf16_t)z;
        }
        apart = cut && any_special<D>(lk, 0);
        if (!apart) pair_sums<D, true>(acc, y, lk, lk, ds, p);
    }
    if (apart) {
        const int key0 = 32 * (subs - 1);
        auto part = [&](int key, int query) { return !CAUSAL || key <= query; };
        add_turned_apart<D>(acc, kp + (int64_t)key0 * a.ks, a.ks, seq.len - key0, a.d, ds, part);
        add_turned_apart<D>(y, kp + (int64_t)key0 * a.ks, a.ks, seq.len - key0, a.d, p, part);
    }
    rest += __shfl_xor(rest, 32, 64);

    float *stat = reinterpret_cast<float *>(lds + 4 * PLACE + (B::OWN ? 32 * RB : 0)); // [4][32]
    __syncthreads();
    join_put<D>(base, acc);
    join_put<D>(base + D * 512, y); // 4 wavefronts x D / 32 x 4 KB after the other
    if (lane < 32) stat[wave * 32 + me] = rest;
    __syncthreads();
    rest = (stat[me] + stat[32 + me]) + (stat[64 + me] + stat[96 + me]);
    if (wave == 0 && lane < have) {
        a.nlse2[(int64_t)head * a.rows + row + lane] = nlse2;
        a.delta[(int64_t)head * a.rows + row + lane] = delta + rest;
    }
    if (wave >= D / 32) return;
    const float one[4] = {1.f, 1.f, 1.f, 1.f};
    f32x16 sum[1] = {join_get<D>(base, one)};
    const f32x16 ys = join_get<D>(base + D * 512, one);
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[0][i] = fmaf(-rest, ys[i], sum[0][i]);
    put_rows<32>(a.dq + row * a.dqs + (int64_t)head * a.d + 32 * wave, a.dqs, have, a.d - 32 * wave, sum, a.scale);
}

// ---------------------------------------------------------------------------
// dk and dv: 128 keys a workgroup, 32 a wavefront, which holds them, their values and both gradients in registers; 32 queries and their
// do at a time in LDS, of all heads of the group one after the other.  S = q K^T has a key's scores in one column.
// The first keys of a long causal sequence have all of its queries to go through, and a launch ends with its longest workgroup, so the
// queries may be dealt to several (attn_splits), whose sums another launch adds up in order.
// 4001 + 6143 tokens of 32/8 heads of 128: 859 us, 1.03 PFLOP/s, matrix units 57 % busy, LDS reads 43 %, waiting 37 % (a barrier for every 32
// queries, and two splits' workgroups of unequal lengths); 8 x 256..1024 tokens of 32 heads 131 us, 32 x 1..128 of 12 of 64 11 us: first loads.
// Measured and not kept: eight wavefronts a workgroup (950 instead of 1025 us then, but 32 x 1..128 16.2 instead of 11.6), queries from
// the last to the first (373 instead of 325), the next tile's operands asked for before the barrier (2529 instead of 2397 there and back).
// ---------------------------------------------------------------------------
template <int D, bool CAUSAL> __global__ __launch_bounds__(256, 2) void k_attn_dkv(const AttnArgs a)
{
    using B = AttnBack<D>;
    constexpr int BN = 128, RING = B::RING;
    __shared__ __attribute__((aligned(1024))) char lds[RING * B::SLOT + B::HELD + RING * 256]; // 32 queries and their do a slot; v; -lse log2(e) and delta
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), me = lane & 31;
    const AttnWork w = attn_work(a.kv_heads);
    const int split = w.number % a.splits;
    const AttnSeq seq = attn_seq<BN, CAUSAL, true>(a, w.number / a.splits);
    if (seq.len < 1) return;
    const int hk = w.head, key0 = seq.tile * BN + wave * 32, have = min(32, seq.len - key0);
    const int64_t row = seq.start + key0;
    const int first = CAUSAL ? seq.tile * BN : 0, per = (seq.len - first + 31) / 32; // subtiles of a head
    const int from_tile = (int)((int64_t)per * a.group * split / a.splits), tiles = (int)((int64_t)per * a.group * (split + 1) / a.splits) - from_tile; // of this workgroup
    const uint32_t at = lds_address(lds);
    const AttnLane<D> own(at + RING * B::SLOT + wave * 32 * AttnTile<D>::RB); // this wavefront's rows

    AttnDma<D, 32> fq, fd;
    fq.plan(a.qs, a.d);
    fd.plan(a.dos, a.d);
    if (a.d != D) clear_tiles<RING * B::SLOT + B::HELD>(lds);
    auto slot = [&](int tile) { return at + (uint32_t)(tile % RING) * B::SLOT; };
    auto stats = [&](int tile) { return at + RING * B::SLOT + B::HELD + (uint32_t)(tile % RING) * 256; };
    // the tile to be fetched next: its number, how many rows of its head are left, and where they are
    const int head0 = hk * a.group + from_tile / per, skip = from_tile % per * 32;
    int f_tile = 0, f_rest = seq.len - first - skip;
    const bf16_t *f_q = a.q + (int64_t)(seq.start + first + skip) * a.qs + (int64_t)head0 * a.d;
    const bf16_t *f_d = a.d_o + (int64_t)(seq.start + first + skip) * a.dos + (int64_t)head0 * a.d;
    const float *f_s = (lane < 32 ? a.nlse2 : a.delta) + (int64_t)head0 * a.rows + seq.start + first + skip;
    auto issue = [&]() {
        fq.issue(f_q, slot(f_tile), f_rest);
        fd.issue(f_d, slot(f_tile) + B::TILE, f_rest);
        // every wavefront fetches them, so that all have as many transfers under way
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
                     : : "s"(__builtin_amdgcn_readfirstlane(stats(f_tile))), "v"(f_s + min(me, f_rest - 1)) : "memory", "m0");
        ++f_tile;
        f_rest -= 32;
        f_q += 32 * a.qs, f_d += 32 * a.dos, f_s += 32;
        if (f_rest <= 0) { // on to the next head
            f_rest = seq.len - first;
            f_q += a.d - (int64_t)per * 32 * a.qs, f_d += a.d - (int64_t)per * 32 * a.dos, f_s += a.rows - (int64_t)per * 32;
        }
    };
    bf16x8 k[D / 16], v[B::REGS];
    if constexpr (B::OWN) {
        AttnDma<D, 128> fv; // a wavefront's transfers are its own 32 rows
        fv.plan(a.vs, a.d);
        fv.issue(a.v + (int64_t)(seq.start + seq.tile * BN) * a.vs + (int64_t)hk * a.d, at + RING * B::SLOT, seq.len - seq.tile * BN);
    }
    if (tiles > 0) issue();
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        k[ks] = along_mem(a.k + row * a.ks + (int64_t)hk * a.d, a.ks, have, a.d, ks);
        if constexpr (!B::OWN) v[ks] = along_mem(a.v + row * a.vs + (int64_t)hk * a.d, a.vs, have, a.d, ks);
    }
    if (RING > 2 && tiles > 1) issue();
    f32x16 dk[D / 32], dv[D / 32], s, dp;
#pragma unroll
    for (int t = 0; t < D / 32; ++t) dk[t] = dv[t] = zeros16();
    bf16x8 p[2], ds[2];
    int n = 0; // tiles so far
    auto arrive = [&]() {
        if (RING > 2 && n + 1 < tiles) wait_vm<fq.N + fd.N + 1>();
        else wait_vm<0>();
        __syncthreads();
        if (n + RING - 1 < tiles) issue();
        ++n;
    };
    auto queries = [&]() { return AttnLane<D>(slot(n - 1)); }; // the tile that has arrived
    auto grads = [&]() { return AttnLane<D>(slot(n - 1) + B::TILE); };
    auto weigh = [&](auto in) { // p and ds; in(row): does the row see the lane's key
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const uint32_t st = stats(n - 1) + 16 * (lane >> 5) + 32 * g;
            const f32x4 nl = *reinterpret_cast<lds_f32x4>(st), dl = *reinterpret_cast<lds_f32x4>(st + 128);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int i = 4 * g + x;
                const float e = __builtin_amdgcn_exp2f(fmaf(s[i], a.c2, nl[x])), z = e * (dp[i] - dl[x]);
                p[i >> 3][i & 7] = (bf16_t)(in(row_of(i)) ? e : 0.f);
                ds[i >> 3][i & 7] = (bf16_t)(in(row_of(i)) ? z : 0.f);
            }
        }
    };
    // this wavefront's subtiles of a head: the first ones, where causal queries see none of its keys; then the diagonal, the main ones, and
    // one that ends with the sequence
    const int idle = have < 1 ? per : CAUSAL ? wave : 0, odd_end = seq.len % 32 != 0 && per - idle > (CAUSAL ? 1 : 0);
    bool apart = false; // some subtile at a mask's border has to be added row by row
    int left = tiles;
#pragma unroll 1
    for (int j0 = from_tile % per; left > 0; j0 = 0) { // subtiles j0..j1 - 1 of a head
        const int j1 = min(per, j0 + left);
        left -= j1 - j0;
        for (int j = j0; j < min(idle, j1); ++j) arrive();
        if (idle >= j1) continue;
        const int middle = min(j1, per - odd_end) - max(j0, idle + (CAUSAL ? 1 : 0));
#pragma unroll 1
        for (int side = 0; side < 2; ++side) {
            if (side == 0 ? CAUSAL && j0 <= idle : odd_end && j1 == per) {
                const int qr = side == 0 ? key0 : seq.len & ~31;
                arrive();
                if (any_special<D>(queries(), 0) || any_special<D>(grads(), 0)) {
                    apart = true;
                } else {
                    pair_products<D>(s, dp, queries(), grads(), k, v, own);
                    const int from = CAUSAL && qr == key0 ? me : 0, to = seq.len - qr; // the queries that see the lane's key
                    weigh([&](int r) { return r >= from && r < to; });
                    pair_sums<D, false>(dv, dk, grads(), queries(), p, ds);
                }
            }
            if (side == 0) {
                for (int i = 0; i < middle; ++i) {
                    arrive();
                    pair_products<D>(s, dp, queries(), grads(), k, v, own);
                    weigh([](int) { return true; });
                    pair_sums<D, false>(dv, dk, grads(), queries(), p, ds);
                }
            }
        }
    }
    if (have > 0 && apart) { // such subtiles again, their rows from memory
#pragma unroll 1
        for (int which = 0; which < 2 * a.group; ++which) {
            const int head = hk * a.group + which / 2, qr = which % 2 == 0 ? key0 : seq.len & ~31, to = seq.len - qr;
            const int tile = which / 2 * per + (qr - first) / 32 - from_tile;
            if ((which % 2 == 0 ? !CAUSAL : !odd_end) || tile < 0 || tile >= tiles) continue;
            const int64_t r0 = seq.start + qr;
            const bf16_t *qp = a.q + r0 * a.qs + (int64_t)head * a.d, *dp_ = a.d_o + r0 * a.dos + (int64_t)head * a.d;
            const int64_t st = (int64_t)head * a.rows + r0;
            s = zeros16(), dp = zeros16();
            uint32_t bad = 0;
#pragma unroll 1
            for (int ks = 0; ks < D / 16; ++ks) {
                const bf16x8 x = along_mem(qp, a.qs, to, a.d, ks), z = along_mem(dp_, a.dos, to, a.d, ks);
                const bf16x8 kk = along_mem(a.k + row * a.ks + (int64_t)hk * a.d, a.ks, have, a.d, ks), vv = along_mem(a.v + row * a.vs + (int64_t)hk * a.d, a.vs, have, a.d, ks);
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, kk, s, 0, 0, 0);
                dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(z, vv, dp, 0, 0, 0);
                bad |= special(x) | special(z);
            }
            if (!__any(bad != 0)) continue; // this one is in
            const int from = CAUSAL && qr == key0 ? me : 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = row_of(i);
                const bool in = r >= from && r < to;
                const float e = in ? __builtin_amdgcn_exp2f(fmaf(s[i], a.c2, a.nlse2[st + min(r, to - 1)])) : 0.f;
                p[i >> 3][i & 7] = (bf16_t)e;
                ds[i >> 3][i & 7] = (bf16_t)(in ? e * (dp[i] - a.delta[st + min(r, to - 1)]) : 0.f);
            }
            auto part = [&](int query, int) { return query >= from; };
            add_turned_apart<D>(dv, dp_, a.dos, to, a.d, p, part);
            add_turned_apart<D>(dk, qp, a.qs, to, a.d, ds, part);
        }
    }
    if (have < 1) return;
    if (a.splits == 1) {
        put_rows<D>(a.dk + row * a.dks + (int64_t)hk * a.d, a.dks, have, a.d, dk, a.scale);
        put_rows<D>(a.dv + row * a.dvs + (int64_t)hk * a.d, a.dvs, have, a.d, dv, 1.f);
        return;
    }
    const int64_t cols = (int64_t)a.kv_heads * a.d;
    float *to = a.part + (((int64_t)split * a.rows + row + me) * 2 * a.kv_heads + hk) * a.d;
    if (me < have) {
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int c = 32 * t + 8 * g + 4 * (lane >> 5);
                if (c >= a.d) continue;
                *reinterpret_cast<f32x4 *>(to + c) = f32x4{dk[t][4 * g], dk[t][4 * g + 1], dk[t][4 * g + 2], dk[t][4 * g + 3]};
                *reinterpret_cast<f32x4 *>(to + cols + c) = f32x4{dv[t][4 * g], dv[t][4 * g + 1], dv[t][4 * g + 2], dv[t][4 * g + 3]};
            }
    }
}

// The splits' sums, in order: eight values a thread of dk or dv.  Bound by memory: 10144 rows, two splits of 8 heads of 128, 32 us (166 MB read, 42
// written: 6.5 TB/s, partly from the last cache).
__global__ __launch_bounds__(256) void k_attn_join(const AttnArgs a)
{
    const int chunks = a.kv_heads * a.d / 8;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, r = id / (2 * chunks);
    const int c = (int)(id - r * 2 * chunks), first = min(max(a.off[0], 0), a.rows), end = min(max(a.off[a.batch], 0), a.rows);
    if (r < first || r >= end) return;
    const bool is_v = c >= chunks;
    const float *from = a.part + r * 2 * a.kv_heads * a.d + (int64_t)c * 8;
    f32x4 x = *reinterpret_cast<const f32x4 *>(from), y = *reinterpret_cast<const f32x4 *>(from + 4);
    for (int s = 1; s < a.splits; ++s) {
        from += (int64_t)a.rows * 2 * a.kv_heads * a.d;
        x += *reinterpret_cast<const f32x4 *>(from);
        y += *reinterpret_cast<const f32x4 *>(from + 4);
    }
    const float by = is_v ? 1.f : a.scale;
    bf16x8 z;
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = (bf16_t)(x[e] * by), z[4 + e] = (bf16_t)(y[e] * by);
    *reinterpret_cast<bf16x8 *>((is_v ? a.dv + r * a.dvs : a.dk + r * a.dks) + (int64_t)(is_v ? c - chunks : c) * 8) = z;
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
static inline bool at_aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// What scores are taken times; infinite, it would make a score of 0 no number
static float attn_c2(const pac_attn *a) { return a->scale * 1.4426950408889634f; }
static pac_status check_attn(const pac_attn *a, int32_t batch, int64_t rows)
{
    if (!a) return PAC_ERR_NULL;
    if (a->heads < 1 || a->heads > 4096 || a->kv_heads < 1 || a->heads % a->kv_heads || a->d < 8 || a->d > 128 || a->d % 8 ||
        (a->causal != 0 && a->causal != 1) || !(a->scale > 0.f) || !std::isfinite(attn_c2(a)) || batch < 0)
        return PAC_ERR_SHAPE;
    if (rows < 0 || rows > INT32_MAX) return PAC_ERR_RANGE;
    if ((rows / 128 + batch) * a->heads >= 1 << 23) return PAC_ERR_UNSUPPORTED;
    return PAC_OK;
}
struct AttnRows { // a matrix of states
    const void *at;
    int64_t stride, cols;
};
static pac_status check_rows(const AttnRows &m)
{
    const int64_t cols = m.cols;
    if (m.stride < cols) return PAC_ERR_RANGE;
    if (m.stride % 8 || !at_aligned(m.at, 16)) return PAC_ERR_ALIGN;
    return m.stride > 1 << 24 ? PAC_ERR_UNSUPPORTED : PAC_OK;
}
static Span rows_span(const AttnRows &m, int64_t rows) { return Span(m.at, rows, m.stride * 2, m.cols * 2); }

static AttnArgs attn_args(const pac_attn *a, const int32_t *off, int32_t batch, int64_t rows)
{
    AttnArgs r{};
    r.off = off; r.batch = batch; r.rows = (int)rows;
    r.heads = a->heads; r.kv_heads = a->kv_heads; r.group = a->heads / a->kv_heads; r.d = a->d;
    r.scale = a->scale; r.c2 = attn_c2(a);
    return r;
}
// Numbers of a head's tiles of `of` rows, all sequences together (attn_seq)
static unsigned attn_numbers(int32_t batch, int64_t rows, int of) { return (unsigned)(rows / of + batch); }
static int64_t stat_bytes(const pac_attn *a, int64_t rows) { return (rows * a->heads * 4 + 255) / 256 * 256; }

// Whether a call's rows are few: forward and dq then take 32 rows a workgroup and deal the keys to its wavefronts.  Up to 64 values a head two such
// workgroups share a compute unit, past that one has it alone.  Us, 128 rows / 32 rows a workgroup (workgroups of 128 rows in brackets):
//   causal, 128 values, forward   1000 tokens of 10 heads (80) 24.0 / 16.1, 1788 of 6 (84) 36.1 / 22.0, 4000 of 5 (160) 70.2 / 61.1, 1600 of 12 (156)
//                                 32.2 / 32.5, but 1000 of 20 (160) 25.3 / 28.0, 2000 of 12 (192) 38.9 / 42.5, 4000 of 8 (256) 73.0 / 83.9
//           64 values             2000 of 12 (192) 27.4 / 19.7, 8000 of 4 (252) 92.5 / 71.9, but 1000 of 40 (320) 18.5 / 23.0, 4000 of 12 (384) 54.2 / 61.6
//   not causal, 128 values        1500 of 5 (60) 31.6 / 20.6, but 1600 of 6 (78) 32.1 / 37.4; all tiles take as long there
//           64 values             4000 of 4 (128) 48.1 / 33.9, 1000 of 16 (128) 17.1 / 12.8, but 2000 of 16 (256) 30.6 / 38.7
// and there and back as these or better.  The rule counts workgroups and does not know how long their chains of keys are, which is what decides near its bounds: at 160
// it takes the faster form for 4000 tokens of 5 heads and the slower one for 1000 of 20.  Below some 100 tokens there is nothing to deal: 19 tokens 8.2 / 8.7.
static bool attn_few(const pac_attn *a, int32_t batch, int64_t rows)
{
    const int64_t most = a->d > 64 ? (a->causal ? 160 : 72) : (a->causal ? 256 : 128);
    return (rows / 128 + batch) * a->heads <= most && rows >= 128 * (int64_t)batch;
}
// Starts a kernel with that much LDS
template <typename K> static bool attn_launch(K kernel, unsigned blocks, int lds, hipStream_t st, const AttnArgs &r)
{
    if (lds > 64 << 10 && hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess) return false;
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), lds, st, r);
    return true;
}
template <int D> static int few_lds(bool back)
{
    const int place = 4 * AttnBack<D>::TILE;
    return back ? 4 * place + (AttnBack<D>::OWN ? 32 * AttnTile<D>::RB : 0) + 512 : 4 * place + 1024;
}

// Workgroups that share a tile of keys in dk and dv, i.e. parts that its queries are dealt into: by estimated time.  A subtile of 32 x 32 takes
// 1.8 us at 128 values a head, 1.26 at 64; a launch takes as long as its longest workgroup (the first keys of a sequence of average length), or as all
// of them together at 384 a time, and a tenth of the other (lengths are on the device: a batch of one long and many short or empty sequences is taken for
// one of average ones, and its long one gets fewer parts than alone); more than 512 workgroups slow each other by 13 %; sums that go through memory cost
// 2 us and their bytes, written and read, at 6.7 TB/s.  The estimate's best among 1, 2, 3, 4, 6, 8, 12, 16 is 0.9 % slower on the average than the best measured
// over 27 calls; there and back, us, 1 / 2 / 4 / 8 / 16 parts (the estimate's choice): 4001 + 6143 tokens of 32/8 heads of 128 2179 / 2044 / 2063 / 2185 /
// 2495 (2), 2048 of 32/8 416 / 293 / 245 / 253 / 313 (6: 242), 4 x 300..600 of 32/8 178 / 134 / 119 / 137 / 179 (4), 500 of 64 heads of 64 on one key head
// 1026 / 537 / 287 / 143 / 105 (16), 16 x 100..200 of 16/4 heads of 64 73 / 58 / 53 / 57 / 70 (3: 52), 4 x 1024 of 8 heads of 64 114 / 128 / 154 / 214 / 360 (1).
constexpr int64_t kAttnTarget = 1300, kAttnSplits = 64; // workgroups and parts at most
static int attn_splits(const pac_attn *a, int32_t batch, int64_t rows)
{
    const int64_t groups = (rows / 128 + batch) * a->kv_heads;
    if (groups < 1 || batch < 1) return 1;
    const double longest = (double)rows / batch * (a->heads / a->kv_heads) / 32; // subtiles
    const double each = 1.8 * (0.4 + 0.6 / 128 * a->d), all = longest * (a->causal ? 0.5 : 1) * groups * each * 1.13 / 384;
    const double bytes = (double)rows * a->kv_heads * a->d * 8;
    double best = 0;
    int splits = 1;
    for (int64_t s = 1; s <= kAttnSplits && (s == 1 || (s * groups <= kAttnTarget && s <= longest)); ++s) {
        const double chain = longest / s * each * (groups * s > 512 ? 1.13 : 1);
        const double t = (chain > all ? chain + 0.1 * all : all + 0.1 * chain) + (s > 1 ? 2 + 0.3e-6 * bytes * s : 0);
        if (s == 1 || t < best) best = t, splits = (int)s;
    }
    return splits;
}
static int64_t part_bytes(const pac_attn *a, int64_t rows, int64_t splits) { return splits < 2 ? 0 : rows * 2 * a->kv_heads * a->d * 4 * splits; }
static int64_t attn_bytes(const pac_attn *a, int32_t batch, int64_t rows) { return 2 * stat_bytes(a, rows) + part_bytes(a, rows, attn_splits(a, batch, rows)); }

template <typename F> static void by_width(int d, const F &f)
{
    if (d <= 32) f(std::integral_constant<int, 32>());
    else if (d <= 64) f(std::integral_constant<int, 64>());
    else if (d <= 96) f(std::integral_constant<int, 96>());
    else f(std::integral_constant<int, 128>());
}

} // namespace pac

using namespace pac;

extern "C" {

pac_status pac_attn_forward(const pac_attn *a, const int32_t *offsets, int32_t batch, int64_t rows, const void *q, int64_t q_stride,
                            const void *k, int64_t k_stride, const void *v, int64_t v_stride, void *o, int64_t o_stride, float *lse,
                            void *hip_stream)
{
    pac_status s = check_attn(a, batch, rows);
    if (s != PAC_OK) return s;
    if (batch == 0 || rows == 0) return PAC_OK;
    if (!offsets || !q || !k || !v || !o) return PAC_ERR_NULL;
    const int64_t qc = (int64_t)a->heads * a->d, kc = (int64_t)a->kv_heads * a->d;
    const AttnRows qm{q, q_stride, qc}, km{k, k_stride, kc}, vm{v, v_stride, kc}, om{o, o_stride, qc};
    for (const AttnRows &m : {qm, km, vm, om})
        if ((s = check_rows(m)) != PAC_OK) return s;
    if (!at_aligned(offsets, 4) || !at_aligned(lse, 4)) return PAC_ERR_ALIGN;
    const Span os = rows_span(om, rows), ls(lse, lse ? rows * a->heads * 4 : 0), off(offsets, ((int64_t)batch + 1) * 4);
    const Span qs = rows_span(qm, rows), ks = rows_span(km, rows), vs = rows_span(vm, rows);
    if (shares(os, {qs, ks, vs, ls, off}) || shares(ls, {qs, ks, vs, off})) return PAC_ERR_RANGE;
    AttnArgs r = attn_args(a, offsets, batch, rows);
    r.q = static_cast<const bf16_t *>(q); r.qs = q_stride;
    r.k = static_cast<const bf16_t *>(k); r.ks = k_stride;
    r.v = static_cast<const bf16_t *>(v); r.vs = v_stride;
    r.out = static_cast<bf16_t *>(o); r.os = o_stride;
    r.lse = lse;
    (void)hipGetLastError();
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    bool ok = true;
    by_width(a->d, [&](auto n) {
        constexpr int D = decltype(n)::value;
        if (attn_few(a, batch, rows)) {
            const unsigned grid = attn_numbers(batch, rows, 32) * r.heads;
            ok = a->causal ? attn_launch(k_attn_fwd_few<D, true>, grid, few_lds<D>(false), st, r) : attn_launch(k_attn_fwd_few<D, false>, grid, few_lds<D>(false), st, r);
            return;
        }
        const dim3 grid(attn_numbers(batch, rows, 128) * r.heads);
        if (a->causal) hipLaunchKernelGGL((k_attn_fwd<D, true>), grid, dim3(256), 0, st, r);
        else hipLaunchKernelGGL((k_attn_fwd<D, false>), grid, dim3(256), 0, st, r);
    });
    if (!ok) return PAC_ERR_DEVICE;
    return hipGetLastError() == hipSuccess ? PAC_OK : PAC_ERR_DEVICE;
}

int64_t pac_attn_workspace_bytes(const pac_attn *a, int32_t batch, int64_t rows)
{
    if (check_attn(a, batch, rows) != PAC_OK) return -1;
    // splits become fewer as tiles become more: room for as many (row, split) pairs as a call of at most this size may have
    int64_t most = rows * (a->heads / a->kv_heads) / 32, pairs;
    most = most > kAttnSplits ? kAttnSplits : most;
    pairs = most < 2 ? 0 : rows * most;
    const int64_t filled = kAttnTarget * 128 / a->kv_heads + 128 * kAttnSplits;
    if (pairs > filled) pairs = filled;
    return 2 * stat_bytes(a, rows) + pairs * 2 * a->kv_heads * a->d * 4;
}

int64_t pac_attn_backward_bytes(const pac_attn *a, int32_t batch, int64_t rows)
{
    return check_attn(a, batch, rows) == PAC_OK ? attn_bytes(a, batch, rows) : -1;
}

pac_status pac_attn_backward(const pac_attn *a, const int32_t *offsets, int32_t batch, int64_t rows, const void *q, int64_t q_stride,
                             const void *k, int64_t k_stride, const void *v, int64_t v_stride, const void *o, int64_t o_stride,
                             const float *lse, const void *do_, int64_t do_stride, void *dq, int64_t dq_stride, void *dk,
                             int64_t dk_stride, void *dv, int64_t dv_stride, void *workspace, int64_t workspace_bytes, void *hip_stream)
{
    pac_status s = check_attn(a, batch, rows);
    if (s != PAC_OK) return s;
    if (batch == 0 || rows == 0) return PAC_OK;
    if (!offsets || !q || !k || !v || !o || !lse || !do_ || !dq || !dk || !dv || !workspace) return PAC_ERR_NULL;
    const int64_t qc = (int64_t)a->heads * a->d, kc = (int64_t)a->kv_heads * a->d;
    const AttnRows qm{q, q_stride, qc}, km{k, k_stride, kc}, vm{v, v_stride, kc}, om{o, o_stride, qc}, dom{do_, do_stride, qc};
    const AttnRows dqm{dq, dq_stride, qc}, dkm{dk, dk_stride, kc}, dvm{dv, dv_stride, kc};
    for (const AttnRows &m : {qm, km, vm, om, dom, dqm, dkm, dvm})
        if ((s = check_rows(m)) != PAC_OK) return s;
    if (!at_aligned(offsets, 4) || !at_aligned(lse, 4) || !at_aligned(workspace, 16)) return PAC_ERR_ALIGN;
    const int64_t need = attn_bytes(a, batch, rows);
    if (workspace_bytes < need) return PAC_ERR_WORKSPACE;
    const Span qs = rows_span(qm, rows), ks = rows_span(km, rows), vs = rows_span(vm, rows), os = rows_span(om, rows);
    const Span ds = rows_span(dom, rows), ls(lse, rows * a->heads * 4), off(offsets, ((int64_t)batch + 1) * 4);
    const Span outs[] = {rows_span(dqm, rows), rows_span(dkm, rows), rows_span(dvm, rows), Span(workspace, need)};
    for (const Span &u : outs) {
        if (shares(u, {qs, ks, vs, os, ds, ls, off})) return PAC_ERR_RANGE;
        for (const Span &x : outs)
            if (&u != &x && share(u, x)) return PAC_ERR_RANGE;
    }
    AttnArgs r = attn_args(a, offsets, batch, rows);
    r.q = static_cast<const bf16_t *>(q); r.qs = q_stride;
    r.k = static_cast<const bf16_t *>(k); r.ks = k_stride;
    r.v = static_cast<const bf16_t *>(v); r.vs = v_stride;
    r.o = static_cast<const bf16_t *>(o); r.os = o_stride;
    r.d_o = static_cast<const bf16_t *>(do_); r.dos = do_stride;
    r.dq = static_cast<bf16_t *>(dq); r.dqs = dq_stride;
    r.dk = static_cast<bf16_t *>(dk); r.dks = dk_stride;
    r.dv = static_cast<bf16_t *>(dv); r.dvs = dv_stride;
    r.lse = const_cast<float *>(lse);
    r.nlse2 = static_cast<float *>(workspace);
    r.delta = reinterpret_cast<float *>(static_cast<char *>(workspace) + stat_bytes(a, rows));
    r.part = reinterpret_cast<float *>(static_cast<char *>(workspace) + 2 * stat_bytes(a, rows));
    r.splits = attn_splits(a, batch, rows);
    const unsigned tiles = attn_numbers(batch, rows, 128);
    (void)hipGetLastError();
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    bool ok = true;
    by_width(a->d, [&](auto n) {
        constexpr int D = decltype(n)::value;
        if (attn_few(a, batch, rows)) {
            const unsigned grid = attn_numbers(batch, rows, 32) * r.heads;
            ok = a->causal ? attn_launch(k_attn_dq_few<D, true>, grid, few_lds<D>(true), st, r) : attn_launch(k_attn_dq_few<D, false>, grid, few_lds<D>(true), st, r);
            if (!ok) return;
        } else if (a->causal) {
            hipLaunchKernelGGL((k_attn_dq<D, true>), dim3(tiles * r.heads), dim3(256), 0, st, r);
        } else {
            hipLaunchKernelGGL((k_attn_dq<D, false>), dim3(tiles * r.heads), dim3(256), 0, st, r);
        }
        if (a->causal) hipLaunchKernelGGL((k_attn_dkv<D, true>), dim3(tiles * r.kv_heads * r.splits), dim3(256), 0, st, r);
        else hipLaunchKernelGGL((k_attn_dkv<D, false>), dim3(tiles * r.kv_heads * r.splits), dim3(256), 0, st, r);
    });
    if (!ok) return PAC_ERR_DEVICE;
    if (r.splits > 1) hipLaunchKernelGGL(k_attn_join, dim3((unsigned)((rows * 2 * kc / 8 + 255) / 256)), dim3(256), 0, st, r);
    return hipGetLastError() == hipSuccess ? PAC_OK : PAC_ERR_DEVICE;
}

} // extern "C"
