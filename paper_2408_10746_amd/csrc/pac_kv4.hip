// A key and value cache in microscaled 4-bit floating point: its writing and reading back, and single-token attention over it
// (declared in include/pac_kv4.h).
#include "../../include/pac_kv4.h"
#include "pac_gemm.h"
#include "pac_span.h"
#include <cfloat>
#include <cmath>

namespace pac {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

static inline bool kv_aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// ---------------------------------------------------------------------------
// The order inside a page.  A head of NB blocks of 32 takes 34 NB bytes a token; the page's tokens of one head lie together:
//   K codes [page][16 NB]   V codes [page / 4][16 lanes][4 tokens][NB]   K scales [page][NB]   V scales [page / 4][NB][4 tokens]
// so that attention's lanes load what their matrix instructions contract, in 4 NB contiguous bytes, 16 lanes side by side:
//   K  lane (token, g), g = 0..3, holds 8 NB values of its token, chunk i of eight of them: values kv4_k_at(g, i)..+7
//   V  lane c = 0..15 holds two values a token and byte j of NB, of four tokens: the pair (even, odd) kv4_v_at(c, j)
// With one, two or four blocks a lane's values are neighbours and lie in one block; three blocks don't divide by 4 and 16 lanes,
// so that there chunk i and byte j are a lane's share of block i, j.
// ---------------------------------------------------------------------------
template <int NB> __host__ __device__ constexpr int kv4_k_at(int g, int i) { return NB == 3 ? 32 * i + 8 * g : 8 * NB * g + 8 * i; }
template <int NB> __host__ __device__ constexpr int kv4_v_at(int c, int j) { return NB == 3 ? 32 * j + 2 * c : 2 * (NB * c + j); }

struct Kv4 {
    char *at;
    int64_t pages;
    int shift, kv_heads, d; // page = 1 << shift
};

// one head's part of a page
__device__ __forceinline__ char *kv4_part(const Kv4 &c, int64_t page, int head, int nb)
{
    return c.at + ((page * c.kv_heads + head) * (34 * (int64_t)nb) << c.shift);
}

// A value's scale is the exponent field of a float, which is the scale byte itself (0: 2^-127, 255: NaN).
__device__ __forceinline__ float kv4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

struct Kv4Io {
    Kv4 c;
    const int64_t *slots;
    void *k, *v;
    int64_t k_stride, v_stride;
    int rows;
    int64_t threads; // rows in fours x kv_heads x 2 x 16 NB
};

// Where thread `id` of a conversion works: four threads a block of 32, eight values each.  Four rows of one head's keys, then of its
// values, lie next to each other, because four tokens of V share their bytes' lines and should meet in one wavefront.
template <int NB> struct Kv4Unit {
    int64_t slot;
    int row, head, col; // col: first value of eight
    bool is_v;
    __device__ __forceinline__ Kv4Unit(const Kv4Io &a, int64_t id)
    {
        const uint32_t part = (uint32_t)(id / (16 * NB)), in = (uint32_t)(id - (int64_t)part * (16 * NB)); // four rows of a head's keys or values
        const uint32_t heads = part >> 1, rows = heads / (uint32_t)a.c.kv_heads;
        is_v = part & 1;
        head = (int)(heads - rows * (uint32_t)a.c.kv_heads);
        row = (int)(4 * rows + in / (4 * NB));
        col = (int)(in % (4 * NB)) * 8;
        slot = row < a.rows ? a.slots[row] : -1;
        if (slot >> a.c.shift >= a.c.pages) slot = -1;
    }
};

// Bytes of a unit's codes: four bytes in a row for K, and for V of four blocks; else pieces `step` bytes apart.
template <int NB> __device__ __forceinline__ char *kv4_codes(const Kv4Io &a, const Kv4Unit<NB> &u, char *part, int tok)
{
    const int b = u.col >> 5, g = u.col >> 3 & 3;
    if (!u.is_v) return part + (int64_t)tok * (16 * NB) + (NB == 3 ? 12 * g + 4 * b : u.col >> 1);
    char *v = part + ((int64_t)(16 * NB) << a.c.shift) + (int64_t)(tok >> 2) * (64 * NB) + (tok & 3) * NB;
    const int p = u.col >> 1; // the first pair; pair p lies in byte j of lane c
    return NB == 3 ? v + 12 * (4 * g) + b : v + (p / NB) * (4 * NB) + p % NB;
}
template <int NB> __device__ __forceinline__ char *kv4_scales(const Kv4Io &a, const Kv4Unit<NB> &u, char *part, int tok)
{
    char *s = part + ((int64_t)(32 * NB) << a.c.shift);
    const int b = u.col >> 5;
    return u.is_v ? s + ((int64_t)NB << a.c.shift) + (tok >> 2) * (4 * NB) + 4 * b + (tok & 3) : s + (int64_t)tok * NB + b;
}
// offset of byte p = 0..3 of a unit of V
template <int NB> __device__ constexpr int kv4_v_byte(int p) { return NB == 3 ? 12 * p : (p / NB) * (4 * NB) + p % NB; }

// scale = 2^(exponent of the absmax - 2), codes = values / scale rounded once by the conversion instruction: exact but for that.
// Bound by memory: 8192 tokens of 8 heads of 128 in bf16, 34 MB in and 9 out, 11 to 13 us (3.3 to 3.9 TB/s); 48 tokens a launch's time, 3.2 us.
// With one token a wavefront, whose bytes of V lie in other wavefronts' lines, in and out took 26 us and now take 21.
template <typename T, int NB, bool VEC>
__global__ __launch_bounds__(256) void k_kv4_write(const Kv4Io a)
{
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= a.threads) return; // whole groups of four lanes leave, here and below: the exchanges stay within four
    const Kv4Unit<NB> u(a, id);
    if (u.slot < 0) return;
    const T *src = static_cast<const T *>(u.is_v ? a.v : a.k) + (int64_t)u.row * (u.is_v ? a.v_stride : a.k_stride) + (int64_t)u.head * a.c.d + u.col;
    float v[8];
    if (u.col >= a.c.d) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.f;
    } else if constexpr (!VEC) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)src[e];
    } else if constexpr (sizeof(T) == 2) {
        const bf16x8 r = *reinterpret_cast<const bf16x8 *>(src);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)r[e];
    } else {
        const f32x4 r0 = *reinterpret_cast<const f32x4 *>(src), r1 = *reinterpret_cast<const f32x4 *>(src + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = r0[e], v[4 + e] = r1[e];
    }
    uint32_t top = 0; // bits of the absmax, which order as values do, infinities and NaN among them
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
    const uint32_t ex = top >> 23; // floor(log2) + 127; 0 for what is below 2^-126, whose scale is the least anyhow
    const bool none = ex == 255;
    const uint32_t byte = none ? 255u : ex > 2 ? ex - 2 : 0u;
    uint32_t w = 0;
    if (!none) {
        const float s = kv4_scale(byte);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], s, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], s, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], s, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], s, 3);
    }
    const int tok = (int)(u.slot & ((1 << a.c.shift) - 1));
    char *part = kv4_part(a.c, u.slot >> a.c.shift, u.head, NB), *to = kv4_codes<NB>(a, u, part, tok);
    if (!u.is_v || NB == 4) *reinterpret_cast<uint32_t *>(to) = w;
    else if (NB == 2) {
        *reinterpret_cast<uint16_t *>(to) = (uint16_t)w;
        *reinterpret_cast<uint16_t *>(to + kv4_v_byte<NB>(2)) = (uint16_t)(w >> 16);
    } else {
#pragma unroll
        for (int p = 0; p < 4; ++p) to[kv4_v_byte<NB>(p)] = (char)(w >> 8 * p);
    }
    if ((id & 3) == 0) *kv4_scales<NB>(a, u, part, tok) = (char)byte;
}

// value = code scale, exact.  Bound by memory: 8192 tokens of 8 heads of 128, 9 MB in and 34 out, 9 to 10 us.
template <typename T, int NB, bool VEC>
__global__ __launch_bounds__(256) void k_kv4_read(const Kv4Io a)
{
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= a.threads) return;
    const Kv4Unit<NB> u(a, id);
    if (u.slot < 0 || u.col >= a.c.d) return;
    const int tok = (int)(u.slot & ((1 << a.c.shift) - 1));
    char *part = kv4_part(a.c, u.slot >> a.c.shift, u.head, NB), *from = kv4_codes<NB>(a, u, part, tok);
    uint32_t w = 0;
    if (!u.is_v || NB == 4) w = *reinterpret_cast<const uint32_t *>(from);
    else if (NB == 2) w = *reinterpret_cast<const uint16_t *>(from) | (uint32_t)*reinterpret_cast<const uint16_t *>(from + kv4_v_byte<NB>(2)) << 16;
    else {
#pragma unroll
        for (int p = 0; p < 4; ++p) w |= (uint32_t)(uint8_t)from[kv4_v_byte<NB>(p)] << 8 * p;
    }
    const float s = kv4_scale((uint8_t)*kv4_scales<NB>(a, u, part, tok));
    const bf16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1);
    const bf16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3);
    const bf16x8 r{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
    T *dst = static_cast<T *>(u.is_v ? a.v : a.k) + (int64_t)u.row * (u.is_v ? a.v_stride : a.k_stride) + (int64_t)u.head * a.c.d + u.col;
    if constexpr (!VEC) {
#pragma unroll
        for (int e = 0; e < 8; ++e) dst[e] = (T)r[e];
    } else if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<bf16x8 *>(dst) = r;
    } else {
        *reinterpret_cast<f32x4 *>(dst) = f32x4{(float)r[0], (float)r[1], (float)r[2], (float)r[3]};
        *reinterpret_cast<f32x4 *>(dst + 4) = f32x4{(float)r[4], (float)r[5], (float)r[6], (float)r[7]};
    }
}

// ---------------------------------------------------------------------------
// attention over the cache
// ---------------------------------------------------------------------------
struct Kv4Attend {
    Kv4 c;
    int heads, group, tiles; // query heads, of a key and value head, tiles of 16 of those
    float c2;                // scale log2(e)
    const int32_t *table, *lens;
    int table_len, splits, batch;
    int coarse; // sequences start in the order of lens >> coarse, -1: in their own
    int64_t table_stride;
    const bf16_t *q;
    int64_t q_stride;
    bf16_t *o;
    int64_t o_stride;
    float *part;  // [batch][heads][splits][32 NB]: unscaled o of the splits
    float2 *stat; // [batch][heads][splits]: largest score (-infinity: no tokens), sum
};

constexpr int kKvStep = 32;               // tokens of a wavefront's step
// Tokens that one workgroup of 16 wavefronts goes through instead of several of four.  One launch against two; us, with at most 512 / 1024 / 2048:
// 700 tokens of 32 heads of 128 11.6 / 8.9 / 9.1, 4 x 900..1000 of 32/8 12.0 / 9.3 / 9.1, 8 x 900..1000 of 32 14.5 / 10.9 / 10.9, 8 x 500..1500 of
// 32/8 11.9 / 11.8 / 10.8, 2000 tokens of 32 11.7 / 11.4 / 12.7.
constexpr int kKvShort = 1024;
// Tokens that are worth a workgroup of their own, us with 128 / 256 / 512: 8 x 1..4096 tokens of 32/8 heads of 128 13.3 / 14.6 / 14.1, 16 x
// 1..4096 15.3 / 16.4 / 18.9, 30000 of one sequence 17.1 / 17.4 / 16.9.
constexpr int kKvLeast = 128;
// Workgroups wanted: the card once, four a compute unit.  With 768 / 1024 / 1536 / 2048 of them, us, caches that take turns: 4 x 60001..65536 tokens
// of 32/8 heads of 128 57.6 / 59.4 / 64.3 / 63.1, 64 x 1..4096 40.1 / 40.0 / 41.4 / 41.6, 32 x 1..4096 23.3 / 22.9 / 24.9 / 26.0, 32 x
// 1000..3000 of 16 heads of 64 22.3 / 22.1 / 23.6 / 24.1, but 4 x 1..65536 41.7 / 35.3 / 34.0 / 36.8, 16 x 1..32768 75.3 / 69.3 / 70.4 / 69.6.
constexpr int kKvTarget = 1024;
constexpr int kKvSplits = 128;            // of a sequence, at most

// tokens of a split of a sequence of len tokens, and how many splits have any
__host__ __device__ inline int kv4_per_split(int len, int splits)
{
    const int per = (int)(((int64_t)len + splits - 1) / splits + 127) / 128 * 128;
    return per > kKvLeast ? per : kKvLeast;
}
__host__ __device__ inline int kv4_tokens(int len, int table_len, int shift)
{
    const int64_t most = (int64_t)table_len << shift;
    return len < 0 ? 0 : len > most ? (int)most : len;
}

__device__ __forceinline__ uint32_t pair_lo(bf16x2 a, bf16x2 b) { return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x05040100u); }
__device__ __forceinline__ uint32_t pair_hi(bf16x2 a, bf16x2 b) { return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x07060302u); }

// byte `at` of a lane's codes of V, as the bf16 pair (even value, odd value)
template <int AT> __device__ __forceinline__ bf16x2 v_pair(const uint32_t *w, float s) { return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[AT / 4], s, AT % 4); }

// What a lane holds of a step's 32 tokens: two tiles of 16 tokens of K, two groups of four tokens of V.  Where a page has 16 tokens or
// more (WIDE), a tile lies in one page, whose place is the same for all lanes: its entry in the table comes through scalars, and a lane's
// places are constant distances from there (32 x 1000..3000 tokens of 16 heads of 64, pages of 16: 30 us by lanes, 26 so).  Else a lane looks up
// the pages of its tokens.  Entries are fetched a step before the codes, so that a
// step waits for one trip to memory and not for two.
template <int NB, bool WIDE> struct Kv4Step {
    static constexpr int S = NB == 3 ? 3 : 1;
    uint32_t k[2][NB], v[2][NB], ks[2][S], vs[2][S];
    bool ok[2]; // the lane's group of V's tokens, which are the tokens of its scores, is there

    // the lane's part of the tables: pages of its two tokens of K, of its two groups of V
    struct Pages {
        int k[2], v[WIDE ? 1 : 2]; // (WIDE: a tile's keys and values are in one page)
        __device__ __forceinline__ void look(const Kv4Attend &a, const int32_t *table, int t0, int end, int lane)
        {
            if constexpr (WIDE) {
#pragma unroll
                for (int x = 0; x < 2; ++x) k[x] = t0 + 16 * x < end ? table[(t0 + 16 * x) >> a.c.shift] : -1;
            } else {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int tk = t0 + 16 * x + (lane & 15), tv = t0 + 16 * x + 4 * (lane >> 4);
                    k[x] = tk < end ? table[tk >> a.c.shift] : -1;
                    v[x] = tv < end ? table[tv >> a.c.shift] : -1;
                }
            }
        }
    };
    // codes and scales of a token of K at w and sc, of four tokens of V at w and sc
    __device__ __forceinline__ void load_k(int x, const char *w, const char *sc, int g)
    {
        __builtin_memcpy(k[x], __builtin_assume_aligned(w, NB == 3 ? 4 : 4 * NB), 4 * NB);
#pragma unroll
        for (int j = 0; j < S; ++j) ks[x][j] = (uint8_t)sc[NB == 3 ? j : g * NB / 4];
    }
    __device__ __forceinline__ void load_v(int x, const char *w, const char *sc, int r)
    {
        __builtin_memcpy(v[x], __builtin_assume_aligned(w, NB == 3 ? 4 : 4 * NB), 4 * NB);
#pragma unroll
        for (int j = 0; j < S; ++j) vs[x][j] = reinterpret_cast<const uint32_t *>(sc)[NB == 3 ? j : r * NB / 16];
    }
    __device__ __forceinline__ void load(const Kv4Attend &a, const Pages &p, int head, int t0, int end, int lane)
    {
        const int r = lane & 15, g = lane >> 4, sh = a.c.shift, in = (1 << sh) - 1;
        const int64_t codes = (int64_t)(16 * NB) << sh;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            ok[x] = false;
#pragma unroll
            for (int j = 0; j < NB; ++j) k[x][j] = v[x][j] = 0;
#pragma unroll
            for (int j = 0; j < S; ++j) ks[x][j] = vs[x][j] = 0;
        }
        if constexpr (WIDE) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int page = __builtin_amdgcn_readfirstlane(p.k[x]), tok = t0 + 16 * x & in;
                if (page < 0 || page >= a.c.pages) continue;
                // (a page has places for all of the tile's tokens, also past the sequence's end)
                const char *at = kv4_part(a.c, page, head, NB), *kc = at + tok * (16 * NB), *kx = at + 2 * codes + tok * NB;
                load_k(x, kc + r * (16 * NB) + 4 * NB * g, kx + r * NB, g);
                load_v(x, kc + codes + g * (64 * NB) + r * (4 * NB), kx + ((int64_t)NB << sh) + g * (4 * NB), r);
                ok[x] = true;
            }
        } else {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int tk = t0 + 16 * x + r & in, tv = t0 + 16 * x + 4 * g & in;
                if (p.k[x] >= 0 && p.k[x] < a.c.pages) {
                    const char *at = kv4_part(a.c, p.k[x], head, NB);
                    load_k(x, at + tk * (16 * NB) + 4 * NB * g, at + 2 * codes + tk * NB, g);
                }
                if (p.v[x] >= 0 && p.v[x] < a.c.pages) {
                    const char *at = kv4_part(a.c, p.v[x], head, NB);
                    load_v(x, at + codes + (tv >> 2) * (64 * NB) + r * (4 * NB), at + 2 * codes + ((int64_t)NB << sh) + (tv >> 2) * (4 * NB), r);
                    ok[x] = true;
                }
            }
        }
    }
};

// The j-th sequence to be started, and its tokens.  Workgroups start in the order of their numbers; where the longest may take several times as
// long as others (kv4_coarse), of every 64 neighbouring sequences those with most tokens come first, in steps of 2^coarse tokens.
struct Kv4Seq {
    int b, len;
};
__device__ __forceinline__ Kv4Seq kv4_seq(const Kv4Attend &a, int j)
{
    if (a.coarse < 0) return Kv4Seq{j, kv4_tokens(a.lens[j], a.table_len, a.c.shift)};
    const int lane = threadIdx.x & 63, b0 = j & ~63;
    const int len = b0 + lane < a.batch ? kv4_tokens(a.lens[b0 + lane], a.table_len, a.c.shift) : -1, n = len >> a.coarse;
    j &= 63;
    int x = 0, longer = 0; // the n of the one looked for is the largest x with more than j of n >= x
#pragma unroll
    for (int bit = 8; bit; bit /= 2) {
        const int c = __builtin_popcountll(__ballot(n >= x + bit));
        longer = c > j ? longer : c;
        x = c > j ? x + bit : x;
    }
    const uint64_t there = __ballot(n == x);
    const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(there >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)there, 0));
    const int at = __builtin_ctzll(__ballot(n == x && before == j - longer));
    return Kv4Seq{b0 + at, __builtin_amdgcn_readlane(len, at)};
}

// What parts' largest scores are taken relative to: the largest of them, or anything where none has a token (all are -infinity and weigh 0)
__device__ __forceinline__ float kv4_finite(float most) { return most == -INFINITY ? 0.f : most; }

// One (sequence, tile of 16 query heads of a key and value head, split) a workgroup.  Scores are computed turned round, tokens by heads:
// S^T = K q^T, so that a lane has one head's scores of 8 tokens (its column of the result) and these are, in place, the operand of
// o^T = V^T p^T, whose columns are heads again: maxima, sums and rescaling stay inside a lane or go over the four lanes of a head.
// The wavefronts take steps of 32 tokens in turn, a step's loads ahead.
// Bound by memory: 4 x 60001..65536 tokens of 32/8 heads of 128, 273 MB, 47 us where the cache was just read (5.8 TB/s), 59 for the whole call over
// caches that take turns; 64 x 1..4096 tokens, 150 MB, 33 to 34 us in one launch, the call 37 to 39.  700 tokens of 32 heads 7.5 us, a launch and three trips to memory.
// (Without page entries a step ahead, and pages looked up by every lane, 4 x 65536 tokens took 125 us; two steps of codes ahead were slower.)
template <int NB, bool WIDE, int WAVES>
__global__ __launch_bounds__(64 * WAVES, WAVES == 4 ? 3 : 4) void k_kv4_attend(const Kv4Attend a)
{
    constexpr int DP = 32 * NB, STRIDE = WAVES * kKvStep, PITCH = DP + 4;
    extern __shared__ float join[]; // [WAVES][heads of a tile][PITCH]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    int id = blockIdx.x;
    const int split = id % a.splits;
    id /= a.splits;
    const int tile = id % a.tiles;
    id /= a.tiles;
    const int hk = id % a.c.kv_heads;
    const Kv4Seq seq = kv4_seq(a, id / a.c.kv_heads);
    const int b = seq.b, len = seq.len, per = WAVES == 16 ? len : kv4_per_split(len, a.splits);
    const int begin = (int64_t)split * per < len ? split * per : len, end = len - begin < per ? len : begin + per;
    if (split > 0 && begin >= end) return;
    const int32_t *table = a.table + b * a.table_stride;
    const int head0 = hk * a.group + tile * 16, mine = min(16, a.group - tile * 16);

    Kv4Step<NB, WIDE> st;
    typename Kv4Step<NB, WIDE>::Pages pages;
    int t0 = begin + wave * kKvStep;
    pages.look(a, table, t0, end, lane);
    bf16x8 q[NB];
    const bf16_t *qr = a.q + b * a.q_stride + (int64_t)(head0 + r) * a.c.d;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        const int at = kv4_k_at<NB>(g, i);
        q[i] = bf16x8{};
        if (r < mine && at < a.c.d) q[i] = *reinterpret_cast<const bf16x8 *>(qr + at);
    }
    f32x4 acc[2 * NB];
#pragma unroll
    for (int n = 0; n < 2 * NB; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
    float top = -FLT_MAX, sum = 0.f; // scores are taken relative to `top`, which stays within 2^8 of the largest so far
    bool some = false;               // has this wavefront met a token?

    if (t0 < end) st.load(a, pages, hk, t0, end, lane);
    pages.look(a, table, t0 + STRIDE, end, lane);
    for (; t0 < end; t0 += STRIDE) {
        Kv4Step<NB, WIDE> now = st;
        if (t0 + STRIDE < end) {
            st.load(a, pages, hk, t0 + STRIDE, end, lane);
            pages.look(a, table, t0 + 2 * STRIDE, end, lane);
        }
        f32x4 s[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            s[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const float sc = kv4_scale(now.ks[x][NB == 3 ? i : 0]);
                const bf16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(now.k[x][i], sc, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(now.k[x][i], sc, 1);
                const bf16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(now.k[x][i], sc, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(now.k[x][i], sc, 3);
                const bf16x8 kf{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
                s[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[i], s[x], 0, 0, 0);
            }
        }
        // tokens that are not there, past the end or in a page outside the cache
        const bool whole = t0 + kKvStep <= end && __all(now.ok[0] && now.ok[1]);
        const int keep = end - t0 - 4 * g;
        some = some || whole || __any((now.ok[0] && keep > 0) || (now.ok[1] && keep > 16));
        if (!whole) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
#pragma unroll
                for (int i = 0; i < 4; ++i) s[x][i] = now.ok[x] && 16 * x + i < keep ? s[x][i] : -INFINITY;
                // V's may hold anything, no value among them: their scales become the least one
                if (keep - 16 * x < 4) {
                    const uint32_t mask = keep - 16 * x <= 0 ? 0u : (1u << 8 * (keep - 16 * x)) - 1u;
#pragma unroll
                    for (int j = 0; j < (NB == 3 ? 3 : 1); ++j) now.vs[x][j] &= mask;
                }
            }
        }
        float most = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3]));
        most = fmaxf(most, fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3]))) * a.c2;
        if (__any(most > top + 8.f)) {
            most = fmaxf(most, __shfl_xor(most, 16, 64));
            most = fmaxf(most, __shfl_xor(most, 32, 64));
            const float next = most > top + 8.f ? most : top, by = __builtin_amdgcn_exp2f(top - next);
            top = next;
            sum *= by;
#pragma unroll
            for (int n = 0; n < 2 * NB; ++n) acc[n] *= by;
        }
        bf16x8 p;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = __builtin_amdgcn_exp2f(fmaf(s[x][i], a.c2, -top));
                sum += e;
                p[4 * x + i] = (bf16_t)e;
            }
#define PAC_KV4_PAIR(X, T, J) v_pair<(T) * NB + (J)>(now.v[X], kv4_scale(now.vs[X][NB == 3 ? (J) : 0] >> 8 * (T) & 255u))
#define PAC_KV4_BYTE(J)                                                                                                           \
    if constexpr ((J) < NB) {                                                                                                     \
        const bf16x2 a0 = PAC_KV4_PAIR(0, 0, J), a1 = PAC_KV4_PAIR(0, 1, J), a2 = PAC_KV4_PAIR(0, 2, J), a3 = PAC_KV4_PAIR(0, 3, J); \
        const bf16x2 b0 = PAC_KV4_PAIR(1, 0, J), b1 = PAC_KV4_PAIR(1, 1, J), b2 = PAC_KV4_PAIR(1, 2, J), b3 = PAC_KV4_PAIR(1, 3, J); \
        const u32x4 lo{pair_lo(a0, a1), pair_lo(a2, a3), pair_lo(b0, b1), pair_lo(b2, b3)};                                       \
        const u32x4 hi{pair_hi(a0, a1), pair_hi(a2, a3), pair_hi(b0, b1), pair_hi(b2, b3)};                                       \
        acc[2 * (J)] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, lo), p, acc[2 * (J)], 0, 0, 0);         \
        acc[2 * (J) + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, hi), p, acc[2 * (J) + 1], 0, 0, 0); \
    }
        PAC_KV4_BYTE(0)
        PAC_KV4_BYTE(1)
        PAC_KV4_BYTE(2)
        PAC_KV4_BYTE(3)
#undef PAC_KV4_BYTE
#undef PAC_KV4_PAIR
    }
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);

    // the wavefronts' results, each relative to its own `top`; -infinity says that there were no tokens, which a sum of 0 does not: the scores of all
    // of them may be -infinity, and o is no number then
    const int heads = min(16, a.group);
    auto joined = [&](int w, int h) { return join + (w * heads + h) * PITCH; };
    float *row = joined(wave, r);
    if (r < mine) {
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = kv4_v_at<NB>(4 * g + i, j);
                row[at] = acc[2 * j][i];
                row[at + 1] = acc[2 * j + 1][i];
            }
        if (g == 0) {
            row[DP] = some ? top : -INFINITY;
            row[DP + 1] = sum;
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < mine * DP; e += 64 * WAVES) {
        const int h = e / DP, at = e % DP;
        float most = joined(0, h)[DP], l = 0.f, v = 0.f;
#pragma unroll
        for (int w = 1; w < WAVES; ++w) most = fmaxf(most, joined(w, h)[DP]);
        const float from = kv4_finite(most);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float by = __builtin_amdgcn_exp2f(joined(w, h)[DP] - from);
            l += by * joined(w, h)[DP + 1];
            v += by * joined(w, h)[at];
        }
        if (len <= per) { // the whole sequence was this workgroup's
            if (at < a.c.d) a.o[b * a.o_stride + (int64_t)(head0 + h) * a.c.d + at] = (bf16_t)(most == -INFINITY ? 0.f : v / l);
        } else {
            const int64_t to = ((int64_t)b * a.heads + head0 + h) * a.splits + split;
            a.part[to * DP + at] = v;
            if (at == 0) a.stat[to] = float2{most, l};
        }
    }
}

// The splits of a sequence's head (at most kKvSplits), each weighed by 2^(its largest score - the largest): 4.7 to 5.4 us, a launch and two trips to
// memory.  A thread adds up four values of every SETS-th split, then the sets are added in order.
template <int NB>
__global__ __launch_bounds__(256) void k_kv4_join(const Kv4Attend a)
{
    constexpr int DP = 32 * NB, QUADS = DP / 4, SETS = 256 / QUADS;
    __shared__ float by[kKvSplits], parts[4];
    __shared__ f32x4 sums[SETS][QUADS];
    const int b = blockIdx.x / a.heads, h = blockIdx.x % a.heads, tid = threadIdx.x;
    const int len = kv4_tokens(a.lens[b], a.table_len, a.c.shift), per = kv4_per_split(len, a.splits);
    if (len <= per) return;
    const int n = (int)(((int64_t)len + per - 1) / per);
    const float2 *stat = a.stat + ((int64_t)b * a.heads + h) * a.splits;
    const f32x4 *part = reinterpret_cast<const f32x4 *>(a.part + ((int64_t)b * a.heads + h) * a.splits * DP);
    // weights: every wavefront finds the largest score of all splits for itself
    const int lane = tid & 63;
    float most = -INFINITY;
    for (int s = lane; s < n; s += 64) most = fmaxf(most, stat[s].x);
#pragma unroll
    for (int x = 1; x < 64; x *= 2) most = fmaxf(most, __shfl_xor(most, x, 64));
    float l = 0.f;
    if (tid < n) {
        by[tid] = __builtin_amdgcn_exp2f(stat[tid].x - kv4_finite(most));
        l = by[tid] * stat[tid].y;
    }
#pragma unroll
    for (int x = 1; x < 64; x *= 2) l += __shfl_xor(l, x, 64);
    if (lane == 0) parts[tid >> 6] = l;
    __syncthreads();
    l = (parts[0] + parts[1]) + (parts[2] + parts[3]);
    const int set = tid / QUADS, at = tid % QUADS;
    if (set < SETS) {
        f32x4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
        for (int s = set; s < n; s += SETS) v += by[s] * part[(int64_t)s * QUADS + at];
        sums[set][at] = v;
    }
    __syncthreads();
    if (tid >= a.c.d) return;
    float v = 0.f;
#pragma unroll
    for (int x = 0; x < SETS; ++x) v += sums[x][tid / 4][tid % 4];
    a.o[b * a.o_stride + (int64_t)h * a.c.d + tid] = (bf16_t)(most == -INFINITY ? 0.f : v / l);
}
static_assert(kKvSplits <= 256, "a thread a split");

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
static int kv4_blocks(const pac_kv4 *c) { return (c->d + 31) / 32; }
static pac_status check_kv4(const pac_kv4 *c)
{
    if (!c) return PAC_ERR_NULL;
    if (c->pages < 0 || c->pages > INT32_MAX || c->page < 8 || c->page > 65536 || (c->page & (c->page - 1)) || c->kv_heads < 1 ||
        c->kv_heads > 4096 || c->d < 8 || c->d > 128 || c->d % 8)
        return PAC_ERR_SHAPE;
    // its bytes have to be a number
    return c->pages * c->page > ((int64_t)1 << 62) / (c->kv_heads * 34 * kv4_blocks(c)) ? PAC_ERR_SHAPE : PAC_OK;
}
static int64_t kv4_bytes(const pac_kv4 *c) { return c->pages * c->page * c->kv_heads * 34 * kv4_blocks(c); }
static Kv4 kv4_of(const pac_kv4 *c)
{
    int shift = 0;
    while (1 << shift < c->page) ++shift;
    return Kv4{static_cast<char *>(c->at), c->pages, shift, c->kv_heads, c->d};
}

// Splits of the long axis: workgroups for four a compute unit, none of fewer than kKvLeast tokens.  Two cases take one workgroup of 16 wavefronts for every
// sequence and head instead (0 splits), which saves the second launch: short sequences that leave most of the card idle (kKvShort), and as many
// sequences by heads as come to two or three such workgroups a compute unit, the longest first, which else would be two splits each.  The latter,
// us, splits / 16 wavefronts, 32/8 heads of 128: 64 x 1..4096 tokens 40.6 / 38.6, 64 x 1..1000 19.3 / 15.8, 64 x 1500 30.2 / 28.8, 64 x
// 3500..4096 59.5 / 57.7, 100 x 1..16000 174 / 173; but with more workgroups, which have one split each, 256 x 1..4096 121.9 / 130.3, 40 x 1..4096 of 32
// heads 69.8 / 78.9.
static int kv4_splits(const pac_kv4 *c, int heads, int batch, int table_len)
{
    const int64_t base = (int64_t)batch * c->kv_heads * ((heads / c->kv_heads + 15) / 16), most = (int64_t)table_len * c->page;
    const int64_t want = (kKvTarget + base - 1) / base, fit = (most + kKvLeast - 1) / kKvLeast;
    if (fit > 1 && ((most <= kKvShort && base <= 256) || (base >= kKvTarget / 2 && base < kKvTarget))) return 0;
    const int64_t s = want < fit ? want : fit;
    return (int)(s < 1 ? 1 : s > kKvSplits ? kKvSplits : s);
}
// In which steps of 2^.. tokens, at most 16 of them, sequences are sorted by their lengths (-1: not at all).  Worth the look at 64 lengths where a
// workgroup may have many tokens and the card is filled a few times at most; us, in order / sorted, 32/8 heads of 128 over caches that take turns:
// 32 x 1..4096 tokens (1024 a workgroup at most) 26.3 / 23.2, 4 x 1..65536 (2048) 38.6 / 35.5, 16 x 1..32768
// (4096) 79.2 / 69.5, 256 x 1..4096 (4096) 127.7 / 121.7, of 32 heads without sharing 40 x 1..4096 84.3 / 69.2; lengths alike 59.2 / 59.4 (4 x
// 60001..65536); but 16 x 1..4096 (512) 18.6 / 19.8, and where workgroups are many anyhow, 200 x 1..2048 of 32 heads
// of 64, 110.1 / 114.3.
static int kv4_coarse(int batch, int64_t base, int64_t most, int splits)
{
    if (batch < 2 || base > 4096 || (splits ? most <= 512 * (int64_t)splits : base <= 256)) return -1;
    int c = 0;
    while (most >> c > 15) ++c;
    return c;
}
static pac_status check_attend(const pac_kv4 *c, int32_t heads, int32_t batch, int32_t table_len)
{
    const pac_status s = check_kv4(c);
    if (s != PAC_OK) return s;
    if (heads < 1 || heads > 4096 || heads % c->kv_heads || batch < 0 || table_len < 0) return PAC_ERR_SHAPE;
    // (the kernel's token numbers run up to two of its steps past a sequence's end)
    if ((int64_t)table_len * c->page > INT32_MAX - 4096 || (int64_t)batch * c->kv_heads * ((heads / c->kv_heads + 15) / 16) >= 1 << 23 ||
        (int64_t)batch * heads >= 1 << 23)
        return PAC_ERR_UNSUPPORTED;
    return PAC_OK;
}
static int64_t attend_bytes(const pac_kv4 *c, int32_t heads, int32_t batch, int splits)
{
    return splits < 2 ? 0 : (int64_t)batch * heads * splits * (2 + 32 * kv4_blocks(c)) * 4;
}

template <typename F> static void by_blocks(int nb, const F &f)
{
    if (nb == 1) f(std::integral_constant<int, 1>());
    else if (nb == 2) f(std::integral_constant<int, 2>());
    else if (nb == 3) f(std::integral_constant<int, 3>());
    else f(std::integral_constant<int, 4>());
}

static pac_status kv4_convert(const pac_kv4 *c, int64_t rows, const int64_t *slots, void *k, int64_t k_stride, void *v, int64_t v_stride,
                              int32_t dtype, bool read, void *hip_stream)
{
    const pac_status s = check_kv4(c);
    if (s != PAC_OK) return s;
    if (dtype != PAC_BF16 && dtype != PAC_F32) return PAC_ERR_SHAPE;
    const int64_t cols = (int64_t)c->kv_heads * c->d, size = dtype == PAC_F32 ? 4 : 2;
    if (rows < 0 || k_stride < cols || v_stride < cols) return PAC_ERR_RANGE;
    if (rows == 0) return PAC_OK;
    if (!slots || !k || !v || (c->pages && !c->at)) return PAC_ERR_NULL;
    if (!kv_aligned(c->at, 16) || !kv_aligned(slots, 8) || !kv_aligned(k, size) || !kv_aligned(v, size)) return PAC_ERR_ALIGN;
    if (rows * c->kv_heads < rows || rows * (int64_t)c->kv_heads > INT32_MAX) return PAC_ERR_UNSUPPORTED;
    const Span cache(c->at, c->pages ? kv4_bytes(c) : 0), ks(k, rows, k_stride * size, cols * size), vs(v, rows, v_stride * size, cols * size), sl(slots, rows * 8);
    if (shares(cache, {ks, vs, sl}) || (read && (shares(ks, {vs, sl}) || shares(vs, {sl})))) return PAC_ERR_RANGE;
    if (c->pages == 0) return PAC_OK;
    const int nb = kv4_blocks(c);
    const int64_t threads = (rows + 3) / 4 * c->kv_heads * 2 * 16 * nb, blocks = (threads + 255) / 256;
    if (blocks >= 1 << 24) return PAC_ERR_UNSUPPORTED;
    const Kv4Io a{kv4_of(c), slots, k, v, k_stride, v_stride, (int)rows, threads};
    const bool vec = kv_aligned(k, 16) && kv_aligned(v, 16) && k_stride * size % 16 == 0 && v_stride * size % 16 == 0;
    (void)hipGetLastError();
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    by_blocks(nb, [&](auto n) {
        constexpr int NB = decltype(n)::value;
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, st, a); };
        if (read) {
            if (dtype == PAC_F32) vec ? go(k_kv4_read<float, NB, true>) : go(k_kv4_read<float, NB, false>);
            else vec ? go(k_kv4_read<bf16_t, NB, true>) : go(k_kv4_read<bf16_t, NB, false>);
        } else {
            if (dtype == PAC_F32) vec ? go(k_kv4_write<float, NB, true>) : go(k_kv4_write<float, NB, false>);
            else vec ? go(k_kv4_write<bf16_t, NB, true>) : go(k_kv4_write<bf16_t, NB, false>);
        }
    });
    return hipGetLastError() == hipSuccess ? PAC_OK : PAC_ERR_DEVICE;
}

} // namespace pac

using namespace pac;

extern "C" {

int64_t pac_kv4_bytes(const pac_kv4 *c) { return check_kv4(c) == PAC_OK ? kv4_bytes(c) : -1; }

pac_status pac_kv4_write(const pac_kv4 *c, int64_t rows, const int64_t *slots, const void *k, int64_t k_stride, const void *v,
                         int64_t v_stride, int32_t dtype, void *hip_stream)
{
    return kv4_convert(c, rows, slots, const_cast<void *>(k), k_stride, const_cast<void *>(v), v_stride, dtype, false, hip_stream);
}

pac_status pac_kv4_read(const pac_kv4 *c, int64_t rows, const int64_t *slots, void *k, int64_t k_stride, void *v, int64_t v_stride,
                        int32_t dtype, void *hip_stream)
{
    return kv4_convert(c, rows, slots, k, k_stride, v, v_stride, dtype, true, hip_stream);
}

int64_t pac_kv4_attend_workspace_bytes(const pac_kv4 *c, int32_t heads, int32_t batch, int32_t table_len)
{
    if (check_attend(c, heads, batch, table_len) != PAC_OK) return -1;
    // splits grow as the batch shrinks: room for the most partial results that a batch of at most this size makes
    const int64_t base = (int64_t)c->kv_heads * ((heads / c->kv_heads + 15) / 16);
    const int64_t fit = ((int64_t)table_len * c->page + kKvLeast - 1) / kKvLeast;
    int64_t pairs = (kKvTarget + 2 * base) / base + batch; // (sequence, split) pairs: want x batch <= kKvTarget / base + batch
    if (pairs > fit * batch) pairs = fit * batch;
    if (pairs > kKvSplits * (int64_t)batch) pairs = kKvSplits * (int64_t)batch;
    return pairs * heads * (2 + 32 * kv4_blocks(c)) * 4;
}

int64_t pac_kv4_attend_bytes(const pac_kv4 *c, int32_t heads, int32_t batch, int32_t table_len)
{
    if (check_attend(c, heads, batch, table_len) != PAC_OK) return -1;
    return batch == 0 ? 0 : attend_bytes(c, heads, batch, kv4_splits(c, heads, batch, table_len));
}

pac_status pac_kv4_attend(const pac_kv4 *c, int32_t heads, float scale, int32_t batch, const int32_t *table, int32_t table_len,
                          int64_t table_stride, const int32_t *lens, const void *q, int64_t q_stride, void *o, int64_t o_stride,
                          void *workspace, int64_t workspace_bytes, void *hip_stream)
{
    const pac_status s = check_attend(c, heads, batch, table_len);
    if (s != PAC_OK) return s;
    const int64_t cols = (int64_t)heads * c->d;
    const float c2 = scale * 1.4426950408889634f; // what scores are taken times; infinite, it would make a score of 0 no number
    if (!(scale > 0.f) || !std::isfinite(c2) || q_stride < cols || o_stride < cols || table_stride < table_len) return PAC_ERR_RANGE;
    if (batch == 0) return PAC_OK;
    const int splits = kv4_splits(c, heads, batch, table_len);
    const int64_t need = attend_bytes(c, heads, batch, splits);
    if (!lens || !q || !o || (table_len && !table) || (c->pages && !c->at) || (need && !workspace)) return PAC_ERR_NULL;
    if (!kv_aligned(c->at, 16) || !kv_aligned(table, 4) || !kv_aligned(lens, 4) || !kv_aligned(q, 16) || !kv_aligned(o, 16) ||
        (need && !kv_aligned(workspace, 16)) || q_stride % 8 || o_stride % 8)
        return PAC_ERR_ALIGN;
    if (need && workspace_bytes < need) return PAC_ERR_WORKSPACE;
    const Span cache(c->at, c->pages ? kv4_bytes(c) : 0), qs(q, batch, q_stride * 2, cols * 2), os(o, batch, o_stride * 2, cols * 2);
    const Span ts(table_len ? table : nullptr, batch, table_stride * 4, (int64_t)table_len * 4), ls(lens, (int64_t)batch * 4), ws(need ? workspace : nullptr, need);
    if (shares(os, {cache, qs, ts, ls, ws}) || shares(ws, {cache, qs, ts, ls})) return PAC_ERR_RANGE;
    Kv4Attend a{};
    a.c = kv4_of(c);
    a.heads = heads; a.group = heads / c->kv_heads; a.tiles = (a.group + 15) / 16;
    a.c2 = c2;
    a.table = table; a.lens = lens; a.table_len = table_len; a.splits = splits < 1 ? 1 : splits; a.batch = batch;
    a.coarse = kv4_coarse(batch, (int64_t)batch * c->kv_heads * a.tiles, (int64_t)table_len * c->page, splits);
    a.table_stride = table_stride;
    a.q = static_cast<const bf16_t *>(q); a.q_stride = q_stride;
    a.o = static_cast<bf16_t *>(o); a.o_stride = o_stride;
    a.part = static_cast<float *>(workspace);
    a.stat = reinterpret_cast<float2 *>(a.part + (int64_t)batch * heads * a.splits * 32 * kv4_blocks(c));
    (void)hipGetLastError();
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const unsigned blocks = (unsigned)((int64_t)batch * c->kv_heads * a.tiles * a.splits);
    const int waves = splits ? 4 : 16, lds = waves * (a.group < 16 ? a.group : 16) * (32 * kv4_blocks(c) + 4) * 4;
    bool fits = true;
    by_blocks(kv4_blocks(c), [&](auto n) {
        constexpr int NB = decltype(n)::value;
        auto go = [&](auto kernel) {
            if (lds > 64 << 10) fits = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess;
            if (fits) hipLaunchKernelGGL(kernel, dim3(blocks), dim3(64 * waves), lds, st, a);
        };
        if (splits) c->page >= 16 ? go(k_kv4_attend<NB, true, 4>) : go(k_kv4_attend<NB, false, 4>);
        else c->page >= 16 ? go(k_kv4_attend<NB, true, 16>) : go(k_kv4_attend<NB, false, 16>);
        if (fits && splits > 1) hipLaunchKernelGGL((k_kv4_join<NB>), dim3((unsigned)(batch * heads)), dim3(256), 0, st, a);
    });
    if (!fits) return PAC_ERR_DEVICE;
    return hipGetLastError() == hipSuccess ? PAC_OK : PAC_ERR_DEVICE;
}

} // extern "C"
