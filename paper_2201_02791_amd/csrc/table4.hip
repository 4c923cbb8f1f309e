// Embedding tables of 4-bit numbers, and the scores of questions against every row of one.
//
// A row is cut into groups of 32 elements; a group has a scale s, a bf16 number, and its elements are numbers c of the format
// e2m1 (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives) times s.  s is the smallest bf16 number, 2^-126 or more, with
// 6 s >= the group's largest magnitude, so nothing saturates, and 1.328125 2^125 at most, so that 6 s is a float (elements past bf16's
// largest number become that); 4.5 bits an element in all.
//
// Encoding compares magnitudes with the borders between two numbers, s times 1/4, 3/4, 5/4, 7/4, 5/2, 7/2 and 5: products
// of at most 11 bits, exact in fp32, so that every element goes to the nearest number (of two as near, to the even code).
//
// Both ways are bound by memory: a million rows of 256 floats 219 us encoded, 5.3 TB/s, and 252 us back, 4.6 TB/s.
#include "common.h"
#include "split_bf16.h"

#include <algorithm>

namespace {

constexpr int G = KGE_TABLE4_GROUP;
static_assert(G == 32, "a group is one step of the matrix instruction and 16 bytes of codes");

typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef floatx4 floatx4u __attribute__((aligned(4)));
typedef unsigned uintx2 __attribute__((ext_vector_type(2)));
typedef uintx2 uintx2h __attribute__((aligned(2)));

struct __attribute__((packed, aligned(4))) F4 { float x[4]; };
struct __attribute__((packed, aligned(2))) H4 { uint16_t x[4]; };

__device__ __forceinline__ float bf16_float(uint16_t h) { return __uint_as_float((uint32_t)h << 16); }

// n elements of four from element `at` of X, the others zero
template <bool BF16>
__device__ __forceinline__ void load4(const void *X, int64_t at, int n, float x[4])
{
    if (BF16) {
        const uint16_t *a = (const uint16_t *)X + at;
        if (n >= 4) {
            const H4 q = *reinterpret_cast<const H4 *>(a);
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = bf16_float(q.x[k]);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = k < n ? bf16_float(a[k]) : 0.f;
        }
    } else {
        const float *a = (const float *)X + at;
        if (n >= 4) {
            const F4 q = *reinterpret_cast<const F4 *>(a);
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = q.x[k];
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = k < n ? a[k] : 0.f;
        }
    }
}

// the bits of the smallest bf16 number, 2^-126 or more, six of which reach `most`, or of the largest six of which are a float; NaN where a member is not
// finite
__device__ __forceinline__ uint32_t group_scale(uint32_t most)
{
    if (most == 0u) return 0u;
    if (most >= 0x7f800000u) return 0x7fc00000u;
    const float a = __uint_as_float(most);
    float s = __uint_as_float(max(__float_as_uint(a * (1.f / 6.f)) & 0xffff0000u, 0x00800000u));
#pragma unroll
    for (int k = 0; k < 2; ++k)      // the product is rounded and then cut: at most two steps short
        if (6.f * s < a) s = __uint_as_float(__float_as_uint(s) + 0x10000u);
    return min(__float_as_uint(s), 0x7e2a0000u);
}

__device__ __forceinline__ uint32_t code_of(float x, float s)
{
    const float a = fabsf(x);
    const uint32_t c = (a > 0.25f * s) + (a >= 0.75f * s) + (a > 1.25f * s) + (a >= 1.75f * s) + (a > 2.5f * s) + (a >= 3.5f * s) + (a > 5.f * s);
    return c | (x < 0.f ? 8u : 0u);
}

// The codes of four elements.  The conversion instruction rounds x / s, here formed by a reciprocal and a product that are off by less than 2^-22:
// where quotients that much smaller and larger have the same codes, those are the codes; else the borders decide
__device__ __forceinline__ uint32_t codes_of(const float x[4], float s, float inverse)
{
    float up[4], down[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float q = fmaf(x[k], inverse, 0.f);                // of minus zero plus zero
        up[k] = q * (1.f + 0x1p-22f);
        down[k] = q * (1.f - 0x1p-22f);
    }
    uint32_t a = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, up[0], up[1], 1.f, 0);
    a = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(a, up[2], up[3], 1.f, 1);
    uint32_t b = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, down[0], down[1], 1.f, 0);
    b = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(b, down[2], down[3], 1.f, 1);
    if (a != b) {
        a = 0u;
#pragma unroll
        for (int k = 0; k < 4; ++k) a |= code_of(x[k], s) << (4 * k);
    }
    return a & 0xffffu;
}

// A block takes `BLOCK_GROUPS` groups side by side in the table.  Where one of them is: rows behind the block's first, and the group in its row.
// A row has up to 128 groups, so the quotient of a number below 384 by them is a product and a shift
struct Block {
    int64_t first, row0;           // group, and the row that it is in
    uint32_t into, groups, per, left;     // groups of that row before it; groups that the block has
};
struct Place { uint32_t more; int32_t g; bool in; };
constexpr int BLOCK_GROUPS = 256;
__device__ __forceinline__ Block block_of(int64_t n_rows, int32_t groups)
{
    Block b;
    b.first = (int64_t)blockIdx.x * BLOCK_GROUPS;
    b.row0 = b.first / groups;
    b.into = (uint32_t)(b.first - b.row0 * groups);
    b.groups = (uint32_t)groups;
    b.per = 65536u / (uint32_t)groups + 1u;
    b.left = (uint32_t)min((int64_t)BLOCK_GROUPS, n_rows * groups - b.first);
    return b;
}
__device__ __forceinline__ Place place_of(const Block &b, uint32_t local)
{
    Place p;
    const uint32_t at = b.into + local;
    p.more = at * b.per >> 16;
    p.g = (int32_t)(at - p.more * b.groups);
    p.in = local < b.left;
    return p;
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }
constexpr int NEAR = 0xb1, PAIR = 0x4e;       // quad_perm: lanes 1 apart, 2 apart

// Four lanes to a group: lane i has elements 4 i .. + 3 and 16 + 4 i .. + 3, so that four lanes load 64 bytes side by side.  Their codes are halves
// of words: lanes change halves in pairs, and each has a word.
template <bool BF16>
__global__ __launch_bounds__(256) void k_table4_encode(const void *__restrict__ X, int64_t ldx, int64_t n_rows, int32_t d, int32_t groups,
                                                       uint32_t *__restrict__ codes, uint16_t *__restrict__ scales)
{
    constexpr int SETS = BLOCK_GROUPS / 64;
    const Block b = block_of(n_rows, groups);
    const int64_t from = b.row0 * ldx;
    const uint32_t lane4 = threadIdx.x & 3;
    float x[SETS][8];
#pragma unroll
    for (int i = 0; i < SETS; ++i) {
        const Place p = place_of(b, 64 * i + (threadIdx.x >> 2));
        const int32_t c = p.g * G + 4 * (int32_t)lane4, n = p.in ? d - c : 0;
        const int64_t at = from + (int64_t)p.more * ldx + c;
        load4<BF16>(X, at, n, x[i]);
        load4<BF16>(X, at + 16, n - 16, x[i] + 4);
    }
    codes += b.first * 4;
    scales += b.first;
#pragma unroll
    for (int i = 0; i < SETS; ++i) {
        uint32_t most = 0u;
#pragma unroll
        for (int k = 0; k < 8; ++k) most = max(most, __float_as_uint(x[i][k]) & 0x7fffffffu);
        most = max(most, dpp<NEAR>(most));
        most = max(most, dpp<PAIR>(most));
        const uint32_t bits = group_scale(most);
        const float s = __uint_as_float(bits);
        uint32_t a = 0u, c = 0u;
        if (s > 0.f) {
            const float inverse = __builtin_amdgcn_rcpf(s);
            a = codes_of(x[i], s, inverse);
            c = codes_of(x[i] + 4, s, inverse);
        }
        const bool odd = lane4 & 1u;
        const uint32_t other = dpp<NEAR>(odd ? a : c), local = 64 * i + (threadIdx.x >> 2);
        if (local < b.left) {
            codes[local * 4 + (lane4 & 1u) * 2 + (lane4 >> 1)] = odd ? other | c << 16 : a | other << 16;
            if (lane4 == 0u) scales[local] = (uint16_t)(bits >> 16);
        }
    }
}

// Eight lanes to a group, which store their 4 elements side by side, 1 KB a wavefront, past the caches (a million rows of 256, us: 64 bytes side by
// side 389, 1 KB 304, past the caches 253; 14541 x 200: 7.0, 6.8, 5.4).  ids null: rows in order
template <bool BF16>
__global__ __launch_bounds__(256) void k_table4_decode(const uint16_t *__restrict__ codes, const uint16_t *__restrict__ scales, int64_t n_rows, int32_t d,
                                                       int32_t groups, const int32_t *__restrict__ ids, int64_t n_out, void *__restrict__ out, int64_t ldo)
{
    constexpr int SETS = BLOCK_GROUPS / 32;
    const Block b = block_of(n_out, groups);
    const uint32_t lane8 = threadIdx.x & 7;
    uint32_t w[SETS];
    float s[SETS];
#pragma unroll
    for (int i = 0; i < SETS; ++i) {
        const uint32_t local = 32 * i + (threadIdx.x >> 3);
        w[i] = 0u;
        s[i] = __uint_as_float(0x7fc00000u);                     // a row that the table does not have
        if (local >= b.left) continue;
        if (!ids) {
            w[i] = (codes + b.first * 8)[local * 8 + lane8];
            s[i] = bf16_float((scales + b.first)[local]);
        } else {
            const Place p = place_of(b, local);
            const int64_t src = ids[b.row0 + p.more];
            if (src >= 0 && src < n_rows) {
                w[i] = codes[(src * groups + p.g) * 8 + lane8];
                s[i] = bf16_float(scales[src * groups + p.g]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < SETS; ++i) {
        const Place p = place_of(b, 32 * i + (threadIdx.x >> 3));
        const int32_t c = p.g * G + 4 * (int32_t)lane8;
        const int n = p.in ? d - c : 0;
        if (n <= 0) continue;
        const int64_t at = b.row0 * ldo + (int64_t)p.more * ldo + c;
        const floatx2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], 1.f, 0), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], 1.f, 1);
        const float y[4] = {lo.x * s[i], lo.y * s[i], hi.x * s[i], hi.y * s[i]};
        if (BF16) {
            uint16_t *o = (uint16_t *)out + at;
            H4 q;
#pragma unroll
            for (int k = 0; k < 4; ++k) q.x[k] = __builtin_bit_cast(uint16_t, (__bf16)y[k]);
            if (n >= 4) __builtin_nontemporal_store(__builtin_bit_cast(uintx2, q), reinterpret_cast<uintx2h *>(o));
            else {
#pragma unroll
                for (int k = 0; k < 3; ++k) if (k < n) o[k] = q.x[k];
            }
        } else {
            float *o = (float *)out + at;
            if (n >= 4) __builtin_nontemporal_store(floatx4{y[0], y[1], y[2], y[3]}, reinterpret_cast<floatx4u *>(o));
            else {
#pragma unroll
                for (int k = 0; k < 3; ++k) if (k < n) o[k] = y[k];
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------- scores
//
//   S[q][i] = sum over groups g of s_ig (sum over the group of c_igk x_qk),   x_q = X[fixed_q] * M[rel_q]
//
// The inner sum is one v_mfma_f32_16x16x32_bf16 for 16 rows of the table: its columns are table rows, its rows are questions.
// Codes become bf16 numbers, which hold them exactly, by v_cvt_scalef32_pk_bf16_fp4, two an instruction; a question is the exact
// sum of three bf16 numbers (a bf16 question without M is one).  So no product is rounded; sums are fp32, and the scale
// multiplies a whole group's sum.
//
// A lane loads the 16 bytes of a whole group of its row (four groups of 16 rows a load); four registers by four groups of
// lanes are then transposed by lane swaps, so that each matrix instruction meets one group: the table stays in plain order.
//
// Up to four questions: their parts are rows 4 part + question of one instruction, and the parts' sums are added at the end.
// More: 16 questions a tile, the parts' products chained, smallest first.  A lane's results are one table row's in either case, with the one
// scale: with the operands changed over it would have four rows of one question to store at once, but need four scales, and 16 lanes would
// store to 16 questions' rows (16 questions to a million rows of 256 98 us instead of 51).
//
// Measured, a million rows of 256: one question 31 us, 4.8 TB/s, 369 vector instructions for 32 rows (with addresses formed anew for each load
// 564, and 40 us); 16 questions 47 us; 37 bf16 questions to 2.9 million rows of 128 149 us, 4.3 TB/s, two thirds of it results.

struct Questions {
    const void *X;
    const float *M;
    const int32_t *fixed, *rel;
    int64_t ldx, ldm, n_x, n_m, n;
};

// elements k .. k + 7 of question q, zeros past its end
template <bool BF16>
__device__ __forceinline__ void question8(const Questions &Q, int64_t q, int32_t k, int32_t d, float x[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.f;
    if (q >= Q.n || k >= d) return;
    const int64_t i = Q.fixed ? Q.fixed[q] : q, r = Q.rel ? Q.rel[q] : q;
    const bool bad = i < 0 || i >= Q.n_x || (Q.M && (r < 0 || r >= Q.n_m));
    if (!bad) {
        load4<BF16>(Q.X, i * Q.ldx + k, d - k, x);
        load4<BF16>(Q.X, i * Q.ldx + k + 4, d - k - 4, x + 4);
        if (Q.M) {
            float m[8];
            load4<false>(Q.M, r * Q.ldm + k, d - k, m);
            load4<false>(Q.M, r * Q.ldm + k + 4, d - k - 4, m + 4);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= m[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(0x7fc00000u);
    }
}

// part p of x: what bf16 cuts off x, of the rest what it cuts off, and what is left; their sum is x, but for bits below 2^-133, bf16's last
__device__ __forceinline__ uint32_t part_of(float x, int p)
{
    const uint32_t hi = __float_as_uint(x) & 0xffff0000u;
    if (split_not_finite(x)) return p == 0 ? (x != x ? 0x7fc0u : hi >> 16) : 0u;
    if (p == 0) return hi >> 16;
    const float r = x - __uint_as_float(hi);
    const uint32_t mid = __float_as_uint(r) & 0xffff0000u;
    if (p == 1) return mid >> 16;
    return __float_as_uint(r - __uint_as_float(mid)) >> 16;
}
__device__ __forceinline__ uint4 parts_of(const float x[8], int p)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = part_of(x[2 * i], p) | part_of(x[2 * i + 1], p) << 16;
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// four registers by four groups of 16 lanes, transposed
__device__ __forceinline__ void transpose4(uint32_t r[4])
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uintx2 t = __builtin_amdgcn_permlane32_swap(r[i], r[i + 2], false, false);
        r[i] = t.x; r[i + 2] = t.y;
    }
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const uintx2 t = __builtin_amdgcn_permlane16_swap(r[i], r[i + 1], false, false);
        r[i] = t.x; r[i + 1] = t.y;
    }
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ split_bf16x8 codes_bf16(uint32_t w)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 2), e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 3);
    return split_bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, e.x, e.y};
}

// What a wavefront has of four groups of 16 rows: their codes, a group a lane, and its row's four scales
struct Four { uint4 w; H4 s; };

__device__ __forceinline__ Four four_groups(const uint4 *__restrict__ codes, const uint16_t *__restrict__ scales, int64_t row, int32_t groups, int32_t g0, int j)
{
    Four f;
    const int64_t at = row * groups + g0;
    if (g0 + 4 <= groups) {
        f.w = codes[at + j];
        f.s = *reinterpret_cast<const H4 *>(scales + at);
    } else {
        f.w = make_uint4(0u, 0u, 0u, 0u);
        if (g0 + j < groups) f.w = codes[at + j];
#pragma unroll
        for (int h = 0; h < 4; ++h) f.s.x[h] = g0 + h < groups ? scales[at + h] : 0;
    }
    return f;
}

// PARTS: of a question; TILES: of 16 questions, 0: up to FEW questions (1 or 4), their parts as rows of one tile; a wavefront takes 32 rows at a
// time, and has the next four groups on their way while it multiplies.
// LDS: [group][tile][part] 1 KB each, what a lane hands the matrix instruction
template <bool BF16, int PARTS, int TILES, int FEW>
__global__ __launch_bounds__(256) void k_table4_scores(const uint4 *__restrict__ codes, const uint16_t *__restrict__ scales, int64_t n_rows, int32_t d,
                                                       int32_t groups, Questions Q, float *__restrict__ out, int64_t ldo)
{
    constexpr int SUMS = TILES ? 4 : FEW;                                        // of a lane's four that are wanted
    constexpr int T = TILES ? TILES : 1, P = TILES ? PARTS : 1, PER = T * P;     // operands of a group
    extern __shared__ uint4 s_q[];
    const int lane = threadIdx.x & 63, i16 = lane & 15, j = lane >> 4;
    const int64_t q0 = (int64_t)blockIdx.y * (TILES ? 16 * TILES : 4);
    const int64_t tiles = (n_rows + 31) >> 5, step = (int64_t)gridDim.x * 4;
    int64_t tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    // this lane's codes and scales of its row of a tile; what is inside the table and has four groups goes by them
    const uint4 *code = codes + (tile * 32 + i16) * groups + j;
    const uint16_t *scale = scales + (tile * 32 + i16) * groups;
    const int64_t stride = step * 32 * groups;
    const auto fetch = [&](int64_t t, int32_t g, Four f[2]) {
        if (t * 32 + 32 <= n_rows && g + 4 <= groups) {
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                f[a].w = code[16 * a * groups + g];
                f[a].s = *reinterpret_cast<const H4 *>(scale + 16 * a * groups + g);
            }
        } else {
#pragma unroll
            for (int a = 0; a < 2; ++a) f[a] = four_groups(codes, scales, min(t * 32 + 16 * a + i16, n_rows - 1), groups, g, j);
        }
    };
    Four now[2];                   // on their way while the questions are laid out
    fetch(tile, 0, now);
    for (int e = threadIdx.x; e < groups * T * 64; e += 256) {                   // a lane's part of a group's operands
        const int l = e & 63, op = e >> 6, row = l & 15, k = op / T * G + 8 * (l >> 4);
        float x[8];
        if (TILES) {
            question8<BF16>(Q, q0 + 16 * (op % T) + row, k, d, x);
#pragma unroll
            for (int p = 0; p < P; ++p) s_q[(op * P + p) * 64 + l] = parts_of(x, p);
        } else if (row < 4) {
            question8<BF16>(Q, q0 + row, k, d, x);
#pragma unroll
            for (int p = 0; p < 4; ++p) s_q[op * 64 + l + 4 * p] = p < PARTS ? parts_of(x, p) : make_uint4(0u, 0u, 0u, 0u);
        }
    }
    __syncthreads();
    if (tile >= tiles) return;
    floatx4 acc[2][T];
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int t = 0; t < T; ++t) acc[a][t] = floatx4{0.f, 0.f, 0.f, 0.f};
    float *mine = out + (q0 + 4 * j) * ldo;      // of this lane's first question, and how many there are from it on
    const int left = (int)min(Q.n - q0 - 4 * j, (int64_t)(16 * T));
    int32_t g0 = 0;
    for (;;) {
        const bool last = g0 + 4 >= groups;
        const int64_t next_tile = last ? tile + step : tile;
        const int32_t next_g0 = last ? 0 : g0 + 4;
        Four next[2];
        if (last) { code += stride; scale += stride; }
        if (next_tile < tiles) fetch(next_tile, next_g0, next);
        uint32_t r[2][4];
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            r[a][0] = now[a].w.x; r[a][1] = now[a].w.y; r[a][2] = now[a].w.z; r[a][3] = now[a].w.w;
            transpose4(r[a]);
        }
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            if (g0 + h >= groups) break;
            const split_bf16x8 c0 = codes_bf16(r[0][h]), c1 = codes_bf16(r[1][h]);
            const float s0 = bf16_float(now[0].s.x[h]), s1 = bf16_float(now[1].s.x[h]);
#pragma unroll
            for (int t = 0; t < T; ++t) {
                floatx4 v0 = {0.f, 0.f, 0.f, 0.f}, v1 = v0;
#pragma unroll
                for (int p = P - 1; p >= 0; --p) {
                    const split_bf16x8 q = __builtin_bit_cast(split_bf16x8, s_q[((g0 + h) * PER + t * P + p) * 64 + lane]);
                    v0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q, c0, v0, 0, 0, 0);
                    v1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q, c1, v1, 0, 0, 0);
                }
#pragma unroll
                for (int k = 0; k < SUMS; ++k) {
                    acc[0][t][k] = fmaf(s0, v0[k], acc[0][t][k]);
                    acc[1][t][k] = fmaf(s1, v1[k], acc[1][t][k]);
                }
            }
        }
        if (last) {
            // a lane holds its row's sums with rows 4 j .. 4 j + 3 of each tile of questions
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                const int64_t row = tile * 32 + 16 * a + i16;
                if (TILES) {
                    float *o = mine + row;
#pragma unroll
                    for (int t = 0; t < T; ++t)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (16 * t + k < left && row < n_rows) o[(16 * t + k) * ldo] = acc[a][t][k];
                } else {
                    float sum = 0.f;
#pragma unroll
                    for (int k = 0; k < SUMS; ++k) {
                        const float v = acc[a][0][k];
                        const float all = PARTS == 3 ? __shfl(v, i16, 64) + (__shfl(v, i16 + 16, 64) + __shfl(v, i16 + 32, 64)) : __shfl(v, i16, 64);
                        if (j == k) sum = all;
                    }
                    if (j < SUMS && q0 + j < Q.n && row < n_rows) out[(q0 + j) * ldo + row] = sum;
                }
#pragma unroll
                for (int t = 0; t < T; ++t) acc[a][t] = floatx4{0.f, 0.f, 0.f, 0.f};
            }
            if (next_tile >= tiles) break;
        }
        tile = next_tile;
        g0 = next_g0;
#pragma unroll
        for (int a = 0; a < 2; ++a) now[a] = next[a];
    }
}

constexpr int LDS_MOST = 160 << 10;

template <bool BF16, int PARTS, int TILES, int FEW = 4>
int launch_scores(const kge_table4 *t, int32_t groups, const Questions &Q, float *scores, int64_t lds, hipStream_t st)
{
    const int bytes = groups * (TILES ? TILES * PARTS : 1) * 1024;
    const int64_t batches = cdiv(Q.n, TILES ? 16 * TILES : 4), tiles = cdiv(t->n_rows, 32);
    int64_t blocks = cdiv(tiles, 4);
    // as many as run at once: registers leave room for four to a compute unit with up to 16 questions, else for three.  37 questions to 2.9 million
    // rows: 1024 blocks 187 us, 768 151
    const int64_t most = 256ll * std::max(1, std::min(TILES <= 1 ? 4 : 3, LDS_MOST / bytes));
    if (blocks > most) blocks = most;
    auto kernel = k_table4_scores<BF16, PARTS, TILES, FEW>;
    if (bytes > 64 << 10) KGE_HIP(hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
    for (int64_t b = 0; b < batches; b += 65535) {
        Questions part = Q;
        const int64_t q = b * (TILES ? 16 * TILES : 4);
        const int64_t here = batches - b < 65535 ? batches - b : 65535;
        part.n = Q.n - q;
        if (part.fixed) part.fixed += q; else part.X = (const char *)part.X + q * part.ldx * (BF16 ? 2 : 4);
        if (part.rel) part.rel += q; else if (part.M) part.M += q * part.ldm;
        if (!part.fixed) part.n_x -= q;
        if (!part.rel) part.n_m -= q;
        kernel<<<dim3((unsigned)blocks, (unsigned)here), 256, bytes, st>>>((const uint4 *)t->codes, t->scales, t->n_rows, t->d, groups, part, scores + q * lds, lds);
        KGE_LAUNCH_CHECK();
    }
    return KGE_OK;
}

template <bool BF16, int PARTS>
int scores_of(const kge_table4 *t, int32_t groups, const Questions &Q, float *scores, int64_t lds, hipStream_t st)
{
    const int tile = groups * PARTS * 1024;
    if (Q.n == 1) return launch_scores<BF16, PARTS, 0, 1>(t, groups, Q, scores, lds, st);
    if (Q.n <= 4 || tile > LDS_MOST) return launch_scores<BF16, PARTS, 0>(t, groups, Q, scores, lds, st);
    if (Q.n <= 16 || 2 * tile > LDS_MOST) return launch_scores<BF16, PARTS, 1>(t, groups, Q, scores, lds, st);
    if (Q.n <= 32 || 3 * tile > LDS_MOST) return launch_scores<BF16, PARTS, 2>(t, groups, Q, scores, lds, st);
    if (Q.n <= 48 || 4 * tile > LDS_MOST) return launch_scores<BF16, PARTS, 3>(t, groups, Q, scores, lds, st);
    return launch_scores<BF16, PARTS, 4>(t, groups, Q, scores, lds, st);
}

int check_table(const kge_table4 *t)
{
    KGE_REQUIRE(t, KGE_EINVAL, "NULL argument");
    KGE_REQUIRE(t->d >= 1 && t->d <= 4096, KGE_EINVAL, "rows have 1 to 4096 elements");
    KGE_REQUIRE(t->n_rows >= 0, KGE_EINVAL, "negative number of rows");
    KGE_REQUIRE(t->n_rows <= 0x7fffffffll, KGE_ERANGE, "2^31 rows or more");
    KGE_REQUIRE(t->n_rows == 0 || (t->codes && t->scales), KGE_EINVAL, "NULL codes or scales");
    KGE_REQUIRE((uintptr_t)t->codes % 16 == 0 && (uintptr_t)t->scales % 2 == 0, KGE_EINVAL, "codes must be aligned to 16 bytes, scales to 2");
    return KGE_OK;
}

int check_rows(const char *name, const void *p, int64_t n, int64_t ld, int32_t d, int32_t dtype)
{
    KGE_REQUIRE(dtype == KGE_DT_F32 || dtype == KGE_DT_BF16, KGE_EINVAL, "%s: bad type", name);
    KGE_REQUIRE(ld >= d && ld <= (1ll << 40), KGE_EINVAL, "%s: the row stride is less than a row", name);
    KGE_REQUIRE(n == 0 || p, KGE_EINVAL, "%s: NULL", name);
    KGE_REQUIRE((uintptr_t)p % (dtype == KGE_DT_F32 ? 4 : 2) == 0, KGE_EINVAL, "%s: not aligned to its elements", name);
    return KGE_OK;
}

}  // namespace

extern "C" int kge_table4_encode(const kge_table4 *table, int32_t dtype, const void *X, int64_t ldx, void *stream)
{
    int rc = check_table(table);
    if (rc == KGE_OK) rc = check_rows("X", X, table->n_rows, ldx, table->d, dtype);
    if (rc != KGE_OK || table->n_rows == 0) return rc;
    hipStream_t st = (hipStream_t)stream;
    const int32_t groups = (int32_t)cdiv(table->d, G);
    const int64_t blocks = cdiv(table->n_rows * groups, BLOCK_GROUPS);
    KGE_REQUIRE(blocks <= 0x7fffffffll / 256, KGE_ERANGE, "2^31 groups or more");
    KGE_PROF("table4_encode", st);
    (dtype == KGE_DT_BF16 ? k_table4_encode<true> : k_table4_encode<false>)<<<(unsigned)blocks, 256, 0, st>>>(X, ldx, table->n_rows, table->d, groups,
                                                                                                            (uint32_t *)table->codes, table->scales);
    KGE_LAUNCH_CHECK();
    return KGE_OK;
}

extern "C" int kge_table4_decode(const kge_table4 *table, const int32_t *rows, int64_t n, int32_t dtype, void *out, int64_t ldo, void *stream)
{
    int rc = check_table(table);
    KGE_REQUIRE(rc != KGE_OK || n >= 0, KGE_EINVAL, "negative number of rows");
    KGE_REQUIRE(rc != KGE_OK || rows || n <= table->n_rows, KGE_EINVAL, "more rows than the table has");
    if (rc == KGE_OK) rc = check_rows("out", out, n, ldo, table->d, dtype);
    if (rc != KGE_OK || n == 0) return rc;
    hipStream_t st = (hipStream_t)stream;
    const int32_t groups = (int32_t)cdiv(table->d, G);
    KGE_REQUIRE(n <= 0x7fffffffll && cdiv(n * groups, BLOCK_GROUPS) <= 0x7fffffffll / 256, KGE_ERANGE, "2^31 groups or more");
    KGE_PROF("table4_decode", st);
    (dtype == KGE_DT_BF16 ? k_table4_decode<true> : k_table4_decode<false>)<<<(unsigned)cdiv(n * groups, BLOCK_GROUPS), 256, 0, st>>>(
        (const uint16_t *)table->codes, table->scales, table->n_rows, table->d, groups, rows, n, out, ldo);
    KGE_LAUNCH_CHECK();
    return KGE_OK;
}

extern "C" int kge_table4_scores(const kge_table4 *table, int32_t dtype, const void *X, int64_t ldx, int64_t n_x, const int32_t *fixed,
                                 const float *M, int64_t ldm, int64_t n_m, const int32_t *rel, int64_t n_questions, float *scores, int64_t lds,
                                 void *stream)
{
    int rc = check_table(table);
    if (rc != KGE_OK) return rc;
    KGE_REQUIRE(n_x >= 0 && n_m >= 0 && n_questions >= 0, KGE_EINVAL, "negative size");
    KGE_REQUIRE(n_questions <= 0x7fffffffll, KGE_ERANGE, "2^31 questions or more");
    rc = check_rows("X", X, n_questions, ldx, table->d, dtype);
    if (rc == KGE_OK && M) rc = check_rows("M", M, n_m, ldm, table->d, KGE_DT_F32);
    if (rc != KGE_OK) return rc;
    KGE_REQUIRE(fixed || n_questions <= n_x, KGE_EINVAL, "without fixed every question is a row of X");
    KGE_REQUIRE(M || !rel, KGE_EINVAL, "rel names rows of M: M is NULL");
    KGE_REQUIRE(!M || rel || n_questions <= n_m, KGE_EINVAL, "without rel every question has a row of M");
    KGE_REQUIRE((uintptr_t)fixed % 4 == 0 && (uintptr_t)rel % 4 == 0, KGE_EINVAL, "fixed and rel must be aligned to their elements");
    KGE_REQUIRE(lds >= table->n_rows, KGE_EINVAL, "scores: the row stride is less than a row");
    if (n_questions == 0 || table->n_rows == 0) return KGE_OK;
    KGE_REQUIRE(scores && (uintptr_t)scores % 4 == 0, KGE_EINVAL, "scores: NULL or not aligned");
    const Questions Q{X, M, fixed, rel, ldx, ldm, n_x, n_m, n_questions};
    const int32_t groups = (int32_t)cdiv(table->d, G);
    hipStream_t st = (hipStream_t)stream;
    KGE_PROF("table4_scores", st);
    if (dtype == KGE_DT_F32) return scores_of<false, 3>(table, groups, Q, scores, lds, st);
    if (M) return scores_of<true, 3>(table, groups, Q, scores, lds, st);
    return scores_of<true, 1>(table, groups, Q, scores, lds, st);
}
