// Embedding tables of 4-bit numbers, and the scores of questions against every row of one.
//
// A row is cut into groups of 32 elements; a group has a scale s, a bf16 number, and its elements are numbers c of the format
// e2m1 (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives) times s.  s is the smallest bf16 number, 2^-126 or more, with
// 6 s >= the group's largest magnitude, so nothing saturates; 4.5 bits an element in all.
//
// Encoding compares magnitudes with the borders between two numbers, s times 1/4, 3/4, 5/4, 7/4, 5/2, 7/2 and 5: products
// of at most 11 bits, exact in fp32, so that every element goes to the nearest number (of two as near, to the even code).
#include "common.h"
#include "split_bf16.h"

namespace {

constexpr int G = KGE_TABLE4_GROUP;
static_assert(G == 32, "a group is one step of the matrix instruction and 16 bytes of codes");

typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef unsigned uintx2 __attribute__((ext_vector_type(2)));

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

// the bits of the smallest bf16 number, 2^-126 or more, six of which reach `most`; NaN where a member is not finite
__device__ __forceinline__ uint32_t group_scale(uint32_t most)
{
    if (most == 0u) return 0u;
    if (most >= 0x7f800000u) return 0x7fc00000u;
    const float a = __uint_as_float(most);
    float s = __uint_as_float(max(__float_as_uint(a * (1.f / 6.f)) & 0xffff0000u, 0x00800000u));
#pragma unroll
    for (int k = 0; k < 2; ++k)      // the product is rounded and then cut: at most two steps short
        if (6.f * s < a) s = __uint_as_float(__float_as_uint(s) + 0x10000u);
    return __float_as_uint(s);
}

__device__ __forceinline__ uint32_t code_of(float x, float s)
{
    const float a = fabsf(x);
    const uint32_t c = (a > 0.25f * s) + (a >= 0.75f * s) + (a > 1.25f * s) + (a >= 1.75f * s) + (a > 2.5f * s) + (a >= 3.5f * s) + (a > 5.f * s);
    return c | (x < 0.f ? 8u : 0u);
}

// 4 lanes to a group, 8 elements each
template <bool BF16>
__global__ __launch_bounds__(256) void k_table4_encode(const void *__restrict__ X, int64_t ldx, int64_t n_rows, int32_t d, int32_t groups,
                                                       uint32_t *__restrict__ codes, uint16_t *__restrict__ scales)
{
    const int64_t first = (int64_t)blockIdx.x * 64;              // this block's first group
    const int64_t row0 = first / groups;
    const uint32_t local = (uint32_t)(first - row0 * groups) + (threadIdx.x >> 2);
    const int64_t row = row0 + local / (uint32_t)groups;
    const int32_t g = (int32_t)(local % (uint32_t)groups), j = threadIdx.x & 3;
    const int32_t c = g * G + 8 * j;
    const int n = row < n_rows ? d - c : 0;
    float x[8];
    load4<BF16>(X, row * ldx + c, n, x);
    load4<BF16>(X, row * ldx + c + 4, n - 4, x + 4);
    uint32_t most = 0u;
#pragma unroll
    for (int k = 0; k < 8; ++k) most = max(most, __float_as_uint(x[k]) & 0x7fffffffu);
    most = max(most, (uint32_t)__shfl_xor((int)most, 1, 64));
    most = max(most, (uint32_t)__shfl_xor((int)most, 2, 64));
    const uint32_t bits = group_scale(most);
    const float s = __uint_as_float(bits);
    uint32_t w = 0u;
    if (s > 0.f) {
#pragma unroll
        for (int k = 0; k < 8; ++k) w |= code_of(x[k], s) << (4 * k);
    }
    if (row < n_rows) {
        const int64_t at = row * groups + g;
        codes[at * 4 + j] = w;
        if (j == 0) scales[at] = (uint16_t)(bits >> 16);
    }
}

// 4 lanes to a group, 8 elements each; ids null: rows in order
template <bool BF16>
__global__ __launch_bounds__(256) void k_table4_decode(const uint32_t *__restrict__ codes, const uint16_t *__restrict__ scales, int64_t n_rows, int32_t d,
                                                       int32_t groups, const int32_t *__restrict__ ids, int64_t n_out, void *__restrict__ out, int64_t ldo)
{
    const int64_t first = (int64_t)blockIdx.x * 64;
    const int64_t row0 = first / groups;
    const uint32_t local = (uint32_t)(first - row0 * groups) + (threadIdx.x >> 2);
    const int64_t row = row0 + local / (uint32_t)groups;
    const int32_t g = (int32_t)(local % (uint32_t)groups), j = threadIdx.x & 3;
    const int32_t c = g * G + 8 * j;
    if (row >= n_out || c >= d) return;
    const int64_t src = ids ? ids[row] : row;
    float s = __uint_as_float(0x7fc00000u);                      // a row that the table does not have
    uint32_t w = 0u;
    if (src >= 0 && src < n_rows) {
        const int64_t at = src * groups + g;
        w = codes[at * 4 + j];
        s = bf16_float(scales[at]);
    }
    float y[8];
    const floatx2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 1);
    const floatx2 p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 3);
    y[0] = p0.x * s; y[1] = p0.y * s; y[2] = p1.x * s; y[3] = p1.y * s;
    y[4] = p2.x * s; y[5] = p2.y * s; y[6] = p3.x * s; y[7] = p3.y * s;
    const int n = d - c;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (BF16) {
            uint16_t *o = (uint16_t *)out + row * ldo + c + 4 * h;
            H4 q;
#pragma unroll
            for (int k = 0; k < 4; ++k) q.x[k] = __builtin_bit_cast(uint16_t, (__bf16)y[4 * h + k]);
            if (n >= 4 * h + 4) *reinterpret_cast<H4 *>(o) = q;
            else {
#pragma unroll
                for (int k = 0; k < 3; ++k) if (4 * h + k < n) o[k] = q.x[k];
            }
        } else {
            float *o = (float *)out + row * ldo + c + 4 * h;
            if (n >= 4 * h + 4) *reinterpret_cast<F4 *>(o) = F4{{y[4 * h], y[4 * h + 1], y[4 * h + 2], y[4 * h + 3]}};
            else {
#pragma unroll
                for (int k = 0; k < 3; ++k) if (4 * h + k < n) o[k] = y[4 * h + k];
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
// More: 16 questions a tile, the parts' products chained, smallest first.

struct Questions {
    const void *X;
    const float *M;
    const int32_t *fixed, *rel;
    int64_t ldx, ldm, n_x, n_m, n;
};

template <bool BF16>
__device__ __forceinline__ float question(const Questions &Q, int64_t q, int32_t k, int32_t d)
{
    if (q >= Q.n || k >= d) return 0.f;
    const int64_t i = Q.fixed ? Q.fixed[q] : q, r = Q.rel ? Q.rel[q] : q;
    if (i < 0 || i >= Q.n_x || (Q.M && (r < 0 || r >= Q.n_m))) return __uint_as_float(0x7fc00000u);
    const float x = BF16 ? bf16_float(((const uint16_t *)Q.X)[i * Q.ldx + k]) : ((const float *)Q.X)[i * Q.ldx + k];
    return Q.M ? x * Q.M[r * Q.ldm + k] : x;
}

// part p of x: what bf16 cuts off x, of the rest what it cuts off, and what is left; their sum is x
__device__ __forceinline__ uint16_t part_of(float x, int p)
{
    const uint32_t hi = __float_as_uint(x) & 0xffff0000u;
    if (split_not_finite(x)) return p == 0 ? (x != x ? 0x7fc0 : hi >> 16) : 0;
    if (p == 0) return hi >> 16;
    const float r = x - __uint_as_float(hi);
    const uint32_t mid = __float_as_uint(r) & 0xffff0000u;
    if (p == 1) return mid >> 16;
    return __float_as_uint(r - __uint_as_float(mid)) >> 16;
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

// PARTS: of a question; TILES: of 16 questions, 0: up to four questions, their parts as rows of one tile.
// LDS: [group][tile][part] 1 KB each, what a lane hands the matrix instruction
template <bool BF16, int PARTS, int TILES>
__global__ __launch_bounds__(256) void k_table4_scores(const uint4 *__restrict__ codes, const uint16_t *__restrict__ scales, int64_t n_rows, int32_t d,
                                                       int32_t groups, Questions Q, float *__restrict__ out, int64_t ldo)
{
    constexpr int T = TILES ? TILES : 1, P = TILES ? PARTS : 1, PER = T * P;     // operands of a group
    extern __shared__ uint4 s_q[];
    const int lane = threadIdx.x & 63, i16 = lane & 15, j = lane >> 4;
    const int64_t q0 = (int64_t)blockIdx.y * (TILES ? 16 * TILES : 4);
    uint16_t *sq = (uint16_t *)s_q;
    for (int e = threadIdx.x; e < groups * PER * 512; e += 256) {                // element e: lane and place in its 8 numbers
        const int at = e & 7, l = (e >> 3) & 63, op = e >> 9;
        const int g = op / PER, t = op % PER / P, p = op % P, row = l & 15, k = g * G + 8 * (l >> 4) + at;
        if (TILES) sq[e] = part_of(question<BF16>(Q, q0 + 16 * t + row, k, d), p);
        else sq[e] = row >> 2 < PARTS ? part_of(question<BF16>(Q, q0 + (row & 3), k, d), row >> 2) : 0;
    }
    __syncthreads();
    const int64_t tiles = (n_rows + 15) >> 4, step = (int64_t)gridDim.x * 4;
    for (int64_t tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); tile < tiles; tile += step) {
        const int64_t row = tile * 16 + i16, src = row < n_rows ? row : n_rows - 1;
        floatx4 acc[T];
#pragma unroll
        for (int t = 0; t < T; ++t) acc[t] = floatx4{0.f, 0.f, 0.f, 0.f};
        for (int g0 = 0; g0 < groups; g0 += 4) {
            uint4 w = make_uint4(0u, 0u, 0u, 0u);
            if (g0 + j < groups) w = codes[src * groups + g0 + j];
            float s[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) s[h] = bf16_float(scales[src * groups + min(g0 + h, groups - 1)]);
            uint32_t r[4] = {w.x, w.y, w.z, w.w};
            transpose4(r);
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                if (g0 + h >= groups) break;
                const split_bf16x8 c = codes_bf16(r[h]);
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    floatx4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int p = P - 1; p >= 0; --p)
                        v = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(split_bf16x8, s_q[((g0 + h) * PER + t * P + p) * 64 + lane]), c, v, 0, 0, 0);
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[t][k] = fmaf(s[h], v[k], acc[t][k]);
                }
            }
        }
        // a lane holds its row's sums with rows 4 j .. 4 j + 3 of each tile of questions
        if (TILES) {
#pragma unroll
            for (int t = 0; t < T; ++t)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int64_t q = q0 + 16 * t + 4 * j + k;
                    if (q < Q.n && row < n_rows) out[q * ldo + row] = acc[t][k];
                }
        } else {
            float v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[k] = acc[0][k];
                if (PARTS == 3) {
                    const float mid = __shfl(v[k], i16 + 16, 64), low = __shfl(v[k], i16 + 32, 64);
                    v[k] = __shfl(v[k], i16, 64) + (mid + low);
                } else v[k] = __shfl(v[k], i16, 64);
            }
            const float mine = j == 0 ? v[0] : j == 1 ? v[1] : j == 2 ? v[2] : v[3];
            if (q0 + j < Q.n && row < n_rows) out[(q0 + j) * ldo + row] = mine;
        }
    }
}

constexpr int LDS_MOST = 160 << 10;

template <bool BF16, int PARTS, int TILES>
int launch_scores(const kge_table4 *t, int32_t groups, const Questions &Q, float *scores, int64_t lds, hipStream_t st)
{
    const int bytes = groups * (TILES ? TILES * PARTS : 1) * 1024;
    const int64_t batches = cdiv(Q.n, TILES ? 16 * TILES : 4), tiles = cdiv(t->n_rows, 16);
    int64_t blocks = cdiv(tiles, 4);
    if (blocks > 2048) blocks = 2048;
    auto kernel = k_table4_scores<BF16, PARTS, TILES>;
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
    if (Q.n <= 4 || tile > LDS_MOST) return launch_scores<BF16, PARTS, 0>(t, groups, Q, scores, lds, st);
    if (Q.n <= 16 || 2 * tile > LDS_MOST) return launch_scores<BF16, PARTS, 1>(t, groups, Q, scores, lds, st);
    if (Q.n <= 32 || 4 * tile > LDS_MOST) return launch_scores<BF16, PARTS, 2>(t, groups, Q, scores, lds, st);
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
    const int64_t blocks = cdiv(table->n_rows * groups, 64);
    KGE_REQUIRE(blocks <= 0x7fffffffll / 256, KGE_ERANGE, "2^29 groups or more");
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
    KGE_REQUIRE(n <= 0x7fffffffll && cdiv(n * groups, 64) <= 0x7fffffffll / 256, KGE_ERANGE, "2^29 groups or more");
    KGE_PROF("table4_decode", st);
    (dtype == KGE_DT_BF16 ? k_table4_decode<true> : k_table4_decode<false>)<<<(unsigned)cdiv(n * groups, 64), 256, 0, st>>>(
        (const uint32_t *)table->codes, table->scales, table->n_rows, table->d, groups, rows, n, out, ldo);
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
