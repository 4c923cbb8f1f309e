// What the dense layer's kernels share: accesses of eight elements at any element's address, the activations, and the
// arguments of a product C[i][j] = sum_k A[i][k] B[k][j].
#pragma once
#include "common.h"
#include "split_bf16.h"

#include <type_traits>

namespace dense {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

enum { FORWARD = 0, INPUT = 1, WEIGHTS = 2 };

__device__ __forceinline__ float bf(uint32_t w16) { return __uint_as_float(w16 << 16); }

// 8 consecutive elements from a (n of them exist; the others read as zeros).  Rows may start at any element: the loads ask
// for no more alignment than an element has
struct __attribute__((packed, aligned(4))) F8 { float x[8]; };
struct __attribute__((packed, aligned(2))) H8 { uint32_t w[4]; };
__device__ __forceinline__ void load8(const float *a, float x[8])
{
    const F8 q = *reinterpret_cast<const F8 *>(a);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = q.x[k];
}
__device__ __forceinline__ uint4 load8(const uint16_t *a)
{
    const H8 q = *reinterpret_cast<const H8 *>(a);
    return make_uint4(q.w[0], q.w[1], q.w[2], q.w[3]);
}
__device__ __forceinline__ void load8(const float *a, int n, float x[8])
{
    if (n >= 8) load8(a, x);
    else {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = 0.f;
        if (n > 0) {               // past the end the last element again: no branch parts the loads
#pragma unroll
            for (int k = 0; k < 7; ++k) x[k] = a[min(k, n - 1)];
#pragma unroll
            for (int k = 1; k < 7; ++k) x[k] = k < n ? x[k] : 0.f;
        }
    }
}
__device__ __forceinline__ uint4 load8(const uint16_t *a, int n)
{
    if (n >= 8) return load8(a);
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    if (n > 0) {
        uint32_t x[7];
#pragma unroll
        for (int k = 0; k < 7; ++k) x[k] = a[min(k, n - 1)];
#pragma unroll
        for (int k = 0; k < 7; ++k) w[k >> 1] |= k < n ? x[k] << (16 * (k & 1)) : 0u;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void spread(uint4 q, float x[8])
{
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) { x[2 * k] = bf(w[k] & 0xffffu); x[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u); }
}

// e^-z from the instruction for 2^x; below 2^-126 it is zero beside the one that it is added to.  Rounding the argument leaves it up to
// 1.2 (1 + |z|) 2^-24 of itself off, and the instruction and the reciprocal's a unit in the last place each.  Where that is many units, z
// far below zero, silu is small with e^z: over [-100, 100] it is at most 0.65 x 2^-22 of the larger of one and itself off.  Its derivative
// is at most 2^-20 off, at z near 16, where 1 - s has no more digits in fp32.  A second step for the argument's rest would cost the backward
// pass, which is bound by act', two more instructions an element
__device__ __forceinline__ float exp_minus(float z) { return __builtin_amdgcn_exp2f(z * -1.44269504f); }
template <int ACT>
__device__ __forceinline__ float act_of(float z)
{
    return ACT == KGE_ACT_RELU ? (z < 0.f ? 0.f : z) : ACT == KGE_ACT_SILU ? z * __builtin_amdgcn_rcpf(1.f + exp_minus(z)) : z;
}
// dP = dy act'(z).  ReLU chooses: where z is not above zero nothing of dy is left, an infinity or NaN neither (a NaN is not above)
template <int ACT>
__device__ __forceinline__ float through_act(float dy, float z)
{
    if (ACT == KGE_ACT_RELU) return z > 0.f ? dy : 0.f;
    if (ACT == KGE_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.f + exp_minus(z));
        return dy * (s * (1.f + z * (1.f - s)));
    }
    return dy;
}
// the same of two bf16 numbers under ReLU
__device__ __forceinline__ uint32_t relu_pair(uint32_t dy, uint32_t z)
{
    return (bf(z & 0xffffu) > 0.f ? dy & 0xffffu : 0u) | (__uint_as_float(z & 0xffff0000u) > 0.f ? dy & 0xffff0000u : 0u);
}

// the first n of 8 numbers to a (n >= 8: all)
__device__ __forceinline__ void store8(float *a, int n, const float x[8])
{
    if (n >= 8) {
        F8 q;
#pragma unroll
        for (int k = 0; k < 8; ++k) q.x[k] = x[k];
        *reinterpret_cast<F8 *>(a) = q;
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) if (k < n) a[k] = x[k];
    }
}
__device__ __forceinline__ void store8(uint16_t *a, int n, const float x[8])
{
    H8 q;
#pragma unroll
    for (int k = 0; k < 4; ++k) q.w[k] = split_round(x[2 * k], x[2 * k + 1]);
    if (n >= 8) *reinterpret_cast<H8 *>(a) = q;
    else {
#pragma unroll
        for (int k = 0; k < 8; ++k) if (k < n) a[k] = (uint16_t)(q.w[k >> 1] >> (16 * (k & 1)));
    }
}

__device__ __forceinline__ float elem(const float *a) { return *a; }
__device__ __forceinline__ float elem(const uint16_t *a) { return bf(*a); }
__device__ __forceinline__ void put(float *a, float x) { *a = x; }
__device__ __forceinline__ void put(uint16_t *a, float x) { *a = __builtin_bit_cast(uint16_t, (__bf16)x); }

template <class T>
struct Args {
    const T *A, *B;                // as stored (see the table above)
    int64_t lda, ldb;
    const T *pre;                  // laid out like the operand that is dP (A of INPUT, B of WEIGHTS)
    int64_t ldpre;
    int64_t M;                     // rows of the result
    int32_t N;                     // its columns
    int64_t K;                     // terms
    int64_t chunk;                 // terms per block (WEIGHTS; K otherwise)
    int32_t tiles_n;
    uint32_t wide;                 // blocks in front of those of the last, narrow columns
    int64_t tiles_m;
    T *C, *pre_out;                // FORWARD: Y, pre;  INPUT: dX
    int64_t ldc, ldp;
    const T *add;                  // FORWARD: R;  INPUT: add
    int64_t ldadd;
    const float *bias;
    float *part, *part_b;          // WEIGHTS: [chunks][M][N] sums, [chunks][N] sums of dP's columns (or null)
};

template <int PARTS>
__device__ __forceinline__ void to_lds(const float x[8], unsigned char *at, int plane)
{
    uint32_t w[3][4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const Split3 s = split_pair(x[2 * k], x[2 * k + 1]);
        w[0][k] = s.w[0]; w[1][k] = s.w[1]; w[2][k] = s.w[2];
    }
#pragma unroll
    for (int p = 0; p < PARTS; ++p) *reinterpret_cast<uint4 *>(at + p * plane) = make_uint4(w[p][0], w[p][1], w[p][2], w[p][3]);
}

// dense_rows_*.hip: FORWARD and INPUT for long matrices of narrow rows, at most ROWS_TERMS terms
template <class T> constexpr int32_t ROWS_TERMS = sizeof(T) == 4 ? 128 : 256;
// whether whole tiles of 32 rows may go through that kernel's loop without branches: chunks of 8 elements that exist or do not, and
// rows of the result at words of 4 bytes that 31 bits reach
template <class T>
bool rows_counted(const Args<T> &a)
{
    auto words = [](const T *p, int64_t ld) { return ((uintptr_t)p % 4) == 0 && (ld * (int64_t)sizeof(T)) % 4 == 0 && ld * 32 * (int64_t)sizeof(T) < 0x7fff0000; };
    return a.K % 8 == 0 && a.N % 8 == 0 && words(a.C, a.ldc) && (!a.pre_out || words(a.pre_out, a.ldp));
}
// Where it pays (us against the tiled kernel's, forward / input gradient).  fp32, 65 terms and more, 16384 rows and more: 16.9 / 13.8
// against 20.5 / 18.7 at 16000 x 128 x 128, 298 / 301 against 402 / 343 at 10^6; with 64 terms 207 / 220 against 214 / 181.  bf16: the tiles
// split nothing, and loading all of B into every block costs about 20 us: 51.7 / 58.1 against 42.4 / 66.0 at 128000 x 256 x 256,
// 315 / 421 against 358 / 505 at 10^6, and 99 / 155 against 83 / 109 with 64 terms; 777 / 705 against 646 / 687 at 10^6 x 100 x 500, in the
// loop with branches.
template <class T>
bool rows_pay(const Args<T> &a)
{
    if (a.K <= 64 || a.K > ROWS_TERMS<T>) return false;
    return sizeof(T) == 4 ? a.M >= 16384 : a.M >= 200000 && rows_counted(a);
}
template <int MODE, class T> int launch_rows(const Args<T> &a, int act, hipStream_t st);
template <> int launch_rows<FORWARD, float>(const Args<float> &a, int act, hipStream_t st);
template <> int launch_rows<FORWARD, uint16_t>(const Args<uint16_t> &a, int act, hipStream_t st);
template <> int launch_rows<INPUT, float>(const Args<float> &a, int act, hipStream_t st);
template <> int launch_rows<INPUT, uint16_t>(const Args<uint16_t> &a, int act, hipStream_t st);

// dense_few.hip: FORWARD and INPUT of few results.  Its time grows with blocks x terms where the tiled kernel's grows with the terms
// alone: at 1024 blocks of 32 x 32, 18.9 / 28.2 us against 22.7 / 46.9 (1000 terms, bf16) and 29.6 / 42.9 against 63.0 / 78.3 (fp32); at
// 2048, 31.5 / 51.3 against 21.8 / 49.4 and 51.8 / 79.0 against 67.4 / 81.0.
template <class T>
bool few_pay(const Args<T> &a) { return cdiv(a.M, 32) * cdiv(a.N, 32) <= (sizeof(T) == 4 ? 2048 : 1024); }
template <int MODE, class T> int launch_few(Args<T> a, int act, hipStream_t st);

}  // namespace dense
