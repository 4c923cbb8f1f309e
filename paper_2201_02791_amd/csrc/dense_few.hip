// Dense layer, forward product and input gradient, of few results: single rows, small batches, narrow layers.
//
// Tiles of 128 x 128 would leave most of the chip without one and walk through the terms one after another.  Here a block
// has 32 x 32 results and its eight wavefronts share the terms: each loads its operands from memory straight into the
// order of the matrix instruction (8 consecutive terms of a row a lane; of W, whose columns lie side by side, 32
// neighbours a load), without LDS and without a barrier until their eight sums meet there.  What bounds it is the latency of
// two or three dependent loads; rows past the last repeat it, their results are not stored.  One row of 1024 by 1024 bf16: 4.7 us on
// the device (17 us in the tiled kernel), 10 with the host's part of the call.
#include "dense.h"

using namespace dense;

namespace {

constexpr int NW = 8, NT = 64 * NW, LD = 33;

template <int MODE, class T, int ACT>
__global__ __launch_bounds__(NT) void k_dense_few(Args<T> a)
{
    constexpr bool F32 = sizeof(T) == 4, SOFT = !F32 && MODE == INPUT && ACT == KGE_ACT_SILU, GRAD = MODE == INPUT && ACT != KGE_ACT_IDENTITY;
    constexpr int P = F32 ? 3 : SOFT ? 2 : 1, PB = F32 ? 3 : 1;
    __shared__ float sums[NW][32 * LD];
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t m0 = (int64_t)(blockIdx.x / (uint32_t)a.tiles_n) * 32;
    const int32_t n0 = (int32_t)(blockIdx.x % (uint32_t)a.tiles_n) * 32;
    const int32_t K = (int32_t)a.K;
    const int64_t m = min(m0 + (lane & 31), a.M - 1);
    const int32_t n = min(n0 + (lane & 31), a.N - 1);
    const int kl = 8 * (lane >> 5);
    const T *const pa = a.A + m * a.lda + kl, *const pg = GRAD ? a.pre + m * a.ldpre + kl : nullptr;
    const T *const pb = MODE == FORWARD ? a.B + (int64_t)kl * a.ldb + n : a.B + (int64_t)n * a.ldb + kl;

    floatx16 acc;
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = 0.f;
    struct Step { float x[8], z[8], y[8]; };
    auto load = [&](Step &h, int32_t k, auto whole) __attribute__((always_inline)) {
        constexpr bool WHOLE = decltype(whole)::value;
        auto eight = [&](const T *p, float *to) __attribute__((always_inline)) {
            if constexpr (F32) {
                if (WHOLE) load8(p, to);
                else load8(p, K - k - kl, to);
            } else spread(WHOLE ? load8(p) : load8(p, K - k - kl), to);
        };
        eight(pa + k, h.x);
        if (GRAD) eight(pg + k, h.z);
        if (MODE == FORWARD) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const T v = pb[(int64_t)(WHOLE ? k + i : min(k + i, K - 1 - kl)) * a.ldb];
                h.y[i] = WHOLE || k + kl + i < K ? elem(&v) : 0.f;
            }
        } else eight(pb + k, h.y);
    };
    auto multiply = [&](Step &h) __attribute__((always_inline)) {
        if (GRAD) {
#pragma unroll
            for (int i = 0; i < 8; ++i) h.x[i] = through_act<ACT>(h.x[i], h.z[i]);
        }
        uint32_t fx[3][4], fy[3][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Split3 s = split_pair(h.x[2 * i], h.x[2 * i + 1]), u = split_pair(h.y[2 * i], h.y[2 * i + 1]);
#pragma unroll
            for (int p = 0; p < 3; ++p) { fx[p][i] = s.w[p]; fy[p][i] = u.w[p]; }
        }
        // smallest products first; of three parts each, those of 2^-24 of the product and below are left out
#pragma unroll
        for (int s = P + PB - 2; s >= 0; --s) {
            if (P == 3 && PB == 3 && s > 2) continue;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int q = s - p;
                if (q < 0 || q >= PB) continue;
                acc = split_mfma(make_uint4(fx[p][0], fx[p][1], fx[p][2], fx[p][3]), make_uint4(fy[q][0], fy[q][1], fy[q][2], fy[q][3]), acc);
            }
        }
    };
    // wavefront w takes every eighth step of 16 terms, the loads of two at a time
    const std::true_type whole{};
    int32_t k = 16 * w;
    Step s0, s1;
    for (; k + 16 * NW + 16 <= K; k += 32 * NW) {
        load(s0, k, whole);
        load(s1, k + 16 * NW, whole);
        multiply(s0);
        multiply(s1);
    }
    for (; k < K; k += 16 * NW) {
        if (k + 16 <= K) load(s0, k, whole);
        else load(s0, k, std::false_type());
        multiply(s0);
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) sums[w][(8 * (v >> 2) + 4 * (lane >> 5) + (v & 3)) * LD + (lane & 31)] = acc[v];
    __syncthreads();
    // two neighbours in a row of results a thread
    const int r = t >> 4, c = 2 * (t & 15);
    const int64_t mi = m0 + r;
    if (mi >= a.M) return;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int32_t ni = n0 + c + j;
        if (ni >= a.N) continue;
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i) x += sums[i][r * LD + c + j];
        if (P + PB > 2 && split_not_finite(x)) {       // once more from fp32 products, term by term
            x = 0.f;
            for (int32_t i = 0; i < K; ++i) {
                float y = elem(a.A + mi * a.lda + i);
                if (GRAD) y = through_act<ACT>(y, elem(a.pre + mi * a.ldpre + i));
                x = fmaf(y, elem(MODE == FORWARD ? a.B + (int64_t)i * a.ldb + ni : a.B + (int64_t)ni * a.ldb + i), x);
                if (x != x) break;             // a NaN stays one: of inputs that are all NaN one term is read
            }
        }
        if (MODE == FORWARD) {
            if (a.bias) x += a.bias[ni];
            if (a.pre_out) put(a.pre_out + mi * a.ldp + ni, x);
            x = act_of<ACT>(x);
        }
        if (a.add) x += elem(a.add + mi * a.ldadd + ni);
        put(a.C + mi * a.ldc + ni, x);
    }
}

}  // namespace

namespace dense {

template <int MODE, class T>
int launch_few(Args<T> a, int act, hipStream_t st)
{
    a.tiles_n = (int32_t)cdiv(a.N, 32);
    const int64_t blocks = cdiv(a.M, 32) * a.tiles_n;
    KGE_REQUIRE(blocks <= 0x7fffffffLL, KGE_ERANGE, "dense: too large for one launch");
    if (act == KGE_ACT_RELU) k_dense_few<MODE, T, KGE_ACT_RELU><<<(unsigned)blocks, NT, 0, st>>>(a);
    else if (act == KGE_ACT_SILU) k_dense_few<MODE, T, KGE_ACT_SILU><<<(unsigned)blocks, NT, 0, st>>>(a);
    else k_dense_few<MODE, T, KGE_ACT_IDENTITY><<<(unsigned)blocks, NT, 0, st>>>(a);
    KGE_LAUNCH_CHECK();
    return KGE_OK;
}
template int launch_few<FORWARD, float>(Args<float>, int, hipStream_t);
template int launch_few<FORWARD, uint16_t>(Args<uint16_t>, int, hipStream_t);
template int launch_few<INPUT, float>(Args<float>, int, hipStream_t);
template int launch_few<INPUT, uint16_t>(Args<uint16_t>, int, hipStream_t);

}  // namespace dense
