// Dense layer, forward product and input gradient, for long matrices of narrow rows: C = A B with B held in registers.
//
// A layer of 128 or 256 columns reads and writes a row or two for every row of products, so the rows set the time and the
// matrix cores have time to spare.  A block stays: each of its wavefronts loads the B operands of its 32 columns once, all
// K terms of them (and splits them once, fp32), and then tiles of rows stream by.  While a tile is multiplied, the next
// one's rows (and R or `add`) are on their way to registers; from there they go to LDS as bf16 parts, dY becoming dP, and
// every wavefront reads all of them.  The sums return through LDS, in the place of the rows, so that bias, activation,
// residual and stores work on 16 to 32 consecutive bytes per lane.
//
// LDS rows are 16 bytes longer than their terms: an odd number of 16-byte chunks apart, eight rows meet all banks.
// Blocks of the several column groups of a wide result run on one XCD in step, so that the rows come from HBM once.
#include "dense.h"

using namespace dense;

namespace {

template <class T>
struct RowArgs {
    Args<T> a;
    int32_t act, groups;           // column groups
    int64_t lanes, tiles;          // blocks per group (a multiple of 8), row tiles
};

// KS: steps of 16 terms; WN: wavefronts side by side, 32 columns each; RB: blocks of 32 rows per wavefront and tile
template <int MODE, class T, bool SOFT, int KS, int WN, int RB>
struct Rows {
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr int P = F32 ? 3 : SOFT ? 2 : 1, PB = F32 ? 3 : 1;
    static constexpr int WM = WN >= 4 ? 1 : 4 / WN, NW = WN * WM, NT = 64 * NW, TR = 32 * RB * WM;
    static constexpr int STRIDE = KS * 32 + 16, PLANE = TR * STRIDE;
    static constexpr int OUT = 32 * WN + 8;                        // floats per row of sums: 4 rows further, 32 banks further
    static constexpr int CH = TR * KS * 2 / NT;         // chunks of 8 terms per thread and tile
    static constexpr int LDS = P * PLANE > TR * OUT * 4 ? P * PLANE : TR * OUT * 4;
};

template <bool RAW, int CH>
struct Chunks {
    uint4 q[RAW ? CH : 1];
    float x[RAW ? 1 : CH][8];
};

template <int MODE, class T, bool SOFT, int KS, int WN, int RB>
__global__ __launch_bounds__((Rows<MODE, T, SOFT, KS, WN, RB>::NT), 2) void k_dense_rows(RowArgs<T> r)
{
    typedef Rows<MODE, T, SOFT, KS, WN, RB> S;
    constexpr int P = S::P, PB = S::PB, NT = S::NT, TR = S::TR, CH = S::CH;
    constexpr bool F32 = S::F32;
    const Args<T> &a = r.a;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];

    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), wn = w % WN, wm = w / WN;
    // workgroup i runs on XCD i % 8: a row tile's column groups are neighbours there
    const int64_t seq = blockIdx.x >> 3;
    const int32_t n0 = (int32_t)(seq % r.groups) * 32 * WN;
    int64_t tile = (seq / r.groups) * 8 + (blockIdx.x & 7);
    const int32_t K = (int32_t)a.K;

    // B operand: column lane % 32 of the wavefront's 32, terms 16 ks + 8 (lane / 32) ..
    uint4 fb[PB][KS];
    {
        const int32_t n = n0 + 32 * wn + (lane & 31);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int32_t k = 16 * ks + 8 * (lane >> 5);
            float x[8];
            if (MODE == FORWARD) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = n < a.N && k + i < K ? elem(a.B + (int64_t)(k + i) * a.ldb + n) : 0.f;
            } else if constexpr (F32) load8(a.B + (int64_t)n * a.ldb + k, n < a.N ? K - k : 0, x);
            else spread(load8(a.B + (int64_t)n * a.ldb + k, n < a.N ? K - k : 0), x);
            uint32_t word[3][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Split3 s = split_pair(x[2 * i], x[2 * i + 1]);
#pragma unroll
                for (int p = 0; p < PB; ++p) word[p][i] = s.w[p];
            }
#pragma unroll
            for (int p = 0; p < PB; ++p) fb[p][ks] = make_uint4(word[p][0], word[p][1], word[p][2], word[p][3]);
        }
    }
    // the sums that this thread finishes: 8 columns, the same in every tile
    constexpr int OC = 4 * WN;                                     // chunks of 8 columns in a row of sums
    const int oc = t % OC;
    const int32_t on = n0 + 8 * oc;
    const int ocount = a.N - on;                                   // columns of it that exist (8 or more: all)
    float bias[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) bias[k] = MODE == FORWARD && a.bias && k < ocount ? a.bias[on + k] : 0.f;

    const bool grad = MODE == INPUT && r.act != KGE_ACT_IDENTITY;
    Chunks<!F32, CH> hx, hg;
    Chunks<!F32, 2 * RB> hr;
    auto load = [&](auto &h, int j, const T *p, int n) __attribute__((always_inline)) {
        if constexpr (F32) load8(p, n, h.x[j]);
        else h.q[j] = load8(p, n);
    };
    // a thread's chunks: the same one of every (NT / 2 KS)th row
    static_assert(NT % (2 * KS) == 0 && CH * NT == TR * KS * 2, "whole rows");
    const int tr = t / (2 * KS), tc = t % (2 * KS);
    const int tn = K - 8 * tc;
    const T *pa = a.A + (tile * TR + tr) * a.lda + 8 * tc, *pg = grad ? a.pre + (tile * TR + tr) * a.ldpre + 8 * tc : nullptr;
    const int64_t step_a = NT / (2 * KS) * a.lda, step_g = NT / (2 * KS) * a.ldpre;
    auto fetch = [&](int64_t ti) __attribute__((always_inline)) {
        if (K == 16 * KS && ti * TR + TR <= a.M) {
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                if constexpr (F32) load8(pa + j * step_a, hx.x[j]);
                else hx.q[j] = load8(pa + j * step_a);
            }
            if (grad) {
#pragma unroll
                for (int j = 0; j < CH; ++j) {
                    if constexpr (F32) load8(pg + j * step_g, hg.x[j]);
                    else hg.q[j] = load8(pg + j * step_g);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const int n = ti * TR + j * (NT / (2 * KS)) + tr < a.M ? tn : 0;
                load(hx, j, pa + j * step_a, n);
                if (grad) load(hg, j, pg + j * step_g, n);
            }
        }
        pa += r.lanes * TR * a.lda;
        if (grad) pg += r.lanes * TR * a.ldpre;
    };
    auto stage = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            unsigned char *at = smem + (j * (NT / (2 * KS)) + tr) * S::STRIDE + 16 * tc;
            if constexpr (P == 1) {
                uint4 q = hx.q[j];
                if (grad) {        // ReLU
                    const uint4 z = hg.q[j];
                    q = make_uint4(relu_pair(q.x, z.x), relu_pair(q.y, z.y), relu_pair(q.z, z.z), relu_pair(q.w, z.w));
                }
                *reinterpret_cast<uint4 *>(at) = q;
            } else {
                float x[8], z[8];
                if constexpr (F32) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) { x[k] = hx.x[j][k]; z[k] = hg.x[j][k]; }
                } else {
                    spread(hx.q[j], x);
                    spread(hg.q[j], z);
                }
                if (SOFT) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] *= act_grad<KGE_ACT_SILU>(z[k]);
                } else if (grad) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] *= act_grad<KGE_ACT_RELU>(z[k]);
                }
                to_lds<P>(x, at, S::PLANE);
            }
        }
    };

    if (tile < r.tiles) fetch(tile);
    for (; tile < r.tiles; tile += r.lanes) {
        stage();
        __syncthreads();
        const int64_t m0 = tile * TR;
        if (a.add) {
#pragma unroll
            for (int j = 0; j < 2 * RB; ++j) {
                const int64_t m = m0 + (j * NT + t) / OC;
                load(hr, j, a.add + m * a.ldadd + on, m < a.M ? ocount : 0);
            }
        }
        if (tile + r.lanes < r.tiles) fetch(tile + r.lanes);
        floatx16 acc[RB];
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][v] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            uint4 fa[P][RB];
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < RB; ++i)
                    fa[p][i] = *reinterpret_cast<const uint4 *>(smem + p * S::PLANE + (32 * (wm * RB + i) + (lane & 31)) * S::STRIDE +
                                                                32 * ks + 16 * (lane >> 5));
            // smallest products first; of three parts each, those of 2^-24 of the product and below are left out
#pragma unroll
            for (int s = P + PB - 2; s >= 0; --s) {
                if (P == 3 && PB == 3 && s > 2) continue;
#pragma unroll
                for (int pa = 0; pa < P; ++pa) {
                    const int pb = s - pa;
                    if (pb < 0 || pb >= PB) continue;
#pragma unroll
                    for (int i = 0; i < RB; ++i) acc[i] = split_mfma(fa[pa][i], fb[pb][ks], acc[i]);
                }
            }
        }
        __syncthreads();           // every wavefront is done with the rows
        float *const out = reinterpret_cast<float *>(smem);
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v)
                out[(32 * (wm * RB + i) + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3)) * S::OUT + 32 * wn + (lane & 31)] = acc[i][v];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 2 * RB; ++j) {
            const int row = (j * NT + t) / OC;
            const int64_t m = m0 + row;
            const float *from = out + row * S::OUT + 8 * oc;
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = from[k];
            if (m >= a.M || ocount <= 0) continue;
            if (P + PB > 2) {      // a sum that is not finite: once more from fp32 products, term by term
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (!split_not_finite(x[k]) || k >= ocount) continue;
                    float s = 0.f;
                    for (int32_t i = 0; i < K; ++i) {
                        float y = elem(a.A + m * a.lda + i);
                        if (grad) y *= act_grad(elem(a.pre + m * a.ldpre + i), r.act);
                        s = fmaf(y, elem(MODE == FORWARD ? a.B + (int64_t)i * a.ldb + on + k : a.B + (int64_t)(on + k) * a.ldb + i), s);
                    }
                    x[k] = s;
                }
            }
            if (MODE == FORWARD) {
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] += bias[k];
                if (a.pre_out) store8(a.pre_out + m * a.ldp + on, ocount, x);
                if (r.act == KGE_ACT_RELU) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = act_of<KGE_ACT_RELU>(x[k]);
                } else if (r.act == KGE_ACT_SILU) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = act_of<KGE_ACT_SILU>(x[k]);
                }
            }
            if (a.add) {
                float y[8];
                if constexpr (F32) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] = hr.x[j][k];
                } else spread(hr.q[j], y);
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] += y[k];
            }
            store8(a.C + m * a.ldc + on, ocount, x);
        }
        __syncthreads();           // the sums' place is the next rows'
    }
}

template <int MODE, class T, bool SOFT, int KS, int WN, int RB>
int launch_one(const Args<T> &a, int act, hipStream_t st)
{
    typedef Rows<MODE, T, SOFT, KS, WN, RB> S;
    RowArgs<T> r;
    r.a = a;
    r.act = act;
    r.groups = (int32_t)cdiv(a.N, 32 * WN);
    r.tiles = cdiv(a.M, S::TR);
    // one block of 8 wavefronts or two of 4 per compute unit, as registers and LDS allow
    const int64_t at_once = 256 * (S::NW == 8 || 2 * S::LDS > 160 * 1024 ? 1 : 2);
    r.lanes = (int64_t)align_up((size_t)cdiv(at_once, r.groups), 8);
    if (r.lanes > (int64_t)align_up((size_t)r.tiles, 8)) r.lanes = (int64_t)align_up((size_t)r.tiles, 8);
    auto kernel = k_dense_rows<MODE, T, SOFT, KS, WN, RB>;
    if (S::LDS > 64 * 1024) KGE_HIP(hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS));
    kernel<<<(unsigned)(r.lanes * r.groups), S::NT, S::LDS, st>>>(r);
    KGE_LAUNCH_CHECK();
    return KGE_OK;
}

template <int MODE, class T, bool SOFT, int KS, int RB>
int launch_columns(const Args<T> &a, int act, hipStream_t st)
{
    // the narrowest group that takes the columns; of wider results, groups of 256 unless groups of 128 leave fewer empty
    if (a.N <= 64) return launch_one<MODE, T, SOFT, KS, 2, 1>(a, act, st);
    if (cdiv(a.N, 128) * 128 < cdiv(a.N, 256) * 256) return launch_one<MODE, T, SOFT, KS, 4, RB>(a, act, st);
    return launch_one<MODE, T, SOFT, KS, 8, RB>(a, act, st);
}

template <int MODE, class T, bool SOFT>
int launch_terms(const Args<T> &a, int act, hipStream_t st)
{
    if (a.K <= 64) return launch_columns<MODE, T, SOFT, 4, 2>(a, act, st);
    // fp32, B in registers: 12 a step of 16 terms, 96 of them at 128 terms.  156 for 208 terms left too few: the next tile's rows went to
    // scratch memory, and 14541 rows of 203 took 95 us where the tiled kernel took 55
    if constexpr (sizeof(T) == 4) return launch_columns<MODE, T, SOFT, 8, MODE == INPUT ? 1 : 2>(a, act, st);
    else {
        if (a.K <= 128) return launch_columns<MODE, T, SOFT, 8, 2>(a, act, st);
        return launch_columns<MODE, T, SOFT, 16, 2>(a, act, st);
    }
}

}  // namespace

namespace dense {

template <int MODE, class T>
int launch_rows(const Args<T> &a, int act, hipStream_t st)
{
    if constexpr (MODE == INPUT) {
        if (act == KGE_ACT_SILU) return launch_terms<MODE, T, true>(a, act, st);
    }
    return launch_terms<MODE, T, false>(a, act, st);
}
template int launch_rows<FORWARD, float>(const Args<float> &, int, hipStream_t);
template int launch_rows<FORWARD, uint16_t>(const Args<uint16_t> &, int, hipStream_t);
template int launch_rows<INPUT, float>(const Args<float> &, int, hipStream_t);
template int launch_rows<INPUT, uint16_t>(const Args<uint16_t> &, int, hipStream_t);

}  // namespace dense
