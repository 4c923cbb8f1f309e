// Dense layer, forward product and input gradient, for long matrices of narrow rows: C = A B with B held in registers.
//
// A layer of 128 or 256 columns reads and writes a row or two for every row of products, so the rows set the time and the
// matrix cores have time to spare.  A block stays: each of its wavefronts loads the B operands of its 32 columns once, all
// K terms of them (and splits them once, fp32), and then tiles of rows stream by.  While one tile is multiplied, the next
// goes from registers to LDS as bf16 parts, dY becoming dP, and the one after that is on its way to registers, so that
// loads are in flight all the time; every wavefront reads all of a tile.  Of the two wavefronts that share a SIMD (blocks of
// eight) one stages while the other multiplies.  The sums pass through LDS, so that bias, activation, residual and
// stores work on 16 to 32 consecutive bytes per lane.
//
// Loads and stores of a wavefront finish in order, and a wait names how many may be left.  The compiler can count them only
// where no branch decides whether one is issued, so a tile that is all there goes through a loop without such branches: what is
// optional (R or `add`, pre) is a template argument, and the lanes whose columns lie past the result store through a buffer
// descriptor that drops them.  With branches in the loop it waited for everything, stores included: a million rows of 256
// bf16 numbers, input gradient with SiLU, took 546 us, and 465 so.  Measured: 2.9 million fp32 rows of 128 to 128 with R = X and pre
// 900 us, 4.9 TB/s (1134 us with branches and R read again); a million bf16 rows of 256 to 256 with pre 307 us, 5.0 TB/s.
//
// LDS rows are 16 bytes longer than their terms: an odd number of 16-byte chunks apart, eight rows meet all banks.
// Blocks of the several column groups of a wide result run on one XCD in step, so that the rows come from HBM once.
#pragma once
#include "dense.h"

namespace dense {

template <class T>
struct RowArgs {
    Args<T> a;
    int32_t act, groups;           // column groups
    int32_t counted;               // whole tiles may go through the loop without branches
    int64_t lanes, tiles, whole;   // blocks per group (a multiple of 8), row tiles, those that are all there
};

enum { ADD_NONE = 0, ADD_ROWS = 1, ADD_SELF = 2 };      // nothing; rows of their own; R is X: its rows are in LDS already

// KS: steps of 16 terms; WN: wavefronts side by side, 32 columns each
template <int MODE, class T, int ACT, int KS, int WN>
struct Rows {
    static constexpr bool F32 = sizeof(T) == 4, SOFT = !F32 && MODE == INPUT && ACT == KGE_ACT_SILU;
    static constexpr int P = F32 ? 3 : SOFT ? 2 : 1, PB = F32 ? 3 : 1;
    static constexpr int NT = 64 * WN, TR = 32;
    static constexpr int STRIDE = KS * 32 + 16, PLANE = TR * STRIDE, BUFFER = P * PLANE;
    static constexpr int OUT = 32 * WN + 8;                        // floats per row of sums: 4 rows further, 32 banks further
    static constexpr int CH = TR * KS * 2 / NT;                    // chunks of 8 terms per thread and tile
    static constexpr int LDS = 2 * BUFFER + TR * OUT * 4;
    static_assert(NT % (2 * KS) == 0 && CH * NT == TR * KS * 2, "a thread's chunks are the same one of several rows");
};

template <bool F32, int CH>
struct Chunks {
    uint4 q[F32 ? 1 : CH];
    float x[F32 ? CH : 1][8];
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// the first 8 bytes x sizeof(T) of a row's chunk, `at` bytes behind the descriptor's address
__device__ __forceinline__ void store_counted(__amdgpu_buffer_rsrc_t to, uint32_t at, const float x[8], const float *)
{
    const u32x4 lo = {__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    const u32x4 hi = {__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7])};
    __builtin_amdgcn_raw_buffer_store_b128(lo, to, at, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b128(hi, to, at + 16u, 0, 0);
}
__device__ __forceinline__ void store_counted(__amdgpu_buffer_rsrc_t to, uint32_t at, const float x[8], const uint16_t *)
{
    const u32x4 q = {split_round(x[0], x[1]), split_round(x[2], x[3]), split_round(x[4], x[5]), split_round(x[6], x[7])};
    __builtin_amdgcn_raw_buffer_store_b128(q, to, at, 0, 0);
}
constexpr uint32_t NOWHERE = 0x80000000u;      // past every descriptor's end, and still so with 16 bytes more

// ACT: INPUT's; a FORWARD's is a number in the arguments (no access to memory depends on it)
template <int MODE, class T, int ACT, int KS, int WN, int ADD, bool PRE>
__global__ __launch_bounds__(64 * WN, 2) void k_dense_rows(RowArgs<T> r)
{
    typedef Rows<MODE, T, ACT, KS, WN> S;
    constexpr int P = S::P, PB = S::PB, NT = S::NT, TR = S::TR, CH = S::CH;
    constexpr bool F32 = S::F32, GRAD = MODE == INPUT && ACT != KGE_ACT_IDENTITY;
    const Args<T> &a = r.a;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];

    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
    // workgroup i runs on XCD i % 8: a row tile's column groups are neighbours there
    const int64_t seq = blockIdx.x >> 3;
    const int32_t n0 = (int32_t)(seq % r.groups) * 32 * WN;
    int64_t tile = (seq / r.groups) * 8 + (blockIdx.x & 7);
    const int32_t K = (int32_t)a.K;
    if (tile >= r.tiles) return;   // uniform over the block

    // B operand: column lane % 32 of the wavefront's 32, terms 16 ks + 8 (lane / 32) ..
    uint4 fb[PB][KS];
    {
        const int32_t n = n0 + 32 * w + (lane & 31);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int32_t k = 16 * ks + 8 * (lane >> 5);
            float x[8];
            if (MODE == FORWARD) {                                 // columns side by side: places past the end read the last one's
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float y = elem(a.B + (int64_t)min(k + i, K - 1) * a.ldb + min(n, a.N - 1));
                    x[i] = n < a.N && k + i < K ? y : 0.f;
                }
            } else if constexpr (F32) load8(a.B + (int64_t)min(n, a.N - 1) * a.ldb + k, n < a.N ? K - k : 0, x);
            else spread(load8(a.B + (int64_t)min(n, a.N - 1) * a.ldb + k, n < a.N ? K - k : 0), x);
            uint32_t word[3][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Split3 s = split_pair(x[2 * i], x[2 * i + 1]);
#pragma unroll
                for (int p = 0; p < PB; ++p) word[p][i] = s.w[p];
            }
#pragma unroll
            for (int p = 0; p < PB; ++p) fb[p][ks] = make_uint4(word[p][0], word[p][1], word[p][2], word[p][3]);
            if (ks % 4 == 3) __builtin_amdgcn_sched_barrier(0);    // loads of four steps in flight, not of all
        }
    }
    // the sums that this thread finishes: 8 columns of two rows
    constexpr int OC = 4 * WN;                                     // chunks of 8 columns in a row of sums
    static_assert(2 * NT == TR * OC, "two chunks a thread");
    const int oc = t % OC, orow = t / OC;
    const int32_t on = n0 + 8 * oc;
    const int ocount = a.N - on;                                   // columns of it that exist (8 or more: all)
    float bias[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) bias[k] = MODE == FORWARD && a.bias && k < ocount ? a.bias[on + k] : 0.f;

    Chunks<F32, CH> hx, hg;
    Chunks<F32, 2> hr;
    const int tr = t / (2 * KS), tc = t % (2 * KS);
    constexpr int RS = NT / (2 * KS);                              // rows between a thread's chunks
    const int tn = K - 8 * tc;                                     // terms of its chunks that exist
    const int tc_in = tn > 0 ? tc : 0;                             // without branches: an empty chunk reads the row's first ..
    const uint32_t keep = tn > 0 ? 0xffffffffu : 0u;               // .. and takes nothing of it
    const T *pa = a.A + (tile * TR + tr) * a.lda + 8 * tc_in, *pg = GRAD ? a.pre + (tile * TR + tr) * a.ldpre + 8 * tc_in : nullptr;
    const T *pr = ADD == ADD_ROWS ? a.add + (tile * TR + orow) * a.ldadd + (ocount > 0 ? on : 0) : nullptr;

    auto load = [&](auto &h, int j, const T *p) __attribute__((always_inline)) {
        if constexpr (F32) load8(p, h.x[j]);
        else h.q[j] = load8(p);
    };
    auto load_some = [&](auto &h, int j, const T *p, int n) __attribute__((always_inline)) {
        if constexpr (F32) load8(p, n, h.x[j]);
        else h.q[j] = load8(p, n);
    };
    auto fetch = [&](int64_t ti, auto counted) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            if constexpr (decltype(counted)::value) {
                load(hx, j, pa + j * RS * a.lda);
                if (GRAD) load(hg, j, pg + j * RS * a.ldpre);
            } else {
                const int n = ti * TR + j * RS + tr < a.M ? tn : 0;
                load_some(hx, j, pa + j * RS * a.lda, n);
                if (GRAD) load_some(hg, j, pg + j * RS * a.ldpre, n);
            }
        }
        pa += r.lanes * TR * a.lda;
        if (GRAD) pg += r.lanes * TR * a.ldpre;
    };
    auto stage = [&](unsigned char *rows) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            unsigned char *at = rows + (j * RS + tr) * S::STRIDE + 16 * tc;
            if constexpr (P == 1) {
                uint4 q = hx.q[j];
                q.x &= keep; q.y &= keep; q.z &= keep; q.w &= keep;
                if (GRAD) {        // ReLU
                    const uint4 z = hg.q[j];
                    q = make_uint4(relu_pair(q.x, z.x), relu_pair(q.y, z.y), relu_pair(q.z, z.z), relu_pair(q.w, z.w));
                }
                *reinterpret_cast<uint4 *>(at) = q;
            } else {
                float x[8], z[8];
                if constexpr (F32) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) { x[k] = __uint_as_float(__float_as_uint(hx.x[j][k]) & keep); z[k] = GRAD ? hg.x[j][k] : 0.f; }
                } else {
                    uint4 q = hx.q[j];
                    q.x &= keep; q.y &= keep; q.z &= keep; q.w &= keep;
                    spread(q, x);
                    spread(hg.q[j], z);
                }
                if (GRAD) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        x[k] = through_act<ACT>(x[k], z[k]);
                        if (ACT == KGE_ACT_SILU) x[k] = __uint_as_float(__float_as_uint(x[k]) & keep);      // 0 times the pre of a row's first chunk
                    }
                }
                to_lds<P>(x, at, S::PLANE);
            }
        }
    };

    // two sums, of even and odd steps: a product need not wait for the one before it
    floatx16 acc[2];
    auto multiply = [&](const unsigned char *rows) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][v] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            uint4 fa[P];
#pragma unroll
            for (int p = 0; p < P; ++p)
                fa[p] = *reinterpret_cast<const uint4 *>(rows + p * S::PLANE + (lane & 31) * S::STRIDE + 32 * ks + 16 * (lane >> 5));
            // smallest products first; of three parts each, those of 2^-24 of the product and below are left out
#pragma unroll
            for (int s = P + PB - 2; s >= 0; --s) {
                if (P == 3 && PB == 3 && s > 2) continue;
#pragma unroll
                for (int pa = 0; pa < P; ++pa) {
                    const int pb = s - pa;
                    if (pb < 0 || pb >= PB) continue;
                    acc[ks & 1] = split_mfma(fa[pa], fb[pb][ks], acc[ks & 1]);
                }
            }
        }
    };

    float *const out = reinterpret_cast<float *>(smem + 2 * S::BUFFER);
    const bool late = WN == 8 && w >= 4;         // wavefronts i and i + 4 share a SIMD
    int side = 0;
    auto step = [&](auto counted) __attribute__((always_inline)) {
        constexpr bool COUNTED = decltype(counted)::value;
        const int64_t m0 = tile * TR;
        const unsigned char *const rows = smem + side * S::BUFFER;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if constexpr (ADD == ADD_ROWS) {
                const T *p = pr + j * (TR / 2) * a.ldadd;
                if constexpr (COUNTED) load(hr, j, p);
                else load_some(hr, j, p, m0 + j * (TR / 2) + orow < a.M ? ocount : 0);
            } else if constexpr (ADD == ADD_SELF) {
                // the parts of a finite number add up to it exactly
                const unsigned char *p = rows + (j * (TR / 2) + orow) * S::STRIDE + (ocount > 0 ? 2 * on : 0);
                if constexpr (F32) {
                    float y[3][8];
#pragma unroll
                    for (int q = 0; q < 3; ++q) spread(*reinterpret_cast<const uint4 *>(p + q * S::PLANE), y[q]);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        hr.x[j][k] = y[0][k] + (y[1][k] + y[2][k]);
                        if (split_not_finite(hr.x[j][k]) && m0 + j * (TR / 2) + orow < a.M && k < ocount)
                            hr.x[j][k] = elem(a.A + (m0 + j * (TR / 2) + orow) * a.lda + on + k);
                    }
                } else hr.q[j] = *reinterpret_cast<const uint4 *>(p);
            }
        }
        if (ADD == ADD_ROWS) pr += r.lanes * TR * a.ldadd;
        if (late) multiply(rows);
        unsigned char *const other = smem + (side ^ 1) * S::BUFFER;      // last read a barrier ago
        if constexpr (COUNTED) {
            stage(other);
            fetch(tile + 2 * r.lanes, counted);
        } else {
            if (tile + r.lanes < r.tiles) stage(other);
            if (tile + 2 * r.lanes < r.tiles) fetch(tile + 2 * r.lanes, counted);
        }
        if (!late) multiply(rows);
        __syncthreads();           // the next tile is there, and the last one's sums are out of `out`
#pragma unroll
        for (int v = 0; v < 16; ++v) out[(8 * (v >> 2) + 4 * (lane >> 5) + (v & 3)) * S::OUT + 32 * w + (lane & 31)] = acc[0][v] + acc[1][v];
        __syncthreads();
        // raw descriptors of this tile's rows, of which lanes past the last column store nothing (counted steps)
        const __amdgpu_buffer_rsrc_t to_c = __builtin_amdgcn_make_buffer_rsrc(a.C + m0 * a.ldc, 0, (int)(TR * a.ldc * sizeof(T)), 0x00020000);
        const __amdgpu_buffer_rsrc_t to_p =
            __builtin_amdgcn_make_buffer_rsrc(PRE ? a.pre_out + m0 * a.ldp : a.C, 0, (int)(PRE ? TR * a.ldp * sizeof(T) : 0), 0x00020000);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int row = j * (TR / 2) + orow;
            const int64_t m = m0 + row;
            float *from = out + row * S::OUT + 8 * oc;
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = from[k];
            if (P + PB > 2) {      // a sum that is not finite: once more from fp32 products, term by term
                bool bad = false;
#pragma unroll
                for (int k = 0; k < 8; ++k) bad |= split_not_finite(x[k]);
                if (bad && m < a.M) {
                    for (int k = 0; k < 8 && k < ocount; ++k) {
                        if (!split_not_finite(from[k])) continue;
                        float s = 0.f;
                        for (int32_t i = 0; i < K; ++i) {
                            float y = elem(a.A + m * a.lda + i);
                            if (GRAD) y = through_act<ACT>(y, elem(a.pre + m * a.ldpre + i));
                            s = fmaf(y, elem(MODE == FORWARD ? a.B + (int64_t)i * a.ldb + on + k : a.B + (int64_t)(on + k) * a.ldb + i), s);
                            if (s != s) break;     // a NaN stays one: of inputs that are all NaN one term is read
                        }
                        from[k] = s;
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = from[k];
                }
            }
            const bool some = COUNTED || (m < a.M && ocount > 0);
            if (MODE == FORWARD) {
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] += bias[k];
                if constexpr (PRE) {
                    if constexpr (COUNTED) store_counted(to_p, ocount > 0 ? (uint32_t)((row * a.ldp + on) * sizeof(T)) : NOWHERE, x, a.pre_out);
                    else if (some) store8(a.pre_out + m * a.ldp + on, ocount, x);
                }
                if (r.act == KGE_ACT_RELU) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = act_of<KGE_ACT_RELU>(x[k]);
                } else if (r.act == KGE_ACT_SILU) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = act_of<KGE_ACT_SILU>(x[k]);
                }
            }
            if constexpr (ADD != ADD_NONE) {
                float y[8];
                if constexpr (F32) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] = hr.x[j][k];
                } else spread(hr.q[j], y);
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] += y[k];
            }
            if constexpr (COUNTED) store_counted(to_c, ocount > 0 ? (uint32_t)((row * a.ldc + on) * sizeof(T)) : NOWHERE, x, a.C);
            else if (some) store8(a.C + m * a.ldc + on, ocount, x);
        }
        tile += r.lanes;
        side ^= 1;
    };

    const std::true_type counted{};
    const std::false_type guarded{};
    fetch(tile, guarded);
    stage(smem);
    if (tile + r.lanes < r.tiles) fetch(tile + r.lanes, guarded);
    __syncthreads();
    if (r.counted)
        while (tile + 2 * r.lanes < r.whole) step(counted);
    while (tile < r.tiles) step(guarded);
}

template <int MODE, class T, int ACT, int KS, int WN, int ADD, bool PRE>
int launch_one(const Args<T> &a, int act, hipStream_t st)
{
    typedef Rows<MODE, T, ACT, KS, WN> S;
    RowArgs<T> r;
    r.a = a;
    r.act = act;
    r.groups = (int32_t)cdiv(a.N, 32 * WN);
    r.tiles = cdiv(a.M, S::TR);
    r.whole = a.M / S::TR;
    r.counted = rows_counted(a);
    // one block of 8 wavefronts or two of 4 per compute unit, as LDS allows
    const int64_t at_once = WN == 8 || 2 * S::LDS > 160 * 1024 ? 256 : 512;
    static_assert(S::LDS <= 160 * 1024, "LDS of a compute unit");
    // The groups of a row tile are on one XCD, and no XCD has more blocks than run there at once: with one more, three groups of 400000
    // rows of 128 terms took 992 us in place of 700 (768 columns fp32), 493 in place of 332 (bf16)
    r.lanes = r.groups < at_once / 8 ? 8 * (at_once / 8 / r.groups) : 8;
    if (r.lanes > (int64_t)align_up((size_t)r.tiles, 8)) r.lanes = (int64_t)align_up((size_t)r.tiles, 8);
    auto kernel = k_dense_rows<MODE, T, ACT, KS, WN, ADD, PRE>;
    if (S::LDS > 64 * 1024) KGE_HIP(hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS));
    kernel<<<(unsigned)(r.lanes * r.groups), S::NT, S::LDS, st>>>(r);
    KGE_LAUNCH_CHECK();
    return KGE_OK;
}

template <int MODE, class T, int ACT, int KS, int WN>
int launch_options(const Args<T> &a, int act, hipStream_t st)
{
    if constexpr (MODE == INPUT) {
        if (a.add) return launch_one<MODE, T, ACT, KS, WN, ADD_ROWS, false>(a, act, st);
        return launch_one<MODE, T, ACT, KS, WN, ADD_NONE, false>(a, act, st);
    } else {
        // R = X as it lies: its chunks are those that are staged
        const bool self = a.add == a.A && a.ldadd == a.lda && a.N == a.K && a.K % 8 == 0;
        if (a.pre_out) {
            if (self) return launch_one<MODE, T, ACT, KS, WN, ADD_SELF, true>(a, act, st);
            if (a.add) return launch_one<MODE, T, ACT, KS, WN, ADD_ROWS, true>(a, act, st);
            return launch_one<MODE, T, ACT, KS, WN, ADD_NONE, true>(a, act, st);
        }
        if (self) return launch_one<MODE, T, ACT, KS, WN, ADD_SELF, false>(a, act, st);
        if (a.add) return launch_one<MODE, T, ACT, KS, WN, ADD_ROWS, false>(a, act, st);
        return launch_one<MODE, T, ACT, KS, WN, ADD_NONE, false>(a, act, st);
    }
}

template <int MODE, class T, int ACT>
int launch_shape(const Args<T> &a, int act, hipStream_t st)
{
    // groups of 256 columns unless groups of 128 leave fewer empty
    const bool wide = cdiv(a.N, 128) * 128 >= cdiv(a.N, 256) * 256;
    // fp32, B in registers: 12 a step of 16 terms, 96 of them at 128 terms; 156 for 208 terms left too few for the rows on their way
    if constexpr (sizeof(T) == 2) {
        if (a.K > 128) return wide ? launch_options<MODE, T, ACT, 16, 8>(a, act, st) : launch_options<MODE, T, ACT, 16, 4>(a, act, st);
    }
    return wide ? launch_options<MODE, T, ACT, 8, 8>(a, act, st) : launch_options<MODE, T, ACT, 8, 4>(a, act, st);
}

}  // namespace dense
