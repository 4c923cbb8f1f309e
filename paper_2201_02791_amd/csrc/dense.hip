// Dense layer on the rows of a feature matrix, with everything around the product in its epilogue, and its backward pass.
//
//   forward    pre = X W + b;  Y = act(pre) + R
//   backward   dP = dY * act'(pre);  dX = dP W^T + add;  dW = X^T dP;  db = sum over rows of dP
//
// One kernel for the three products C[i][j] = sum_k A[i][k] B[k][j]; they differ in how an operand lies in memory:
//
//   forward     A = X: terms k side by side          B = W: columns j side by side
//   input       A = dP: terms side by side           B = W^T: terms side by side
//   weights     A = X^T: columns i side by side      B = dP: columns side by side       (terms: the rows of X)
//
// A block has a tile of results: 128 x 128 on four wavefronts, 64 x 64 each on v_mfma_f32_32x32x16_bf16; 64 x 128 where 128 x 128 would
// leave compute units with one or two (fp32 forward and input gradient); 128 x 32 for the last columns of those where few are left; and
// for the weights' gradient what its narrow side fits, 128 x 32, 128 x 64, 32 x 128, or 256 x 128 on eight wavefronts (wide bf16 ones).
// Operands reach LDS through registers, where they become bf16 and where dY turns into dP: act' is never stored, and the next terms are
// loaded while some are multiplied; the 256 x 128 tile has two buffers and stages one while it multiplies the other.  An operand whose
// terms lie side by side is read back with ds_read_b128 from rows of terms, one whose columns do with the transposing ds_read_b64_tr_b16
// from rows of columns; the chunks of 16 bytes of a row are XOR-ed with its number so that neither meets a bank twice.
//
// fp32 numbers become three bf16 parts and six products (split_bf16.h): 417 TFLOP/s where the fp32 instruction has 157.
// bf16 numbers enter as they are, and so does dP of bf16 rows under identity and ReLU; under SiLU dP is an fp32 number:
// two parts (2^-17) where the result is rounded to bf16, three where it is a weights' gradient in fp32.  Sums that are
// not finite come again from fp32 products: infinities do not survive a split.  Of the nine products of three parts the three below
// 2^-24 of the product are left out: dW of 290001 x 128 x 32, numbers of spread one, is 7.8e-7 of its root mean square off (the
// library's fp32 product 2.9e-6).
//
// What bounds it: fp32, the matrix cores and the splitting beside them (128000 x 1000 x 1000 forward 1575 us, 975 TFLOP/s of bf16
// products, 163 of fp32; the library's fp32 product alone does 153); bf16, the operands' way through LDS, a read of 1 KB per instruction
// of 32 cycles (64000 x 1024 x 1024: 203 us, 662 TFLOP/s; the library does 1205 at 8192 x 8192 x 8192 without bias or activation); with
// SiLU, a wide layer's backward pass is bound by act', formed again for every 128 columns of the result (404 us in place of 181).
//
// The weights' gradient sums over as many rows as there are: they are cut into chunks so that about as many blocks run as
// the chip holds, each writes its sums to the workspace and a second launch adds them in a fixed order.
#include "dense.h"

#include <algorithm>

using namespace dense;

namespace {

// what a thread holds of an operand's next tile: chunks of 8 elements as they lie in memory
template <bool F32, int CH>
struct Held {
    uint4 q[F32 ? 1 : CH];
    float x[F32 ? CH : 1][8];
};

// A block's tile of BM x BN results, WM x WN wavefronts, (BM / WM) x (BN / WN) each
template <int MODE, class T, int ACT, int BM, int BN, int WM, int WN>
struct Shape {
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr bool SOFT = !F32 && ACT == KGE_ACT_SILU;          // dP of bf16 rows that is no bf16 number
    static constexpr int PA = F32 ? 3 : MODE == INPUT && SOFT ? 2 : 1;
    static constexpr int PB = F32 ? 3 : MODE == WEIGHTS && SOFT ? 3 : 1;
    static constexpr bool ROWA = MODE != WEIGHTS, ROWB = MODE == INPUT;    // terms side by side
    static constexpr int NT = 64 * WM * WN, MI = BM / 32 / WM, NJ = BN / 32 / WN;
    static constexpr int BK = (PA + PB > 2 && (MODE != WEIGHTS || (BM > 32 && BN > 32))) || BM == 256 ? 32 : 64;
    static constexpr int ALLA = BM * BK / 8, ALLB = BN * BK / 8;         // chunks of 8; with fewer than threads, several hold the same one
    static constexpr int CHA = ALLA / NT, CHB = ALLB < NT ? 1 : ALLB / NT;
    static constexpr int PLANEA = BM * BK * 2, PLANEB = BN * BK * 2;
    static constexpr int BUFFER = PA * PLANEA + PB * PLANEB;
    // a block that has its compute unit to itself stages one tile while it multiplies another
    static constexpr bool TWO = BM == 256;
    // per SIMD: 168 registers, so that three blocks share a compute unit where one of fp32 numbers alone would leave it for two
    static constexpr int WAVES = F32 && MODE != WEIGHTS ? (BM == 64 ? 4 : MODE == FORWARD ? 3 : 2) : 1;
    static constexpr int OUT = 32 * NJ + 8;                            // floats per row of results in LDS: 4 rows further, 32 banks further
    static constexpr int TILES = (TWO ? 2 : 1) * BUFFER, RESULTS = WM * WN * 32 * OUT * 4;
    static constexpr int LDS = TILES > RESULTS ? TILES : RESULTS;
    static_assert(CHA * NT == ALLA && (CHB * NT == ALLB || (MODE != WEIGHTS && NT % ALLB == 0)), "whole chunks");
    static_assert(LDS >= NT * 32, "the columns' sums");
};

// The place of chunk (r, c) of a tile: rows of BK terms (a row is 64 or 128 bytes), or rows of W columns, whose blocks of 64
// bytes are what a transposing read takes from four rows at a time
template <int BK>
__device__ __forceinline__ int term_place(int r, int c)
{
    constexpr int PER = BK / 8;
    return r * (2 * BK) + ((c ^ (PER == 4 ? (r >> 1) & 3 : r & 7)) << 4);
}
template <int W>
__device__ __forceinline__ int column_swap(int k) { return W >= 128 ? k & 3 : W == 64 ? (k >> 1) & 1 : 0; }
template <int W>
__device__ __forceinline__ int column_place(int k, int c) { return k * (2 * W) + ((c ^ (4 * column_swap<W>(k))) << 4); }

// the tile at row m0 and column n0 of the result, its terms those of a chunk
template <int MODE, class T, int ACT, int BM, int BN, int WM, int WN>
__device__ __forceinline__ void tile_at(const Args<T> &a, int64_t m0, int32_t n0, int64_t chunk, unsigned char *smem)
{
    typedef Shape<MODE, T, ACT, BM, BN, WM, WN> S;
    constexpr int BK = S::BK, PA = S::PA, PB = S::PB, NT = S::NT, MI = S::MI, NJ = S::NJ;
    const int64_t k_beg = chunk * a.chunk, k_end = min(k_beg + a.chunk, a.K);
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), wm = w / WN, wn = w % WN;
    const int tb = S::ALLB < NT ? t % S::ALLB : t;

    struct Set {
        Held<S::F32, S::CHA> a, p;
        Held<S::F32, S::CHB> b, q; // p, q: pre of the operand that is dP
    };
    Set set;
    constexpr bool GRAD = MODE != FORWARD && ACT != KGE_ACT_IDENTITY;

    // chunk j of this thread in a tile of terms: row (j NT + t) / (BK / 8); of W columns: term (j NT + t) / (W / 8).  The chunk
    // in the row is the same for every j
    constexpr int TC = BK / 8, AC = BM / 8, BC = BN / 8;
    static_assert(NT % TC == 0 && NT % AC == 0 && NT % BC == 0, "one chunk of a row per thread");
    // Where this thread's chunks lie when k0 = k_beg, and how far apart the tiles are.  Rows and columns past the result's read the
    // last row or the first chunk in their place: what they add up to is not stored.  Only terms past the end have to be zeros.
    struct Walk { const T *p[(S::CHA > S::CHB ? S::CHA : S::CHB)]; int64_t tile; };
    auto walk = [&](int t, const T *base, int64_t ld, auto terms, auto per, auto chunks, int64_t outer0, int64_t outer_n) __attribute__((always_inline)) -> Walk {
        constexpr int PER = decltype(per)::value;
        Walk x;
#pragma unroll
        for (int j = 0; j < decltype(chunks)::value; ++j) {
            const int r = (j * NT + t) / PER, c = t % PER;
            if constexpr (decltype(terms)::value) x.p[j] = base + min(outer0 + r, outer_n - 1) * ld + k_beg + 8 * c;
            else x.p[j] = base + (k_beg + r) * ld + (outer0 + 8 * c < outer_n ? outer0 + 8 * c : 0);
        }
        x.tile = decltype(terms)::value ? BK : BK * ld;
        return x;
    };
    const std::integral_constant<bool, S::ROWA> ra{};
    const std::integral_constant<bool, S::ROWB> rb{};
    const std::integral_constant<int, S::ROWA ? TC : AC> ca{};
    const std::integral_constant<int, S::ROWB ? TC : BC> cb{};
    const std::integral_constant<int, S::CHA> na{};
    const std::integral_constant<int, S::CHB> nb{};
    Walk wa = walk(t, a.A, a.lda, ra, ca, na, m0, a.M), wb = walk(tb, a.B, a.ldb, rb, cb, nb, n0, a.N), wp{};
    if constexpr (GRAD) wp = MODE == INPUT ? walk(t, a.pre, a.ldpre, ra, ca, na, m0, a.M) : walk(tb, a.pre, a.ldpre, rb, cb, nb, n0, a.N);
    // Tiles up to here load whole chunks: their terms all exist, and a chunk that the end of a row of columns cuts reads on into the
    // next row, which the last one (the last eight, should they be narrower than a chunk) does not have
    const bool cut = (!S::ROWA && a.M % 8 != 0) || (!S::ROWB && a.N % 8 != 0);
    const int64_t k_whole = min(k_end, cut ? a.K - 8 : a.K) - BK;

    auto fetch = [&](Set &h, int64_t k0, auto counted) __attribute__((always_inline)) {
        auto one = [&](int t, auto &h, int j, const Walk &x, auto terms, auto per, int64_t outer0, int64_t outer_n, auto whole) __attribute__((always_inline)) {
            constexpr int PER = decltype(per)::value;
            if constexpr (decltype(whole)::value) {
                if constexpr (S::F32) load8(x.p[j], h.x[j]);
                else h.q[j] = load8(x.p[j]);
            } else {
                const int left = (int)min((int64_t)BK, k_end - k0);
                const int r = (j * NT + t) / PER, c = t % PER;
                int n;
                if constexpr (decltype(terms)::value) n = outer0 + r < outer_n ? left - 8 * c : 0;
                else n = r < left ? (int)max((int64_t)0, min((int64_t)8, outer_n - outer0 - 8 * c)) : 0;
                if constexpr (S::F32) load8(x.p[j], n, h.x[j]);
                else h.q[j] = load8(x.p[j], n);
            }
        };
        auto all = [&](auto whole) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < S::CHA; ++j) {
                one(t, h.a, j, wa, ra, ca, m0, a.M, whole);
                if constexpr (MODE == INPUT && GRAD) one(t, h.p, j, wp, ra, ca, m0, a.M, whole);
            }
#pragma unroll
            for (int j = 0; j < S::CHB; ++j) {
                one(tb, h.b, j, wb, rb, cb, n0, a.N, whole);
                if constexpr (MODE == WEIGHTS && GRAD) one(tb, h.q, j, wp, rb, cb, n0, a.N, whole);
            }
        };
        if constexpr (decltype(counted)::value) all(std::true_type());
        else if (k0 <= k_whole) all(std::true_type());
        else all(std::false_type());
#pragma unroll
        for (int j = 0; j < S::CHA; ++j) {
            wa.p[j] += wa.tile;
            if constexpr (MODE == INPUT && GRAD) wp.p[j] += wp.tile;
        }
#pragma unroll
        for (int j = 0; j < S::CHB; ++j) {
            wb.p[j] += wb.tile;
            if constexpr (MODE == WEIGHTS && GRAD) wp.p[j] += wp.tile;
        }
    };

    floatx16 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    float col[8];                  // WEIGHTS: sums of dP over this thread's rows, its 8 columns
#pragma unroll
    for (int k = 0; k < 8; ++k) col[k] = 0.f;
    const bool sum_columns = MODE == WEIGHTS && a.part_b && m0 == 0;

    // registers -> LDS, dY -> dP on the way
    auto stage = [&](const Set &set, unsigned char *la) __attribute__((always_inline)) {
        unsigned char *const lb = la + PA * S::PLANEA;
        auto one = [&](int t, const auto &h, const auto &hg, int j, unsigned char *lds, auto terms, auto per, auto parts, int plane, auto grad,
                       bool columns) __attribute__((always_inline)) {
            constexpr int PER = decltype(per)::value, P = decltype(parts)::value;
            const int r = (j * NT + t) / PER, c = t % PER;
            unsigned char *at = lds;
            if constexpr (decltype(terms)::value) at += term_place<BK>(r, c);
            else at += column_place<PER * 8>(r, c);
            if constexpr (P == 1) {
                uint4 q = h.q[j];
                if constexpr (decltype(grad)::value) {   // ReLU
                    const uint4 z = hg.q[j];
                    q = make_uint4(relu_pair(q.x, z.x), relu_pair(q.y, z.y), relu_pair(q.z, z.z), relu_pair(q.w, z.w));
                }
                *reinterpret_cast<uint4 *>(at) = q;
                if (columns) {
                    float x[8];
                    spread(q, x);
#pragma unroll
                    for (int k = 0; k < 8; ++k) col[k] += x[k];
                }
            } else {
                float x[8], z[8];
                if constexpr (S::F32) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = h.x[j][k];
                } else spread(h.q[j], x);
                if constexpr (decltype(grad)::value) {
                    if constexpr (S::F32) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) z[k] = hg.x[j][k];
                    } else spread(hg.q[j], z);
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = through_act<ACT>(x[k], z[k]);
                }
                to_lds<P>(x, at, plane);
                if (columns)
#pragma unroll
                    for (int k = 0; k < 8; ++k) col[k] += x[k];
            }
        };
#pragma unroll
        for (int j = 0; j < S::CHA; ++j)
            one(t, set.a, set.p, j, la, ra, ca, std::integral_constant<int, PA>(), S::PLANEA, std::integral_constant<bool, MODE == INPUT && GRAD>(), false);
#pragma unroll
        for (int j = 0; j < S::CHB; ++j)
            one(tb, set.b, set.q, j, lb, rb, cb, std::integral_constant<int, PB>(), S::PLANEB, std::integral_constant<bool, MODE == WEIGHTS && GRAD>(),
                sum_columns);
    };

    // operand of the matrix instruction: row (or column) lane % 32 of block `blk` of 32, terms ks + 8 (lane / 32) ..
    const int l16 = lane & 15, kr0 = 8 * (lane >> 5) + (l16 >> 2);
    const int lc = (16 * ((lane >> 4) & 1) + 4 * (l16 & 3)) * 2;
    auto frag = [&](const unsigned char *lds, auto terms, auto width, int blk, int ks) __attribute__((always_inline)) -> uint4 {
        if constexpr (decltype(terms)::value)
            return *reinterpret_cast<const uint4 *>(lds + term_place<BK>(32 * blk + (lane & 31), ks / 8 + (lane >> 5)));
        else {
            constexpr int W = decltype(width)::value;
            // rows kr0 and kr0 + 4 of a step, and those of later steps, are swapped alike
            const unsigned char *p = lds + (ks + kr0) * (2 * W) + (((blk ^ column_swap<W>(kr0)) << 6) + lc);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)p);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)(p + 4 * 2 * W));
            return __builtin_bit_cast(uint4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    };

    // a wavefront whose results all lie past the end leaves the matrix cores to the others
    const bool idle = BM == 64 && n0 + 32 * NJ * wn >= a.N;
    auto multiply = [&](const unsigned char *la) __attribute__((always_inline)) {
        if (idle) return;
        const unsigned char *const lb = la + PA * S::PLANEA;
#pragma unroll
        for (int ks = 0; ks < BK; ks += 16) {
            uint4 fa[PA][MI], fb[PB][NJ];
#pragma unroll
            for (int p = 0; p < PA; ++p)
#pragma unroll
                for (int i = 0; i < MI; ++i)
                    fa[p][i] = frag(la + p * S::PLANEA, std::integral_constant<bool, S::ROWA>(), std::integral_constant<int, BM>(), MI * wm + i, ks);
#pragma unroll
            for (int p = 0; p < PB; ++p)
#pragma unroll
                for (int j = 0; j < NJ; ++j)
                    fb[p][j] = frag(lb + p * S::PLANEB, std::integral_constant<bool, S::ROWB>(), std::integral_constant<int, BN>(), NJ * wn + j, ks);
            // smallest products first; of three parts each, those of 2^-24 of the product and below are left out
#pragma unroll
            for (int s = PA + PB - 2; s >= 0; --s) {
                if (PA == 3 && PB == 3 && s > 2) continue;
#pragma unroll
                for (int pa = 0; pa < PA; ++pa) {
                    const int pb = s - pa;
                    if (pb < 0 || pb >= PB) continue;
#pragma unroll
                    for (int i = 0; i < MI; ++i)
#pragma unroll
                        for (int j = 0; j < NJ; ++j) acc[i][j] = split_mfma(fa[pa][i], fb[pb][j], acc[i][j]);
                }
            }
        }
    };

    const std::true_type counted{};
    const std::false_type guarded{};
    if constexpr (S::TWO) {
        // Tile i is multiplied out of buffer i mod 2 while tile i + 1 goes from its registers to the other buffer and the loads of
        // tile i + 3 are issued into these; those of tile i + 2 are on their way.  Of the two wavefronts that share a SIMD one
        // stages while the other multiplies, and then the other way round.
        const int64_t tiles = cdiv(k_end - k_beg, BK);
        const bool late = w >= WM * WN / 2;
        Set other;
        fetch(set, k_beg, guarded);
        if (tiles > 1) fetch(other, k_beg + BK, guarded);
        stage(set, smem);
        if (tiles > 2) fetch(set, k_beg + 2 * BK, guarded);
        __syncthreads();
        auto step = [&](int64_t i, Set &next, int side, auto how) __attribute__((always_inline)) {
            constexpr bool COUNTED = decltype(how)::value;
            const unsigned char *const now = smem + side * S::BUFFER;
            if (!late) multiply(now);
            if (COUNTED || i + 1 < tiles) stage(next, smem + (side ^ 1) * S::BUFFER);       // last read a barrier ago
            if (COUNTED || i + 3 < tiles) fetch(next, k_beg + (i + 3) * BK, how);
            if (late) multiply(now);
            __syncthreads();
        };
        int64_t i = 0;
        for (; k_beg + (i + 4) * BK <= k_whole; i += 2) {
            step(i, other, 0, counted);
            step(i + 1, set, 1, counted);
        }
        for (; i < tiles; i += 2) {
            step(i, other, 0, guarded);
            if (i + 1 < tiles) step(i + 1, set, 1, guarded);
        }
    } else {
        fetch(set, k_beg, guarded);
        for (int64_t k0 = k_beg; k0 < k_end; k0 += BK) {
            stage(set, smem);
            __syncthreads();
            if (k0 + BK < k_end) fetch(set, k0 + BK, guarded);
            multiply(smem);
            __syncthreads();
        }
    }

    // Results pass through LDS, a wavefront's 32 rows at a time in a place of its own, so that bias, activation, residual and stores
    // work on 8 consecutive columns a lane
    float *const out = reinterpret_cast<float *>(smem) + w * (32 * S::OUT);
    constexpr int OC = 4 * NJ;
    const int oc = lane % OC;
    const int64_t n = n0 + 32 * NJ * wn + 8 * oc;
    const int count = (int)max((int64_t)0, min((int64_t)8, a.N - n));
    float bias[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) bias[k] = MODE == FORWARD && a.bias && k < count ? a.bias[n + k] : 0.f;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        if (idle) break;
        __builtin_amdgcn_wave_barrier();
        // register v of lane l: row 8 (v / 4) + 4 (l / 32) + v % 4 and column l % 32 of the 32 x 32 block
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) out[(8 * (v >> 2) + 4 * (lane >> 5) + (v & 3)) * S::OUT + 32 * j + (lane & 31)] = acc[i][j][v];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int q = 0; q < 2 * NJ; ++q) {
            const int r = q * (64 / OC) + lane / OC;
            const int64_t m = m0 + 32 * (MI * wm + i) + r;
            float *from = out + r * S::OUT + 8 * oc;
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = from[k];
            if (m >= a.M || count == 0) continue;
            if (PA + PB > 2) {     // a sum that is not finite: once more from fp32 products, term by term
                bool bad = false;
#pragma unroll
                for (int k = 0; k < 8; ++k) bad |= k < count && split_not_finite(x[k]);
                if (bad) {
                    for (int c = 0; c < count; ++c) {
                        if (!split_not_finite(from[c])) continue;
                        float s = 0.f;
                        for (int64_t k = k_beg; k < k_end; ++k) {
                            float y = elem(S::ROWA ? a.A + m * a.lda + k : a.A + k * a.lda + m);
                            float z = elem(S::ROWB ? a.B + (n + c) * a.ldb + k : a.B + k * a.ldb + n + c);
                            if (MODE == INPUT && GRAD) y = through_act<ACT>(y, elem(a.pre + m * a.ldpre + k));
                            if (MODE == WEIGHTS && GRAD) z = through_act<ACT>(z, elem(a.pre + k * a.ldpre + n + c));
                            s = fmaf(y, z, s);
                            if (s != s) break;     // a NaN stays one: of inputs that are all NaN one term is read
                        }
                        from[c] = s;
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = from[k];
                }
            }
            if (MODE == WEIGHTS) {
                store8(a.part + (chunk * a.M + m) * a.N + n, count, x);
                continue;
            }
            if (MODE == FORWARD) {
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] += bias[k];
                if (a.pre_out) store8(a.pre_out + m * a.ldp + n, count, x);
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = act_of<ACT>(x[k]);
            }
            if (a.add) {
                float y[8];
                if constexpr (S::F32) load8(a.add + m * a.ldadd + n, count, y);
                else spread(load8(a.add + m * a.ldadd + n, count), y);
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] += y[k];
            }
            store8(a.C + m * a.ldc + n, count, x);
        }
    }
    if (MODE == WEIGHTS && sum_columns) {        // NT / BC threads hold the same columns: added in their order
        __syncthreads();
        float *s = reinterpret_cast<float *>(smem);
#pragma unroll
        for (int k = 0; k < 8; ++k) s[(t / BC) * BN + (t % BC) * 8 + k] = col[k];
        __syncthreads();
        if (t < BN && n0 + t < a.N) {
            float x = 0.f;
#pragma unroll 16
            for (int r = 0; r < NT / BC; ++r) x += s[r * BN + t];
            a.part_b[chunk * a.N + n0 + t] = x;
        }
    }
}

// NARROW: the last columns, 32 or fewer, have tiles of 128 x 32 behind the others
template <int MODE, class T, int ACT, int BM, int BN, int WM, int WN, bool NARROW>
__global__ __launch_bounds__(64 * WM * WN, (Shape<MODE, T, ACT, BM, BN, WM, WN>::WAVES)) void k_dense(Args<T> a)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    // block -> (tile of rows, tile of columns, chunk of terms).  Workgroup i runs on XCD i % 8, each with its own L2: the
    // tiles that read the same long rows follow one another on one XCD
    int64_t tm, chunk = 0;
    int32_t tn;
    if (MODE == WEIGHTS) {
        const int64_t tiles = a.tiles_m * a.tiles_n, chunks = cdiv(a.K, a.chunk);
        if (chunks >= 8) {
            const int64_t seq = blockIdx.x >> 3;
            chunk = (seq / tiles) * 8 + (blockIdx.x & 7);
            const int64_t t = seq % tiles;
            tm = t / a.tiles_n; tn = (int32_t)(t % a.tiles_n);
        } else {
            chunk = blockIdx.x / tiles;
            const int64_t t = blockIdx.x % tiles;
            tm = t / a.tiles_n; tn = (int32_t)(t % a.tiles_n);
        }
        if (chunk >= chunks) return;
    } else if (NARROW && blockIdx.x >= a.wide) {
        if constexpr (NARROW) tile_at<MODE, T, ACT, 128, 32, 4, 1>(a, (int64_t)(blockIdx.x - a.wide) * 128, a.tiles_n * BN, 0, smem);
        return;
    } else if (a.tiles_m >= 64) {
        const int64_t seq = blockIdx.x >> 3;
        tm = (seq / a.tiles_n) * 8 + (blockIdx.x & 7);
        tn = (int32_t)(seq % a.tiles_n);
        if (tm >= a.tiles_m) return;
    } else {
        tm = blockIdx.x / a.tiles_n;
        tn = (int32_t)(blockIdx.x % a.tiles_n);
    }
    tile_at<MODE, T, ACT, BM, BN, WM, WN>(a, tm * BM, tn * BN, chunk, smem);
}

// dW and db from the chunks' sums: 64 elements of either a block, four a lane, Y runs of chunks side by side, then these in their
// order.  One element a lane took 28 us in place of 12 at 3 chunks of 1500 x 1500, and 13.5 in place of 10 at 128 of 256 x 256
template <int Y>
__global__ __launch_bounds__(16 * Y) void k_dense_sum(const float *__restrict__ part, const float *__restrict__ part_b, int64_t chunks, int64_t nw,
                                                    int64_t nb, float *__restrict__ dW, float *__restrict__ db)
{
    struct __attribute__((packed, aligned(4))) F4 { float x[4]; };
    __shared__ float s[Y][68];
    const int x = 4 * (threadIdx.x & 15), y = threadIdx.x >> 4;
    const int64_t blocks_w = cdiv(nw, 64);
    const bool w = blockIdx.x < blocks_w;
    const int64_t n = w ? nw : nb, i0 = (w ? blockIdx.x : blockIdx.x - blocks_w) * 64, left = n - i0 - x;
    const float *const from = (w ? part : part_b) + i0 + x;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (left >= 4) {
        auto at = [&](int64_t c) { return *reinterpret_cast<const F4 *>(from + c * n); };
        int64_t c = y;
        for (; c + 3 * Y < chunks; c += 4 * Y) {       // four loads on their way, added in the chunks' order
            F4 z[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) z[k] = at(c + Y * k);
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += z[k].x[e];
        }
        for (; c < chunks; c += Y) {
            const F4 z = at(c);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += z.x[e];
        }
    } else {
        for (int64_t c = y; c < chunks; c += Y)
#pragma unroll
            for (int e = 0; e < 3; ++e) if (e < left) v[e] += from[c * n + e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) s[y][x + e] = v[e];
    __syncthreads();
    const int t = threadIdx.x;
    if (t < 64 && i0 + t < n) {
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < Y; ++r) sum += s[r][t];
        (w ? dW : db)[i0 + t] = sum;
    }
}

constexpr int32_t MAX_D = 65536;

int check(const kge_dense *L, int64_t n_rows)
{
    KGE_REQUIRE(L, KGE_EINVAL, "NULL argument");
    KGE_REQUIRE(L->d_in >= 1 && L->d_out >= 1 && L->d_in <= MAX_D && L->d_out <= MAX_D, KGE_EINVAL, "dense: widths are 1 to %d", MAX_D);
    KGE_REQUIRE(L->dtype == KGE_DT_F32 || L->dtype == KGE_DT_BF16, KGE_EINVAL, "dense: bad type");
    KGE_REQUIRE(L->act == KGE_ACT_IDENTITY || L->act == KGE_ACT_RELU || L->act == KGE_ACT_SILU, KGE_EINVAL, "dense: bad act");
    KGE_REQUIRE(n_rows >= 0, KGE_EINVAL, "dense: negative number of rows");
    KGE_REQUIRE(n_rows <= 0x7fffffffLL, KGE_ERANGE, "dense: at most 2^31 - 1 rows");
    return KGE_OK;
}

// The weights' gradient has the smallest tile that takes a narrow side whole: what is empty of a tile is multiplied all the same.  bf16
// results of 129 rows and 65 columns and more take a tile of 256 x 128, so that dY becomes dP in one block alone for up to 256 rows (a
// million rows of 256 x 256, SiLU: 781 us with tiles of 128 x 128, 474 with 256 x 256, whose 128 sums a lane leave no registers for
// loads two tiles ahead, 460 with these)
struct Tile { int bm, bn; };
Tile weights_tile(const kge_dense *L)
{
    if (L->d_out <= 32) return {128, 32};
    if (L->d_out <= 64) return {128, 64};
    if (L->d_in <= 32) return {32, 128};
    if (L->dtype == KGE_DT_BF16 && L->d_in > 128 && L->d_out > 64) return {256, 128};
    return {128, 128};
}

// Chunks of rows of the weights' gradient: as many as run at once, at least 256 rows each.  A chunk's tiles run on one XCD: the chip
// holds 512 blocks, but an XCD 64, and one more than that is a second round (29082 x 203 x 517 fp32, 10 tiles: 103 us with 51 chunks,
// 7 of them on some XCDs, 73 with 48; 60000 x 384 x 384 bf16 65 and 44)
int64_t chunk_rows(const kge_dense *L, int64_t n_rows)
{
    const Tile tile = weights_tile(L);
    const int64_t tiles = cdiv(L->d_in, tile.bm) * cdiv(L->d_out, tile.bn), at_once = tile.bm == 256 ? 256 : 512;
    int64_t chunks = tiles <= at_once / 8 ? 8 * (at_once / 8 / tiles) : at_once / tiles;
    if (chunks > cdiv(n_rows, 256)) chunks = cdiv(n_rows, 256);
    if (chunks < 1) chunks = 1;
    return align_up((size_t)cdiv(n_rows > 0 ? n_rows : 1, chunks), 64);
}

template <class F>
void with_act(int act, F f)
{
    if (act == KGE_ACT_RELU) f(std::integral_constant<int, KGE_ACT_RELU>());
    else if (act == KGE_ACT_SILU) f(std::integral_constant<int, KGE_ACT_SILU>());
    else f(std::integral_constant<int, KGE_ACT_IDENTITY>());
}

// Up to three whole tiles of columns and 32 columns or fewer (us with a tile of 128 for these against narrow ones): fp32 112 / 119
// against 92 / 108 (forward with 200 terms / input gradient with 200, 100000 rows, 160 columns), 137 / 160 against 128 / 149 (60000
// rows, 288), 196 / 217 against 192 / 206 (100000, 400), but 233 against 240 with 528; bf16 forward 43 against 34, 44 against 42, 75
// against 64.  A bf16 input gradient splits dP in either: 54 against 59 with 160 columns
template <int MODE, class T>
constexpr bool MAY_NARROW = MODE == FORWARD || (MODE == INPUT && sizeof(T) == 4);
bool narrow_pays(int32_t n) { return n > 128 && n <= 416 && n % 128 >= 1 && n % 128 <= 32; }

// fp32 tiles of 64 x 128 in place of 128 x 128, forward / input gradient, time over that of 128 x 128.  Up to 384 of these: twice as many
// blocks of 64 rows leave no more than three on a compute unit, in place of one or two unequally: 0.81 to 0.98 from 200 to 360 tiles, at 203
// to 768 terms and 203 to 640 columns (but 1.02 at 255 tiles of 768 terms).  Above, W is split and read twice as often for a round that is
// no shorter: 400 tiles 1.01 to 1.05 up to 320 terms, 1.04 to 1.10 from 384 on; 512 0.92 to 1.04, 0.97 to 1.08; 570 0.93 to 1.02, 0.96 to
// 1.05; 640 0.96 to 1.03, 0.99 to 1.06; 700 to 768 0.91 to 1.05 at 200 terms, 0.95 to 1.12 at 512.  Rows of an odd number of terms gain most:
// 14541 x 203 x 517 with SiLU, 570 tiles, 51.7 / 44.7 us against 53.0 / 54.2.
bool half_tall_pays(int64_t m, int32_t n, int64_t terms)
{
    const int64_t tiles = cdiv(m, 128) * cdiv(n, 128);
    return tiles <= 384 || (tiles <= 640 && terms <= 320);
}

template <int MODE, class T, int BM, int BN, int WM, int WN, bool NARROW = false>
int launch_tile(int act, Args<T> a, hipStream_t st)
{
    if constexpr (MAY_NARROW<MODE, T> && !NARROW) {
        if (narrow_pays(a.N)) return launch_tile<MODE, T, BM, BN, WM, WN, true>(act, a, st);
    }
    a.tiles_m = cdiv(a.M, BM);
    a.tiles_n = NARROW ? a.N / BN : (int32_t)cdiv(a.N, BN);
    int64_t blocks = a.tiles_m * a.tiles_n;
    if (MODE == WEIGHTS) {
        const int64_t chunks = cdiv(a.K, a.chunk);
        blocks *= chunks >= 8 ? (int64_t)align_up((size_t)chunks, 8) : chunks;
    } else if (a.tiles_m >= 64) blocks = (int64_t)align_up((size_t)a.tiles_m, 8) * a.tiles_n;
    a.wide = (uint32_t)blocks;
    if (NARROW) blocks += cdiv(a.M, 128);
    KGE_REQUIRE(blocks < (1ll << 32) / (64 * WM * WN), KGE_ERANGE, "dense: too large for one launch");
    hipError_t e = hipSuccess;
    with_act(act, [&](auto act_c) {
        constexpr int ACT = decltype(act_c)::value, WIDE = Shape<MODE, T, ACT, BM, BN, WM, WN>::LDS;
        int lds = WIDE;
        if constexpr (NARROW) lds = std::max(lds, Shape<MODE, T, ACT, 128, 32, 4, 1>::LDS);
        auto kernel = k_dense<MODE, T, ACT, BM, BN, WM, WN, NARROW>;
        if (lds > 64 * 1024) e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e == hipSuccess) kernel<<<(unsigned)blocks, 64 * WM * WN, lds, st>>>(a);
    });
    KGE_HIP(e);
    KGE_LAUNCH_CHECK();
    return KGE_OK;
}

template <int MODE, class T>
int launch(const kge_dense *L, const Args<T> &a, hipStream_t st)
{
    if constexpr (MODE == WEIGHTS) {
        KGE_PROF("dense_weight_grad", st);
        const Tile tile = weights_tile(L);
        if (tile.bn == 32) return launch_tile<MODE, T, 128, 32, 4, 1>(L->act, a, st);
        if (tile.bn == 64) return launch_tile<MODE, T, 128, 64, 2, 2>(L->act, a, st);
        if (tile.bm == 32) return launch_tile<MODE, T, 32, 128, 1, 4>(L->act, a, st);
        if constexpr (sizeof(T) == 2) {
            if (tile.bm == 256) return launch_tile<MODE, T, 256, 128, 4, 2>(L->act, a, st);
        }
        return launch_tile<MODE, T, 128, 128, 2, 2>(L->act, a, st);
    } else {
        if (few_pay(a)) {
            KGE_PROF(MODE == FORWARD ? "dense_few" : "dense_few_input_grad", st);
            return launch_few<MODE, T>(a, L->act, st);
        }
        if (rows_pay(a)) {
            KGE_PROF(MODE == FORWARD ? "dense_rows" : "dense_rows_input_grad", st);
            return launch_rows<MODE, T>(a, L->act, st);
        }
        KGE_PROF(MODE == FORWARD ? "dense" : "dense_input_grad", st);
        if constexpr (sizeof(T) == 4) {
            if (half_tall_pays(a.M, a.N, a.K)) return launch_tile<MODE, T, 64, 128, 1, 4>(L->act, a, st);
        }
        return launch_tile<MODE, T, 128, 128, 2, 2>(L->act, a, st);
    }
}

bool at_element(const void *p, int32_t dtype) { return ((uintptr_t)p % (dtype == KGE_DT_BF16 ? 2 : 4)) == 0; }

template <class T>
int forward(const kge_dense *L, int64_t n, const void *X, int64_t ldx, const void *R, int64_t ldr, void *Y, int64_t ldy, void *pre, int64_t ldp,
            hipStream_t st)
{
    Args<T> a{};
    a.A = (const T *)X; a.lda = ldx; a.B = (const T *)L->W; a.ldb = L->d_out;
    a.M = n; a.N = L->d_out; a.K = a.chunk = L->d_in;
    a.C = (T *)Y; a.ldc = ldy; a.pre_out = (T *)pre; a.ldp = ldp; a.add = (const T *)R; a.ldadd = ldr; a.bias = L->b;
    return launch<FORWARD, T>(L, a, st);
}

template <class T>
int backward(const kge_dense *L, int64_t n, const void *X, int64_t ldx, const void *pre, int64_t ldp, const void *dY, int64_t lddy, const void *add,
             int64_t ldadd, void *dX, int64_t lddx, float *dW, float *db, void *ws, hipStream_t st)
{
    if (dX && n > 0) {
        Args<T> a{};
        a.A = (const T *)dY; a.lda = lddy; a.pre = (const T *)pre; a.ldpre = ldp; a.B = (const T *)L->W; a.ldb = L->d_out;
        a.M = n; a.N = L->d_in; a.K = a.chunk = L->d_out;
        a.C = (T *)dX; a.ldc = lddx; a.add = (const T *)add; a.ldadd = ldadd;
        int rc = launch<INPUT, T>(L, a, st);
        if (rc != KGE_OK) return rc;
    }
    if (dW || db) {
        const int64_t chunk = chunk_rows(L, n), chunks = cdiv(n, chunk), nw = (int64_t)L->d_in * L->d_out;
        Args<T> a{};
        a.part = (float *)ws;
        a.part_b = db ? a.part + chunks * nw : nullptr;
        if (chunks == 1 && dW) { a.part = dW; a.part_b = db; }      // one chunk's sums are the result
        if (n > 0) {
            a.A = (const T *)X; a.lda = ldx; a.B = (const T *)dY; a.ldb = lddy; a.pre = (const T *)pre; a.ldpre = ldp;
            a.M = L->d_in; a.N = L->d_out; a.K = n; a.chunk = chunk;
            int rc = launch<WEIGHTS, T>(L, a, st);
            if (rc != KGE_OK || a.part == dW) return rc;
        }
        KGE_PROF("dense_sum", st);             // without rows: sums of nothing, zeros
        const int64_t w = dW ? nw : 0, b = db ? L->d_out : 0;
        const unsigned blocks = (unsigned)(cdiv(w, 64) + cdiv(b, 64));
        if (chunks > 256) k_dense_sum<64><<<blocks, 1024, 0, st>>>(a.part, a.part_b, chunks, w, b, dW, db);
        else if (chunks > 96) k_dense_sum<32><<<blocks, 512, 0, st>>>(a.part, a.part_b, chunks, w, b, dW, db);
        else if (chunks > 16) k_dense_sum<16><<<blocks, 256, 0, st>>>(a.part, a.part_b, chunks, w, b, dW, db);
        else k_dense_sum<4><<<blocks, 64, 0, st>>>(a.part, a.part_b, chunks, w, b, dW, db);
        KGE_LAUNCH_CHECK();
    }
    return KGE_OK;
}

}  // namespace

extern "C" int kge_dense_forward(const kge_dense *L, int64_t n_rows, const void *X, int64_t ldx, const void *R, int64_t ldr, void *Y, int64_t ldy,
                                 void *pre, int64_t ldp, void *stream)
{
    int rc = check(L, n_rows);
    if (rc != KGE_OK) return rc;
    KGE_REQUIRE(ldx >= L->d_in && ldy >= L->d_out && (!R || ldr >= L->d_out) && (!pre || ldp >= L->d_out), KGE_EINVAL,
                "dense: a row stride is smaller than the row");
    if (n_rows == 0) return KGE_OK;
    KGE_REQUIRE(L->W && X && Y, KGE_EINVAL, "NULL argument");
    KGE_REQUIRE(at_element(L->W, L->dtype) && at_element(X, L->dtype) && at_element(R, L->dtype) && at_element(Y, L->dtype) &&
                    at_element(pre, L->dtype) && at_element(L->b, KGE_DT_F32), KGE_EINVAL, "dense: an array is not aligned to its elements");
    KGE_REQUIRE(Y != X && Y != pre && (!pre || (pre != X && pre != R)), KGE_EINVAL, "dense: Y and pre may not be X or each other, nor pre R");
    KGE_REQUIRE(R != Y || ldr == ldy || n_rows == 1, KGE_EINVAL, "dense: an R that is Y has Y's row stride");
    hipStream_t st = (hipStream_t)stream;
    return L->dtype == KGE_DT_F32 ? forward<float>(L, n_rows, X, ldx, R, ldr, Y, ldy, pre, ldp, st)
                                  : forward<uint16_t>(L, n_rows, X, ldx, R, ldr, Y, ldy, pre, ldp, st);
}

extern "C" size_t kge_dense_workspace_bytes(const kge_dense *L, int64_t n_rows)
{
    if (check(L, n_rows) != KGE_OK) return 0;
    const int64_t chunks = n_rows > 0 ? cdiv(n_rows, chunk_rows(L, n_rows)) : 1;
    return align_up((size_t)chunks * ((size_t)L->d_in * L->d_out + L->d_out) * sizeof(float), 256);
}

extern "C" int kge_dense_backward(const kge_dense *L, int64_t n_rows, const void *X, int64_t ldx, const void *pre, int64_t ldp, const void *dY,
                                  int64_t lddy, const void *add, int64_t ldadd, void *dX, int64_t lddx, float *dW, float *db, void *workspace,
                                  size_t ws_bytes, void *stream)
{
    int rc = check(L, n_rows);
    if (rc != KGE_OK) return rc;
    KGE_REQUIRE(n_rows == 0 || ((L->W || !dX) && (X || !(dW || db)) && dY && (pre || L->act == KGE_ACT_IDENTITY)), KGE_EINVAL, "NULL argument");
    KGE_REQUIRE((!X || ldx >= L->d_in) && (!dY || lddy >= L->d_out) && (!pre || ldp >= L->d_out) && (!add || ldadd >= L->d_in) && (!dX || lddx >= L->d_in),
                KGE_EINVAL, "dense: a row stride is smaller than the row");
    KGE_REQUIRE(!add || dX, KGE_EINVAL, "dense: a gradient to add needs dX");
    KGE_REQUIRE(at_element(L->W, L->dtype) && at_element(X, L->dtype) && at_element(pre, L->dtype) && at_element(dY, L->dtype) &&
                    at_element(add, L->dtype) && at_element(dX, L->dtype) && at_element(dW, KGE_DT_F32) && at_element(db, KGE_DT_F32),
                KGE_EINVAL, "dense: an array is not aligned to its elements");
    if (dW || db) {
        KGE_REQUIRE((int64_t)L->d_in * L->d_out <= 1ll << 28, KGE_ERANGE, "dense: a weights' gradient has at most 2^28 elements");
        KGE_REQUIRE(workspace && ((uintptr_t)workspace % 256) == 0, KGE_EINVAL, "dense: the workspace must be 256-byte aligned");
        KGE_REQUIRE(ws_bytes >= kge_dense_workspace_bytes(L, n_rows), KGE_ENOMEM, "dense: workspace too small");
    }
    KGE_REQUIRE(!dX || n_rows == 0 || (dX != dY && dX != pre && dX != X), KGE_EINVAL, "dense: dX may not be dY, pre or X");
    KGE_REQUIRE(!dX || add != dX || ldadd == lddx || n_rows <= 1, KGE_EINVAL, "dense: an add that is dX has dX's row stride");
    hipStream_t st = (hipStream_t)stream;
    return L->dtype == KGE_DT_F32
               ? backward<float>(L, n_rows, X, ldx, pre, ldp, dY, lddy, add, ldadd, dX, lddx, dW, db, workspace, st)
               : backward<uint16_t>(L, n_rows, X, ldx, pre, ldp, dY, lddy, add, ldadd, dX, lddx, dW, db, workspace, st);
}
