// Draws from rows of scores: temperature, top-k, top-p and min-p, from random numbers that the caller gives.
//
//   weight of a score l in a row whose largest is m:  w = e^((l - m) / temperature), rounded to a multiple of 2^-b,
//   b = min(40, 62 - ceil(log2 columns));  minus infinity and NaN have none
//   in descending order of scores, equal ones in the order of their columns: top-k leaves the first k, top-p of those the
//   shortest beginning whose weights reach top_p of theirs, min-p what has at least min_p times the largest weight
//   the draw: the first column at which the sum of the weights left, in the order of columns, passes u times their total
//
// Weights are whole numbers below 2^63 in all, so that sums are exact: neither the order in which threads add nor the way in
// which rows are split shows in a result.  The exponential is formed in double: a weight is off by one unit at most, and that
// only where it lies next to a half of one.
//
// What top-k and top-p leave is all scores above one and, of those equal to it, the first few: that score is found digit by
// digit of its bits (three digits), from counts or sums of weights by digit in LDS.
#include "common.h"

#include <math.h>

namespace {

typedef unsigned long long u64;

constexpr int THREADS = 1024, WAVES = THREADS / 64;
constexpr int DIGITS = 2048;                  // values of a digit: 11, 11 and 10 bits

struct Sampling {
    float temperature, top_p, min_p;
    int32_t top_k;
    const float *row_temperature, *row_top_p, *row_min_p;
    const int32_t *row_top_k;
};

struct Call {
    Sampling how;
    const void *scores;
    const void *u;
    int32_t *choice;
    float *prob;
    int64_t n_rows, lds;
    int32_t n_cols, n_draws, bits;
    int32_t u64bit;
};

// bits of scores in an order that whole numbers have; 0: no weight.  Both zeros are one.
__device__ __forceinline__ uint32_t key_of(float l)
{
    const uint32_t b = __float_as_uint(l + 0.f);
    const uint32_t k = b ^ ((int32_t)b < 0 ? 0xffffffffu : 0x80000000u);
    return l > -INFINITY ? k : 0u;
}
__device__ __forceinline__ float score_of(uint32_t key) { return __uint_as_float(key ^ ((int32_t)key < 0 ? 0x80000000u : 0xffffffffu)); }

template <bool BF16>
__device__ __forceinline__ uint32_t key_at(const void *row, int64_t c)
{
    return key_of(BF16 ? __uint_as_float((uint32_t)((const uint16_t *)row)[c] << 16) : ((const float *)row)[c]);
}

struct Weigh {
    double most, per, unit, least;           // m, 1 / temperature, 2^b, and the exponent below which a weight rounds to zero
    uint32_t most_key;
    __device__ __forceinline__ u64 operator()(uint32_t key) const
    {
        if (key == 0u) return 0ull;
        if (key == most_key) return (u64)unit;
        const double z = ((double)score_of(key) - most) * per;
        return z > least ? (u64)rint(exp(z) * unit) : 0ull;
    }
};

// ---- a block's sums

__device__ __forceinline__ u64 shfl_up64(u64 v, int off) { return (u64)__shfl_up((long long)v, off, 64); }
__device__ __forceinline__ u64 shfl_xor64(u64 v, int off) { return (u64)__shfl_xor((long long)v, off, 64); }

__device__ __forceinline__ u64 wave_scan(u64 v)
{
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const u64 o = shfl_up64(v, off);
        if ((int)(threadIdx.x & 63) >= off) v += o;
    }
    return v;
}

// inclusive sums over the block's threads, and their total; s: WAVES + 1 words
__device__ __forceinline__ u64 block_scan(u64 v, u64 *s, u64 *total)
{
    const int wave = threadIdx.x >> 6;
    v = wave_scan(v);
    if ((threadIdx.x & 63) == 63) s[wave] = v;
    __syncthreads();
    u64 before = 0ull, all = 0ull;
    for (int i = 0; i < WAVES; ++i) {
        if (i < wave) before += s[i];
        all += s[i];
    }
    __syncthreads();
    *total = all;
    return before + v;
}

__device__ __forceinline__ uint32_t block_max(uint32_t v, u64 *s)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, off, 64));
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    uint32_t all = 0u;
    for (int i = 0; i < WAVES; ++i) all = max(all, (uint32_t)s[i]);
    __syncthreads();
    return all;
}

// The digit at which the sums, from the largest digit down, first reach `goal` (1 or more, at most their total), and the sum of
// the digits above it.  Two digits a thread.
__device__ __forceinline__ int digit_at(const u64 *hist, u64 goal, u64 *s, u64 *s_found, u64 *above)
{
    static_assert(DIGITS == 2 * THREADS, "two digits a thread");
    const int hi = DIGITS - 1 - 2 * (int)threadIdx.x;
    const u64 a = hist[hi], b = hist[hi - 1];
    u64 total;
    const u64 upto = block_scan(a + b, s, &total), before = upto - a - b;
    if (before < goal && goal <= upto) {
        const bool first = goal <= before + a;
        s_found[0] = first ? hi : hi - 1;
        s_found[1] = first ? before : before + a;
    }
    __syncthreads();
    const int digit = (int)s_found[0];
    *above = s_found[1];
    __syncthreads();
    return digit;
}

// One block to a row.
template <bool BF16>
__global__ __launch_bounds__(THREADS) void k_sample_rows(Call o)
{
    __shared__ u64 s_hist[DIGITS];
    __shared__ u64 s_part[WAVES + 1], s_found[2];
    __shared__ u64 s_sums[THREADS];
    const int tid = threadIdx.x;
    for (int64_t r = blockIdx.x; r < o.n_rows; r += gridDim.x) {
        const void *row = (const char *)o.scores + r * o.lds * (BF16 ? 2 : 4);
        const int32_t n = o.n_cols;
        float t = o.how.row_temperature ? o.how.row_temperature[r] : o.how.temperature;
        int32_t k = o.how.row_top_k ? o.how.row_top_k[r] : o.how.top_k;
        if (o.how.row_top_k && o.how.top_k > 0) k = k > 0 ? min(k, o.how.top_k) : o.how.top_k;
        const float p = o.how.row_top_p ? o.how.row_top_p[r] : o.how.top_p, low = o.how.row_min_p ? o.how.row_min_p[r] : o.how.min_p;
        if (!(t > 0.f)) { t = 1.f; k = 1; }
        // the largest score
        uint32_t most = 0u;
        for (int32_t c = tid; c < n; c += THREADS) most = max(most, key_at<BF16>(row, c));
        most = block_max(most, s_part);
        Weigh weigh;
        weigh.unit = (double)(1ull << o.bits);
        weigh.most_key = most; weigh.most = (double)score_of(most); weigh.per = 1.0 / (double)t;
        weigh.least = -0.6931471805599453 * (o.bits + 2);
        // what is left: keys above `cut` and, of those equal to it, the first `ties`
        uint32_t cut = 0u;
        u64 ties = 0ull;
        for (int which = 0; which < 2; ++which) {                // top-k, then top-p
            if (which == 0 ? (k <= 0 || k >= n) : !(p < 1.f)) continue;
            u64 goal = 0ull, all = 0ull;
            uint32_t found = 0u;
            u64 above = 0ull;
            const u64 cut_w = which == 1 && ties > 0ull ? weigh(cut) : 0ull;
            for (int level = 0; level < 3; ++level) {
                const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, width = level == 2 ? 1024 : 2048;
                for (int i = tid; i < DIGITS; i += THREADS) s_hist[i] = 0ull;
                __syncthreads();
                const uint32_t same = level == 0 ? 0u : level == 1 ? 0xffe00000u : 0xfffffc00u;
                u64 mine = 0ull;
                for (int32_t c = tid; c < n; c += THREADS) {
                    const uint32_t key = key_at<BF16>(row, c);
                    if (key == 0u || (key & same) != found || (which == 1 && key <= cut)) continue;
                    const u64 w = which == 0 ? 1ull : weigh(key);
                    if (w) atomicAdd(&s_hist[(key >> shift) & (width - 1)], w);
                    mine += w;
                }
                if (which == 1 && tid == 0 && ties > 0ull && (cut & same) == found) {
                    atomicAdd(&s_hist[(cut >> shift) & (width - 1)], ties * cut_w);
                    mine += ties * cut_w;
                }
                __syncthreads();
                if (level == 0) {
                    block_scan(mine, s_part, &all);
                    if (which == 0) goal = all < (u64)k ? 0ull : (u64)k;
                    else {
                        const double g = ceil((double)p * (double)all);
                        goal = g < 1.0 ? 1ull : (u64)g;
                        if (goal > all) goal = all;
                    }
                    if (goal == 0ull) break;                     // fewer scores than k, or none
                }
                u64 more;
                const int digit = digit_at(s_hist, goal - above, s_part, s_found, &more);
                above += more;
                found |= (uint32_t)digit << shift;
            }
            if (goal == 0ull) continue;
            if (which == 0) { cut = found; ties = goal - above; }
            else {
                const u64 w = weigh(found);
                ties = (goal - above + w - 1ull) / w;
                cut = found;
            }
        }
        const double least_weight = (double)(low > 1.f ? 1.f : low) * weigh.unit;
        // the weights in the order of columns: first their total, then what the draws reach
        u64 total = 0ull;
        for (int pass = 0; pass < 2; ++pass) {
            u64 base = 0ull, equal = 0ull;
            for (int32_t c0 = 0; c0 < n; c0 += THREADS) {
                const int32_t c = c0 + tid;
                const uint32_t key = c < n ? key_at<BF16>(row, c) : 0u;
                bool in = key > cut;
                if (cut != 0u) {
                    u64 here;
                    const u64 before = equal + block_scan(key == cut ? 1ull : 0ull, s_part, &here);
                    if (key == cut) in = before <= ties;
                    equal += here;
                }
                u64 w = in ? weigh(key) : 0ull;
                if ((double)w < least_weight) w = 0ull;
                u64 here;
                const u64 upto = block_scan(w, s_part, &here);
                if (pass == 1 && here) {
                    s_sums[tid] = base + upto;
                    __syncthreads();
                    for (int32_t i = tid; i < o.n_draws; i += THREADS) {
                        const int64_t at = r * o.n_draws + i;
                        const double u = o.u64bit ? ((const double *)o.u)[at] : (double)((const float *)o.u)[at];
                        const double reach = u * (double)total;
                        const u64 goal = reach >= (double)total ? total - 1ull : reach > 0.0 ? min((u64)reach, total - 1ull) : 0ull;
                        if (goal < base || goal >= base + here) continue;
                        int lo = 0, hi = THREADS - 1;            // the first of the sums above the goal
                        while (lo < hi) {
                            const int mid = (lo + hi) >> 1;
                            if (s_sums[mid] > goal) hi = mid;
                            else lo = mid + 1;
                        }
                        o.choice[at] = c0 + lo;
                        if (o.prob) o.prob[at] = (float)((double)(s_sums[lo] - (lo ? s_sums[lo - 1] : base)) / (double)total);
                    }
                    __syncthreads();
                }
                base += here;
            }
            if (pass == 0) {
                total = base;
                if (total == 0ull) {
                    for (int32_t i = tid; i < o.n_draws; i += THREADS) {
                        const int64_t at = r * o.n_draws + i;
                        o.choice[at] = -1;
                        if (o.prob) o.prob[at] = 0.f;
                    }
                    break;
                }
            }
        }
        __syncthreads();
    }
}

int bits_of(int64_t n_cols)
{
    int log = 0;
    while ((1ll << log) < n_cols) ++log;
    return 62 - log < 40 ? 62 - log : 40;
}

int check_call(const kge_sampling *how, int64_t n_rows, int64_t n_cols)
{
    KGE_REQUIRE(how, KGE_EINVAL, "NULL argument");
    KGE_REQUIRE(n_rows >= 0 && n_cols >= 0, KGE_EINVAL, "negative size");
    KGE_REQUIRE(n_rows <= 0x7fffffffll && n_cols <= 0x7fffffffll, KGE_ERANGE, "2^31 rows or columns or more");
    KGE_REQUIRE(how->row_temperature || (how->temperature >= 0.f && how->temperature <= 3.402823466e38f), KGE_EINVAL,
                "temperature must be zero or more, and finite");
    KGE_REQUIRE(how->top_k >= 0, KGE_EINVAL, "top_k must be zero (off) or more");
    KGE_REQUIRE(how->row_top_p || (how->top_p > 0.f && how->top_p <= 1.f), KGE_EINVAL, "top_p must be above zero, and one at most (off)");
    KGE_REQUIRE(how->row_min_p || (how->min_p >= 0.f && how->min_p <= 1.f), KGE_EINVAL, "min_p must be zero (off) to one");
    KGE_REQUIRE((uintptr_t)how->row_temperature % 4 == 0 && (uintptr_t)how->row_top_k % 4 == 0 && (uintptr_t)how->row_top_p % 4 == 0 &&
                    (uintptr_t)how->row_min_p % 4 == 0, KGE_EINVAL, "the rows' settings must be aligned to their elements");
    return KGE_OK;
}

}  // namespace

extern "C" size_t kge_sample_workspace_bytes(const kge_sampling *how, int64_t n_rows, int64_t n_cols)
{
    if (check_call(how, n_rows, n_cols) != KGE_OK) return 0;
    return 256;
}

extern "C" int kge_sample_scores(const kge_sampling *how, int64_t n_rows, int64_t n_cols, const void *scores, int32_t dtype, int64_t lds,
                                 const void *u, int32_t u_bits, int32_t n_draws, int32_t *choice, float *prob, void *workspace,
                                 size_t ws_bytes, void *stream)
{
    int rc = check_call(how, n_rows, n_cols);
    if (rc != KGE_OK) return rc;
    KGE_REQUIRE(dtype == KGE_DT_F32 || dtype == KGE_DT_BF16, KGE_EINVAL, "scores: bad type");
    KGE_REQUIRE(u_bits == 32 || u_bits == 64, KGE_EINVAL, "random numbers have 32 or 64 bits");
    KGE_REQUIRE(n_draws >= 0, KGE_EINVAL, "negative number of draws");
    KGE_REQUIRE(lds >= n_cols && lds <= (1ll << 40), KGE_EINVAL, "scores: the row stride is less than a row");
    if (n_rows == 0 || n_draws == 0) return KGE_OK;
    KGE_REQUIRE((scores || n_cols == 0) && u && choice, KGE_EINVAL, "NULL array");
    KGE_REQUIRE((uintptr_t)scores % (dtype == KGE_DT_F32 ? 4 : 2) == 0 && (uintptr_t)u % (u_bits / 8) == 0 && (uintptr_t)choice % 4 == 0 &&
                    (uintptr_t)prob % 4 == 0, KGE_EINVAL, "an array is not aligned to its elements");
    KGE_REQUIRE(workspace && (uintptr_t)workspace % 256 == 0, KGE_EINVAL, "the workspace is NULL or not aligned to 256 bytes");
    KGE_REQUIRE(ws_bytes >= kge_sample_workspace_bytes(how, n_rows, n_cols), KGE_ENOMEM, "the workspace is too small");
    hipStream_t st = (hipStream_t)stream;
    Call o;
    o.how = Sampling{how->temperature, how->top_p, how->min_p, how->top_k, how->row_temperature, how->row_top_p, how->row_min_p, how->row_top_k};
    o.scores = scores; o.u = u; o.choice = choice; o.prob = prob; o.n_rows = n_rows; o.lds = lds;
    o.n_cols = (int32_t)n_cols; o.n_draws = n_draws; o.bits = bits_of(n_cols); o.u64bit = u_bits == 64;
    KGE_PROF("sample_scores", st);
    const unsigned blocks = (unsigned)(n_rows < 65536 ? n_rows : 65536);
    (dtype == KGE_DT_BF16 ? k_sample_rows<true> : k_sample_rows<false>)<<<blocks, THREADS, 0, st>>>(o);
    KGE_LAUNCH_CHECK();
    return KGE_OK;
}

namespace {

__global__ __launch_bounds__(256) void k_pick_negatives(const int32_t *__restrict__ cand_ent, const uint8_t *__restrict__ cand_side, uint32_t n_cand,
                                                        const int32_t *__restrict__ choice, int64_t n, uint32_t n_neg, int32_t *__restrict__ neg_ent,
                                                        uint8_t *__restrict__ neg_side)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t q = i / n_neg;
        uint32_t c = (uint32_t)choice[i];
        if (c >= n_cand) c = (uint32_t)(i - q * n_neg) % n_cand;
        neg_ent[i] = cand_ent[q * n_cand + c];
        neg_side[i] = cand_side[q * n_cand + c];
    }
}

// candidates whose corrupted triple is the positive itself: their scores become minus infinity
__global__ __launch_bounds__(256) void k_hide_positives(const int32_t *__restrict__ core_h, const int32_t *__restrict__ core_t, int32_t n_core,
                                                        const int32_t *__restrict__ pos, int64_t n, uint32_t n_cand, const int32_t *__restrict__ cand_ent,
                                                        const uint8_t *__restrict__ cand_side, float *__restrict__ scores, int64_t lds)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t q = i / n_cand;
        const int32_t c = pos[q];
        if (c < 0 || c >= n_core) continue;
        if (cand_ent[i] == (cand_side[i] ? core_h[c] : core_t[c])) scores[q * lds + (i - q * n_cand)] = -INFINITY;
    }
}

}  // namespace

extern "C" int kge_hide_positives(const kge_partition *p, const int32_t *pos_core_idx, int64_t n_pos, const int32_t *cand_ent,
                                  const uint8_t *cand_side, int32_t n_cand, float *scores, int64_t lds, void *stream)
{
    KGE_REQUIRE(p, KGE_EINVAL, "NULL partition");
    KGE_REQUIRE(n_pos >= 0 && n_cand >= 0 && lds >= n_cand, KGE_EINVAL, "negative size, or a row stride of less than a row");
    KGE_REQUIRE(n_pos <= 0x7fffffffll, KGE_ERANGE, "2^31 positives or more");
    const int64_t n = n_pos * n_cand;
    if (n == 0) return KGE_OK;
    KGE_REQUIRE(pos_core_idx && cand_ent && cand_side && scores, KGE_EINVAL, "NULL array");
    hipStream_t st = (hipStream_t)stream;
    KGE_PROF("hide_positives", st);
    const int64_t blocks = cdiv(n, 256);
    k_hide_positives<<<(unsigned)(blocks < 65536 ? blocks : 65536), 256, 0, st>>>(p->core_h, p->core_t, (int32_t)p->n_core, pos_core_idx, n,
                                                                               (uint32_t)n_cand, cand_ent, cand_side, scores, lds);
    KGE_LAUNCH_CHECK();
    return KGE_OK;
}

extern "C" int kge_pick_negatives(const int32_t *cand_ent, const uint8_t *cand_side, int32_t n_cand, const int32_t *choice, int64_t n_pos,
                                  int32_t n_neg, int32_t *neg_ent, uint8_t *neg_side, void *stream)
{
    KGE_REQUIRE(n_pos >= 0 && n_neg >= 0 && n_cand >= 0, KGE_EINVAL, "negative size");
    KGE_REQUIRE(n_pos <= 0x7fffffffll, KGE_ERANGE, "2^31 positives or more");
    const int64_t n = n_pos * n_neg;
    if (n == 0) return KGE_OK;
    KGE_REQUIRE(n_cand > 0, KGE_EINVAL, "no candidates to draw from");
    KGE_REQUIRE(cand_ent && cand_side && choice && neg_ent && neg_side, KGE_EINVAL, "NULL array");
    hipStream_t st = (hipStream_t)stream;
    KGE_PROF("pick_negatives", st);
    const int64_t blocks = cdiv(n, 256);
    k_pick_negatives<<<(unsigned)(blocks < 65536 ? blocks : 65536), 256, 0, st>>>(cand_ent, cand_side, (uint32_t)n_cand, choice, n, (uint32_t)n_neg,
                                                                               neg_ent, neg_side);
    KGE_LAUNCH_CHECK();
    return KGE_OK;
}
