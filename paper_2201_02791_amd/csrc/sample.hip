// Draws from rows of scores: temperature, top-k, top-p and min-p, from random numbers that the caller gives.
//
//   weight of a score l in a row whose largest is m:  w = e^((l - m) / temperature), rounded to a multiple of 2^-b,
//   b = min(40, 62 - ceil(log2 columns));  minus infinity and NaN have none
//   in descending order of scores, equal ones in the order of their columns: top-k leaves the first k, top-p of those the
//   shortest beginning whose weights reach top_p of theirs, min-p what has at least min_p times the largest weight
//   the draw: the first column at which the sum of the weights left, in the order of columns, passes u times their total
//
// Weights are whole numbers below 2^62 in all, so that sums are exact: neither the order in which threads add nor the way in
// which rows are split shows in a result, and atomics on them change nothing.
//
// Nothing is sorted.  What top-k and top-p leave is all scores above one and, of those equal to it, the first few ("the cut").
// That score is found digit by digit of its bits, from counts or sums of weights by digit in LDS:
//   up to 1024 columns      a wavefront a row, digits of 8 bits, the row's keys in registers
//   up to 32768 at least    a block a row, digits of 11 or 12 bits; read again by each pass, or up to 16384 columns in registers
//   more, a small top_k     blocks take their part of a row and leave its first k scores (k_part_top); those, in the order
//                           of columns, are a short row for a block
//   more                    a launch for each digit; blocks add their parts' sums by digit to the row's in memory (k_long_digit)
//
// Bound by vector instructions where rows are many (65536 rows of 256, 64 draws each: 35 us, 3.9 TB/s; 16 rows of 2.9 million
// at top_p 0.9: 168 us in six launches), by waits where they are few (one row of a million at top_k 50: 9 + 18 us).
#include "common.h"

#include <math.h>

namespace {

typedef unsigned long long u64;

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
    int32_t n_cols, n_draws, bits, u64bit;
    const uint32_t *part_key;      // [n_rows][n_part]: a row's first scores, in the order of their columns, and the columns
    const int32_t *part_col;
    int32_t n_part;
    double per;                    // 256 / (T ln 2) of the call's temperature
};

__device__ __host__ __forceinline__ double per_of(float t) { return 369.329930467574627508 / (double)(t > 0.f ? t : 1.f); }

// a row's settings
struct Setting { float t, p, low; int32_t k; };

__device__ __forceinline__ Setting setting_of(const Sampling &how, int64_t r)
{
    Setting s;
    s.t = how.row_temperature ? how.row_temperature[r] : how.temperature;
    s.k = how.row_top_k ? how.row_top_k[r] : how.top_k;
    if (how.row_top_k && how.top_k > 0) s.k = s.k > 0 ? min(s.k, how.top_k) : how.top_k;
    s.p = how.row_top_p ? how.row_top_p[r] : how.top_p;
    s.low = how.row_min_p ? how.row_min_p[r] : how.min_p;
    if (!(s.t > 0.f)) { s.t = 1.f; s.k = 1; }
    return s;
}

// ---- scores as whole numbers in their order; 0: no weight.  Both zeros are one.

__device__ __forceinline__ uint32_t key_of(float l)
{
    const uint32_t b = __float_as_uint(l + 0.f);
    const uint32_t k = b ^ ((int32_t)b < 0 ? 0xffffffffu : 0x80000000u);
    return l > -INFINITY ? k : 0u;
}
__device__ __forceinline__ uint32_t key_in_order(float l)          // of a score that has a weight
{
    const uint32_t b = __float_as_uint(l + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float score_of(uint32_t key) { return __uint_as_float(key ^ ((int32_t)key < 0 ? 0x80000000u : 0xffffffffu)); }

// the largest score of keys up to this one: 0x7fffffff would be minus zero, which no key is, and which equals zero
__device__ __forceinline__ float score_upto(uint32_t key) { return score_of(key == 0x7fffffffu ? 0x7ffffffeu : key); }

struct __attribute__((packed, aligned(4))) F4 { float x[4]; };
struct __attribute__((packed, aligned(2))) H4 { uint16_t x[4]; };
struct __attribute__((packed, aligned(4))) U4 { uint32_t x[4]; };

// Where a row's keys come from: scores, or the first scores of its parts
template <bool BF16>
struct Scores {
    static constexpr bool PLAIN = true;
    const void *row;
    int32_t n;
    __device__ __forceinline__ float one(int32_t c) const { return BF16 ? __uint_as_float((uint32_t)((const uint16_t *)row)[c] << 16) : ((const float *)row)[c]; }
    // columns c .. c + 3, all of them in the row
    __device__ __forceinline__ void score4(int32_t c, float l[4]) const
    {
        if (BF16) {
            const H4 q = *reinterpret_cast<const H4 *>((const uint16_t *)row + c);
#pragma unroll
            for (int k = 0; k < 4; ++k) l[k] = __uint_as_float((uint32_t)q.x[k] << 16);
        } else {
            const F4 q = *reinterpret_cast<const F4 *>((const float *)row + c);
#pragma unroll
            for (int k = 0; k < 4; ++k) l[k] = q.x[k];
        }
    }
    __device__ __forceinline__ void whole4(int32_t c, uint32_t key[4]) const
    {
        float l[4];
        score4(c, l);
#pragma unroll
        for (int k = 0; k < 4; ++k) key[k] = key_of(l[k]);
    }
    // 1024 columns of a wavefront from column c0 on: 4 j .. + 3 of each 256 for lane j, minus infinity past the end
    __device__ __forceinline__ void run16(int32_t c0, int lane, float l[16]) const
    {
        const int32_t c = c0 + 4 * lane;
        if (c0 + 1024 <= n) {
#pragma unroll
            for (int j = 0; j < 4; ++j) score4(c + 256 * j, l + 4 * j);
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int32_t at = c + 256 * (j / 4) + j % 4;
                l[j] = at < n ? one(at) : -INFINITY;
            }
        }
    }
    __device__ __forceinline__ uint32_t key(int32_t c) const { return key_of(one(c)); }
    __device__ __forceinline__ int32_t column(int32_t c) const { return c; }
};
struct Parts {
    static constexpr bool PLAIN = false;         // there is a top-k
    const uint32_t *keys;
    const int32_t *col;
    int32_t n;
    __device__ __forceinline__ void whole4(int32_t c, uint32_t key[4]) const
    {
        const U4 q = *reinterpret_cast<const U4 *>(keys + c);
#pragma unroll
        for (int k = 0; k < 4; ++k) key[k] = q.x[k];
    }
    __device__ __forceinline__ uint32_t key(int32_t c) const { return keys[c]; }
    __device__ __forceinline__ int32_t column(int32_t c) const { return col[c]; }
};
// keys of columns c .. c + 3, 0 past the end
template <class Source>
__device__ __forceinline__ void get4(const Source &src, int32_t c, uint32_t key[4])
{
    if (c + 4 <= src.n) src.whole4(c, key);
    else {
#pragma unroll
        for (int k = 0; k < 4; ++k) key[k] = c + k < src.n ? src.key(c + k) : 0u;
    }
}

// ---- weights

// e^z, z = (l - m) / T <= 0, as 2^(x / 256), x = z 256 / ln 2: its nearest whole number n is left in the low bits of x + 3 2^51, what is
// left, r, goes through four terms of the exponential series of r ln 2 / 256 (the fifth is below 2^-54) and n mod 256 through a
// table of 2^(b + j / 256).  Adding 2^52 to the number of units rounds it.  No branch: what is too small is held at `least` and rounds to
// zero.  Double operations are as fast as float ones here.  A weight is off by one unit at most, and that only within 2^-7 of a unit
// of a half of one (x carries an error of |x| 2^-53, 2^-39 at most).
constexpr int POWERS = 256;
struct Weigh {
    double most, per, least;           // m, 256 / (T ln 2), and an x at which a weight rounds to zero
    const double *pow;                 // LDS: 2^(b + j / 256)
    uint32_t most_key;
    int32_t bits;
    bool endless;                      // m is infinite: what is equal to it has all the weight
    __device__ __forceinline__ void init(uint32_t key, float t, const Call &o, const double *table)
    {
        most_key = key;
        most = (double)score_of(key);
        per = o.how.row_temperature ? per_of(t) : o.per;
        bits = o.bits;
        least = -256.0 * (bits + 2);
        pow = table;
        endless = score_of(key) == INFINITY;
    }
    __device__ __forceinline__ u64 unit() const { return 1ull << bits; }
    // the weight of a score of a row whose largest is not infinite, in units, plus 2^52: rounded.  NaN and minus infinity: none
    __device__ __forceinline__ double raised(float l) const
    {
        const double x = __builtin_fmax(((double)l - most) * per, least);
        const double t = x + 0x1.8p52, r = x - (t - 0x1.8p52);
        constexpr double c1 = 0.0027076061740622863, c2 = c1 * c1 / 2.0, c3 = c2 * c1 / 3.0, c4 = c3 * c1 / 4.0;
        const int32_t i = (int32_t)__double_as_longlong(t);
        const double e = fma(r, fma(r, fma(r, fma(r, c4, c3), c2), c1), 1.0) * pow[i & (POWERS - 1)];
        const long long w = __double_as_longlong(e) + ((long long)((i & ~(POWERS - 1)) << 12) << 32);       // times 2^(i >> 8)
        return __longlong_as_double(w) + 0x1p52;
    }
    __device__ __forceinline__ double units(uint32_t key) const
    {
        if (endless) return key == most_key ? (double)unit() : 0.0;
        return raised(score_of(key)) - 0x1p52;
    }
    __device__ __forceinline__ u64 operator()(uint32_t key) const
    {
        if (endless) return key == most_key ? unit() : 0ull;
        return (u64)__double_as_longlong(raised(score_of(key))) & 0xfffffffffffffull;
    }
    // no score of a lower key has a weight: all that round to one unit or more are above m - T ln 2 (b + 2)
    __device__ __forceinline__ uint32_t lowest(float t) const
    {
        const float l = (float)(most - (double)t * (0.6931471805599453 * (bits + 2)));
        return l > -3.402823466e38f ? key_of(l) : 0x00800000u;
    }
};

__device__ __forceinline__ void fill_pow(double *table, int32_t bits)
{
    if (threadIdx.x < POWERS) table[threadIdx.x] = exp2((double)threadIdx.x * (1.0 / POWERS) + bits);
    __syncthreads();
}

// a whole number of up to 52 bits, from and to double
__device__ __forceinline__ u64 whole(double v) { return (u64)__double_as_longlong(v + 0x1p52) & 0xfffffffffffffull; }

// ---- sums over a wavefront and over a team of NT threads (64: a wavefront, more: the block)

template <int CTRL, int ROWS>
__device__ __forceinline__ u64 dpp_add(u64 v)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xf, false);
    return v + ((u64)hi << 32 | lo);
}
// inclusive sums over the lanes: within rows of 16, then the rows before
__device__ __forceinline__ u64 wave_scan(u64 v)
{
    v = dpp_add<0x111, 0xf>(v);
    v = dpp_add<0x112, 0xf>(v);
    v = dpp_add<0x114, 0xf>(v);
    v = dpp_add<0x118, 0xf>(v);
    v = dpp_add<0x142, 0xa>(v);
    return dpp_add<0x143, 0xc>(v);
}
// the same of whole numbers in double, below 2^53
__device__ __forceinline__ double wave_scan(double v)
{
    const auto step = [](double x, int lo, int hi) { return x + __longlong_as_double((long long)((u64)(uint32_t)hi << 32 | (uint32_t)lo)); };
#define SCAN_STEP(CTRL, ROWS) \
    v = step(v, __builtin_amdgcn_update_dpp(0, (int)__double_as_longlong(v), CTRL, ROWS, 0xf, false), \
             __builtin_amdgcn_update_dpp(0, (int)(__double_as_longlong(v) >> 32), CTRL, ROWS, 0xf, false));
    SCAN_STEP(0x111, 0xf)
    SCAN_STEP(0x112, 0xf)
    SCAN_STEP(0x114, 0xf)
    SCAN_STEP(0x118, 0xf)
    SCAN_STEP(0x142, 0xa)
    SCAN_STEP(0x143, 0xc)
#undef SCAN_STEP
    return v;
}
__device__ __forceinline__ u64 lane_of(u64 v, int lane)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane);
    return (u64)hi << 32 | lo;
}
__device__ __forceinline__ double lane_of(double v, int lane) { return __longlong_as_double((long long)lane_of((u64)__double_as_longlong(v), lane)); }
__device__ __forceinline__ u64 wave_sum(u64 v) { return lane_of(wave_scan(v), 63); }
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) { return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false)); }
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    v = dpp_max<0x111, 0xf>(v);
    v = dpp_max<0x112, 0xf>(v);
    v = dpp_max<0x114, 0xf>(v);
    v = dpp_max<0x118, 0xf>(v);
    v = dpp_max<0x142, 0xa>(v);
    v = dpp_max<0x143, 0xc>(v);
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

template <int NT>
struct Team {
    static constexpr int WAVES = NT / 64;
    // LDS written by the team is there for the team
    static __device__ __forceinline__ void sync()
    {
        if (NT == 64) {
            __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "workgroup");
            __builtin_amdgcn_wave_barrier();
        } else __syncthreads();
    }
    static __device__ __forceinline__ int tid() { return NT == 64 ? (int)(threadIdx.x & 63) : (int)threadIdx.x; }
    // inclusive sums over the threads, and their total; s: WAVES words of LDS
    template <class N>
    static __device__ __forceinline__ N scan(N v, void *words, N *total)
    {
        N *s = (N *)words;
        v = wave_scan(v);
        if (NT == 64) { *total = lane_of(v, 63); return v; }
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 63) s[wave] = v;
        __syncthreads();
        const int at = threadIdx.x & 63;
        const N sums = wave_scan(at < WAVES ? s[at] : N(0));
        __syncthreads();
        *total = lane_of(sums, WAVES - 1);
        return v + (wave ? lane_of(sums, wave - 1) : N(0));
    }
    static __device__ __forceinline__ uint32_t most(uint32_t v, u64 *s)
    {
        v = wave_max(v);
        if (NT == 64) return v;
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
        __syncthreads();
        const int at = threadIdx.x & 63;
        v = wave_max(at < WAVES ? (uint32_t)s[at] : 0u);
        __syncthreads();
        return v;
    }
};

// ---- the cut

struct Cut {
    uint32_t key;                  // scores above it are left, 0: all
    bool every;                    // all that are equal to it are, else the first `ties` of them
    u64 ties;
};

// The search for one: which = 0 by counts (top-k), 1 by weights (top-p).  Digits are those of a key's distance from `base`, which is not above
// the key that is searched: few digits where the keys lie close together, and sums that spread over all values of a digit.
constexpr uint32_t LEAST_KEY = 0x00800000u;   // of the lowest number
template <int BITS>
struct Search {
    u64 goal, above;               // the sum that the scores from the cut on reach; the sum of the digits above what is found
    uint32_t base, found;          // digits so far
    int32_t shift, width;          // of the digit that is next
    bool open;
    __device__ __forceinline__ void begin(uint32_t low, uint32_t most)
    {
        goal = above = 0ull;
        base = low; found = 0u;
        const int bits = max(1, 32 - (int)__builtin_clz((most - low) | 1u));
        shift = max(bits - BITS, 0);
        width = bits - shift;
        open = true;
    }
    __device__ __forceinline__ bool in(uint32_t key) const { return key >= base && (((key - base) >> shift) >> width) == found; }
    __device__ __forceinline__ uint32_t digit(uint32_t key) const { return ((key - base) >> shift) & ((1u << width) - 1u); }
    __device__ __forceinline__ void step(int digit, u64 more)
    {
        above += more;
        found = found << width | (uint32_t)digit;
        open = shift > 0;
        width = min(BITS, shift);
        shift -= width;
    }
    __device__ __forceinline__ uint32_t key() const { return base + found; }
    // the least and the largest key that have the digits found
    __device__ __forceinline__ uint32_t first() const { return base + ((found << width) << shift); }
    __device__ __forceinline__ u64 last() const { return first() + ((1ull << (width + shift)) - 1ull); }
};

// The digit at which the sums, from the largest digit down, first reach `goal` (1 or more, their total at most); the sum of the digits above it
// and its own
template <int NT, int BITS>
__device__ __forceinline__ u64 digit_total(const u64 *hist, u64 (&v)[(1 << BITS) / NT], u64 *upto, u64 *s)
{
    constexpr int PER = (1 << BITS) / NT;
    static_assert(PER >= 1, "a thread has a digit");
    const int hi = (1 << BITS) - 1 - PER * Team<NT>::tid();
    u64 sum = 0ull, total;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        v[k] = hist[hi - k];
        sum += v[k];
    }
    *upto = Team<NT>::scan(sum, s, &total);
    return total;
}
template <int NT, int BITS>
__device__ __forceinline__ int digit_at(const u64 (&v)[(1 << BITS) / NT], u64 upto, u64 goal, u64 *s_found, u64 *above, u64 *own, const uint32_t *counts = nullptr)
{
    constexpr int PER = (1 << BITS) / NT;
    const int hi = (1 << BITS) - 1 - PER * Team<NT>::tid();
    u64 before = upto;
#pragma unroll
    for (int k = 0; k < PER; ++k) before -= v[k];
    if (before < goal && goal <= upto) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if (before < goal && goal <= before + v[k]) {
                s_found[0] = hi - k; s_found[1] = before; s_found[2] = v[k];
                if (counts) s_found[3] = counts[k];
            }
            before += v[k];
        }
    }
    Team<NT>::sync();
    const int digit = (int)s_found[0];
    *above = s_found[1]; *own = s_found[2];
    Team<NT>::sync();
    return digit;
}

// what the sums have to reach, from their total; 0: nothing is cut
__device__ __forceinline__ u64 goal_of_count(u64 all, const Setting &set) { return all < (u64)set.k ? 0ull : (u64)set.k; }
__device__ __forceinline__ u64 goal_of_weight(u64 all, const Setting &set)
{
    const double g = ceil((double)set.p * (double)all);
    const u64 goal = g < 1.0 ? 1ull : (u64)g;
    return goal > all ? all : goal;
}

// One score left is the largest, of equal ones the first: nothing to search
__device__ __forceinline__ bool cuts(int which, const Setting &set, int32_t n) { return set.k != 1 && (which == 0 ? set.k > 0 && set.k < n : set.p < 1.f); }
__device__ __forceinline__ Cut first_cut(const Setting &set, uint32_t most) { return set.k == 1 ? Cut{most, false, 1ull} : Cut{0u, true, 0ull}; }

// a search has ended; `own`: the sum at its key
template <class S>
__device__ __forceinline__ Cut cut_at(int which, const S &x, u64 own, const Cut &was, const Weigh &weigh)
{
    Cut c;
    c.key = x.key();
    if (which == 0) {
        c.ties = x.goal - x.above;
        c.every = c.ties == own;
    } else {
        const u64 w = weigh(c.key);
        c.ties = (x.goal - x.above + w - 1ull) / w;
        c.every = c.ties * w == own && (c.key != was.key || was.every);
    }
    return c;
}

// A row's keys, TILES tiles of 4 columns a thread at a time: thread t of NT has columns 4 (NT i + t) .. + 3 of tile i.  ONE: the row has no
// more, and they stay in registers, with the weights of those that top-k leaves where a wavefront has the row (a thread of a block of 1024 has 128
// registers, too few for them); else every pass reads them again, from the caches, and weighs again.
template <int NT, int TILES, bool ONE, class Source>
struct Keys {
    static constexpr int V = 4 * TILES, BATCH = NT * V;
    static constexpr bool HELD = ONE && NT == 64;
    const Source &src;
    uint32_t key[V];
    double w[HELD ? V : 1];
    __device__ __forceinline__ void weigh_all(const Weigh &weigh, const Cut &cut)
    {
        if (!HELD) return;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            w[HELD ? i : 0] = 0.0;
            if (key[i] >= cut.key) w[HELD ? i : 0] = weigh.units(key[i]);
        }
    }
    __device__ __forceinline__ double weight(int i, const Weigh &weigh) const
    {
        if (HELD) return w[HELD ? i : 0];
        uint32_t k = key[i];
        asm volatile("" : "+v"(k));              // the compiler would hold the last pass's weights, in scratch memory
        return weigh.units(k);
    }
    __device__ __forceinline__ explicit Keys(const Source &s) : src(s) { if (ONE) load(0); }
    __device__ __forceinline__ void load(int32_t c0)
    {
        // inside the row no branch parts the loads
        if (c0 + BATCH <= src.n) {
#pragma unroll
            for (int i = 0; i < TILES; ++i) src.whole4(c0 + 4 * (NT * i + Team<NT>::tid()), key + 4 * i);
        } else {
#pragma unroll
            for (int i = 0; i < TILES; ++i) get4(src, c0 + 4 * (NT * i + Team<NT>::tid()), key + 4 * i);
        }
    }
    // f(first column) for each batch from column c0 on, whose keys are then in `key`
    template <class F>
    __device__ __forceinline__ void each(int32_t c0, F f)
    {
        if (ONE) { f(0); return; }
#pragma unroll 1
        for (; c0 < src.n; c0 += BATCH) {
            load(c0);
            f(c0);
        }
    }
};

// The cut of top-k for a wavefront's row, bit by bit from the first at which the largest key and a lower bound differ: a comparison and a count of
// lanes for each key is all a bit takes.  Ends where exactly k keys are not below what is tried.
template <class K>
__device__ __forceinline__ void find_kth(K &keys, int32_t k, uint32_t low, uint32_t most, Cut &cut)
{
    const auto from = [&](uint32_t at) {         // keys not below it
        int n = 0;
#pragma unroll
        for (int i = 0; i < K::V; ++i) n += (int)__popcll(__ballot(keys.key[i] >= at));
        return n;
    };
    if (from(low) < k) return;                   // fewer scores than k
    int bits = 32 - (int)__builtin_clz((most ^ low) | 1u), n = 0;
    uint32_t at = bits < 32 ? most >> bits << bits : 0u;
    for (; bits > 0; --bits) {
        const uint32_t next = at | 1u << (bits - 1);
        const int here = from(next);
        if (here < k) continue;
        at = next;
        n = here;
        if (n == k) break;
    }
    // the least of those keys
    uint32_t least = 0xffffffffu;
#pragma unroll
    for (int i = 0; i < K::V; ++i) least = min(least, keys.key[i] >= at ? keys.key[i] : 0xffffffffu);
    least = ~wave_max(~least);
    const int above = from(least + 1u), all = from(least);
    cut = Cut{least, all == k, (u64)(k - above)};
}

// limit: as soon as no more than so many scores are at or above the least that has the digits found, the search for top-k's cut ends; the cut is
// then that score's key, and true is returned: what is left holds the first k, and may hold more
template <int NT, int BITS, class K>
__device__ __forceinline__ bool find_cut(int which, uint32_t limit, K &keys, const Setting &set, const Weigh &weigh, uint32_t low, uint32_t most, Cut &cut, u64 *hist, u64 *s,
                                         u64 *s_found)
{
    if (!cuts(which, set, keys.src.n)) return false;
    // a wavefront's row has up to 1024 scores: their number fits beside their weights, and where a digit has one score the search ends
    constexpr int PACK = K::HELD ? 11 : 0;
    const int tid = Team<NT>::tid();
    Search<BITS> x;
    x.begin(low, most);
#pragma unroll 1
    for (bool first = true; x.open; first = false) {
        for (int i = tid; i < 1 << BITS; i += NT) hist[i] = 0ull;
        Team<NT>::sync();
        keys.each(0, [&](int32_t) {
#pragma unroll
            for (int i = 0; i < K::V; ++i) {
                const uint32_t key = keys.key[i];
                if (!x.in(key) || (which == 1 && key <= cut.key)) continue;
                const u64 w = which == 0 ? 1ull : whole(keys.weight(i, weigh));
                if (w) atomicAdd(&hist[x.digit(key)], PACK ? w << PACK | 1ull : w);
            }
        });
        if (which == 1 && tid == 0 && cut.key && x.in(cut.key)) {
            const u64 w = cut.ties * weigh(cut.key);
            atomicAdd(&hist[x.digit(cut.key)], PACK ? w << PACK | cut.ties : w);
        }
        Team<NT>::sync();
        u64 v[(1 << BITS) / NT], upto, more, own;
        uint32_t counts[(1 << BITS) / NT];
        const u64 all = digit_total<NT, BITS>(hist, v, &upto, s) >> PACK;
        upto >>= PACK;
#pragma unroll
        for (int k = 0; k < (1 << BITS) / NT; ++k) {
            counts[k] = (uint32_t)v[k] & ((1u << PACK) - 1u);
            v[k] >>= PACK;
        }
        if (first) x.goal = which == 0 ? goal_of_count(all, set) : goal_of_weight(all, set);
        if (x.goal == 0ull) return false;
        const int digit = digit_at<NT, BITS>(v, upto, x.goal - x.above, s_found, &more, &own, PACK ? counts : nullptr);
        const bool lone = PACK && s_found[3] == 1ull;
        Team<NT>::sync();
        x.step(digit, more);
        if (lone && (x.first() > cut.key || cut.every)) {
            cut = Cut{x.first(), true, 1ull};
            return true;
        }
        if (which == 0 && x.above + own <= (u64)limit) {
            cut = Cut{x.first(), true, ~0ull};
            return true;
        }
        if (!x.open) cut = cut_at(which, x, own, cut, weigh);
    }
    return false;
}

// a lower bound of the k-th largest key, from the threads' largest: NT scores at least are not below the least of those
template <int NT>
__device__ __forceinline__ uint32_t low_of(uint32_t mine, int32_t k, u64 *s)
{
    if (k > NT) return LEAST_KEY;
    return max(~Team<NT>::most(~mine, s), LEAST_KEY);
}

// ---- draws

__device__ __forceinline__ double random_of(const Call &o, int64_t at) { return o.u64bit ? ((const double *)o.u)[at] : (double)((const float *)o.u)[at]; }

__device__ __forceinline__ u64 goal_of_draw(const Call &o, int64_t at, u64 total)
{
    const double reach = random_of(o, at) * (double)total;
    return reach >= (double)total ? total - 1ull : reach > 0.0 ? min((u64)reach, total - 1ull) : 0ull;
}
// totals that a double holds
__device__ __forceinline__ double goal_of_draw(const Call &o, int64_t at, double total)
{
    return fmin(fmax(floor(random_of(o, at) * total), 0.0), total - 1.0);
}

__device__ __forceinline__ void answer(const Call &o, int64_t at, int32_t column, double w, double inverse)
{
    o.choice[at] = column;
    if (o.prob) o.prob[at] = (float)(w * inverse);
}
// 1 / total, to 2^-50: the instruction's 2^-14 or better squared twice
__device__ __forceinline__ double inverse_of(double total)
{
    double y = __builtin_amdgcn_rcp(total);
    y = fma(fma(-total, y, 1.0), y, y);
    return fma(fma(-total, y, 1.0), y, y);
}

// the least weight that min-p leaves
__device__ __forceinline__ u64 least_weight(const Setting &set, const Weigh &weigh)
{
    if (!(set.low > 0.f)) return 1ull;
    const double low = set.low > 1.f ? 1.0 : (double)set.low;
    const u64 least = (u64)ceil(low * (double)weigh.unit());
    return least ? least : 1ull;
}

__device__ __forceinline__ u64 ties_of(const uint32_t key[4], const Cut &cut)
{
    u64 n = 0ull;
#pragma unroll
    for (int k = 0; k < 4; ++k) n += key[k] == cut.key ? 1ull : 0ull;
    return n;
}

// The weights w that are left of 4 columns a lane, 256 columns of a wavefront in order: of keys above the cut and of the ties that are, and no fewer
// units than `least`; *equal: ties of the cut before them, counted on
__device__ __forceinline__ void left4(const uint32_t key[4], const Cut &cut, u64 least, u64 *equal, double w[4])
{
    if (least == 1ull && cut.key == 0u) return;
    if (least > 1ull) {
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = w[k] >= (double)least ? w[k] : 0.0;
    }
    if (cut.every) {
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = key[k] >= cut.key ? w[k] : 0.0;
        return;
    }
    const u64 mine = ties_of(key, cut), upto = wave_scan(mine);
    u64 rank = *equal + upto - mine;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const bool tie = key[k] == cut.key;
        w[k] = key[k] > cut.key || (tie && rank < cut.ties) ? w[k] : 0.0;
        rank += tie ? 1ull : 0ull;
    }
    *equal += lane_of(upto, 63);
}

// The first of n sums, ascending, above the goal
template <class N>
__device__ __forceinline__ int first_above(const N *sums, int n, N goal)
{
    int lo = 0, hi = n - 1;
#pragma unroll 1
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid] > goal) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// Of 256 columns, 4 a lane from column c on, the one at which the weights left pass the goal, if one does; `before`: the weights before them.
// The weights left of them all
template <class Source>
__device__ __forceinline__ u64 pick4(const Call &o, int64_t at, const Source &src, int32_t c, const uint32_t key[4], const Cut &cut, const Weigh &weigh, u64 least,
                                     u64 *equal, u64 goal, u64 before, u64 total)
{
    double w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = weigh.units(key[k]);
    left4(key, cut, least, equal, w);
    const double here = w[0] + w[1] + w[2] + w[3], upto = wave_scan(here);
    u64 from = before + whole(upto - here);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const u64 x = whole(w[k]);
        if (goal >= from && goal < from + x) answer(o, at, src.column(c + k), w[k], inverse_of((double)total));
        from += x;
    }
    return whole(lane_of(upto, 63));
}

constexpr int RUN = 256;           // columns that a wavefront weighs at once
constexpr int64_t ROW_MOST = RUN * 1024;      // columns of a row that a block takes: a thread has a run

// A row of which up to FEW scores, top-k's among them, are at or above the cut: one wavefront has them, one a lane, and counts for each those before
// it, by score and by column
constexpr int FEW = 64;
template <int NT, class K>
__device__ __forceinline__ void draw_few(const Call &o, int64_t first, K &keys, const Setting &set, const Weigh &weigh, const Cut &cut, uint32_t *list, u64 *s_found)
{
    uint32_t *count = (uint32_t *)s_found;                       // list: keys, then columns, then sums
    if (threadIdx.x == 0) *count = 0u;
    __syncthreads();
    keys.each(0, [&](int32_t c0) {
#pragma unroll
        for (int i = 0; i < K::V; ++i) {
            if (keys.key[i] < cut.key) continue;
            const uint32_t at = atomicAdd(count, 1u);
            list[at] = keys.key[i];
            list[FEW + at] = c0 + 4 * (NT * (i / 4) + threadIdx.x) + i % 4;
        }
    });
    __syncthreads();
    if (threadIdx.x < 64) {
        typedef Team<64> W;
        u64 *sum = (u64 *)(list + 2 * FEW);
        const int n = __builtin_amdgcn_readfirstlane((int)*count), lane = threadIdx.x;
        const uint32_t key = lane < n ? list[lane] : 0u, at = lane < n ? list[FEW + lane] : ~0u;
        const u64 order = (u64)key << 32 | (uint32_t)~at;
        int by_score = 0, by_column = 0;
        for (int j = 0; j < n; ++j) {
            by_score += lane_of(order, j) > order;
            by_column += (uint32_t)__builtin_amdgcn_readlane((int)at, j) < at;
        }
        if (lane >= n) by_score = by_column = lane;
        u64 w = lane < n && by_score < set.k ? weigh(key) : 0ull;
        if (set.p < 1.f) {
            sum[by_score] = w;
            W::sync();
            const u64 mine = sum[lane], upto = wave_scan(mine);
            W::sync();
            sum[lane] = upto - mine;
            W::sync();
            if (sum[by_score] >= goal_of_weight(lane_of(upto, 63), set)) w = 0ull;
            W::sync();
        }
        if (w < least_weight(set, weigh)) w = 0ull;
        sum[by_column] = w;
        W::sync();
        const u64 mine = sum[lane], upto = wave_scan(mine), total = lane_of(upto, 63);
        W::sync();
        sum[lane] = upto - mine;
        W::sync();
        const u64 before = sum[by_column];
        const double inverse = inverse_of((double)total);
        for (int32_t i = 0; i < o.n_draws; ++i) {
            const u64 goal = goal_of_draw(o, first + i, total);
            if (goal >= before && goal < before + w) answer(o, first + i, keys.src.column((int32_t)at), (double)w, inverse);
        }
    }
    __syncthreads();
}

// The sums by column of a row that a wavefront holds (w: its weights left, 4 columns a lane a tile), 1024 weights of 2^40 units at most, which a
// double holds; a lane finds a draw by halving.  A place is left free after every 32 sums: lanes that halve read places a power of two apart, which would
// be in a few of the banks (65536 rows of 256, 64 draws: 46 us without, and with a search that takes any length, 40)
constexpr int padded(int i) { return i + i / 32; }
template <int TILES, class W, class Source>
__device__ __forceinline__ void draw_by_column(const Call &o, int64_t first, const Source &src, double *to, W weights)
{
    typedef Team<64> T;
    const int lane = T::tid();
    double total = 0.0;
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        double w[4];
        weights(i, w);
        w[1] += w[0]; w[2] += w[1]; w[3] += w[2];
        const double upto = wave_scan(w[3]), base = total + (upto - w[3]);
#pragma unroll
        for (int k = 0; k < 4; ++k) to[padded(256 * i) + 4 * lane + (lane >> 3) + k] = base + w[k];
        total += lane_of(upto, 63);
    }
    T::sync();
    const double inverse = inverse_of(total);
    for (int32_t i = lane; i < o.n_draws; i += 64) {
        const double goal = goal_of_draw(o, first + i, total);
        int place = 0;                                           // of the first sum above the goal
#pragma unroll
        for (int step = 128 * TILES; step > 0; step /= 2)
            if (to[place + padded(step - 1)] <= goal) place += padded(step);
        const int at = place - place / 33;
        answer(o, first + i, src.column(at), to[place] - (place ? to[place - 1 - (at % 32 == 0)] : 0.0), inverse);
    }
    T::sync();
}

// The sums of the runs of 256 columns are there (sums; ties: of the cut, by runs, their number before each); a wavefront weighs the run of a draw
// again
template <int NT, class Source>
__device__ __forceinline__ void draw_by_run(const Call &o, int64_t first, const Source &src, const Cut &cut, const Weigh &weigh, u64 least, u64 *sums, const u64 *ties, u64 *s)
{
    typedef Team<NT> T;
    const int tid = T::tid(), wave = NT == 64 ? 0 : (int)(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int runs = (src.n + RUN - 1) / RUN;
    u64 total;
    T::sync();
    const u64 mine = tid < runs ? sums[tid] : 0ull;
    const u64 upto = T::scan(mine, s, &total);
    if (tid < runs) sums[tid] = upto;
    T::sync();
    for (int32_t i = wave; i < o.n_draws; i += NT / 64) {
        const u64 goal = goal_of_draw(o, first + i, total);
        const int run = first_above(sums, runs, goal);
        const int32_t c = RUN * run + 4 * lane;
        uint32_t again[4];
        get4(src, c, again);
        u64 equal = cut.every ? 0ull : ties[run];
        pick4(o, first + i, src, c, again, cut, weigh, least, &equal, goal, run ? sums[run - 1] : 0ull, total);
    }
    T::sync();
}

// A row of which neither top-k nor top-p takes anything: its scores are no more than numbers, their order does not matter
template <int NT, int TILES, bool ONE, bool BF16>
__device__ __forceinline__ void draw_plain(const Call &o, int64_t first, const Setting &set, const Scores<BF16> &src, u64 *sums, u64 *s, const double *pow)
{
    typedef Team<NT> T;
    constexpr int V = 4 * TILES, BATCH = NT * V, WAVES = NT / 64;
    const int wave = NT == 64 ? 0 : (int)(threadIdx.x >> 6), lane = threadIdx.x & 63;
    float l[V];
    const auto load = [&](int32_t c0) {
        if (c0 + BATCH <= src.n) {
#pragma unroll
            for (int i = 0; i < TILES; ++i) src.score4(c0 + 4 * (NT * i + T::tid()), l + 4 * i);
        } else {
#pragma unroll
            for (int i = 0; i < TILES; ++i) {
                const int32_t c = c0 + 4 * (NT * i + T::tid());
                if (c + 4 <= src.n) src.score4(c, l + 4 * i);
                else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) l[4 * i + k] = c + k < src.n ? src.one(c + k) : -INFINITY;
                }
            }
        }
    };
    float mine = -INFINITY;
#pragma unroll 1
    for (int32_t c0 = 0; c0 < src.n; c0 += BATCH) {
        load(c0);
#pragma unroll
        for (int k = 0; k < V; ++k) mine = l[k] > mine ? l[k] : mine;          // the instruction for the larger one makes NaN of a signalling NaN
    }
    const uint32_t most = T::most(key_of(mine), s);
    if (most == 0u) {
        for (int32_t i = T::tid(); i < o.n_draws; i += NT) answer(o, first + i, -1, 0.0, 1.0);
        return;
    }
    Weigh weigh;
    weigh.init(most, set.t, o, pow);
    const u64 least = least_weight(set, weigh);
    const double fewest = (double)least;
    const auto weigh4 = [&](int i, double w[4]) {
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = weigh.raised(l[4 * i + k]) - 0x1p52;
        if (weigh.endless) {
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = l[4 * i + k] == INFINITY ? (double)weigh.unit() : 0.0;
        }
        if (least > 1ull) {
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = w[k] >= fewest ? w[k] : 0.0;
        }
    };
    if constexpr (ONE && NT == 64) draw_by_column<TILES>(o, first, src, (double *)sums, weigh4);
    else {
        const int runs = (src.n + RUN - 1) / RUN;
#pragma unroll 1
        for (int32_t c0 = 0; c0 < src.n; c0 += BATCH) {
            if (!ONE) load(c0);
#pragma unroll
            for (int i = 0; i < TILES; ++i) {
                double w[4];
                weigh4(i, w);
                const u64 sum = whole(lane_of(wave_scan(w[0] + w[1] + w[2] + w[3]), 63));
                const int run = c0 / RUN + i * WAVES + wave;
                if (lane == 0 && run < runs) sums[run] = sum;
            }
        }
        draw_by_run<NT>(o, first, src, Cut{0u, true, 0ull}, weigh, least, sums, nullptr, s);
    }
}

// One row.  Up to 1024 columns the sums by column are in LDS, and a lane finds a draw by halving; beyond, the sums by runs of 256
// columns are (sums[run]: of runs 0 .. run; ties[run], where not all ties are left: their number before the run), and a wavefront
// weighs the run of a draw again.
template <int NT, int TILES, bool ONE, int BITS, class Source>
__device__ __forceinline__ void draw_row(const Call &o, int64_t r, const Source &src, u64 *hist, u64 *sums, u64 *ties, u64 *s, u64 *s_found, const double *pow)
{
    typedef Team<NT> T;
    typedef Keys<NT, TILES, ONE, Source> K;
    constexpr int V = K::V, WAVES = NT / 64;
    const int tid = T::tid(), wave = NT == 64 ? 0 : (int)(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const Setting set = setting_of(o.how, r);
    if constexpr (Source::PLAIN) {
        if (set.k != 1 && !cuts(0, set, src.n) && !cuts(1, set, src.n)) {
            draw_plain<NT, TILES, ONE>(o, r * o.n_draws, set, src, sums, s, pow);
            return;
        }
    }
    K keys(src);
    uint32_t mine = 0u;
    keys.each(0, [&](int32_t) {
#pragma unroll
        for (int i = 0; i < V; ++i) mine = max(mine, keys.key[i]);
    });
    const uint32_t most = T::most(mine, s);
    const int64_t first = r * o.n_draws;
    if (most == 0u) {                                            // a row without weights
        for (int32_t i = tid; i < o.n_draws; i += NT) answer(o, first + i, -1, 0.0, 1.0);
        return;
    }
    if (set.k == 1) {                                            // the first column of the largest score
        uint32_t at = ~0u;
        keys.each(0, [&](int32_t c0) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (keys.key[i] == most) at = min(at, (uint32_t)(c0 + 4 * (NT * (i / 4) + tid) + i % 4));
        });
        at = ~T::most(~at, s);
        for (int32_t i = tid; i < o.n_draws; i += NT) answer(o, first + i, src.column((int32_t)at), 1.0, 1.0);
        return;
    }
    Weigh weigh;
    weigh.init(most, set.t, o, pow);
    Cut cut{0u, true, 0ull};
    if (cuts(0, set, src.n)) {
        const uint32_t low = low_of<NT>(mine, set.k, s);
        if constexpr (K::HELD) find_kth(keys, set.k, low, most, cut);
        else {
            const uint32_t limit = NT > 64 && set.k <= FEW && o.n_draws <= FEW ? FEW : 0u;
            const bool few = find_cut<NT, BITS>(0, limit, keys, set, weigh, low, most, cut, hist, s, s_found);
            if constexpr (NT > 64) {
                if (few) {
                    draw_few<NT>(o, first, keys, set, weigh, cut, (uint32_t *)sums, s_found);
                    return;
                }
            }
        }
    }
    keys.weigh_all(weigh, cut);
    find_cut<NT, BITS>(1, 0u, keys, set, weigh, max(cut.key, weigh.lowest(set.t)), most, cut, hist, s, s_found);
    const u64 least = least_weight(set, weigh);
    if constexpr (K::HELD) {
        u64 equal = 0ull;                                        // ties in the tiles before
        draw_by_column<TILES>(o, first, src, (double *)sums, [&](int i, double w[4]) {
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = keys.weight(4 * i + k, weigh);
            left4(keys.key + 4 * i, cut, least, &equal, w);
        });
    } else {
        const int runs = (src.n + RUN - 1) / RUN;
        if (!cut.every) {
            keys.each(0, [&](int32_t c0) {
#pragma unroll
                for (int i = 0; i < TILES; ++i) {
                    const u64 mine = wave_sum(ties_of(keys.key + 4 * i, cut));
                    const int run = c0 / RUN + i * WAVES + wave;
                    if (lane == 0 && run < runs) ties[run] = mine;
                }
            });
            T::sync();
            const u64 mine = tid < runs ? ties[tid] : 0ull;
            u64 all;
            const u64 upto = T::scan(mine, s, &all);
            if (tid < runs) ties[tid] = upto - mine;
            T::sync();
        }
        keys.each(0, [&](int32_t c0) {
#pragma unroll
            for (int i = 0; i < TILES; ++i) {
                const int run = c0 / RUN + i * WAVES + wave;
                u64 equal = cut.every || run >= runs ? 0ull : ties[run];
                double w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = keys.weight(4 * i + k, weigh);
                left4(keys.key + 4 * i, cut, least, &equal, w);
                const u64 sum = whole(lane_of(wave_scan(w[0] + w[1] + w[2] + w[3]), 63));
                if (lane == 0 && run < runs) sums[run] = sum;
            }
        });
        draw_by_run<NT>(o, first, src, cut, weigh, least, sums, ties, s);
    }
}

// What a kernel's rows are: scores, scores of which the host knows that nothing is cut (half the registers and no sums by digit: 65536 rows of 256, 64
// draws, 40 us as a branch of the first kernel, 35 here), the first scores of parts
enum { CUT, PLAIN, PARTS };
// NT 64: four rows a block, a wavefront each.  Wavefronts at once to a SIMD: what LDS and registers leave room for
constexpr int waves_of(int nt, int tiles, bool one, int kind)
{
    if (kind == PLAIN) return nt == 64 && one ? (tiles == 1 ? 8 : 4) : nt == 1024 ? 4 : 6;
    return nt == 64 && one ? (tiles == 1 ? 5 : 3) : 4;
}
template <bool BF16, int NT, int TILES, bool ONE, int KIND>
__global__ __launch_bounds__(NT == 64 ? 256 : NT) __attribute__((amdgpu_waves_per_eu(waves_of(NT, TILES, ONE, KIND)))) void k_rows(Call o)
{
    constexpr int BITS = NT == 64 ? 8 : NT == 256 ? 11 : 12, TEAMS = NT == 64 ? 4 : 1, COLUMNS = 4 * TILES * NT;
    constexpr bool BY_COLUMN = ONE && NT == 64;
    __shared__ u64 s_hist[TEAMS][KIND == PLAIN ? 1 : 1 << BITS], s_sums[TEAMS][BY_COLUMN ? padded(COLUMNS) : NT], s_ties[TEAMS][BY_COLUMN || KIND == PLAIN ? 1 : NT];
    __shared__ u64 s_part[TEAMS][16], s_found[TEAMS][4];
    __shared__ double s_pow[POWERS];
    fill_pow(s_pow, o.bits);
    const int team = NT == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    for (int64_t r = (int64_t)blockIdx.x * TEAMS + team; r < o.n_rows; r += (int64_t)gridDim.x * TEAMS) {
        if constexpr (KIND == PARTS) {
            const Parts src{o.part_key + r * o.n_part, o.part_col + r * o.n_part, o.n_part};
            draw_row<NT, TILES, ONE, BITS>(o, r, src, s_hist[team], s_sums[team], s_ties[team], s_part[team], s_found[team], s_pow);
        } else {
            const Scores<BF16> src{(const char *)o.scores + r * o.lds * (BF16 ? 2 : 4), o.n_cols};
            if constexpr (KIND == PLAIN) draw_plain<NT, TILES, ONE>(o, r * o.n_draws, setting_of(o.how, r), src, s_sums[team], s_part[team], s_pow);
            else draw_row<NT, TILES, ONE, BITS>(o, r, src, s_hist[team], s_sums[team], s_ties[team], s_part[team], s_found[team], s_pow);
        }
    }
}

// ---- long rows, few scores left: the first k of a row are among the first k of its parts

template <bool BF16, int NT, int TILES>
__global__ __launch_bounds__(NT) void k_part_top(Call o, int64_t row0, int32_t parts, int32_t most_k, int32_t slots, uint32_t *__restrict__ part_key, int32_t *__restrict__ part_col)
{
    typedef Team<NT> T;
    constexpr int BITS = NT == 1024 ? 12 : 11;
    __shared__ u64 s_hist[1 << BITS], s_part[16], s_found[4];
    const int64_t r = row0 + blockIdx.x / (unsigned)parts;
    const int32_t part = (int32_t)(blockIdx.x % (unsigned)parts);
    constexpr int COLUMNS = 4 * TILES * NT;
    const int32_t c0 = part * COLUMNS, n = min(COLUMNS, o.n_cols - c0);
    const Scores<BF16> src{(const char *)o.scores + (r * o.lds + c0) * (BF16 ? 2 : 4), n};
    Setting set = setting_of(o.how, r);
    set.k = set.k > 0 ? min(set.k, most_k) : most_k;
    const int tid = T::tid();
    Keys<NT, TILES, true, Scores<BF16>> keys(src);
    Cut cut{0u, true, 0ull};
    if (set.k == 1) {
        uint32_t most = 0u;
#pragma unroll
        for (int i = 0; i < 4 * TILES; ++i) most = max(most, keys.key[i]);
        cut = first_cut(set, T::most(most, s_part));
    } else {
        const Weigh none{};
        uint32_t mine = 0u;
#pragma unroll
        for (int i = 0; i < 4 * TILES; ++i) mine = max(mine, keys.key[i]);
        const uint32_t most = T::most(mine, s_part);
        if (most) find_cut<NT, BITS>(0, (uint32_t)slots, keys, set, none, low_of<NT>(mine, set.k, s_part), most, cut, s_hist, s_part, s_found);
    }
    uint32_t *out_key = part_key + (r * parts + part) * slots;
    int32_t *out_col = part_col + (r * parts + part) * slots;
    u64 base = 0ull;                                             // scores written, and in the upper half ties met
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        const uint32_t *key = keys.key + 4 * i;
        u64 mine = 0ull;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t x = key[k];
            mine += x > cut.key ? 1ull : x == cut.key && x ? 1ull << 32 : 0ull;
        }
        u64 all;
        u64 before = base + T::scan(mine, s_part, &all) - mine;
        base += all;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t x = key[k];
            const bool tie = x == cut.key && x;
            const u64 ties = min(before >> 32, cut.ties);
            if (x > cut.key || (tie && (before >> 32) < cut.ties)) {
                const uint32_t at = (uint32_t)before + (uint32_t)ties;
                out_key[at] = x;
                out_col[at] = c0 + 4 * (NT * i + tid) + k;
            }
            before += x > cut.key ? 1ull : tie ? 1ull << 32 : 0ull;
        }
    }
    const int32_t written = (int32_t)((uint32_t)base + (uint32_t)min(base >> 32, cut.ties));
    for (int32_t i = written + tid; i < slots; i += NT) out_key[i] = 0u;
}

// ---- long rows: a launch a digit.  Once top-p's first digit is found, what has a larger one is left for certain: the next launch sums its weights, by
// runs of columns, beside the sums by the second digit, and lists the scores with the first; the third digit and the sums of what is
// left of the list read the list alone.  A part with more of them than its list has room for is read again.
// Where draws are few nothing is summed by runs: a part's weights above the first digit are sums of its own sums by digit, and a draw weighs
// the part that it is in.

struct State {                     // of a row, after a launch
    Search<11> x;
    Cut cut;
    uint32_t most;
};

struct Long {
    Call o;
    int64_t row0;                  // first row of this batch
    int32_t parts, part;           // blocks to a row, and columns to a block (a multiple of LONG_RUN)
    uint32_t *most;                // [rows][parts]
    u64 *hist;                     // [rows][6][2048]
    State *state;                  // [rows][7]
    u64 *part_sum, *part_ties;     // [rows][parts]: weights above the cut, ties of it
    u64 *run_sum, *run_ties;       // [rows][parts][part / LONG_RUN]; null: a draw weighs its part again
    u64 *part_hist;                // beside that [rows][parts][2048]: the parts' sums by top-p's first digit
    uint2 *list;                   // [rows][parts][part / LIST_PART]: scores with top-p's first digit, and their columns
    uint32_t *listed;              // [rows][parts]: their number, which may be more than there is room for
};
constexpr int LIST_PART = 4;
constexpr int LONG_T = 256, LONG_DIGITS = 2048;
constexpr int LONG_RUN = 1024;      // columns whose weights are summed

template <bool BF16>
__global__ __launch_bounds__(LONG_T) void k_long_most(Long a)
{
    __shared__ u64 s_part[16];
    const int64_t r = blockIdx.x / (unsigned)a.parts;
    const int32_t part = (int32_t)(blockIdx.x % (unsigned)a.parts), c0 = part * a.part;
    const Scores<BF16> src{(const char *)a.o.scores + (a.row0 + r) * a.o.lds * (BF16 ? 2 : 4), min(a.o.n_cols, c0 + a.part)};
    uint32_t most = 0u;
    Keys<LONG_T, 4, false, Scores<BF16>> keys(src);
    keys.each(c0, [&](int32_t) {
#pragma unroll
        for (int k = 0; k < 16; ++k) most = max(most, keys.key[k]);
    });
    most = Team<LONG_T>::most(most, s_part);
    if (threadIdx.x == 0) a.most[r * a.parts + part] = most;
    for (int32_t i = part * LONG_T + threadIdx.x; i < 6 * LONG_DIGITS; i += a.parts * LONG_T) a.hist[r * 6 * LONG_DIGITS + i] = 0ull;
}

// The row's state after stage `prev` (3 which + level), from the sums by digit that its launch left; prev < 0: before the first.
// `before`: the stage before that; `next`: which search the launch begins, or -1
__device__ __forceinline__ State advance(const Long &a, int64_t r, int before, int prev, int next, const Setting &set, Weigh *weigh, const double *pow, u64 *s,
                                         u64 *s_found)
{
    typedef Team<LONG_T> T;
    State st;
    if (prev < 0) {
        uint32_t most = 0u;
        for (int32_t i = threadIdx.x; i < a.parts; i += LONG_T) most = max(most, a.most[r * a.parts + i]);
        st.most = T::most(most, s);
        st.cut = first_cut(set, st.most);
        st.x.open = false;
    } else st = a.state[r * 7 + 1 + before];
    weigh->init(st.most, set.t, a.o, pow);
    if (prev >= 0 && st.x.open) {
        const int which = prev / 3, level = prev % 3;
        u64 v[LONG_DIGITS / LONG_T], upto, more, own;
        const u64 all = digit_total<LONG_T, 11>(a.hist + (r * 6 + prev) * LONG_DIGITS, v, &upto, s);
        if (level == 0) st.x.goal = which == 0 ? goal_of_count(all, set) : goal_of_weight(all, set);
        if (st.x.goal) {
            const int digit = digit_at<LONG_T, 11>(v, upto, st.x.goal - st.x.above, s_found, &more, &own);
            st.x.step(digit, more);
            if (!st.x.open) st.cut = cut_at(which, st.x, own, st.cut, *weigh);
        } else st.x.open = false;
    }
    if (next >= 0) {
        if (st.most && cuts(next, set, a.o.n_cols)) st.x.begin(next == 0 ? LEAST_KEY : max(st.cut.key, weigh->lowest(set.t)), st.most);
        else st.x.open = false;
    }
    return st;
}

// sums by digit of a search's level - of top-p's the first; prev: the stage of the launch before, `before` the one before that
template <bool BF16>
__global__ __launch_bounds__(LONG_T) void k_long_digit(Long a, int which, int level, int before, int prev)
{
    __shared__ u64 s_hist[LONG_DIGITS], s_part[16], s_found[4];
    __shared__ double s_pow[POWERS];
    fill_pow(s_pow, a.o.bits);
    const int64_t r = blockIdx.x / (unsigned)a.parts;
    const int32_t part = (int32_t)(blockIdx.x % (unsigned)a.parts), c0 = part * a.part;
    const Setting set = setting_of(a.o.how, a.row0 + r);
    Weigh weigh;
    const State st = advance(a, r, before, prev, level == 0 ? which : -1, set, &weigh, s_pow, s_part, s_found);
    if (part == 0 && threadIdx.x == 0) a.state[r * 7 + 1 + prev] = st;
    if (!st.x.open) return;
    for (int i = threadIdx.x; i < LONG_DIGITS; i += LONG_T) s_hist[i] = 0ull;
    __syncthreads();
    const Scores<BF16> src{(const char *)a.o.scores + (a.row0 + r) * a.o.lds * (BF16 ? 2 : 4), min(a.o.n_cols, c0 + a.part)};
    // what has the digits found before lies between two scores; of it top-p counts what is above top-k's cut
    const uint32_t low = st.x.first(), high = (uint32_t)min(st.x.last(), (u64)st.most);
    const float from = score_of(which == 1 && st.cut.key >= low ? st.cut.key + 1u : low), upto = score_upto(high);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    auto add = [&](float l, u64 w) { atomicAdd(&s_hist[st.x.digit(key_in_order(l))], w); };
    for (int32_t c0w = c0 + LONG_RUN * wave; c0w < src.n; c0w += LONG_RUN * (LONG_T / 64)) {
        float l[16];
        src.run16(c0w, lane, l);
        if (which == 0) {
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if (l[k] >= from && l[k] <= upto) add(l[k], 1ull);
        } else if (!weigh.endless) {
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if (l[k] >= from) add(l[k], (u64)__double_as_longlong(weigh.raised(l[k])) & 0xfffffffffffffull);
        } else {
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if (l[k] >= from && l[k] == INFINITY) add(l[k], weigh.unit());
        }
    }
    if (which == 1 && part == 0 && threadIdx.x == 0 && st.cut.key && st.x.in(st.cut.key))
        atomicAdd(&s_hist[st.x.digit(st.cut.key)], st.cut.ties * weigh(st.cut.key));
    __syncthreads();
    u64 *hist = a.hist + (r * 6 + which * 3 + level) * LONG_DIGITS;
    for (int i = threadIdx.x; i < LONG_DIGITS; i += LONG_T)
        if (s_hist[i]) atomicAdd(&hist[i], s_hist[i]);
    if (which == 1 && a.part_hist)
        for (int i = threadIdx.x; i < LONG_DIGITS; i += LONG_T) a.part_hist[(int64_t)blockIdx.x * LONG_DIGITS + i] = s_hist[i];
}

// scores that a search's digits found leave open, from top-k's cut on
struct Range { float from, upto; };
__device__ __forceinline__ Range range_of(const State &st)
{
    return Range{score_of(max(st.x.first(), st.cut.key)), score_upto((uint32_t)min(st.x.last(), (u64)st.most))};
}

// Of 16 columns a lane, the weights of scores from `edge` on (above the cut, and what is equal to it if all that is is left), no fewer units than
// `least`; 1024 weights of 2^40 units are a whole number that a double holds
__device__ __forceinline__ u64 run_weight(const float l[16], float edge, u64 least, const Weigh &weigh)
{
    double lanes = 0.0;
    if (weigh.endless) {
#pragma unroll
        for (int k = 0; k < 16; ++k) lanes += l[k] == INFINITY && l[k] >= edge ? (double)weigh.unit() : 0.0;
    } else if (least <= 1ull) {
#pragma unroll
        for (int k = 0; k < 16; ++k) lanes += weigh.raised(l[k] >= edge ? l[k] : -INFINITY) - 0x1p52;
    } else {
        const double fewest = (double)least;
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const double v = weigh.raised(l[k] >= edge ? l[k] : -INFINITY) - 0x1p52;
            lanes += v >= fewest ? v : 0.0;
        }
    }
    return whole(lane_of(wave_scan(lanes), 63));
}
__device__ __forceinline__ u64 run_ties(const float l[16], float tie)
{
    u64 t = 0ull;
#pragma unroll
    for (int k = 0; k < 16; ++k) t += l[k] == tie ? 1ull : 0ull;
    return wave_sum(t);
}
__device__ __forceinline__ float edge_of(const Cut &cut) { return cut.key == 0u ? -INFINITY : score_of(cut.every ? cut.key : cut.key + 1u); }

// The weights above the cut and the ties of it, by runs of columns and by part.  Where top-p's search is open (its first digit is found), what is
// above that digit counts; what has it is listed, and its weights go to the sums by the second digit
// Six blocks to a compute unit, so that the 1424 of 16 rows of 2.9 million run at once (51 us, of five 57)
template <bool BF16>
__global__ __launch_bounds__(LONG_T) __attribute__((amdgpu_waves_per_eu(6))) void k_long_sums(Long a, int before, int prev, int slot)
{
    __shared__ u64 s_hist[LONG_DIGITS], s_part[16], s_found[4];
    __shared__ double s_pow[POWERS];
    __shared__ uint32_t s_listed;
    if (threadIdx.x == 0) s_listed = 0u;
    fill_pow(s_pow, a.o.bits);
    const int64_t r = blockIdx.x / (unsigned)a.parts, here = blockIdx.x;
    const int32_t part = (int32_t)(blockIdx.x % (unsigned)a.parts), c0 = part * a.part;
    const Setting set = setting_of(a.o.how, a.row0 + r);
    Weigh weigh;
    const State st = advance(a, r, before, prev, -1, set, &weigh, s_pow, s_part, s_found);
    if (part == 0 && threadIdx.x == 0) a.state[r * 7 + slot] = st;
    const bool open = st.x.open;
    if (open) {
        for (int i = threadIdx.x; i < LONG_DIGITS; i += LONG_T) s_hist[i] = 0ull;
        __syncthreads();
    }
    const u64 least = least_weight(set, weigh);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const Scores<BF16> src{(const char *)a.o.scores + (a.row0 + r) * a.o.lds * (BF16 ? 2 : 4), min(a.o.n_cols, c0 + a.part)};
    const int32_t runs = a.part / LONG_RUN;
    const Range maybe = range_of(st);
    const bool above = st.x.last() < st.most, count_ties = !open && !st.cut.every;
    const float edge = !open ? edge_of(st.cut) : above ? score_of((uint32_t)st.x.last() + 1u) : NAN;
    // The sums by the first digit hold what min-p takes: they serve where it takes nothing above that digit, by more than a weight's rounding
    const bool by_digit = open && a.part_hist && (least <= 1ull || !above || weigh((uint32_t)st.x.last() + 1u) >= least + 2ull);
    uint2 *list = a.list + here * (a.part / LIST_PART);
    u64 sum = 0ull, ties = 0ull;
    for (int32_t i = wave; i < runs && c0 + LONG_RUN * i < src.n; i += LONG_T / 64) {
        float l[16];
        src.run16(c0 + LONG_RUN * i, lane, l);
        const u64 w = st.most && !by_digit ? run_weight(l, edge, least, weigh) : 0ull, t = count_ties ? run_ties(l, score_of(st.cut.key)) : 0ull;
        if (lane == 0 && a.run_sum) {
            a.run_sum[here * runs + i] = w;
            a.run_ties[here * runs + i] = t;
        }
        sum += w;
        ties += t;
        if (open) {
            uint32_t hits = 0u;
#pragma unroll
            for (int k = 0; k < 16; ++k) hits |= l[k] >= maybe.from && l[k] <= maybe.upto ? 1u << k : 0u;
#pragma unroll 1
            while (hits) {                                       // few: read again, so that no register is named by a number
                const int k = __builtin_ctz(hits);
                hits &= hits - 1u;
                const int32_t c = c0 + LONG_RUN * i + RUN * (k / 4) + 4 * lane + k % 4;
                const float x = src.one(c);
                const uint32_t key = key_in_order(x), at = atomicAdd(&s_listed, 1u);
                if (at < (uint32_t)(a.part / LIST_PART)) list[at] = make_uint2(__float_as_uint(x), (uint32_t)c);
                if (key > st.cut.key) atomicAdd(&s_hist[st.x.digit(key)], weigh(key));
            }
        }
    }
    if (by_digit) {
        for (int i = (int)st.x.found + 1 + (int)threadIdx.x; i < LONG_DIGITS; i += LONG_T) sum += a.part_hist[here * LONG_DIGITS + i];
        sum = wave_sum(sum);
    }
    // every lane of a wavefront has its sums
    if (lane == 0) { s_part[wave] = sum; s_part[8 + wave] = ties; }
    if (open && part == 0 && threadIdx.x == 0 && st.cut.key && st.x.in(st.cut.key)) atomicAdd(&s_hist[st.x.digit(st.cut.key)], st.cut.ties * weigh(st.cut.key));
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = ties = 0ull;
        for (int i = 0; i < LONG_T / 64; ++i) { sum += s_part[i]; ties += s_part[8 + i]; }
        a.part_sum[here] = sum;
        a.part_ties[here] = ties;
        a.listed[here] = s_listed;
    }
    if (!open) return;
    u64 *hist = a.hist + (r * 6 + 4) * LONG_DIGITS;
    for (int i = threadIdx.x; i < LONG_DIGITS; i += LONG_T)
        if (s_hist[i]) atomicAdd(&hist[i], s_hist[i]);
}

// f(score, column) for what a part's list holds, or should: scores in `range`
template <bool BF16, class F>
__device__ __forceinline__ void each_listed(const Long &a, int64_t here, const Scores<BF16> &src, int32_t c0, const Range &range, F f)
{
    const uint32_t n = a.listed[here];
    if (n <= (uint32_t)(a.part / LIST_PART)) {
        const uint2 *list = a.list + here * (a.part / LIST_PART);
        for (uint32_t i = threadIdx.x; i < n; i += LONG_T) f(__uint_as_float(list[i].x), (int32_t)list[i].y);
    } else {
#pragma unroll 1
        for (int32_t c = c0 + (int)threadIdx.x; c < src.n; c += LONG_T) {
            const float l = src.one(c);
            if (l >= range.from && l <= range.upto) f(l, c);
        }
    }
}

// sums by top-p's third digit
template <bool BF16>
__global__ __launch_bounds__(LONG_T) void k_long_third(Long a)
{
    __shared__ u64 s_hist[LONG_DIGITS], s_part[16], s_found[4];
    __shared__ double s_pow[POWERS];
    fill_pow(s_pow, a.o.bits);
    const int64_t r = blockIdx.x / (unsigned)a.parts, here = blockIdx.x;
    const int32_t part = (int32_t)(blockIdx.x % (unsigned)a.parts), c0 = part * a.part;
    const Setting set = setting_of(a.o.how, a.row0 + r);
    Weigh weigh;
    const State st = advance(a, r, 3, 4, -1, set, &weigh, s_pow, s_part, s_found);
    if (part == 0 && threadIdx.x == 0) a.state[r * 7 + 5] = st;
    if (!st.x.open) return;
    for (int i = threadIdx.x; i < LONG_DIGITS; i += LONG_T) s_hist[i] = 0ull;
    __syncthreads();
    const Scores<BF16> src{(const char *)a.o.scores + (a.row0 + r) * a.o.lds * (BF16 ? 2 : 4), min(a.o.n_cols, c0 + a.part)};
    each_listed(a, here, src, c0, range_of(a.state[r * 7 + 4]), [&](float l, int32_t) {
        const uint32_t key = key_in_order(l);
        if (key > st.cut.key && st.x.in(key)) atomicAdd(&s_hist[st.x.digit(key)], weigh(key));
    });
    if (part == 0 && threadIdx.x == 0 && st.cut.key && st.x.in(st.cut.key)) atomicAdd(&s_hist[st.x.digit(st.cut.key)], st.cut.ties * weigh(st.cut.key));
    __syncthreads();
    u64 *hist = a.hist + (r * 6 + 5) * LONG_DIGITS;
    for (int i = threadIdx.x; i < LONG_DIGITS; i += LONG_T)
        if (s_hist[i]) atomicAdd(&hist[i], s_hist[i]);
}

// what is left of the lists, added to the sums by runs and parts
template <bool BF16>
__global__ __launch_bounds__(LONG_T) void k_long_rest(Long a)
{
    constexpr int RUNS_MOST = 32;
    __shared__ u64 s_part[16], s_found[4], s_sum[RUNS_MOST], s_ties[RUNS_MOST];
    __shared__ double s_pow[POWERS];
    if (threadIdx.x < RUNS_MOST) s_sum[threadIdx.x] = s_ties[threadIdx.x] = 0ull;
    fill_pow(s_pow, a.o.bits);
    const int64_t r = blockIdx.x / (unsigned)a.parts, here = blockIdx.x;
    const int32_t part = (int32_t)(blockIdx.x % (unsigned)a.parts), c0 = part * a.part;
    const Setting set = setting_of(a.o.how, a.row0 + r);
    Weigh weigh;
    const State st = advance(a, r, 4, 5, -1, set, &weigh, s_pow, s_part, s_found), was = a.state[r * 7 + 4];
    if (part == 0 && threadIdx.x == 0) a.state[r * 7 + 6] = st;
    if (!was.x.open) return;                                     // nothing was listed: the sums are whole
    const u64 least = least_weight(set, weigh);
    const Scores<BF16> src{(const char *)a.o.scores + (a.row0 + r) * a.o.lds * (BF16 ? 2 : 4), min(a.o.n_cols, c0 + a.part)};
    each_listed(a, here, src, c0, range_of(was), [&](float l, int32_t c) {
        const uint32_t key = key_in_order(l);
        if (key < st.cut.key) return;
        const int run = (c - c0) / LONG_RUN;
        if (key == st.cut.key && !st.cut.every) atomicAdd(&s_ties[run], 1ull);
        else {
            const u64 w = weigh(key);
            if (w >= least) atomicAdd(&s_sum[run], w);
        }
    });
    __syncthreads();
    const int32_t runs = a.part / LONG_RUN;
    if (threadIdx.x < 64) {
        const int i = threadIdx.x;
        u64 w = 0ull, t = 0ull;
        if (i < runs && c0 + LONG_RUN * i < src.n) {
            w = s_sum[i];
            t = s_ties[i];
            if (a.run_sum) {
                a.run_sum[here * runs + i] += w;
                a.run_ties[here * runs + i] = t;
            }
        }
        w = wave_sum(w);
        t = wave_sum(t);
        if (i == 0) {
            a.part_sum[here] += w;
            a.part_ties[here] = t;
        }
    }
}

// Of n items in order, with weights above the cut and ties of it, the one at which the weights left pass `goal`: its number, and what comes
// before it (weights left, ties).  n_found 0: only the total.  All lanes of a wavefront alike.
struct Found { int32_t item; u64 before, ties, total; };
__device__ __forceinline__ Found find_item(const u64 *sum, const u64 *tie, int32_t n, u64 before, u64 ties, u64 left, u64 w_tie, bool search, u64 goal)
{
    Found f{-1, 0ull, 0ull, before};
    const int lane = threadIdx.x & 63;
    for (int32_t i0 = 0; i0 < n; i0 += 64) {
        const int32_t i = i0 + lane;
        u64 w = i < n ? sum[i] : 0ull, mine_ties = 0ull, upto_ties = 0ull;
        if (w_tie) {
            mine_ties = i < n ? tie[i] : 0ull;
            upto_ties = ties + wave_scan(mine_ties);
            const u64 first = upto_ties - mine_ties;
            w += (min(upto_ties, left) - min(first, left)) * w_tie;
        }
        const u64 upto = f.total + wave_scan(w);
        if (search && f.item < 0) {
            const u64 hit = __ballot(upto > goal);
            if (hit) {
                const int at = __builtin_ctzll(hit);
                f.item = i0 + at;
                f.before = lane_of(upto - w, at);
                f.ties = w_tie ? lane_of(upto_ties - mine_ties, at) : 0ull;
                return f;
            }
        }
        f.total = lane_of(upto, 63);
        if (w_tie) ties = lane_of(upto_ties, 63);
    }
    return f;
}

// A draw by WAVES wavefronts: one, which finds the run in its part, or those of a block, which weigh the part again
template <bool BF16, int WAVES>
__global__ __launch_bounds__(WAVES > 1 ? 64 * WAVES : 256) void k_long_draw(Long a, int64_t first, int64_t n)
{
    constexpr int RUNS_MOST = 32;
    __shared__ u64 s_sum[WAVES > 1 ? RUNS_MOST : 1], s_ties[WAVES > 1 ? RUNS_MOST : 1];
    __shared__ double s_pow[POWERS];
    fill_pow(s_pow, a.o.bits);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t draw = first + (WAVES > 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + wave);
    if (draw >= n) return;
    const int64_t r = draw / a.o.n_draws, at = a.row0 * a.o.n_draws + draw;
    const State st = a.state[r * 7 + 6];
    const Setting set = setting_of(a.o.how, a.row0 + r);
    Weigh weigh;
    weigh.init(st.most, set.t, a.o, s_pow);
    const u64 least = least_weight(set, weigh);
    u64 w_tie = st.most && !st.cut.every ? weigh(st.cut.key) : 0ull;
    if (w_tie < least) w_tie = 0ull;
    const u64 *sum = a.part_sum + r * a.parts, *tie = a.part_ties + r * a.parts;
    const u64 total = find_item(sum, tie, a.parts, 0ull, 0ull, st.cut.ties, w_tie, false, 0ull).total;
    if (total == 0ull) {
        if (lane == 0 && (WAVES == 1 || wave == 0)) answer(a.o, at, -1, 0.0, 1.0);
        return;
    }
    const u64 goal = goal_of_draw(a.o, at, total);
    const Found p = find_item(sum, tie, a.parts, 0ull, 0ull, st.cut.ties, w_tie, true, goal);
    const Scores<BF16> src{(const char *)a.o.scores + (a.row0 + r) * a.o.lds * (BF16 ? 2 : 4), a.o.n_cols};
    const int32_t c0 = p.item * a.part, last = (src.n - c0 + LONG_RUN - 1) / LONG_RUN, runs = min(a.part / LONG_RUN, last);       // the row may end in this part
    const u64 *run_sum = a.run_sum, *run_tie = a.run_ties;
    if (WAVES == 1) {
        run_sum += (r * a.parts + p.item) * (a.part / LONG_RUN);
        run_tie += (r * a.parts + p.item) * (a.part / LONG_RUN);
    } else {
        const float edge = edge_of(st.cut);
        for (int32_t i = wave; i < runs; i += WAVES) {
            float l[16];
            src.run16(c0 + LONG_RUN * i, lane, l);
            const u64 w = run_weight(l, edge, least, weigh), t = st.cut.every ? 0ull : run_ties(l, score_of(st.cut.key));
            if (lane == 0) { s_sum[i] = w; s_ties[i] = t; }
        }
        __syncthreads();
        if (wave > 0) return;
        run_sum = s_sum;
        run_tie = s_ties;
    }
    const Found f = find_item(run_sum, run_tie, runs, p.before, p.ties, st.cut.ties, w_tie, true, goal);
    u64 equal = f.ties, upto = f.before;
#pragma unroll 1
    for (int i = 0; i < LONG_RUN / RUN && upto <= goal; ++i) {
        const int32_t c = c0 + LONG_RUN * f.item + RUN * i + 4 * lane;
        uint32_t key[4];
        get4(src, c, key);
        upto += pick4(a.o, at, src, c, key, st.cut, weigh, least, &equal, goal, upto, total);
    }
}

// ---- host

int bits_of(int64_t n_cols)
{
    int log = 0;
    while ((1ll << log) < n_cols) ++log;
    return 62 - log < 40 ? 62 - log : 40;
}

constexpr int64_t LONG_BLOCKS = (1 << 22) - 1;           // of one launch: fewer than 2^32 threads
static_assert(LONG_BLOCKS * 1024 < 1ll << 32, "k_part_top has 1024 threads to a block");

// Up to KGE_SAMPLE_ROW columns a block takes a row whole, up to twice as many where there are rows for half the compute units, up to ROW_MOST where for
// all; else rows are split.  Nothing cut / top_k 50 / top_p 0.9, us, whole against split:
//   1 x 17000      18 / 17 / 40 against 18 / 19 / 33         256 x 65000     31 / 40 / 103 against 43 / 50 / 97
//   1 x 65000      30 / 26 / 86 against 18 / 19 / 33         256 x 262144    103 / 123 / 414 against 111 / 135 / 240
//   64 x 130000    38 / 51 / 170 against 29 / 36 / 69        600 x 65000     76 / 102 / 296 against 79 / 92 / 170
//   100 x 65000    23 / 31 / 93 against 26 / 32 / 63         600 x 262144    281 / 388 / 1087 against 279 / 295 / 556
//   128 x 40000    19 / 22 / 65 against 23 / 29 / 58         2048 x 40000    116 / 169 / 435 against 235 / 171 / 474
//   128 x 65000    24 / 33 / 95 against 28 / 35 / 70         2048 x 262144   753 / 1042 / 2951 against 888 / 960 / 1810
// The rule goes by sizes alone and suits draws of which nothing is cut and small top_k; with a top_p most of these rows would rather be split.
constexpr int64_t BLOCK_ROW = 65536;

// How a call runs, by its sizes and what the host knows of its settings
struct Plan {
    int32_t most_k, slots;         // 0: rows, or digits in launches; else k_part_top's
    int32_t parts, part, rows;     // parts of a row, columns of a part, rows a batch
    size_t off_most, off_hist, off_state, off_sum, off_ties, off_run, off_run_ties, off_part_hist, off_list, off_listed, bytes;
};

// Whether parts may keep their sums by digit: parts that are several times as many scores
template <class How>
bool parts_digits(const How &how, int64_t part) { return part >= 16384 && (how.row_top_p || how.top_p < 1.f); }

Plan plan_of(const kge_sampling *how, int64_t n_rows, int64_t n_cols)
{
    Plan p{};
    p.bytes = 256;
    if (n_cols <= KGE_SAMPLE_ROW || (n_cols <= BLOCK_ROW && n_rows >= 128) || (n_cols <= ROW_MOST && n_rows >= 256) || n_rows == 0) return p;
    const bool greedy = !how->row_temperature && how->temperature == 0.f;
    int64_t k = greedy ? 1 : how->top_k;
    if (k > 0) {
        // parts of 4096 columns where their scores left are a row of 16384 at most, else of 16384.  A few more places than k spare most parts
        // all digits but the first
        const int64_t slots = k == 1 ? 1 : (k + k / 8 + 15) / 8 * 8;
        for (int64_t part = 4096; part <= 16384; part *= 4) {
            const int64_t parts = cdiv(n_cols, part);
            if (k <= part && parts * slots <= (part == 4096 ? 16384 : BLOCK_ROW)) {
                p.most_k = (int32_t)k; p.slots = (int32_t)slots; p.parts = (int32_t)parts; p.part = (int32_t)part;
                p.rows = (int32_t)(n_rows < LONG_BLOCKS / parts ? n_rows : LONG_BLOCKS / parts);
                p.bytes = align_up((size_t)n_rows * parts * slots * 4, 256) * 2;
                return p;
            }
        }
    }
    // about 2048 blocks, of 4096 to 32768 columns
    int64_t part = 4096;
    while (part < 32768 && n_rows * cdiv(n_cols, part) > 2048) part *= 2;
    p.part = (int32_t)part; p.parts = (int32_t)cdiv(n_cols, part);
    p.rows = (int32_t)(n_rows < 4096 ? n_rows : 4096);
    if (p.rows > LONG_BLOCKS / p.parts) p.rows = (int32_t)(LONG_BLOCKS / p.parts);
    if (p.rows < 1) p.rows = 1;
    const size_t rows = (size_t)p.rows, parts = rows * p.parts, runs = parts * (part / LONG_RUN);
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at = align_up(at + bytes, 256); return here; };
    p.off_most = take(parts * 4);
    p.off_hist = take(rows * 6 * LONG_DIGITS * 8);
    p.off_state = take(rows * 7 * sizeof(State));
    p.off_sum = take(parts * 8);
    p.off_ties = take(parts * 8);
    p.off_run = take(runs * 8);
    p.off_run_ties = take(runs * 8);
    p.off_part_hist = take(parts_digits(*how, p.part) ? parts * LONG_DIGITS * 8 : 0);
    p.off_list = take(how->row_top_p || how->top_p < 1.f ? parts * (part / LIST_PART) * 8 : 0);     // of top-p's search alone
    p.off_listed = take(parts * 4);
    p.bytes = at;
    return p;
}

template <bool BF16, int NT, int TILES, bool ONE, int KIND>
int launch_rows(const Call &o, hipStream_t st)
{
    // a table of powers a block: its wavefronts take rows in turn
    const int64_t blocks = NT == 64 ? cdiv(o.n_rows, 4) : o.n_rows, most = NT == 64 ? 2048 : 65536;
    k_rows<BF16, NT, TILES, ONE, KIND><<<(unsigned)(blocks < most ? blocks : most), NT == 64 ? 256 : NT, 0, st>>>(o);
    KGE_LAUNCH_CHECK();
    return KGE_OK;
}

// rows that are taken whole
template <bool BF16, int KIND>
int launch_whole(const Call &o, hipStream_t st)
{
    if (o.n_cols <= 256) return launch_rows<BF16, 64, 1, true, KIND>(o, st);
    if (o.n_cols <= 1024) return launch_rows<BF16, 64, 4, true, KIND>(o, st);
    // Rows of little more: a wavefront a row, which reads them again, or a block.  No settings, us, wavefront / block: 16384 x 1100 68 / 110, 8192 x 2000
    // 38 / 56, 4096 x 2000 21 / 30; top_p 0.9: 196 / 343, 128 / 185, 67 / 96
    if (o.n_cols <= 2048 && o.n_rows >= 4096) return launch_rows<BF16, 64, 4, false, KIND>(o, st);
    if (o.n_cols <= 4096) return launch_rows<BF16, 256, 4, false, KIND>(o, st);
    // Rows enough for several blocks to a compute unit: small ones, whose waits overlap.  No settings, us, 256 threads / 1024: 2048 x 14541 51 / 73, 600 x
    // 60000 70 / 77, 600 x 14541 21 / 27; top_p 0.9: 178 / 226, 276 / 270, 79 / 87
    if (o.n_cols <= RUN * 256 && o.n_rows >= 512) return launch_rows<BF16, 256, 4, false, KIND>(o, st);
    if (o.n_cols <= 16384) return launch_rows<BF16, 1024, 4, true, KIND>(o, st);
    return launch_rows<BF16, 1024, 4, false, KIND>(o, st);
}

template <bool BF16>
int launch_call(Call o, const Plan &p, char *ws, hipStream_t st)
{
    if (p.parts == 0) {
        const bool cut = o.how.row_temperature || !(o.how.temperature > 0.f) || o.how.row_top_k || o.how.top_k > 0 || o.how.row_top_p || o.how.top_p < 1.f;
        return cut ? launch_whole<BF16, CUT>(o, st) : launch_whole<BF16, PLAIN>(o, st);
    }
    if (p.most_k) {
        uint32_t *part_key = (uint32_t *)ws;
        int32_t *part_col = (int32_t *)(ws + p.bytes / 2);
        for (int64_t row0 = 0; row0 < o.n_rows; row0 += p.rows) {
            const int64_t rows = o.n_rows - row0 < p.rows ? o.n_rows - row0 : p.rows;
            if (p.part == 4096) k_part_top<BF16, 256, 4><<<(unsigned)(rows * p.parts), 256, 0, st>>>(o, row0, p.parts, p.most_k, p.slots, part_key, part_col);
            else k_part_top<BF16, 1024, 4><<<(unsigned)(rows * p.parts), 1024, 0, st>>>(o, row0, p.parts, p.most_k, p.slots, part_key, part_col);
            KGE_LAUNCH_CHECK();
        }
        o.part_key = part_key; o.part_col = part_col; o.n_part = p.parts * p.slots;
        if (o.n_part <= 1024) return launch_rows<false, 64, 4, true, PARTS>(o, st);
        if (o.n_part <= 4096) return launch_rows<false, 256, 4, false, PARTS>(o, st);
        if (o.n_part <= 16384) return launch_rows<false, 1024, 4, true, PARTS>(o, st);
        return launch_rows<false, 1024, 4, false, PARTS>(o, st);
    }
    Long a;
    a.o = o; a.parts = p.parts; a.part = p.part;
    a.most = (uint32_t *)(ws + p.off_most); a.hist = (u64 *)(ws + p.off_hist); a.state = (State *)(ws + p.off_state);
    a.part_sum = (u64 *)(ws + p.off_sum); a.part_ties = (u64 *)(ws + p.off_ties);
    a.run_sum = (u64 *)(ws + p.off_run); a.run_ties = (u64 *)(ws + p.off_run_ties);
    a.list = (uint2 *)(ws + p.off_list); a.listed = (uint32_t *)(ws + p.off_listed);
    const bool by_count = o.how.row_top_k || o.how.top_k > 1;
    const bool by_weight = o.how.row_top_p || o.how.top_p < 1.f;
    // Draws that weigh a quarter of the row again at most.  top_p 0.9, 4 draws, us, weighing again / sums by runs: 16 x 2.9 million 168 / 185, 40 x a million
    // 145 / 155; parts of 4096, 1 x 2.9 million 66 / 62
    const bool again = parts_digits(o.how, p.part) && o.n_draws <= o.n_cols / p.part / 4;
    if (again) a.run_sum = a.run_ties = nullptr;
    a.part_hist = again ? (u64 *)(ws + p.off_part_hist) : nullptr;
    for (a.row0 = 0; a.row0 < o.n_rows; a.row0 += p.rows) {
        const int64_t rows = o.n_rows - a.row0 < p.rows ? o.n_rows - a.row0 : p.rows;
        const unsigned blocks = (unsigned)(rows * p.parts);
        k_long_most<BF16><<<blocks, LONG_T, 0, st>>>(a);
        KGE_LAUNCH_CHECK();
        int before = -2, prev = -1;
        for (int which = 0; which < 2; ++which) {
            if (which == 0 ? !by_count : !by_weight) continue;
            for (int level = 0; level < (which == 0 ? 3 : 1); ++level) {
                k_long_digit<BF16><<<blocks, LONG_T, 0, st>>>(a, which, level, before, prev);
                before = prev;
                prev = 3 * which + level;
            }
            KGE_LAUNCH_CHECK();
        }
        k_long_sums<BF16><<<blocks, LONG_T, 0, st>>>(a, before, prev, by_weight ? 4 : 6);
        KGE_LAUNCH_CHECK();
        if (by_weight) {
            k_long_third<BF16><<<blocks, LONG_T, 0, st>>>(a);
            k_long_rest<BF16><<<blocks, LONG_T, 0, st>>>(a);
            KGE_LAUNCH_CHECK();
        }
        const int64_t draws = rows * o.n_draws;
        for (int64_t d = 0; d < draws; d += LONG_BLOCKS) {
            const int64_t here = draws - d < LONG_BLOCKS ? draws - d : LONG_BLOCKS;
            if (again) k_long_draw<BF16, 16><<<(unsigned)here, 1024, 0, st>>>(a, d, draws);
            else k_long_draw<BF16, 1><<<(unsigned)cdiv(here, 4), 256, 0, st>>>(a, d, d + here);
            KGE_LAUNCH_CHECK();
        }
    }
    return KGE_OK;
}

int check_call(const kge_sampling *how, int64_t n_rows, int64_t n_cols)
{
    KGE_REQUIRE(how, KGE_EINVAL, "NULL argument");
    KGE_REQUIRE(n_rows >= 0 && n_cols >= 0, KGE_EINVAL, "negative size");
    KGE_REQUIRE(n_rows <= 0x7fffffffll && n_cols <= 0x7fff0000ll, KGE_ERANGE, "2^31 rows, or more than 2^31 - 2^16 columns");
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
    return plan_of(how, n_rows, n_cols).bytes;
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
    const Plan p = plan_of(how, n_rows, n_cols);
    if (n_cols > KGE_SAMPLE_ROW) {
        KGE_REQUIRE(workspace && (uintptr_t)workspace % 256 == 0, KGE_EINVAL, "the workspace is NULL or not aligned to 256 bytes");
        KGE_REQUIRE(ws_bytes >= p.bytes, KGE_ENOMEM, "the workspace is too small");
    }
    hipStream_t st = (hipStream_t)stream;
    Call o;
    o.how = Sampling{how->temperature, how->top_p, how->min_p, how->top_k, how->row_temperature, how->row_top_p, how->row_min_p, how->row_top_k};
    o.scores = scores; o.u = u; o.choice = choice; o.prob = prob; o.n_rows = n_rows; o.lds = lds;
    o.n_cols = (int32_t)n_cols; o.n_draws = n_draws; o.bits = bits_of(n_cols); o.u64bit = u_bits == 64;
    o.part_key = nullptr; o.part_col = nullptr; o.n_part = 0; o.per = per_of(how->temperature);
    KGE_PROF("sample_scores", st);
    return dtype == KGE_DT_BF16 ? launch_call<true>(o, p, (char *)workspace, st) : launch_call<false>(o, p, (char *)workspace, st);
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
