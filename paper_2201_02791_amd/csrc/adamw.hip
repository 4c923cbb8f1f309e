// One AdamW step over a list of tensors (decoupled weight decay, Loshchilov & Hutter 2019), in one launch per
// LIST_MAX tensors (of up to 2^26 wavefronts of work).
//
//   m <- b1 m + (1 - b1) g;  v <- b2 v + (1 - b2) g^2;  p <- p - lr (wd p + (m / c1) / (sqrt(v / c2) + eps)),  c = 1 - b^t
//
// Moments of 32 bits are floats.  Moments of 8 bits share a scale, a power of two, among the KGE_ADAMW_BLOCK consecutive
// elements of a row that one wavefront (or part of one, for short rows) holds: m is kept in e4m3, v in e5m2, whose
// 32 octaves span the squares of what 16 octaves of gradients are.  The update itself takes the new moments as they are
// in fp32, before they are rounded.
//
// Why rounding needs an offset: v moves by 1 - b2, a thousandth, per step, and e5m2 numbers are up to a quarter apart, so
// rounding to nearest would leave v where it is for ever.  A number between two of the format's goes to the upper one
// where its place between them plus an offset u(element, step) in [0, 1) reaches one: over steps the mean is the number.
// u is a hash of a multiply-add of both, one 32-bit multiplication for the two offsets of an element; 0x9E3779B9 is 2^32 over the golden
// section, the other two multipliers are odd constants known from published 32-bit hashes.  (Multiples of the
// golden section in its place, without the hash, meet [0, 1) more evenly, but an average that only falls waits for them
// in step: it came out at half its value after three time constants, where these offsets keep its mean.)  A step's
// variance is (1 - b2) D v^2 for numbers D v apart and is forgotten at 2 (1 - b2): v spreads by sqrt(D / 2), at most
// sqrt(1/8), and sqrt(v) by half of that.  A v that is not zero is kept at or above e5m2's smallest number, so that no
// step divides by a v that was lost.
//
// fp contraction is off: every operation on the moments rounds once, in the order written above, so that the same states
// come out wherever this arithmetic is repeated.
//
// Bandwidth bound: an element of 32-bit moments takes 28 bytes (16 read, 12 written), one of 8-bit moments 16.  Measured on the
// large graph's model (a table of 10^6 x 256 of which 9 rows in 10 are taken, and 29 million other parameters): 1241 us,
// 5.4 TB/s, and 728 us, 5.3 TB/s.  The latter was bound by its vector instructions, 105 an element and 770 us, until the blocks'
// maxima went through rotations (a DPP instruction each) and root and reciprocal were single instructions.  With the step number in device
// memory every thread forms the corrections' powers in double: a million rows of 256, 1303 -> 1305 us at step 10 and 1301 -> 1307 at
// step 100000 with 32 bits, 723 -> 776 and 717 -> 903 with 8, whose instructions have no time to spare.
#include "common.h"

#include <math.h>

#pragma clang fp contract(off)

namespace {

constexpr int BLOCK = KGE_ADAMW_BLOCK;        // 64 lanes x 4 elements
static_assert(BLOCK == 256, "one wavefront holds a block, 4 elements a lane");
constexpr int64_t MOST_WAVES = (1ll << 32) / 64 - 4;      // a launch has fewer than 2^32 threads: a list of more takes several
constexpr int64_t MOST_ELEMENTS = 1ll << 36;  // no card holds as many with their gradients
static_assert(MOST_WAVES % 4 == 0, "whole blocks");
constexpr int LIST_MAX = 28;                  // tensors per launch: their descriptions are launch arguments, below 4 KB

struct Tensor {
    float *p;
    const float *g;
    void *m, *v;
    float *ms, *vs;
    uint16_t *copy;
    const uint8_t *mask;
    int64_t d, n_rows, nb;         // nb: blocks of a row
    int64_t first;                 // first unit, in wavefronts, of this tensor in the launch
    float wd;
    int32_t how;                   // lanes of a unit (low byte), HOW_*
};
enum { HOW_WHOLE = 1 << 8, HOW_8BIT = 1 << 9, HOW_NONZERO = 1 << 10 };

struct List {
    Tensor t[LIST_MAX];
    int32_t n;
    float lr, b1, b2, eps, omb1, omb2, inv_c1, inv_c2;
    const int64_t *t_dev;          // the step number in device memory, or null
    const float *factor;           // what gradients are multiplied by, in device memory (k_adamw<true>)
    int64_t step;
    int64_t base;                  // the launch's first wavefront
};
static_assert(sizeof(List) <= 4096, "launch arguments");

typedef float floatx2 __attribute__((ext_vector_type(2)));

struct Four { float x[4]; };
// four elements at any element's address
struct __attribute__((packed, aligned(4))) F4 { float x[4]; };
struct __attribute__((packed, aligned(1))) C4 { uint32_t w; };
struct __attribute__((packed, aligned(2))) H4 { uint32_t w[2]; };

// n elements of four; WHOLE: rows are a multiple of four, n is four
template <bool WHOLE>
__device__ __forceinline__ Four load4(const float *a, int n)
{
    Four r{};
    if (WHOLE || n >= 4) {
        const F4 q = *reinterpret_cast<const F4 *>(a);
#pragma unroll
        for (int k = 0; k < 4; ++k) r.x[k] = q.x[k];
    } else {
#pragma unroll
        for (int k = 0; k < 3; ++k) r.x[k] = k < n ? a[k] : 0.f;
    }
    return r;
}

template <bool WHOLE>
__device__ __forceinline__ void store4(float *a, const Four &r, int n)
{
    if (WHOLE || n >= 4) *reinterpret_cast<F4 *>(a) = F4{{r.x[0], r.x[1], r.x[2], r.x[3]}};
    else {
#pragma unroll
        for (int k = 0; k < 3; ++k) if (k < n) a[k] = r.x[k];
    }
}

template <bool WHOLE>
__device__ __forceinline__ uint32_t load_codes(const uint8_t *a, int n)
{
    if (WHOLE || n >= 4) return reinterpret_cast<const C4 *>(a)->w;
    uint32_t r = 0u;
#pragma unroll
    for (int k = 0; k < 3; ++k) if (k < n) r |= (uint32_t)a[k] << (8 * k);
    return r;
}

template <bool WHOLE>
__device__ __forceinline__ void store_codes(uint8_t *a, uint32_t r, int n)
{
    if (WHOLE || n >= 4) reinterpret_cast<C4 *>(a)->w = r;
    else {
#pragma unroll
        for (int k = 0; k < 3; ++k) if (k < n) a[k] = (uint8_t)(r >> (8 * k));
    }
}

// largest of the magnitudes' bit patterns over the unit's lanes (a NaN is larger than all): rotations inside a row of 16 lanes,
// which cost one instruction each, then the rows
template <int N>
__device__ __forceinline__ uint32_t most_rotated(uint32_t v)
{
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 | N, 0xf, 0xf, false));
}
__device__ __forceinline__ uint32_t most_of(uint32_t v, int lanes)
{
    if (lanes >= 16) {
        v = most_rotated<8>(v);
        v = most_rotated<4>(v);
        v = most_rotated<2>(v);
        v = most_rotated<1>(v);
        if (lanes >= 32) v = max(v, (uint32_t)__shfl_xor((int)v, 16, 64));
        if (lanes == 64) v = max(v, (uint32_t)__shfl_xor((int)v, 32, 64));
        return v;
    }
    for (int off = lanes >> 1; off > 0; off >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, off, 64));
    return v;
}

// The power of two (its bits) that brings a block's largest magnitude to between half of the format's largest number,
// 1.75 x 2^TOP, and that number; 0 for a block of zeros, NaN for one with a number that is not finite.
template <int TOP>
__device__ __forceinline__ uint32_t scale_bits(uint32_t most)
{
    if (most == 0u) return 0u;
    if (most >= 0x7f800000u) return 0x7fc00000u;
    const int e = (int)(most >> 23) - TOP + ((most & 0x7fffffu) > 0x600000u);
    return (uint32_t)max(e, 1) << 23;
}

// a scaled magnitude, to a number of the format with DIGITS bits behind the point and normal numbers from 2^LEAST on; the offset
// in units of 2^-16.  Both products are by powers of two: the sum is what rounds, whether it is fused or not
template <int DIGITS, int LEAST>
__device__ __forceinline__ float round_up_by(float y, float offset)
{
    const uint32_t e = max(__float_as_uint(y) & 0x7f800000u, (uint32_t)(127 + LEAST) << 23);
    const float per = __uint_as_float(((uint32_t)(254 + DIGITS) << 23) - e);
    return floorf(__builtin_fmaf(offset, 0x1p-16f, y * per)) * __uint_as_float(e - ((uint32_t)DIGITS << 23));
}

// the two offsets of an element, 16 bits each, from its index and the step (times their multipliers)
__device__ __forceinline__ uint32_t offsets_of(uint32_t x) { return (x ^ (x >> 16)) * 0x2C1B3C6Du; }

// One block of a row by the `lanes` lanes of a unit: element i0 + 4 lane .., n of its four inside the row (n <= 0: none).
template <bool WHOLE, bool EIGHT, bool SCALED>
__device__ __forceinline__ void update(const List &o, const Tensor &T, int64_t at, int n, int64_t scale_at, int lanes, float inv_c1,
                                       float inv_c2, uint32_t step, float factor, bool on)
{
    const bool any = on && n > 0;
    Four p{}, g{}, m{}, v{};
    uint32_t cm = 0u, cv = 0u;
    float sm = 0.f, sv = 0.f;
    if (any) {
        p = load4<WHOLE>(T.p + at, n);
        g = load4<WHOLE>(T.g + at, n);
        if (EIGHT) {
            cm = load_codes<WHOLE>((const uint8_t *)T.m + at, n);
            cv = load_codes<WHOLE>((const uint8_t *)T.v + at, n);
            sm = T.ms[scale_at]; sv = T.vs[scale_at];
        } else {
            m = load4<WHOLE>((const float *)T.m + at, n);
            v = load4<WHOLE>((const float *)T.v + at, n);
        }
    }
    if (EIGHT) {
        const floatx2 m0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)cm, false), m1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)cm, true);
        const floatx2 v0 = __builtin_amdgcn_cvt_pk_f32_bf8((int)cv, false), v1 = __builtin_amdgcn_cvt_pk_f32_bf8((int)cv, true);
        m.x[0] = m0.x * sm; m.x[1] = m0.y * sm; m.x[2] = m1.x * sm; m.x[3] = m1.y * sm;
        v.x[0] = v0.x * sv; v.x[1] = v0.y * sv; v.x[2] = v1.x * sv; v.x[3] = v1.y * sv;
    }
    uint32_t most_m = 0u, most_v = 0u;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (SCALED) g.x[k] *= factor;
        m.x[k] = o.b1 * m.x[k] + o.omb1 * g.x[k];
        v.x[k] = o.b2 * v.x[k] + (o.omb2 * g.x[k]) * g.x[k];
        // root and reciprocal are off by a unit in the last place, of the step and not of the parameter.  The instruction for the root
        // need not keep numbers below 2^-126, which count only beside an eps of no size
        const float w = v.x[k] * inv_c2;
        const float step_k = m.x[k] * inv_c1 * __builtin_amdgcn_rcpf((o.eps >= 0x1p-40f ? __builtin_amdgcn_sqrtf(w) : sqrtf(w)) + o.eps);
        p.x[k] -= o.lr * (T.wd * p.x[k] + step_k);
        if (EIGHT && any && (WHOLE || k < n)) {
            most_m = max(most_m, __float_as_uint(m.x[k]) & 0x7fffffffu);
            most_v = max(most_v, __float_as_uint(v.x[k]) & 0x7fffffffu);
        }
    }
    if (EIGHT) {                     // all lanes of the wavefront take part in the exchange
        const uint32_t km = scale_bits<8>(most_of(most_m, lanes)), kv = scale_bits<15>(most_of(most_v, lanes));
        const float im = km ? __uint_as_float((254u << 23) - km) : 0.f, iv = kv ? __uint_as_float((254u << 23) - kv) : 0.f;
        float q[4], r[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t x = offsets_of(((uint32_t)at + (uint32_t)k) * 0xC2B2AE35u + step * 0x9E3779B9u);
            q[k] = copysignf(round_up_by<3, -6>(fabsf(m.x[k]) * im, (float)(x & 0xffffu)), m.x[k]);
            r[k] = fmaxf(round_up_by<2, -14>(v.x[k] * iv, (float)(x >> 16)), v.x[k] > 0.f ? 0x1p-16f : 0.f);
        }
        cm = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false), true);
        cv = (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(r[2], r[3], __builtin_amdgcn_cvt_pk_bf8_f32(r[0], r[1], 0, false), true);
        if (any) {
            store_codes<WHOLE>((uint8_t *)T.m + at, cm, n);
            store_codes<WHOLE>((uint8_t *)T.v + at, cv, n);
            if ((threadIdx.x & (lanes - 1)) == 0) { T.ms[scale_at] = __uint_as_float(km); T.vs[scale_at] = __uint_as_float(kv); }
        }
    }
    if (!any) return;
    store4<WHOLE>(T.p + at, p, n);
    if (!EIGHT) {
        store4<WHOLE>((float *)T.m + at, m, n);
        store4<WHOLE>((float *)T.v + at, v, n);
    }
    if (T.copy) {
        uint16_t c[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) c[k] = __builtin_bit_cast(uint16_t, (__bf16)p.x[k]);
        if (WHOLE || n >= 4) *reinterpret_cast<H4 *>(T.copy + at) = H4{{c[0] | (uint32_t)c[1] << 16, c[2] | (uint32_t)c[3] << 16}};
        else {
#pragma unroll
            for (int k = 0; k < 3; ++k) if (k < n) T.copy[at + k] = c[k];
        }
    }
}

template <bool WHOLE, bool EIGHT, bool SCALED>
__device__ __forceinline__ void unit(const List &o, const Tensor &T, int64_t w, float inv_c1, float inv_c2, uint32_t step, float factor)
{
    const int lane = threadIdx.x & 63, lanes = T.how & 0xff;
    const int l = lane & (lanes - 1);
    if (T.how & HOW_NONZERO) {       // a unit is a row: first whether its gradient has anything, then block after block
        const int64_t row = w * (64 / lanes) + lane / lanes;
        const bool in = row < T.n_rows;
        bool some = false;
        for (int64_t b = 0; b < T.nb; ++b) {
            const int64_t c = b * BLOCK + 4 * l;
            if (in && c < T.d) {
                const Four g = load4<WHOLE>(T.g + row * T.d + c, (int)min((int64_t)4, T.d - c));
                some |= (g.x[0] != 0.f) | (g.x[1] != 0.f) | (g.x[2] != 0.f) | (g.x[3] != 0.f);
            }
        }
        const uint64_t mine = lanes == 64 ? ~0ull : ((1ull << lanes) - 1ull) << (lane & ~(lanes - 1));
        const bool on = (__ballot(some) & mine) != 0ull;
        for (int64_t b = 0; b < T.nb; ++b) {
            const int64_t c = b * BLOCK + 4 * l;
            update<WHOLE, EIGHT, SCALED>(o, T, row * T.d + c, in ? (int)min((int64_t)4, T.d - c) : 0, row * T.nb + b, lanes, inv_c1,
                                         inv_c2, step, factor, on);
        }
        return;
    }
    int64_t row, b = 0;
    if (lanes == 64) {               // nb > 1 only where a unit is a whole wavefront
        row = T.nb == 1 ? w : T.n_rows == 1 ? 0 : w / T.nb;
        b = w - row * T.nb;
    } else row = w * (64 / lanes) + lane / lanes;
    const bool in = row < T.n_rows;
    const int64_t c = b * BLOCK + 4 * l;
    const bool on = in && (!T.mask || T.mask[row]);
    update<WHOLE, EIGHT, SCALED>(o, T, row * T.d + c, in ? (int)min((int64_t)4, T.d - c) : 0, row * T.nb + b, lanes, inv_c1, inv_c2, step,
                                 factor, on);
}

// SCALED: gradients times a factor from device memory, which the norm of them all may have left there; one that is NaN, of
// gradients that are not finite, leaves everything as it is.  A million rows of 256: 1316 -> 1319 us with 32-bit moments, 711 -> 707 with 8
template <bool SCALED>
__global__ __launch_bounds__(256) void k_adamw(List o)
{
    const float factor = SCALED ? *o.factor : 1.f;
    if (SCALED && factor != factor) return;
    // the bias corrections of a step number in device memory, in double like the host's
    float inv_c1 = o.inv_c1, inv_c2 = o.inv_c2;
    int64_t step = o.step;
    if (o.t_dev) {
        step = *o.t_dev;
        double p1 = 1.0, p2 = 1.0, q1 = o.b1, q2 = o.b2;
        for (uint64_t e = step > 0 ? (uint64_t)step : 1ull; e; e >>= 1) {
            if (e & 1ull) { p1 *= q1; p2 *= q2; }
            q1 *= q1; q2 *= q2;
        }
        inv_c1 = (float)(1.0 / (1.0 - p1)); inv_c2 = (float)(1.0 / (1.0 - p2));
    }
    const int64_t w = o.base + (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int i = 0;
    while (i + 1 < o.n && w >= o.t[i + 1].first) ++i;
    const Tensor &T = o.t[i];
    const int64_t mine = w - T.first;
    if (T.how & HOW_8BIT) {
        if (T.how & HOW_WHOLE) unit<true, true, SCALED>(o, T, mine, inv_c1, inv_c2, (uint32_t)step, factor);
        else unit<false, true, SCALED>(o, T, mine, inv_c1, inv_c2, (uint32_t)step, factor);
    } else {
        if (T.how & HOW_WHOLE) unit<true, false, SCALED>(o, T, mine, inv_c1, inv_c2, (uint32_t)step, factor);
        else unit<false, false, SCALED>(o, T, mine, inv_c1, inv_c2, (uint32_t)step, factor);
    }
}

bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

}  // namespace

namespace {

int adamw_step(const kge_adamw *opt, const kge_adamw_tensor *tensors, int32_t n_tensors, const float *factor, void *stream)
{
    KGE_REQUIRE(opt && (tensors || n_tensors == 0), KGE_EINVAL, "NULL argument");
    KGE_REQUIRE(n_tensors >= 0, KGE_EINVAL, "negative number of tensors");
    KGE_REQUIRE(opt->beta1 >= 0.f && opt->beta1 < 1.f && opt->beta2 >= 0.f && opt->beta2 < 1.f, KGE_EINVAL,
                "beta1 and beta2 must be in [0, 1)");
    KGE_REQUIRE(aligned(opt->t_dev, 8), KGE_EINVAL, "t_dev is not aligned to its type");
    KGE_REQUIRE(opt->t_dev || opt->t >= 1, KGE_EINVAL, "AdamW's step number t starts at 1");
    for (int32_t i = 0; i < n_tensors; ++i) {
        const kge_adamw_tensor &x = tensors[i];
        KGE_REQUIRE(x.n_rows >= 0 && x.d >= 0, KGE_EINVAL, "tensor %d: negative size", i);
        KGE_REQUIRE(x.state_bits == 32 || x.state_bits == 8, KGE_EINVAL, "tensor %d: moments have 32 or 8 bits", i);
        KGE_REQUIRE(x.rows == KGE_ROWS_ALL || x.rows == KGE_ROWS_MASK || x.rows == KGE_ROWS_NONZERO, KGE_EINVAL,
                    "tensor %d: bad choice of rows", i);
        KGE_REQUIRE(x.d == 0 || x.n_rows <= (MOST_ELEMENTS - 1) / x.d, KGE_ERANGE, "tensor %d: 2^36 elements or more", i);
        if (x.n_rows == 0 || x.d == 0) continue;
        KGE_REQUIRE(x.param && x.grad && x.m && x.v, KGE_EINVAL, "tensor %d: NULL parameter, gradient or moment", i);
        KGE_REQUIRE((x.state_bits == 8) == (x.m_scale != nullptr) && (x.state_bits == 8) == (x.v_scale != nullptr), KGE_EINVAL,
                    "tensor %d: scales belong to moments of 8 bits, and to those alone", i);
        KGE_REQUIRE((x.rows == KGE_ROWS_MASK) == (x.row_mask != nullptr), KGE_EINVAL,
                    "tensor %d: a row mask belongs to KGE_ROWS_MASK, and to that alone", i);
        KGE_REQUIRE(x.rows != KGE_ROWS_NONZERO || x.d <= 65536, KGE_EINVAL,
                    "tensor %d: KGE_ROWS_NONZERO takes rows of at most 65536 elements", i);
        KGE_REQUIRE(aligned(x.param, 4) && aligned(x.grad, 4) && aligned(x.copy, 2) &&
                        (x.state_bits == 8 || (aligned(x.m, 4) && aligned(x.v, 4))) && aligned(x.m_scale, 4) && aligned(x.v_scale, 4),
                    KGE_EINVAL, "tensor %d: an array is not aligned to its elements", i);
    }
    hipStream_t st = (hipStream_t)stream;
    List o;
    o.lr = opt->lr; o.b1 = opt->beta1; o.b2 = opt->beta2; o.eps = opt->eps;
    o.omb1 = (float)(1.0 - (double)opt->beta1); o.omb2 = (float)(1.0 - (double)opt->beta2);
    o.factor = factor;
    o.t_dev = opt->t_dev; o.step = opt->t_dev ? 0 : opt->t;
    o.inv_c1 = o.inv_c2 = 1.f;
    if (!opt->t_dev) {
        o.inv_c1 = (float)(1.0 / (1.0 - pow((double)opt->beta1, (double)opt->t)));
        o.inv_c2 = (float)(1.0 / (1.0 - pow((double)opt->beta2, (double)opt->t)));
    }
    KGE_PROF("adamw", st);
    for (int32_t i = 0; i < n_tensors;) {
        o.n = 0;
        int64_t waves = 0;
        for (; i < n_tensors && o.n < LIST_MAX; ++i) {
            const kge_adamw_tensor &x = tensors[i];
            if (x.n_rows == 0 || x.d == 0) continue;
            const bool eight = x.state_bits == 8;
            Tensor T;
            T.p = x.param; T.g = x.grad; T.m = x.m; T.v = x.v; T.ms = x.m_scale; T.vs = x.v_scale; T.copy = x.copy; T.mask = x.row_mask;
            T.d = x.d; T.n_rows = x.n_rows; T.wd = x.weight_decay;
            // nothing of a step that takes all rows and keeps no scales goes by rows
            if (!eight && x.rows == KGE_ROWS_ALL) { T.d = x.n_rows * x.d; T.n_rows = 1; }
            T.nb = cdiv(T.d, BLOCK);
            int lanes = 1;
            while (lanes < 64 && 4 * lanes < T.d) lanes *= 2;
            T.how = lanes | (T.d % 4 == 0 ? HOW_WHOLE : 0) | (eight ? HOW_8BIT : 0) | (x.rows == KGE_ROWS_NONZERO ? HOW_NONZERO : 0);
            const int64_t units = x.rows == KGE_ROWS_NONZERO || T.nb == 1 ? cdiv(T.n_rows, 64 / lanes) : T.n_rows * T.nb;
            T.first = waves;
            waves += units;
            o.t[o.n++] = T;
        }
        if (o.n == 0) continue;
        for (o.base = 0; o.base < waves; o.base += MOST_WAVES) {
            const int64_t left = waves - o.base;
            (factor ? k_adamw<true> : k_adamw<false>)<<<(unsigned)cdiv(left < MOST_WAVES ? left : MOST_WAVES, 4), 256, 0, st>>>(o);
            KGE_LAUNCH_CHECK();
        }
    }
    return KGE_OK;
}

}  // namespace

extern "C" int kge_adamw_step(const kge_adamw *opt, const kge_adamw_tensor *tensors, int32_t n_tensors, void *stream)
{
    return adamw_step(opt, tensors, n_tensors, nullptr, stream);
}

extern "C" int kge_adamw_step_scaled(const kge_adamw *opt, const kge_adamw_tensor *tensors, int32_t n_tensors, const float *factor, void *stream)
{
    KGE_REQUIRE(factor && aligned(factor, 4), KGE_EINVAL, "factor: the address of a float is wanted");
    return adamw_step(opt, tensors, n_tensors, factor, stream);
}
