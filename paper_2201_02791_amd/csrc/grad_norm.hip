// The norm of all gradients of a model and their scaling to a largest norm.
//
//   norm = sqrt(sum over tensors and elements of g^2);  factor = min(1, max_norm / norm);  g <- factor g
//
// Squares are formed and added in double: the square of a float is exact there, nothing overflows, and the order of the sum
// (lanes, wavefronts, blocks, always the same for the same sizes) shows in no bit of the float that comes out but by chance.
// The matrix cores have no part in it, and the vector unit takes double additions at the rate of float ones.
//
// Two launches: blocks that each leave one sum in the workspace, then blocks that all add those sums up in the same order and
// scale what is theirs; for the norm alone one block adds them up.  No atomics, nothing to clear beforehand.
// Bandwidth bound: 265 million floats, of which 239 million count (958 MB), 158 us (6.1 TB/s, a part of it from the last-level cache; 195 us after
// their scaling) and scaled 334 us, 5.7 TB/s.  Scaling goes from the last gradient to the first, the cache's order, and stores past it (359 us without).
// (One block for a small model, in one launch, waits longer for its loads than the second launch takes: 43,000 elements 16.6 us against
// 5.3 + 6.0.)
#include "common.h"

#include <math.h>

namespace {

constexpr int LIST_MAX = 48;                  // tensors per launch: their descriptions are launch arguments, below 4 KB
constexpr int BLOCKS_MAX = 2048;              // sums a launch leaves
constexpr int SLOTS = 4;                      // a unit of work: so many times 4 elements for each lane of a wavefront
constexpr int64_t MOST_ELEMENTS = 1ll << 36;

struct Tensor {
    void *g;
    const uint8_t *mask;
    int64_t d, n_rows, nb;         // nb: blocks of 256 elements of a row
    int64_t first;                 // first unit of this tensor in the launch
    int32_t lanes, bf16;           // lanes that share a row's block
};
struct List {
    Tensor t[LIST_MAX];
    int64_t units;
    int32_t n;
};
static_assert(sizeof(List) <= 3584, "launch arguments");

struct __attribute__((packed, aligned(4))) F4 { float x[4]; };
struct __attribute__((packed, aligned(2))) H4 { uint16_t x[4]; };

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef floatx4 floatx4u __attribute__((aligned(4)));

struct Four { float x[4]; };

// n elements of four at element `at`, the others zero
__device__ __forceinline__ Four load4(const Tensor &T, int64_t at, int n)
{
    Four r{};
    if (T.bf16) {
        const uint16_t *a = (const uint16_t *)T.g + at;
        if (n >= 4) {
            const H4 q = *reinterpret_cast<const H4 *>(a);
#pragma unroll
            for (int k = 0; k < 4; ++k) r.x[k] = __uint_as_float((uint32_t)q.x[k] << 16);
        } else {
#pragma unroll
            for (int k = 0; k < 3; ++k) if (k < n) r.x[k] = __uint_as_float((uint32_t)a[k] << 16);
        }
    } else {
        const float *a = (const float *)T.g + at;
        if (n >= 4) {
            const F4 q = *reinterpret_cast<const F4 *>(a);
#pragma unroll
            for (int k = 0; k < 4; ++k) r.x[k] = q.x[k];
        } else {
#pragma unroll
            for (int k = 0; k < 3; ++k) if (k < n) r.x[k] = a[k];
        }
    }
    return r;
}

__device__ __forceinline__ void store4(const Tensor &T, int64_t at, int n, const Four &r)
{
    if (T.bf16) {
        uint16_t *a = (uint16_t *)T.g + at;
        H4 q;
#pragma unroll
        for (int k = 0; k < 4; ++k) q.x[k] = __builtin_bit_cast(uint16_t, (__bf16)r.x[k]);
        if (n >= 4) *reinterpret_cast<H4 *>(a) = q;
        else {
#pragma unroll
            for (int k = 0; k < 3; ++k) if (k < n) a[k] = q.x[k];
        }
    } else {
        float *a = (float *)T.g + at;
        if (n >= 4) __builtin_nontemporal_store(floatx4{r.x[0], r.x[1], r.x[2], r.x[3]}, reinterpret_cast<floatx4u *>(a));
        else {
#pragma unroll
            for (int k = 0; k < 3; ++k) if (k < n) a[k] = r.x[k];
        }
    }
}

// Where slot s of a tensor has this lane's elements: their index, and how many of four are inside a row that counts
__device__ __forceinline__ int place(const Tensor &T, int64_t s, int lane, int64_t *at)
{
    int64_t row, b = 0;
    if (T.lanes == 64) {
        row = T.n_rows == 1 ? 0 : T.nb == 1 ? s : s / T.nb;
        b = s - row * T.nb;
    } else row = s * (64 / T.lanes) + lane / T.lanes;
    const int64_t c = b * 256 + 4 * (lane & (T.lanes - 1));
    *at = row * T.d + c;
    const bool on = row < T.n_rows && c < T.d && (!T.mask || T.mask[row]);
    return on ? (int)min((int64_t)4, T.d - c) : 0;
}

__device__ __forceinline__ const Tensor &tensor_of(const List &o, int64_t unit)
{
    int i = 0;
    while (i + 1 < o.n && unit >= o.t[i + 1].first) ++i;
    return o.t[i];
}

// the same sum in every thread of a block of 256
__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double s_part[4];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = (s_part[0] + s_part[1]) + (s_part[2] + s_part[3]);
    __syncthreads();
    return v;
}

// a wavefront's sum of squares over units w, w + waves, ..
__device__ __forceinline__ double squares(const List &o, int64_t w, int64_t waves, int lane)
{
    double a[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 1
    for (int64_t u = w; u < o.units; u += waves) {
        const Tensor &T = tensor_of(o, u);
        Four x[SLOTS];
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            int64_t at;
            const int n = place(T, (u - T.first) * SLOTS + s, lane, &at);
            x[s] = load4(T, at, n);
        }
#pragma unroll
        for (int s = 0; s < SLOTS; ++s)
#pragma unroll
            for (int k = 0; k < 4; ++k) a[k] = fma((double)x[s].x[k], (double)x[s].x[k], a[k]);
    }
    return (a[0] + a[1]) + (a[2] + a[3]);
}

// its units scaled, the last first: what was read last the last-level cache still has
__device__ __forceinline__ void scale_by(const List &o, int64_t w, int64_t waves, int lane, float f)
{
#pragma unroll 1
    for (int64_t v = w; v < o.units; v += waves) {
        const int64_t u = o.units - 1 - v;
        const Tensor &T = tensor_of(o, u);
        Four x[SLOTS];
        int64_t at[SLOTS];
        int n[SLOTS];
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            n[s] = place(T, (u - T.first) * SLOTS + s, lane, &at[s]);
            x[s] = load4(T, at[s], n[s]);
        }
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
#pragma unroll
            for (int k = 0; k < 4; ++k) x[s].x[k] *= f;
            if (n[s] > 0) store4(T, at[s], n[s], x[s]);
        }
    }
}

__global__ __launch_bounds__(256) void k_square_sums(List o, double *__restrict__ sums)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const double v = block_sum(squares(o, (int64_t)blockIdx.x * 4 + wave, (int64_t)gridDim.x * 4, threadIdx.x & 63));
    if (threadIdx.x == 0) sums[blockIdx.x] = v;
}

// what follows from the sum of all squares.  One that is not finite: a factor that is NaN, and no step that counts
__device__ __forceinline__ float finish(double v, double max_norm, float *norm, float *factor, int64_t *t_dev)
{
    const double root = sqrt(v);
    const float f = !(v < INFINITY) ? NAN : v > 0.0 && max_norm < root ? (float)(max_norm / root) : 1.f;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        if (norm) *norm = (float)root;
        if (factor) *factor = f;
        if (t_dev && f == f) ++*t_dev;
    }
    return f;
}

// the blocks' sums, added by every block alike
__device__ __forceinline__ double all_sums(const double *__restrict__ sums, int n_sums)
{
    double v = 0.0;
    for (int i = threadIdx.x; i < n_sums; i += 256) v += sums[i];
    return block_sum(v);
}

__global__ __launch_bounds__(256) void k_norm(const double *__restrict__ sums, int n_sums, double max_norm, float *norm, float *factor, int64_t *t_dev)
{
    finish(all_sums(sums, n_sums), max_norm, norm, factor, t_dev);
}

__global__ __launch_bounds__(256) void k_norm_scale(List o, const double *__restrict__ sums, int n_sums, double max_norm, float *norm, float *factor)
{
    const float f = finish(all_sums(sums, n_sums), max_norm, norm, factor, nullptr);
    if (f == 1.f) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    scale_by(o, (int64_t)blockIdx.x * 4 + wave, (int64_t)gridDim.x * 4, threadIdx.x & 63, f);
}

int64_t lists_of(int32_t n_tensors) { return cdiv(n_tensors > 0 ? n_tensors : 1, LIST_MAX); }

// the tensors from number `from` on, as many as one launch takes
void make_list(const kge_grad_tensor *tensors, int32_t n_tensors, int32_t from, List *o)
{
    o->n = 0;
    o->units = 0;
    for (int32_t i = from; i < n_tensors && i < from + LIST_MAX; ++i) {
        const kge_grad_tensor &x = tensors[i];
        if (x.n_rows == 0 || x.d == 0) continue;
        Tensor T;
        T.g = x.grad; T.mask = x.row_mask; T.d = x.d; T.n_rows = x.n_rows; T.bf16 = x.dtype == KGE_DT_BF16;
        if (!T.mask) { T.d = x.n_rows * x.d; T.n_rows = 1; }
        T.nb = cdiv(T.d, 256);
        T.lanes = 1;
        while (T.lanes < 64 && 4 * T.lanes < T.d) T.lanes *= 2;
        T.first = o->units;
        o->units += cdiv(T.lanes == 64 ? T.n_rows * T.nb : cdiv(T.n_rows, 64 / T.lanes), SLOTS);
        o->t[o->n++] = T;
    }
}

int check_list(const kge_grad_tensor *tensors, int32_t n_tensors, double max_norm)
{
    KGE_REQUIRE(n_tensors >= 0, KGE_EINVAL, "negative number of tensors");
    KGE_REQUIRE(tensors || n_tensors == 0, KGE_EINVAL, "NULL argument");
    KGE_REQUIRE(max_norm >= 0.0, KGE_EINVAL, "max_norm must be zero or more");
    for (int32_t i = 0; i < n_tensors; ++i) {
        const kge_grad_tensor &x = tensors[i];
        KGE_REQUIRE(x.n_rows >= 0 && x.d >= 0, KGE_EINVAL, "tensor %d: negative size", i);
        KGE_REQUIRE(x.dtype == KGE_DT_F32 || x.dtype == KGE_DT_BF16, KGE_EINVAL, "tensor %d: bad type", i);
        KGE_REQUIRE(x.d == 0 || x.n_rows <= (MOST_ELEMENTS - 1) / x.d, KGE_ERANGE, "tensor %d: 2^36 elements or more", i);
        if (x.n_rows == 0 || x.d == 0) continue;
        KGE_REQUIRE(x.grad, KGE_EINVAL, "tensor %d: NULL gradient", i);
        KGE_REQUIRE((uintptr_t)x.grad % (x.dtype == KGE_DT_F32 ? 4 : 2) == 0, KGE_EINVAL, "tensor %d: not aligned to its elements", i);
    }
    return KGE_OK;
}

// t_dev: with the norm alone
int run(const kge_grad_tensor *tensors, int32_t n_tensors, double max_norm, bool scale, float *norm, float *factor, int64_t *t_dev,
        void *workspace, size_t ws_bytes, hipStream_t st)
{
    int rc = check_list(tensors, n_tensors, max_norm);
    if (rc != KGE_OK) return rc;
    KGE_REQUIRE((norm || factor || scale) && (uintptr_t)norm % 4 == 0 && (uintptr_t)factor % 4 == 0, KGE_EINVAL,
                "norm and factor: addresses of a float each are wanted, one of them at least");
    KGE_REQUIRE(workspace && (uintptr_t)workspace % 256 == 0, KGE_EINVAL, "the workspace is NULL or not aligned to 256 bytes");
    KGE_REQUIRE(ws_bytes >= kge_grad_norm_workspace_bytes(n_tensors), KGE_ENOMEM, "the workspace is too small");
    double *sums = (double *)workspace;
    int n_sums = 0;
    List o;
    KGE_PROF("grad_norm", st);
    for (int32_t from = 0; from < n_tensors; from += LIST_MAX) {
        make_list(tensors, n_tensors, from, &o);
        if (o.n == 0) continue;
        const int64_t blocks = cdiv(o.units, 4) < BLOCKS_MAX ? cdiv(o.units, 4) : BLOCKS_MAX;
        k_square_sums<<<(unsigned)blocks, 256, 0, st>>>(o, sums + n_sums);
        KGE_LAUNCH_CHECK();
        n_sums += (int)blocks;
    }
    bool told = false;
    for (int32_t from = 0; scale && from < n_tensors; from += LIST_MAX) {
        if (n_tensors > LIST_MAX) make_list(tensors, n_tensors, from, &o);      // one list: it is there already
        if (o.n == 0) continue;
        const int64_t blocks = cdiv(o.units, 4) < BLOCKS_MAX ? cdiv(o.units, 4) : BLOCKS_MAX;
        k_norm_scale<<<(unsigned)blocks, 256, 0, st>>>(o, sums, n_sums, max_norm, told ? nullptr : norm, told ? nullptr : factor);
        KGE_LAUNCH_CHECK();
        told = true;
    }
    if (!told) {
        k_norm<<<1, 256, 0, st>>>(sums, n_sums, max_norm, norm, factor, t_dev);
        KGE_LAUNCH_CHECK();
    }
    return KGE_OK;
}

}  // namespace

extern "C" size_t kge_grad_norm_workspace_bytes(int32_t n_tensors)
{
    if (n_tensors < 0) {
        kge_set_error("negative number of tensors");
        return 0;
    }
    return (size_t)lists_of(n_tensors) * BLOCKS_MAX * sizeof(double);
}

extern "C" int kge_grad_norm(const kge_grad_tensor *tensors, int32_t n_tensors, double max_norm, float *norm, float *factor, void *workspace,
                             size_t ws_bytes, void *stream)
{
    return run(tensors, n_tensors, max_norm, false, norm, factor, nullptr, workspace, ws_bytes, (hipStream_t)stream);
}

extern "C" int kge_grad_norm_step(const kge_grad_tensor *tensors, int32_t n_tensors, double max_norm, float *norm, float *factor,
                                  int64_t *t_dev, void *workspace, size_t ws_bytes, void *stream)
{
    KGE_REQUIRE(t_dev && (uintptr_t)t_dev % 8 == 0, KGE_EINVAL, "t_dev: the address of an int64 is wanted");
    return run(tensors, n_tensors, max_norm, false, norm, factor, t_dev, workspace, ws_bytes, (hipStream_t)stream);
}

extern "C" int kge_clip_grads(const kge_grad_tensor *tensors, int32_t n_tensors, double max_norm, float *norm, float *factor, void *workspace,
                              size_t ws_bytes, void *stream)
{
    return run(tensors, n_tensors, max_norm, true, norm, factor, nullptr, workspace, ws_bytes, (hipStream_t)stream);
}
