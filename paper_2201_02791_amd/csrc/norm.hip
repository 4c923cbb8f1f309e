// Layer norm of rows (Ba, Kiros & Hinton 2016) and its backward pass.
//
//   mean = (1/d) sum x;  rstd = 1 / sqrt((1/d) sum (x - mean)^2 + eps);  xh = (x - mean) rstd;  y = xh gamma + beta
//   u = dy gamma;  dx = rstd (u - mean(u) - xh mean(u xh));  dgamma = sum over rows of dy xh;  dbeta = sum of dy
//
// A row is read once and stays in registers: the deviations are taken from the mean itself, not from a difference of two
// large sums.  A group of G lanes holds a row of up to 4 G V elements, 4 consecutive ones per lane and step; G is part of a
// wavefront for rows of up to 128 elements, a wavefront up to 2048 and a block of 256 or 1024 threads beyond, where the
// sums of a row go through LDS.  Backward: blocks take rows in turn and keep the sums for dgamma and dbeta of their
// columns in registers over all their rows, 2 x 4 V per lane; a second launch adds the blocks' rows in a fixed order, so
// that the result repeats bit for bit.  Statistics and sums are fp32 whatever the rows' type.
//
// Bandwidth bound: forward a row is read and written once, backward two rows are read and one is written.  Rows of up to 256
// elements are taken four at a time per group, of up to 512 two, so that a lane's loads cover the memory's latency: 2.9 million
// fp32 rows of 128 forward 566 us, 5.3 TB/s (589 us one at a time); a million bf16 rows of 256 with fp32 gradients backward
// 380 us, 5.4 TB/s (455 us).
#include "common.h"

#include <type_traits>

namespace {

// four elements at any element's address
struct __attribute__((packed, aligned(4))) F4 { float x[4]; };
struct __attribute__((packed, aligned(2))) H4 { uint32_t w[2]; };

template <class T> struct Elem;
template <> struct Elem<float> {
    static __device__ __forceinline__ void load(const float *a, float x[4])
    {
        const F4 q = *reinterpret_cast<const F4 *>(a);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = q.x[k];
    }
    static __device__ __forceinline__ void store(float *a, const float x[4]) { *reinterpret_cast<F4 *>(a) = F4{{x[0], x[1], x[2], x[3]}}; }
    static __device__ __forceinline__ float one(const float *a) { return *a; }
    static __device__ __forceinline__ void put(float *a, float x) { *a = x; }
};
template <> struct Elem<__bf16> {
    static __device__ __forceinline__ void load(const __bf16 *a, float x[4])
    {
        const H4 q = *reinterpret_cast<const H4 *>(a);
        x[0] = __uint_as_float(q.w[0] << 16); x[1] = __uint_as_float(q.w[0] & 0xffff0000u);
        x[2] = __uint_as_float(q.w[1] << 16); x[3] = __uint_as_float(q.w[1] & 0xffff0000u);
    }
    static __device__ __forceinline__ void store(__bf16 *a, const float x[4])
    {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        const bf16x4 q = {(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
        *reinterpret_cast<H4 *>(a) = __builtin_bit_cast(H4, q);
    }
    static __device__ __forceinline__ float one(const __bf16 *a) { return (float)*a; }
    static __device__ __forceinline__ void put(__bf16 *a, float x) { *a = (__bf16)x; }
};

// WHOLE: d is a multiple of 4, so that a lane's four elements are all inside the row or all outside
template <bool WHOLE, class T>
__device__ __forceinline__ void get4(const T *a, int n, float x[4])
{
    if (WHOLE ? n > 0 : n >= 4) Elem<T>::load(a, x);
    else {
        x[0] = x[1] = x[2] = x[3] = 0.f;
        if (!WHOLE && n > 0) {                   // past the end the last element again: no branch parts the loads
#pragma unroll
            for (int k = 0; k < 3; ++k) x[k] = Elem<T>::one(a + min(k, n - 1));
            x[1] = n > 1 ? x[1] : 0.f;
            x[2] = n > 2 ? x[2] : 0.f;
        }
    }
}
template <bool WHOLE, class T>
__device__ __forceinline__ void put4(T *a, int n, const float x[4])
{
    if (WHOLE ? n > 0 : n >= 4) Elem<T>::store(a, x);
    else if (!WHOLE) {
#pragma unroll
        for (int k = 0; k < 3; ++k) if (k < n) Elem<T>::put(a + k, x[k]);
    }
}

// sum over the G lanes of a row's group; every lane gets it.  Groups of more than a wavefront are a whole block (then all
// its threads call this together); each sum of a kernel has an LDS row of its own, `side`, so that one barrier is enough.
template <int G>
__device__ __forceinline__ float group_sum(float v, float (*lds)[16], int side)
{
#pragma unroll
    for (int off = (G < 64 ? G : 64) >> 1; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    if constexpr (G > 64) {
        if ((threadIdx.x & 63) == 0) lds[side][threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < G / 64; ++w) v += lds[side][w];
    }
    return v;
}

// rows that a group has in flight: what one lane's loads leave of the memory's rate
constexpr int rows_at_once(int V) { return V == 1 ? 4 : V == 2 ? 2 : 1; }

template <int G, int V, bool WHOLE, class TX, class TY>
__global__ __launch_bounds__(G > 256 ? G : 256) void k_norm_forward(const TX *__restrict__ X, int64_t ldx, int64_t n, int32_t d,
                                                                     const float *__restrict__ gamma, const float *__restrict__ beta, float eps,
                                                                     TY *__restrict__ Y, int64_t ldy, float *__restrict__ mean_out,
                                                                     float *__restrict__ rstd_out)
{
    constexpr int NT = G > 256 ? G : 256, ROWS = NT / G, U = rows_at_once(V);
    __shared__ float lds[3][16];
    const int l = threadIdx.x & (G - 1);
    const int64_t row0 = (int64_t)blockIdx.x * (ROWS * U) + threadIdx.x / G;
    float x[U][V][4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t row = row0 + u * ROWS;     // whether it exists is uniform over the group; the exchanges below stay inside it
#pragma unroll
        for (int c = 0; c < V; ++c) {
            const int at = (c * G + l) * 4;
            get4<WHOLE>(X + row * ldx + at, row < n ? d - at : 0, x[u][c]);
        }
    }
    const float inv_d = 1.f / (float)d;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t row = row0 + u * ROWS;
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < V; ++c) s += (x[u][c][0] + x[u][c][1]) + (x[u][c][2] + x[u][c][3]);
        float mean = group_sum<G>(s, lds, 0) * inv_d;
        // the deviations' own mean is what rounding left of the row's: it is taken out of them and of their mean square, so that a
        // row of one value has neither
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int c = 0; c < V; ++c) {
            const int left = d - (c * G + l) * 4;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                x[u][c][k] -= mean;
                if (k < left) { s1 += x[u][c][k]; s2 += x[u][c][k] * x[u][c][k]; }
            }
        }
        const float rest = group_sum<G>(s1, lds, 1) * inv_d;
        const float square = group_sum<G>(s2, lds, 2) * inv_d;
        const float var = square - rest * rest;
        const float rstd = 1.f / sqrtf((var < 0.f ? 0.f : var) + eps);      // a NaN stays one
        mean += rest;
        if (row >= n) continue;
#pragma unroll
        for (int c = 0; c < V; ++c) {
            const int at = (c * G + l) * 4, left = d - at;
            float g[4] = {1.f, 1.f, 1.f, 1.f}, b[4] = {0.f, 0.f, 0.f, 0.f};
            if (gamma) get4<WHOLE>(gamma + at, left, g);
            if (beta) get4<WHOLE>(beta + at, left, b);
#pragma unroll
            for (int k = 0; k < 4; ++k) x[u][c][k] = (x[u][c][k] - rest) * rstd * g[k] + b[k];
            put4<WHOLE>(Y + row * ldy + at, left, x[u][c]);
        }
        if (l == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }
    }
}

// sums_g, sums_b (each if wanted): the block's sums of dy xh and of dy, `step` elements behind those of the block before
template <int G, int V, bool WHOLE, class TX, class TY>
__global__ __launch_bounds__(G > 256 ? G : 256) void k_norm_backward(const TX *__restrict__ X, int64_t ldx, int64_t n, int32_t d,
                                                                      const float *__restrict__ gamma, const float *__restrict__ mean_in,
                                                                      const float *__restrict__ rstd_in, const TY *__restrict__ dY,
                                                                      int64_t lddy, TX *__restrict__ dX, int64_t lddx, float *__restrict__ sums_g,
                                                                      float *__restrict__ sums_b, int64_t step)
{
    constexpr int NT = G > 256 ? G : 256, ROWS = NT / G;
    __shared__ float sums[ROWS > 1 ? NT * 4 * V : 1];
    const int l = threadIdx.x & (G - 1), sub = threadIdx.x / G;
    const float inv_d = 1.f / (float)d;
    float g[V][4], dg[V][4], db[V][4];
#pragma unroll
    for (int c = 0; c < V; ++c) {
        const int at = (c * G + l) * 4;
        if (gamma) get4<WHOLE>(gamma + at, d - at, g[c]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (!gamma) g[c][k] = 1.f;
            dg[c][k] = db[c][k] = 0.f;
        }
    }
    constexpr int U = rows_at_once(V);
    int side = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * (ROWS * U); row0 < n; row0 += (int64_t)gridDim.x * (ROWS * U)) {
        float x[U][V][4], g_y[U][V][4], mean[U], rstd[U];
#pragma unroll
        for (int q = 0; q < U; ++q) {
            const int64_t row = row0 + q * ROWS + sub;
            const bool in = row < n;
            mean[q] = in ? mean_in[row] : 0.f;
            rstd[q] = in ? rstd_in[row] : 0.f;
#pragma unroll
            for (int c = 0; c < V; ++c) {
                const int at = (c * G + l) * 4;
                get4<WHOLE>(X + row * ldx + at, in ? d - at : 0, x[q][c]);
                get4<WHOLE>(dY + row * lddy + at, in ? d - at : 0, g_y[q][c]);
            }
        }
#pragma unroll
        for (int q = 0; q < U; ++q) {
            const int64_t row = row0 + q * ROWS + sub;
            float su = 0.f, sx = 0.f;
#pragma unroll
            for (int c = 0; c < V; ++c) {
                const int left = d - (c * G + l) * 4;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float &xh = x[q][c][k], &u = g_y[q][c][k];
                    xh = k < left ? (xh - mean[q]) * rstd[q] : 0.f;
                    dg[c][k] += u * xh;
                    db[c][k] += u;
                    u *= g[c][k];
                    su += u;
                    sx += u * xh;
                }
            }
            if (!dX) continue;                   // uniform over the grid
            if constexpr (G > 64) {
                // two sums, one barrier: they travel in the two halves of the row that `side` names
                for (int off = 32; off > 0; off >>= 1) { su += __shfl_xor(su, off, 64); sx += __shfl_xor(sx, off, 64); }
                __shared__ float two[2][2][16];
                if ((threadIdx.x & 63) == 0) { two[side][0][threadIdx.x >> 6] = su; two[side][1][threadIdx.x >> 6] = sx; }
                __syncthreads();
                su = sx = 0.f;
#pragma unroll
                for (int w = 0; w < G / 64; ++w) { su += two[side][0][w]; sx += two[side][1][w]; }
                side ^= 1;
            } else {
                su = group_sum<G>(su, nullptr, 0);
                sx = group_sum<G>(sx, nullptr, 0);
            }
            su *= inv_d; sx *= inv_d;
            if (row >= n) continue;
#pragma unroll
            for (int c = 0; c < V; ++c) {
                const int at = (c * G + l) * 4;
#pragma unroll
                for (int k = 0; k < 4; ++k) x[q][c][k] = rstd[q] * (g_y[q][c][k] - su - x[q][c][k] * sx);
                put4<WHOLE>(dX + row * lddx + at, d - at, x[q][c]);
            }
        }
    }
    if (!sums_g && !sums_b) return;
    if (sums_g) sums_g += blockIdx.x * step;
    if (sums_b) sums_b += blockIdx.x * step;
    if constexpr (ROWS > 1) {                    // the block's groups, in their order
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (which) __syncthreads();
#pragma unroll
            for (int c = 0; c < V; ++c)
#pragma unroll
                for (int k = 0; k < 4; ++k) sums[sub * 4 * V * G + (c * G + l) * 4 + k] = which ? db[c][k] : dg[c][k];
            __syncthreads();
            float *const to = which ? sums_b : sums_g;
            for (int i = threadIdx.x; to && i < d; i += NT) {
                float s = 0.f;
#pragma unroll
                for (int r = 0; r < ROWS; ++r) s += sums[r * 4 * V * G + i];
                to[i] = s;
            }
        }
    } else {
#pragma unroll
        for (int c = 0; c < V; ++c) {
            const int at = (c * G + l) * 4;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (at + k < d) {
                    if (sums_g) sums_g[at + k] = dg[c][k];
                    if (sums_b) sums_b[at + k] = db[c][k];
                }
        }
    }
}

// column sums of part [blocks][2 d]: 32 columns a block, 32 rows side by side, then these in their order
__global__ __launch_bounds__(1024) void k_norm_sum(const float *__restrict__ part, int32_t blocks, int32_t d, float *__restrict__ dgamma,
                                                   float *__restrict__ dbeta)
{
    __shared__ float s[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + x;
    float v = 0.f;
    if (c < 2 * d) {
        int r = y;
        for (; r + 7 * 32 < blocks; r += 8 * 32) {       // eight loads on their way, added in the rows' order
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = part[(int64_t)(r + 32 * k) * 2 * d + c];
#pragma unroll
            for (int k = 0; k < 8; ++k) v += x[k];
        }
        for (; r < blocks; r += 32) v += part[(int64_t)r * 2 * d + c];
    }
    s[y][x] = v;
    __syncthreads();
    if (y == 0 && c < 2 * d) {
        v = 0.f;
#pragma unroll
        for (int r = 0; r < 32; ++r) v += s[r][x];
        float *out = c < d ? dgamma : dbeta;
        if (out) out[c < d ? c : c - d] = v;
    }
}

constexpr int32_t MAX_D = 16384;

// rows that a block holds at a time, for rows of d elements
int rows_of(int32_t d) { return d <= 64 ? 16 : d <= 128 ? 8 : d <= 2048 ? 4 : 1; }
int64_t backward_blocks(int64_t n, int32_t d)
{
    const int64_t most = d <= 2048 ? 1024 : 512, want = cdiv(n, rows_of(d) * rows_at_once(d <= 256 ? 1 : d <= 512 ? 2 : 4));
    return want < most ? want : most;
}

int check(const kge_norm *L, int64_t n_rows)
{
    KGE_REQUIRE(L, KGE_EINVAL, "NULL argument");
    KGE_REQUIRE(L->d >= 1 && L->d <= MAX_D, KGE_EINVAL, "layer norm: rows have 1 to %d elements", MAX_D);
    KGE_REQUIRE((L->x_dtype == KGE_DT_F32 || L->x_dtype == KGE_DT_BF16) && (L->y_dtype == KGE_DT_F32 || L->y_dtype == KGE_DT_BF16),
                KGE_EINVAL, "layer norm: bad type");
    KGE_REQUIRE(L->eps >= 0.f, KGE_EINVAL, "layer norm: eps must not be negative");
    KGE_REQUIRE(n_rows >= 0, KGE_EINVAL, "layer norm: negative number of rows");
    KGE_REQUIRE(n_rows <= 0x7fffffffLL, KGE_ERANGE, "layer norm: at most 2^31 - 1 rows");
    return KGE_OK;
}

size_t bytes_of(int32_t dtype) { return dtype == KGE_DT_BF16 ? 2 : 4; }

// calls f(G, V) with the group and the steps that rows of d elements take
template <class F>
void with_shape(int32_t d, F f)
{
    if (d <= 64) f(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
    else if (d <= 128) f(std::integral_constant<int, 32>(), std::integral_constant<int, 1>());
    else if (d <= 256) f(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
    else if (d <= 512) f(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
    else if (d <= 1024) f(std::integral_constant<int, 64>(), std::integral_constant<int, 4>());
    else if (d <= 2048) f(std::integral_constant<int, 64>(), std::integral_constant<int, 8>());
    else if (d <= 4096) f(std::integral_constant<int, 256>(), std::integral_constant<int, 4>());
    else if (d <= 8192) f(std::integral_constant<int, 256>(), std::integral_constant<int, 8>());
    else f(std::integral_constant<int, 1024>(), std::integral_constant<int, 4>());
}
template <class F>
void with_types(const kge_norm *L, bool whole, F f)
{
    auto types = [&](auto v) {
        if (L->x_dtype == KGE_DT_F32) {
            if (L->y_dtype == KGE_DT_F32) f(v, float{}, float{});
            else f(v, float{}, __bf16{});
        } else {
            if (L->y_dtype == KGE_DT_F32) f(v, __bf16{}, float{});
            else f(v, __bf16{}, __bf16{});
        }
    };
    if (whole) types(std::true_type());
    else types(std::false_type());
}

}  // namespace

extern "C" int kge_layer_norm_forward(const kge_norm *L, int64_t n_rows, const void *X, int64_t ldx, void *Y, int64_t ldy, float *mean,
                                      float *rstd, void *stream)
{
    int rc = check(L, n_rows);
    if (rc != KGE_OK) return rc;
    const int32_t d = L->d;
    KGE_REQUIRE(ldx >= d && ldy >= d, KGE_EINVAL, "layer norm: a row stride is smaller than the row");
    if (n_rows == 0) return KGE_OK;
    KGE_REQUIRE(X && Y, KGE_EINVAL, "NULL argument");
    KGE_REQUIRE(((uintptr_t)X % bytes_of(L->x_dtype)) == 0 && ((uintptr_t)Y % bytes_of(L->y_dtype)) == 0 &&
                    ((uintptr_t)L->gamma % 4) == 0 && ((uintptr_t)L->beta % 4) == 0 && ((uintptr_t)mean % 4) == 0 && ((uintptr_t)rstd % 4) == 0,
                KGE_EINVAL, "layer norm: an array is not aligned to its elements");
    hipStream_t st = (hipStream_t)stream;
    KGE_PROF("layer_norm", st);
    with_shape(d, [&](auto G, auto V) {
        with_types(L, d % 4 == 0, [&](auto v, auto tx, auto ty) {
            typedef decltype(tx) TX;
            typedef decltype(ty) TY;
            constexpr int nt = G.value > 256 ? G.value : 256, rows = nt / G.value * rows_at_once(V.value);
            constexpr int64_t most = (int64_t)rows * (0x7fffffff / nt);      // a launch has fewer than 2^32 threads
            for (int64_t r = 0; r < n_rows; r += most) {
                const int64_t n = n_rows - r < most ? n_rows - r : most;
                k_norm_forward<G.value, V.value, v.value, TX, TY><<<(unsigned)cdiv(n, rows), nt, 0, st>>>(
                    (const TX *)X + r * ldx, ldx, n, d, L->gamma, L->beta, L->eps, (TY *)Y + r * ldy, ldy, mean ? mean + r : nullptr,
                    rstd ? rstd + r : nullptr);
            }
        });
    });
    KGE_LAUNCH_CHECK();
    return KGE_OK;
}

extern "C" size_t kge_layer_norm_workspace_bytes(const kge_norm *L, int64_t n_rows)
{
    if (check(L, n_rows) != KGE_OK) return 0;
    return align_up((size_t)(n_rows > 0 ? backward_blocks(n_rows, L->d) : 1) * 2 * L->d * sizeof(float), 256);
}

extern "C" int kge_layer_norm_backward(const kge_norm *L, int64_t n_rows, const void *X, int64_t ldx, const float *mean, const float *rstd,
                                       const void *dY, int64_t lddy, void *dX, int64_t lddx, float *dgamma, float *dbeta, void *workspace,
                                       size_t ws_bytes, void *stream)
{
    int rc = check(L, n_rows);
    if (rc != KGE_OK) return rc;
    const int32_t d = L->d;
    KGE_REQUIRE(ldx >= d && lddy >= d && (!dX || lddx >= d), KGE_EINVAL, "layer norm: a row stride is smaller than the row");
    KGE_REQUIRE(n_rows == 0 || (X && mean && rstd && dY), KGE_EINVAL, "NULL argument");
    KGE_REQUIRE(((uintptr_t)X % bytes_of(L->x_dtype)) == 0 && ((uintptr_t)dX % bytes_of(L->x_dtype)) == 0 &&
                    ((uintptr_t)dY % bytes_of(L->y_dtype)) == 0 && ((uintptr_t)L->gamma % 4) == 0 && ((uintptr_t)mean % 4) == 0 &&
                    ((uintptr_t)rstd % 4) == 0 && ((uintptr_t)dgamma % 4) == 0 && ((uintptr_t)dbeta % 4) == 0,
                KGE_EINVAL, "layer norm: an array is not aligned to its elements");
    const bool want = dgamma || dbeta;
    hipStream_t st = (hipStream_t)stream;
    if (want) {
        KGE_REQUIRE(workspace && ((uintptr_t)workspace % 256) == 0, KGE_EINVAL, "layer norm: the workspace must be 256-byte aligned");
        KGE_REQUIRE(ws_bytes >= kge_layer_norm_workspace_bytes(L, n_rows), KGE_ENOMEM, "layer norm: workspace too small");
    }
    const int64_t blocks = backward_blocks(n_rows, d);
    // one block's sums are the result
    float *const sums_g = !want ? nullptr : blocks == 1 ? dgamma : (float *)workspace;
    float *const sums_b = !want ? nullptr : blocks == 1 ? dbeta : (float *)workspace + d;
    if (n_rows > 0 && (want || dX)) {
        KGE_PROF("layer_norm_bwd", st);
        with_shape(d, [&](auto G, auto V) {
            with_types(L, d % 4 == 0, [&](auto v, auto tx, auto ty) {
                typedef decltype(tx) TX;
                typedef decltype(ty) TY;
                constexpr int nt = G.value > 256 ? G.value : 256;
                k_norm_backward<G.value, V.value, v.value, TX, TY><<<(unsigned)blocks, nt, 0, st>>>(
                    (const TX *)X, ldx, n_rows, d, L->gamma, mean, rstd, (const TY *)dY, lddy, (TX *)dX, lddx, sums_g, sums_b, 2 * (int64_t)d);
            });
        });
        KGE_LAUNCH_CHECK();
    }
    if (want && blocks != 1) {                   // without rows: sums of nothing, zeros
        KGE_PROF("layer_norm_sum", st);
        k_norm_sum<<<(unsigned)cdiv(2 * (int64_t)d, 32), 1024, 0, st>>>((const float *)workspace, (int32_t)blocks, d, dgamma, dbeta);
        KGE_LAUNCH_CHECK();
    }
    return KGE_OK;
}
