// Layer norm over the rows of a matrix, forward and backward with the reduction of the weights' gradients (gfx950).
//   mu = mean x, r = (mean (x - mu)^2 + eps)^-1/2, xh = (x - mu) r, y = xh gamma + beta
//   g = dy gamma:  dx = r (g - mean g - xh mean(g xh)),  dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy
// A few operations an element: bound by HBM traffic.
#include "row_ops.h"

namespace omni {

// One workgroup per row.  The row stays in registers between its three uses (mean, squares about the mean, output) where
// BLOCK * CHUNKS chunks hold it; CHUNKS == 0: a longer row is read three times, the second and third time from the caches.
// The squares are summed about the mean, not as mean x^2 - mu^2, which cancels where |mu| is large against the spread.
template <typename T, int BLOCK, int CHUNKS>
__global__ __launch_bounds__(BLOCK) void layer_norm_forward_kernel(const T *x, int64_t ldx, int64_t rows, int n, float eps, const float *__restrict__ gamma,
                                                                   const float *__restrict__ beta, T *y, int64_t ldy, float *__restrict__ mean, float *__restrict__ rstd)
{
    constexpr int V = CHUNK<T>, KEPT = CHUNKS > 0 ? CHUNKS : 1;
    __shared__ float lds[BLOCK / 64];
    const int64_t r = grid_row();
    if (r >= rows) return;
    const T *row = x + r * ldx;
    T *out = y + r * ldy;
    const int chunks = CHUNKS > 0 ? CHUNKS : (n + BLOCK * V - 1) / (BLOCK * V);
    float v[KEPT][V], sum[1] = {0.f};
    for (int c = 0; c < chunks; ++c) {
        float(&w)[V] = v[CHUNKS > 0 ? c : 0];
        load_chunk(row, (c * BLOCK + (int)threadIdx.x) * V, n, 0.f, w);
#pragma unroll
        for (int j = 0; j < V; ++j) sum[0] += w[j];
    }
    block_join<BLOCK>(sum, lds, Add());
    const float mu = sum[0] / (float)n;
    sum[0] = 0.f;
    for (int c = 0; c < chunks; ++c) {
        const int at = (c * BLOCK + (int)threadIdx.x) * V;
        float(&w)[V] = v[CHUNKS > 0 ? c : 0];
        if (CHUNKS == 0) load_chunk(row, at, n, 0.f, w);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float d = at + j < n ? w[j] - mu : 0.f;
            sum[0] += d * d;
        }
    }
    block_join<BLOCK>(sum, lds, Add());
    const float rs = 1.0f / sqrtf(sum[0] / (float)n + eps);
    if (threadIdx.x == 0) {
        if (mean != nullptr) mean[r] = mu;
        if (rstd != nullptr) rstd[r] = rs;
    }
    for (int c = 0; c < chunks; ++c) {
        const int at = (c * BLOCK + (int)threadIdx.x) * V;
        float(&w)[V] = v[CHUNKS > 0 ? c : 0], ga[V], be[V];
        if (at >= n) break;
        if (CHUNKS == 0) load_chunk(row, at, n, 0.f, w);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            ga[j] = gamma != nullptr && at + j < n ? gamma[at + j] : 1.f;
            be[j] = beta != nullptr && at + j < n ? beta[at + j] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < V; ++j) w[j] = (w[j] - mu) * rs * ga[j] + be[j];
        store_chunk(out, at, n, w);
    }
}

// The data gradient, one workgroup per row, x and dy in registers between the sums and the output in the same way.
template <typename T, int BLOCK, int CHUNKS>
__global__ __launch_bounds__(BLOCK) void layer_norm_dx_kernel(const T *x, int64_t ldx, const T *dy, int64_t lddy, int64_t rows, int n, const float *__restrict__ gamma,
                                                              const float *__restrict__ mean, const float *__restrict__ rstd, T *dx, int64_t lddx)
{
    constexpr int V = CHUNK<T>, KEPT = CHUNKS > 0 ? CHUNKS : 1;
    __shared__ float lds[2 * (BLOCK / 64)];
    const int64_t r = grid_row();
    if (r >= rows) return;
    const T *xr = x + r * ldx, *dr = dy + r * lddy;
    T *out = dx + r * lddx;
    const float mu = mean[r], rs = rstd[r];
    const int chunks = CHUNKS > 0 ? CHUNKS : (n + BLOCK * V - 1) / (BLOCK * V);
    float xh[KEPT][V], g[KEPT][V], sums[2] = {0.f, 0.f};
    auto take = [&](int at, float(&a)[V], float(&b)[V]) {
        load_chunk(xr, at, n, mu, a);
        load_chunk(dr, at, n, 0.f, b);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            a[j] = (a[j] - mu) * rs;
            if (gamma != nullptr && at + j < n) b[j] *= gamma[at + j];
        }
    };
    for (int c = 0; c < chunks; ++c) {
        float(&a)[V] = xh[CHUNKS > 0 ? c : 0], (&b)[V] = g[CHUNKS > 0 ? c : 0];
        take((c * BLOCK + (int)threadIdx.x) * V, a, b);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            sums[0] += b[j];
            sums[1] += b[j] * a[j];
        }
    }
    block_join<BLOCK>(sums, lds, Add());
    const float mg = sums[0] / (float)n, mgx = sums[1] / (float)n;
    for (int c = 0; c < chunks; ++c) {
        const int at = (c * BLOCK + (int)threadIdx.x) * V;
        if (at >= n) break;
        float(&a)[V] = xh[CHUNKS > 0 ? c : 0], (&b)[V] = g[CHUNKS > 0 ? c : 0], o[V];
        if (CHUNKS == 0) take(at, a, b);
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = rs * (b[j] - mg - a[j] * mgx);
        store_chunk(out, at, n, o);
    }
}

// dgamma and dbeta: a workgroup adds LN_COLS chunks of columns over one range of rows, 256 / LN_COLS rows at a time, and
// joins them in LDS; `part` [ranges][2][n] receives the range's sums (one range: they go straight to dgamma and dbeta).
constexpr int LN_COLS = 8;

template <typename T>
__global__ __launch_bounds__(256) void layer_norm_weights_kernel(const T *__restrict__ x, int64_t ldx, const T *__restrict__ dy, int64_t lddy, int64_t rows, int n,
                                                                 const float *__restrict__ mean, const float *__restrict__ rstd, int64_t range, float *__restrict__ part,
                                                                 float *__restrict__ dgamma, float *__restrict__ dbeta)
{
    constexpr int V = CHUNK<T>, LANES = 256 / LN_COLS;
    __shared__ float lds[2][V][256 + 8];
    const int col = threadIdx.x % LN_COLS, lane = threadIdx.x / LN_COLS, at = (blockIdx.x * LN_COLS + col) * V;
    const int64_t r0 = blockIdx.y * range, r1 = r0 + range < rows ? r0 + range : rows;
    float ga[V], be[V];
#pragma unroll
    for (int j = 0; j < V; ++j) ga[j] = be[j] = 0.f;
    if (at < n)
        for (int64_t r = r0 + lane; r < r1; r += LANES) {
            const float mu = mean[r], rs = rstd[r];
            float a[V], b[V];
            load_chunk(x + r * ldx, at, n, mu, a);
            load_chunk(dy + r * lddy, at, n, 0.f, b);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                ga[j] += b[j] * ((a[j] - mu) * rs);
                be[j] += b[j];
            }
        }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        lds[0][j][threadIdx.x] = ga[j];
        lds[1][j][threadIdx.x] = be[j];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * V * LN_COLS; i += 256) {
        const int which = i / (V * LN_COLS), c = i / V % LN_COLS, j = i % V;
        float s = 0.f;
        for (int l = 0; l < LANES; ++l) s += lds[which][j][l * LN_COLS + c];
        const int to = (blockIdx.x * LN_COLS + c) * V + j;
        if (to >= n) continue;
        if (part != nullptr) part[((int64_t)blockIdx.y * 2 + which) * n + to] = s;
        else if (which == 0 && dgamma != nullptr) dgamma[to] = s;
        else if (which == 1 && dbeta != nullptr) dbeta[to] = s;
    }
}

__global__ __launch_bounds__(256) void layer_norm_join_kernel(const float *__restrict__ part, int ranges, int n, float *__restrict__ dgamma, float *__restrict__ dbeta)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= 2 * (int64_t)n) return;
    float s = 0.f;
    for (int k = 0; k < ranges; ++k) s += part[(int64_t)k * 2 * n + i];
    if (i < n) {
        if (dgamma != nullptr) dgamma[i] = s;
    } else if (dbeta != nullptr) {
        dbeta[i - n] = s;
    }
}

// Ranges of rows of the weights' gradients: about four workgroups per compute unit, 64 rows each at least.  Never fewer for
// more rows; no rows are one empty range, whose sums are zero.
static int64_t weight_ranges(int dtype, int64_t rows, int64_t n)
{
    const int64_t cols = LN_COLS * (16 / (int64_t)elem_size(dtype)), tiles = (n + cols - 1) / cols;
    const int64_t most = (rows + 63) / 64, want = (1024 + tiles - 1) / tiles, ranges = want < most ? want : most;
    return ranges > 1 ? ranges : 1;
}

size_t layer_norm_workspace(int dtype, int64_t rows, int64_t n)
{
    const int64_t ranges = weight_ranges(dtype, rows, n);
    return ranges > 1 ? (size_t)ranges * 2 * n * sizeof(float) : 0;
}

// BLOCK and CHUNKS by the row's length: the smallest workgroup that holds the row in at most four chunks a thread
#define OMNI_LN_BY_LENGTH(LAUNCH)                          \
    do {                                                   \
        const int64_t chunks = (n + CHUNK<T> - 1) / CHUNK<T>; \
        if (chunks <= 64) LAUNCH(64, 1);                   \
        else if (chunks <= 256) LAUNCH(64, 4);             \
        else if (chunks <= 512) LAUNCH(256, 2);            \
        else if (chunks <= 1024) LAUNCH(256, 4);           \
        else if (chunks <= 2048) LAUNCH(512, 4);           \
        else if (chunks <= 4096) LAUNCH(1024, 4);          \
        else LAUNCH(1024, 0);                              \
    } while (0)

template <typename T> static int forward(const LayerNormArgs &a, float eps, const float *beta, T *y, int64_t ldy, float *mean, float *rstd, hipStream_t s)
{
    const int64_t n = a.width;
#define OMNI_LN_FORWARD(B, C)                                                                                                              \
    hipLaunchKernelGGL((layer_norm_forward_kernel<T, B, C>), row_grid(a.rows), dim3(B), 0, s, (const T *)a.x, a.ldx, a.rows, (int)n, eps, a.gamma, beta, \
                       y, ldy, mean, rstd)
    OMNI_LN_BY_LENGTH(OMNI_LN_FORWARD);
#undef OMNI_LN_FORWARD
    OMNI_LAUNCH_CHECK();
    return OMNI_OK;
}

int launch_layer_norm_forward(const LayerNormArgs &a, float eps, const float *beta, void *y, int64_t ldy, float *mean, float *rstd, hipStream_t s)
{
    ProfScope prof(KID_LAYER_NORM, s, 0.0, 2.0 * (double)a.rows * a.width * elem_size(a.dtype));
    return a.dtype == OMNI_BF16 ? forward<bf16_t>(a, eps, beta, (bf16_t *)y, ldy, mean, rstd, s) : forward<float>(a, eps, beta, (float *)y, ldy, mean, rstd, s);
}

template <typename T>
static int backward(const LayerNormArgs &a, const T *dy, int64_t lddy, const float *mean, const float *rstd, T *dx, int64_t lddx, float *dgamma, float *dbeta, float *part,
                    hipStream_t s)
{
    const int64_t n = a.width;
    const T *x = (const T *)a.x;
    if (dgamma != nullptr || dbeta != nullptr) {  // first: dx may be written over x or dy
        const int64_t ranges = weight_ranges(a.dtype, a.rows, n), range = (a.rows + ranges - 1) / ranges, cols = LN_COLS * CHUNK<T>;
        hipLaunchKernelGGL(layer_norm_weights_kernel<T>, dim3((unsigned)((n + cols - 1) / cols), (unsigned)ranges), dim3(256), 0, s, x, a.ldx, dy, lddy, a.rows, (int)n,
                           mean, rstd, range, ranges > 1 ? part : nullptr, dgamma, dbeta);
        OMNI_LAUNCH_CHECK();
        if (ranges > 1) {
            hipLaunchKernelGGL(layer_norm_join_kernel, dim3((unsigned)((2 * n + 255) / 256)), dim3(256), 0, s, part, (int)ranges, (int)n, dgamma, dbeta);
            OMNI_LAUNCH_CHECK();
        }
    }
    if (dx != nullptr) {
#define OMNI_LN_DX(B, C) \
    hipLaunchKernelGGL((layer_norm_dx_kernel<T, B, C>), row_grid(a.rows), dim3(B), 0, s, x, a.ldx, dy, lddy, a.rows, (int)n, a.gamma, mean, rstd, dx, lddx)
        OMNI_LN_BY_LENGTH(OMNI_LN_DX);
#undef OMNI_LN_DX
        OMNI_LAUNCH_CHECK();
    }
    return OMNI_OK;
}

int launch_layer_norm_backward(const LayerNormArgs &a, const void *dy, int64_t lddy, const float *mean, const float *rstd, void *dx, int64_t lddx, float *dgamma,
                               float *dbeta, float *part, hipStream_t s)
{
    ProfScope prof(KID_LAYER_NORM, s, 0.0, (dx != nullptr ? 3.0 : 2.0) * (double)a.rows * a.width * elem_size(a.dtype));
    return a.dtype == OMNI_BF16 ? backward<bf16_t>(a, (const bf16_t *)dy, lddy, mean, rstd, (bf16_t *)dx, lddx, dgamma, dbeta, part, s)
                                : backward<float>(a, (const float *)dy, lddy, mean, rstd, (float *)dx, lddx, dgamma, dbeta, part, s);
}

}  // namespace omni
