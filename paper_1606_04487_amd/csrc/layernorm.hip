// Layer norm over the rows of a matrix, forward and backward with the reduction of the weights' gradients (gfx950).
//   mu = mean x, r = (mean (x - mu)^2 + eps)^-1/2, xh = (x - mu) r, y = xh gamma + beta
//   g = dy gamma:  dx = r (g - mean g - xh mean(g xh)),  dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy
// A few operations an element: bound by memory.
#include "row_ops.h"

namespace omni {

// The sums of N values over the TEAM threads that share a row, to each of them.  lds [N][16] is this join's own: a later join
// with another buffer lies between two uses of one, so one barrier is enough.
template <int TEAM, int N> __device__ __forceinline__ void team_join(float (&v)[N], float (*lds)[16])
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_join(v[i], Add());
    if (TEAM == 64) return;
    constexpr int WAVES = TEAM / 64;
    const int wave = threadIdx.x / 64, first = wave / WAVES * WAVES;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) lds[i][wave] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float r = lds[i][first];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) r += lds[i][first + w];
        v[i] = r;
    }
}

// CHUNK floats of a vector over the columns, or `fill`
template <Fit FIT, int V> __device__ __forceinline__ void load_columns(const float *p, int at, int n, float fill, float (&v)[V])
{
    if (p != nullptr && at + V <= n) {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            const float4 f = *reinterpret_cast<const float4 *>(p + at + j);
            v[j] = f.x, v[j + 1] = f.y, v[j + 2] = f.z, v[j + 3] = f.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = FIT != WHOLE && p != nullptr && at + j < n ? p[at + j] : fill;
    }
}

// ------------------------------------------------------------------------------------------------ forward
// BLOCK threads per row, CHUNKS chunks each, which stay in registers between the row's three uses (mean, squares about the mean,
// output); a workgroup goes on to further rows with gamma and beta in registers too and the next row's loads in flight, since
// from the caches the two of them are 8 bytes an element where a bf16 element itself is 4, read and written.
// The squares are summed about the mean, not as mean x^2 - mu^2, which cancels where |mu| is large against the spread.
template <typename T, int BLOCK, int CHUNKS, Fit FIT>
__global__ __launch_bounds__(BLOCK, BLOCK <= 512 ? (FIT == CUT && BLOCK == 512 ? 4 : 6) : 4) void layer_norm_forward_kernel(const T *x, int64_t ldx, int64_t rows, int n, float eps, const float *__restrict__ gamma,
                                                                   const float *__restrict__ beta, T *y, int64_t ldy, float *__restrict__ mean, float *__restrict__ rstd)
{
    constexpr int V = CHUNK<T>;
    __shared__ float lds[2][1][16];
    const int tid = threadIdx.x;
    float ga[CHUNKS][V], be[CHUNKS][V];
    Raw<T> next[CHUNKS];
    int64_t r = grid_row();
    if (r >= rows) return;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        next[c] = load_raw<FIT>(x + r * ldx, (c * BLOCK + tid) * V, n);
        load_columns<FIT, V>(gamma, (c * BLOCK + tid) * V, n, 1.f, ga[c]);
        load_columns<FIT, V>(beta, (c * BLOCK + tid) * V, n, 0.f, be[c]);
    }
    for (;;) {
        float v[CHUNKS][V], sum[1] = {0.f}, sq[1] = {0.f};
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            settle<FIT>(next[c], (c * BLOCK + tid) * V, n);
            unpack(next[c].w, v[c]);
        }
        const int64_t r2 = r + (int64_t)gridDim.x * gridDim.y;
        if (r2 < rows)
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) next[c] = load_raw<FIT>(x + r2 * ldx, (c * BLOCK + tid) * V, n);
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int j = 0; j < V; ++j) sum[0] += v[c][j];
        team_join<BLOCK>(sum, lds[0]);
        const float mu = sum[0] / (float)n;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int at = (c * BLOCK + tid) * V;
            float q = 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                v[c][j] -= mu;
                if (FIT == WHOLE || at + j < n) q += v[c][j] * v[c][j];
            }
            sq[0] += FIT != WHOLE || at < n ? q : 0.f;
        }
        team_join<BLOCK>(sq, lds[1]);
        const float rs = 1.0f / sqrtf(sq[0] / (float)n + eps);
        if (tid == 0) {
            if (mean != nullptr) mean[r] = mu;
            if (rstd != nullptr) rstd[r] = rs;
        }
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
#pragma unroll
            for (int j = 0; j < V; ++j) v[c][j] = v[c][j] * rs * ga[c][j] + be[c][j];
            store_chunk<FIT>(y + r * ldy, (c * BLOCK + tid) * V, n, v[c], false);
        }
        if (r2 >= rows) return;
        r = r2;
    }
}

// Longer rows: a workgroup of 1024 per row, which keeps the first LONG_KEPT chunks a thread as they lie in memory; what a row has
// beyond them is read three times, the second and third time from the caches.
constexpr int LONG_KEPT = 8;

// A thread's sum over its chunks of such a row, chunks of a row of 2^24 fp32 elements being 4096: 64 of them at a time, so that no
// value is one of 2^14 in a row whose roundings may all go the same way (0.1 in each of 2^24 columns, in one row: a mean of 0.099985).
struct LongSum {
    float whole = 0.f, part = 0.f;
    int count = 0;
    __device__ __forceinline__ void operator+=(float chunk)
    {
        part += chunk;
        if (++count % 64 == 0) whole += part, part = 0.f;
    }
    __device__ __forceinline__ float total() const { return whole + part; }
};

template <typename T>
__global__ __launch_bounds__(1024) void layer_norm_forward_long_kernel(const T *x, int64_t ldx, int64_t rows, int n, float eps, const float *__restrict__ gamma,
                                                                       const float *__restrict__ beta, T *y, int64_t ldy, float *__restrict__ mean, float *__restrict__ rstd)
{
    constexpr int V = CHUNK<T>, STEP = 1024 * V;
    __shared__ float lds[2][1][16];
    const int64_t r = grid_row();
    if (r >= rows) return;
    const T *row = x + r * ldx;
    const int first = threadIdx.x * V;
    Raw<T> kept[LONG_KEPT];
    LongSum all, squares;
#pragma unroll
    for (int c = 0; c < LONG_KEPT; ++c) kept[c] = load_raw<CUT>(row, first + c * STEP, n);
    // f(v, at) for every chunk of the thread that begins inside the row, zero outside it
    auto each = [&](auto f) {
        float v[V];
#pragma unroll
        for (int c = 0; c < LONG_KEPT; ++c)
            if (first + c * STEP < n) {
                unpack(kept[c].w, v);
                f(v, first + c * STEP);
            }
        for (int at = first + LONG_KEPT * STEP; at < n; at += STEP) {
            load_chunk(row, at, n, v);
            f(v, at);
        }
    };
#pragma unroll
    for (int c = 0; c < LONG_KEPT; ++c) settle<CUT>(kept[c], first + c * STEP, n);
    each([&](float(&v)[V], int) {
        float q = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) q += v[j];
        all += q;
    });
    float sum[1] = {all.total()};
    team_join<1024>(sum, lds[0]);
    const float mu = sum[0] / (float)n;
    each([&](float(&v)[V], int at) {
        float q = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float d = at + j < n ? v[j] - mu : 0.f;
            q += d * d;
        }
        squares += q;
    });
    float sq[1] = {squares.total()};
    team_join<1024>(sq, lds[1]);
    const float rs = 1.0f / sqrtf(sq[0] / (float)n + eps);
    if (threadIdx.x == 0) {
        if (mean != nullptr) mean[r] = mu;
        if (rstd != nullptr) rstd[r] = rs;
    }
    each([&](float(&v)[V], int at) {
        float w[V];
        load_columns<CUT, V>(gamma, at, n, 1.f, w);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = (v[j] - mu) * rs * w[j];
        load_columns<CUT, V>(beta, at, n, 0.f, w);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] += w[j];
        store_chunk<CUT>(y + r * ldy, at, n, v, false);
    });
}

// ------------------------------------------------------------------------------------------------ backward
__device__ __forceinline__ bool on16(const void *p) { return ((uintptr_t)p & 15) == 0; }

template <typename T> struct NormBackward {
    const T *x, *dy;
    int64_t ldx, lddy, rows;
    int n;
    const float *gamma, *mean, *rstd;
    T *dx;
    int64_t lddx;
    float *dgamma, *dbeta, *part;  // part [ranges or workgroups][2][n], null: the sums go to dgamma and dbeta themselves
    int tiles, tile;               // tiles of columns, and their chunks
    int64_t range;                 // rows of a range
    bool past;                     // dx goes past the caches
};

// The weights' gradients of one tile of columns, TILE chunks across, over one range of rows by a workgroup of 1024: 1024 / TILE
// rows at a time, four of them a thread in flight.
template <int TILE, Fit FIT, typename T> __device__ __forceinline__ void norm_columns(const NormBackward<T> &a, int tile, int64_t which, float *lds)
{
    constexpr int V = CHUNK<T>, LANES = 1024 / TILE, ROWS = 4;
    const int col = threadIdx.x % TILE, lane = threadIdx.x / TILE, at = (tile * TILE + col) * V;
    const int64_t r1 = (which + 1) * a.range < a.rows ? (which + 1) * a.range : a.rows;
    float s[2 * V];
#pragma unroll
    for (int j = 0; j < 2 * V; ++j) s[j] = 0.f;
    for (int64_t r = which * a.range + lane; r < r1; r += ROWS * LANES) {
        Raw<T> x[ROWS], d[ROWS];
        float mu[ROWS], rs[ROWS];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int64_t k = r + i * LANES < r1 ? r + i * LANES : r;
            x[i] = load_raw<FIT>(a.x + k * a.ldx, at, a.n);
            d[i] = load_raw<FIT>(a.dy + k * a.lddy, at, a.n);
            mu[i] = a.mean[k];
            rs[i] = a.rstd[k];
        }
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            if (r + i * LANES >= r1) break;
            float xv[V], dv[V];
            settle<FIT>(x[i], at, a.n);
            settle<FIT>(d[i], at, a.n);
            unpack(x[i].w, xv);
            unpack(d[i].w, dv);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                s[j] += dv[j] * ((xv[j] - mu[i]) * rs[i]);
                s[V + j] += dv[j];
            }
        }
    }
    // the rows of a wavefront, then the 16 wavefronts: lds [16][2 V][TILE]
#pragma unroll
    for (int j = 0; j < 2 * V; ++j) s[j] = join_strided<TILE>(s[j], Add());
    if ((threadIdx.x & 63) < TILE)
#pragma unroll
        for (int j = 0; j < 2 * V; ++j) lds[((threadIdx.x / 64) * 2 * V + j) * TILE + col] = s[j];
    __syncthreads();
    if (threadIdx.x < 2 * V * TILE) {
        const int v = threadIdx.x / (V * TILE), c = threadIdx.x / V % TILE, j = threadIdx.x % V, to = (tile * TILE + c) * V + j;
        float r = 0.f;
        for (int w = 0; w < 16; ++w) r += lds[(w * 2 * V + v * V + j) * TILE + c];
        if (to < a.n) {
            if (a.part != nullptr) a.part[(which * 2 + v) * a.n + to] = r;
            else if (v == 0 && a.dgamma != nullptr) a.dgamma[to] = r;
            else if (v == 1 && a.dbeta != nullptr) a.dbeta[to] = r;
        }
    }
}

// Tiles of 8 chunks, 128 bytes of a row and so a cache line, where there are enough of them to occupy the chip, else of 4 (2048 x 4096
// fp32: 27 us with tiles of 8, 38 of 4; 2000 x 2000 bf16: 15.8 and 13.2): a compute unit has only so many lines under way.
constexpr int LN_TILE = 8, LN_NARROW = 4, LN_LDS = 16 * 2 * 8 * LN_TILE;
template <Fit FIT, typename T> __device__ __forceinline__ void norm_columns(const NormBackward<T> &a, int id, float *lds)
{
    const int tile = id % a.tiles, which = id / a.tiles;
    if (FIT == TINY || a.tile == LN_NARROW) norm_columns<LN_NARROW, FIT>(a, tile, which, lds);
    else norm_columns<LN_TILE, FIT>(a, tile, which, lds);
}

// TEAM threads per row, 1024 / TEAM rows at a time, x and dy in registers between the sums and the output.  The first
// tiles x ranges workgroups (`columns` of them, counted over a grid's x and y: 2^28 columns are 2^23 tiles of fp32) take the weights' gradients; the two kinds run beside each other, and what one
// reads the other finds in the caches.  With WEIGHTS there are none of that kind: a workgroup goes on to further rows, the next
// row's loads in flight, adds their part of the weights' gradients in registers and leaves its sums in `part`.
template <typename T, int TEAM, int CHUNKS, bool WEIGHTS, Fit FIT>
__global__ __launch_bounds__(1024, 4) void layer_norm_backward_kernel(NormBackward<T> a, int columns)
{
    constexpr int V = CHUNK<T>, TEAMS = 1024 / TEAM;
    __shared__ float lds[2][2][16];
    __shared__ float sums[WEIGHTS ? 1 : LN_LDS];
    const int64_t id = WEIGHTS ? blockIdx.x : grid_row() - columns, step = (int64_t)gridDim.x * TEAMS;
    if (!WEIGHTS && id < 0) {
        norm_columns<FIT>(a, (int)id + columns, sums);
        return;
    }
    if (!WEIGHTS && (a.dx == nullptr || id * TEAMS >= a.rows)) return;
    const int team = threadIdx.x / TEAM, lane = threadIdx.x % TEAM;
    const float inv_n = 1.0f / (float)a.n;
    float ga[CHUNKS][V], dg[CHUNKS][V], db[CHUNKS][V];
    // rows in flight: two in fp32 (8192 x 4096: 95 us with one, 80 with two), whose chunks are half as many values (16384 x 4096 bf16:
    // 82 us with one, 95 with two)
    constexpr int AHEAD = WEIGHTS && V == 4 && CHUNKS == 1 ? 2 : 1;
    Raw<T> nx[AHEAD][CHUNKS], nd[AHEAD][CHUNKS];
    float nmu[AHEAD], nrs[AHEAD];
    auto fetch = [&](int i, int64_t r) {
        if (r >= a.rows) {  // not loaded: zeros from settle, which has nothing to say of a TINY chunk
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
                if (FIT == TINY) nx[i][c] = nd[i][c] = {{0, 0, 0, 0}};
            return;
        }
        nmu[i] = a.mean[r];
        nrs[i] = a.rstd[r];
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            nx[i][c] = load_raw<FIT>(a.x + r * a.ldx, (c * TEAM + lane) * V, a.n);
            nd[i][c] = load_raw<FIT>(a.dy + r * a.lddy, (c * TEAM + lane) * V, a.n);
        }
    };
    int64_t r = id * TEAMS + team;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) fetch(i, r + i * step);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        if (WEIGHTS) load_columns<FIT, V>(a.gamma, (c * TEAM + lane) * V, a.n, 1.f, ga[c]);
#pragma unroll
        for (int j = 0; j < V; ++j) dg[c][j] = db[c][j] = 0.f;
    }
    for (int turn = 0;; turn ^= 1, r += step) {
        float xh[CHUNKS][V], d[CHUNKS][V], s[2] = {0.f, 0.f};
        const float mu = nmu[0], rs = nrs[0];
        const int n = r < a.rows ? a.n : 0;  // a row past the last one has no elements: zeros, which add nothing
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            settle<FIT>(nx[0][c], (c * TEAM + lane) * V, n);
            settle<FIT>(nd[0][c], (c * TEAM + lane) * V, n);
            unpack(nx[0][c].w, xh[c]);
            unpack(nd[0][c].w, d[c]);
#pragma unroll
            for (int j = 0; j < V; ++j) xh[c][j] = (c * TEAM + lane) * V + j < n ? (xh[c][j] - mu) * rs : 0.f;
        }
        const bool more = WEIGHTS && r - team + step < a.rows;  // (the same for the whole workgroup)
        if (more) {
#pragma unroll
            for (int i = 0; i + 1 < AHEAD; ++i) {
                nmu[i] = nmu[i + 1], nrs[i] = nrs[i + 1];
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) nx[i][c] = nx[i + 1][c], nd[i][c] = nd[i + 1][c];
            }
            fetch(AHEAD - 1, r + AHEAD * step);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            if (!WEIGHTS) load_columns<FIT, V>(a.gamma, (c * TEAM + lane) * V, a.n, 1.f, ga[c]);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (WEIGHTS) {
                    dg[c][j] += d[c][j] * xh[c][j];
                    db[c][j] += d[c][j];
                }
                d[c][j] *= ga[c][j];
                s[0] += d[c][j];
                s[1] += d[c][j] * xh[c][j];
            }
        }
        team_join<TEAM>(s, lds[turn]);
        const float mg = s[0] * inv_n, mgx = s[1] * inv_n;
        if (a.dx != nullptr && r < a.rows)
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
#pragma unroll
                for (int j = 0; j < V; ++j) d[c][j] = rs * (d[c][j] - mg - xh[c][j] * mgx);
                store_chunk<FIT>(a.dx + r * a.lddx, (c * TEAM + lane) * V, a.n, d[c], a.past && on16(a.dx + r * a.lddx));
            }
        if (!more) break;
    }
    if (!WEIGHTS || a.part == nullptr) return;
    // the teams' sums, a team after the other
    float *part = a.part + id * 2 * a.n;
    extern __shared__ float rows_lds[];  // [2][CHUNKS][V][TEAM]
    for (int t = TEAMS - 1; t > 0; --t) {
        __syncthreads();
        if (team == t)
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    rows_lds[(c * V + j) * TEAM + lane] = dg[c][j];
                    rows_lds[((CHUNKS + c) * V + j) * TEAM + lane] = db[c][j];
                }
        __syncthreads();
        if (team == 0)
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    dg[c][j] += rows_lds[(c * V + j) * TEAM + lane];
                    db[c][j] += rows_lds[((CHUNKS + c) * V + j) * TEAM + lane];
                }
    }
    if (team == 0)
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            store_floats<V>(part, (c * TEAM + lane) * V, a.n, dg[c]);
            store_floats<V>(part + a.n, (c * TEAM + lane) * V, a.n, db[c]);
        }
}

// Rows of more chunks than that: the first LONG_KEPT chunks a thread of x and dy are kept as they lie in memory, what is beyond
// them is read a second time from the caches.
template <typename T> __global__ __launch_bounds__(1024) void layer_norm_backward_long_kernel(NormBackward<T> a, int columns)
{
    constexpr int V = CHUNK<T>, STEP = 1024 * V, KEPT = LONG_KEPT / 2;
    __shared__ float lds[2][16];
    __shared__ float sums[LN_LDS];
    const int64_t r = grid_row() - columns;
    if (r < 0) {
        norm_columns<CUT>(a, (int)r + columns, sums);
        return;
    }
    if (a.dx == nullptr || r >= a.rows) return;
    const T *xr = a.x + r * a.ldx, *dr = a.dy + r * a.lddy;
    const float mu = a.mean[r], rs = a.rstd[r];
    const int first = threadIdx.x * V;
    Raw<T> kx[KEPT], kd[KEPT];
    LongSum gs, gxs;
#pragma unroll
    for (int c = 0; c < KEPT; ++c) {
        kx[c] = load_raw<CUT>(xr, first + c * STEP, a.n);
        kd[c] = load_raw<CUT>(dr, first + c * STEP, a.n);
    }
    // f(xh, g, at) for every chunk of the thread; g is zero outside the row
    auto each = [&](auto f) {
        float x[V], d[V], g[V];
        auto give = [&](int at) {
            load_columns<CUT, V>(a.gamma, at, a.n, 1.f, g);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                x[j] = at + j < a.n ? (x[j] - mu) * rs : 0.f;
                d[j] *= g[j];
            }
            f(x, d, at);
        };
#pragma unroll
        for (int c = 0; c < KEPT; ++c)
            if (first + c * STEP < a.n) {
                unpack(kx[c].w, x);
                unpack(kd[c].w, d);
                give(first + c * STEP);
            }
        for (int at = first + KEPT * STEP; at < a.n; at += STEP) {
            load_chunk(xr, at, a.n, x);
            load_chunk(dr, at, a.n, d);
            give(at);
        }
    };
#pragma unroll
    for (int c = 0; c < KEPT; ++c) {
        settle<CUT>(kx[c], first + c * STEP, a.n);
        settle<CUT>(kd[c], first + c * STEP, a.n);
    }
    each([&](float(&x)[V], float(&d)[V], int) {
        float q = 0.f, qx = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            q += d[j];
            qx += d[j] * x[j];
        }
        gs += q;
        gxs += qx;
    });
    float s[2] = {gs.total(), gxs.total()};
    team_join<1024>(s, lds);
    const float mg = s[0] / (float)a.n, mgx = s[1] / (float)a.n;
    each([&](float(&x)[V], float(&d)[V], int at) {
#pragma unroll
        for (int j = 0; j < V; ++j) d[j] = rs * (d[j] - mg - x[j] * mgx);
        store_chunk<CUT>(a.dx + r * a.lddx, at, a.n, d, a.past && on16(a.dx + r * a.lddx));
    });
}

// The sums of the parts, 64 columns by 16 parts at a time.
__global__ __launch_bounds__(1024) void layer_norm_join_kernel(const float *__restrict__ part, int parts, int n, float *__restrict__ dgamma, float *__restrict__ dbeta)
{
    __shared__ float lds[16][64];
    const int col = threadIdx.x % 64, lane = threadIdx.x / 64;
    const int64_t i = (int64_t)blockIdx.x * 64 + col;
    float s = 0.f;
    if (i < 2 * (int64_t)n)
#pragma unroll 8
        for (int k = lane; k < parts; k += 16) s += part[(int64_t)k * 2 * n + i];
    lds[lane][col] = s;
    __syncthreads();
    if (lane > 0 || i >= 2 * (int64_t)n) return;
    for (int l = 1; l < 16; ++l) s += lds[l][col];
    if (i < n) {
        if (dgamma != nullptr) dgamma[i] = s;
    } else if (dbeta != nullptr) {
        dbeta[i - n] = s;
    }
}

// ------------------------------------------------------------------------------------------------ host side
// How the weights' gradients are added.  fused: by the workgroups that take the rows, whose sums (8 bytes a column and workgroup,
// written and read once) are then less than x and dy read again; else beside them, by tiles of columns over ranges of rows.
// Rows of at most 8192 elements, 8 values a thread: with 16 the registers do not hold a row and both sums (4096 x 16384 bf16: 201 us
// fused, 133 beside; 4096 x 8192 fp32: 85 and 126).  More than 2048 of them (2048 x 4096 bf16: 19.5 and 19.7; 1024 x 4096: 17 and 11).
constexpr int64_t FUSED_MOST = 8192;
struct WeightsPlan { bool fused; int tile; int64_t parts, tiles; };

static WeightsPlan weights_plan(int dtype, int64_t rows, int64_t n)
{
    const int64_t v = 16 / (int64_t)elem_size(dtype), chunks = (n + v - 1) / v;
    WeightsPlan p = {false, chunks >= 128 * LN_TILE ? LN_TILE : LN_NARROW, 1, 0};
    p.tiles = (chunks + p.tile - 1) / p.tile;
    if (rows > 2048 && n <= FUSED_MOST) {
        p.fused = true;
        p.parts = 256;  // one workgroup per compute unit
        return p;
    }
    // about four workgroups per compute unit, 2048 rows each at least
    const int64_t most = rows / 2048, want = (1024 + p.tiles - 1) / p.tiles;
    p.parts = want < most ? want : most;
    if (p.parts < 1) p.parts = 1;
    return p;
}

size_t layer_norm_workspace(int dtype, int64_t rows, int64_t n)
{
    // what fewer rows need is never more: 256 parts where rows > 2048, else at most rows / 2048
    const WeightsPlan p = weights_plan(dtype, rows, n);
    return p.fused || p.parts > 1 ? (size_t)p.parts * 2 * n * sizeof(float) : 0;
}

template <typename T, int BLOCK, int CHUNKS>
static void launch_forward(const LayerNormArgs &a, float eps, const float *beta, T *y, int64_t ldy, float *mean, float *rstd, hipStream_t s)
{
    // workgroups that are resident at once: 24 wavefronts per compute unit
    const int64_t most = 256 * (24 / (BLOCK / 64)), groups = a.rows < most ? a.rows : most;
#define OMNI_LN_FORWARD(FIT)                                                                                                                                              \
    hipLaunchKernelGGL((layer_norm_forward_kernel<T, BLOCK, CHUNKS, FIT>), row_grid(groups), dim3(BLOCK), 0, s, (const T *)a.x, a.ldx, a.rows, (int)a.width, eps, a.gamma, beta, y, \
                       ldy, mean, rstd)
    if (a.width % CHUNK<T> == 0) OMNI_LN_FORWARD(WHOLE);
    else if (BLOCK > 64 || CHUNKS > 1 || a.width > CHUNK<T>) OMNI_LN_FORWARD(CUT);
    else OMNI_LN_FORWARD((BLOCK == 64 && CHUNKS == 1 ? TINY : CUT));
#undef OMNI_LN_FORWARD
}

template <typename T> static int forward(const LayerNormArgs &a, float eps, const float *beta, T *y, int64_t ldy, float *mean, float *rstd, hipStream_t s)
{
    const int64_t chunks = (a.width + CHUNK<T> - 1) / CHUNK<T>;
    if (chunks <= 64) launch_forward<T, 64, 1>(a, eps, beta, y, ldy, mean, rstd, s);
    else if (chunks <= 128) launch_forward<T, 64, 2>(a, eps, beta, y, ldy, mean, rstd, s);
    else if (chunks <= 256) launch_forward<T, 256, 1>(a, eps, beta, y, ldy, mean, rstd, s);
    else if (chunks <= 512) launch_forward<T, 256, 2>(a, eps, beta, y, ldy, mean, rstd, s);
    else if (chunks <= 1024) launch_forward<T, 512, 2>(a, eps, beta, y, ldy, mean, rstd, s);
    else if (chunks <= 2048) launch_forward<T, 1024, 2>(a, eps, beta, y, ldy, mean, rstd, s);
    else
        hipLaunchKernelGGL(layer_norm_forward_long_kernel<T>, row_grid(a.rows), dim3(1024), 0, s, (const T *)a.x, a.ldx, a.rows, (int)a.width, eps, a.gamma, beta, y, ldy, mean, rstd);
    OMNI_LAUNCH_CHECK();
    return OMNI_OK;
}

int launch_layer_norm_forward(const LayerNormArgs &a, float eps, const float *beta, void *y, int64_t ldy, float *mean, float *rstd, hipStream_t s)
{
    ProfScope prof(KID_LAYER_NORM, s, 0.0, 2.0 * (double)a.rows * a.width * elem_size(a.dtype));
    return a.dtype == OMNI_BF16 ? forward<bf16_t>(a, eps, beta, (bf16_t *)y, ldy, mean, rstd, s) : forward<float>(a, eps, beta, (float *)y, ldy, mean, rstd, s);
}

template <typename T, int TEAM, int CHUNKS> static void launch_backward(const NormBackward<T> &b, bool fused, int64_t columns, int64_t parts, bool dx, hipStream_t s)
{
    constexpr int64_t TEAMS = 1024 / TEAM;
    const int64_t groups = (b.rows + TEAMS - 1) / TEAMS;
    const size_t lds = TEAMS > 1 ? 2 * CHUNKS * CHUNK<T> * TEAM * sizeof(float) : 0;
    const Fit fit = b.n % CHUNK<T> == 0 ? WHOLE : TEAM == 64 && b.n < CHUNK<T> ? TINY : CUT;
    constexpr bool FUSES = TEAM * CHUNKS * CHUNK<T> <= FUSED_MOST;
#define OMNI_LN_BACKWARD(FIT)                                                                                                                                               \
    do {                                                                                                                                                                    \
        if (FUSES && fused) hipLaunchKernelGGL((layer_norm_backward_kernel<T, TEAM, CHUNKS, FUSES, FIT>), dim3((unsigned)parts), dim3(1024), lds, s, b, 0);                 \
        else hipLaunchKernelGGL((layer_norm_backward_kernel<T, TEAM, CHUNKS, false, FIT>), row_grid(columns + (dx ? groups : 0)), dim3(1024), 0, s, b, (int)columns);          \
    } while (0)
    if (fit == WHOLE) OMNI_LN_BACKWARD(WHOLE);
    else if (fit == CUT) OMNI_LN_BACKWARD(CUT);
    else OMNI_LN_BACKWARD((TEAM == 64 ? TINY : CUT));
#undef OMNI_LN_BACKWARD
}

template <typename T> static int backward_launch(const NormBackward<T> &b, bool fused, int64_t columns, int64_t parts, bool dx, hipStream_t s)
{
    const int64_t chunks = (b.n + CHUNK<T> - 1) / CHUNK<T>;
    if (chunks <= 64) launch_backward<T, 64, 1>(b, fused, columns, parts, dx, s);
    else if (chunks <= 128) launch_backward<T, 128, 1>(b, fused, columns, parts, dx, s);
    else if (chunks <= 256) launch_backward<T, 256, 1>(b, fused, columns, parts, dx, s);
    else if (chunks <= 512) launch_backward<T, 512, 1>(b, fused, columns, parts, dx, s);
    else if (chunks <= 1024) launch_backward<T, 1024, 1>(b, fused, columns, parts, dx, s);
    else if (chunks <= 2048) launch_backward<T, 1024, 2>(b, fused, columns, parts, dx, s);
    else hipLaunchKernelGGL(layer_norm_backward_long_kernel<T>, row_grid(columns + (dx ? b.rows : 0)), dim3(1024), 0, s, b, (int)columns);
    OMNI_LAUNCH_CHECK();
    return OMNI_OK;
}

template <typename T>
static int backward(const LayerNormArgs &a, const T *dy, int64_t lddy, const float *mean, const float *rstd, T *dx, int64_t lddx, float *dgamma, float *dbeta, float *part,
                    hipStream_t s)
{
    const bool weights = dgamma != nullptr || dbeta != nullptr;
    WeightsPlan p = weights_plan(a.dtype, a.rows, a.width);
    const int64_t range = p.fused ? a.rows : (a.rows + p.parts - 1) / p.parts, columns = p.tiles * p.parts;
    NormBackward<T> b = {(const T *)a.x, dy, a.ldx, lddy, a.rows, (int)a.width, a.gamma, mean, rstd, dx, lddx, dgamma, dbeta, p.parts > 1 ? part : nullptr, (int)p.tiles, p.tile, range, past_caches(a.dtype, a.rows, a.width)};
    int st;
    if (!weights) {  // (the resident workgroups are the faster ones for many rows, also without sums to leave)
        b.part = nullptr;
        if (dx == nullptr) return OMNI_OK;
        return backward_launch(b, p.fused, 0, p.parts, true, s);
    }
    if (p.fused) {
        if ((st = backward_launch(b, true, 0, p.parts, true, s)) != OMNI_OK) return st;
    } else if (dx != nullptr && ((const void *)dx == a.x || dx == dy)) {  // dx is written over what the sums are taken from: after them
        if ((st = backward_launch(b, false, columns, 0, false, s)) != OMNI_OK) return st;
        if ((st = backward_launch(b, false, 0, 0, true, s)) != OMNI_OK) return st;
    } else if ((st = backward_launch(b, false, columns, 0, dx != nullptr, s)) != OMNI_OK) {
        return st;
    }
    if (p.parts > 1) {
        hipLaunchKernelGGL(layer_norm_join_kernel, dim3((unsigned)((2 * a.width + 63) / 64)), dim3(1024), 0, s, part, (int)p.parts, (int)a.width, dgamma, dbeta);
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
