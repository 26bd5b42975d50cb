// Device helpers of the kernels that walk the rows of a matrix (layernorm.hip, logits.hip): a row of n elements is read in
// chunks of 16 bytes, a workgroup works on one row or on a piece of one, and its sums are joined in a fixed order.
#pragma once

#include "common.h"

namespace omni {

// elements of a 16-byte chunk
template <typename T> constexpr int CHUNK = 16 / (int)sizeof(T);

template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) ChunkBits { uint32_t w[4]; };  // of any element alignment

__device__ __forceinline__ void unpack(const uint32_t (&w)[4], float (&v)[8])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float(w[j] << 16);
        v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(const uint32_t (&w)[4], float (&v)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(w[j]);
}
__device__ __forceinline__ void pack(const float (&v)[8], uint32_t (&w)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = f32x2_to_bf16x2(v[2 * j], v[2 * j + 1]);
}
__device__ __forceinline__ void pack(const float (&v)[4], uint32_t (&w)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(v[j]);
}

__device__ __forceinline__ float element(const float *p) { return *p; }
__device__ __forceinline__ float element(const bf16_t *p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void set_element(float *p, float v) { *p = v; }
__device__ __forceinline__ void set_element(bf16_t *p, float v) { *p = f32_to_bf16(v); }

// 16 bytes moved down by `bytes` (up, if negative), zero behind them
__device__ __forceinline__ void shift_bytes(uint32_t (&w)[4], int bytes)
{
    uint64_t lo = w[0] | (uint64_t)w[1] << 32, hi = w[2] | (uint64_t)w[3] << 32;
    if (bytes > 0) {
        if (bytes >= 8) lo = hi, hi = 0;
        const int k = bytes % 8 * 8;
        if (k > 0) lo = lo >> k | hi << (64 - k), hi >>= k;
    } else if (bytes < 0) {
        if (bytes <= -8) hi = lo, lo = 0;
        const int k = -bytes % 8 * 8;
        if (k > 0) hi = hi << k | lo >> (64 - k), lo <<= k;
    }
    w[0] = (uint32_t)lo, w[1] = (uint32_t)(lo >> 32), w[2] = (uint32_t)hi, w[3] = (uint32_t)(hi >> 32);
}

// Elements [at, at + CHUNK) of a row of n as they lie in memory, zero outside the row, in two steps: load_raw starts the load,
// settle is called where the chunk is used.  A chunk that is partly outside is cut from the row's first or last 16 bytes, which
// are loaded whole: a load that needs a branch or its data at once keeps the loads around it from staying in flight (layer norm
// of 8192 x 5001 bf16, whose rows end inside a chunk, with the cut at the load: forward 57 us, backward 95).
// Nor may a kernel ask at each load whether the row holds a chunk at all (1023 x 1001 fp32: backward 10.8 us, 7.5 without).
// WHOLE: n is a multiple of the chunk, so a chunk is inside or outside; TINY: n is less than a chunk, which is loaded by elements.
enum Fit { WHOLE, CUT, TINY };
template <typename T> using Raw = ChunkBits<T>;
template <Fit FIT, typename T> __device__ __forceinline__ Raw<T> load_raw(const T *row, int at, int n)
{
    constexpr int V = CHUNK<T>;
    if (FIT != TINY) return *reinterpret_cast<const ChunkBits<T> *>(row + (at < 0 ? 0 : at < n - V ? at : n - V));
    Raw<T> b = {{0, 0, 0, 0}};
    float v[V];
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = at + j >= 0 && at + j < n ? element(row + at + j) : 0.f;
    pack(v, b.w);
    return b;
}
template <Fit FIT, typename T> __device__ __forceinline__ void settle(Raw<T> &b, int at, int n)
{
    constexpr int V = CHUNK<T>;
    if (FIT == TINY) return;
    if (FIT == WHOLE) {
#pragma unroll
        for (int j = 0; j < 4; ++j) b.w[j] = at < n ? b.w[j] : 0;
        return;
    }
    if (at >= 0 && at + V <= n) return;
    if (at >= n || at + V <= 0) b = {{0, 0, 0, 0}};
    else shift_bytes(b.w, (at < 0 ? at : at + V - n) * (int)sizeof(T));
}
// ... as floats, of a row of at least a chunk
template <typename T> __device__ __forceinline__ void load_chunk(const T *row, int at, int n, float (&v)[CHUNK<T>])
{
    Raw<T> b = load_raw<CUT>(row, at, n);
    settle<CUT>(b, at, n);
    unpack(b.w, v);
}
template <int V> __device__ __forceinline__ void store_floats(float *p, int at, int n, const float (&v)[V])
{
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (at + j < n) p[at + j] = v[j];
}
// past: the chunk lies on 16 bytes and goes past the caches.
template <typename T> __device__ __forceinline__ void store_whole(T *p, const float (&v)[CHUNK<T>], bool past)
{
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    ChunkBits<T> b;
    pack(v, b.w);
    if (past) __builtin_nontemporal_store(words{b.w[0], b.w[1], b.w[2], b.w[3]}, reinterpret_cast<words *>(p));
    else *reinterpret_cast<ChunkBits<T> *>(p) = b;
}
template <Fit FIT, typename T> __device__ __forceinline__ void store_chunk(T *row, int at, int n, const float (&v)[CHUNK<T>], bool past)
{
    if (FIT != TINY && at >= 0 && at + CHUNK<T> <= n) {
        store_whole(row + at, v, past);
    } else if (FIT != WHOLE) {
#pragma unroll
        for (int j = 0; j < CHUNK<T>; ++j)
            if (at + j >= 0 && at + j < n) set_element(row + at + j, v[j]);
    }
}

// Results of this many bytes, which with what they are computed from are more than the 256 MB of the last cache, are stored past the
// caches: gradients of 4096 x 65536 bf16 178 us instead of 184 (210 and 222 where the loss is computed, too), layer norm's dx of 16384 x
// 4096 bf16 64 instead of 71.  Not its y, which is the next thing read (16384 x 4096 bf16: 49 us past the caches, 44 into them).
inline bool past_caches(int dtype, int64_t rows, int64_t width) { return (double)rows * width * elem_size(dtype) >= 134217728.0; }

// ---------------------------------------------------------------- one workgroup per row
// Rows run over a grid's x and then its y: 2^20 workgroups of 1024 threads are what x takes.
constexpr int64_t ROW_GRID = 1 << 20;
inline dim3 row_grid(int64_t rows) { return dim3((unsigned)(rows < ROW_GRID ? rows : ROW_GRID), (unsigned)((rows + ROW_GRID - 1) / ROW_GRID)); }
__device__ __forceinline__ int64_t grid_row() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }  // the last may be past the rows

// ---------------------------------------------------------------- joins over a wavefront and a workgroup
// Lane i gets lane i ^ 1, i ^ 2, its mirror in 8 and in 16, then the other half of 32 and of 64: every lane ends with the
// same value, added in the same order.
template <int CTRL> __device__ __forceinline__ float dpp(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
template <typename OP> __device__ __forceinline__ float join16(float v, OP op)  // over 16 lanes
{
    v = op(v, dpp<0xb1>(v));   // quad_perm 1 0 3 2
    v = op(v, dpp<0x4e>(v));   // quad_perm 2 3 0 1
    v = op(v, dpp<0x141>(v));  // row_half_mirror
    return op(v, dpp<0x140>(v));  // row_mirror
}
template <typename OP> __device__ __forceinline__ float wave_join(float v, OP op)
{
    v = join16(v, op);
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
// over the lanes whose numbers are equal modulo STRIDE (2, 4 or 8)
template <int STRIDE, typename OP> __device__ __forceinline__ float join_strided(float v, OP op)
{
    if (STRIDE <= 2) v = op(v, dpp<0x4e>(v));   // quad_perm 2 3 0 1
    if (STRIDE <= 4) v = op(v, dpp<0x124>(v));  // row_ror 4
    v = op(v, dpp<0x128>(v));                   // row_ror 8
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
struct Add { __device__ __forceinline__ float operator()(float a, float b) const { return a + b; } };
struct MinBits { __device__ __forceinline__ float operator()(float a, float b) const { return __uint_as_float(min(__float_as_uint(a), __float_as_uint(b))); } };  // of whole numbers
struct Max { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };

// The workgroup's sum (or maximum) of N values a thread, to every thread.  `lds` holds N * BLOCK / 64 floats; the barrier in
// front lets it be used again at once.
template <int BLOCK, int N, typename OP> __device__ __forceinline__ void block_join(float (&v)[N], float *lds, OP op)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_join(v[i], op);
    if (BLOCK == 64) return;
    constexpr int WAVES = BLOCK / 64;
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) lds[i * WAVES + threadIdx.x / 64] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float r = lds[i * WAVES];
        for (int w = 1; w < WAVES; ++w) r = op(r, lds[i * WAVES + w]);
        v[i] = r;
    }
}

}  // namespace omni
