// What is read off a network's logits (gfx950): log probabilities of given classes with the entropy and the top
// alternatives, and the distillation loss, each with its gradient.
//   z = (x - m) / T, m = max x, s = sum e^z:  ln p_i = z_i - ln s,  H = ln s - sum z e^z / s
// A row is read once: every thread keeps a running maximum and the sums relative to it, and the threads' are joined.  z is
// formed as a difference first, so a row of the type's lowest values is a uniform one and not an empty one; a class of -inf
// has no probability and a row of nothing else none at all (m = -inf, s = 0).  A NaN or +inf makes the row's results NaN.
#include "row_ops.h"

// Products and sums are fused where fmaf says so and nowhere else: a row's sums are then the same bits in every variant of a
// kernel, whatever else it computes.
#pragma clang fp contract(off)

namespace omni {

// An exponent is one rounded product with log2 e, so a power e^z is off by about |z| 2^-24 (and 0 below 2^-126), its square and fourth
// power, taken for T = 1 beside T = 2 and 4, by twice and four times that.  That is 1 to 3 times 1e-7 of fp32 results, up to 3 times
// what an exponential with the low part of log2 e leaves (plain forms in torch: 0.6 to 1.3 times 1e-7), and nothing in bf16; the low
// part would be one more instruction an element, in loops of about ten that bound these kernels or come near it.
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
// z below which e^z is zero; -inf is raised to it where it is multiplied with e^z
constexpr float Z_LEAST = -16384.f;

__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }  // one instruction, 1 ulp; results below 2^-126 are zero

// ------------------------------------------------------------------------------------------------ a row's pieces
// 16-byte chunks that start where memory is aligned: chunk c covers elements [c * V - shift, c * V - shift + V).  Chunks lo to
// hi - 1 are whole; the elements outside them, at most 2 (V - 1), are taken one a thread.
template <typename T> struct RowSplit {
    int shift, lo, hi, head, edges;
    __device__ __forceinline__ RowSplit(const T *row, int n)
    {
        constexpr int V = CHUNK<T>;
        shift = (int)(((uintptr_t)row / sizeof(T)) % V);
        lo = shift > 0 ? 1 : 0;
        hi = (n + shift) / V;
        if (hi < lo) hi = lo;
        head = shift > 0 ? V - shift : 0;
        if (head > n) head = n;
        const int tail = n + shift - hi * V;
        edges = head + (tail > 0 && hi * V >= shift && head < n ? tail : 0);
    }
    __device__ __forceinline__ int edge(int i, int n) const { return i < head ? i : n - edges + i; }
    __device__ __forceinline__ int first(int c) const { return c * CHUNK<T> - shift; }
};

// A chunk of the row as it lies in memory.  NT: it is used once, so it goes past the caches (rows read straight through:
// 6.9 TB/s, 6.2 through the caches; 2^29 bytes in rows of 64 to 256 KB).
template <typename T, bool NT> __device__ __forceinline__ uint4 raw_chunk(const T *row, int at)
{
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    const words *p = reinterpret_cast<const words *>(row + at);
    const words w = NT ? __builtin_nontemporal_load(p) : *p;
    return make_uint4(w.x, w.y, w.z, w.w);
}
template <typename T> __device__ __forceinline__ void unpack(const uint4 &b, float *v)
{
    const uint32_t w[4] = {b.x, b.y, b.z, b.w};
    float u[CHUNK<T>];
    unpack(w, u);
#pragma unroll
    for (int j = 0; j < CHUNK<T>; ++j) v[j] = u[j];
}

// Values in the order of whole numbers (-0 counts as 0), with the index below: larger key = larger value, then lower index.
__device__ __forceinline__ uint32_t ordered(float v)
{
    const uint32_t b = __float_as_uint(v + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t k) { return __uint_as_float((int32_t)k < 0 ? k & 0x7fffffffu : ~k); }
constexpr uint32_t ORDERED_NOTHING = 0x007fffffu;  // ordered(-inf)

// ------------------------------------------------------------------------------------------------ running sums
// Powers of two throughout: e^z = 2^(c (x - m)), c = log2 e / T.  s = sum of them, and in t
enum Also {
    NOTHING,
    Z_TIMES,   // sum z e^z: the entropy's
    AT_ONE,    // the sum at T = 1, by a second exponential
    SQUARED,   // ... which at T = 2 is the first one's square
    SQUARED2,  // ... and at T = 4 its fourth power
};
// All are relative to the power h = m c as fp32 rounds it, so that an exponent is one fused product and sum, x c - h; finish()
// takes the rounding, m c - h < 2^-4, out of them.  Where m c is so large that its rounding is a power of its own (masks of the
// type's lowest value, m of +inf) they are relative to m c itself and the difference x - m is taken first.
struct Sums {
    float m, h, s, t;
    __device__ __forceinline__ float m0() const { return m == -INFINITY ? 0.f : m; }
    __device__ __forceinline__ bool far() const { return !(fabsf(h) < 1048576.f); }
    __device__ __forceinline__ float rounding(float c) const { return far() ? 0.f : fmaf(m0(), c, -h); }  // exact
};

template <int ALSO> __device__ __forceinline__ float at_one(float e, float d) { return ALSO == SQUARED ? e * e : ALSO == SQUARED2 ? (e * e) * (e * e) : exp2_fast(d * LOG2E); }

template <int ALSO> __device__ __forceinline__ void rescale(Sums &a, float m, float c)
{
    if (a.m == m) return;
    const Sums b = {m, m * c, a.s, a.t};
    if (a.m > -INFINITY) {  // (else there is nothing so far, or NaN, which stays)
        const float z = fmaf(a.m - m, c, b.rounding(c) - a.rounding(c)), f = exp2_fast(z);
        if (ALSO == Z_TIMES) a.t = f > 0.f ? (a.t + z * a.s) * f : 0.f;
        if (ALSO >= AT_ONE) a.t *= at_one<ALSO>(f, a.m - m);
        a.s *= f;
    }
    a.m = m;
    a.h = b.h;
}

// To sums relative to m itself.
template <int ALSO> __device__ __forceinline__ void finish(Sums &a, float c)
{
    const float z = -a.rounding(c), f = exp2_fast(z);
    if (ALSO == Z_TIMES) a.t = (a.t + z * a.s) * f;
    if (ALSO > AT_ONE) a.t *= at_one<ALSO>(f, 0.f);
    a.s *= f;
}

// Takes N elements in; returns their largest.
template <int ALSO, int N> __device__ __forceinline__ float absorb(Sums &a, const float (&x)[N], float c)
{
    float g = x[0];
#pragma unroll
    for (int j = 1; j < N; ++j) g = fmaxf(g, x[j]);
    if (g > a.m) rescale<ALSO>(a, g, c);
    if (__any(a.far())) {  // the difference first
        const float m = a.m0(), r = a.rounding(c);
        for (int j = 0; j < N; ++j) {
            const float d = x[j] - m, z = fmaf(d, c, r), e = exp2_fast(z);
            a.s += e;
            if (ALSO == Z_TIMES) a.t += fmaxf(z, Z_LEAST) * e;
            if (ALSO >= AT_ONE) a.t += at_one<ALSO>(e, d);
        }
        return g;
    }
    // two chains of sums
    float s1 = 0.f, t1 = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const float z = fmaf(x[j], c, -a.h), e = exp2_fast(z);
        (j % 2 ? s1 : a.s) += e;
        float &t = j % 2 ? t1 : a.t;
        if (ALSO == Z_TIMES) t = fmaf(fmaxf(z, Z_LEAST), e, t);
        if (ALSO == AT_ONE) t += exp2_fast((x[j] - a.m0()) * LOG2E);
        if (ALSO == SQUARED) t = fmaf(e, e, t);
        if (ALSO == SQUARED2) t = fmaf(e * e, e * e, t);
    }
    a.s += s1;
    a.t += t1;
    return g;
}

template <int ALSO, int BLOCK> __device__ __forceinline__ void join(Sums &a, float c, float *lds)
{
    float m[1] = {a.m}, v[2];
    block_join<BLOCK>(m, lds, Max());
    rescale<ALSO>(a, m[0], c);
    v[0] = a.s, v[1] = a.t;
    block_join<BLOCK>(v, lds, Add());
    a.s = v[0], a.t = v[1];
    finish<ALSO>(a, c);
}

constexpr int PAIR = 2, BATCH = 4;  // chunks whose sums are taken together; chunks a thread has in flight

// The largest of every thread's elements by slots of a few batches, in halves of ordered() keys: which chunks of a row can hold
// one of its largest elements.  Batches of slot i are i << shift and so on.
constexpr int SLOTS = 16;
template <int BLOCK> struct Slots {
    uint16_t most[SLOTS][BLOCK];
};

// The sums over a row; the thread's own maximum (for the top alternatives) goes to *own.  KEPT chunks a thread, the first ones,
// are loaded at once and stay in `kept`; the others follow in batches, the next batch in flight while one is summed.  The slots'
// maxima go to `slots` (null: they are not wanted).
template <typename T, int BLOCK, int ALSO, bool NT, int KEPT>
__device__ __forceinline__ Sums row_sums(const T *row, int n, const RowSplit<T> &sp, float c, float *own, float *lds, uint4 (&kept)[KEPT > 0 ? KEPT : 1],
                                         Slots<BLOCK> *slots = nullptr, int shift = 0)
{
    constexpr int V = CHUNK<T>;
    static_assert(KEPT % BATCH == 0 && BATCH % PAIR == 0, "whole batches of whole pairs");
    Sums a = {-INFINITY, 0.f, 0.f, 0.f};  // (no maximum yet: h = 0)
    const int tid = threadIdx.x, last = sp.hi - 1;
    auto take = [&](const uint4 *b, int at, bool whole) {  // two chunks; those past the last one, which repeat it, count as -inf
        float x[PAIR * V];
#pragma unroll
        for (int u = 0; u < PAIR; ++u) {
            unpack<T>(b[u], x + u * V);
            if (!whole)
#pragma unroll
                for (int j = 0; j < V; ++j) x[u * V + j] = at + u * BLOCK <= last ? x[u * V + j] : -INFINITY;
        }
        return absorb<ALSO>(a, x, c);
    };
    auto load = [&](uint4 &b, int at) { b = raw_chunk<T, NT>(row, sp.first(at < last ? at : last)); };
    int at = sp.lo + tid, first = sp.lo, batch = 0;
    float most = -INFINITY;
    auto take_batch = [&](const uint4 *b) {
        if ((batch & ((1 << shift) - 1)) == 0) most = -INFINITY;
#pragma unroll
        for (int u = 0; u < BATCH; u += PAIR)
            if (first + u * BLOCK < sp.hi) most = fmaxf(most, take(b + u, at + u * BLOCK, first + (u + PAIR) * BLOCK <= sp.hi));
        if (slots != nullptr) slots->most[batch >> shift][tid] = (uint16_t)(ordered(most) >> 16);
    };
    if (KEPT > 0 && sp.lo < sp.hi) {
#pragma unroll
        for (int u = 0; u < KEPT; ++u) load(kept[u], at + u * BLOCK);
#pragma unroll
        for (int u = 0; u < KEPT; u += BATCH) {
            if (first < sp.hi) take_batch(kept + u);
            at += BATCH * BLOCK;
            first += BATCH * BLOCK;
            ++batch;
        }
    }
    if (first < sp.hi) {
        uint4 b[BATCH], next[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u) load(b[u], at + u * BLOCK);
        for (;; ++batch) {
            const bool more = first + BATCH * BLOCK < sp.hi;
            if (more)
#pragma unroll
                for (int u = 0; u < BATCH; ++u) load(next[u], at + (BATCH + u) * BLOCK);
            take_batch(b);
            if (!more) break;
#pragma unroll
            for (int u = 0; u < BATCH; ++u) b[u] = next[u];
            at += BATCH * BLOCK;
            first += BATCH * BLOCK;
        }
    }
    if (tid < sp.edges) {
        const float x[1] = {element(row + sp.edge(tid, n))};
        absorb<ALSO>(a, x, c);
    }
    if (own != nullptr) *own = a.m;
    join<ALSO, BLOCK>(a, c, lds);
    return a;
}

// ------------------------------------------------------------------------------------------------ top alternatives
constexpr int TOP_KEYS = 512, TOP_LIST = 256;

template <int BLOCK> struct TopLds {
    uint64_t keys[TOP_KEYS];
    uint64_t bar;
    alignas(16) uint32_t group[BLOCK];
    int count, listed;
    uint16_t list[TOP_LIST];  // slot * BLOCK + thread
};

// The k largest of a row, k <= 64, in order, by a workgroup of 64 or 256.  The k-th largest of the threads' maxima (of single
// chunks', by one wavefront for k > 16) is a lower bound of the k-th largest element; the elements that reach it are collected, few more
// than k, and ranked by comparing each with all.  A row that the threads keep (KEPT > 0) is looked through where it lies; of others
// only the slots whose maximum reaches the bound are read again, their chunks spread over the workgroup (every chunk of the
// threads that reach it instead: 149 us for 32 of 2048 x 131072 bf16, where the sums alone take 85: the chunks of one thread lie
// in as many cache lines, and half of the row came a second time).  When more elements reach the bound than there is room for
// (equal values), the k-th largest of those collected is a higher bound, and the collection is done again: every key is
// different, so this ends.  Rows of equal values, or with fewer than k above a mask of the type's lowest value, are the slow ones: 5 of
// 2048 x 131072 bf16 374 us instead of 110, of 256 x 1000 fp32 60 instead of 6, as every element counts up one word in LDS.
template <typename T, int BLOCK, int KEPT, typename PUT>
__device__ __forceinline__ void row_top(const T *row, int n, const RowSplit<T> &sp, float own, int k, TopLds<BLOCK> &t, uint4 (&kept)[KEPT > 0 ? KEPT : 1],
                                        const Slots<BLOCK> *slots, int shift, PUT put)
{
    static_assert(BLOCK == 256 || (BLOCK == 64 && KEPT > 0), "groups of a lane");
    constexpr int V = CHUNK<T>, EACH = BLOCK == 64 ? KEPT : 4;  // groups of a lane
    const int tid = threadIdx.x, lane = tid & 63, rest = KEPT > 0 ? sp.hi : sp.lo;
    // The kept chunks are unpacked again where they are looked through, and their indexes taken again: held since the sums, or over the
    // repetitions, they are 166 registers instead of 94 (5 of 4096 x 4096 bf16: 22 us, 13.5 so; of 16384 x 1000: 31 and 21).
    auto as_they_lie = [&]() {
        if (KEPT > 0)
#pragma unroll
            for (int i = 0; i < KEPT; ++i) asm volatile("" : "+v"(kept[i].x), "+v"(kept[i].y), "+v"(kept[i].z), "+v"(kept[i].w));
    };
    uint32_t bound = 0;
    if (tid == 0) t.listed = 0;
    as_they_lie();
    // 16 or fewer: 64 groups bound as well, and every lane counts the maxima above its own.  More: the bound by its bits, from the
    // highest (counting over 256 groups: 32 of 2047 x 50021 bf16 53 us, by bits 47).
    if (k <= 16) {
        float g = own;
        if (BLOCK == 256) {
            g = fmaxf(g, dpp<0xb1>(g));
            g = fmaxf(g, dpp<0x4e>(g));
        }
        if (tid % (BLOCK / 64) == 0) t.group[tid / (BLOCK / 64)] = ordered(g);
        __syncthreads();
        const uint32_t mine = t.group[lane];
        int above = 0;
#pragma unroll
        for (int i = 0; i < 64; i += 4) {
            const uint4 o = *reinterpret_cast<const uint4 *>(t.group + i);
            above += (o.x > mine) + (o.y > mine) + (o.z > mine) + (o.w > mine);
        }
        bound = __float_as_uint(wave_join(__uint_as_float(above < k ? mine : ~0u), MinBits()));
    } else {
        uint32_t u[EACH];
        if constexpr (BLOCK == 64) {  // every chunk is a group
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                float x[V], g = i == 0 && tid < sp.edges ? element(row + sp.edge(tid, n)) : -INFINITY;
                unpack<T>(kept[i], x);
#pragma unroll
                for (int j = 0; j < V; ++j) g = sp.lo + tid + i * 64 < sp.hi ? fmaxf(g, x[j]) : g;
                u[i] = ordered(fmaxf(g, -INFINITY));
            }
        } else {  // every thread is
            t.group[tid] = ordered(own);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < EACH; ++i) u[i] = t.group[i * 64 + lane];
        }
        for (int bit = 31; bit >= (V == 8 ? 16 : 0); --bit) {  // (the lower half of a bf16 value's key says nothing)
            const uint32_t more = bound | (1u << bit);
            int reach = 0;
#pragma unroll
            for (int i = 0; i < EACH; ++i) reach += __popcll(__ballot(u[i] >= more));
            if (reach >= k) bound = more;
            if (reach == k) break;
        }
    }
    if (bound <= ORDERED_NOTHING) bound = ORDERED_NOTHING + 1;  // -inf is nobody's alternative
    const bool able = ordered(own) >= bound;
    // slots that reach the bound; past the list's room, every chunk is looked through
    const int batches = rest < sp.hi ? (sp.hi - rest + BATCH * BLOCK - 1) / (BATCH * BLOCK) : 0;
    if (able)
        for (int i = 0; i << shift < batches; ++i)
            if (slots->most[i][tid] >= bound >> 16) {
                const int to = atomicAdd(&t.listed, 1);
                if (to < TOP_LIST) t.list[to] = (uint16_t)(i * BLOCK + tid);
            }
    uint64_t bar = (uint64_t)bound << 32;
    int found;
    for (;;) {
        __syncthreads();
        if (tid == 0) t.count = 0;
        __syncthreads();
        as_they_lie();
        int at = sp.lo + tid;
        asm volatile("" : "+v"(at));
        const float least = unordered((uint32_t)(bar >> 32));
        auto offer = [&](float x, int i) {
            if (!(x >= least)) return;
            const uint64_t key = ((uint64_t)ordered(x) << 32) | (uint32_t)~i;
            if (key < bar) return;
            const int to = atomicAdd(&t.count, 1);
            if (to < TOP_KEYS) t.keys[to] = key;
        };
        auto offer_chunk = [&](const uint4 &b, int c) {
            float x[V];
            unpack<T>(b, x);
            float most = x[0];
#pragma unroll
            for (int j = 1; j < V; ++j) most = fmaxf(most, x[j]);
            if (!(most >= least)) return;
#pragma unroll
            for (int j = 0; j < V; ++j) offer(x[j], sp.first(c) + j);
        };
        if (able) {
#pragma unroll
            for (int i = 0; i < KEPT; ++i)
                if (at + i * BLOCK < sp.hi) offer_chunk(kept[i], at + i * BLOCK);
            if (tid < sp.edges) offer(element(row + sp.edge(tid, n)), sp.edge(tid, n));
        }
        const int listed = KEPT > 0 ? 0 : t.listed;
        if (listed <= TOP_LIST) {
            const int each = 2 + shift;  // chunks of a slot: BATCH << shift
            for (int i = tid; i < listed << each; i += BLOCK) {
                const int e = t.list[i >> each], q = i & ((1 << each) - 1), c = rest + e % BLOCK + ((e / BLOCK << each) + q) * BLOCK;
                if (c < sp.hi) offer_chunk(raw_chunk<T, false>(row, sp.first(c)), c);
            }
        } else {
            for (int c = rest + tid; c < sp.hi; c += BLOCK) offer_chunk(raw_chunk<T, false>(row, sp.first(c)), c);
        }
        __syncthreads();
        found = t.count;
        if (found <= TOP_KEYS) break;
        for (int i = tid; i < TOP_KEYS; i += BLOCK) {
            int above = 0;
#pragma unroll 8
            for (int j = 0; j < TOP_KEYS; ++j) above += t.keys[j] > t.keys[i];
            if (above == k - 1) t.bar = t.keys[i];
        }
        __syncthreads();
        bar = t.bar;
    }
    for (int i = tid; i < found; i += BLOCK) {
        const uint64_t key = t.keys[i];
        int above = 0;
#pragma unroll 8
        for (int j = 0; j < found; ++j) above += t.keys[j] > key;
        if (above < k) put(above, key);
    }
    for (int i = found + tid; i < k; i += BLOCK) put(i, 0);
}

// An alternative's place in the outputs; a key of 0 is none.
struct TopOut {
    int64_t *index;
    float *lp, m, inv_t, lns;
    __device__ __forceinline__ void operator()(int i, uint64_t key) const
    {
        index[i] = key == 0 ? -1 : (int64_t)(uint32_t)~(uint32_t)key;
        lp[i] = key == 0 ? -INFINITY : (unordered((uint32_t)(key >> 32)) - m) * inv_t - lns;
    }
};

// ------------------------------------------------------------------------------------------------ few long rows
// Where there are fewer rows than the chip has room for, a long row is cut into PARTS_MOST parts (fewer, if they would be shorter
// than PART_LEAST chunks), each a row of its own to one workgroup: one compute unit takes 28 GB/s from memory (a row of 131072
// bf16: 9 us).  The next launch joins the parts' sums, in their order, and their largest elements.  Sums alone gain up to 512 rows
// (loss of 400 x 131072 bf16: 22 us in parts, 29 whole; 511: 27 and 31).  Largest elements are looked for once a part, so fewer rows
// gain, the fewer the shorter they are (5 of 160 x 131072 bf16: 21 and 28, of 400: 38 and 35; of 48 x 50021: 13 and 15, of 256: 19 and 16).
// Loss and gradient read a whole row once and its parts twice (48 x 131072 bf16: 16 and 24; 160: 30 and 28).
constexpr int PART_LEAST = 1024, PARTS_MOST = 64, SPLIT_CHUNKS = 4096;
struct Parts { int count; int64_t length; };  // elements of a part, a multiple of 64; count = 1: the rows are not split
enum Wanted { SUMS, TOPS, BOTH };

// rows from which on they are not split
static int64_t split_rows(int64_t chunks, Wanted w)
{
    if (chunks <= SPLIT_CHUNKS) return 0;
    return w == SUMS ? 512 : w == BOTH ? 96 : chunks / 64 < 384 ? chunks / 64 : 384;
}

static Parts row_parts(int dtype, int64_t rows, int64_t classes, Wanted w)
{
    const int64_t v = 16 / (int64_t)elem_size(dtype);
    if (rows >= split_rows(classes / v, w)) return {1, classes};
    int64_t length = round_up((classes + PARTS_MOST - 1) / PARTS_MOST, 64);
    if (length < PART_LEAST * v) length = PART_LEAST * v;
    return {(int)((classes + length - 1) / length), length};
}

// bytes of the parts' sums, and of their keys behind them
static size_t parts_bytes(int dtype, int64_t rows, int64_t classes, int top)
{
    const Wanted w = top > 0 ? TOPS : SUMS;
    const int64_t from = split_rows(classes / (16 / (int64_t)elem_size(dtype)), w), most = rows < from ? rows : from - 1;  // a workspace for more rows serves fewer
    return from > 0 ? (size_t)most * row_parts(dtype, 0, classes, w).count * (sizeof(float4) + (size_t)top * sizeof(uint64_t)) : 0;
}
size_t logprob_workspace(int dtype, int64_t rows, int64_t classes, int top) { return parts_bytes(dtype, rows, classes, top); }
size_t distill_workspace(int dtype, int64_t rows, int64_t classes) { return parts_bytes(dtype, rows, classes, 0); }

template <typename T, int KEPT, int ALSO, bool TOP>
__global__ __launch_bounds__(256) void row_parts_kernel(const T *__restrict__ logits, int64_t ld, int64_t rows, int n, int parts, int64_t length, float c, int shift, int top,
                                                        float4 *__restrict__ sums, uint64_t *__restrict__ keys)
{
    constexpr int BLOCK = 256;
    __shared__ float lds[2 * (BLOCK / 64)];
    __shared__ TopLds<BLOCK> tl;
    __shared__ Slots<TOP && KEPT == 0 ? BLOCK : 1> sl;
    Slots<BLOCK> *slots = TOP && KEPT == 0 ? reinterpret_cast<Slots<BLOCK> *>(&sl) : nullptr;
    const int64_t id = grid_row(), r = id / parts, p = id % parts, begin = p * length;
    if (r >= rows) return;
    const T *row = logits + r * ld + begin;
    const int mine = (int)(begin + length < n ? length : n - begin);
    const RowSplit<T> sp(row, mine);
    float own;
    uint4 kept[KEPT > 0 ? KEPT : 1];
    const Sums a = row_sums<T, BLOCK, ALSO, true, KEPT>(row, mine, sp, c, &own, lds, kept, slots, shift);
    if (threadIdx.x == 0) sums[id] = make_float4(a.m, a.s, a.t, 0.f);
    if (TOP)
        row_top<T, BLOCK, KEPT>(row, mine, sp, own, top, tl, kept, slots, shift,
                              [&](int i, uint64_t key) { keys[id * top + i] = key == 0 ? 0 : key - (uint64_t)begin; });  // (the index is stored inverted)
}

// The sums of a row from its parts', the same in every wavefront.
template <int ALSO> __device__ __forceinline__ Sums join_parts(const float4 *sums, int parts, float c)
{
    const int lane = threadIdx.x & 63;
    const float4 p = lane < parts ? sums[lane] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
    Sums a = {p.x, 0.f, p.y, p.z};
    const float m = wave_join(a.m, Max());
    // (relative to the maxima themselves)
    if (a.m != m && a.m > -INFINITY) {
        const float d = a.m - m, z = d * c, f = exp2_fast(z);
        if (ALSO == Z_TIMES) a.t = f > 0.f ? (a.t + z * a.s) * f : 0.f;
        if (ALSO >= AT_ONE) a.t *= at_one<ALSO>(f, d);
        a.s *= f;
    }
    a.m = m;
    a.s = wave_join(a.s, Add());
    a.t = wave_join(a.t, Add());
    return a;
}

// The k largest of the parts' k largest by a workgroup of 256, as in row_top: the k-th largest of the threads' maxima is the bound,
// here of whole keys, so that few more than k reach it whatever is equal; by counting (20 of 48 x 131072 bf16: 15.4 us, 17.4 by bits).
// found [parts * k].
template <typename PUT> __device__ __forceinline__ void join_tops(const uint64_t *keys, int total, int k, uint64_t *found, PUT put)
{
    __shared__ alignas(16) uint64_t group[256];
    __shared__ uint64_t kth;
    __shared__ int count;
    const int tid = threadIdx.x;
    uint64_t own = 0;
    for (int i = tid; i < total; i += 256) own = keys[i] > own ? keys[i] : own;
    group[tid] = own;
    if (tid == 0) count = 0, kth = 0;
    __syncthreads();
    // (every key but 0 is different: the one with k - 1 above it is the k-th)
    int over = 0;
#pragma unroll 16
    for (int i = 0; i < 256; i += 2) {
        const ulonglong2 o = *reinterpret_cast<const ulonglong2 *>(group + i);
        over += (o.x > own) + (o.y > own);
    }
    if (over == k - 1) kth = own;
    __syncthreads();
    uint64_t bound = kth;
    if (bound == 0) bound = 1;  // (a key of 0 is none)
    if (own >= bound)
        for (int i = tid; i < total; i += 256)
            if (keys[i] >= bound) found[atomicAdd(&count, 1)] = keys[i];
    __syncthreads();
    const int n = count;
    for (int i = tid; i < n; i += 256) {
        int above = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) above += found[j] > found[i];
        if (above < k) put(above, found[i]);
    }
    for (int i = n + tid; i < k; i += 256) put(i, 0);
}

// ------------------------------------------------------------------------------------------------ log probabilities
struct LogprobOut {
    const int64_t *targets;
    int given;
    float *logprob, *entropy;
    int top;
    int64_t *top_index;
    float *top_logprob, *stats;
};

// What is written of a row apart from its alternatives; returns ln s.
template <typename T, int BLOCK, bool ENTROPY> __device__ __forceinline__ float write_logprobs(const LogprobOut &o, const T *row, int64_t r, int n, const Sums &a, float inv_t)
{
    const bool none = a.m == -INFINITY && a.s == 0.f;
    const float lns = logf(a.s);
    if (threadIdx.x == 0) {
        if (ENTROPY) o.entropy[r] = none ? 0.f : lns - LN2 * a.t / a.s;
        if (o.stats != nullptr) o.stats[2 * r] = a.m, o.stats[2 * r + 1] = a.s;
    }
    for (int i = threadIdx.x; i < o.given; i += BLOCK) {
        const int64_t at = o.targets[r * o.given + i];
        float v = at < 0 ? 0.f : NAN;
        if (at >= 0 && at < n) v = none ? -INFINITY : (element(row + at) - a.m) * inv_t - lns;
        o.logprob[r * o.given + i] = v;
    }
    return lns;
}

template <typename T, int BLOCK, int KEPT, bool ENTROPY>
__global__ __launch_bounds__(BLOCK) void logprob_forward_kernel(const T *__restrict__ logits, int64_t ld, int64_t rows, int n, float c, float inv_t, int shift, LogprobOut o)
{
    __shared__ float lds[2 * (BLOCK / 64)];
    __shared__ TopLds<BLOCK> tl;
    __shared__ Slots<(KEPT > 0) ? 1 : BLOCK> sl;  // rows that are kept whole need none
    Slots<BLOCK> *slots = KEPT > 0 || o.top == 0 ? nullptr : reinterpret_cast<Slots<BLOCK> *>(&sl);
    const int64_t r = grid_row();
    if (r >= rows) return;
    const T *row = logits + r * ld;
    const RowSplit<T> sp(row, n);
    float own;
    uint4 kept[KEPT > 0 ? KEPT : 1];
    const Sums a = row_sums<T, BLOCK, ENTROPY ? Z_TIMES : NOTHING, true, KEPT>(row, n, sp, c, &own, lds, kept, slots, shift);
    const float lns = write_logprobs<T, BLOCK, ENTROPY>(o, row, r, n, a, inv_t);
    if (o.top > 0) row_top<T, BLOCK, KEPT>(row, n, sp, own, o.top, tl, kept, slots, shift, TopOut{o.top_index + r * o.top, o.top_logprob + r * o.top, a.m, inv_t, lns});
}

template <typename T, bool ENTROPY>
__global__ __launch_bounds__(256) void logprob_join_kernel(const T *__restrict__ logits, int64_t ld, int n, int parts, float c, float inv_t, const float4 *__restrict__ sums,
                                                           const uint64_t *__restrict__ keys, LogprobOut o)
{
    extern __shared__ uint64_t tops[];
    const int64_t r = blockIdx.x;
    const Sums a = join_parts<ENTROPY ? Z_TIMES : NOTHING>(sums + r * parts, parts, c);
    const float lns = write_logprobs<T, 256, ENTROPY>(o, logits + r * ld, r, n, a, inv_t);
    if (o.top > 0) join_tops(keys + r * parts * o.top, parts * o.top, o.top, tops, TopOut{o.top_index + r * o.top, o.top_logprob + r * o.top, a.m, inv_t, lns});
}

// ------------------------------------------------------------------------------------------------ gradients
// A row's gradient is a function of the element and the row's sums everywhere but at a few listed classes, where something is
// added.  `value` gives the first; the listed classes are written last, each with all that is added to it in one rounding, by
// the first entry of the list that names it: every entry looks through the list, four at a time (16384 x 1000 bf16 with 32 entries:
// 23.5 us one at a time, 19.9 so; 1 x 1000 fp32, loss and gradient: 6.5 and 5.1).  out may be the logits themselves.
template <int MOST> struct ListLds {
    alignas(16) int at[(MOST + 3) / 4 * 4];  // -1: not in the row
    alignas(16) float add[(MOST + 3) / 4 * 4];
    __device__ __forceinline__ void close(int count)  // fills the last four up; a barrier comes before the list is read by fours
    {
        if ((int)threadIdx.x < (-count & 3)) at[count + threadIdx.x] = -1;
    }
};

// Chunks [c0, c1) of a row, aligned as the output's row is, AHEAD of them loaded before the first is used; `also` may change a
// chunk's values before they are rounded.
template <Fit FIT, typename T, int BLOCK, int AHEAD, typename F, typename G>
__device__ __forceinline__ void write_chunks(const T *in, T *out, int n, int shift, int64_t c0, int64_t c1, bool past, F value, G also)
{
    constexpr int V = CHUNK<T>;
    for (int64_t c = c0 + threadIdx.x; c < c1; c += AHEAD * BLOCK) {
        Raw<T> b[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) b[u] = load_raw<FIT>(in, (int)((c + u * BLOCK < c1 ? c + u * BLOCK : c) * V) - shift, n);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (c + u * BLOCK >= c1) break;
            const int at = (int)((c + u * BLOCK) * V) - shift;
            float x[V];
            settle<FIT>(b[u], at, n);
            unpack(b[u].w, x);
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = value(x[j]);
            also(at, x);
            store_chunk<FIT>(out, at, n, x, past);
        }
    }
}
template <typename T, int BLOCK, int AHEAD, typename F, typename G> __device__ __forceinline__ void write_row(const T *in, T *out, int n, int64_t c0, int64_t c1, bool past, F value, G also)
{
    constexpr int V = CHUNK<T>;
    const int shift = (int)(((uintptr_t)out / sizeof(T)) % V);
    if (c1 > (n + shift + V - 1) / V) c1 = (n + shift + V - 1) / V;
    if (n >= V) write_chunks<CUT, T, BLOCK, AHEAD>(in, out, n, shift, c0, c1, past, value, also);
    else write_chunks<TINY, T, BLOCK, 1>(in, out, n, shift, c0, c1, past, value, also);
}

// The listed classes in the elements that a call of write_row with the same chunks covers: their logits (before), their values
// (after, with a barrier between).
template <typename T, int BLOCK, int MOST> struct ListedOut {
    static constexpr int EACH = (MOST + BLOCK - 1) / BLOCK;
    float x[EACH];
    int from, to;
    __device__ __forceinline__ void read(const T *in, const T *out, int n, int64_t c0, int64_t c1, const ListLds<MOST> &l, int count)
    {
        constexpr int V = CHUNK<T>;
        const int shift = (int)(((uintptr_t)out / sizeof(T)) % V);
        from = c0 == 0 ? 0 : (int)(c0 * V) - shift;
        to = c1 * V - shift < n ? (int)(c1 * V) - shift : n;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int i = threadIdx.x + e * BLOCK;
            if (i < count && l.at[i] >= from && l.at[i] < to) x[e] = element(in + l.at[i]);
        }
    }
    __device__ __forceinline__ void read(const T *in, int n, const ListLds<MOST> &l, int count)  // of the whole row
    {
        from = 0, to = n;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int i = threadIdx.x + e * BLOCK;
            if (i < count && l.at[i] >= 0) x[e] = element(in + l.at[i]);
        }
    }
    template <typename F> __device__ __forceinline__ void write(T *out, const ListLds<MOST> &l, int count, F value)
    {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int i = threadIdx.x + e * BLOCK;
            if (i >= count || l.at[i] < from || l.at[i] >= to) continue;
            const int mine = l.at[i];
            bool first = true;
            float add = 0.f;
            for (int j = 0; j < count; j += 4) {
                const int4 at = *reinterpret_cast<const int4 *>(l.at + j);
                const float4 a = *reinterpret_cast<const float4 *>(l.add + j);
                first &= (at.x != mine || j >= i) & (at.y != mine || j + 1 >= i) & (at.z != mine || j + 2 >= i) & (at.w != mine || j + 3 >= i);
                add += at.x == mine ? a.x : 0.f;
                add += at.y == mine ? a.y : 0.f;
                add += at.z == mine ? a.z : 0.f;
                add += at.w == mine ? a.w : 0.f;
            }
            if (first) set_element(out + l.at[i], value(x[e]) + add);
        }
    }
};

// A workgroup writes 4 chunks a thread of a row (distillation's gradient of 4096 x 65536 bf16: 184 us, 262 with 16 chunks a
// thread).  One wavefront where that is the row, which then needs no barriers (log probabilities' of 16384 x 1000 bf16: 57 us with
// workgroups of 256, 14 so).
struct Pieces { int block, count, chunks; bool past; };  // chunks of a piece; whether it is stored past the caches

static Pieces grad_pieces(int dtype, int64_t rows, int64_t classes)
{
    const int64_t v = 16 / (int64_t)elem_size(dtype);
    const int64_t chunks = (classes + v - 1) / v + 1;  // one more than the row has: they are counted from an aligned address in front of it
    const int block = chunks <= 4 * 64 ? 64 : 256;
    return {block, (int)((chunks + 4 * block - 1) / (4 * block)), 4 * block, past_caches(dtype, rows, classes)};
}

// ONE: at most one target a row, which is added where its chunk is written; else the targets are a list.
template <typename T, int BLOCK, bool ONE>
__global__ __launch_bounds__(BLOCK) void logprob_backward_kernel(const T *logits, int64_t ld, int64_t rows, int n, Pieces pieces, float c, float inv_t,
                                                                 const int64_t *__restrict__ targets, int given, const float *__restrict__ dlogprob,
                                                                 const float *__restrict__ dentropy, const float *__restrict__ entropy, const float *__restrict__ stats,
                                                                 T *out, int64_t ld_out)
{
    constexpr int V = CHUNK<T>;
    __shared__ ListLds<ONE ? 1 : GIVEN_MOST> l;
    const int64_t id = grid_row(), r = id / pieces.count;
    if (r >= rows) return;
    const int64_t c0 = (id % pieces.count) * pieces.chunks, c1 = c0 + pieces.chunks;
    const T *in = logits + r * ld;
    T *to = out + r * ld_out;
    const float m = stats[2 * r], s = stats[2 * r + 1];
    const bool none = m == -INFINITY && s == 0.f;
    int64_t target = -1;
    float all = 0.f;
    auto gradient = [&](int64_t at, float d) { return at < 0 || none ? 0.f : at < n ? d * inv_t : NAN; };
    if (ONE) {
        if (given > 0) {
            target = targets[r];
            all = gradient(target, dlogprob[r]);
        }
    } else {
        for (int i = threadIdx.x; i < given; i += BLOCK) {
            const int64_t at = targets[r * given + i];
            l.at[i] = at < n ? (int)(at < 0 ? -1 : at) : -1;
            l.add[i] = gradient(at, dlogprob[r * given + i]);
        }
        l.close(given);
        __syncthreads();
        // (by every thread: 2047 x 50021 bf16 with 1 or 16 targets 75 us, with 128 93, with 1024, which look through the list besides, 1.9 ms)
        for (int i = 0; i < given; ++i) all += l.add[i];
    }
    // d x = 1/T [ sum dlp (delta - p) - dH p (ln p + H) ] = listed + p (a + b z),  ln p = ln2 z - ln s
    const float dh = dentropy != nullptr ? dentropy[r] * inv_t : 0.f, lns = logf(s);
    const float h = dentropy != nullptr ? entropy[r] : 0.f;
    const float inv_s = none ? 0.f : 1.f / s, a = none ? 0.f : (-all - dh * (h - lns)) * inv_s, b = none ? 0.f : -dh * LN2 * inv_s, m0 = none ? 0.f : m;
    auto value = [&](float x) {
        const float z = fmaxf((x - m0) * c, Z_LEAST);
        return exp2_fast(z) * fmaf(b, z, a);
    };
    if (ONE) {
        const int at0 = target >= 0 && target < n ? (int)target : -V;
        write_row<T, BLOCK, 4>(in, to, n, c0, c1, pieces.past, value, [&](int at, float(&x)[V]) {
            if ((unsigned)(at0 - at) < (unsigned)V)
#pragma unroll
                for (int j = 0; j < V; ++j) x[j] += at + j == at0 ? all : 0.f;
        });
        return;
    }
    ListedOut<T, BLOCK, ONE ? 1 : GIVEN_MOST> listed;
    listed.read(in, to, n, c0, c1, l, given);
    __syncthreads();
    write_row<T, BLOCK, 4>(in, to, n, c0, c1, pieces.past, value, [](int, float(&)[V]) {});
    __syncthreads();
    listed.write(to, l, given, value);
}

template <typename T> static int logprob_backward(const LogitsArgs &a, const int64_t *targets, int given, const float *dlogprob, const float *dentropy, const float *entropy,
                                                  const float *stats, T *out, int64_t ld_out, hipStream_t s)
{
    const Pieces pieces = grad_pieces(a.dtype, a.rows, a.classes);
#define OMNI_LOGPROB_BACKWARD(B, ONE)                                                                                                                                           \
    hipLaunchKernelGGL((logprob_backward_kernel<T, B, ONE>), row_grid(a.rows * pieces.count), dim3(B), 0, s, (const T *)a.logits, a.ld, a.rows, (int)a.classes, pieces, LOG2E / a.temperature, \
                       1.f / a.temperature, targets, given, dlogprob, dentropy, entropy, stats, out, ld_out)
    if (given <= 1 && pieces.block == 64) OMNI_LOGPROB_BACKWARD(64, true);
    else if (given <= 1) OMNI_LOGPROB_BACKWARD(256, true);
    else OMNI_LOGPROB_BACKWARD(256, false);
#undef OMNI_LOGPROB_BACKWARD
    OMNI_LAUNCH_CHECK();
    return OMNI_OK;
}

int launch_logprob_backward(const LogitsArgs &a, const int64_t *targets, int given, const float *dlogprob, const float *dentropy, const float *entropy, const float *stats,
                            void *out, int64_t ld_out, hipStream_t s)
{
    ProfScope prof(KID_LOGPROB, s, 0.0, 2.0 * (double)a.rows * a.classes * elem_size(a.dtype));
    return a.dtype == OMNI_BF16 ? logprob_backward<bf16_t>(a, targets, given, dlogprob, dentropy, entropy, stats, (bf16_t *)out, ld_out, s)
                                : logprob_backward<float>(a, targets, given, dlogprob, dentropy, entropy, stats, (float *)out, ld_out, s);
}

// Slots of 2^shift batches, at most SLOTS of them for a row that may begin anywhere in its first chunk.
static int slot_shift(int64_t chunks, int block)
{
    int shift = 0;
    while (((chunks / (BATCH * block)) >> shift) + 1 > SLOTS) ++shift;
    return shift;
}

// The parts' launch: their sums, and with top > 0 their largest elements.
template <typename T, int ALSO> static int launch_parts(const LogitsArgs &a, const Parts &p, float c, int top, float4 *sums, uint64_t *keys, hipStream_t s)
{
    const int64_t chunks = p.length / CHUNK<T>;
    const int shift = slot_shift(chunks, 256);
    const dim3 grid = row_grid(a.rows * p.count);
#define OMNI_PARTS(K, TOP) \
    hipLaunchKernelGGL((row_parts_kernel<T, K, ALSO, TOP>), grid, dim3(256), 0, s, (const T *)a.logits, a.ld, a.rows, (int)a.classes, p.count, p.length, c, shift, top, sums, keys)
#define OMNI_PARTS_BY_LENGTH(TOP)                 \
    do {                                          \
        if (chunks <= 4 * 256) OMNI_PARTS(4, TOP); \
        else OMNI_PARTS(0, TOP);                  \
    } while (0)
    if constexpr (ALSO == NOTHING || ALSO == Z_TIMES) {
        if (top > 0) OMNI_PARTS_BY_LENGTH(true);
        else OMNI_PARTS_BY_LENGTH(false);
    } else {
        OMNI_PARTS_BY_LENGTH(false);
    }
#undef OMNI_PARTS_BY_LENGTH
#undef OMNI_PARTS
    OMNI_LAUNCH_CHECK();
    return OMNI_OK;
}

template <typename T, bool ENTROPY> static int logprob_forward(const LogitsArgs &a, const LogprobOut &o, void *workspace, hipStream_t s)
{
    const int64_t chunks = a.classes / CHUNK<T>;
    const float inv_t = 1.f / a.temperature, c = LOG2E / a.temperature;
    const Parts p = row_parts(a.dtype, a.rows, a.classes, o.top > 0 ? TOPS : SUMS);
    if (p.count > 1) {
        float4 *sums = (float4 *)workspace;
        uint64_t *keys = (uint64_t *)(sums + a.rows * p.count);
        const int st = launch_parts<T, ENTROPY ? Z_TIMES : NOTHING>(a, p, c, o.top, sums, keys, s);
        if (st != OMNI_OK) return st;
        hipLaunchKernelGGL((logprob_join_kernel<T, ENTROPY>), dim3((unsigned)a.rows), dim3(256), (size_t)p.count * o.top * sizeof(uint64_t), s, (const T *)a.logits, a.ld, (int)a.classes,
                           p.count, c, inv_t, sums, keys, o);
        OMNI_LAUNCH_CHECK();
        return OMNI_OK;
    }
    // short rows stay with one wavefront, which needs no barriers
#define OMNI_LOGPROB(B, K) \
    hipLaunchKernelGGL((logprob_forward_kernel<T, B, K, ENTROPY>), row_grid(a.rows), dim3(B), 0, s, (const T *)a.logits, a.ld, a.rows, (int)a.classes, c, inv_t, slot_shift(chunks, B), o)
    if (chunks <= 256) OMNI_LOGPROB(64, 4);
    else if (chunks <= 512) OMNI_LOGPROB(64, 8);
    else if (chunks <= 1024) OMNI_LOGPROB(256, 4);
    else OMNI_LOGPROB(256, 0);
#undef OMNI_LOGPROB
    OMNI_LAUNCH_CHECK();
    return OMNI_OK;
}

int launch_logprob_forward(const LogitsArgs &a, const int64_t *targets, int given, float *logprob, float *entropy, int top, int64_t *top_index, float *top_logprob,
                           float *stats, void *workspace, hipStream_t s)
{
    ProfScope prof(KID_LOGPROB, s, 0.0, (double)a.rows * a.classes * elem_size(a.dtype));
    const LogprobOut o = {targets, given, logprob, entropy, top, top_index, top_logprob, stats};
    if (a.dtype == OMNI_BF16) return entropy != nullptr ? logprob_forward<bf16_t, true>(a, o, workspace, s) : logprob_forward<bf16_t, false>(a, o, workspace, s);
    return entropy != nullptr ? logprob_forward<float, true>(a, o, workspace, s) : logprob_forward<float, false>(a, o, workspace, s);
}

// ------------------------------------------------------------------------------------------------ distillation
//   q = softmax(t_k / T) over the entries that are there, p = softmax(x / T), p1 = softmax(x)
//   loss = alpha T^2 sum_k q_k (ln q_k - ln p_{i_k}) + (1 - alpha) (-ln p1_label)
//   d x_i = w [ alpha T (p_i - sum_{i_k = i} q_k) + (1 - alpha) (p1_i - [i = label]) ]
// With alpha = 1 or T = 1 one exponential an element serves both softmaxes, else two (TWO).
typedef ListLds<KEPT_MOST + 1> EntryLds;  // the label behind the entries

// The row's entries: at[k], and q_k in add[k].  Returns {ln sum, max, entries that are there, an index out of range}.
struct Entries { float lnsum, max; bool any, bad; };  // bad: an index or a logit that makes the row's results NaN

template <int BLOCK> __device__ __forceinline__ Entries read_entries(const DistillArgs &d, int64_t r, int n, float inv_t, EntryLds &l, float *lds)
{
    Entries e = {0.f, 0.f, false, false};
    float v[2] = {-INFINITY, 0.f};
    for (int i = threadIdx.x; i < d.kept; i += BLOCK) {
        int64_t at = d.index[r * d.kept + i];
        const float t = d.teacher[r * d.kept + i];
        if (t == -INFINITY) at = -1;
        if (at >= n) v[1] = 1.f, at = -1;
        if (at >= 0 && !(t < INFINITY)) v[1] = 1.f;
        if (at >= 0) v[0] = fmaxf(v[0], t);
        l.at[i] = at < 0 ? -1 : (int)at;
        l.add[i] = t;
    }
    block_join<BLOCK>(v, lds, Max());
    e.max = v[0];
    e.bad = v[1] > 0.f;
    e.any = v[0] > -INFINITY;
    float s[1] = {0.f};
    for (int i = threadIdx.x; i < d.kept; i += BLOCK)
        if (l.at[i] >= 0) s[0] += exp2_fast((l.add[i] - e.max) * (inv_t * LOG2E));
    block_join<BLOCK>(s, lds, Add());
    e.lnsum = logf(s[0]);
    return e;
}

template <typename T, int BLOCK, bool TWO>
__device__ __forceinline__ float row_loss(const DistillArgs &d, const T *row, int64_t r, int n, const Sums &a, const Entries &e, const EntryLds &l, float *lds)
{
    // (TWO: a.s at T, a.t at 1; else a.s for whichever is used)
    const float inv_t = 1.f / d.temperature;
    const bool none = a.m == -INFINITY && a.s == 0.f;
    float sum[1] = {0.f};
    if (e.any) {
        // T ln q and T ln p, which stay in range where ln p itself would not (a class masked with the type's lowest value, T < 1)
        const float tlns = d.temperature * logf(a.s), tlnsum = d.temperature * e.lnsum;
        for (int i = threadIdx.x; i < d.kept; i += BLOCK) {
            if (l.at[i] < 0) continue;
            const float lnq = l.add[i] - e.max - tlnsum, q = exp2_fast(lnq * (inv_t * LOG2E));
            const float lnp = none ? -INFINITY : element(row + l.at[i]) - a.m - tlns;
            if (!(q == 0.f)) sum[0] += q * (lnq - lnp);
        }
        block_join<BLOCK>(sum, lds, Add());
    }
    float loss = d.alpha > 0.f && d.kept > 0 ? d.alpha * d.temperature * sum[0] : 0.f;
    if (e.bad) loss = NAN;
    if (d.labels != nullptr && d.alpha < 1.f) {
        const int64_t at = d.labels[r];
        const float lns1 = logf(TWO ? a.t : a.s);
        if (at >= n) loss = NAN;
        else if (at >= 0) loss += (1.f - d.alpha) * (none ? INFINITY : lns1 - (element(row + at) - a.m));
    }
    return loss;
}

// The gradient's coefficients: d x = cT 2^(zT) + c1 2^(z1) + what is listed (entries, then the label).  idle: the row has neither an
// entry nor a label, and so no gradient, whatever its logits are (a row that fills a batch up may hold NaN).
struct Coefs { float ct, c1; int count; bool idle; };

template <int BLOCK, bool TWO> __device__ __forceinline__ Coefs row_coefs(const DistillArgs &d, int64_t r, int n, float m, float s, float s1, const Entries &e, float w, EntryLds &l)
{
    const float inv_t = 1.f / d.temperature, soft = d.alpha * d.temperature * w, hard = (1.f - d.alpha) * w;
    const bool none = m == -INFINITY && s == 0.f;
    Coefs k = {0.f, 0.f, d.kept, !e.any && !e.bad};
    for (int i = threadIdx.x; i < d.kept; i += BLOCK)
        l.add[i] = none || l.at[i] < 0 ? 0.f : -soft * exp2_fast(((l.add[i] - e.max) * inv_t - e.lnsum) * LOG2E);
    if (e.any && !none) k.ct = soft / s;
    if (e.bad) k.ct = NAN;
    if (d.labels != nullptr && d.alpha < 1.f) {
        const int64_t at = d.labels[r];
        if (threadIdx.x == 0) {
            l.at[d.kept] = at >= 0 && at < n ? (int)at : -1;
            l.add[d.kept] = none ? 0.f : -hard;
        }
        ++k.count;
        if (at >= 0 && !none) k.c1 = hard / (TWO ? s1 : s);
        if (at >= n) k.c1 = NAN;
        if (at >= 0) k.idle = false;
    }
    l.close(k.count);
    __syncthreads();
    return k;
}

// The gradient's value at x, ct 2^(zT) + c1 2^(z1).
template <int ALSO> struct Gradient {
    float m, c, ct, c1;
    __device__ __forceinline__ Gradient(const Coefs &k, float max, float scale) : m(max == -INFINITY ? 0.f : max), c(scale), ct(ALSO == NOTHING ? k.ct + k.c1 : k.ct), c1(k.c1) {}
    __device__ __forceinline__ float operator()(float x) const
    {
        const float d = x - m, e = exp2_fast(d * c);
        if (ALSO == NOTHING) return e * ct;
        if (ALSO == SQUARED) return e * fmaf(e, c1, ct);
        if (ALSO == SQUARED2) return e * fmaf(e * e * e, c1, ct);
        return e * ct + exp2_fast(d * LOG2E) * c1;
    }
};

// The loss of a row and what the backward pass needs of it, from the row's sums; returns the row's entries.
template <typename T, int BLOCK, int ALSO>
__device__ __forceinline__ Entries write_loss(const DistillArgs &d, const T *row, int64_t r, int n, const Sums &a, float *loss, float *stats, EntryLds &l, float *lds)
{
    const Entries e = read_entries<BLOCK>(d, r, n, 1.f / d.temperature, l, lds);
    __syncthreads();
    const float v = row_loss<T, BLOCK, ALSO != NOTHING>(d, row, r, n, a, e, l, lds);
    if (threadIdx.x == 0) {
        loss[r] = v;
        if (stats != nullptr) stats[4 * r] = a.m, stats[4 * r + 1] = a.s, stats[4 * r + 2] = ALSO != NOTHING ? a.t : a.s, stats[4 * r + 3] = 0.f;
    }
    return e;
}

// Whole rows: the loss alone.
template <typename T, int BLOCK, int ALSO>
__global__ __launch_bounds__(BLOCK) void distill_loss_kernel(const T *__restrict__ logits, int64_t ld, int64_t rows, int n, DistillArgs d, float c, float *__restrict__ loss,
                                                             float *__restrict__ stats)
{
    __shared__ float lds[2 * (BLOCK / 64)];
    __shared__ EntryLds l;
    const int64_t r = grid_row();
    if (r >= rows) return;
    const T *row = logits + r * ld;
    const RowSplit<T> sp(row, n);
    uint4 none[1];
    const Sums a = row_sums<T, BLOCK, ALSO, true, 0>(row, n, sp, c, nullptr, lds, none);
    write_loss<T, BLOCK, ALSO>(d, row, r, n, a, loss, stats, l, lds);
}

// ... of rows whose sums the parts' launch has taken, by as many threads as the gradient's workgroups have there
constexpr int JOIN_BLOCK = 256;

template <typename T, int ALSO>
__global__ __launch_bounds__(JOIN_BLOCK) void distill_join_kernel(const T *__restrict__ logits, int64_t ld, int n, int parts, DistillArgs d, float c, const float4 *__restrict__ sums,
                                                          float *__restrict__ loss, float *__restrict__ stats)
{
    __shared__ float lds[2 * (JOIN_BLOCK / 64)];
    __shared__ EntryLds l;
    const int64_t r = blockIdx.x;
    const Sums a = join_parts<ALSO>(sums + r * parts, parts, c);
    write_loss<T, JOIN_BLOCK, ALSO>(d, logits + r * ld, r, n, a, loss, stats, l, lds);
}

// The gradient of an idle row.
template <typename T, int BLOCK> __device__ __forceinline__ void write_nothing(const T *in, T *out, int n, int64_t c0, int64_t c1, bool past)
{
    write_row<T, BLOCK, 1>(in, out, n, c0, c1, past, [](float) { return 0.f; }, [](int, float(&)[CHUNK<T>]) {});
}

// Loss and gradient of whole rows.  The row's first KEPT chunks a thread stay in registers from the sums to the gradient; what
// a longer row has beyond them is read again.
template <typename T, int BLOCK, int KEPT, int ALSO>
__global__ __launch_bounds__(BLOCK) void distill_both_kernel(const T *logits, int64_t ld, int64_t rows, int n, DistillArgs d, float c, float *__restrict__ loss, T *out,
                                                             int64_t ld_out, int past)
{
    constexpr int V = CHUNK<T>;
    __shared__ float lds[2 * (BLOCK / 64)];
    __shared__ EntryLds l;
    const int64_t r = grid_row();
    if (r >= rows) return;
    const T *row = logits + r * ld;
    T *to = out + r * ld_out;
    const RowSplit<T> sp(row, n);
    uint4 kept[KEPT];
    const Sums a = row_sums<T, BLOCK, ALSO, false, KEPT>(row, n, sp, c, nullptr, lds, kept);
    const Entries e = write_loss<T, BLOCK, ALSO>(d, row, r, n, a, loss, nullptr, l, lds);
    const Coefs k = row_coefs<BLOCK, ALSO != NOTHING>(d, r, n, a.m, a.s, a.t, e, d.scale * (d.dloss != nullptr ? d.dloss[r] : 1.f), l);
    if (k.idle) return write_nothing<T, BLOCK>(row, to, n, 0, (n + 2 * V) / V, past);
    const Gradient<ALSO> value(k, a.m, c);
    ListedOut<T, BLOCK, KEPT_MOST + 1> listed;
    listed.read(row, n, l, k.count);
    const float edge = (int)threadIdx.x < sp.edges ? element(row + sp.edge(threadIdx.x, n)) : 0.f;
    __syncthreads();
    const bool aligned = past && ((uintptr_t)to / sizeof(T)) % V == sp.shift;
    auto put = [&](const uint4 &b, int c) {
        float x[V];
        unpack<T>(b, x);
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = value(x[j]);
        store_whole(to + sp.first(c), x, aligned);
    };
    int at = sp.lo + threadIdx.x;
#pragma unroll
    for (int u = 0; u < KEPT; ++u)
        if (at + u * BLOCK < sp.hi) put(kept[u], at + u * BLOCK);
    for (at += KEPT * BLOCK; at < sp.hi; at += BLOCK) put(raw_chunk<T, false>(row, sp.first(at)), at);
    if ((int)threadIdx.x < sp.edges) set_element(to + sp.edge(threadIdx.x, n), value(edge));
    __syncthreads();
    listed.write(to, l, k.count, value);
}

// The gradient from given sums: the statistics of an earlier call, or (sums != null) the parts' of this one.  loss != null: the
// row's first workgroup writes the loss, too, for which it reads all over the row -- not where the row is overwritten.
template <typename T, int BLOCK, int ALSO>
__global__ __launch_bounds__(BLOCK) void distill_backward_kernel(const T *logits, int64_t ld, int64_t rows, int n, Pieces pieces, DistillArgs d, float c,
                                                                      const float *__restrict__ stats, const float4 *__restrict__ sums, int parts, float *__restrict__ loss,
                                                                      T *out, int64_t ld_out)
{
    __shared__ float lds[2 * (BLOCK / 64)];
    __shared__ EntryLds l;
    const int64_t id = grid_row(), r = id / pieces.count;
    if (r >= rows) return;
    const int64_t c0 = (id % pieces.count) * pieces.chunks, c1 = c0 + pieces.chunks;
    const T *in = logits + r * ld;
    T *to = out + r * ld_out;
    Sums a;
    if (sums != nullptr) a = join_parts<ALSO>(sums + r * parts, parts, c);
    else a = {stats[4 * r], 0.f, stats[4 * r + 1], stats[4 * r + 2]};
    const Entries e = read_entries<BLOCK>(d, r, n, 1.f / d.temperature, l, lds);
    __syncthreads();
    if (loss != nullptr && c0 == 0) {
        const float v = row_loss<T, BLOCK, ALSO != NOTHING>(d, in, r, n, a, e, l, lds);
        if (threadIdx.x == 0) loss[r] = v;
        __syncthreads();
    }
    const Coefs k = row_coefs<BLOCK, ALSO != NOTHING>(d, r, n, a.m, a.s, a.t, e, d.scale * (d.dloss != nullptr ? d.dloss[r] : 1.f), l);
    if (k.idle) return write_nothing<T, BLOCK>(in, to, n, c0, c1, pieces.past);
    const Gradient<ALSO> value(k, a.m, c);
    ListedOut<T, BLOCK, KEPT_MOST + 1> listed;
    listed.read(in, to, n, c0, c1, l, k.count);
    __syncthreads();
    // (1021 x 32003 fp32: 47 us with one chunk ahead, 50 with four; 4096 x 65536 bf16: 197 and 184)
    write_row<T, BLOCK, sizeof(T) == 4 ? 1 : 4>(in, to, n, c0, c1, pieces.past, value, [](int, float(&)[CHUNK<T>]) {});
    __syncthreads();
    listed.write(to, l, k.count, value);
}

// What t holds: the second softmax is there only where both losses are, at different temperatures.  T = 2 and T = 4 take it as a
// power of the first, in one or two products instead of an exponential, four issue slots.
static Also second_softmax(const DistillArgs &d)
{
    if (!(d.alpha > 0.f && d.alpha < 1.f && d.kept > 0 && d.labels != nullptr && d.temperature != 1.f)) return NOTHING;
    return d.temperature == 2.f ? SQUARED : d.temperature == 4.f ? SQUARED2 : AT_ONE;
}

#define OMNI_BY_SECOND(LAUNCH, ...)                           \
    do {                                                      \
        const Also also = second_softmax(d);                  \
        if (also == NOTHING) LAUNCH(__VA_ARGS__, NOTHING);    \
        else if (also == SQUARED) LAUNCH(__VA_ARGS__, SQUARED); \
        else if (also == SQUARED2) LAUNCH(__VA_ARGS__, SQUARED2); \
        else LAUNCH(__VA_ARGS__, AT_ONE);                     \
    } while (0)

static float distill_scale(const DistillArgs &d) { return LOG2E / (d.alpha > 0.f && d.kept > 0 ? d.temperature : 1.f); }

template <typename T> static int distill_loss(const LogitsArgs &a, const DistillArgs &d, float *loss, float *stats, void *workspace, hipStream_t s)
{
    const float c = distill_scale(d);
    const int64_t chunks = a.classes / CHUNK<T>;
    const Parts p = row_parts(a.dtype, a.rows, a.classes, SUMS);
    if (p.count > 1) {
        float4 *sums = (float4 *)workspace;
        int st = OMNI_OK;
#define OMNI_DISTILL_PARTS(UNUSED, ALSO)                                                                                                                                 \
    do {                                                                                                                                                                 \
        if ((st = launch_parts<T, ALSO>(a, p, c, 0, sums, nullptr, s)) != OMNI_OK) return st;                                                                            \
        hipLaunchKernelGGL((distill_join_kernel<T, ALSO>), dim3((unsigned)a.rows), dim3(JOIN_BLOCK), 0, s, (const T *)a.logits, a.ld, (int)a.classes, p.count, d, c, sums, loss, stats); \
    } while (0)
        OMNI_BY_SECOND(OMNI_DISTILL_PARTS, 0);
#undef OMNI_DISTILL_PARTS
        OMNI_LAUNCH_CHECK();
        return OMNI_OK;
    }
#define OMNI_DISTILL_LOSS(B, ALSO) \
    hipLaunchKernelGGL((distill_loss_kernel<T, B, ALSO>), row_grid(a.rows), dim3(B), 0, s, (const T *)a.logits, a.ld, a.rows, (int)a.classes, d, c, loss, stats)
    if (chunks <= 512) OMNI_BY_SECOND(OMNI_DISTILL_LOSS, 64);
    else OMNI_BY_SECOND(OMNI_DISTILL_LOSS, 256);
#undef OMNI_DISTILL_LOSS
    OMNI_LAUNCH_CHECK();
    return OMNI_OK;
}

int launch_distill_loss(const LogitsArgs &a, const DistillArgs &d, float *loss, float *stats, void *workspace, hipStream_t s)
{
    ProfScope prof(KID_DISTILL, s, 0.0, (double)a.rows * a.classes * elem_size(a.dtype));
    return a.dtype == OMNI_BF16 ? distill_loss<bf16_t>(a, d, loss, stats, workspace, s) : distill_loss<float>(a, d, loss, stats, workspace, s);
}

template <typename T>
static int distill_backward(const LogitsArgs &a, const DistillArgs &d, const float *stats, const float4 *sums, int parts, float *loss, T *out, int64_t ld_out, hipStream_t s)
{
    const float c = distill_scale(d);
    const Pieces pieces = grad_pieces(a.dtype, a.rows, a.classes);
#define OMNI_DISTILL_BACKWARD(B, ALSO)                                                                                                                              \
    hipLaunchKernelGGL((distill_backward_kernel<T, B, ALSO>), row_grid(a.rows * pieces.count), dim3(B), 0, s, (const T *)a.logits, a.ld, a.rows, (int)a.classes, pieces, d, c, stats, \
                       sums, parts, loss, out, ld_out)
    if (pieces.block == 64) OMNI_BY_SECOND(OMNI_DISTILL_BACKWARD, 64);
    else OMNI_BY_SECOND(OMNI_DISTILL_BACKWARD, JOIN_BLOCK);
#undef OMNI_DISTILL_BACKWARD
    OMNI_LAUNCH_CHECK();
    return OMNI_OK;
}

template <typename T> static int distill_both(const LogitsArgs &a, const DistillArgs &d, float *loss, T *out, int64_t ld_out, void *workspace, hipStream_t s)
{
    const float c = distill_scale(d);
    const int64_t chunks = a.classes / CHUNK<T>;
    const Parts p = row_parts(a.dtype, a.rows, a.classes, BOTH);
    if (p.count > 1) {
        float4 *sums = (float4 *)workspace;
        int st = OMNI_OK;
        const bool over = (const void *)out == a.logits;
#define OMNI_DISTILL_PARTS(UNUSED, ALSO)                                                                                                                                 \
    do {                                                                                                                                                                 \
        if ((st = launch_parts<T, ALSO>(a, p, c, 0, sums, nullptr, s)) != OMNI_OK) return st;                                                                            \
        if (over)                                                                                                                                                        \
            hipLaunchKernelGGL((distill_join_kernel<T, ALSO>), dim3((unsigned)a.rows), dim3(JOIN_BLOCK), 0, s, (const T *)a.logits, a.ld, (int)a.classes, p.count, d, c, sums,   \
                               loss, nullptr);                                                                                                                           \
    } while (0)
        OMNI_BY_SECOND(OMNI_DISTILL_PARTS, 0);
#undef OMNI_DISTILL_PARTS
        OMNI_LAUNCH_CHECK();
        return distill_backward<T>(a, d, nullptr, sums, p.count, over ? nullptr : loss, out, ld_out, s);
    }
    const int past = past_caches(a.dtype, a.rows, a.classes);
#define OMNI_DISTILL_BOTH(B, K, ALSO) \
    hipLaunchKernelGGL((distill_both_kernel<T, B, K, ALSO>), row_grid(a.rows), dim3(B), 0, s, (const T *)a.logits, a.ld, a.rows, (int)a.classes, d, c, loss, out, ld_out, past)
    if (chunks <= 256) OMNI_BY_SECOND(OMNI_DISTILL_BOTH, 64, 4);
    else if (chunks <= 1024) OMNI_BY_SECOND(OMNI_DISTILL_BOTH, 256, 4);
    else if (chunks <= 2048) OMNI_BY_SECOND(OMNI_DISTILL_BOTH, 256, 8);
    else if (chunks <= 4096) OMNI_BY_SECOND(OMNI_DISTILL_BOTH, 256, 16);
    else if (chunks <= 8192) OMNI_BY_SECOND(OMNI_DISTILL_BOTH, 512, 16);
    else OMNI_BY_SECOND(OMNI_DISTILL_BOTH, 1024, 16);
#undef OMNI_DISTILL_BOTH
    OMNI_LAUNCH_CHECK();
    return OMNI_OK;
}

int launch_distill_both(const LogitsArgs &a, const DistillArgs &d, float *loss, void *out, int64_t ld_out, void *workspace, hipStream_t s)
{
    ProfScope prof(KID_DISTILL, s, 0.0, 2.0 * (double)a.rows * a.classes * elem_size(a.dtype));
    return a.dtype == OMNI_BF16 ? distill_both<bf16_t>(a, d, loss, (bf16_t *)out, ld_out, workspace, s) : distill_both<float>(a, d, loss, (float *)out, ld_out, workspace, s);
}

int launch_distill_backward(const LogitsArgs &a, const DistillArgs &d, const float *stats, void *out, int64_t ld_out, hipStream_t s)
{
    ProfScope prof(KID_DISTILL, s, 0.0, 2.0 * (double)a.rows * a.classes * elem_size(a.dtype));
    return a.dtype == OMNI_BF16 ? distill_backward<bf16_t>(a, d, stats, nullptr, 0, nullptr, (bf16_t *)out, ld_out, s)
                                : distill_backward<float>(a, d, stats, nullptr, 0, nullptr, (float *)out, ld_out, s);
}

}  // namespace omni
