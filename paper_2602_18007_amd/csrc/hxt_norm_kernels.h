// What the norm (hxt_norm.hip) and its gradient (hxt_norm_grad.hip) share: rows in registers, their totals, and the choice of
// threads.  Both are bound by memory: a row is read once, kept in registers from the first pass over it to the last, and
// every output is written from there.
#ifndef HXT_NORM_KERNELS_H
#define HXT_NORM_KERNELS_H

#include <algorithm>
#include <cstring>

#include "hxt_operators.h"

namespace hxt {
namespace {

constexpr float kE4m3Max = 448.0f, kLeastScale = 0x1p-126f, kLeastEps = 1e-24f;
constexpr int64_t kMostCols = 32768;

enum Source { FROM_TENSORS = 0, FROM_MESSAGE = 1, FROM_MESSAGE_SUMMED = 2 };

struct Rows {                      // of a tensor
    uint8_t *p;
    uint64_t pitch;                // bytes
    __device__ __forceinline__ uint8_t *row(uint64_t r) const { return p + r * pitch; }
};

struct NormArgs {
    uint32_t rows, cols;
    uint32_t first_group;          // number of the launch's first workgroup
    float eps;
    Rows x, residual, h, y, q;     // p == nullptr: not there
    const uint8_t *weight;
    float *scale;
    ChunkGeom g;                   // of the message that x, and with residual_packed the residual, are in
    const uint8_t *packed;
    uint64_t residual_off;         // of the residual in the stream
    bool residual_packed;
    bool nt, nt_packed;            // cache hints of the tensors' rows and of the message
    SumCtx cx;
};

struct NormGradArgs {
    uint32_t rows, cols;
    float eps;
    bool nt, nt_packed;            // cache hints of the tensors' rows and of the message
    Rows h, dy, dh, dx;
    const uint8_t *weight;
    float *partial;                // [gridDim][cols], or nullptr
    ChunkGeom g;                   // of the message that dx goes into
    uint8_t *packed;
};

typedef u32x2 u32x2_any __attribute__((aligned(1)));

// ---- vectors of a row -----------------------------------------------------------------
// Vector v of a row has n elements, V of them or, at the row's end, fewer.

template <typename T, bool NT = false>
__device__ __forceinline__ u32x4 load_row(const uint8_t *row, uint32_t v, uint32_t n)
{
    constexpr uint32_t V = Number<T>::V;
    const uint8_t *at = row + size_t(v) * 16;
    if (n >= V) return load16_any<NT>(at);
    T e[V] = {};
#pragma unroll
    for (uint32_t i = 0; i < V; ++i)
        if (i < n) e[i] = reinterpret_cast<const T *>(at)[i];
    return __builtin_bit_cast(u32x4, e);
}

template <typename T>
__device__ __forceinline__ void store_row(uint8_t *row, uint32_t v, uint32_t n, u32x4 x, bool nt)
{
    constexpr uint32_t V = Number<T>::V;
    uint8_t *at = row + size_t(v) * 16;
    if (n >= V) {
        if (nt) store16_any<true>(at, x);
        else store16_cached(at, x);
        return;
    }
    T out[V];
    __builtin_memcpy(out, &x, 16);
#pragma unroll
    for (uint32_t i = 0; i < V; ++i)
        if (i < n) reinterpret_cast<T *>(at)[i] = out[i];
}

// The same at byte s of a message's stream.  A vector that ends in another chunk than it begins in goes by elements.
template <typename T>
__device__ __forceinline__ u32x4 load_packed(const ChunkGeom &g, const uint8_t *packed, uint64_t s, uint32_t n)
{
    constexpr uint32_t V = Number<T>::V;
    const ChunkAt at = chunk_at(g, s);
    if (n >= V && at.rem + 16 <= g.B) return load16_any<false>(packed + packed_place(g, at));
    T e[V] = {};
#pragma unroll
    for (uint32_t i = 0; i < V; ++i)
        if (i < n) e[i] = *reinterpret_cast<const T *>(packed + packed_place(g, chunk_at(g, s + i * sizeof(T))));
    return __builtin_bit_cast(u32x4, e);
}

template <typename T>
__device__ __forceinline__ void store_packed(const ChunkGeom &g, uint8_t *packed, uint64_t s, uint32_t n, u32x4 x)
{
    constexpr uint32_t V = Number<T>::V;
    const ChunkAt at = chunk_at(g, s);
    if (n >= V && at.rem + 16 <= g.B) {
        store16_any<false>(packed + packed_place(g, at), x);
        return;
    }
    T out[V];
    __builtin_memcpy(out, &x, 16);
#pragma unroll
    for (uint32_t i = 0; i < V; ++i)
        if (i < n) *reinterpret_cast<T *>(packed + packed_place(g, chunk_at(g, s + i * sizeof(T)))) = out[i];
}

// Zeros behind the last tensor byte, up to the stream's end (fewer than 256 bytes, all in the last tensor byte's chunk).
__device__ __forceinline__ void zero_padding(const ChunkGeom &g, uint8_t *packed, uint64_t tensor_bytes, uint32_t t, uint32_t threads)
{
    const uint64_t end = (tensor_bytes + 255) & ~uint64_t(255);
    for (uint64_t s = tensor_bytes + t; s < end; s += threads) packed[packed_place(g, chunk_at(g, s))] = 0;
}

// ---- totals of a row over the G threads that hold it -------------------------------------
template <int G>
__device__ __forceinline__ float row_sum(float v, float *part)
{
    v = wave_sum(v);
    if constexpr (G == 64) return v;
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0;
#pragma unroll
    for (int w = 0; w < G / 64; ++w) s += part[threadIdx.x / G * (G / 64) + w];
    return s;
}

template <int G>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t *part)
{
    v = wave_max(v);
    if constexpr (G == 64) return v;
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    uint32_t m = 0;
#pragma unroll
    for (int w = 0; w < G / 64; ++w) m = max(m, part[threadIdx.x / G * (G / 64) + w]);
    return m;
}

__device__ __forceinline__ uint32_t magnitude(float f) { return __float_as_uint(f) & 0x7FFFFFFFu; }

// 1 / sqrt(mean(h^2) + eps), given the sum of squares.  Where that has left binary32's range although no value is infinite
// (values from about 1e19 on), the row is taken again over its largest value; all threads that meet at a barrier take the same
// way (of two rows in a workgroup, both).
constexpr float kSquaresLeave = 3.0e38f;

template <int G>
__device__ __forceinline__ bool any_row(bool mine)
{
    return G > 64 && G < 256 ? __syncthreads_or(mine) != 0 : mine;
}

template <int G, int EPT, typename Value>
__device__ __forceinline__ float reciprocal_rms(float ss, Value &&value, uint32_t cols, float eps, float *part, uint32_t *part_max)
{
    const float plain = 1.0f / sqrtf(ss / float(cols) + eps);
    if (!any_row<G>(ss > kSquaresLeave)) return plain;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < EPT; ++i) top = max(top, magnitude(value(i)));
    if constexpr (G > 64) __syncthreads();
    top = row_max<G>(top, part_max);
    const float m = __uint_as_float(top), by = ss > kSquaresLeave && top < 0x7F800000u ? m : 1.0f;
    float s = 0;
#pragma unroll
    for (int i = 0; i < EPT; ++i) s += (value(i) / by) * (value(i) / by);
    if constexpr (G > 64) __syncthreads();
    s = row_sum<G>(s, part);
    return by == 1.0f ? plain : 1.0f / (by * sqrtf(s / float(cols) + eps / by / by));
}

// ---- sums of a message on the way ---------------------------------------------------------
// The rows of a workgroup are one run of the stream, no longer than a chunk: it lies in chunk c and, behind its border,
// in chunk c + 1.  A chunk is complete when all its 16-byte vectors have arrived, so arrivals count vectors, and no
// workgroup has to know how the others cut the chunk.
__device__ __forceinline__ void arrive_vectors(const ChunkGeom &g, const SumCtx &cx, uint32_t chunk, unsigned long long value, uint32_t vectors)
{
    if (!vectors) return;
    const uint64_t len = chunk + 1 == g.C ? g.L - uint64_t(chunk) * g.B : g.B;
    const uint32_t expected = uint32_t(len >> 4);
    Acc *a = reinterpret_cast<Acc *>(cx.acc + (size_t(cx.chunks) * cx.fan + chunk) * cx.stride);
    if (vectors != expected) {
        const unsigned long long before = __hip_atomic_fetch_add(&a->sum, value, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::"v"(uint32_t(before)) : "memory");
        if (__hip_atomic_fetch_add(&a->cnt, vectors, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + vectors != expected) return;
        value = __hip_atomic_exchange(&a->sum, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(&a->cnt, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    cx.sums[chunk] = value;
}

struct RunSums {
    uint64_t before = 0, behind = 0;     // words up to the run's chunk border and behind it
};

// A run [from, to) of stream bytes, pads included, and its chunk border (or its end, if that comes first).
struct Run {
    uint64_t from, to, border;
    uint32_t chunk;
    __device__ __forceinline__ Run(const ChunkGeom &g, uint64_t off, uint64_t rb, uint32_t rows, uint32_t first, uint32_t last)
    {
        from = off + first * rb;
        to = off + last * rb;
        if (last == rows) to = (to + 255) & ~uint64_t(255);
        const ChunkAt at = chunk_at(g, from);
        chunk = at.chunk;
        border = min(to, from + (g.B - at.rem));
    }
};

// ---- launches -----------------------------------------------------------------------------

// Threads that hold a row, and elements each of them holds.
struct RowShape {
    int threads, elements;
};

// Of many rows each belongs to as few threads as its values fit into (64 of bf16 and 32 of f32 each): waves on their own wait for
// nobody, and one has a whole row on its way at a time (8192 rows of 3584, bf16, with a residual: 46.7 us, by 256 threads a row
// 65).  Of few rows 256 threads take one, so that its latency is short (one row of 4096 5.7
// us, by one wave 10).
constexpr int64_t kManyRows = 1024;

inline RowShape norm_shape(int64_t rows, int64_t cols, int64_t es)
{
    if (cols <= 512) return {64, 8};
    if (rows < kManyRows && cols <= 8192) return {256, cols <= 2048 ? 8 : (cols <= 4096 ? 16 : 32)};
    if (cols <= 1024) return {64, 16};
    if (cols <= 2048) return {64, 32};
    const int most = es == 2 ? 64 : 32;
    int threads = 64;
    while (int64_t(threads) * most < cols) threads *= 2;
    return {threads, most};
}

// The gradient holds four values an element and the weight's sums: few elements a thread leave room for enough waves (4096 rows of
// 4096, bf16, into a message, with the sums over the workgroups: by 512 threads a row 34.6 us, by 256 36.0, by one wave 47.4).
inline RowShape norm_grad_shape(int64_t cols)
{
    if (cols <= 512) return {64, 8};
    if (cols <= 2048) return {256, 8};
    if (cols <= 4096) return {512, 8};
    if (cols <= 8192) return {512, 16};
    if (cols <= 16384) return {512, 32};
    return {1024, 32};
}

inline int group_threads(RowShape s) { return s.threads < 256 ? 256 : s.threads; }
inline int rows_of(RowShape s) { return group_threads(s) / s.threads; }

template <typename F>
void with_grad_shape(hxt_dtype_t type, RowShape s, F &&f)
{
    auto of = [&]<typename T>() {
        if (s.threads == 64) f.template operator()<T, 64, 8>();
        else if (s.threads == 256) f.template operator()<T, 256, 8>();
        else if (s.threads == 512 && s.elements == 8) f.template operator()<T, 512, 8>();
        else if (s.threads == 512 && s.elements == 16) f.template operator()<T, 512, 16>();
        else if (s.threads == 512) f.template operator()<T, 512, 32>();
        else f.template operator()<T, 1024, 32>();
    };
    if (type == HXT_BF16) of.template operator()<uint16_t>();
    else of.template operator()<uint32_t>();
}

// Calls f<T, threads of a row, elements of a thread>().
template <typename F>
void with_shape(hxt_dtype_t type, RowShape s, F &&f)
{
    const int k = s.threads * 64 + s.elements;
    auto both = [&]<typename T>() {
        if (k == 64 * 64 + 8) f.template operator()<T, 64, 8>();
        else if (k == 64 * 64 + 16) f.template operator()<T, 64, 16>();
        else if (k == 64 * 64 + 32) f.template operator()<T, 64, 32>();
        else if (k == 256 * 64 + 8) f.template operator()<T, 256, 8>();
        else if (k == 256 * 64 + 16) f.template operator()<T, 256, 16>();
        else if (k == 256 * 64 + 32) f.template operator()<T, 256, 32>();
        else return false;
        return true;
    };
    if (type == HXT_BF16) {
        using T = uint16_t;
        if (both.template operator()<T>()) return;
        if (s.threads == 64) f.template operator()<T, 64, 64>();
        else if (s.threads == 128) f.template operator()<T, 128, 64>();
        else if (s.threads == 256) f.template operator()<T, 256, 64>();
        else f.template operator()<T, 512, 64>();
    } else {
        using T = uint32_t;
        if (both.template operator()<T>()) return;
        if (s.threads == 128) f.template operator()<T, 128, 32>();
        else if (s.threads == 512) f.template operator()<T, 512, 32>();
        else f.template operator()<T, 1024, 32>();
    }
}

inline Rows rows_at(const Matrix &m) { return Rows{reinterpret_cast<uint8_t *>(m.p), m.pitch()}; }

inline int64_t element_size(hxt_dtype_t t) { return t == HXT_BF16 ? 2 : (t == HXT_F32 ? 4 : 0); }

// A plan's tensor t holds rows x cols elements of that type, one after another.
inline bool holds(const Plan &p, size_t t, int64_t elems, hxt_dtype_t type)
{
    const TensorPlan &tp = p.tensors[t];
    return tp.elems == uint64_t(elems) && (elems == 0 || (tp.kind == K_CONTIG && tp.dtype == type));
}

inline int check_sizes(int64_t rows, int64_t cols, hxt_dtype_t dtype, float eps)
{
    if (rows < 0 || cols < 1 || !element_size(dtype) || !(eps >= kLeastEps) || eps > 3.0e38f) return HXT_EINVAL;
    if (rows > 0x7FFFFFFF || cols > kMostCols) return HXT_EUNSUPPORTED;
    return HXT_OK;
}

// Rows that lie on 16 bytes are read and written non-temporally: they are new each time.  Others share bursts with their
// neighbours and go through the cache.
inline bool on_vectors(const Matrix &m) { return m.none() || (m.p % 16 == 0 && uint64_t(m.stride * m.es) % 16 == 0); }

}  // namespace
}  // namespace hxt

#endif
