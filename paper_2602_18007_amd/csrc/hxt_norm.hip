// Root-mean-square norm with the residual's addition and an 8-bit output, on tensors and on a received message, and its
// gradient, into tensors and into a message to send (include/hxt.h: hxt_norm ... hxt_pack_norm_grad).
//
// Both are bound by memory: a row is read once, kept in registers as binary32 from the first pass over it to the last,
// and every output is written from there.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>

#include "hxt_operators.h"

using namespace hxt;

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
    float eps;
    Rows x, residual, h, y, q;     // p == nullptr: not there
    const uint8_t *weight;
    float *scale;
    ChunkGeom g;                   // of the message that x, and with residual_packed the residual, are in
    const uint8_t *packed;
    uint64_t residual_off;         // of the residual in the stream
    bool residual_packed;
    SumCtx cx;
};

struct NormGradArgs {
    uint32_t rows, cols;
    float eps;
    Rows h, dy, dh, dx;
    const uint8_t *weight;
    float *partial;                // [gridDim * rows per workgroup][cols], or nullptr
    ChunkGeom g;                   // of the message that dx goes into
    uint8_t *packed;
};

// ---- vectors of a row -----------------------------------------------------------------
// Vector v of a row has n elements, V of them or, at the row's end, fewer.

template <typename T>
__device__ __forceinline__ u32x4 load_row(const uint8_t *row, uint32_t v, uint32_t n)
{
    constexpr uint32_t V = Number<T>::V;
    const uint8_t *at = row + size_t(v) * 16;
    if (n >= V) return load16_any<false>(at);
    T e[V] = {};
#pragma unroll
    for (uint32_t i = 0; i < V; ++i)
        if (i < n) e[i] = reinterpret_cast<const T *>(at)[i];
    return __builtin_bit_cast(u32x4, e);
}

template <typename T>
__device__ __forceinline__ void store_row(uint8_t *row, uint32_t v, uint32_t n, u32x4 x)
{
    constexpr uint32_t V = Number<T>::V;
    uint8_t *at = row + size_t(v) * 16;
    if (n >= V) {
        store16_any<false>(at, x);
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
    for (int w = 0; w < G / 64; ++w) s += part[w];
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
    for (int w = 0; w < G / 64; ++w) m = m > part[w] ? m : part[w];
    return m;
}

__device__ __forceinline__ uint32_t magnitude(float f) { return __float_as_uint(f) & 0x7FFFFFFFu; }

// 1 / sqrt(mean(h^2) + eps), given the sum of squares.  Where that has left binary32's range although no value is infinite
// (values from about 1e19 on), the row is taken again over its largest value; every thread of the row takes the same way.
template <int G, int EPT>
__device__ __forceinline__ float reciprocal_rms(float ss, const float (&h)[EPT], uint32_t cols, float eps, float *part, uint32_t *part_max)
{
    if (ss > 3.0e38f) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < EPT; ++i) top = max(top, magnitude(h[i]));
        if constexpr (G > 64) __syncthreads();
        top = row_max<G>(top, part_max);
        if (top < 0x7F800000u) {
            const float m = __uint_as_float(top);
            float s = 0;
#pragma unroll
            for (int i = 0; i < EPT; ++i) s += (h[i] / m) * (h[i] / m);
            if constexpr (G > 64) __syncthreads();
            s = row_sum<G>(s, part);
            return 1.0f / (m * sqrtf(s / float(cols) + eps / m / m));
        }
    }
    return 1.0f / sqrtf(ss / float(cols) + eps);
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

// One tensor's run [from, to) of stream bytes, pads included; parts: LDS for the waves' sums.
__device__ __forceinline__ void commit_run(const ChunkGeom &g, const SumCtx &cx, uint64_t from, uint64_t to, RunSums s, uint64_t (*parts)[2])
{
    s.before = wave_sum64(s.before);
    s.behind = wave_sum64(s.behind);
    if ((threadIdx.x & 63) == 0) {
        parts[threadIdx.x >> 6][0] = s.before;
        parts[threadIdx.x >> 6][1] = s.behind;
    }
    __syncthreads();
    if (threadIdx.x < 2) {
        uint64_t v = 0;
        for (uint32_t w = 0; w < blockDim.x / 64; ++w) v += parts[w][threadIdx.x];
        const ChunkAt at = chunk_at(g, from);
        const uint64_t border = min(to, from + (g.B - at.rem));
        const uint64_t n = threadIdx.x ? to - border : border - from;
        arrive_vectors(g, cx, at.chunk + threadIdx.x, v, uint32_t(n >> 4));
    }
}

// ---- forward --------------------------------------------------------------------------
template <typename T, int G, int EPT, Source SRC>
__global__ __launch_bounds__(G < 256 ? 256 : G) void k_norm(NormArgs a)
{
    constexpr uint32_t V = Number<T>::V, NV = EPT / V, PER = (G < 256 ? 256 : G) / G;
    __shared__ float part[16];
    __shared__ uint32_t part_max[16], part_top[16];
    __shared__ uint64_t parts[2][16][2];
    const uint32_t t = G < 256 ? threadIdx.x & (G - 1) : threadIdx.x;
    const uint32_t first = blockIdx.x * PER, row = first + (G < 256 ? threadIdx.x / G : 0);
    const bool there = row < a.rows;
    const uint64_t rb = uint64_t(a.cols) * sizeof(T);
    RunSums sums_x, sums_r;
    float h[EPT];
#pragma unroll
    for (int i = 0; i < EPT; ++i) h[i] = 0;
    if (there) {
        u32x4 raw[NV], res[NV];
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i) {
            const uint32_t v = i * G + t, n = v * V < a.cols ? min(V, a.cols - v * V) : 0;
            raw[i] = res[i] = u32x4{0, 0, 0, 0};
            if (!n) continue;
            if constexpr (SRC == FROM_TENSORS) raw[i] = load_row<T>(a.x.row(row), v, n);
            else raw[i] = load_packed<T>(a.g, a.packed, row * rb + v * 16, n);
            if (SRC != FROM_TENSORS && a.residual_packed) res[i] = load_packed<T>(a.g, a.packed, a.residual_off + row * rb + v * 16, n);
            else if (a.residual.p) res[i] = load_row<T>(a.residual.row(row), v, n);
        }
        if constexpr (SRC == FROM_MESSAGE_SUMMED) {
            auto count = [&](uint64_t off, const u32x4 (&vec)[NV], RunSums &s) {
                const uint64_t run = off + uint64_t(first) * rb, border = run + (a.g.B - chunk_at(a.g, run).rem);
                const uint64_t at = off + row * rb;
#pragma unroll
                for (uint32_t i = 0; i < NV; ++i) {      // (vectors past the row's end are zero)
                    const uint64_t w = words_sum(vec[i]);
                    if (at + (i * G + t) * 16 < border) s.before += w;
                    else s.behind += w;
                }
                if (row + 1 == a.rows && t < 16) {       // the tensor's padding
                    const uint64_t p = off + uint64_t(a.rows) * rb + t * 16;
                    if (p < ((off + uint64_t(a.rows) * rb + 255) & ~uint64_t(255))) {
                        const uint64_t w = words_sum(load16_any<false>(a.packed + packed_place(a.g, chunk_at(a.g, p))));
                        if (p < border) s.before += w;
                        else s.behind += w;
                    }
                }
            };
            count(0, raw, sums_x);
            if (a.residual_packed) count(a.residual_off, res, sums_r);
        }
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i) {
            float r[V];
            Number<T>::widen(raw[i], h + i * V);
            Number<T>::widen(res[i], r);
#pragma unroll
            for (uint32_t j = 0; j < V; ++j) h[i * V + j] += r[j];
        }
    }
    if constexpr (SRC == FROM_MESSAGE_SUMMED) {
        const uint64_t last = min(uint64_t(first) + PER, uint64_t(a.rows));
        auto end = [&](uint64_t off) { return last == a.rows ? (off + last * rb + 255) & ~uint64_t(255) : off + last * rb; };
        commit_run(a.g, a.cx, first * rb, end(0), sums_x, parts[0]);
        if (a.residual_packed) commit_run(a.g, a.cx, a.residual_off + first * rb, end(a.residual_off), sums_r, parts[1]);
    }
    float ss = 0;
#pragma unroll
    for (int i = 0; i < EPT; ++i) ss += h[i] * h[i];
    ss = row_sum<G>(ss, part);
    const float rstd = reciprocal_rms<G>(ss, h, a.cols, a.eps, part, part_top);
    uint32_t top = 0;
#pragma unroll
    for (uint32_t i = 0; i < NV; ++i) {
        const uint32_t v = i * G + t, n = there && v * V < a.cols ? min(V, a.cols - v * V) : 0;
        if (!n) continue;
        float *f = h + i * V;
        if (a.h.p) store_row<T>(a.h.row(row), v, n, Number<T>::narrow(f));
        float w[V];
        if (a.weight) Number<T>::widen(load_row<T>(a.weight, v, n), w);
#pragma unroll
        for (uint32_t j = 0; j < V; ++j) {
            f[j] = a.weight ? f[j] * rstd * w[j] : f[j] * rstd;
            top = max(top, magnitude(f[j]));
        }
        if (a.y.p) store_row<T>(a.y.row(row), v, n, Number<T>::narrow(f));
    }
    if (!a.q.p) return;
    top = row_max<G>(top, part_max);
    // A row's largest value becomes 448.  (A tiny row's scale stays a normal number, whose reciprocal is one too.)
    const float scale = top > 0x7F800000u ? __uint_as_float(0x7FC00000u) : fmaxf(__uint_as_float(top) / kE4m3Max, kLeastScale);
    const float inverse = 1.0f / scale;
    if (!there) return;
    if (t == 0) a.scale[row] = scale;
#pragma unroll
    for (uint32_t i = 0; i < NV; ++i) {
        const uint32_t v = i * G + t, n = v * V < a.cols ? min(V, a.cols - v * V) : 0;
        if (!n) continue;
        const float *f = h + i * V;
        uint8_t *to = a.q.row(row) + size_t(v) * V;
        uint32_t w[V / 4];
#pragma unroll
        for (uint32_t j = 0; j < V; j += 4) w[j / 4] = e4m3x4(f[j] * inverse, f[j + 1] * inverse, f[j + 2] * inverse, f[j + 3] * inverse);
        if (n == V) {
            __builtin_memcpy(to, w, V);
        } else {
#pragma unroll
            for (uint32_t j = 0; j < V; ++j)
                if (j < n) to[j] = uint8_t(w[j / 4] >> (8 * (j & 3)));
        }
    }
}

// ---- gradient ---------------------------------------------------------------------------
template <typename T, int G, int EPT, bool PACK>
__global__ __launch_bounds__(G < 256 ? 256 : G) void k_norm_grad(NormGradArgs a)
{
    constexpr uint32_t V = Number<T>::V, NV = EPT / V, PER = (G < 256 ? 256 : G) / G;
    __shared__ float part[2][16], part_s[16], part_g[16];
    __shared__ uint32_t part_top[16];
    const uint32_t t = G < 256 ? threadIdx.x & (G - 1) : threadIdx.x;
    const uint32_t mine = blockIdx.x * PER + (G < 256 ? threadIdx.x / G : 0), all = gridDim.x * PER;
    const uint64_t rb = uint64_t(a.cols) * sizeof(T);
    float w[EPT], dw[EPT];
#pragma unroll
    for (uint32_t i = 0; i < NV; ++i) {
        const uint32_t v = i * G + t, n = v * V < a.cols ? min(V, a.cols - v * V) : 0;
#pragma unroll
        for (uint32_t j = 0; j < V; ++j) {
            w[i * V + j] = 1.0f;
            dw[i * V + j] = 0;
        }
        if (n && a.weight) Number<T>::widen(load_row<T>(a.weight, v, n), w + i * V);
    }
    // rows: blockIdx.x * PER is the same for the whole workgroup, so that all its threads meet at the barriers
    for (uint64_t base = uint64_t(blockIdx.x) * PER; base < a.rows; base += all) {
        const uint64_t row = base + (mine - blockIdx.x * PER);
        const bool there = row < a.rows;
        float h[EPT], dy[EPT];
        u32x4 dh[NV];
        float ss = 0, sg = 0;
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i) {
            const uint32_t v = i * G + t, n = there && v * V < a.cols ? min(V, a.cols - v * V) : 0;
            u32x4 rh = u32x4{0, 0, 0, 0}, rd = rh;
            dh[i] = rh;
            if (n) {
                rh = load_row<T>(a.h.row(row), v, n);
                rd = load_row<T>(a.dy.row(row), v, n);
                if (a.dh.p) dh[i] = load_row<T>(a.dh.row(row), v, n);
            }
            Number<T>::widen(rh, h + i * V);
            Number<T>::widen(rd, dy + i * V);
        }
#pragma unroll
        for (int i = 0; i < EPT; ++i) {
            ss += h[i] * h[i];
            sg += h[i] * (dy[i] * w[i]);
        }
        ss = wave_sum(ss);
        sg = wave_sum(sg);
        if constexpr (G > 64) {
            __syncthreads();               // the last row's sums have been read
            if ((threadIdx.x & 63) == 0) {
                part[0][threadIdx.x >> 6] = ss;
                part[1][threadIdx.x >> 6] = sg;
            }
            __syncthreads();
            ss = sg = 0;
#pragma unroll
            for (int k = 0; k < G / 64; ++k) {
                ss += part[0][k];
                sg += part[1][k];
            }
        }
        const float rstd = reciprocal_rms<G>(ss, h, a.cols, a.eps, part_s, part_top);
        float mean;                         // of g * n
        if (ss > 3.0e38f) {
            float s = 0;
#pragma unroll
            for (int i = 0; i < EPT; ++i) s += h[i] * rstd * (dy[i] * w[i]);
            if constexpr (G > 64) __syncthreads();
            mean = row_sum<G>(s, part_g) / float(a.cols);
        } else {
            mean = sg * rstd / float(a.cols);
        }
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i) {
            const uint32_t v = i * G + t, n = there && v * V < a.cols ? min(V, a.cols - v * V) : 0;
            if (!n) continue;
            float d[V];
            Number<T>::widen(dh[i], d);
#pragma unroll
            for (uint32_t j = 0; j < V; ++j) {
                const uint32_t e = i * V + j;
                const float norm = h[e] * rstd;
                dw[e] += dy[e] * norm;
                d[j] += (dy[e] * w[e] - norm * mean) * rstd;
            }
            const u32x4 out = Number<T>::narrow(d);
            if constexpr (PACK) store_packed<T>(a.g, a.packed, row * rb + v * 16, n, out);
            else store_row<T>(a.dx.row(row), v, n, out);
        }
    }
    if constexpr (PACK)
        if (blockIdx.x == 0) zero_padding(a.g, a.packed, uint64_t(a.rows) * rb, threadIdx.x, blockDim.x);
    if (!a.partial) return;
    float *to = a.partial + size_t(mine) * a.cols;
#pragma unroll
    for (uint32_t i = 0; i < NV; ++i)
#pragma unroll
        for (uint32_t j = 0; j < V; ++j)
            if ((i * G + t) * V + j < a.cols) to[(i * G + t) * V + j] = dw[i * V + j];
}

// Column sums of n rows of partial sums: 4 columns a thread, 16 threads a row, SLICES of the rows side by side, joined in
// order.  Bound by the reading of the rows: 8 of them are in flight per thread.
template <int SLICES>
__global__ __launch_bounds__(16 * SLICES) void k_column_sums(const float *__restrict__ partial, uint32_t n, uint32_t cols, const float *add, float *to)
{
    __shared__ float part[SLICES][64];
    typedef f32x4 f32x4_any __attribute__((aligned(4)));
    const uint32_t quad = threadIdx.x & 15, slice = threadIdx.x >> 4, col = blockIdx.x * 64 + quad * 4;
    f32x4 s = {0, 0, 0, 0};
    if (col + 4 <= cols) {
#pragma unroll 8
        for (uint32_t r = slice; r < n; r += SLICES) s += *reinterpret_cast<const f32x4_any *>(partial + size_t(r) * cols + col);
    } else {
        for (uint32_t r = slice; r < n; r += SLICES)
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                if (col + i < cols) s[i] += partial[size_t(r) * cols + col + i];
    }
    *reinterpret_cast<f32x4 *>(&part[slice][quad * 4]) = s;
    __syncthreads();
    const uint32_t c = blockIdx.x * 64 + threadIdx.x;
    if (threadIdx.x >= 64 || c >= cols) return;
    float sum = 0;
#pragma unroll 8
    for (int k = 0; k < SLICES; ++k) sum += part[k][threadIdx.x];
    to[c] = add ? add[c] + sum : sum;
}

// ---- launches -----------------------------------------------------------------------------

// Threads that hold a row, and elements each of them holds.
struct RowShape {
    int threads, elements;
};

RowShape norm_shape(int64_t cols)
{
    if (cols <= 512) return {64, 8};
    if (cols <= 2048) return {256, 8};
    if (cols <= 4096) return {256, 16};
    if (cols <= 8192) return {256, 32};
    if (cols <= 16384) return {512, 32};
    return {512, 64};
}

template <typename F>
void with_shape(RowShape s, F &&f)
{
    if (s.threads == 64) f.template operator()<64, 8>();
    else if (s.elements == 8) f.template operator()<256, 8>();
    else if (s.elements == 16) f.template operator()<256, 16>();
    else if (s.threads == 256) f.template operator()<256, 32>();
    else if (s.elements == 32) f.template operator()<512, 32>();
    else f.template operator()<512, 64>();
}

int rows_of(RowShape s) { return s.threads == 64 ? 4 : 1; }

template <typename F>
void with_type(hxt_dtype_t t, F &&f)
{
    if (t == HXT_F32) f.template operator()<uint32_t>();
    else f.template operator()<uint16_t>();
}

Rows rows_at(const Matrix &m) { return Rows{reinterpret_cast<uint8_t *>(m.p), m.pitch()}; }

int64_t element_size(hxt_dtype_t t) { return t == HXT_BF16 ? 2 : (t == HXT_F32 ? 4 : 0); }

// A plan's tensor t holds rows x cols elements of that type, one after another.
bool holds(const Plan &p, size_t t, int64_t elems, hxt_dtype_t type)
{
    const TensorPlan &tp = p.tensors[t];
    return tp.elems == uint64_t(elems) && (elems == 0 || (tp.kind == K_CONTIG && tp.dtype == type));
}

int check_sizes(int64_t rows, int64_t cols, hxt_dtype_t dtype, float eps)
{
    if (rows < 0 || cols < 1 || !element_size(dtype) || !(eps >= kLeastEps) || eps > 3.0e38f) return HXT_EINVAL;
    if (rows > 0x7FFFFFFF || cols > kMostCols) return HXT_EUNSUPPORTED;
    return HXT_OK;
}

struct Norm {
    Matrix x, residual, h, y, q;
    explicit Norm(const hxt_norm_t &a)
        : x(a.x, a.rows, a.cols, a.x_stride, element_size(a.dtype)), residual(a.residual, a.rows, a.cols, a.residual_stride, x.es),
          h(a.h, a.rows, a.cols, a.h_stride, x.es), y(a.y, a.rows, a.cols, a.y_stride, x.es), q(a.q, a.rows, a.cols, a.q_stride, 1)
    {
    }
};

int check_norm(const hxt_norm_t *a, bool message)
{
    if (!a) return HXT_EINVAL;
    int rc = check_sizes(a->rows, a->cols, a->dtype, a->eps);
    if (rc != HXT_OK) return rc;
    if ((!a->h && !a->y && !a->q) || (a->q && !a->scale)) return HXT_EINVAL;
    if (message ? a->x != nullptr : (!a->x && a->rows > 0)) return HXT_EINVAL;
    const Norm m(*a);
    for (const Matrix *r : {&m.x, &m.residual})
        if ((rc = check_read(*r)) != HXT_OK) return rc;
    for (const Matrix *w : {&m.h, &m.y, &m.q})
        if ((rc = check_write(*w)) != HXT_OK) return rc;
    const Matrix weight(a->weight, 1, a->cols, 0, m.x.es), scale(a->q ? a->scale : nullptr, 1, a->rows, 0, 4);
    if ((rc = check_read(weight)) != HXT_OK || (rc = check_read(scale)) != HXT_OK) return rc;
    const bool h_in_place = !m.h.none();
    for (const Matrix *in : {&m.x, &m.residual}) {
        if (!m.h.disjoint(*in) && !m.h.is(*in)) return HXT_EOVERLAP;
        if (!m.y.disjoint(*in) && !(m.y.is(*in) && !h_in_place)) return HXT_EOVERLAP;
        if (!m.q.disjoint(*in) || !scale.disjoint(*in)) return HXT_EOVERLAP;
    }
    for (const Matrix *out : {&m.h, &m.y, &m.q, &scale})
        if (!out->disjoint(weight)) return HXT_EOVERLAP;
    if (!m.h.disjoint(m.y) || !m.h.disjoint(m.q) || !m.y.disjoint(m.q) || !scale.disjoint(m.h) || !scale.disjoint(m.y) || !scale.disjoint(m.q))
        return HXT_EOVERLAP;
    return HXT_OK;
}

NormArgs norm_args(const hxt_norm_t &a)
{
    const Norm m(a);
    NormArgs n;
    std::memset(&n, 0, sizeof n);
    n.rows = uint32_t(a.rows);
    n.cols = uint32_t(a.cols);
    n.eps = a.eps;
    n.x = rows_at(m.x);
    n.residual = rows_at(m.residual);
    n.h = rows_at(m.h);
    n.y = rows_at(m.y);
    n.q = rows_at(m.q);
    n.x.pitch = uint64_t(a.x_stride * m.x.es);
    n.residual.pitch = uint64_t(a.residual_stride * m.x.es);
    n.weight = static_cast<const uint8_t *>(a.weight);
    n.scale = a.scale;
    return n;
}

template <Source SRC>
void launch_norm(const NormArgs &n, hxt_dtype_t dtype, hipStream_t st)
{
    const RowShape shape = norm_shape(n.cols);
    const uint32_t per = uint32_t(rows_of(shape));
    with_type(dtype, [&]<typename T>() {
        with_shape(shape, [&]<int G, int EPT>() { k_norm<T, G, EPT, SRC><<<(n.rows + per - 1) / per, G < 256 ? 256 : G, 0, st>>>(n); });
    });
}

// Workgroups of the gradient: each leaves one row of partial weight gradients per row that it holds at a time.
uint32_t grad_groups(int64_t rows, RowShape s)
{
    const int64_t per = rows_of(s);
    return uint32_t(std::min<int64_t>((rows + per - 1) / per, s.threads == 512 ? 512 : 768));
}

struct NormGrad {
    Matrix h, dy, dh, dx;
    explicit NormGrad(const hxt_norm_grad_t &a)
        : h(a.h, a.rows, a.cols, a.h_stride, element_size(a.dtype)), dy(a.dy, a.rows, a.cols, a.dy_stride, h.es),
          dh(a.dh, a.rows, a.cols, a.dh_stride, h.es), dx(a.dx, a.rows, a.cols, a.dx_stride, h.es)
    {
    }
};

int check_norm_grad(const hxt_norm_grad_t *a, bool message)
{
    if (!a) return HXT_EINVAL;
    int rc = check_sizes(a->rows, a->cols, a->dtype, a->eps);
    if (rc != HXT_OK) return rc;
    const bool some = a->rows > 0;
    if ((some && (!a->h || !a->dy)) || (message ? a->dx != nullptr : (some && !a->dx))) return HXT_EINVAL;
    const NormGrad m(*a);
    for (const Matrix *r : {&m.h, &m.dy, &m.dh})
        if ((rc = check_read(*r)) != HXT_OK) return rc;
    if ((rc = check_write(m.dx)) != HXT_OK) return rc;
    const Matrix weight(a->weight, 1, a->cols, 0, m.h.es), dweight(a->dweight, 1, a->cols, 0, 4), add(a->dweight ? a->dweight_add : nullptr, 1, a->cols, 0, 4);
    for (const Matrix *r : {&weight, &dweight, &add})
        if ((rc = check_read(*r)) != HXT_OK) return rc;
    const size_t need = a->dweight ? hxt_norm_grad_work_bytes(a->rows, a->cols) : 0;
    const Matrix work(need ? a->work : nullptr, 1, int64_t(need), 0, 1);
    if (need && (!a->work || a->work_bytes < need)) return HXT_EINVAL;
    if (need && reinterpret_cast<uintptr_t>(a->work) % 16) return HXT_EALIGN;
    for (const Matrix *in : {&m.h, &m.dy, &m.dh}) {
        if (!m.dx.disjoint(*in) && !m.dx.is(*in)) return HXT_EOVERLAP;
        if (!dweight.disjoint(*in) || !work.disjoint(*in)) return HXT_EOVERLAP;
    }
    for (const Matrix *out : {&m.dx, &dweight, &work})
        if (!out->disjoint(weight) || (!out->disjoint(add) && !(out == &dweight && dweight.is(add)))) return HXT_EOVERLAP;
    if (!m.dx.disjoint(dweight) || !m.dx.disjoint(work) || !dweight.disjoint(work)) return HXT_EOVERLAP;
    return HXT_OK;
}

int run_norm_grad(const hxt_norm_grad_t &a, const Plan *p, uint8_t *packed, hipStream_t st)
{
    const NormGrad m(a);
    NormGradArgs n;
    std::memset(&n, 0, sizeof n);
    n.rows = uint32_t(a.rows);
    n.cols = uint32_t(a.cols);
    n.eps = a.eps;
    n.h = rows_at(m.h);
    n.dy = rows_at(m.dy);
    n.dh = rows_at(m.dh);
    n.dx = rows_at(m.dx);
    n.h.pitch = uint64_t(a.h_stride * m.h.es);
    n.dy.pitch = uint64_t(a.dy_stride * m.h.es);
    n.dh.pitch = uint64_t(a.dh_stride * m.h.es);
    n.weight = static_cast<const uint8_t *>(a.weight);
    n.partial = a.dweight ? static_cast<float *>(a.work) : nullptr;
    if (p) n.g = p->geom;
    n.packed = packed;
    const RowShape shape = norm_shape(a.cols);
    const uint32_t groups = a.rows ? grad_groups(a.rows, shape) : 0;
    if (groups)
        with_type(a.dtype, [&]<typename T>() {
            with_shape(shape, [&]<int G, int EPT>() {
                if (p) k_norm_grad<T, G, EPT, true><<<groups, G < 256 ? 256 : G, 0, st>>>(n);
                else k_norm_grad<T, G, EPT, false><<<groups, G < 256 ? 256 : G, 0, st>>>(n);
            });
        });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return operator_fail(e);
    return a.dweight ? operator_column_sums(static_cast<const float *>(a.work), groups * uint32_t(rows_of(shape)), uint32_t(a.cols), a.dweight_add, a.dweight, st) : HXT_OK;
}

}  // namespace

int hxt::operator_column_sums(const float *partial, uint32_t n, uint32_t cols, const float *add, float *to, hipStream_t st)
{
    if (n <= 64) k_column_sums<16><<<(cols + 63) / 64, 256, 0, st>>>(partial, n, cols, add, to);
    else k_column_sums<64><<<(cols + 63) / 64, 1024, 0, st>>>(partial, n, cols, add, to);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HXT_OK : operator_fail(e);
}

extern "C" {

int hxt_norm(const hxt_norm_t *a, void *stream)
{
    int rc = check_norm(a, false);
    if (rc != HXT_OK || a->rows == 0) return rc;
    if ((rc = operator_device()) != HXT_OK) return rc;
    launch_norm<FROM_TENSORS>(norm_args(*a), a->dtype, static_cast<hipStream_t>(stream));
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HXT_OK : operator_fail(e);
}

int hxt_unpack_norm(const hxt_plan_t *plan, const void *packed, const hxt_norm_t *a, uint64_t *sums, void *stream)
{
    if (!plan) return HXT_EINVAL;
    int rc = check_norm(a, true);
    if (rc != HXT_OK) return rc;
    const Plan &p = operator_plan(plan);
    const size_t n = p.tensors.size();
    if (n < 1 || n > 2) return HXT_EUNSUPPORTED;
    if (n == 2 && a->residual) return HXT_EINVAL;
    for (size_t t = 0; t < n; ++t)
        if (!holds(p, t, a->rows * a->cols, a->dtype)) return HXT_EUNSUPPORTED;
    if ((rc = operator_message(plan, packed)) != HXT_OK || p.C == 0) return rc;
    const Norm m(*a);
    const Matrix message(packed, 1, int64_t(p.C * p.B), 0, 1), sum(sums, 1, int64_t(p.C), 0, 8), scale(a->q ? a->scale : nullptr, 1, a->rows, 0, 4);
    if (sum.p % 8) return HXT_EALIGN;
    for (const Matrix *out : {&m.h, &m.y, &m.q, &scale})
        if (!out->disjoint(message) || !out->disjoint(sum)) return HXT_EOVERLAP;
    NormArgs na = norm_args(*a);
    na.g = p.geom;
    na.packed = static_cast<const uint8_t *>(packed);
    na.residual_packed = n == 2;
    na.residual_off = n == 2 ? p.tensors[1].stream_off : 0;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const uint64_t rb = m.x.row_bytes();
    if (sums && rb % 16 == 0 && p.B >= rb * uint64_t(rows_of(norm_shape(a->cols)))) {       // the sums come with the rows
        struct Enqueue {
            NormArgs &n;
            hxt_dtype_t dtype;
            hipStream_t st;
        } e{na, a->dtype, st};
        return operator_unpack_sums(plan, sums, st, [](void *ctx, const SumCtx &cx) {
            Enqueue &x = *static_cast<Enqueue *>(ctx);
            x.n.cx = cx;
            launch_norm<FROM_MESSAGE_SUMMED>(x.n, x.dtype, x.st);
        }, &e);
    }
    launch_norm<FROM_MESSAGE>(na, a->dtype, st);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return operator_fail(e);
    return sums ? operator_sums(plan, packed, sums, false, st) : HXT_OK;
}

size_t hxt_norm_grad_work_bytes(int64_t rows, int64_t cols)
{
    if (rows <= 0 || cols <= 0 || rows > 0x7FFFFFFF || cols > kMostCols) return 0;
    const RowShape s = norm_shape(cols);
    return size_t(grad_groups(rows, s)) * size_t(rows_of(s)) * size_t(cols) * sizeof(float);
}

int hxt_norm_grad(const hxt_norm_grad_t *a, void *stream)
{
    int rc = check_norm_grad(a, false);
    if (rc != HXT_OK || (a->rows == 0 && !a->dweight)) return rc;
    if ((rc = operator_device()) != HXT_OK) return rc;
    return run_norm_grad(*a, nullptr, nullptr, static_cast<hipStream_t>(stream));
}

int hxt_pack_norm_grad(const hxt_plan_t *plan, const hxt_norm_grad_t *a, void *packed, uint64_t *sums, void *stream)
{
    if (!plan) return HXT_EINVAL;
    int rc = check_norm_grad(a, true);
    if (rc != HXT_OK) return rc;
    const Plan &p = operator_plan(plan);
    if (p.tensors.size() != 1 || !holds(p, 0, a->rows * a->cols, a->dtype)) return HXT_EUNSUPPORTED;
    if ((rc = operator_message(plan, packed)) != HXT_OK) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (p.C == 0) return a->dweight ? run_norm_grad(*a, nullptr, nullptr, st) : HXT_OK;
    const NormGrad m(*a);
    const size_t need = a->dweight ? hxt_norm_grad_work_bytes(a->rows, a->cols) : 0;
    const Matrix message(packed, 1, int64_t(p.C * p.B), 0, 1), sum(sums, 1, int64_t(p.C), 0, 8);
    if (sum.p % 8) return HXT_EALIGN;
    const Matrix weight(a->weight, 1, a->cols, 0, m.h.es), dweight(a->dweight, 1, a->cols, 0, 4),
        add(a->dweight ? a->dweight_add : nullptr, 1, a->cols, 0, 4), work(need ? a->work : nullptr, 1, int64_t(need), 0, 1);
    for (const Matrix *o : {&m.h, &m.dy, &m.dh, &weight, &dweight, &add, &work, &sum})
        if (!o->disjoint(message)) return HXT_EOVERLAP;
    for (const Matrix *o : {&m.h, &m.dy, &m.dh, &weight, &dweight, &add, &work})
        if (!o->disjoint(sum)) return HXT_EOVERLAP;
    if ((rc = run_norm_grad(*a, &p, static_cast<uint8_t *>(packed), st)) != HXT_OK) return rc;
    return sums ? operator_sums(plan, packed, sums, true, st) : HXT_OK;
}

}  // extern "C"
