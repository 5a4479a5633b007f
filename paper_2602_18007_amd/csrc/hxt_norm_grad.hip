// Gradient of the root-mean-square norm, into tensors and into a message to send (include/hxt.h: hxt_norm_grad,
// hxt_pack_norm_grad), and sums over the rows of partial sums.
#include "hxt_norm_kernels.h"

using namespace hxt;

namespace {

// Each row belongs to G threads: both sums of a row (of h^2 and of h dy w) come from one reading, the gradient from the registers.
// A workgroup walks the rows in strides of the grid and keeps the sums of dy n of its columns in registers.  Bound by memory: 4096 x
// 4096 bf16 with dh into a message 30.6 us (134 MB and 8 MB of partial sums, 4.7 TB/s), the sums' own launch 4.7.
template <typename T, int G, int EPT, bool PACK>
__global__ __launch_bounds__(G < 256 ? 256 : G) void k_norm_grad(NormGradArgs a)
{
    constexpr uint32_t V = Number<T>::V, NV = EPT / V, THREADS = G < 256 ? 256 : G, PER = THREADS / G;
    __shared__ float part[2][16], part_s[16], part_g[16];
    __shared__ __attribute__((aligned(16))) float joined[PER > 1 ? G * EPT : 1];
    __shared__ uint32_t part_top[16];
    const uint32_t t = threadIdx.x % G, group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / (G / 64);
    const uint64_t rb = uint64_t(a.cols) * sizeof(T);
    // Rows and the weight stay as they are in memory and are widened where they are used: half the registers, of bf16.
    u32x4 w[NV], h[NV], dy[NV], dh[NV];
    float dw[EPT];
    auto elements = [&](uint32_t i) {                     // of this thread's vector i
        const uint32_t v = i * G + t;
        return v * V < a.cols ? min(V, a.cols - v * V) : 0;
    };
#pragma unroll
    for (uint32_t i = 0; i < NV; ++i) {
        w[i] = u32x4{0, 0, 0, 0};
        if (a.weight) {
            if (elements(i)) w[i] = load_row<T>(a.weight, i * G + t, elements(i));
        } else {
            float one[V];
#pragma unroll
            for (uint32_t j = 0; j < V; ++j) one[j] = 1.0f;
            w[i] = Number<T>::narrow(one);
        }
#pragma unroll
        for (uint32_t j = 0; j < V; ++j) dw[i * V + j] = 0;
    }
    // rows: the first of a round is the same for the whole workgroup, so that all its threads meet at the barriers
    for (uint64_t base = uint64_t(blockIdx.x) * PER; base < a.rows; base += uint64_t(gridDim.x) * PER) {
        const uint64_t row = base + group;
        const bool there = row < a.rows;
        auto read = [&]<bool NT>() {
            const uint8_t *at_h = a.h.row(row), *at_dy = a.dy.row(row), *at_dh = a.dh.row(row);
#pragma unroll
            for (uint32_t i = 0; i < NV; ++i) {
                const uint32_t n = there ? elements(i) : 0;
                h[i] = n ? load_row<T, NT>(at_h, i * G + t, n) : u32x4{0, 0, 0, 0};
                dy[i] = n ? load_row<T, NT>(at_dy, i * G + t, n) : u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (uint32_t i = 0; i < NV; ++i) {
                const uint32_t n = there && a.dh.p ? elements(i) : 0;
                dh[i] = n ? load_row<T, NT>(at_dh, i * G + t, n) : u32x4{0, 0, 0, 0};
            }
        };
        if (a.nt) read.template operator()<true>();
        else read.template operator()<false>();
        float ss = 0, sg = 0;
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i) {
            float x[V], g[V], u[V];
            Number<T>::widen(h[i], x);
            Number<T>::widen(dy[i], g);
            Number<T>::widen(w[i], u);
#pragma unroll
            for (uint32_t j = 0; j < V; ++j) {
                ss += x[j] * x[j];
                sg += x[j] * (g[j] * u[j]);
            }
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
                ss += part[0][threadIdx.x / G * (G / 64) + k];
                sg += part[1][threadIdx.x / G * (G / 64) + k];
            }
        }
        auto element = [&](const u32x4 (&v)[NV], int i) {
            float x[V];
            Number<T>::widen(v[i / V], x);
            return x[i % V];
        };
        const float rstd = reciprocal_rms<G, EPT>(ss, [&](int i) { return element(h, i); }, a.cols, a.eps, part_s, part_top);
        float mean = sg * rstd / float(a.cols);                 // of g * n
        // Where the sum of squares or this one has left binary32's range: once more, from the normed row.
        const bool left = ss > kSquaresLeave || !(fabsf(sg) <= kSquaresLeave);
        if (any_row<G>(left)) {
            float s = 0;
#pragma unroll
            for (int i = 0; i < EPT; ++i) s += element(h, i) * rstd * (element(dy, i) * element(w, i));
            if constexpr (G > 64) __syncthreads();
            s = row_sum<G>(s, part_g);
            if (left) mean = s / float(a.cols);
        }
        // (widened again, not kept from the sums: that would be twice the registers)
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i) asm volatile("" : "+v"(h[i]), "+v"(dy[i]), "+v"(w[i]));
        const ChunkAt place = chunk_at(a.g, PACK ? row * rb : 0);
        uint8_t *to = PACK ? (place.rem + rb <= a.g.B ? a.packed + packed_place(a.g, place) : nullptr) : a.dx.row(row);     // (a row in one chunk)
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i) {
            const uint32_t v = i * G + t, n = there ? elements(i) : 0;
            if (!n) continue;
            float x[V], g[V], u[V], d[V];
            Number<T>::widen(h[i], x);
            Number<T>::widen(dy[i], g);
            Number<T>::widen(w[i], u);
            Number<T>::widen(dh[i], d);
#pragma unroll
            for (uint32_t j = 0; j < V; ++j) {
                const float norm = x[j] * rstd;
                dw[i * V + j] += g[j] * norm;
                d[j] += (g[j] * u[j] - norm * mean) * rstd;
            }
            const u32x4 out = Number<T>::narrow(d);
            if (!PACK || to) store_row<T>(to, v, n, out, PACK ? a.nt_packed : a.nt);
            else store_packed<T>(a.g, a.packed, row * rb + v * 16, n, out);
        }
    }
    if constexpr (PACK)
        if (blockIdx.x == 0) zero_padding(a.g, a.packed, uint64_t(a.rows) * rb, threadIdx.x, blockDim.x);
    if (!a.partial) return;
    // The rows that a workgroup holds at a time are joined in their order.
    if constexpr (PER > 1) {
        for (uint32_t k = 0; k < PER; ++k) {
            if (group == k)
#pragma unroll
                for (uint32_t i = 0; i < NV; ++i)
#pragma unroll
                    for (uint32_t j = 0; j < V; j += 4) {
                        f32x4 &sum = *reinterpret_cast<f32x4 *>(joined + (i * G + t) * V + j);
                        const f32x4 mine = {dw[i * V + j], dw[i * V + j + 1], dw[i * V + j + 2], dw[i * V + j + 3]};
                        sum = k ? sum + mine : mine;
                    }
            __syncthreads();
        }
        float *to = a.partial + size_t(blockIdx.x) * a.cols;
        for (uint32_t c = threadIdx.x; c < a.cols; c += THREADS) to[c] = joined[c];
    } else {
        float *to = a.partial + size_t(blockIdx.x) * a.cols;
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i)
#pragma unroll
            for (uint32_t j = 0; j < V; ++j)
                if ((i * G + t) * V + j < a.cols) to[(i * G + t) * V + j] = dw[i * V + j];
    }
}

// Column sums of n rows of partial sums: 4 columns a thread, 16 threads a row, SLICES of the rows side by side, joined in
// order.  Bound by the reading of the rows: 8 of them are in flight per thread.
template <int SLICES>
__global__ __launch_bounds__(16 * SLICES) void k_column_sums(const float *__restrict__ partial, uint32_t n, uint32_t cols, const float *add, float *to)
{
    __shared__ __attribute__((aligned(16))) float part[SLICES][64];
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

// Workgroups of the gradient: two a CU.  Each leaves one row of partial weight gradients, so that more of them cost more than they
// bring (34.6 us with 512, 41.0 with 1024).
constexpr int64_t kGradGroups = 512;
uint32_t grad_groups(int64_t rows, RowShape s)
{
    const int64_t per = rows_of(s);
    return uint32_t(std::min<int64_t>((rows + per - 1) / per, kGradGroups));
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

int run_norm_grad(const hxt_norm_grad_t &a, const Plan *p, uint8_t *packed, bool nt_packed, hipStream_t st)
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
    n.nt = on_vectors(m.h) && on_vectors(m.dy) && on_vectors(m.dh) && on_vectors(m.dx);
    n.nt_packed = nt_packed;
    const RowShape shape = norm_grad_shape(a.cols);
    const uint32_t groups = a.rows ? grad_groups(a.rows, shape) : 0;
    if (groups)
        with_grad_shape(a.dtype, shape, [&]<typename T, int G, int EPT>() {
            if (p) k_norm_grad<T, G, EPT, true><<<groups, group_threads(shape), 0, st>>>(n);
            else k_norm_grad<T, G, EPT, false><<<groups, group_threads(shape), 0, st>>>(n);
        });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return operator_fail(e);
    return a.dweight ? operator_column_sums(static_cast<const float *>(a.work), groups, uint32_t(a.cols), a.dweight_add, a.dweight, st) : HXT_OK;
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

size_t hxt_norm_grad_work_bytes(int64_t rows, int64_t cols)
{
    if (rows <= 0 || cols <= 0 || rows > 0x7FFFFFFF || cols > kMostCols) return 0;
    return size_t(grad_groups(rows, norm_grad_shape(cols))) * size_t(cols) * sizeof(float);
}

int hxt_norm_grad(const hxt_norm_grad_t *a, void *stream)
{
    int rc = check_norm_grad(a, false);
    if (rc != HXT_OK || (a->rows == 0 && !a->dweight)) return rc;
    if ((rc = operator_device()) != HXT_OK) return rc;
    return run_norm_grad(*a, nullptr, nullptr, false, static_cast<hipStream_t>(stream));
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
    if (p.C == 0) return a->dweight ? run_norm_grad(*a, nullptr, nullptr, false, st) : HXT_OK;
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
    if ((rc = run_norm_grad(*a, &p, static_cast<uint8_t *>(packed), operator_packed_nontemporal(plan, false), st)) != HXT_OK) return rc;
    return sums ? operator_sums(plan, packed, sums, true, st) : HXT_OK;
}

}  // extern "C"
