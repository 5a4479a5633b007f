// Root-mean-square norm with the residual's addition and an 8-bit output, on tensors and on a received message
// (include/hxt.h: hxt_norm, hxt_unpack_norm).
#include "hxt_norm_kernels.h"

using namespace hxt;

namespace {

// ---- forward --------------------------------------------------------------------------
// Each row belongs to G threads, EPT values each, read once: x (of a message through its chunks) plus the residual as binary32,
// then the sum of squares, then the outputs, of q after one more total.  Bound by memory: a 4096 x 4096 message of x and residual
// into h and 8 bits with its sums 25.3 us (117 MB, 4.6 TB/s), 8192 x 3584 with a residual into h and y 46.3 us (235 MB, 5.1 TB/s).
template <typename T, int G, int EPT, Source SRC>
__global__ __launch_bounds__(G < 256 ? 256 : G) void k_norm(NormArgs a)
{
    constexpr uint32_t V = Number<T>::V, NV = EPT / V, PER = (G < 256 ? 256 : G) / G, WAVES = (G < 256 ? 256 : G) / 64;
    __shared__ float part[16];
    __shared__ uint32_t part_max[16], part_top[16];
    __shared__ uint64_t parts[SRC == FROM_MESSAGE_SUMMED ? WAVES : 1][4];
    const uint32_t t = threadIdx.x % G, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t first = (a.first_group + blockIdx.x) * PER, row = first + wave / (G / 64);
    const bool there = row < a.rows;
    const uint64_t rb = uint64_t(a.cols) * sizeof(T);
    float h[EPT];
#pragma unroll
    for (int i = 0; i < EPT; ++i) h[i] = 0;
    if (there) {
        u32x4 raw[NV], res[NV];
        // a row of the message that lies in one chunk, as most do, is read like a tensor's
        auto read = [&](const Rows &tensor, bool in_message, uint64_t off, u32x4 (&v)[NV]) {
            const uint8_t *at = tensor.p ? tensor.row(row) : nullptr;
            if (in_message) {
                const ChunkAt c = chunk_at(a.g, off + row * rb);
                at = c.rem + rb <= a.g.B ? a.packed + packed_place(a.g, c) : nullptr;
            }
            auto all = [&]<bool NT>() {
#pragma unroll
                for (uint32_t i = 0; i < NV; ++i) {
                    const uint32_t k = i * G + t, n = k * V < a.cols ? min(V, a.cols - k * V) : 0;
                    v[i] = n ? load_row<T, NT>(at, k, n) : u32x4{0, 0, 0, 0};
                }
            };
            if (at && (in_message ? a.nt_packed : a.nt)) {
                all.template operator()<true>();
            } else if (at) {
                all.template operator()<false>();
            } else {
#pragma unroll
                for (uint32_t i = 0; i < NV; ++i) {
                    const uint32_t k = i * G + t, n = k * V < a.cols ? min(V, a.cols - k * V) : 0;
                    v[i] = in_message && n ? load_packed<T>(a.g, a.packed, off + row * rb + k * 16, n) : u32x4{0, 0, 0, 0};
                }
            }
        };
        read(a.x, SRC != FROM_TENSORS, 0, raw);
        read(a.residual, SRC != FROM_TENSORS && a.residual_packed, a.residual_off, res);
        if constexpr (SRC == FROM_MESSAGE_SUMMED) {
            const uint32_t last = min(first + PER, a.rows);
            auto count = [&](uint64_t off, const u32x4 (&vec)[NV], uint64_t *to) {
                const Run run(a.g, off, rb, a.rows, first, last);
                RunSums s;
                const uint64_t at = off + row * rb;
                auto add = [&](uint64_t p, u32x4 v) {
                    if (p < run.border) s.before += words_sum(v);
                    else s.behind += words_sum(v);
                };
#pragma unroll
                for (uint32_t i = 0; i < NV; ++i) add(at + (i * G + t) * 16, vec[i]);        // (vectors past the row's end are zero)
                if (row + 1 == a.rows && t < 16) {           // the tensor's padding
                    const uint64_t p = off + uint64_t(a.rows) * rb + t * 16;
                    if (p < run.to) add(p, load16_any<false>(a.packed + packed_place(a.g, chunk_at(a.g, p))));
                }
                s.before = wave_sum64(s.before);
                if (run.border < run.to) s.behind = wave_sum64(s.behind);
                if ((threadIdx.x & 63) == 63) {
                    to[0] = s.before;
                    to[1] = s.behind;
                }
            };
            count(0, raw, parts[wave]);
            if (a.residual_packed) count(a.residual_off, res, parts[wave] + 2);
        }
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i) {
            float r[V];
            Number<T>::widen(raw[i], h + i * V);
            Number<T>::widen(res[i], r);
#pragma unroll
            for (uint32_t j = 0; j < V; ++j) h[i * V + j] += r[j];
        }
    } else if constexpr (SRC == FROM_MESSAGE_SUMMED) {
        if ((threadIdx.x & 63) < 4) parts[wave][threadIdx.x & 3] = 0;
    }
    float ss = 0;
#pragma unroll
    for (int i = 0; i < EPT; ++i) ss += h[i] * h[i];
    ss = row_sum<G>(ss, part);
    const float rstd = reciprocal_rms<G, EPT>(ss, [&](int i) { return h[i]; }, a.cols, a.eps, part, part_top);
    uint32_t top = 0;
#pragma unroll
    for (uint32_t i = 0; i < NV; ++i) {
        const uint32_t v = i * G + t, n = there && v * V < a.cols ? min(V, a.cols - v * V) : 0;
        if (!n) continue;
        float *f = h + i * V;
        if (a.h.p) store_row<T>(a.h.row(row), v, n, Number<T>::narrow(f), a.nt);
        float w[V];
        if (a.weight) Number<T>::widen(load_row<T>(a.weight, v, n), w);
#pragma unroll
        for (uint32_t j = 0; j < V; ++j) {
            f[j] = a.weight ? f[j] * rstd * w[j] : f[j] * rstd;
            top = max(top, magnitude(f[j]));
        }
        if (a.y.p) store_row<T>(a.y.row(row), v, n, Number<T>::narrow(f), a.nt);
    }
    if (a.q.p) {
        top = row_max<G>(top, part_max);
        // A row's largest value becomes 448.
        const float scale = top > 0x7F800000u ? __uint_as_float(0x7FC00000u) : fmaxf(__uint_as_float(top) / kE4m3Max, kLeastScale);
        if (there && t == 0) a.scale[row] = scale;
        // y / scale as binary32 rounds it: the product with 1 / scale, put right by what it leaves.  Tiny rows are lifted first, so that
        // this is a normal number; of an infinite scale nothing is taken away (finite values are 0 in it, infinite ones NaN).  (4096 x
        // 4096 with a residual: 25.3 us, with the product alone 24.8.)
        const bool tiny = scale < 0x1p-60f;               // (a row's threads are whole waves)
        const float unit = tiny ? scale * 0x1p64f : scale, inverse = 1.0f / unit, taken = unit < INFINITY ? unit : 0.0f;
        if (tiny) {
#pragma unroll
            for (int i = 0; i < EPT; ++i) h[i] *= 0x1p64f;
        }
        auto quotient = [&](float v) {
            const float about = v * inverse;
            return fmaf(fmaf(-about, taken, v), inverse, about);
        };
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i) {
            const uint32_t v = i * G + t, n = there && v * V < a.cols ? min(V, a.cols - v * V) : 0;
            if (!n) continue;
            const float *f = h + i * V;
            uint8_t *to = a.q.row(row) + size_t(v) * V;
            uint32_t w[V / 4];
#pragma unroll
            for (uint32_t j = 0; j < V; j += 4) w[j / 4] = e4m3x4(quotient(f[j]), quotient(f[j + 1]), quotient(f[j + 2]), quotient(f[j + 3]));
            if (n == V) {
                if constexpr (V == 8) {
                    if (a.nt) __builtin_nontemporal_store(u32x2{w[0], w[1]}, reinterpret_cast<u32x2_any *>(to));
                    else __builtin_memcpy(to, w, V);
                } else {
                    __builtin_memcpy(to, w, V);
                }
            } else {
#pragma unroll
                for (uint32_t j = 0; j < V; ++j)
                    if (j < n) to[j] = uint8_t(w[j / 4] >> (8 * (j & 3)));
            }
        }
    }
    if constexpr (SRC == FROM_MESSAGE_SUMMED) {
        // Last, so that nothing waits for the atomics.  (With several waves a row, the sums were there before row_sum's barrier.)
        if constexpr (G == 64) __syncthreads();
        if (threadIdx.x < 4 && (threadIdx.x < 2 || a.residual_packed)) {
            uint64_t v = 0;
#pragma unroll
            for (uint32_t w = 0; w < WAVES; ++w) v += parts[w][threadIdx.x];
            const Run run(a.g, threadIdx.x < 2 ? 0 : a.residual_off, rb, a.rows, first, min(first + PER, a.rows));
            const uint64_t n = threadIdx.x & 1 ? run.to - run.border : run.border - run.from;
            arrive_vectors(a.g, a.cx, run.chunk + (threadIdx.x & 1), v, uint32_t(n >> 4));
        }
    }
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
    if ((!a->h && !a->y && !a->q && a->rows > 0) || (a->q && !a->scale)) return HXT_EINVAL;
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
    n.nt = on_vectors(m.x) && on_vectors(m.residual) && on_vectors(m.h) && on_vectors(m.y);
    n.weight = static_cast<const uint8_t *>(a.weight);
    n.scale = a.scale;
    return n;
}

template <Source SRC>
void launch_norm(NormArgs n, hxt_dtype_t dtype, hipStream_t st)
{
    const RowShape shape = norm_shape(n.rows, n.cols, element_size(dtype));
    const uint32_t per = uint32_t(rows_of(shape));
    in_launches((uint64_t(n.rows) + per - 1) / per, uint32_t(group_threads(shape)), [&](uint32_t first, uint32_t count) {
        n.first_group = first;
        with_shape(dtype, shape, [&]<typename T, int G, int EPT>() { k_norm<T, G, EPT, SRC><<<count, group_threads(shape), 0, st>>>(n); });
    });
}

}  // namespace

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
    const Matrix weight(a->weight, 1, a->cols, 0, m.x.es);
    for (const Matrix *in : {&m.residual, &weight, &message})
        if (!in->disjoint(sum)) return HXT_EOVERLAP;
    NormArgs na = norm_args(*a);
    na.g = p.geom;
    na.packed = static_cast<const uint8_t *>(packed);
    na.nt_packed = operator_packed_nontemporal(plan, true);
    na.residual_packed = n == 2;
    na.residual_off = n == 2 ? p.tensors[1].stream_off : 0;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const uint64_t rb = m.x.row_bytes();
    if (sums && rb % 16 == 0 && p.B <= uint64_t(1) << 35 && p.B >= rb * uint64_t(rows_of(norm_shape(a->rows, a->cols, m.x.es)))) {       // the sums come with the rows (and a chunk's vectors are counted in 32 bits)
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

}  // extern "C"
