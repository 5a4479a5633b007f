// Matrix products with their epilogue, into tensors and into a message to send, and their gradients (include/hxt.h:
// hxt_product ... hxt_product_grad): argument checks and launches.  The kernels are in hxt_product_kernels.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <array>
#include <cstring>

#include "hxt_product_kernels.h"
#include "hxt_product_rules.h"

using namespace hxt;

namespace {

constexpr int64_t kMostDepth = int64_t(1) << 24, kMostSize = 0x7FFFFFFF, kMostStride = int64_t(1) << 22;

int64_t element_size(hxt_dtype_t t) { return t == HXT_BF16 ? 2 : (t == HXT_F32 ? 4 : (t == HXT_E4M3 ? 1 : 0)); }

template <typename F>
int launched(F &&f)
{
    f();
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HXT_OK : operator_fail(e);
}

// The same for `groups` workgroups of so many threads: launch(arguments, workgroups).
template <typename F>
int launched(ProductArgs a, uint64_t groups, uint32_t threads, F &&launch)
{
    return launched([&] {
        in_launches(groups, threads, [&](uint32_t first, uint32_t count) {
            a.first_group = first;
            launch(a, count);
        });
    });
}

// A kernel with more than 64 KiB of dynamic LDS says so before it is launched.
int allow_lds(const void *kernel, uint32_t bytes)
{
    if (bytes <= 65536) return HXT_OK;
    const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, int(bytes));
    return e == hipSuccess ? HXT_OK : operator_fail(e);
}

template <Factor F, int TM, int TN, int WM, int WN, bool PA, bool QA, bool DIRECT>
int launch_tiles(const ProductArgs &a, hipStream_t st)
{
    constexpr uint32_t lds = product_lds(TM, TN, WM, WN, PA, QA);
    if (const int rc = allow_lds(reinterpret_cast<const void *>(&k_product<F, TM, TN, WM, WN, PA, QA, DIRECT>), lds); rc != HXT_OK) return rc;
    return launched(a, uint64_t(a.tiles_m) * a.tiles_n * a.splits, 64 * WM * WN, [&](const ProductArgs &run, uint32_t groups) {
        k_product<F, TM, TN, WM, WN, PA, QA, DIRECT><<<groups, 64 * WM * WN, lds, st>>>(run);
    });
}

// A row of 16-byte vectors at 16-byte multiples, in columns too where the rows are the contraction index.
bool vectors(const Operand &o, bool across, int64_t es)
{
    return reinterpret_cast<uintptr_t>(o.p) % 16 == 0 && o.stride % 16 == 0 && (!across || (int64_t(o.rows) * es) % 16 == 0);
}

template <Factor F, int WAVES>
int launch_rows(const ProductArgs &a, hipStream_t st)
{
    constexpr uint32_t lds = rows_lds(WAVES);
    return launched(a, up(a.e.n, 16), 64 * WAVES, [&](const ProductArgs &run, uint32_t groups) { k_product_rows<F, WAVES><<<groups, 64 * WAVES, lds, st>>>(run); });
}

template <Factor F>
int launch_ring(const ProductArgs &a, hipStream_t st)
{
    constexpr uint32_t lds = kRing * 2 * 64 * kStep;
    if (const int rc = allow_lds(reinterpret_cast<const void *>(&k_product_ring<F>), lds); rc != HXT_OK) return rc;
    return launched(a, uint64_t(a.tiles_m) * a.tiles_n * a.splits, 256, [&](const ProductArgs &run, uint32_t groups) { k_product_ring<F><<<groups, 256, lds, st>>>(run); });
}

// Copies an operand's rows to `to`.
template <Factor F>
int align_rows(Operand &o, bool across, uint8_t *to, hipStream_t st)
{
    using E = std::conditional_t<F == F_E4M3, uint8_t, uint16_t>;
    const uint32_t rows = across ? o.depth : o.rows, cols = across ? o.rows : o.depth, vectors = up(uint64_t(cols) * sizeof(E), 16);
    const uint64_t count = uint64_t(rows) * vectors;
    const int rc = launched([&] {
        in_launches((count + 255) / 256, 256, [&](uint32_t first, uint32_t groups) {
            k_product_align<E><<<groups, 256, 0, st>>>(o.p, o.stride, cols, count, vectors, reinterpret_cast<u32x4 *>(to), first);
        });
    });
    o.p = to;
    o.stride = int64_t(vectors) * 16;
    if (across) o.rows = uint32_t(vectors * 16 / sizeof(E));           // (the zeros behind are columns of their own, not stored)
    return rc;
}

template <Factor F, bool PA, bool QA>
int run_product(ProductArgs a, uint8_t *work, size_t work_bytes, hipStream_t st)
{
    constexpr int64_t es = F == F_E4M3 ? 1 : 2;
    const int64_t m = a.e.m, n = a.e.n, depth = a.p.depth;
    const bool p_direct = vectors(a.p, PA, es), q_direct = vectors(a.q, QA, es);
    const Way way = way_for(m, n, depth, es, PA, QA, p_direct, q_direct, work_bytes);
    const Shape &s = way.shape;
    int rc;
    if (way.copy_p && (rc = align_rows<F>(a.p, PA, work + way.p_at, st)) != HXT_OK) return rc;
    if (way.copy_q && (rc = align_rows<F>(a.q, QA, work + way.q_at, st)) != HXT_OK) return rc;
    a.tiles_m = up(a.e.m, s.tile);
    a.tiles_n = up(a.e.n, s.tile);
    a.splits = s.splits;
    a.split_steps = s.split_steps;
    a.work = reinterpret_cast<float *>(work);
    if constexpr (!PA && !QA)          // 16 waves where the workgroups do not fill the chip twice
        if (s.tile == 16) return a.e.n <= 8192 ? launch_rows<F, 16>(a, st) : launch_rows<F, 8>(a, st);
    if (!way.direct) rc = launch_tiles<F, 128, 128, 2, 2, PA, QA, false>(a, st);
    else if (s.tile == 256) {
        a.tiles_n -= s.half;
        rc = launch_tiles<F, 256, 256, 2, 4, PA, QA, true>(a, st);
        if (rc == HXT_OK && s.half) {
            a.n_first = a.tiles_n * 256;
            a.tiles_n = up(n - a.n_first, 128);
            rc = launch_tiles<F, 256, 128, 4, 2, PA, QA, true>(a, st);
        }
    }
    else if (s.tile == 128) rc = launch_tiles<F, 128, 128, 2, 2, PA, QA, true>(a, st);
    else if constexpr (!PA && !QA) rc = launch_ring<F>(a, st);
    else rc = HXT_EUNSUPPORTED;        // (not reached: rings are for operands along)
    if (rc != HXT_OK || a.splits <= 1) return rc;
    const uint64_t groups = uint64_t((a.e.n + 3) / 4) * a.e.m;
    return launched([&] { k_product_join<<<up(groups, 256), 256, 0, st>>>(a.work, a.splits, a.e); });
}

// One row's stride is no distance between rows: any is taken, and only whether it is a whole number of vectors is kept, by
// which a way is chosen.
bool far(const Matrix &m) { return !m.none() && m.rows > 1 && m.stride > kMostStride; }
int64_t row_stride(const Matrix &m) { return (m.rows > 1 ? m.stride : m.stride % 16) * m.es; }

Operand operand(const Matrix &m, bool across)
{
    return Operand{reinterpret_cast<const uint8_t *>(m.p), row_stride(m), uint32_t(across ? m.cols : m.rows), uint32_t(across ? m.rows : m.cols)};
}

// ---- forward --------------------------------------------------------------------------------
struct Product {
    Matrix a, b, a_scale, b_scale, bias, residual, pre, c, work;
    explicit Product(const hxt_product_t &x)
        : a(x.a, x.m, x.k, x.a_stride, element_size(x.dtype)), b(x.b, x.n, x.k, x.b_stride, element_size(x.dtype)),
          a_scale(x.a_scale, 1, x.m, 0, 4), b_scale(x.b_scale, 1, x.n, 0, 4), bias(x.bias, 1, x.n, 0, 2),
          residual(x.residual, x.m, x.n, x.residual_stride, element_size(x.out_dtype)), pre(x.pre, x.m, x.n, x.pre_stride, 2),
          c(x.c, x.m, x.n, x.c_stride, element_size(x.out_dtype)),
          work(x.work, 1, x.work ? int64_t(x.work_bytes) : 0, 0, 1)
    {
    }
};

int check_sizes(int64_t m, int64_t n, int64_t k)
{
    if (m < 0 || n < 0 || k < 0) return HXT_EINVAL;
    if (m > kMostSize || n > kMostSize || k > kMostDepth) return HXT_EUNSUPPORTED;
    const uint64_t tiles = uint64_t(up(m, 16)) * up(n, 16);
    return m > 0 && n > 0 && (tiles >> 30 || uint64_t(m) * uint64_t(n) >> 40) ? HXT_EUNSUPPORTED : HXT_OK;
}

int check_product(const hxt_product_t *x, bool message)
{
    if (!x) return HXT_EINVAL;
    if ((x->dtype != HXT_BF16 && x->dtype != HXT_E4M3) || (x->out_dtype != HXT_BF16 && x->out_dtype != HXT_F32)) return HXT_EINVAL;
    if (x->act < HXT_ACT_NONE || x->act > HXT_ACT_SILU) return HXT_EINVAL;
    if (x->dtype != HXT_E4M3 && (x->a_scale || x->b_scale)) return HXT_EINVAL;
    if (x->dtype == HXT_E4M3 && x->out_dtype == HXT_F32) return HXT_EUNSUPPORTED;
    int rc = check_sizes(x->m, x->n, x->k);
    if (rc != HXT_OK) return rc;
    const bool some = x->m > 0 && x->n > 0;
    if ((some && x->k > 0 && (!x->a || !x->b)) || (message ? x->c != nullptr : (some && !x->c))) return HXT_EINVAL;
    const Product p(*x);
    for (const Matrix *r : {&p.a, &p.b, &p.residual}) {
        if ((rc = check_read(*r)) != HXT_OK) return rc;
        if (far(*r)) return HXT_EUNSUPPORTED;
    }
    for (const Matrix *w : {&p.pre, &p.c}) {
        if ((rc = check_write(*w)) != HXT_OK) return rc;
        if (far(*w)) return HXT_EUNSUPPORTED;
    }
    for (const Matrix *r : {&p.a_scale, &p.b_scale, &p.bias})
        if ((rc = check_read(*r)) != HXT_OK) return rc;
    if (x->work_bytes > (size_t(1) << 62) || p.work.cols < int64_t(hxt_product_work_bytes(x->m, x->n, x->k, x->dtype))) return HXT_EINVAL;
    if (p.work.p % 16) return HXT_EALIGN;
    for (const Matrix *out : {&p.pre, &p.c, &p.work}) {
        for (const Matrix *in : {&p.a, &p.b, &p.a_scale, &p.b_scale, &p.bias})
            if (!out->disjoint(*in)) return HXT_EOVERLAP;
        if (!out->disjoint(p.residual) && !(out == &p.c && out->is(p.residual))) return HXT_EOVERLAP;
    }
    if (!p.pre.disjoint(p.c) || !p.pre.disjoint(p.work) || !p.c.disjoint(p.work)) return HXT_EOVERLAP;
    return HXT_OK;
}

int launch_forward(const hxt_product_t &x, const Plan *plan, void *packed, hipStream_t st)
{
    const Product p(x);
    ProductArgs a;
    std::memset(&a, 0, sizeof a);
    a.p = operand(p.a, false);
    a.q = operand(p.b, false);
    Epilogue &e = a.e;
    e.m = uint32_t(x.m);
    e.n = uint32_t(x.n);
    e.m_scale = x.a_scale;
    e.n_scale = x.b_scale;
    e.bias = static_cast<const uint16_t *>(x.bias);
    e.act = x.act;
    e.residual = static_cast<const uint8_t *>(x.residual);
    e.residual_stride = row_stride(p.residual);
    e.pre = static_cast<uint8_t *>(x.pre);
    e.pre_stride = int64_t(p.pre.pitch());
    e.out = static_cast<uint8_t *>(plan ? packed : x.c);
    e.out_stride = int64_t(p.c.pitch());
    e.out32 = x.out_dtype == HXT_F32;
    e.message = plan != nullptr;
    if (plan) e.g = plan->geom;
    uint8_t *work = static_cast<uint8_t *>(x.work);
    return x.dtype == HXT_E4M3 ? run_product<F_E4M3, false, false>(a, work, p.work.cols, st) : run_product<F_BF16, false, false>(a, work, p.work.cols, st);
}

// ---- gradients ---------------------------------------------------------------------------------
// Bands of rows whose column sums are taken side by side for dbias.
uint32_t bias_bands(int64_t m, int64_t n)
{
    const uint32_t across = up(uint64_t(n), 512);
    return std::max(1u, std::min(up(uint64_t(m), 16), 2048 / std::min(across, 2048u)));
}

size_t partial_bytes(int64_t m, int64_t n) { return (size_t(bias_bands(m, n)) * size_t(n) * sizeof(float) + 255) / 256 * 256; }

struct ProductGrad {
    Matrix dc, pre, a, b, dz, da, db, db_add, dbias, dbias_add, work;
    explicit ProductGrad(const hxt_product_grad_t &x)
        : dc(x.dc, x.m, x.n, x.dc_stride, 2), pre(x.act == HXT_ACT_NONE ? nullptr : x.pre, x.m, x.n, x.pre_stride, 2),
          a(x.db ? x.a : nullptr, x.m, x.k, x.a_stride, 2), b(x.da ? x.b : nullptr, x.n, x.k, x.b_stride, 2), dz(x.dz, x.m, x.n, x.dz_stride, 2),
          da(x.da, x.m, x.k, x.da_stride, 2), db(x.db, x.n, x.k, x.db_stride, element_size(x.db_dtype)),
          db_add(x.db ? x.db_add : nullptr, x.n, x.k, x.db_add_stride, element_size(x.db_dtype)), dbias(x.dbias, 1, x.n, 0, 4),
          dbias_add(x.dbias ? x.dbias_add : nullptr, 1, x.n, 0, 4), work(x.work, 1, x.work ? int64_t(x.work_bytes) : 0, 0, 1)
    {
    }
};

int check_product_grad(const hxt_product_grad_t *x)
{
    if (!x) return HXT_EINVAL;
    if ((x->db_dtype != HXT_BF16 && x->db_dtype != HXT_F32) || x->act < HXT_ACT_NONE || x->act > HXT_ACT_SILU) return HXT_EINVAL;
    int rc;
    for (const auto &[m, n, k] : {std::array<int64_t, 3>{x->m, x->n, x->k}, {x->m, x->k, x->n}, {x->n, x->k, x->m}})
        if ((rc = check_sizes(m, n, k)) != HXT_OK) return rc;
    const bool some = x->m > 0 && x->n > 0;
    if (some && (!x->dc || (x->act != HXT_ACT_NONE && (!x->pre || !x->dz)))) return HXT_EINVAL;
    if (some && x->k > 0 && ((x->da && !x->b) || (x->db && !x->a))) return HXT_EINVAL;
    const ProductGrad p(*x);
    for (const Matrix *r : {&p.dc, &p.pre, &p.a, &p.b, &p.db_add}) {
        if ((rc = check_read(*r)) != HXT_OK) return rc;
        if (far(*r)) return HXT_EUNSUPPORTED;
    }
    for (const Matrix *w : {&p.dz, &p.da, &p.db}) {
        if ((rc = check_write(*w)) != HXT_OK) return rc;
        if (far(*w)) return HXT_EUNSUPPORTED;
    }
    for (const Matrix *r : {&p.dbias, &p.dbias_add})
        if ((rc = check_read(*r)) != HXT_OK) return rc;
    if (x->work_bytes > (size_t(1) << 62) || p.work.cols < int64_t(hxt_product_grad_work_bytes(x->m, x->n, x->k))) return HXT_EINVAL;
    if (p.work.p % 16) return HXT_EALIGN;
    const Matrix *outs[] = {&p.dz, &p.da, &p.db, &p.dbias, &p.work};
    for (const Matrix *out : outs) {
        for (const Matrix *in : {&p.dc, &p.pre, &p.a, &p.b, &p.db_add, &p.dbias_add}) {
            const bool allowed = (out == &p.dz && (in == &p.dc || in == &p.pre)) || (out == &p.db && in == &p.db_add) || (out == &p.dbias && in == &p.dbias_add);
            if (!out->disjoint(*in) && !(allowed && out->is(*in))) return HXT_EOVERLAP;
        }
        for (const Matrix *other : outs)
            if (other != out && !out->disjoint(*other)) return HXT_EOVERLAP;
    }
    return HXT_OK;
}

Epilogue plain(const Matrix &out, bool f32)
{
    Epilogue e;
    std::memset(&e, 0, sizeof e);
    e.m = uint32_t(out.rows);
    e.n = uint32_t(out.cols);
    e.out = reinterpret_cast<uint8_t *>(out.p);
    e.out_stride = int64_t(out.pitch());
    e.out32 = f32;
    return e;
}

int launch_grad(const hxt_product_grad_t &x, hipStream_t st)
{
    const ProductGrad p(x);
    int rc;
    float *partial = static_cast<float *>(x.work);
    uint8_t *work = x.work ? static_cast<uint8_t *>(x.work) + partial_bytes(x.m, x.n) : nullptr;
    const size_t room = x.work ? x.work_bytes - std::min(x.work_bytes, partial_bytes(x.m, x.n)) : 0;
    Matrix dz = p.dz;                                    // what the products read
    if (x.act == HXT_ACT_NONE) dz = p.dc;
    const bool copies = x.act != HXT_ACT_NONE;
    if (x.n > 0 && x.m > 0 && (copies || x.dbias)) {
        DzArgs d;
        std::memset(&d, 0, sizeof d);
        d.m = uint32_t(x.m);
        d.n = uint32_t(x.n);
        d.dc = static_cast<const uint8_t *>(x.dc);
        d.pre = static_cast<const uint8_t *>(x.pre);
        d.dc_stride = row_stride(p.dc);
        d.pre_stride = row_stride(p.pre);
        d.dz = copies ? static_cast<uint8_t *>(x.dz) : nullptr;
        d.dz_stride = int64_t(p.dz.pitch());
        d.act = x.act;
        d.partial = x.dbias ? partial : nullptr;
        const dim3 grid(up(uint64_t(x.n), 512), bias_bands(x.m, x.n));
        if ((rc = launched([&] { k_product_dz<<<grid, 256, 0, st>>>(d); })) != HXT_OK) return rc;
    }
    if (x.dbias && x.n > 0) {
        const uint32_t bands = x.m > 0 ? bias_bands(x.m, x.n) : 0;
        if ((rc = operator_column_sums(partial, bands, uint32_t(x.n), x.dbias_add, x.dbias, st)) != HXT_OK) return rc;
    }
    if (x.da && x.m > 0 && x.k > 0) {
        ProductArgs a;
        std::memset(&a, 0, sizeof a);
        a.p = operand(dz, false);
        a.q = operand(p.b, true);
        a.p.depth = a.q.depth = uint32_t(x.n);
        a.e = plain(p.da, false);
        if ((rc = run_product<F_BF16, false, true>(a, work, room, st)) != HXT_OK) return rc;
    }
    if (x.db && x.n > 0 && x.k > 0) {
        ProductArgs a;
        std::memset(&a, 0, sizeof a);
        a.p = operand(dz, true);
        a.q = operand(p.a, true);
        a.p.depth = a.q.depth = uint32_t(x.m);
        a.e = plain(p.db, x.db_dtype == HXT_F32);
        a.e.residual = reinterpret_cast<const uint8_t *>(p.db_add.p);
        a.e.residual_stride = row_stride(p.db_add);
        if ((rc = run_product<F_BF16, true, true>(a, work, room, st)) != HXT_OK) return rc;
    }
    return HXT_OK;
}

}  // namespace

extern "C" {

size_t hxt_product_work_bytes(int64_t m, int64_t n, int64_t k, hxt_dtype_t dtype)
{
    if (check_sizes(m, n, k) != HXT_OK || (dtype != HXT_BF16 && dtype != HXT_E4M3)) return 0;
    return work_for(m, n, k, element_size(dtype), false, false);
}

int hxt_product(const hxt_product_t *x, void *stream)
{
    int rc = check_product(x, false);
    if (rc != HXT_OK || x->m == 0 || x->n == 0) return rc;
    if ((rc = operator_device()) != HXT_OK) return rc;
    return launch_forward(*x, nullptr, nullptr, static_cast<hipStream_t>(stream));
}

int hxt_pack_product(const hxt_plan_t *plan, const hxt_product_t *x, void *packed, uint64_t *sums, void *stream)
{
    if (!plan) return HXT_EINVAL;
    int rc = check_product(x, true);
    if (rc != HXT_OK) return rc;
    const Plan &p = operator_plan(plan);
    if (p.tensors.size() != 1) return HXT_EUNSUPPORTED;
    const TensorPlan &t = p.tensors[0];
    if (t.elems != uint64_t(x->m) * uint64_t(x->n) || (t.elems && (t.kind != K_CONTIG || t.dtype != x->out_dtype))) return HXT_EUNSUPPORTED;
    if ((rc = operator_message(plan, packed)) != HXT_OK || p.C == 0) return rc;
    const Product m(*x);
    const Matrix message(packed, 1, int64_t(p.C * p.B), 0, 1), sum(sums, 1, int64_t(p.C), 0, 8);
    if (sum.p % 8) return HXT_EALIGN;
    for (const Matrix *o : {&m.a, &m.b, &m.a_scale, &m.b_scale, &m.bias, &m.residual, &m.pre, &m.work})
        if (!o->disjoint(message) || !o->disjoint(sum)) return HXT_EOVERLAP;
    if (!sum.disjoint(message)) return HXT_EOVERLAP;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if ((rc = launch_forward(*x, &p, packed, st)) != HXT_OK) return rc;
    return sums ? operator_sums(plan, packed, sums, true, st) : HXT_OK;
}

size_t hxt_product_grad_work_bytes(int64_t m, int64_t n, int64_t k)
{
    if (check_sizes(m, n, k) != HXT_OK || check_sizes(m, k, n) != HXT_OK || check_sizes(n, k, m) != HXT_OK) return 0;
    if (m == 0 || n == 0) return 0;
    return partial_bytes(m, n) + std::max(work_for(m, k, n, 2, false, true), work_for(n, k, m, 2, true, true));
}

int hxt_product_grad(const hxt_product_grad_t *x, void *stream)
{
    int rc = check_product_grad(x);
    if (rc != HXT_OK) return rc;
    if ((rc = operator_device()) != HXT_OK) return rc;
    return launch_grad(*x, static_cast<hipStream_t>(stream));
}

}  // extern "C"
