// What the operators at the ends of a stage (hxt_norm.hip, hxt_norm_grad.hip, hxt_product.hip) share: checks of their arguments, places in a
// packed buffer, number formats, and the parts of the plan's bookkeeping that hxt_device.hip lends them.
#ifndef HXT_OPERATORS_H
#define HXT_OPERATORS_H

#include <hip/hip_runtime.h>

#include <cstdint>

#include "hxt_internal.h"
#include "hxt_kernels.h"

namespace hxt {

// ---- from hxt_device.hip ------------------------------------------------------------
int operator_fail(hipError_t e);                                           // remembers e, returns HXT_EHIP
int operator_device();                                                     // HXT_EHIP if there is no HIP device
int operator_message(const hxt_plan_t *plan, const void *packed);          // the checks of hxt_pack / hxt_unpack
const Plan &operator_plan(const hxt_plan_t *plan);
bool operator_packed_nontemporal(const hxt_plan_t *plan, bool load);       // the packed side's cache hint
// Sums of a packed buffer by a pass of its own, with the accumulators of hxt_pack (send) or hxt_unpack.
int operator_sums(const hxt_plan_t *plan, const void *packed, uint64_t *sums, bool send, hipStream_t st);
// Calls enqueue(ctx, cx) while the accumulators of hxt_unpack are this call's.
int operator_unpack_sums(const hxt_plan_t *plan, uint64_t *sums, hipStream_t st, void (*enqueue)(void *ctx, const SumCtx &cx), void *ctx);

// to[c] = add[c] (nullptr: 0) + the sum over n rows of partial[.][c], in an order fixed by n (hxt_norm_grad.hip).
int operator_column_sums(const float *partial, uint32_t n, uint32_t cols, const float *add, float *to, hipStream_t st);

// ---- argument checks (host) ----------------------------------------------------------
// A matrix as the calls take it.
struct Matrix {
    uintptr_t p;
    int64_t rows, cols, stride;       // stride in elements
    int64_t es;

    Matrix(const void *base, int64_t rows_, int64_t cols_, int64_t stride_, int64_t es_)
        : p(reinterpret_cast<uintptr_t>(base)), rows(rows_), cols(cols_), stride(stride_), es(es_) {}
    bool none() const { return !p; }
    bool empty() const { return !p || rows == 0 || cols == 0; }
    uint64_t row_bytes() const { return uint64_t(cols * es); }
    uint64_t pitch() const { return rows > 1 ? uint64_t(stride * es) : row_bytes(); }
    uint64_t extent() const { return uint64_t(rows - 1) * pitch() + row_bytes(); }
    bool is(const Matrix &o) const { return p == o.p && es == o.es && pitch() == o.pitch(); }
    // No byte in common: apart, or columns next to each other in one wider buffer.
    bool disjoint(const Matrix &o) const
    {
        if (empty() || o.empty() || p + extent() <= o.p || o.p + o.extent() <= p) return true;
        if (pitch() != o.pitch() || rows == 1 || o.rows == 1) return false;
        const Matrix &a = p <= o.p ? *this : o, &b = p <= o.p ? o : *this;
        const uint64_t d = (b.p - a.p) % a.pitch();
        return a.row_bytes() <= d && d + b.row_bytes() <= a.pitch();
    }
};

constexpr int64_t kMostElements = int64_t(1) << 40;      // of a matrix, stride included

// what is read, if it is given
inline int check_read(const Matrix &m)
{
    if (m.none()) return HXT_OK;
    if (m.stride < 0) return HXT_EINVAL;
    if (m.p % uintptr_t(m.es)) return HXT_EALIGN;
    if (m.rows > 1 && m.stride > kMostElements / (m.rows - 1)) return HXT_EUNSUPPORTED;
    return HXT_OK;
}

// what is written
inline int check_write(const Matrix &m)
{
    const int rc = check_read(m);
    if (rc != HXT_OK || m.none()) return rc;
    return m.rows > 1 && m.stride < m.cols ? HXT_EINVAL : HXT_OK;
}

// ---- launches ----------------------------------------------------------------------------
// HIP takes fewer than 2^32 threads in a launch.  Calls launch(first, count) for `groups` workgroups of that many threads, in as many
// launches as they need; a run begins at a multiple of 8, so that workgroups go to the same XCDs as in one launch.
template <typename F>
inline void in_launches(uint64_t groups, uint32_t threads, F &&launch)
{
    const uint64_t most = 0xFFFFFFFFu / threads / 8 * 8;
    for (uint64_t first = 0; first < groups; first += most) launch(uint32_t(first), uint32_t(groups - first < most ? groups - first : most));
}

// ---- places in a packed buffer ---------------------------------------------------------
HXT_HD uint64_t packed_place(const ChunkGeom &g, ChunkAt at)
{
    const uint32_t slot = fast_div(at.chunk, g.div_k), lane = at.chunk - slot * g.k;
    return (uint64_t(lane) * g.q + (lane < g.r ? lane : g.r) + slot) * g.B + at.rem;
}

// ---- numbers (device) ------------------------------------------------------------------
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float bf16_to_f32(uint32_t bits) { return __uint_as_float(bits << 16); }

// Two values rounded to bf16, to nearest even (one instruction).
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi)
{
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{lo, hi}), b2));
}
__device__ __forceinline__ uint16_t bf16_of(float v) { return uint16_t(bf16x2(v, v)); }

// Four values rounded to e4m3, to nearest even; |values| < 464 or NaN.
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d)
{
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true));
}

// Elements of 16 bytes as binary32, and back.
template <typename T> struct Number;
template <> struct Number<uint16_t> {          // bf16
    static constexpr int V = 8;
    static __device__ __forceinline__ void widen(u32x4 v, float *f)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(v[i] << 16);
            f[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ u32x4 narrow(const float *f)
    {
        return u32x4{bf16x2(f[0], f[1]), bf16x2(f[2], f[3]), bf16x2(f[4], f[5]), bf16x2(f[6], f[7])};
    }
    static __device__ __forceinline__ uint16_t one(float f) { return bf16_of(f); }
};
template <> struct Number<uint32_t> {          // f32
    static constexpr int V = 4;
    static __device__ __forceinline__ void widen(u32x4 v, float *f)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
    }
    static __device__ __forceinline__ u32x4 narrow(const float *f)
    {
        return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    }
    static __device__ __forceinline__ uint32_t one(float f) { return __float_as_uint(f); }
};

// Totals over the 64 lanes of a wave, in every lane: steps inside rows of 16 lanes, then across them.
template <int CTRL, typename F>
__device__ __forceinline__ uint32_t dpp_step(uint32_t v, F &&f)
{
    return f(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), CTRL, 0xF, 0xF, false)));
}
template <typename F>
__device__ __forceinline__ uint32_t wave_total(uint32_t v, F &&f)       // f(v, 0) == v
{
    v = dpp_step<0x111>(v, f);        // row_shr 1, 2, 4, 8: lane 15 of a row has the row's total
    v = dpp_step<0x112>(v, f);
    v = dpp_step<0x114>(v, f);
    v = dpp_step<0x118>(v, f);
    v = dpp_step<0x142>(v, f);        // row_bcast 15, 31
    v = dpp_step<0x143>(v, f);
    return uint32_t(__builtin_amdgcn_readlane(int(v), 63));
}
__device__ __forceinline__ float wave_sum(float x)
{
    return __uint_as_float(wave_total(__float_as_uint(x), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x)
{
    return wave_total(x, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
__device__ __forceinline__ uint64_t wave_sum64(uint64_t v)       // the total in lane 63
{
    v = dpp_plus<0x111>(v);
    v = dpp_plus<0x112>(v);
    v = dpp_plus<0x114>(v);
    v = dpp_plus<0x118>(v);
    v = dpp_plus<0x142>(v);
    return dpp_plus<0x143>(v);
}

}  // namespace hxt

#endif
