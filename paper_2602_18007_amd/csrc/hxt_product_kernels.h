// Matrix products on the matrix cores (gfx950): device code of hxt_product.hip.
//
// out[m][n] = sum over the contraction index of P(m, .) * Q(n, .), tile by tile: a workgroup owns TM x TN results in
// registers and walks the contraction in steps of 128 bytes a row (64 bf16, 128 e4m3).  A step's two operand tiles lie in
// LDS, twice, so that the next step's loads run under this step's matrix instructions.
//
// An operand is either along (its rows are m or n, the contraction index is adjacent) or across (its rows are the contraction
// index: b in da = dz b, both factors in db = dz^T a), which the transposing LDS loads turn on the way into registers.
#ifndef HXT_PRODUCT_KERNELS_H
#define HXT_PRODUCT_KERNELS_H

#include "hxt_operators.h"

namespace hxt {

enum Factor { F_BF16 = 0, F_E4M3 = 1 };

struct Operand {
    const uint8_t *p;
    int64_t stride;               // bytes between rows
    uint32_t rows;                // m or n: outer extent of the products
    uint32_t depth;               // contraction extent
};

// What happens to a product before it is stored; see hxt_product_t.
struct Epilogue {
    uint32_t m, n;
    const float *m_scale, *n_scale;
    const uint16_t *bias;
    int act;
    const uint8_t *residual;      // of the output's type
    int64_t residual_stride;      // bytes, as the other strides
    uint8_t *pre;
    int64_t pre_stride;
    uint8_t *out;                 // rows of a tensor, or the packed buffer of a message of one tensor
    int64_t out_stride;
    bool out32, message;
    ChunkGeom g;
};

struct ProductArgs {
    Operand p, q;
    uint32_t tiles_m, tiles_n;
    uint32_t splits;              // parts of the contraction; > 1: partial sums go to work[split][m][n]
    uint32_t split_steps;         // steps of one part
    float *work;
    Epilogue e;
};

// ---- epilogue ---------------------------------------------------------------------------

__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }

// z/2 (1 + tanh u) is z * sigmoid(2u), which keeps its relative precision where tanh nears -1.
constexpr float kGelu2A = 1.5957691216057308f, kGeluB = 0.044715f;
__device__ __forceinline__ float activate(float z, int act)
{
    if (act == HXT_ACT_RELU) return z > 0 ? z : z * 0.0f;               // (0 times NaN stays NaN)
    if (act == HXT_ACT_SILU) return z * sigmoid(z);
    if (act == HXT_ACT_GELU) return z * sigmoid(kGelu2A * z * (1.0f + kGeluB * z * z));
    return z;
}

__device__ __forceinline__ float activate_grad(float z, int act)
{
    if (act == HXT_ACT_RELU) return z > 0 ? 1.0f : 0.0f;
    if (act == HXT_ACT_SILU) {
        const float s = sigmoid(z);
        return s * (1.0f + z * (1.0f - s));
    }
    if (act == HXT_ACT_GELU) {
        const float s = sigmoid(kGelu2A * z * (1.0f + kGeluB * z * z));
        const float t = s * (1.0f - s);                // 0 where z^2 may leave the range
        return t == 0 ? s : s + z * t * kGelu2A * (1.0f + 3.0f * kGeluB * z * z);
    }
    return 1.0f;
}

// W neighbouring elements as binary32, and back; the address is element aligned, the hardware takes it.
template <int W>
__device__ __forceinline__ void load_bf16(const uint8_t *p, float *f)
{
    uint16_t e[W];
    __builtin_memcpy(e, p, 2 * W);
#pragma unroll
    for (int i = 0; i < W; ++i) f[i] = bf16_to_f32(e[i]);
}

template <int W>
__device__ __forceinline__ void store_numbers(uint8_t *p, const float *f, bool f32)
{
    if (f32) {
        __builtin_memcpy(p, f, 4 * W);
        return;
    }
    uint32_t w[W / 2];
#pragma unroll
    for (int i = 0; i < W / 2; ++i) w[i] = bf16x2(f[2 * i], f[2 * i + 1]);
    __builtin_memcpy(p, w, 2 * W);
}

// Finishes results (m, n0 .. n0 + W - 1) from their sums.
template <int W>
__device__ __forceinline__ void finish(const Epilogue &e, uint32_t m, uint32_t n0, float *z)
{
    if (m >= e.m || n0 >= e.n) return;
    const uint32_t es = e.out32 ? 4 : 2, count = e.n - n0;
    const float ms = e.m_scale ? e.m_scale[m] : 1.0f;
    const uint64_t s = (uint64_t(m) * e.n + n0) * es;
    if (count >= W) {
        if (e.m_scale || e.n_scale) {
            float ns[W];
            if (e.n_scale) __builtin_memcpy(ns, e.n_scale + n0, 4 * W);
#pragma unroll
            for (int i = 0; i < W; ++i) z[i] *= e.n_scale ? ms * ns[i] : ms;
        }
        if (e.bias) {
            float b[W];
            load_bf16<W>(reinterpret_cast<const uint8_t *>(e.bias + n0), b);
#pragma unroll
            for (int i = 0; i < W; ++i) z[i] += b[i];
        }
        if (e.pre) store_numbers<W>(e.pre + m * e.pre_stride + 2 * size_t(n0), z, false);
        if (e.act != HXT_ACT_NONE) {
#pragma unroll
            for (int i = 0; i < W; ++i) z[i] = activate(z[i], e.act);
        }
        if (e.residual) {
            float r[W];
            const uint8_t *at = e.residual + m * e.residual_stride + size_t(n0) * es;
            if (e.out32) __builtin_memcpy(r, at, 4 * W);
            else load_bf16<W>(at, r);
#pragma unroll
            for (int i = 0; i < W; ++i) z[i] += r[i];
        }
        if (!e.message) {
            store_numbers<W>(e.out + m * e.out_stride + size_t(n0) * es, z, e.out32);
            return;
        }
        const ChunkAt at = chunk_at(e.g, s);
        if (at.rem + W * es <= e.g.B) {
            store_numbers<W>(e.out + packed_place(e.g, at), z, e.out32);
            return;
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if (uint32_t(i) >= count) continue;
            const uint32_t n = n0 + i;
            z[i] *= e.n_scale ? ms * e.n_scale[n] : ms;
            if (e.bias) z[i] += bf16_to_f32(e.bias[n]);
            if (e.pre) reinterpret_cast<uint16_t *>(e.pre + m * e.pre_stride)[n] = bf16_of(z[i]);
            z[i] = activate(z[i], e.act);
            if (e.residual) {
                const uint8_t *row = e.residual + m * e.residual_stride;
                z[i] += e.out32 ? reinterpret_cast<const float *>(row)[n] : bf16_to_f32(reinterpret_cast<const uint16_t *>(row)[n]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < W; ++i) {                 // the row's end, or a chunk border: element by element
        if (uint32_t(i) >= count) continue;
        uint8_t *at = e.message ? e.out + packed_place(e.g, chunk_at(e.g, s + i * es)) : e.out + m * e.out_stride + size_t(n0 + i) * es;
        if (e.out32) *reinterpret_cast<float *>(at) = z[i];
        else *reinterpret_cast<uint16_t *>(at) = bf16_of(z[i]);
    }
}

// Zeros between a message's last element and the end of its stream.
__device__ __forceinline__ void pad_message(const Epilogue &e)
{
    const uint64_t bytes = uint64_t(e.m) * e.n * (e.out32 ? 4 : 2), end = (bytes + 255) & ~uint64_t(255);
    for (uint64_t s = bytes + threadIdx.x; s < end; s += blockDim.x) e.out[packed_place(e.g, chunk_at(e.g, s))] = 0;
}

// ---- operand tiles in LDS ------------------------------------------------------------------
constexpr int kStep = 128;        // bytes of a row per step, of operands along; across: kStep / 2 rows

// One operand's tile: T rows of m or n.
//   along:  T rows of 128 bytes; 16-byte piece c of row r lies at place c ^ turn(r), so that the 16 rows that a fragment load
//           touches at once lie in 16 different places of the banks' 256 bytes (neighbouring rows are 128 bytes apart)
//   across: 64 rows (contraction) of 2 T bytes; piece c of row k lies at place c ^ turn(k), two by two (a transposing
//           load takes 32 bytes of each of 8 rows per half wave)
template <int T, bool ACROSS, int ES, int THREADS>
struct TileOf {
    static constexpr int BYTES = T * kStep;
    static constexpr int PIECES = BYTES / 16, EACH = (PIECES + THREADS - 1) / THREADS;
    static constexpr int LINE = ACROSS ? T / 8 : 8;              // pieces of an LDS row
    static constexpr int DEPTH = ACROSS ? 64 : kStep / ES;       // contraction elements of a step

    static __device__ __forceinline__ int turn(int row)
    {
        if (ACROSS) return (((row & 3) | ((row >> 3) & 1) << 2) << 1) & (LINE - 1);
        return (row >> 1) & 7;
    }

    // Piece `id` of the tile: its row, and the first byte of that row it holds.
    static __device__ __forceinline__ void piece(int id, int &row, int &byte)
    {
        row = id / LINE;
        byte = ((id % LINE) ^ turn(row)) * 16;
    }

    // Straight from memory into LDS, 16 bytes a lane: the whole step lies inside the contraction, rows past the operand's end
    // repeat its last one (across: columns the last 8), what comes of them is never stored.
    static __device__ __forceinline__ void load_direct(const Operand &o, uint32_t row0, uint32_t step, uint8_t *lds)
    {
        const uint8_t *base = ACROSS ? o.p + int64_t(step) * DEPTH * o.stride : o.p + int64_t(step) * kStep + int64_t(row0) * o.stride;
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int id = j * THREADS + int(threadIdx.x);
            if (PIECES % THREADS && id >= PIECES) continue;
            int row, byte;
            piece(id, row, byte);
            uint64_t at;
            if (ACROSS) at = uint64_t(row) * uint64_t(o.stride) + min(2 * row0 + uint32_t(byte), 2 * o.rows - 16);
            else at = uint64_t(min(uint32_t(row), o.rows - 1 - row0)) * uint64_t(o.stride) + uint32_t(byte);
            uint8_t *to = lds + (j * THREADS + __builtin_amdgcn_readfirstlane(int(threadIdx.x) & ~63)) * 16;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(base + at),
                                             (__attribute__((address_space(3))) void *)to, 16, 0, 0);
        }
    }

    // Through registers: any alignment, zeros outside the operand.
    static __device__ __forceinline__ void load_any(const Operand &o, uint32_t row0, uint32_t step, uint8_t *lds)
    {
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int id = j * THREADS + int(threadIdx.x);
            if (PIECES % THREADS && id >= PIECES) continue;
            int row, byte;
            piece(id, row, byte);
            const uint64_t r = ACROSS ? uint64_t(step) * DEPTH + row : uint64_t(row0) + row;
            const uint64_t c = ACROSS ? row0 + byte / ES : uint64_t(step) * DEPTH + byte / ES;
            const uint64_t rows = ACROSS ? o.depth : o.rows, cols = ACROSS ? o.rows : o.depth;
            u32x4 v = u32x4{0, 0, 0, 0};
            if (r < rows && c < cols) {
                const uint8_t *at = o.p + r * o.stride + c * ES;
                if (c + 16 / ES <= cols) {
                    v = load16_any<false>(at);
                } else {
                    using E = std::conditional_t<ES == 1, uint8_t, uint16_t>;
                    E e[16 / ES];
#pragma unroll
                    for (uint32_t i = 0; i < 16 / ES; ++i) e[i] = c + i < cols ? reinterpret_cast<const E *>(at)[i] : E(0);
                    v = __builtin_bit_cast(u32x4, e);
                }
            }
            *reinterpret_cast<u32x4 *>(lds + id * 16) = v;
        }
    }

    // Fragment f of those that start at tile row `first`: for half h of the step, lane l's 16 bytes are row l % 16's, contraction
    // elements (4h + l / 16) * 8 .. + 7 (of e4m3: * 16 .. + 15).
    static __device__ __forceinline__ u32x4 fragment(const uint8_t *lds, int first, int f, int h)
    {
        const int l = int(threadIdx.x) & 63, r = l & 15, q = l >> 4;
        if constexpr (!ACROSS) {
            const int row = first + 16 * f + r;
            return *reinterpret_cast<const u32x4 *>(lds + row * kStep + (((4 * h + q) ^ turn(row)) * 16));
        } else {
            typedef short s4 __attribute__((ext_vector_type(4)));
            u32x4 v;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int k = 32 * h + 8 * q + 4 * j + (r >> 2);
                const int col = first + 16 * f + 4 * (r & 3);
                const uint8_t *at = lds + k * (2 * T) + (((col >> 3) ^ turn(k)) * 16) + (col & 4) * 2;
                const s4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)at);
                const u32x2 w = __builtin_bit_cast(u32x2, x);
                v[2 * j] = w.x;
                v[2 * j + 1] = w.y;
            }
            return v;
        }
    }
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// Tiles in an order that keeps neighbours on one XCD's L2: workgroups go to the eight XCDs in turn, so each XCD takes a run of
// consecutive tiles, and consecutive tiles are blocks 8 tiles high.
__device__ __forceinline__ void tile_at(uint32_t id, uint32_t all, uint32_t tm, uint32_t tn, uint32_t &i, uint32_t &j)
{
    const uint32_t xcd = id & 7, each = all >> 3, more = all & 7;
    uint32_t t = xcd * each + min(xcd, more) + (id >> 3);
    const uint32_t per_band = 8 * tn, band = t / per_band;
    t -= band * per_band;
    const uint32_t high = min(8u, tm - band * 8);
    i = band * 8 + t % high;
    j = t / high;
}

// Rows of a wave's results that are turned in LDS at a time, and the LDS of a workgroup.
HXT_HD constexpr int epilogue_rows(int tm, int tn, int wm, int wn)
{
    int rows = tm / wm;
    while (wm * wn * rows * (tn / wn + 4) * 4 > 147456) rows /= 2;
    return rows;
}
HXT_HD constexpr int product_lds(int tm, int tn, int wm, int wn)
{
    const int loop = 2 * (tm + tn) * kStep, end = wm * wn * epilogue_rows(tm, tn, wm, wn) * (tn / wn + 4) * 4;
    return loop > end ? loop : end;
}

// Four neighbours of one part's sums.
__device__ __forceinline__ void store_part(float *part, uint32_t rows, uint32_t cols, uint32_t m, uint32_t n, f32x4 v)
{
    if (m >= rows || n >= cols) return;
    typedef f32x4 f32x4_any __attribute__((aligned(4)));
    float *at = part + size_t(m) * cols + n;
    if (n + 4 <= cols) {
        *reinterpret_cast<f32x4_any *>(at) = v;
        return;
    }
    at[0] = v.x;
    if (n + 1 < cols) at[1] = v.y;
    if (n + 2 < cols) at[2] = v.z;
}

template <Factor F, int TM, int TN, int WM, int WN, bool P_ACROSS, bool Q_ACROSS, bool DIRECT>
__global__ __launch_bounds__(64 * WM * WN) void k_product(ProductArgs a)
{
    constexpr int THREADS = 64 * WM * WN, ES = F == F_E4M3 ? 1 : 2;
    constexpr int RM = TM / WM / 16, RN = TN / WN / 16;
    using TileP = TileOf<TM, P_ACROSS, ES, THREADS>;
    using TileQ = TileOf<TN, Q_ACROSS, ES, THREADS>;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    constexpr int BUFFER = TileP::BYTES + TileQ::BYTES;

    const uint32_t tiles = a.tiles_m * a.tiles_n;
    const uint32_t split = a.splits > 1 ? blockIdx.x / tiles : 0;
    uint32_t ti, tj;
    tile_at(blockIdx.x - split * tiles, tiles, a.tiles_m, a.tiles_n, ti, tj);
    const uint32_t m0 = ti * TM, n0 = tj * TN;
    const int wave = int(threadIdx.x) >> 6, wm = wave / WN, wn = wave % WN;
    const uint32_t depth = a.p.depth, all_steps = (depth + TileP::DEPTH - 1) / TileP::DEPTH;
    const uint32_t first = split * a.split_steps, last = min(all_steps, first + a.split_steps);
    const uint32_t whole = depth / TileP::DEPTH;                   // steps that lie inside the contraction

    f32x4 acc[RM][RN];
#pragma unroll
    for (int i = 0; i < RM; ++i)
#pragma unroll
        for (int j = 0; j < RN; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

    auto load = [&](uint32_t step, uint8_t *to) {
        if (DIRECT && step < whole) {
            TileP::load_direct(a.p, m0, step, to);
            TileQ::load_direct(a.q, n0, step, to + TileP::BYTES);
        } else {
            TileP::load_any(a.p, m0, step, to);
            TileQ::load_any(a.q, n0, step, to + TileP::BYTES);
        }
    };
    if (first < last) load(first, lds);
    for (uint32_t step = first; step < last; ++step) {
        uint8_t *now = lds + ((step - first) & 1) * BUFFER, *next = lds + ((step - first + 1) & 1) * BUFFER;
        // this step's tiles have arrived, and all waves have read the last step's
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (step + 1 < last) load(step + 1, next);
        u32x4 p[2][RM], q[2][RN];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < RM; ++i) p[h][i] = TileP::fragment(now, wm * (TM / WM), i, h);
#pragma unroll
            for (int j = 0; j < RN; ++j) q[h][j] = TileQ::fragment(now + TileP::BYTES, wn * (TN / WN), j, h);
            if constexpr (F == F_BF16) {
#pragma unroll
                for (int i = 0; i < RM; ++i)
#pragma unroll
                    for (int j = 0; j < RN; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, q[h][j]), __builtin_bit_cast(bf16x8, p[h][i]),
                                                                            acc[i][j], 0, 0, 0);
            }
        }
        if constexpr (F == F_E4M3) {
            auto both = [](u32x4 lo, u32x4 hi) {
                return i32x8{int(lo.x), int(lo.y), int(lo.z), int(lo.w), int(hi.x), int(hi.y), int(hi.z), int(hi.w)};
            };
#pragma unroll
            for (int i = 0; i < RM; ++i)
#pragma unroll
                for (int j = 0; j < RN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(both(q[0][j], q[1][j]), both(p[0][i], p[1][i]), acc[i][j], 0, 0, 0, 0,
                                                                                 0, 0);
        }
    }

    // Lane l has, of fragment (i, j), row 16i + l % 16 and columns 16j + 4 (l / 16) .. + 3.  Every wave turns its results in LDS, ROUND
    // rows at a time, so that lanes finish 8 neighbours each and rows are stored in one piece (the rows in LDS are 16 bytes apart in
    // the banks).
    __syncthreads();                                     // all waves are through with the operand tiles
    constexpr int COLS = TN / WN, ROWS = TM / WM, ROUND = epilogue_rows(TM, TN, WM, WN), PITCH = COLS + 4, RUNS = COLS / 8;
    float *mine = reinterpret_cast<float *>(lds) + wave * (ROUND * PITCH);
    const int l = int(threadIdx.x) & 63;
#pragma unroll
    for (int r0 = 0; r0 < ROWS; r0 += ROUND) {
#pragma unroll
        for (int i = 0; i < ROUND / 16; ++i)
#pragma unroll
            for (int j = 0; j < RN; ++j)
                *reinterpret_cast<f32x4 *>(mine + (16 * i + (l & 15)) * PITCH + 16 * j + 4 * (l >> 4)) = acc[r0 / 16 + i][j];
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int at = l; at < ROUND * RUNS; at += 64) {
            const int row = at / RUNS, col = at % RUNS * 8;
            const f32x4 lo = *reinterpret_cast<const f32x4 *>(mine + row * PITCH + col), hi = *reinterpret_cast<const f32x4 *>(mine + row * PITCH + col + 4);
            const uint32_t m = m0 + wm * ROWS + r0 + row, n = n0 + wn * COLS + col;
            if (a.splits > 1) {
                float *part = a.work + size_t(split) * a.e.m * a.e.n;
                store_part(part, a.e.m, a.e.n, m, n, lo);
                store_part(part, a.e.m, a.e.n, m, n + 4, hi);
            } else {
                float z[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
                finish<8>(a.e, m, n, z);
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
    if (a.splits <= 1 && a.e.message && blockIdx.x == 0) pad_message(a.e);
}

// Sums the parts of a product in their order and finishes it, 4 neighbours a thread.
__global__ __launch_bounds__(256) void k_product_join(const float *__restrict__ work, uint32_t splits, Epilogue e)
{
    const uint64_t groups = (e.n + 3) / 4, id = uint64_t(blockIdx.x) * 256 + threadIdx.x;
    if (e.message && blockIdx.x == 0) pad_message(e);
    if (id >= groups * e.m) return;
    const uint32_t m = uint32_t(id / groups), n0 = 4 * uint32_t(id - m * groups);
    float z[4] = {0, 0, 0, 0};
    const size_t part = size_t(e.m) * e.n;
    const float *at = work + size_t(m) * e.n + n0;
    for (uint32_t s = 0; s < splits; ++s, at += part) {
        if (n0 + 4 <= e.n) {
            float v[4];
            __builtin_memcpy(v, at, 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) z[i] += v[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n0 + i < e.n) z[i] += at[i];
        }
    }
    finish<4>(e, m, n0, z);
}

// ---- dz and the bias gradient ----------------------------------------------------------------
struct DzArgs {
    uint32_t m, n;
    const uint8_t *dc, *pre;
    int64_t dc_stride, pre_stride, dz_stride;      // bytes
    uint8_t *dz;                                   // nullptr: not stored
    int act;
    float *partial;                                // [gridDim.y][n] column sums, or nullptr
};

// 64 lanes x 8 columns, 4 waves on every fourth row of a band; a band's column sums go to partial.
__global__ __launch_bounds__(256) void k_product_dz(DzArgs a)
{
    __shared__ float part[4][512];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n0 = blockIdx.x * 512 + lane * 8;
    float sum[8] = {};
    if (n0 < a.n) {
        const uint32_t count = min(8u, a.n - n0);
        for (uint64_t m = uint64_t(blockIdx.y) * 4 + wave; m < a.m; m += uint64_t(gridDim.y) * 4) {
            float d[8], z[8];
            const uint8_t *from = a.dc + m * a.dc_stride + 2 * size_t(n0), *pre = a.pre + m * a.pre_stride + 2 * size_t(n0);
            uint8_t *to = a.dz + m * a.dz_stride + 2 * size_t(n0);
            if (count == 8) {
                load_bf16<8>(from, d);
                if (a.act != HXT_ACT_NONE) {
                    load_bf16<8>(pre, z);
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[i] *= activate_grad(z[i], a.act);
                }
                if (a.dz) store_numbers<8>(to, d, false);
            } else {
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i) {
                    d[i] = 0;
                    if (i >= count) continue;
                    d[i] = bf16_to_f32(reinterpret_cast<const uint16_t *>(from)[i]);
                    if (a.act != HXT_ACT_NONE) d[i] *= activate_grad(bf16_to_f32(reinterpret_cast<const uint16_t *>(pre)[i]), a.act);
                    if (a.dz) reinterpret_cast<uint16_t *>(to)[i] = bf16_of(d[i]);
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += d[i];
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) part[wave][lane * 8 + i] = sum[i];
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < 512 && blockIdx.x * 512 + c < a.n; c += 256)
        a.partial[size_t(blockIdx.y) * a.n + blockIdx.x * 512 + c] = (part[0][c] + part[1][c]) + (part[2][c] + part[3][c]);
}

// Column sums of `bands` rows, added to `add`.
__global__ __launch_bounds__(256) void k_product_dbias(const float *__restrict__ partial, uint32_t bands, uint32_t n, const float *add, float *dbias)
{
    const uint32_t c = blockIdx.x * 256 + threadIdx.x;
    if (c >= n) return;
    float s = 0;
    for (uint32_t b = 0; b < bands; ++b) s += partial[size_t(b) * n + c];
    dbias[c] = add ? add[c] + s : s;
}

}  // namespace hxt

#endif
