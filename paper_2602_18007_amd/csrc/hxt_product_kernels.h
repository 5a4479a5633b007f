// Matrix products on the matrix cores (gfx950): device code of hxt_product.hip.
//
// out[m][n] = sum over the contraction index of P(m, .) * Q(n, .), tile by tile: a workgroup owns TM x TN results in
// registers and walks the contraction in steps of 128 bytes a row (64 bf16, 128 e4m3).  A step's two operand tiles lie in
// LDS, twice, so that the next step's loads run under this step's matrix instructions.
//
// Bound by the matrix cores, at the clock that the power limit leaves: 4096 x 4096 x 14336 bf16 in 256 x 256 tiles 341 to 365 us on one card
// and another (1320 to 1410 TFLOP/s); the matrix pipes are busy for 68% of the cycles, at 2.04 GHz, and with operands of zeros 63% at 2.43 GHz
// (303 us); 8192 x 8192 x 8192 745, of zeros 616.  16 x 16 x 32 instructions rather than 32 x 32 x 16, whose accumulators'
// traffic costs power (zeros 599, data 821 us).
//
// An operand is either along (its rows are m or n, the contraction index is adjacent) or across (its rows are the contraction
// index: b in da = dz b, both factors in db = dz^T a), which the transposing LDS loads turn on the way into registers.
#ifndef HXT_PRODUCT_KERNELS_H
#define HXT_PRODUCT_KERNELS_H

#include "hxt_operators.h"
#include "hxt_product_rules.h"

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
    uint32_t n_first;             // column of the first tile
    uint32_t first_group;         // number of the launch's first workgroup
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
    if (act == HXT_ACT_RELU) return z <= 0 ? 0.0f : z;                  // (NaN is not <= 0 and stays; minus infinity is)
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

// z * s * t, where neither s * t nor z * s has to lie in binary32's range (hxt_norm's scales go down to 2^-126): s's exponent is added
// last.  (A sum of 8-bit products is 0 or between 2^-18 and 2^42.)
__device__ __forceinline__ float scaled(float z, float s, float t)
{
    return __builtin_ldexpf(z * (__builtin_amdgcn_frexp_mantf(s) * t), __builtin_amdgcn_frexp_expf(s));
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
            for (int i = 0; i < W; ++i) z[i] = scaled(z[i], ms, e.n_scale ? ns[i] : 1.0f);
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
            if (e.m_scale || e.n_scale) z[i] = scaled(z[i], ms, e.n_scale ? e.n_scale[n] : 1.0f);
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
typedef int i32x4 __attribute__((ext_vector_type(4)));

// One operand's tile: T rows of m or n, in LDS as the direct loads leave it, in blocks of 1024 bytes that one wave writes.
//   along:  T rows of 128 bytes; 16-byte piece c of row r lies at place c ^ turn(r), so that the 16 rows that a fragment load
//           touches at once lie in 16 different places of the banks' 256 bytes (neighbouring rows are 128 bytes apart)
//   across: 64 rows (contraction) of 2 T bytes, blocks 32 bytes further apart than they are long.  A transposing load takes 32
//           bytes of rows 8q + 4j + s for all q and s below 4: these lie in 16 different blocks, 8 of which (half a wave's) share
//           no bank; rows that differ in j (and with T = 128 in the step's half) share a block.
// Either way the places of a wave's fragments are constant offsets from one address per lane (along: from one per half).
template <int T, bool ACROSS, int ES, int THREADS>
struct TileOf {
    static constexpr int PIECES = T * kStep / 16, EACH = (PIECES + THREADS - 1) / THREADS;
    static constexpr int BLOCK = ACROSS ? 1056 : 1024, BYTES = PIECES / 64 * BLOCK;
    static constexpr int DEPTH = ACROSS ? 64 : kStep / ES;       // contraction elements of a step
    static_assert(!ACROSS || ((T == 128 || T == 256) && ES == 2));

    static __device__ __forceinline__ int turn(int row) { return (row >> 1) & 7; }

    // Piece `id` of the tile: its row, and the first byte of that row it holds.
    static __device__ __forceinline__ void piece(int id, int &row, int &byte)
    {
        if constexpr (ACROSS) {
            const int block = id >> 6, at = (id & 63) * 16, in = at / (2 * T);
            const int half = T == 256 ? block >> 4 : in >> 1;
            row = 32 * half + 8 * ((block >> 2) & 3) + 4 * (in & 1) + (block & 3);
            byte = at % (2 * T);
        } else {
            row = id / 8;
            byte = ((id % 8) ^ turn(row)) * 16;
        }
    }
    static __device__ __forceinline__ int place(int id) { return (id >> 6) * BLOCK + (id & 63) * 16; }

    // Straight from memory into LDS, 16 bytes a lane: steps that lie inside the contraction.  Rows past the operand's end repeat its
    // last one (across: columns the last 8), what comes of them is never stored.  A lane's offsets are the same for every step;
    // the base moves.
    static __device__ __forceinline__ void offsets(const Operand &o, uint32_t row0, uint32_t (&at)[EACH])
    {
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            int row, byte;
            piece(j * THREADS + int(threadIdx.x), row, byte);
            if (ACROSS) at[j] = uint32_t(row) * uint32_t(o.stride) + min(2 * row0 + uint32_t(byte), 2 * o.rows - 16);
            else at[j] = min(uint32_t(row), o.rows - 1 - row0) * uint32_t(o.stride) + uint32_t(byte);
        }
    }
    // The descriptor of a step's base, and load j of the EACH that bring a tile.  The load is written out because the compiler, where
    // it knows of loads into LDS, waits for all of them before every transposing read; the kernel's own waits and barriers
    // order them.  It has no register for a result; m0 says where the wave's block goes, 16 bytes a lane.
    static __device__ __forceinline__ i32x4 descriptor(const Operand &o, uint32_t row0, uint32_t step)
    {
        const uint64_t base = reinterpret_cast<uint64_t>(o.p) + (ACROSS ? uint64_t(step) * DEPTH * uint64_t(o.stride)
                                                                        : uint64_t(step) * kStep + uint64_t(row0) * uint64_t(o.stride));
        return i32x4{__builtin_amdgcn_readfirstlane(int(uint32_t(base))), __builtin_amdgcn_readfirstlane(int(uint32_t(base >> 32) & 0xFFFFu)), -1, 0x00020000};
    }
    static __device__ __forceinline__ void load_direct(i32x4 from, const uint32_t (&at)[EACH], uint32_t lds, int j)
    {
        if (PIECES % THREADS && j * THREADS + int(threadIdx.x) >= PIECES) return;
        const uint32_t to = __builtin_amdgcn_readfirstlane(int(lds + (threadIdx.x >> 6) * BLOCK)) + j * (THREADS / 64) * BLOCK;
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"          // (m0 is reserved; naming it keeps the compiler from carrying a value of its own past here)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(at[j]), "s"(from) : "memory", "m0");
#pragma clang diagnostic pop
    }

    // Through registers: any alignment, zeros outside the operand.
    static __device__ __forceinline__ void fetch(const Operand &o, uint32_t row0, uint32_t step, u32x4 (&v)[EACH])
    {
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            int row, byte;
            piece(j * THREADS + int(threadIdx.x), row, byte);
            const uint64_t r = ACROSS ? uint64_t(step) * DEPTH + row : uint64_t(row0) + row;
            const uint64_t c = ACROSS ? row0 + byte / ES : uint64_t(step) * DEPTH + byte / ES;
            const uint64_t rows = ACROSS ? o.depth : o.rows, cols = ACROSS ? o.rows : o.depth;
            v[j] = u32x4{0, 0, 0, 0};
            if (r < rows && c < cols) {
                const uint8_t *at = o.p + r * o.stride + c * ES;
                if (c + 16 / ES <= cols) {
                    v[j] = load16_any<false>(at);
                } else {
                    using E = std::conditional_t<ES == 1, uint8_t, uint16_t>;
                    E e[16 / ES];
#pragma unroll
                    for (uint32_t i = 0; i < 16 / ES; ++i) e[i] = c + i < cols ? reinterpret_cast<const E *>(at)[i] : E(0);
                    v[j] = __builtin_bit_cast(u32x4, e);
                }
            }
        }
    }
    static __device__ __forceinline__ void put(uint8_t *lds, const u32x4 (&v)[EACH])
    {
#pragma unroll
        for (int j = 0; j < EACH; ++j)
            if (!(PIECES % THREADS) || j * THREADS + int(threadIdx.x) < PIECES) *reinterpret_cast<u32x4 *>(lds + place(j * THREADS + int(threadIdx.x))) = v[j];
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
                // row 32h + 8q + 4j + r / 4, columns first + 16f + 4 (r % 4) .. + 3
                const uint8_t *at = lds + (4 * q + (r >> 2)) * BLOCK + (4 * (r & 3) + first) * 2 + 32 * f +
                                    (T == 256 ? 16 * h * BLOCK + j * 512 : (2 * h + j) * 256);
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
// consecutive tiles, and consecutive tiles are blocks 8 tiles high (bf16 4096 x 4096 x 14336 341 us, 4 high 342, 16 high 355;
// 4096 x 14336 x 4096 381, 377 and 404, of 8 bits 204, 200 and 218).
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
HXT_HD constexpr int product_lds(int tm, int tn, int wm, int wn, bool p_across, bool q_across)
{
    const int loop = 2 * (tm * kStep / 1024 * (p_across ? 1056 : 1024) + tn * kStep / 1024 * (q_across ? 1056 : 1024)), end = wm * wn * epilogue_rows(tm, tn, wm, wn) * (tn / wn + 4) * 4;
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

// 16 x 16 results: c += of DEEP times 64 bytes a row; e4m3's instruction takes 128.
template <Factor F, int DEEP>
__device__ __forceinline__ void multiply_pieces(f32x4 &c, const u32x4 (&q)[DEEP], const u32x4 (&p)[DEEP])
{
    if constexpr (F == F_BF16) {
#pragma unroll
        for (int h = 0; h < DEEP; ++h) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, q[h]), __builtin_bit_cast(bf16x8, p[h]), c, 0, 0, 0);
    } else {
        static_assert(DEEP == 2);
        auto both = [](const u32x4 (&v)[2]) { return i32x8{int(v[0].x), int(v[0].y), int(v[0].z), int(v[0].w), int(v[1].x), int(v[1].y), int(v[1].z), int(v[1].w)}; };
        c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(both(q), both(p), c, 0, 0, 0, 0, 0, 0);
    }
}

// A wave's ROWS x COLS results from LDS to where they go, 8 neighbours a lane: (m, n) is the first.
template <int ROWS, int COLS, int PITCH>
__device__ __forceinline__ void finish_rows(const ProductArgs &a, uint32_t split, const float *mine, uint32_t m0, uint32_t n0)
{
    constexpr int RUNS = COLS / 8;
#pragma unroll 1
    for (int at = int(threadIdx.x) & 63; at < ROWS * RUNS; at += 64) {
        const int row = at / RUNS, col = at % RUNS * 8;
        const f32x4 lo = *reinterpret_cast<const f32x4 *>(mine + row * PITCH + col), hi = *reinterpret_cast<const f32x4 *>(mine + row * PITCH + col + 4);
        const uint32_t m = m0 + row, n = n0 + col;
        if (a.splits > 1) {
            float *part = a.work + size_t(split) * a.e.m * a.e.n;
            store_part(part, a.e.m, a.e.n, m, n, lo);
            store_part(part, a.e.m, a.e.n, m, n + 4, hi);
        } else {
            float z[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            finish<8>(a.e, m, n, z);
        }
    }
}

// Calls f<0>, f<1>, .. f<N - 1>.
template <int N, int AT = 0, typename F>
__device__ __forceinline__ void each(F &&f)
{
    if constexpr (AT < N) {
        f.template operator()<AT>();
        each<N, AT + 1>(f);
    }
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

    const uint32_t tiles = a.tiles_m * a.tiles_n, group = a.first_group + blockIdx.x;
    const uint32_t split = a.splits > 1 ? group / tiles : 0;
    uint32_t ti, tj;
    tile_at(group - split * tiles, tiles, a.tiles_m, a.tiles_n, ti, tj);
    const uint32_t m0 = ti * TM, n0 = a.n_first + tj * TN;
    const int wave = int(threadIdx.x) >> 6, wm = wave / WN, wn = wave % WN;
    const uint32_t depth = a.p.depth, all_steps = (depth + TileP::DEPTH - 1) / TileP::DEPTH;
    const uint32_t first = split * a.split_steps, last = min(all_steps, first + a.split_steps);
    const uint32_t whole = depth / TileP::DEPTH;                   // steps that lie inside the contraction

    f32x4 acc[RM][RN];
#pragma unroll
    for (int i = 0; i < RM; ++i)
#pragma unroll
        for (int j = 0; j < RN; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

    // A step is PHASES parts of its matrix instructions.  While one runs, the fragments of the next are read: bf16 by halves of
    // the step's depth and of the wave's rows, e4m3 (whose instructions take the whole depth) by quarters of the rows.
    constexpr int PHASES = 4, HALVES = F == F_BF16 ? 2 : 1, PARTS = PHASES / HALVES, PI = RM / PARTS, DEEP = 2 / HALVES;
    static_assert(RM % PARTS == 0);
    u32x4 p[2][PI][DEEP], q[HALVES][RN][DEEP];
    const int p_first = wm * (TM / WM), q_first = wn * (TN / WN);
    auto read_p = [&]<int PH, int I, int D>(const uint8_t *from, u32x4 (&to)[PI][DEEP]) {
        to[I][D] = TileP::fragment(from, p_first, PH % PARTS * PI + I, PH / PARTS + D);
    };
    auto read_q = [&]<int PH, int J, int D>(const uint8_t *from, u32x4 (&to)[RN][DEEP]) {
        to[J][D] = TileQ::fragment(from + TileP::BYTES, q_first, J, PH / PARTS + D);
    };
    auto multiply = [&]<int PH, int I, int J>(const u32x4 (&pp)[PI][DEEP], const u32x4 (&qq)[RN][DEEP]) {
        multiply_pieces<F>(acc[PH % PARTS * PI + I][J], qq[J], pp[I]);
    };
    constexpr int READS_P = PI * DEEP, READS_Q = RN * DEEP, MATRIX = PI * RN, LOADS = TileP::EACH + TileQ::EACH;
    uint32_t step = first;
    if constexpr (DIRECT) {
        const uint32_t steps = min(last, whole) > first ? min(last, whole) - first : 0;
        uint32_t at_p[TileP::EACH], at_q[TileQ::EACH];
        TileP::offsets(a.p, m0, at_p);
        TileQ::offsets(a.q, n0, at_q);
        // The eight XCDs begin at eighths of the contraction: in step they would ask the same memory channels for the same columns
        // (4096 x 4096 x 14336 362 -> 352 us, 8192 x 8192 x 8192 802 -> 767).
        const uint32_t begin = (blockIdx.x & 7) * (steps >> 3);
        const uint32_t lds0 = uint32_t(uintptr_t((__attribute__((address_space(3))) uint8_t *)lds));
        i32x4 from_p, from_q;
        auto aim = [&](uint32_t s) {                     // at step s's tiles
            s += begin;
            if (s >= steps) s -= steps;
            from_p = TileP::descriptor(a.p, m0, first + s);
            from_q = TileQ::descriptor(a.q, n0, first + s);
        };
        auto load = [&]<int L>(uint32_t to) {
            if constexpr (L < TileP::EACH) TileP::load_direct(from_p, at_p, to, L);
            else TileQ::load_direct(from_q, at_q, to + TileP::BYTES, L - TileP::EACH);
        };
        auto read = [&]<int PH, int U, int SET>(const uint8_t *from) {       // unit U of what phase PH needs
            if constexpr (U < READS_P) read_p.template operator()<PH, U / DEEP, U % DEEP>(from, p[PH & 1]);
            else read_q.template operator()<PH, (U - READS_P) / DEEP, (U - READS_P) % DEEP>(from, q[SET]);
        };
        if (steps) {
            aim(0);
            each<LOADS>([&]<int L>() { load.template operator()<L>(lds0); });
            if (steps > 1) {
                aim(1);
                each<LOADS>([&]<int L>() { load.template operator()<L>(lds0 + BUFFER); });
            }
            __builtin_amdgcn_s_waitcnt(0);
            __syncthreads();
            each<READS_P + READS_Q>([&]<int U>() { read.template operator()<0, U, 0>(lds); });
        }
        // One step, whose tiles are in buffer PAR.  INNER: two more follow, so that nothing has to be asked and the schedule is one
        // piece: between two matrix instructions few reads from LDS and loads, so that none of them holds up the next.
        auto one = [&]<int PAR, bool INNER>(uint32_t s) {
            const uint8_t *now = lds + PAR * BUFFER, *next = lds + (1 - PAR) * BUFFER;
            each<PHASES>([&]<int PH>() {
                constexpr bool TURN = PH + 1 == PHASES;
                constexpr int SET = PH / PARTS, NEXT = (PH + 1) % PHASES, AFTER = NEXT / PARTS;
                constexpr bool NEW_Q = NEXT % PARTS == 0, IN_PLACE = NEW_Q && AFTER == SET;
                const bool go_on = INNER || !TURN || s + 1 < steps, more = TURN && (INNER || s + 2 < steps);
                const uint8_t *from = TURN ? next : now;
                if constexpr (TURN) {
                    if (more) aim(s + 2);
                    // all waves have what they need of this step's tiles, and the next step's have arrived
                    if (go_on) {
                        __builtin_amdgcn_s_waitcnt(0);
                        __syncthreads();
                    }
                }
                if (!INNER) {
                    if (go_on) each<READS_P>([&]<int U>() { read.template operator()<NEXT, U, AFTER>(from); });
                    if (NEW_Q && !IN_PLACE && go_on) each<READS_Q>([&]<int U>() { read.template operator()<NEXT, READS_P + U, AFTER>(from); });
                    if (more) each<LOADS>([&]<int L>() { load.template operator()<L>(lds0 + PAR * BUFFER); });
                }
                __builtin_amdgcn_sched_barrier(0);
                // column by column of the wave's results, so that a q fragment is free PI instructions later
                each<MATRIX>([&]<int M>() {
                    if constexpr (INNER) {
                        constexpr int READS = READS_P + (NEW_Q && !IN_PLACE ? READS_Q : 0), EARLY = IN_PLACE ? MATRIX / 2 : MATRIX * 3 / 4;
                        constexpr int LO = M < EARLY ? READS * M / EARLY : READS, HI = M + 1 < EARLY ? READS * (M + 1) / EARLY : READS;
                        each<HI - LO>([&]<int U>() { read.template operator()<NEXT, LO + U, AFTER>(from); });
                        if constexpr (IN_PLACE && M > 0 && M % PI == 0)
                            each<DEEP>([&]<int U>() { read.template operator()<NEXT, READS_P + (M / PI - 1) * DEEP + U, AFTER>(from); });
                        if constexpr (TURN) {
                            constexpr int L0 = LOADS * M / MATRIX, L1 = LOADS * (M + 1) / MATRIX;
                            each<L1 - L0>([&]<int L>() { load.template operator()<L0 + L>(lds0 + PAR * BUFFER); });
                        }
                    }
                    multiply.template operator()<PH, M % PI, M / PI>(p[PH & 1], q[SET]);
                    __builtin_amdgcn_sched_barrier(0);
                });
                if constexpr (INNER && IN_PLACE) each<DEEP>([&]<int U>() { read.template operator()<NEXT, READS_P + (RN - 1) * DEEP + U, AFTER>(from); });
                if (!INNER && IN_PLACE && go_on) each<READS_Q>([&]<int U>() { read.template operator()<NEXT, READS_P + U, AFTER>(from); });
            });
        };
        uint32_t s = 0;
        for (; s + 3 < steps; s += 2) {
            one.template operator()<0, true>(s);
            one.template operator()<1, true>(s + 1);
        }
        for (; s < steps; s += 2) {
            one.template operator()<0, false>(s);
            if (s + 1 < steps) one.template operator()<1, false>(s + 1);
        }
        step += steps;
    }
    // Operands of any alignment, and the part of a step that is left at the contraction's end.
    if (step < last) {
        u32x4 vp[TileP::EACH], vq[TileQ::EACH];
        TileP::fetch(a.p, m0, step, vp);
        TileQ::fetch(a.q, n0, step, vq);
        if (DIRECT) __syncthreads();                     // the buffers have been read
        for (uint32_t s = 0; step < last; ++step, ++s) {
            uint8_t *now = lds + (s & 1) * BUFFER;       // (read last in step s - 2, before the last barrier)
            TileP::put(now, vp);
            TileQ::put(now + TileP::BYTES, vq);
            __syncthreads();
            if (step + 1 < last) {
                TileP::fetch(a.p, m0, step + 1, vp);
                TileQ::fetch(a.q, n0, step + 1, vq);
            }
            each<PHASES>([&]<int PH>() {
                each<READS_P>([&]<int U>() { read_p.template operator()<PH, U / DEEP, U % DEEP>(now, p[0]); });
                if constexpr (PH % PARTS == 0) each<READS_Q>([&]<int U>() { read_q.template operator()<PH, U / DEEP, U % DEEP>(now, q[0]); });
                each<MATRIX>([&]<int M>() { multiply.template operator()<PH, M / RN, M % RN>(p[0], q[0]); });
            });
        }
    }

    // Lane l has, of fragment (i, j), row 16i + l % 16 and columns 16j + 4 (l / 16) .. + 3.  Every wave turns its results in LDS, ROUND
    // rows at a time, so that lanes finish 8 neighbours each and rows are stored in one piece (the rows in LDS are 16 bytes apart in
    // the banks).
    __syncthreads();                                     // all waves are through with the operand tiles
    constexpr int COLS = TN / WN, ROWS = TM / WM, ROUND = epilogue_rows(TM, TN, WM, WN), PITCH = COLS + 4;
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
        finish_rows<ROUND, COLS, PITCH>(a, split, mine, m0 + wm * ROWS + r0, n0 + wn * COLS);
        __builtin_amdgcn_wave_barrier();
    }
    if (a.splits <= 1 && a.e.message && group == 0 && !a.n_first) pad_message(a.e);
}

// ---- tens of rows -------------------------------------------------------------------------------
// The same tiles where reading b is what takes time: 64 x 64 results a workgroup and RING steps' tiles in LDS, all but one of them
// on their way, so that a CU keeps RING - 1 times 16 KiB in flight.  Operands along, in vectors.
constexpr int kRing = 8;

template <Factor F>
__global__ __launch_bounds__(256) void k_product_ring(ProductArgs a)
{
    constexpr int T = 64, ES = F == F_E4M3 ? 1 : 2, R = 2;                   // four waves of 32 x 32
    using Tile = TileOf<T, false, ES, 256>;
    constexpr int BUFFER = 2 * Tile::BYTES, LOADS = 2 * Tile::EACH;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const uint32_t tiles = a.tiles_m * a.tiles_n, group = a.first_group + blockIdx.x, split = a.splits > 1 ? group / tiles : 0, tile = group - split * tiles;
    const uint32_t m0 = tile % a.tiles_m * T, n0 = tile / a.tiles_m * T;
    const int wave = int(threadIdx.x) >> 6, wm = wave >> 1, wn = wave & 1;
    const uint32_t depth = a.p.depth, all_steps = (depth + Tile::DEPTH - 1) / Tile::DEPTH, whole = depth / Tile::DEPTH;
    const uint32_t first = split * a.split_steps, last = min(all_steps, first + a.split_steps);
    const uint32_t steps = min(last, whole) > first ? min(last, whole) - first : 0;
    f32x4 acc[R][R];
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < R; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    auto compute = [&](const uint8_t *at) {
        u32x4 p[R][2], q[R][2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < R; ++i) {
                p[i][h] = Tile::fragment(at, 32 * wm, i, h);
                q[i][h] = Tile::fragment(at + Tile::BYTES, 32 * wn, i, h);
            }
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < R; ++j) multiply_pieces<F>(acc[i][j], q[j], p[i]);
    };
    uint32_t at_p[Tile::EACH], at_q[Tile::EACH];
    Tile::offsets(a.p, m0, at_p);
    Tile::offsets(a.q, n0, at_q);
    const uint32_t lds0 = uint32_t(uintptr_t((__attribute__((address_space(3))) uint8_t *)lds));
    // workgroups begin at different steps, so that they do not ask the same memory channels at the same time (64 x 14336 x 4096 29.8 ->
    // 27.8 us)
    const uint32_t begin = steps ? group % steps : 0;
    auto turned = [&](uint32_t s) { return s + begin < steps ? s + begin : s + begin - steps; };
    auto load = [&](uint32_t s) {                            // (past the end the last step again, into a buffer that is not read)
        const uint32_t to = lds0 + s % kRing * BUFFER, step = first + turned(min(s, steps - 1));
        const i32x4 from_p = Tile::descriptor(a.p, m0, step), from_q = Tile::descriptor(a.q, n0, step);
#pragma unroll
        for (int j = 0; j < Tile::EACH; ++j) {
            Tile::load_direct(from_p, at_p, to, j);
            Tile::load_direct(from_q, at_q, to + Tile::BYTES, j);
        }
    };
    if (steps) {
#pragma unroll 1
        for (uint32_t s = 0; s + 1 < kRing; ++s) load(s);
        for (uint32_t s = 0; s < steps; ++s) {
            // of this wave's loads, all but those of the RING - 2 steps behind this one have arrived, and it has read the last step's tiles
            constexpr int behind = (kRing - 2) * LOADS;
            static_assert(behind < 64);
            __builtin_amdgcn_s_waitcnt((behind & 15) | (behind >> 4) << 14 | 7 << 4);
            asm volatile("s_barrier" ::: "memory");
            load(s + kRing - 1);
            compute(lds + s % kRing * BUFFER);
        }
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (last > whole && whole >= first) {                    // the part of a step that is left at the contraction's end
        u32x4 vp[Tile::EACH], vq[Tile::EACH];
        Tile::fetch(a.p, m0, whole, vp);
        Tile::fetch(a.q, n0, whole, vq);
        Tile::put(lds, vp);
        Tile::put(lds + Tile::BYTES, vq);
        __syncthreads();
        compute(lds);
        __syncthreads();
    }
    constexpr int PITCH = 36;
    float *mine = reinterpret_cast<float *>(lds) + wave * (32 * PITCH);
    const int l = int(threadIdx.x) & 63;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < R; ++j) *reinterpret_cast<f32x4 *>(mine + (16 * i + (l & 15)) * PITCH + 16 * j + 4 * (l >> 4)) = acc[i][j];
    __builtin_amdgcn_wave_barrier();
    finish_rows<32, 32, PITCH>(a, split, mine, m0 + 32 * wm, n0 + 32 * wn);
    if (a.splits <= 1 && a.e.message && group == 0) pad_message(a.e);
}

// ---- few rows ---------------------------------------------------------------------------------
// Products of at most 16 rows: every row of b is read once, straight into the registers of the matrix instruction, and nothing is
// shared but the rows of a, which stay in the L2.  A workgroup owns 16 columns; its waves take the contraction's 128-byte pieces
// in turn, and their sums are joined in LDS in the waves' order.  Bound by the reading of b (1 x 4096 x 14336, bf16, 16 waves:
// 23.6 us, 5.0 TB/s, of which 5 are the ramp and the end; with b read non-temporally 25.4, with 3 pieces a batch 27.3, by 8 waves
// 26.0).  Any alignment: the vectors of a fragment are read wherever they lie.
HXT_HD constexpr int rows_lds(int waves) { return waves * 16 * 20 * 4; }

template <Factor F, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_product_rows(ProductArgs a)
{
    constexpr int ES = F == F_E4M3 ? 1 : 2, UNROLL = 2, PITCH = 20;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    float *parts = reinterpret_cast<float *>(lds);
    const int l = int(threadIdx.x) & 63, r = l & 15, g = l >> 4;
    const uint32_t wave = threadIdx.x >> 6, n0 = (a.first_group + blockIdx.x) * 16;
    // rows past the end repeat the last one, what comes of them is not stored
    const uint8_t *at_a = a.p.p + int64_t(min(uint32_t(r), a.e.m - 1)) * a.p.stride + 16 * g;
    const uint8_t *at_b = a.q.p + int64_t(min(n0 + r, a.e.n - 1)) * a.q.stride + 16 * g;
    f32x4 acc = {0, 0, 0, 0};
    // Batches of UNROLL pieces a wave; the next one is asked for before this one is multiplied.
    const uint32_t pieces = a.p.depth / (kStep / ES), batches = (pieces + UNROLL * WAVES - 1) / (UNROLL * WAVES);
    u32x4 x[2][UNROLL][2], y[2][UNROLL][2];
    auto load = [&](uint32_t b, u32x4 (&xs)[UNROLL][2], u32x4 (&ys)[UNROLL][2]) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const uint64_t at = uint64_t(min(wave + WAVES * (b * UNROLL + u), pieces - 1)) * kStep;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                ys[u][h] = load16_any<false>(at_b + at + 64 * h);
                xs[u][h] = load16_any<false>(at_a + at + 64 * h);
            }
        }
    };
    auto use = [&](uint32_t b, const u32x4 (&xs)[UNROLL][2], const u32x4 (&ys)[UNROLL][2]) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
            if (wave + WAVES * (b * UNROLL + u) < pieces) multiply_pieces<F>(acc, ys[u], xs[u]);
    };
    if (batches) load(0, x[0], y[0]);
    for (uint32_t b = 0; b < batches; b += 2) {
        if (b + 1 < batches) load(b + 1, x[1], y[1]);
        use(b, x[0], y[0]);
        if (b + 1 >= batches) break;
        if (b + 2 < batches) load(b + 2, x[0], y[0]);
        use(b + 1, x[1], y[1]);
    }
    if (a.p.depth % (kStep / ES) && wave == pieces % WAVES) {       // the piece that the contraction ends in, zeros behind
        auto part = [&](const uint8_t *at, int h) {
            using E = std::conditional_t<ES == 1, uint8_t, uint16_t>;
            const uint32_t from = (pieces * kStep + 64 * h + 16 * g) / ES;
            E e[16 / ES];
#pragma unroll
            for (uint32_t i = 0; i < 16 / ES; ++i) e[i] = from + i < a.p.depth ? reinterpret_cast<const E *>(at + uint64_t(pieces) * kStep + 64 * h)[i] : E(0);
            return __builtin_bit_cast(u32x4, e);
        };
        const u32x4 xs[2] = {part(at_a, 0), part(at_a, 1)}, ys[2] = {part(at_b, 0), part(at_b, 1)};
        multiply_pieces<F>(acc, ys, xs);
    }
    *reinterpret_cast<f32x4 *>(parts + (wave * 16 + r) * PITCH + 4 * g) = acc;       // row l % 16, columns 4 (l / 16) .. + 3
    __syncthreads();
    if (threadIdx.x < 32) {
        const uint32_t m = threadIdx.x / 2, col = threadIdx.x % 2 * 8;
        float z[8] = {};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const f32x4 lo = *reinterpret_cast<const f32x4 *>(parts + (w * 16 + m) * PITCH + col), hi = *reinterpret_cast<const f32x4 *>(parts + (w * 16 + m) * PITCH + col + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                z[i] += lo[i];
                z[4 + i] += hi[i];
            }
        }
        finish<8>(a.e, m, n0 + col, z);
    }
    if (a.e.message && n0 == 0) pad_message(a.e);
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
    if (n0 + 4 <= e.n) {
#pragma unroll 4
        for (uint32_t s = 0; s < splits; ++s) {             // (several parts on their way at a time)
            float v[4];
            __builtin_memcpy(v, at + s * part, 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) z[i] += v[i];
        }
    } else {
        for (uint32_t s = 0; s < splits; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n0 + i < e.n) z[i] += at[s * part + i];
    }
    finish<4>(e, m, n0, z);
}

// Rows copied to 16-byte multiples, vectors a row, zeros behind the row's end.
template <typename E>
__global__ __launch_bounds__(256) void k_product_align(const uint8_t *__restrict__ from, int64_t stride, uint32_t cols, uint64_t count, uint32_t vectors,
                                                       u32x4 *__restrict__ to, uint32_t first_group)
{
    const uint64_t id = (uint64_t(first_group) + blockIdx.x) * 256 + threadIdx.x;
    if (id >= count) return;
    constexpr uint32_t V = 16 / sizeof(E);
    const uint64_t row = id / vectors;
    const uint32_t col = uint32_t(id - row * vectors) * V;
    const uint8_t *at = from + row * stride + size_t(col) * sizeof(E);
    if (col + V <= cols) {
        to[id] = load16_any<false>(at);
        return;
    }
    E e[V];
#pragma unroll
    for (uint32_t i = 0; i < V; ++i) e[i] = col + i < cols ? reinterpret_cast<const E *>(at)[i] : E(0);
    to[id] = __builtin_bit_cast(u32x4, e);
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

// 64 lanes x 8 columns, 4 waves on every fourth row of a band; a band's column sums go to partial.  Bound by memory (4096 x 14336: 61 us,
// 5.8 TB/s).
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

}  // namespace hxt

#endif
