// Which kernel serves a product, and what its workspace holds: rules on sizes alone, without HIP, so that they can be tested without a
// GPU.
#ifndef HXT_PRODUCT_RULES_H
#define HXT_PRODUCT_RULES_H

#include <algorithm>
#include <cstddef>
#include <cstdint>
#include <utility>

namespace hxt {

constexpr int kStep = 128;        // bytes of a row per step, of operands along; across: kStep / 2 rows

// ---- which kernel ---------------------------------------------------------------------------
struct Shape {
    uint32_t tile;                 // 16: k_product_rows, 64: k_product_ring, else k_product's
    uint32_t splits, split_steps;
    uint32_t half;                 // of 256 x 256 tiles: columns of tiles at the end that go as 256 x 128
    double us;                     // what it is expected to take
};

inline uint32_t up(uint64_t n, uint64_t to) { return uint32_t((n + to - 1) / to); }

// Which kernel, and in how many parts of the contraction: the least time by these measured costs in us.
//   A step (128 bytes of the contraction) of a full round of workgroups, a round being what the chip holds at a time:
//   256 x 256 tiles, one a CU, 1.5 (4096 x 4096 x 14336: 341 us in one round of 224 steps), 256 x 128 0.9; 128 x 128, two a CU, 1.0 (448 us in two
//   rounds), one a CU 0.65; through registers (operands not in vectors) 1.6; the ring of 64 x 64, one a CU, 0.42 (64 x 14336 x
//   4096: 27.8 us in one round of 64 steps; as 128 x 128 tiles in four parts 34.9).  A round's ramp and end 4 (ring 2.5); joining
//   the parts 4 and what they take to be written and read at 5 TB/s.  Where whole rounds of 256 x 256 tiles leave few, these go as
//   256 x 128 in a launch of their own (4096 x 14336 x 4096: 8 bits 214 -> 204 us, bf16 396 -> 381).
//   Up to 4 rows (16 where the ring cannot serve them) k_product_rows: 1 x 4096 x 14336 23.6 us against 27.5 as a ring in four
//   parts; 8 x 14336 x 4096 29.5 against 26.
inline Shape shape_for(int64_t m, int64_t n, int64_t depth, int64_t es, bool along, bool direct)
{
    const uint32_t steps = std::max(1u, up(uint64_t(depth), uint64_t(kStep / es)));
    if (along && m <= (direct ? 4 : 16)) return Shape{16, 1, steps, 0, 0};
    Shape best{128, 1, steps, 0, 0};
    double least = 1e30;
    for (const uint32_t tile : {64u, 128u, 256u}) {
        if ((tile != 128 && !direct) || (tile == 64 && !along)) continue;
        const uint64_t tiles = uint64_t(up(m, tile)) * up(n, tile);
        for (uint32_t s = 1; s <= 16 && (s == 1 || (steps / s >= 4 && tiles * s <= 512)); s *= 2) {
            const uint32_t each = up(steps, s);
            const double rounds = double((tiles * s + 255) / 256);       // of one workgroup a CU
            double t = tile == 64 ? rounds * (0.42 * each + 2.5) : (tile == 256 ? rounds * (1.5 * each + 4) : 0);
            if (tile == 128) t = (direct ? double(uint64_t(rounds) / 2) + 0.65 * double(uint64_t(rounds) % 2) : 0.8 * (rounds + 1)) * each + 2 * (rounds + 1);
            if (s > 1) t += 4.0 + double(m) * double(n) * s * 8 / 5e6;
            if (t < least) {
                least = t;
                best = Shape{tile, s, each, 0, t};
            }
            // what is left behind whole rounds, in half tiles that fill one
            const uint64_t tm = up(m, 256), tn = up(n, 256), whole = tile == 256 && s == 1 ? tiles / 256 * 256 / tm : 0;
            if (whole && whole < tn && (tn - whole) * 2 * tm <= 256) {
                const double u = double((tm * whole + 255) / 256) * (1.5 * each + 4) + 0.9 * each + 8;
                if (u < least) {
                    least = u;
                    best = Shape{tile, s, each, uint32_t(tn - whole), u};
                }
            }
        }
    }
    return best;
}

inline uint64_t up256(uint64_t n) { return (n + 255) / 256 * 256; }

inline uint64_t parts_bytes(const Shape &s, int64_t m, int64_t n) { return s.splits > 1 ? up256(uint64_t(s.splits) * m * n * sizeof(float)) : 0; }

// A copy of rows x cols elements whose rows begin at 16-byte multiples.
inline uint64_t copy_bytes(int64_t rows, int64_t cols, int64_t es) { return up256(uint64_t(rows) * ((uint64_t(cols * es) + 15) / 16 * 16)); }

// Operands whose rows are not in vectors (odd row lengths or pitches) are copied first where the workspace has room and the
// copies, written and read at 4.5 TB/s, cost less than the way through registers (4096 x 4096 x 4095: 246 us through registers,
// 131 copied).  s: the way without copies, and after the call the chosen one.
inline bool worth_copying(Shape &s, int64_t m, int64_t n, int64_t depth, int64_t es, bool along, uint64_t copied)
{
    Shape with = shape_for(m, n, depth, es, along, true);
    with.us += 3 + double(copied) * 2 / 4.5e6;
    if (s.tile == 16 || with.us >= s.us) return false;
    s = with;
    return true;
}

// Workspace of a product: the parts of its sums, and copies of operands whose rows are no whole vectors.
inline size_t work_for(int64_t m, int64_t n, int64_t depth, int64_t es, bool p_across, bool q_across)
{
    if (m <= 0 || n <= 0 || depth <= 0) return 0;
    const bool along = !p_across && !q_across;
    Shape direct = shape_for(m, n, depth, es, along, true), any = shape_for(m, n, depth, es, along, false);
    uint64_t need = std::max(parts_bytes(direct, m, n), parts_bytes(any, m, n)), copies = 0;
    for (const auto &[across, outer] : {std::pair{p_across, m}, {q_across, n}})
        if ((across ? outer : depth) * es % 16) copies += across ? copy_bytes(depth, outer, es) : copy_bytes(outer, depth, es);
    if (copies && worth_copying(any, m, n, depth, es, along, copies)) need = std::max(need, parts_bytes(any, m, n) + copies);
    return size_t(need);
}

struct Way {
    Shape shape;
    bool direct;                   // tiles are loaded straight into LDS
    bool copy_p, copy_q;           // operands copied to whole vectors first, to these places in the workspace
    uint64_t p_at, q_at;
};

// p_direct, q_direct: the operand's rows are whole vectors at 16-byte multiples.  Of an empty contraction nothing is read, nor copied.
inline Way way_for(int64_t m, int64_t n, int64_t depth, int64_t es, bool p_across, bool q_across, bool p_direct, bool q_direct, size_t work_bytes)
{
    const bool along = !p_across && !q_across;
    Way w{{}, (p_direct && q_direct) || depth == 0, false, false, 0, 0};
    w.shape = shape_for(m, n, depth, es, along, w.direct);
    if (w.direct) return w;
    const uint64_t p_bytes = p_direct ? 0 : (p_across ? copy_bytes(depth, m, es) : copy_bytes(m, depth, es));
    const uint64_t q_bytes = q_direct ? 0 : (q_across ? copy_bytes(depth, n, es) : copy_bytes(n, depth, es));
    Shape copied = w.shape;
    if (!worth_copying(copied, m, n, depth, es, along, p_bytes + q_bytes) || parts_bytes(copied, m, n) + p_bytes + q_bytes > work_bytes) return w;
    const uint64_t at = parts_bytes(copied, m, n);
    return Way{copied, true, !p_direct, !q_direct, at, at + p_bytes};
}

}  // namespace hxt

#endif
