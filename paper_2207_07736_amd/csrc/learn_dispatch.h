// learn_dispatch.h -- which form of a learner's kernel a call runs, how its work is cut,
// and what workspace that takes, as functions of its sizes alone (plain C++).
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace rlsim_dev {

inline uint64_t up_to(uint64_t x, uint64_t multiple) { return (x + multiple - 1u) / multiple * multiple; }
inline uint64_t least(uint64_t a, uint64_t b) { return a < b ? a : b; }
inline uint64_t most(uint64_t a, uint64_t b) { return a > b ? a : b; }

// ---- the gated recurrence ----------------------------------------------------------
constexpr uint32_t kScanMark = 16u;               // steps between marks, and of a run of loads
constexpr uint32_t kScanMapEntries = 1u << 22;    // most segments x channels of a call
constexpr uint32_t kScanSegments = 1024u;

struct ScanCut { uint32_t segments, seg_len; };
// Segments of time for `threads` threads' channels.  A cut call reads its rows twice, so few
// are cut: where there are fewer than two waves to a CU, or four if the steps are many (one
// thread's run of 16 steps takes 4 us whatever the others do).  What is cut is cut into
// segments of 32 steps at least, and no more workgroups than run at once: `per_cu` of 256
// threads on each CU (1,024 x 37 x 336 fp16 backward 82 us with 800 workgroups where 768 run at
// once, 37 x 320 with 768 of them 63).  Forward and backward, us, uncut / cut:
//   200 x 4,096 x 64 fp32 338 / 531     1,000 x 1,024 x 64 bf16 652 / 359
//   200 x 1,024 x 64 fp32 122 / 122     1,000 x 2,048 x 64 bf16 687 / 677
inline ScanCut scan_cut(uint64_t threads, uint64_t channels, uint32_t T, uint32_t cus, uint32_t per_cu)
{
    const uint64_t enough = (T <= 256u ? 128ull : 256ull) * cus, groups = (threads + 255u) / 256u;
    uint64_t s = threads >= enough ? 1u : most((uint64_t)per_cu * cus / groups, 1u);
    s = least(s, T / 32u);
    s = least(s, kScanSegments);
    s = least(s, channels ? kScanMapEntries / channels : 1u);
    if (s < 2u) return {1u, T};
    const uint32_t len = (uint32_t)up_to((T + s - 1u) / s, kScanMark);
    return {(T + len - 1u) / len, len};
}

// ---- clipping --------------------------------------------------------------------
constexpr uint32_t kClipTensors = 96u;            // of one launch: their table has to fit its arguments
constexpr uint32_t kClipBlocks = 6144u;           // most blocks of a call, beyond one to a tensor
constexpr uint64_t kClipSmall = 1u << 15;         // elements that one workgroup takes alone
// Elements of a block.  About 2,048 blocks, all of them at once, up to 50 M elements; larger
// ones leave too few, and as every workgroup of the scaling adds up all blocks' sums, smaller
// ones too many.  us at 1,984 / 4,096 / 8,192 / 16,384 blocks: 61 tensors of 50 M in place
// 35.5 / 38.2, 48 of 400 M bf16 into others 442 / 428 / 423 / 475.
inline uint64_t clip_chunk(uint64_t total)
{
    if (total <= kClipSmall) return 1024u;
    const uint64_t few = least(most(total / 2048u, 8192u), 24576u);
    return up_to(most(few, (total + kClipBlocks - 1u) / kClipBlocks), 2048u);
}

// ---- the output layer's cross entropy ------------------------------------------------
// Products of rows run in 16-bit matrix instructions.  fp32 rows are scaled and cut into
// two fp16 parts of 11 bits each; the three products that reach 22 bits are summed.  (Three
// bf16 parts and six products, 24 bits, took 187 us instead of 148 at 2,048 x 256 on 4,096; the
// matrix units' own fp32 products run at a sixteenth of the rate.)
constexpr uint32_t kXentK = 32u;                  // elements of a step along the summed dimension
struct XentShape {
    uint32_t rows, dim, vocab, parts;
    uint32_t dim_k, rows_k;                       // padded to whole steps
    uint32_t piece;                               // entries of the vocabulary at a time
};
inline XentShape xent_shape(uint32_t rows, uint32_t dim, uint32_t vocab, uint32_t parts)
{
    XentShape s{rows, dim, vocab, parts, (uint32_t)up_to(dim, kXentK), (uint32_t)up_to(rows, kXentK), 0u};
    // both of dz's arrays stay in the last-level cache: 64 MB each (128 MB each, 4,096 x 4,096 on
    // 131,072 bf16: 15.3 ms instead of 15.1)
    uint64_t p = least((1ull << 25) / ((uint64_t)parts * s.rows_k), (1ull << 25) / ((uint64_t)parts * s.dim_k));
    p = most(p / 256u * 256u, 256u);
    s.piece = (uint32_t)least(p, up_to(vocab, 256u));
    return s;
}

// The tile of a product M x N, and how many workgroups share the summed dimension of one
// (only sums may be shared).  256 x 256 where that gives every CU one and the sum is long
// enough to pay for its ends; us, 256 / 128: 4,096 x 4,096 on 131,072 bf16 14,340 / 19,490,
// 4,096 x 256 on 8,192 142 / 149, and 7 x 1,024 on 32,000 (one step) 27 / 19 for dmatrix.
// Shares for one workgroup to a CU (two to a CU: 512 x 512 on 8,192 bf16 71 us instead of
// 57, for the sums' writes and reads).
struct XentTile { uint32_t m, n, span, share; };  // span: entries along m of one wave
constexpr uint32_t kXentShareTiles = 1024u;
inline XentTile xent_tile(uint32_t M, uint32_t N, uint64_t steps, bool sums, uint32_t cus)
{
    const uint64_t big = ((M + 255ull) / 256u) * ((N + 255ull) / 256u);
    XentTile t = N <= 32u ? XentTile{128u, 32u, 32u, 1u} : big >= cus && steps >= 8u ? XentTile{256u, 256u, 128u, 1u} : XentTile{128u, 128u, 64u, 1u};
    const uint64_t tiles = (uint64_t)((M + t.m - 1u) / t.m) * ((N + t.n - 1u) / t.n), wanted = cus;
    if (!sums || tiles >= wanted || t.m == 256u) return t;
    const uint64_t s = least(least(wanted / tiles, steps / 4u), least(kXentShareTiles / tiles, 64u));
    t.share = s < 2u ? 1u : (uint32_t)s;
    return t;
}
// Floats that hold a product's shares: its tiles times 128 x 128 at most, or the product.
inline uint64_t xent_share_floats(uint64_t rows, uint64_t dim4) { return most(rows * dim4, (uint64_t)kXentShareTiles * 128u * 128u); }

// Where few rows decide a gradient, the rounding of dz to 16 bits can be well above the mean
// beside the result's own: the errors of some calls of 1 to 54 rows were 1.5 to 1.8 times
// those of exact factors (of many rows they average to 1.1, or 1.4 with weights).  So dz has
// two parts: for dhidden of up to 16 rows, the second part as 16 rows more, which the smallest tile
// has room for; and for dmatrix of fp16 calls of up to 1,024 rows (of bf16 ones it is fp16, and
// fine enough).
constexpr uint32_t kXentStackRows = 16u, kXentFewRows = 1024u;

struct XentWork {                                 // byte offsets
    uint64_t info, zt, stats, refs, part, up_n, up_m, x, xm, w, dz, dz_w, dx, dw, end;
};
inline XentWork xent_work(const XentShape& s)
{
    XentWork o{};
    uint64_t at = 0u;
    auto take = [&at](uint64_t bytes) { const uint64_t p = at; at += up_to(bytes, 256u); return p; };
    const uint64_t P2 = 2ull * s.parts, dim4 = up_to(s.dim, 4u);
    o.refs = take(8u);
    o.info = take(32ull * s.rows_k);
    o.zt = take(4ull * s.rows_k);
    o.stats = take(12ull * s.rows_k);
    o.part = take(8ull * s.rows_k * (up_to(s.vocab, 256u) / 32u));
    o.up_n = take(4ull * s.rows_k);
    o.up_m = take(4ull * s.piece);
    o.x = take(P2 * s.rows * s.dim_k);
    o.xm = take(P2 * s.rows_k * s.dim_k);
    o.w = take(P2 * s.piece * s.dim_k);
    o.dz = take(P2 * s.rows_k * s.piece);
    o.dz_w = take(4ull * s.rows_k * s.piece);
    o.dx = take(4u * xent_share_floats(s.rows, dim4));
    o.dw = take(4ull * kXentShareTiles * 128u * 128u);
    o.end = at;
    return o;
}
// Entries of the vocabulary in one launch for the losses: its tiles' threads stay below 2^32.
inline uint64_t xent_width(uint32_t rows_k) { return most((1ull << 36) / rows_k / 256u * 256u, 256u); }
// A handle's workspace: enough for every call within its bounds.
inline uint64_t xent_bound(uint32_t rows, uint32_t dim, uint32_t vocab, uint32_t parts)
{
    const XentShape s = xent_shape(rows, dim, vocab, parts);
    XentShape b = s;
    XentWork o = xent_work(b);
    // smaller rows or dim widen the piece: its arrays are bounded by their products
    const uint64_t P2 = 2ull * parts, piece_all = up_to(vocab, 256u);
    const uint64_t by_dim = least(P2 * piece_all * s.dim_k, most(2ull << 25, P2 * 256u * s.dim_k));
    const uint64_t by_rows = least(P2 * piece_all * s.rows_k, most(2ull << 25, P2 * 256u * s.rows_k));
    return o.up_m + up_to(4ull * piece_all, 256u) + 2u * up_to(P2 * (uint64_t)s.rows_k * s.dim_k, 256u) + up_to(by_dim, 256u) + 3u * up_to(by_rows, 256u)
           + (o.end - o.dx) + 4096u;
}

}  // namespace rlsim_dev
