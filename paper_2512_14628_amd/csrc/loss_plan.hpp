// How hsadmm_softmax_loss cuts its products and lays out its workspace: host arithmetic only, without HIP, so that it also compiles
// by itself (tests/test_loss_plan_cpu.py sweeps it).
#ifndef LOSS_PLAN_HPP
#define LOSS_PLAN_HPP
#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace {

// Bytes of logits, and then their gradients, that hsadmm_softmax_loss holds at once.  A piece costs its logits a second time: 8192 x 2048 x
// 131072 in bf16, a twentieth padding, 11.9 ms in one piece of 2^31 bytes, 13.3 in two, 14.1 in four, 14.6 in eight; 16384 rows, in two,
// 26.5 for twice 11.9.  So more than this would save a tenth to a fifth of the largest calls only, for a workspace of as many more
// gigabytes beside the model.
constexpr int64_t kLossHeld = 1ll << 31;
constexpr int kInputRows = 256;          // rows of the held copies are rounded up to this ...
constexpr int kInputCols = 64;           // ... and their columns to this (128 bytes at least)
constexpr int kLossHeadBytes = 512;

// The tile of a product: b by b elements of the output (kNarrow: 128 by 32), in `splits` parts of the k axis.
constexpr int kNarrow = 32, kNarrowTile = 128;
struct ProductPlan {
    int b;
    int splits;
    int64_t k_part;
    bool fills;          // tiles enough for the chip without parts
};

// The largest tile that has a workgroup for each of the chip's 256 compute units: 256 (16-bit types only, and more than 128 rows: half of
// the tile would be rows that do not exist, and that kSums and the slabs have no room for; where parts of the k axis are allowed they
// count too), 128, 64.  Fewer tiles of 64 than that: parts, of tiles of 128 in 16 bits if those then fill the chip.  The
// number of parts is the one that leaves the fewest places on the chip idle in the last round (a hundredth off for each: their sums
// are written and read); parts of tiles of 64 that fill the chip are none.  Up to 32 rows the tile is 128 x 32.  us (parts):
//   tiles of 128 / 256   inputs' gradients of 3690 x 2048 x 32768, bf16 799 / 652 (2)
//   tiles of 64 / 128    rows x 1568 x 3479, 560 rows: bf16 18.9 (1), 20.7 (2) / 23.6 (1), 22.4 (2); fp32 67 (1) / 108 (1), 81 (3)
//                        256 x 16384 x 2048, bf16 97.8 (1), 32.4 (8) / 30.3 (8), 28.0 (16); 256 x 2048 x 1000, fp32 14.5 (8), 49 (1) / 16.6 (16)
//   128 x 32 / 128 x 128 x 2048 x 131072, bf16: one row 92 / 102, 32 rows 99 / 115, 33 rows 147 / 116
inline ProductPlan plan_product(int64_t out_p, int64_t out_q, int64_t k, bool sixteen, bool narrow, bool parts)
{
    constexpr int64_t kUnits = 256;
    const auto tiles = [&](int64_t b) { return narrow ? (out_p + kNarrowTile - 1) / kNarrowTile : ((out_p + b - 1) / b) * ((out_q + b - 1) / b); };
    const auto most_parts = [&](int64_t b) { return parts ? std::max<int64_t>(1, k / (4 * b)) : 1; };
    ProductPlan r{};
    r.b = narrow ? kNarrow
        : sixteen && out_q > 128 && tiles(256) * most_parts(256) >= kUnits ? 256
        : tiles(128) >= kUnits ? 128
        : sixteen && tiles(64) < kUnits && tiles(128) * most_parts(128) >= kUnits ? 128 : 64;
    const int64_t n = tiles(r.b);
    r.fills = n >= kUnits;
    r.splits = 1;
    if (parts && k > 0 && !(r.b == 64 && r.fills)) {
        const int64_t at_once = kUnits * (r.b == 256 ? 1 : r.b == 128 || !sixteen ? 2 : 4);        // workgroups that share the chip
        const int64_t most = std::min<int64_t>({r.b >= 128 ? most_parts(r.b) : std::max<int64_t>(1, k / 128), std::max<int64_t>(1, 2 * at_once / n), 64});
        double best = 0.0;
        for (int64_t s = 1; s <= most; ++s) {
            const int64_t rounds = (n * s + at_once - 1) / at_once;
            const double part = (double)(n * s) / (double)(rounds * at_once) * (1.0 - 0.01 * (double)s);
            if (part > best) { best = part; r.splits = (int)s; }
        }
    }
    r.k_part = std::max<int64_t>(64, (k + r.splits * 64 - 1) / (r.splits * 64) * 64);
    r.splits = (int)std::max<int64_t>(1, (k + r.k_part - 1) / r.k_part);
    return r;
}

constexpr int64_t kFewTerms = 256;

// How hsadmm_softmax_loss cuts its products, and where its scratch lies in the workspace.
struct LossScratch {
    size_t head, row, label, place, held_loss, picked, own, rounded, stat, slab, rows, packed, parts, grads, sums, total;
    int64_t Np, Dp;             // rows and columns of the held inputs
    int64_t Vc;                 // classes of a piece, a multiple of 256
    int pieces;
    bool pack;                  // W's rows are copied before they are used (not whole pieces of 16 bytes)
    bool small;                 // logits in fp32 and in parts, joined by rows
    bool rest_inputs, rest_weights;     // the products with what the rounding of the logits' gradients leaves are added
    ProductPlan logits, inputs, weights;
    int slab_elems;
    int64_t slabs;
    bool launches;              // the products' tiles fit their grids
};

// Whether a product's tiles fit one launch.
inline bool launches(const ProductPlan& how, int64_t out_p, int64_t out_q)
{
    const int64_t bp = how.b == kNarrow ? kNarrowTile : how.b, threads = how.b == 256 ? 512 : 256;
    return ((out_p + bp - 1) / bp) * ((out_q + how.b - 1) / how.b) * how.splits + 8 < (1ll << 32) / threads;
}

// For n rows on a layer of V rows of D elements of `size` bytes, `off` elements into its arena; `held`: bytes of logits held at once.
inline LossScratch loss_scratch(int64_t held, int32_t V, int32_t D, int64_t off, int64_t n, int64_t size, bool gradients)
{
    LossScratch s{};
    const bool narrow = n <= kNarrow, sixteen = size == 2;
    // (up to 128 rows no tile is longer, plan_product)
    s.Np = n <= 128 ? 128 : (n + kInputRows - 1) / kInputRows * kInputRows;
    s.Dp = ((int64_t)D + kInputCols - 1) / kInputCols * kInputCols;
    s.pack = D * size % 16 != 0 || off * size % 16 != 0;
    const int64_t most = std::max<int64_t>(256, held / size / s.Np / 256 * 256);
    s.pieces = gradients || s.pack ? (int)((V + most - 1) / most) : 1;
    s.Vc = ((V + s.pieces - 1) / s.pieces + 255) / 256 * 256;
    s.pieces = (int)((V + s.Vc - 1) / s.Vc);
    s.logits = plan_product(V, n, s.Dp, sixteen, narrow, false);
    // The gradients of the logits are rounded to 16 bits.  Of the label's what the rounding leaves is always added.  The other classes'
    // roundings differ in sign: together they are off by sqrt(sum of p^2) of a rounding, little where the softmax is spread over many
    // classes.  A vocabulary of a few classes is none: there, and in the weights' gradient of a few rows, what is left of all
    // roundings is multiplied too, twice the time of a product that is short (fp16, error against 64 bits 0.00031 without, 0.00022 with;
    // the output's own rounding is 0.00021).
    const bool fits = s.pieces == 1 && 4 * s.Np * s.Vc <= held;
    s.rest_inputs = gradients && sixteen && fits && V <= kFewTerms;
    s.rest_weights = gradients && sixteen && fits && (n <= kFewTerms || V <= kFewTerms);
    // (tiles of 64 are for so few logits that they are joined by rows as well)
    s.small = (s.pieces == 1 && (!s.logits.fills || s.logits.b == 64)) || s.rest_inputs || s.rest_weights;
    if (s.small) s.logits = plan_product(V, n, s.Dp, sixteen, narrow, true);
    else if (!narrow && s.logits.b == 64) s.logits.b = 128;
    s.inputs = plan_product(D, n, s.Vc, sixteen, narrow, true);
    s.weights = plan_product(D, std::min<int64_t>(V, s.Vc), n, sixteen, false, false);
    s.slab_elems = s.logits.b == kNarrow ? 32 : s.logits.b / 2;
    s.slabs = s.small ? 0 : (V + 255) / 256 * (256 / s.slab_elems);
    s.launches = launches(s.logits, V, n) && launches(s.inputs, D, n) && launches(s.weights, D, std::min<int64_t>(V, s.Vc));
    size_t at = 0;
    const auto take = [&](int64_t bytes) { const size_t here = at; at = (at + (size_t)bytes + 255) / 256 * 256; return here; };
    s.head = take(kLossHeadBytes);
    s.row = take(4 * s.Np);
    s.label = take(4 * s.Np);
    s.place = take(4 * s.Np);
    s.held_loss = take(4 * s.Np);
    s.picked = take(4 * s.Np);
    s.own = take(gradients ? 4 * s.Np : 0);
    s.rounded = take(gradients ? 4 * s.Np : 0);
    s.stat = take(8 * s.Np);
    s.slab = take(8 * s.slabs * s.Np);
    s.rows = take(size * s.Np * s.Dp);
    s.packed = take(s.pack ? size * s.Vc * s.Dp : 0);
    s.parts = take(s.small ? 4 * (int64_t)s.logits.splits * s.Np * s.Vc : 0);
    s.grads = take(gradients ? size * s.Np * s.Vc * (s.rest_inputs || s.rest_weights ? 2 : 1) : 0);
    s.sums = take(gradients ? 4 * (int64_t)s.inputs.splits * s.Np * s.Dp : 0);
    s.total = at;
    return s;
}

}  // namespace
#endif
