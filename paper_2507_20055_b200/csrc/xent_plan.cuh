// How the linear cross entropy cuts its work: sizes of a handle's workspace, and pieces, tiles and slots of a call.  Host
// arithmetic alone (xent_splits runs on the device too), so that every extent can be checked against its buffer without a GPU.
#pragma once
#include <algorithm>
#include <cstddef>

#include "../../include/cert.h"

#ifdef __CUDACC__
#define CERT_BOTH __host__ __device__
#else
#define CERT_BOTH
#endif

namespace cert {

constexpr int kXentPairRows = 256;                    // rows of A per CTA pair
constexpr size_t kProbBytes = size_t(256) << 20;
constexpr size_t kWeightBytes = size_t(256) << 20;    // copy of a piece, where every call needs one
constexpr size_t kWeightBytesSpare = size_t(32) << 20;
constexpr size_t kSplitBytes = size_t(64) << 20;

// How many ranges K is cut into where there are fewer tiles than CTA pairs: what the pairs' waves cost in steps of 64 of K,
// with 8 steps for starting and ending a tile and the slabs' later addition (an eighth of a step per tile and slab).  Only
// counts that fill one, two, three or four waves are looked at.  The kernels work it out from the number of rows that
// count, which only the device knows; every thread does, so it is a handful of 32-bit operations.
CERT_BOTH inline int xent_splits(int tiles, int num_kb, int segs, int pairs, int most) {
    if (tiles <= 0 || most <= 1) return 1;
    int best = 1;
    float least = (float)((tiles + pairs - 1) / pairs) * (float)(num_kb * segs + 8);
    for (int waves = 1; waves <= 4; ++waves) {
        int s = pairs * waves / tiles;
        if (s > most) s = most;
        if (s > num_kb) s = num_kb;
        if (s <= best) continue;
        const float cost = (float)((tiles * s + pairs - 1) / pairs) * (float)((num_kb + s - 1) / s * segs + 8) + 0.125f * (float)(tiles * s);
        if (cost < least) { least = cost; best = s; }
    }
    return best;
}

inline long long xent_up(long long x, long long m) { return (x + m - 1) / m * m; }
inline long long xent_div(long long a, long long b) { return (a + b - 1) / b; }

// What a handle holds, in elements or bytes as the names say.
struct XentSizes {
    int D, V, Dp, Vp, parts;
    long long row_bytes;             // of the padded copies of x and the weights
    size_t rows_pad, wbuf_bytes, partial_cap, prob_bytes, dx32_floats, dw32_floats, colsum_floats;
};

inline XentSizes xent_sizes(int max_rows, int features, int classes, int type, bool with_grad) {
    XentSizes s = {};
    s.D = features;
    s.V = classes;
    s.parts = type == CERT_TYPE_F32 ? 3 : 1;
    s.Dp = (int)xent_up(features, 64);
    s.Vp = (int)xent_up(classes, 256);
    s.row_bytes = (long long)s.parts * s.Dp * 2;
    s.rows_pad = (size_t)xent_up(max_rows, kXentPairRows);
    const bool copies = s.parts > 1 || features % 8 != 0;
    // at least one piece of 256 classes fits whatever the sizes
    const long long w_want = std::min<long long>(s.Vp * s.row_bytes, (long long)(copies ? kWeightBytes : kWeightBytesSpare));
    s.wbuf_bytes = (size_t)std::max<long long>(w_want, std::min<long long>(s.Vp, 256) * s.row_bytes);
    // two slots per column tile: narrow tiles only where few rows share them
    s.partial_cap = std::max((size_t)(2 * xent_div(s.Vp, 256)) * s.rows_pad, (size_t)(2 * xent_div(s.Vp, 64)) * std::min<size_t>(s.rows_pad, 1024));
    // room for tiles that do not divide the classes (or a piece that is copied)
    s.partial_cap += (size_t)2 * s.rows_pad * (size_t)(copies ? xent_div(s.Vp * s.row_bytes, (long long)s.wbuf_bytes) : 1);
    if (with_grad) {
        const size_t prob_row = s.rows_pad * s.parts * 2;
        s.prob_bytes = std::max(std::min((size_t)s.Vp * prob_row, kProbBytes), (size_t)std::min<long long>(s.Vp, 256) * prob_row);
        s.dx32_floats = std::max(s.rows_pad * s.Dp, std::min(kSplitBytes / 4, 32 * s.rows_pad * s.Dp));
        // dW's sums over many rows are only split where the classes alone give few tiles
        s.dw32_floats = (size_t)s.Vp * s.Dp <= (1u << 21) ? std::min<size_t>(kSplitBytes / 4, (size_t)32 * s.Vp * s.Dp) : 64;
        s.colsum_floats = s.prob_bytes / (s.parts * 2) / 32;
    }
    return s;
}

// Column tile of the products over a row panel.  For 64 of K a pair's MMAs take 2 bn cycles, and each of its CTAs takes in 128
// rows of A (fewer where there are fewer) and bn / 2 of B at the 57 bytes per cycle that a multiprocessor gets from L2 (the
// rate of bulk copies measured with cert_peak_microbench); a tile costs 8 such steps more to start and end.  A width that
// divides the work into whole waves may win over a wider one (65536 classes, 74 pairs: 293 tiles of 224, four waves, instead
// of 256 of 256, also four).
inline int xent_pick_bn(int rows, int N, int K, int segs, int pairs, int unit) {
    int best = 256;
    double cost = 1e30;
    const int tiles_m = (int)xent_div(std::max(rows, 1), kXentPairRows);
    for (int bn = 256; bn >= 64; bn -= unit) {
        const double waves = (double)xent_div((long long)tiles_m * xent_div(N, bn), pairs);
        const double step = std::max(2.0 * bn, (std::min(rows, 128) * 128.0 + bn * 64.0) / 57.0);
        const double c = waves * (step * xent_div(K, 64) * segs + 8 * 512);
        if (c < cost * 0.999) { cost = c; best = bn; }
    }
    return best;
}

// Column tile and most ranges of K for a gradient's product of tiles_m row panels: as xent_splits, over both.
inline void xent_pick_split(int tiles_m, int N, int num_kb, int segs, int pairs, int most, int &bn, int &splits) {
    double least = 1e30;
    for (int b = 256; b >= 128; b /= 2) {
        const int tiles = tiles_m * (int)xent_div(N, b);
        const int s = xent_splits(tiles, num_kb, segs, pairs, most);
        const double waves = (double)xent_div((long long)tiles * s, pairs);
        const double cost = waves * ((double)xent_div(num_kb, s) * segs * (256 + b) / 512 + 8) + (s > 1 ? tiles * s / 8.0 * b / 256 : 0.0);
        if (cost < least * 0.999) { least = cost; bn = b; splits = s; }
    }
}

// (max, sum) pairs per row that the statistics of all classes leave, two for each column tile: a piece of the classes that
// is copied is tiled by itself, and its last tile may be a narrow one.
inline long long xent_slots(int V, int piece, int bn) {
    const long long whole = V / piece, rest = V - whole * piece;
    return 2 * (whole * xent_div(piece, bn) + xent_div(rest, bn));
}

// How a call is cut.
struct XentPlan {
    int rows_pad, tiles_m, segs;
    int copy_piece;                  // classes whose weights are read (or copied) at a time
    int piece, pieces;               // classes whose probabilities are held at a time
    int dx_kb, bn_dx, dx_most, bn_dw, dw_most;
    size_t slab, dw_slab;            // floats of a K range's sums for dx and dW
    bool by_row;                     // one product for statistics and probabilities
    int bn_lse;
};

inline XentPlan xent_plan(const XentSizes &s, int rows, bool direct, bool want_grad, int pairs) {
    XentPlan p = {};
    p.rows_pad = (int)xent_up(std::max(rows, 1), kXentPairRows);
    p.tiles_m = p.rows_pad / kXentPairRows;
    p.segs = s.parts == 1 ? 1 : 6;
    // the weights are read in place where TMA can, else piece by piece from a padded copy
    p.copy_piece = direct ? s.Vp : (int)std::min<long long>(s.Vp, (long long)s.wbuf_bytes / s.row_bytes / 256 * 256);
    const long long prob_row = (long long)p.rows_pad * s.parts * 2;
    p.piece = !want_grad ? s.Vp : (int)std::min<long long>(p.copy_piece, std::min<long long>(s.Vp, (long long)s.prob_bytes / prob_row / 256 * 256));
    p.pieces = (int)xent_div(s.V, p.piece);
    p.slab = (size_t)p.rows_pad * s.Dp;
    p.dw_slab = (size_t)std::min(p.piece, s.V) * s.Dp;
    p.dx_kb = (int)xent_div(std::min(p.piece, s.V), 64);
    p.bn_dx = p.bn_dw = 256;
    p.dx_most = p.dw_most = 1;
    if (want_grad) {
        // where the row and column tiles are too few, K is split and the slabs are added afterwards
        xent_pick_split(p.tiles_m, s.D, p.dx_kb, p.segs, pairs, (int)std::min<size_t>(32, std::max<size_t>(1, s.dx32_floats / p.slab)), p.bn_dx, p.dx_most);
        const int tiles_v = (int)xent_div(std::min(p.piece, s.V), kXentPairRows);
        xent_pick_split(tiles_v, s.D, p.rows_pad / 64, p.segs, pairs,
                        p.pieces == 1 ? (int)std::min<size_t>(32, std::max<size_t>(1, s.dw32_floats / p.dw_slab)) : 1, p.bn_dw, p.dw_most);
        // (fewer rows may count than there are: the device may want more ranges than the host)
        if (p.dx_most > 1) p.dx_most = (int)std::min<size_t>(32, s.dx32_floats / p.slab);
    }
    // ROW saves a second product of the logits but its warps wait for one another.  With against without it, bfloat16, 8192
    // rows, 4096 features, with gradients: 128 classes 136 us against 150, 256 classes 155 against 154 (float32 408 against 475).
    // The loss alone would gain from 65 classes on (1024 rows, 1024 features: 64 classes 15.5 us against 16.5, 256 classes 20.7
    // against 16.7), but then it would not be, to the bit, the loss that the call with gradients returns.
    p.by_row = s.V <= 256 && p.pieces == 1 && p.copy_piece >= s.V;
    if (!p.by_row) {
        // wider tiles until their pairs fit; 256 always do, since pieces are whole multiples of it
        p.bn_lse = xent_pick_bn(rows, std::min(s.V, p.copy_piece), s.D, p.segs, pairs, 32);
        while (p.bn_lse < 256 && (size_t)xent_slots(s.V, p.copy_piece, p.bn_lse) * p.rows_pad > s.partial_cap) p.bn_lse += 32;
    }
    return p;
}

// Whether the 32 columns from col0 on of a piece of N classes read the bias: the float32 copy of it ends at V rounded up to
// 256, the last piece's last tile may end behind that (its columns from N on are no classes).
CERT_BOTH inline bool xent_reads_bias(int col0, int N) { return col0 < N; }

// Column tile of a piece's probabilities.
inline int xent_prob_bn(const XentSizes &s, const XentPlan &p, int rows, int width, int pairs) {
    return p.by_row ? (s.V <= 64 ? 64 : s.V <= 128 ? 128 : 256) : xent_pick_bn(rows, width, s.D, p.segs, pairs, 64);
}

}  // namespace cert
