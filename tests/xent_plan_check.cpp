// Goes through the linear cross entropy's host arithmetic as a call does and compares every extent with its buffer.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <cmath>

#include "../paper_2507_20055_b200/csrc/xent_plan.cuh"

using namespace cert;

static bool fits(const char *what, long long max_rows, long long rows, long long d, long long v, int type, bool direct, long long used, long long has) {
    if (used <= has) return true;
    std::printf("%s: %lld of %lld, max_rows %lld rows %lld features %lld classes %lld type %d in place %d\n", what, used, has, max_rows, rows, d, v,
                type, (int)direct);
    return false;
}

// The extents of one call; false where one leaves its buffer.
extern "C" int check_call(int max_rows, int rows, int d, int v, int type, int direct, int grad, int pairs) {
    const XentSizes s = xent_sizes(max_rows, d, v, type, true);
    const XentPlan p = xent_plan(s, rows, direct != 0, grad != 0, pairs);
#define FITS(what, used, has) if (!fits(what, max_rows, rows, d, v, type, direct != 0, (long long)(used), (long long)(has))) return 0
    if (!p.by_row) {
        long long slots = 0;
        for (int c0 = 0; c0 < v; c0 += p.copy_piece) {
            const int width = std::min(p.copy_piece, v - c0);
            slots += 2 * xent_div(width, p.bn_lse);
            for (int col0 = 0; col0 < width; col0 += 32)
                if (xent_reads_bias(col0, width)) FITS("bias read for statistics", c0 + col0 + 32, s.Vp);
        }
        FITS("slots", slots * p.rows_pad, s.partial_cap);
        FITS("slots counted", xent_slots(v, p.copy_piece, p.bn_lse), slots);
        FITS("slots counted", slots, xent_slots(v, p.copy_piece, p.bn_lse));
    }
    if (!direct) FITS("copied weights", p.copy_piece * s.row_bytes, s.wbuf_bytes);
    FITS("rows", p.rows_pad, s.rows_pad);
    if (grad) {
        FITS("probabilities", (long long)p.rows_pad * s.parts * 2 * p.piece, s.prob_bytes);
        FITS("column sums", (long long)p.rows_pad / 32 * p.piece, s.colsum_floats);
        FITS("dx sums", (long long)p.dx_most * (long long)p.slab, s.dx32_floats);
        if (p.dw_most > 1) FITS("dW sums", (long long)p.dw_most * (long long)p.dw_slab, s.dw32_floats);
        for (int c0 = 0; c0 < v; c0 += p.piece) {
            const int width = std::min(p.piece, v - c0), bn = xent_prob_bn(s, p, rows, width, pairs);
            const int end = (int)std::min<long long>(xent_up(width, bn), p.by_row ? bn : p.piece);
            for (int col0 = 0; col0 < end; col0 += 32)
                if (p.by_row || xent_reads_bias(col0, width)) FITS("bias read for probabilities", c0 + col0 + 32, s.Vp);
        }
        FITS("pieces", p.piece, p.copy_piece);
        FITS("piece in tiles of 256", p.piece % 256, 0);
    }
    FITS("copied piece in tiles of 256", p.copy_piece % 256, 0);
    return 1;
}

extern "C" int sweep(unsigned seed, int calls, int pairs) {
    std::mt19937 g(seed);
    auto log_between = [&](double lo, double hi) { return (int)std::lround(std::exp(std::uniform_real_distribution<double>(std::log(lo), std::log(hi))(g))); };
    int bad = 0;
    for (int i = 0; i < calls; ++i) {
        const int max_rows = log_between(1, 65536), rows = std::min(max_rows, g() % 3 ? log_between(1, max_rows + 0.4) : max_rows);
        const int d = std::max(1, g() % 4 ? log_between(8, 16384) / 8 * 8 : log_between(1, 16384)), v = log_between(17, 600000);
        const int type = (int)(g() % 3);
        const bool direct = type != CERT_TYPE_F32 && g() % 2 && d % 8 == 0;
        bad += !check_call(max_rows, std::max(1, rows), d, v, type, direct, (int)(g() % 2), pairs);
    }
    return bad;
}

int main(int argc, char **argv) {
    const int bad = sweep(1, argc > 1 ? std::atoi(argv[1]) : 100000, 74);
    std::printf("%d calls out of range\n", bad);
    return bad != 0;
}
