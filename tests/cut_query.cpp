// What librkblock would take for a size (csrc/rkb_cut.h), for the tests: see cuts.py.
#include "rkb_cut.h"

using namespace rkb;

static void put(int *out, const cut &c)
{
    out[0] = c.tm;
    out[1] = c.bufs;
    out[2] = c.splits;
}

// few rows; together; two parts; the pair's buffers and splits; tile rows, buffers and splits of g and u, dx, dwg and dwu
extern "C" void gated_cuts(int64_t rows, int64_t d, int64_t f, int *out)
{
    const cut sums = sums_cut(rows, d, f);
    const backward_cut c(rows, d, f);
    out[0] = few_rows_win(rows, f, d, sums.us);
    out[1] = c.together;
    out[2] = c.fine;
    out[3] = c.both.bufs;
    out[4] = c.both.splits;
    put(out + 5, sums);
    put(out + 8, c.x);
    put(out + 11, c.w);
}

extern "C" void weight_grad_cut(int64_t rows, int64_t n, int64_t k, int *out) { put(out, choose_cut(n, k, rows, 1, 1, 1, false)); }
