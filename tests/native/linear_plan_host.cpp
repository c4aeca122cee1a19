// The division of the integer products (cf_linear_plan.h) as the host compiler sees it, for tests.
#include "../../paper_2508_18850_amd/csrc/cf_linear_plan.h"

using namespace cf::linear;

extern "C" {

int lp_ways() { return kNumWays; }
int lp_way(int n_out, int rows, int cus) { return way_of(n_out, rows, cus); }
void lp_sizes(int way, int *sizes) { sizes[0] = kWays[way].rows, sizes[1] = kWays[way].cols, sizes[2] = kWays[way].tiles; }
int lp_stream_grid(int row_blocks, int col_blocks) { return (int)stream_grid(row_blocks, col_blocks); }
void lp_stream_blocks(int row_blocks, int col_blocks, int *m, int *n)
{
    for (int i = 0; i < lp_stream_grid(row_blocks, col_blocks); ++i) {
        const Block b = stream_block(i, row_blocks, col_blocks);
        m[i] = b.m, n[i] = b.n;
    }
}

}  // extern "C"
