// How a product of 8-bit integers is divided (cf_linear.hip): the ways, the choice between them, which workgroup takes what.  Nothing but functions of
// plain values, so that a host compiler can run what the library and its kernels run.
#ifndef CF_LINEAR_PLAN_H
#define CF_LINEAR_PLAN_H

namespace cf {
namespace linear {

// The ways to divide a product.  What a step of 128 codes of the sum takes a workgroup that has a compute unit for itself, and one among others on it, in
// us; a call takes about 3 us more.  (Measured at 4096 to 11008 codes and 1 to 8192 rows, all ways at each; a wavefront of the tiles waits for its
// operands and multiplies by turns, so that a step of a tile that is alone takes 1.5 times as long as the matrix units need for it or more.  The way that they
// give takes up to 7 % longer than the best one at 18 shapes of 65 to 8192 rows and 512 to 12288 outputs: 256 x 4096 -> 6144 16.5 us, 15.4 in tiles of
// 64 x 64.  Under many rows with few outputs reading the rows counts, which they do not know: 4096 x 4096 -> 128 12.5 us, 10.3 in blocks of 64 x 64.)
struct Way {
    int rows, cols, threads;       // of a workgroup
    bool tiles;
    float alone, among;
};
constexpr Way kWays[] = {
    {16, 16, 256, false, 0.085f, 0.087f}, {16, 32, 256, false, 0.145f, 0.16f}, {32, 32, 256, false, 0.17f, 0.145f},
    {64, 32, 256, false, 0.23f, 0.23f},   {64, 64, 256, false, 0.27f, 0.28f},  {64, 64, 256, true, 0.31f, 0.26f},
    {128, 64, 256, true, 0.42f, 0.44f},   {256, 128, 512, true, 1.0f, 1.11f},  {256, 256, 512, true, 1.5f, 1.87f},
};
constexpr int kNumWays = sizeof kWays / sizeof *kWays;

constexpr int blocks_of(int n, int size) { return (n + size - 1) / size; }

// index of the way whose steps take the least time
inline int way_of(int n_out, int rows, int cus)
{
    int best = 0;
    double least = 0;
    for (int i = 0; i < kNumWays; ++i) {
        const Way &w = kWays[i];
        const long long workgroups = (long long)blocks_of(rows, w.rows) * blocks_of(n_out, w.cols), on_one = (workgroups + cus - 1) / cus;
        const float shared = (float)on_one * w.among;
        const double step = on_one == 1 && workgroups * 4 <= cus * 3 ? w.alone : w.alone > shared ? w.alone : shared;
        if (i == 0 || step < least) best = i, least = step;
    }
    return best;
}

// Workgroup i runs on die i mod 8.
struct Block {
    int m, n;                      // of the rows, of the outputs; n is none of the product's where a workgroup has nothing to do
};

// Few rows: each die takes every eighth block of outputs, whose row blocks follow each other there.  What is left of the outputs, up to seven blocks of
// them, is dealt to all dies alike, block by block of the rows: whole outputs would be the work of some dies alone, without the others' compute units
// (8192 x 4096 -> 128, two blocks, on two dies: 42.2 us, on eight 15.2; 4096 x 4096 -> 64 18.1 and 8.0).  All outputs dealt like that, a range of them
// to a die, take 3 to 7 % more where there are hundreds (200 x 4096 -> 4096 11.7 us, 10.9).
constexpr unsigned left_of(int row_blocks, int col_blocks) { return (unsigned)(col_blocks & 7) * (unsigned)row_blocks; }
constexpr unsigned stream_grid(int row_blocks, int col_blocks)
{
    return 8 * ((unsigned)(col_blocks >> 3) * (unsigned)row_blocks + (left_of(row_blocks, col_blocks) + 7) / 8);
}
constexpr Block stream_block(unsigned index, int row_blocks, int col_blocks)
{
    const unsigned die = index & 7, turn = index >> 3, rows = (unsigned)row_blocks, whole = (unsigned)(col_blocks >> 3) * rows;
    if (turn < whole) return Block{(int)(turn % rows), (int)(8 * (turn / rows) + die)};
    const unsigned unit = die * ((left_of(row_blocks, col_blocks) + 7) / 8) + turn - whole;
    return Block{(int)(unit % rows), (int)(unit / rows) + (col_blocks & ~7)};
}

}  // namespace linear
}  // namespace cf

#endif
