// Which kernel a call of the 4-bit layer takes, how its work is cut and what scratch the arg-max wants: functions of its sizes alone.  Host code,
// in a header of its own so that the tests can compile it without the kernels.
#pragma once
#include <algorithm>
#include <stddef.h>
#include <stdint.h>

#include "../../include/whalesplit.h"

namespace ws {

constexpr int W4_MAX_ROWS = WS_W4_MAX_ROWS;
constexpr int64_t W4_MAX_PITCH = WS_W4_MAX_PITCH;                            // 16 rows are addressed with 31 bits
constexpr int W4_MAX_CLASSES = WS_W4_MAX_CLASSES;                            // a whole last group's biases are addressed with 32 bits, the last KiB of them left over
constexpr int W4_STEP = 128;                 // features that the lanes of a wave cover with 16 bytes of codes each
constexpr int W4_FEW_WAVES = 8;              // of a workgroup of w4_few
constexpr int W4_FEW_MOST = 2048;            // 16 classes x 32 rows that w4_few takes at most, whatever the number of features
constexpr int W4_MAX_PARTS = 4096;           // candidates of a row at most
constexpr int W4_STREAM_GROUPS = 256;        // workgroups of w4_stream at most, one to a compute unit
constexpr size_t W4_STREAM_LDS = 160 * 1024;

// How a call is run.  us of the launch, fp32 logits of bf16 features, codes not in any cache (one MI355X); - where a kernel cannot run:
//   rows x features x classes    w4_stream RING 1, 2    w4_few       w4_tiles
//    1 x 2048 x 100000           24.0  24.9             29           35
//   16 x 2048 x 100000           27.0  27.2             31           37
//   32 x 2048 x 100000           31.4  33.9             51           40
//    1 x  512 x 100000            8.2  10.3             10.7         11.9
//    1 x 2048 x 12500             8.2   7.6              6.6         11.6
//   16 x 2048 x 12500             9.6                    7.4         12.3
//   32 x 2048 x 12500            12.2  11.3              9.0         13.0
//   32 x 2048 x 16000            12.6                    9.7         13.2
//   32 x 2048 x 20000            13.2                   15.6         13.4
//    1 x 8192 x 12500            24.5  17.0             28           37
//    1 x 4096 x 4000             10.3   8.9              5.4         17.8
//    1 x 4096 x 1000             10.1   8.6              4.8         17.4
//    8 x  512 x 2000              3.2   4.8              3.9          4.7
//   64 x  512 x 12500                                    7.8          6.3
//   64 x 1024 x 1000                                     4.9          7.7
//   64 x 1024 x 12500                                    8.4          8.7
//   40 x 2048 x 12500                                   12.2         12.5
//   64 x 2048 x 12500                                   14.3         13.4
//   96 x 2048 x 12500                                   19.7         17.8
//  128 x 2048 x 3000                                     7.9         11.7
//  256 x 2048 x 3000                                    12.3         11.9
//   64 x 4096 x 6000                                    15.2         21.3
//   96 x 4096 x 6000                                    21.4         21.6
//  128 x 4096 x 6000                                    27.3         21.5
//   64 x 4096 x 12500                                   29.3         22.0
//  256 x 4096 x 1000                                     8.7         19.2
//  128 x 8192 x 1000                                    12.4         34
//  256 x 8192 x 4000                                    75           36
//   19 x 4096 x 100000          50.6                    97           82
//   20 x 4096 x 100000           -                      94           82
//   32 x 4096 x 100000           -                     102           84
//   19 x 4096 x 12500           19.1                    16.5         21.4
//   20 x 4096 x 12500            -                      16.7         21.5
//    9 x 8192 x 12500           20.7 (RING 2)           31           38
//   10 x 8192 x 12500            -                      31           38
//   32 x 8192 x 12500            -                      45           39
//    9 x 8192 x 100000         102                                  160
//   10 x 8192 x 100000           -                                  160
// A wave of w4_stream takes whole rows of 16 classes: with few of them most waves have nothing to do, and w4_few shares the rows out, while its
// workgroups fit the compute units at once.  Short rows stay on w4_stream, or with more rows of the batch than it holds on w4_tiles, whose time per
// step hardly depends on how many tiles there are: w4_few is faster for less than two rounds of its workgroups (17 to 32 rows of 8192 features and
// 782 tiles of classes are three, and still go there: 45 us where w4_tiles takes 39).
// What w4_stream takes is bounded by LDS, which holds the features of all rows: 19 rows of 4096, 9 of 8192.  One more row, on another kernel,
// takes up to 1.6 times as long; features in pieces would move that border.
enum W4Way { W4_STREAM, W4_FEW, W4_TILES };
struct W4Plan {
    W4Way way;
    int groups;                              // workgroups along the classes
    int ring;                                // w4_stream
    int S, CT, row_groups;                   // w4_few
    int NT;                                  // w4_tiles
    bool wide;                               //   eight waves, not four
};

static size_t w4_stream_lds(int B, int D) {
    const size_t steps = (D + W4_STEP - 1) / W4_STEP;
    return 4 * (((size_t)B * (64 * steps + 16) + 255) & ~(size_t)255);
}

static void plan_w4_tiles(W4Plan& p, int B, int C, bool top1) {
    const int64_t tiles = ((int64_t)C + 15) / 16;
    const int row_tiles = (B + 15) / 16;
    // Blocks of rows of one height, up to 8 tiles of 16 with CT = 4 tiles of classes, up to 4 with CT = 2; eight waves to a workgroup, or four.  The
    // tall ones for logits only (the arg-max's candidates take registers, too: 256 x 2048 x 100 000 153 us with 6 tiles, 134 with 4), and
    // whatever is larger only while there are workgroups for most compute units (80 x 2048 x 50 000: 45 us with four waves, 42 with eight);
    // two tiles of 16 rows if that makes a workgroup for each at most (64 x 4096 x 12 500 29.3 us with four, 22.0; 128 of these rows 30.4, 33.5).
    auto shape = [&](int most_rows, int classes) {
        const int blocks = (row_tiles + most_rows - 1) / most_rows;
        p.NT = (row_tiles + blocks - 1) / blocks;
        p.groups = (int)((tiles + classes - 1) / classes);
        return (int64_t)p.groups * blocks;
    };
    p.wide = (!top1 && row_tiles > 4 && shape(8, 32) >= 160) || shape(4, 16) >= 160;
    if (!p.wide && shape(2, 8) > 256) shape(4, 8);
    if (p.NT <= 4) p.NT = p.NT <= 2 ? 2 : 4;
}

static W4Plan w4_plan(int B, int D, int C, bool top1) {
    W4Plan p = {W4_TILES, 0, 1, 1, 1, 1, 0, false};
    const int64_t tiles = ((int64_t)C + 15) / 16;
    const int steps = (D + W4_STEP - 1) / W4_STEP;
    const bool fits = B <= 32 && w4_stream_lds(B, D) <= W4_STREAM_LDS;
    const int row_blocks = (B + 31) / 32;
    const int64_t most = fits ? (steps <= 32 ? 1024 : 512) : steps <= 8 ? W4_FEW_MOST : steps <= 16 ? 1536 : 1024;      // 16 classes x 32 rows shared out
    if (steps >= 8 && steps <= 8 * W4_FEW_WAVES && tiles * row_blocks <= most) {
        p.way = W4_FEW;
        while (W4_FEW_WAVES * p.S < steps) p.S *= 2;
        // as many classes to a workgroup as the registers hold, while there are workgroups for most compute units; with the 32 rows' features in
        // LDS one workgroup fits a unit, and more of them than units would go one after the other (32 x 4096 x 6000 13.4 us, 9.5)
        p.CT = p.S <= 2 ? 4 : p.S == 4 ? 2 : 1;
        if (p.S > 1 && (B <= 16 ? tiles < 192 * p.CT : tiles * row_blocks <= 256)) p.CT = 1;
        p.groups = (int)((tiles + p.CT - 1) / p.CT);
        // blocks of rows side by side as far as there are compute units, evenly many one after the other
        const int side = p.groups < 256 ? 256 / p.groups : 1, turns = (row_blocks + side - 1) / side;
        p.row_groups = (row_blocks + turns - 1) / turns;
    } else if (fits) {
        p.way = W4_STREAM;
        p.groups = tiles < W4_STREAM_GROUPS ? (int)tiles : W4_STREAM_GROUPS;
        p.ring = steps > 32 && tiles <= 1024 ? 2 : 1;
    } else {
        plan_w4_tiles(p, B, C, top1);
    }
    return p;
}

// Candidates of a row: one of each workgroup along the classes.  w4_tiles' workgroups walk the groups, and with very many rows there are fewer
// of them: a launch counts its threads with 32 bits.
static int w4_parts(const W4Plan& p, int B) {
    int parts = p.groups < W4_MAX_PARTS ? p.groups : W4_MAX_PARTS;
    if (p.way == W4_TILES)
        while ((int64_t)parts * ((B + 31) / 32) > 1 << 20) parts /= 2;
    return parts;
}

// The most of them that any number of features makes.
static int w4_most_parts(int B, int C) {
    const int64_t tiles = ((int64_t)C + 15) / 16;
    W4Plan p = {W4_TILES, 0, 1, 1, 1, 1, 0, false};
    plan_w4_tiles(p, B, C, true);
    int64_t most = w4_parts(p, B);
    if (B <= 32) most = std::max(most, std::min<int64_t>(tiles, W4_STREAM_GROUPS));
    if (tiles * ((B + 31) / 32) <= W4_FEW_MOST) most = std::max(most, tiles);
    return (int)most;
}

}  // namespace ws
