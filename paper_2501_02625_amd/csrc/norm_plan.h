// The rules by which the norm's gradient forms the sums of the columns: plain host functions, for the launcher, for the workspace query and for a
// host program that asks.
#pragma once
#include <cstdint>

namespace halo {

// Workgroups of a launch that sums columns: the threads of a compute unit that they hold are 1024, or 512 where a row takes more than 4096 columns
// (1024 lanes, or four groups of 512): every one more writes a part of the sums and has fewer rows to have on their way.  EX, G_W and
// G_B in bf16, 256 / 512 / 768 workgroups: 8192 x 4096 (512 lanes) 53.8 us / 47.4 / 53.6, 2048 x 8192 with 1024 lanes 27.1 / 36 / 42, 1024 x
// 14336 (512 lanes, four groups) 38.4 / 46.4 / 53.6, 8192 x 512 12.1 / 10.4 / 9.8.
constexpr int64_t kMostNormBwd = 512;
inline int64_t most_norm_bwd(int64_t cols) { return cols > 4096 ? kMostNormBwd / 2 : kMostNormBwd; }
// Rows that a workgroup of these has at once.
inline int norm_bwd_teams(int64_t cols) { return cols <= 64 ? 32 : cols <= 128 ? 16 : cols <= 256 ? 8 : cols <= 1024 ? 4 : 1; }

// Few rows: E_X and the sums of the columns in one launch, by workgroups of their own, which read E and X once more.  512 rows at most, 256 up
// to 512 columns, and in fp32 432 from 4097 to 8192, from where on the second reading costs more than the second launch.
// Layer norm with a base in a graph, rows x columns, one launch / parts and their sum:
//   bf16  64 x 512 4.5 us / 6.0, 256 x 512 5.3 / 6.5, 512 x 256 6.6 / 6.2 and 512 x 64 6.4 / 5.6 (not taken), 512 x 2048 7.3 / 11.2, 512 x 4096
//         7.4 / 16.2, 512 x 8192 13.1 / 16.8, 512 x 14336 21.6 / 29.1, 512 x 32768 42 / 49; not taken 768 x 4096 9.6 / 16.3, 1024 x 4096 12.6 /
//         16.4, 1024 x 8192 21.4 / 20.6
//   fp32  256 x 512 6.6 / 6.6, 256 x 64 6.5 / 5.6 (taken: the host's part of a second launch, 3 us, is not in these), 512 x 512 9.4 / 6.6 (not
//         taken), 512 x 4096 13.1 / 16.5; 5000 columns, 416 rows 14.2 / 15.6, 448 16.7 / 15.8, 512 17.8 / 16.6; 8192, 384 17.0 / 18.1, 416 19.4 /
//         18.7, 512 22.3 / 20.6; 512 x 14336 37 / 42, 512 x 32768 114 / 128; 1024 x 8192 36.9 / 29.4 (not taken)
inline bool norm_bwd_one_launch(int64_t rows, int64_t cols, bool f32) {
    return rows > 0 && rows <= (cols <= 512 ? 256 : f32 && cols > 4096 && cols <= 8192 ? 432 : 512);
}

// Rows without room in registers for the sums beside them: these have a launch of their own.
constexpr bool norm_bwd_apart(int64_t cols, bool f32) { return cols > (f32 ? 8192 : 16384); }

// Of more rows: the parts that are written to the workspace, at most.
inline int64_t norm_bwd_parts(int64_t rows, int64_t cols, bool f32) {
    const bool apart = norm_bwd_apart(cols, f32);
    const int64_t rows_each = apart ? 16 : norm_bwd_teams(cols), most = apart ? 2048 / ((cols + 511) / 512) : most_norm_bwd(cols);
    const int64_t parts = (rows + rows_each - 1) / rows_each;
    return parts < most ? parts : most;
}

}  // namespace halo
