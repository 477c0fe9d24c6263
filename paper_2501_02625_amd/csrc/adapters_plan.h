// Rules that choose between ways to run the low-rank adapters: plain host functions, for the launchers and for a host program that asks
// which way a call goes.
#pragma once
#include <cstdint>

namespace halo {
namespace adapters {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Tokens of a workgroup of wide_kernel (adapters_wide.hip), for b tokens and a result of `wide` columns: 256 (128 above rank 64: the thin
// values' pieces take up to 96 KB of LDS) once such tiles times strips of 512 columns are as many as the compute units (3417 x 11976, rank 64: 60 us,
// shorter ones 85), 64 down to two strips a compute unit, 16 below: 19.5 us instead of 21.8 at 2048 x 4096, rank 16, which is one strip; but
// 45.6 instead of 39 at 1547 x 12984, rank 32, with 2.5 of them.  Above rank 64 tiles of 64 have no place between: where they make two strips a
// compute unit, tiles of 128 make one.
inline int wide_tile_tokens(int64_t b, int64_t wide, int max_rank) {
    constexpr int64_t kComputeUnits = 256;
    const int64_t strips = ceil_div(wide, 512);
    const int tall = max_rank > 64 ? 128 : 256;
    if (ceil_div(b, tall) * strips >= kComputeUnits) return tall;
    return tall > 128 && ceil_div(b, 64) * strips >= 2 * kComputeUnits ? 64 : 16;
}

}  // namespace adapters
}  // namespace halo
