// Launchers of the low-rank adapters of many requests (adapters.hip) and of dropout (dropout.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "philox.h"

namespace halo {

constexpr int kMaxAdapterRank = 128;
constexpr int kMaxAdapterSlots = 32768;       // with the most cuts of 2^22 tokens still a grid dimension (65535)

// The pool: U bf16 [slots x max_rank x m], V bf16 [slots x n x max_rank], of which adapter a's first ranks[a] rows of U and columns of
// V are used (ranks null: max_rank); scale fp32 [slots] or null (1).  adapter_of [b]: the adapter of each token, none where it is not
// in [0, slots).
struct AdapterPool {
    const uint16_t* U;
    const uint16_t* V;
    const int32_t* ranks;
    const float* scale;
    const int32_t* adapter_of;
    int64_t b, m, n;
    int slots, max_rank;
};

struct AdaptersFwd {
    AdapterPool pool;
    const uint16_t* X; int64_t ld_x;
    const void* base; int64_t ld_base;       // null: zero
    void* Y; int64_t ld_y;
    int out_f32;                             // base and Y fp32 instead of bf16
    float* T;                                // [b x max_rank]
    DropoutMask drop;
    void* workspace;
};

struct AdaptersBwd {
    AdapterPool pool;
    const uint16_t* E; int64_t ld_e;
    const uint16_t* X; int64_t ld_x;
    const float* T;
    const void* base; int64_t ld_base;
    void* EX; int64_t ld_ex;                 // null: not wanted, and so the next two
    int out_f32;
    float* GU;
    float* GV;
    DropoutMask drop;
    void* workspace;
};

size_t adapters_fwd_workspace(int64_t b, int64_t m, int64_t n, int slots, int max_rank);
size_t adapters_bwd_workspace(int64_t b, int64_t m, int64_t n, int slots, int max_rank, bool drop);
hipError_t launch_adapters_fwd(const AdaptersFwd& a, hipStream_t s);
hipError_t launch_adapters_bwd(const AdaptersBwd& a, hipStream_t s);

struct DropoutArgs {
    const void* in; int64_t ld_in;
    const void* residual; int64_t ld_res;    // null: none
    void* out; int64_t ld_out;
    int64_t rows, cols;
    int f32;                                 // all three fp32 instead of bf16
    DropoutMask drop;
};
hipError_t launch_dropout(const DropoutArgs& a, hipStream_t s);

}  // namespace halo
