// Interface between the host code of the page operators and their kernels.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace taper {

constexpr int kLayersPerLaunch = 64, kMovesInArguments = 256;

struct PoolPointers {
    void* base[kLayersPerLaunch];
};
struct PageMove {
    int32_t src, dst;
};
struct MoveArguments {  // short lists travel with the launch
    PageMove move[kMovesInArguments];
};
// A destination page of a join: n_tokens tokens of sequence seq from token0 on.
struct PackPage {
    int32_t dst, seq, token0, n_tokens;
};
struct PackArgs {
    const PackPage* pages;
    const int32_t* bt;         // [n_seqs][bt_stride]
    const int32_t* run_start;  // [n_seqs + 1] CSR over runs (the prefix, then the segments)
    const int32_t* run_token;  // first token of each run
    const int32_t* run_entry;  // block-table entry its pages begin at
    int32_t bt_stride, n_pages, kind, n_heads, dim;
};

hipError_t launch_pages_copy(const PoolPointers& pools, int n_layers, const PageMove* list /* device, or null: in args */, const MoveArguments* args,
                             int64_t n_moves, int64_t page_bytes, hipStream_t s);
hipError_t launch_pages_pack(const PoolPointers& pools, int n_layers, const PackArgs& a, hipStream_t s);

}  // namespace taper
