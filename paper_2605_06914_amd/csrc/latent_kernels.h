// Interface between the host code of the latent-cache operators and their kernels (device pointers only).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "taper_latent.h"

namespace taper {

constexpr int kLatentTileTokens = 64;  // tokens a workgroup of the decode kernel takes at a time
constexpr int kLatentTileRows = 128;   // query rows it holds at most
constexpr int kRopeDim = 64;

struct LatentShape {
    int n_heads, latent_dim, head_dim;
    float scale_log2e;  // scale * log2(e)
};

struct PartStats {             // of a partial row
    float m, l;               // running max in log2 units, sum
    signed char exponent[8];  // of each eighth of its columns
};
struct LatentDecodeArgs {
    const int32_t* bt;              // [n_seqs][bt_stride]
    const taper_latent_item* items;
    const int32_t* piece_start;     // [n_seqs + 1]
    const int32_t* piece_row;
    void* q_lat;                    // bf16 [n_seqs * n_heads][latent_dim + 64]
    void* q_rest;                   // bf16 [n_seqs * n_heads][latent_dim]: what q_lat's rounding took away (written where lse is wanted)
    PartStats* stats;               // [n_partial_rows]
    void* part;                     // f16 [n_partial_rows][latent_dim]: rows divided by their own sum and their columns' powers of two
    const void* q;
    const void* w_up;
    const void* pages;
    void* out;
    float* lse;
    int32_t bt_stride, n_seqs, n_items;
};
hipError_t launch_latent_decode(const LatentShape& sh, const LatentDecodeArgs& a, hipStream_t s);

// The normaliser of a row that sees few tokens feels the rounding of their keys, which averages out over many (at 128 tokens and unit
// scores it is off by 2e-5 of some 5): pages that hold positions below this have low parts of their keys, which such rows add.
constexpr int kLowPositions = 128;

// A tile of a prompt's query rows.
struct PromptTile {
    int32_t row0, n_rows;        // rows of q
    int32_t first_pos;           // position of the first row's token in its sequence
    int32_t prefix_len;          // tokens of the shared prefix
    int32_t prefix_e, suffix_e;  // expanded pages of the prefix and of the private tokens begin here (even numbers)
    int32_t page_begin, page_end;  // the pages (of the prefix, an even number, then private ones) this tile's item meets; page_begin is even
    int32_t part_row;            // partial rows of head 0, or -1: the item is its rows' only one and writes the result
    int32_t n_pieces;            // items of the same rows; their partial rows are n_rows apart
    int32_t bundle, n_bundle;    // this item is one of n_bundle from number `bundle` on that meet the same keys (see tile_of_block)
};
struct PromptArgs {
    const int32_t* e_page;       // [n_expanded] physical page of an expanded page
    const int32_t* e_valid;      // [n_expanded] tokens of it that exist
    const int32_t* e_low;        // [n_expanded] number of its page of low parts, -1: it has none
    const PromptTile* tiles;     // [n_tiles], longest first
    const PromptTile* merges;    // [n_merges] row tiles whose keys are cut into pieces
    void* kv;                    // [head of the group][n_expanded / 2][K, K, V of a pair of pages] (see the kernels)
    void* k_low;                 // f16 [head of the group][n_low][K]: 2^11 times what the rounding of keys took away, where lse is wanted
    int32_t* format;             // [head of the group][n_chunks][keys, values]: 1 where four pages are bf16 instead of half precision
    float2* ml;
    float* part;                 // [head][partial rows][head_dim]
    const void* q;
    const void* w_up;
    const void* pages;
    void* out;
    float* lse;
    int32_t n_chunks, units;     // fours of expanded pages; compute units
    int32_t n_low;               // pages of low parts
    int32_t n_expanded, n_tiles, n_merges, n_partial_rows;  // partial rows of one head
    int32_t heads_at_once;
};
hipError_t launch_latent_prompt(const LatentShape& sh, const PromptArgs& a, hipStream_t s);

hipError_t launch_latent_append(int latent_dim, int64_t n, const void* latent, int64_t latent_stride, const void* rope, int64_t rope_stride,
                                const int64_t* slots, void* pages, int64_t n_slots, hipStream_t s);

}  // namespace taper
