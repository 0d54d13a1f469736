// Attention of several query tokens per request over a paged cache: parameters, and what the host side needs to launch it.
#pragma once
#include <cuda.h>

#include "fcsim_kv_device.cuh"

namespace fcsim_kv_dev {

// Tiles of keys after which a walk's output is put aside and begun again (a multiple of 2).  The tensor core cuts its sums off: up to 2^-23 of the sum is
// lost at each of 16 additions a tile (8 over width 128), always towards zero, 2^-12 in so many tiles.  (With 2 048 of them outputs were 1.7e-3 too small.)
constexpr int kAsideTiles = 128;

struct PrefillParams {
    Pool pool;
    const char* q;
    char* out;
    float* lse;
    const int32_t *starts, *table, *lengths;
    int32_t* status;
    int64_t q_row, q_head, table_row;
    int n_rows, n_requests, n_heads, max_length;
    int window, first;               // both 0 where everything is seen; their sum is below max_length
    int box, kept;                   // tokens of a page that one bulk copy brings, 0: none do; `first` rounded up to a multiple of them
    int key_dim, query_tokens;       // tensor maps: whether slots come before heads; tokens of a box of q
    int heads_a_tile, head_tiles;    // query heads that share a block's rows; such tiles of a kv head
    int tokens_a_block;
    int aside;                       // whether a walk may be longer than kAsideTiles
    float scale;
    // workspace
    int* counters;  // [CTAs][2], zero between calls: the parts that are done of the block that begins in a CTA's stretch
    float* parts;   // [CTAs][2][tiles of rows][head_dim of the variant + 2][128]; with `aside`, behind these as much as for one of the 2
    // with `box`: [pages][heads, slots in the order of their strides][head_dim], and q
    CUtensorMap k_map, v_map, q_map;
};

// A variant of the kernel.  The functions return a cudaError_t.
struct PrefillVariant {
    int (*launch)(const PrefillParams&, int grid, int device, cudaStream_t);
    int rows, keys, width;  // rows of a block, keys of a tile, head_dim at most
    bool raw_rows;          // rows of the cache come as they are (or, of 8 bits, so wide that they lie as bulk copies bring them)
};

PrefillVariant prefill_variant_f16(int head_dim);
PrefillVariant prefill_variant_bf16(int head_dim);
PrefillVariant prefill_variant_f16_e4m3(int head_dim);
PrefillVariant prefill_variant_bf16_e4m3(int head_dim);

}  // namespace fcsim_kv_dev
