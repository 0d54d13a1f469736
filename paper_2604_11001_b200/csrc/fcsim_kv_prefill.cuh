// Attention of several query tokens per request over a paged cache: parameters, and what the host side needs to launch it.
#pragma once
#include "fcsim_kv_device.cuh"

namespace fcsim_kv_dev {

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
    int heads_a_tile, head_tiles;    // query heads that share a block's rows; such tiles of a kv head
    int tokens_a_block;
    float scale;
    // workspace
    int* counters;  // [CTAs][2], zero between calls: the parts that are done of the block that begins in a CTA's stretch
    float* parts;   // [CTAs][2][tiles of rows][head_dim of the variant + 2][128]
};

// A variant of the kernel.  The functions return a cudaError_t.
struct PrefillVariant {
    int (*launch)(const PrefillParams&, int grid, int device, cudaStream_t);
    int rows, keys, width;  // rows of a block, keys of a tile, head_dim at most
};

PrefillVariant prefill_variant_f16(int head_dim);
PrefillVariant prefill_variant_bf16(int head_dim);
PrefillVariant prefill_variant_f16_e4m3(int head_dim);
PrefillVariant prefill_variant_bf16_e4m3(int head_dim);

}  // namespace fcsim_kv_dev
