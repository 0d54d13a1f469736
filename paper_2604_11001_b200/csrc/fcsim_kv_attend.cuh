// Attention of one query token per request over a paged cache: parameters, and what the host side needs to launch it.
#pragma once
#include "fcsim_kv_device.cuh"

namespace fcsim_kv_dev {

constexpr int kThreads = 128;
constexpr int kWeightCtas = 6;    // CTAs of the weights' kernel on an SM (100 requests in f16, 4, 6, 8, 12: 53.6, 50.5, 50.5, 54.2 us in all)
constexpr int kMaxDevices = 64;   // devices for which answers of the runtime are remembered
constexpr int kMaxCtas = 4096;   // bound of the grid (the work is divided among the CTAs at run time)

struct AttendParams {
    Pool pool;
    const char* q;
    char* out;
    float* lse;
    const int32_t *table, *lengths;
    int32_t* status;
    int64_t q_row, q_head, table_row;
    int n_requests, n_heads, max_length, add_weight;
    int most_seen, first;  // tokens that a request sees at most: all, or a window and before it the `first` oldest (0 where all are seen)
    float scale;
    int tile_bits;       // tokens a CTA takes at once, of the variant
    // workspace
    int* counters;       // [workers], zero between calls: the parts that are done of the group that begins in a worker's stretch
    float* parts;        // [workers][2][heads of a tile][head_dim + 2]; a worker is a CTA or one of its four warps
    float* stats;        // add_weight: [n_requests][n_heads][4]: largest logit, its unit, 1 / sum, -
    float* logits;       // add_weight: per request [n_heads][tiles * tokens of a tile]
    int64_t logit_tiles; // what `logits` has room for, in tiles
};

// A variant of the kernel.  The functions return a cudaError_t.
struct AttendVariant {
    int (*launch)(const AttendParams&, int grid, cudaStream_t);
    int (*ctas_per_sm)(int device, int* out);  // asked once per device; also raises the kernel's limit of shared memory
    int head_cols, width;          // query heads and elements of its tile
    int tile_bits;                 // its tokens: 64 or 128
};

// The variant for a type of q, a type of cache, a head width and a group of query heads per kv head, with first tokens before a window or without.
AttendVariant attend_variant_f16(int head_dim, int group, bool first);
AttendVariant attend_variant_bf16(int head_dim, int group, bool first);
AttendVariant attend_variant_f16_e4m3(int head_dim, int group, bool first);
AttendVariant attend_variant_bf16_e4m3(int head_dim, int group, bool first);
int launch_weights(const AttendParams&, int grid, cudaStream_t);

}  // namespace fcsim_kv_dev
