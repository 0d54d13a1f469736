// Paged key-value cache: validation and launches of append, attend and evict.  The C ABI is declared in
// include/fcsim_kv.h.
#include "fcsim_kv.h"

#include <math.h>

#include <algorithm>
#include <atomic>

#include "fcsim_kv_attend.cuh"

using namespace fcsim_kv_dev;

namespace {

thread_local int g_last_cuda_error = 0;

int cuda_status(cudaError_t e) {
    if (e == cudaSuccess) return FCSIM_OK;
    g_last_cuda_error = (int)e;
    return FCSIM_ECUDA;
}
int launched() { return cuda_status(cudaGetLastError()); }

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
// a stride in elements whose bytes are a multiple of 16, and not negative
bool good_stride(int64_t s, int bytes) { return s >= 0 && (s * bytes) % 16 == 0; }

// ------------------------------------------------------------------------------------------------ append
struct AppendParams {
    Pool pool;
    const char *q, *k, *v, *q_norm, *k_norm;
    char* q_out;
    const float* rope;
    const int32_t* positions;
    const int64_t* slots;
    int32_t* status;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head;
    int n_tokens, n_heads, rope_dim, n_positions, interleaved;
    float eps;
};

// One row (a head of a token of q, k or v) by a group of LPR lanes, 8 elements a lane.
template <class T, class C, int LPR>
__global__ void __launch_bounds__(256) fcsim_kv_append_kernel(const AppendParams p) {
    const int heads = p.n_heads + 2 * p.pool.n_kv, D = p.pool.head_dim;
    const int lane = threadIdx.x & (LPR - 1);
    const int64_t item = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) / LPR;
    const bool there = item < (int64_t)p.n_tokens * heads;
    const int token = there ? (int)(item / heads) : 0, j = there ? (int)(item - (int64_t)token * heads) : 0;
    const bool is_q = j < p.n_heads, is_v = j >= p.n_heads + p.pool.n_kv;
    const int h = is_q ? j : is_v ? j - p.n_heads - p.pool.n_kv : j - p.n_heads;
    const bool mine = there && lane * 8 < D;
    int position = 0;
    bool turned = p.rope != nullptr, good = true;
    if (turned) {
        position = p.positions[token];
        good = position >= 0 && position < p.n_positions;
        if (!good && there && lane == 0) flag(p.status, FCSIM_KV_BAD_POSITION);
    }
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (mine) {
        const char* src = is_q ? p.q + ((int64_t)token * p.q_row + (int64_t)h * p.q_head) * 2
                        : is_v ? p.v + ((int64_t)token * p.v_row + (int64_t)h * p.v_head) * 2
                               : p.k + ((int64_t)token * p.k_row + (int64_t)h * p.k_head) * 2;
        load8<T>(src + lane * 16, x);
    }
    const char* w = is_q ? p.q_norm : is_v ? nullptr : p.k_norm;
    float sum = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) sum += x[i] * x[i];
#pragma unroll
    for (int m = LPR / 2; m; m >>= 1) sum += __shfl_xor_sync(~0u, sum, m);
    if (w && mine) {
        float y[8];
        load8<T>(w + lane * 16, y);
        const float r = 1.0f / sqrtf(sum / (float)D + p.eps);
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = x[i] * r * y[i];
    }
    if (turned) {
        const int half = p.rope_dim / 2;
        const float* row = p.rope + (int64_t)(good ? position : 0) * p.rope_dim;
        float mate[8];
        // pairs half a rotation apart: the other element sits rope_dim / 16 lanes away, at the same place
        const int first = lane * 8 < half;
        const int other = first ? lane + p.rope_dim / 16 : lane - p.rope_dim / 16;
#pragma unroll
        for (int i = 0; i < 8; i++) mate[i] = __shfl_sync(~0u, x[i], other & (LPR - 1), LPR);
        if (mine && !is_v) {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const int e = lane * 8 + i;
                if (e < p.rope_dim) {
                    if (p.interleaved) {
                        if (!(i & 1)) {
                            const float c = row[e / 2], s = row[half + e / 2], a = x[i], b = x[i + 1];
                            x[i] = a * c - b * s;
                            x[i + 1] = b * c + a * s;
                        }
                    } else {
                        const int a = first ? e : e - half;
                        const float c = row[a], s = row[half + a];
                        x[i] = first ? x[i] * c - mate[i] * s : x[i] * c + mate[i] * s;
                    }
                }
            }
        }
    }
    if (!there) return;
    if (is_q) {
        if (!good) {
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] = 0;
        }
        if (mine) store8<T>(p.q_out + (((int64_t)token * p.n_heads + h) * D + lane * 8) * 2, x);
        return;
    }
    const int64_t slot = p.slots[token];
    if (slot < 0 || !good) return;
    if (slot >= (int64_t)p.pool.n_pages * p.pool.page_size) {
        if (lane == 0) flag(p.status, FCSIM_KV_BAD_PAGE);
        return;
    }
    const int page = (int)((uint32_t)slot / (uint32_t)p.pool.page_size);
    const int place = (int)((uint32_t)slot - (uint32_t)page * (uint32_t)p.pool.page_size);
    if (C::bytes == 1 && mine) {
        const float s = is_v ? p.pool.v_scale[h] : p.pool.k_scale[h];
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = x[i] / s;
    }
    char* dst = (is_v ? p.pool.v : p.pool.k) +
                (page * p.pool.stride_page + place * p.pool.stride_slot + h * p.pool.stride_head + lane * 8) * C::bytes;
    if (mine) store8<C>(dst, x);
    if (!is_v && lane == 0 && p.pool.weight)
        p.pool.weight[((int64_t)page * p.pool.n_kv + h) * p.pool.page_size + place] = 0.0f;
}

template <class T, class C>
int launch_append(const AppendParams& p, cudaStream_t stream) {
    const int lanes = p.pool.head_dim / 8;
    const int64_t rows = (int64_t)p.n_tokens * (p.n_heads + 2 * p.pool.n_kv);
    const int lpr = lanes <= 8 ? 8 : lanes <= 16 ? 16 : 32;
    const int64_t blocks = (rows * lpr + 255) / 256;
    if (blocks > 0x7fffffff) return FCSIM_EINVAL;
    if (lpr == 8) fcsim_kv_append_kernel<T, C, 8><<<(unsigned)blocks, 256, 0, stream>>>(p);
    else if (lpr == 16) fcsim_kv_append_kernel<T, C, 16><<<(unsigned)blocks, 256, 0, stream>>>(p);
    else fcsim_kv_append_kernel<T, C, 32><<<(unsigned)blocks, 256, 0, stream>>>(p);
    return launched();
}

// ------------------------------------------------------------------------------------------------ evict
struct EvictParams {
    Pool pool;
    const int32_t *table, *lengths, *budget, *new_table;
    int32_t *new_lengths, *kept, *status;
    int64_t table_row, new_row;
    int max_length, max_budget, recent, first, bytes;
};

__device__ __forceinline__ int length_of(const int32_t* lengths, int r, int max_length, int32_t* status) {
    int n = lengths[r];
    if (n < 0 || n > max_length) {
        flag(status, FCSIM_KV_BAD_LENGTH);
        n = n < 0 ? 0 : max_length;
    }
    return n;
}

// A weight as an unsigned key of the same order: NaN lowest, -0 as 0.
__device__ __forceinline__ uint32_t order_key(float w) {
    if (w != w) return 0;
    const uint32_t b = __float_as_uint(w + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// One kv head of one request by one CTA: the threshold bit by bit, then places by a running sum, then the copies.
__global__ void __launch_bounds__(256) fcsim_kv_evict_kernel(const EvictParams p) {
    const int r = blockIdx.y, h = blockIdx.x, tid = threadIdx.x;
    const int n = length_of(p.lengths, r, p.max_length, p.status);
    int budget = p.budget[r];
    if (budget < 0 || budget > p.max_budget) {
        flag(p.status, FCSIM_KV_BAD_BUDGET);
        budget = budget < 0 ? 0 : p.max_budget;
    }
    const int keep = min(n, budget), recent = min(p.recent, budget), first = min(p.first, budget - recent);
    // tokens [lo, hi) compete for `places`
    const int lo = keep == n ? n : first, hi = keep == n ? n : n - recent, places = keep - (n - hi) - lo;
    __shared__ int count;
    auto key = [&](int t) {
        const int page = p.table[r * p.table_row + t / p.pool.page_size];
        if (page < 0 || page >= p.pool.n_pages) {
            flag(p.status, FCSIM_KV_BAD_PAGE);
            return 0u;
        }
        return order_key(p.pool.weight[((int64_t)page * p.pool.n_kv + h) * p.pool.page_size + t % p.pool.page_size]);
    };
    uint32_t threshold = 0;
    if (places > 0) {
        for (int bit = 31; bit >= 0; bit--) {  // the largest threshold that at least `places` keys reach
            const uint32_t attempt = threshold | (1u << bit);
            int c = 0;
            for (int t = lo + tid; t < hi; t += 256) c += key(t) >= attempt;
            __syncthreads();
            if (tid == 0) count = 0;
            __syncthreads();
            atomicAdd(&count, c);
            __syncthreads();
            if (count >= places) threshold = attempt;
        }
    }
    int above = 0;
    for (int t = lo + tid; t < hi; t += 256) above += key(t) > threshold;
    __syncthreads();
    if (tid == 0) count = 0;
    __syncthreads();
    atomicAdd(&count, above);
    __syncthreads();
    const int ties = places - count;  // the oldest of the keys equal to the threshold
    int32_t* kept = p.kept + ((int64_t)r * p.pool.n_kv + h) * p.max_budget;
    if (tid == 0) {
        int at = 0, equal = 0;
        for (int t = 0; t < n; t++) {
            bool take = t < lo || t >= hi;
            if (!take && places > 0) {
                const uint32_t k = key(t);
                take = k > threshold || (k == threshold && equal++ < ties);
            }
            if (take) kept[at++] = t;
        }
        for (int i = keep; i < p.max_budget; i++) kept[i] = -1;
        if (h == 0) p.new_lengths[r] = keep;
    }
    __syncthreads();
    const int chunks = p.pool.head_dim * p.bytes / 16;
    for (int i = tid; i < keep * chunks; i += 256) {
        const int row = i / chunks, c = i % chunks, t = kept[row];
        const int page = p.table[r * p.table_row + t / p.pool.page_size];
        const int to = p.new_table[r * p.new_row + row / p.pool.page_size];
        if (page < 0 || page >= p.pool.n_pages || to < 0 || to >= p.pool.n_pages) {
            flag(p.status, FCSIM_KV_BAD_PAGE);
            continue;
        }
        const int64_t from = (page * p.pool.stride_page + (t % p.pool.page_size) * p.pool.stride_slot + h * p.pool.stride_head) * p.bytes + c * 16;
        const int64_t dest = (to * p.pool.stride_page + (row % p.pool.page_size) * p.pool.stride_slot + h * p.pool.stride_head) * p.bytes + c * 16;
        *reinterpret_cast<uint4*>(p.pool.k + dest) = *reinterpret_cast<const uint4*>(p.pool.k + from);
        *reinterpret_cast<uint4*>(p.pool.v + dest) = *reinterpret_cast<const uint4*>(p.pool.v + from);
        if (c == 0)
            p.pool.weight[((int64_t)to * p.pool.n_kv + h) * p.pool.page_size + row % p.pool.page_size] =
                p.pool.weight[((int64_t)page * p.pool.n_kv + h) * p.pool.page_size + t % p.pool.page_size];
    }
}

// ------------------------------------------------------------------------------------------------ validation
int cache_bytes(const fcsim_kv_cache* c) { return c->dtype == FCSIM_KV_E4M3 ? 1 : 2; }

int check_cache(const fcsim_kv_cache* c, Pool* pool) {
    if (!c) return FCSIM_EINVAL;
    if (c->dtype != FCSIM_KV_F16 && c->dtype != FCSIM_KV_BF16 && c->dtype != FCSIM_KV_E4M3) return FCSIM_EINVAL;
    const int bytes = cache_bytes(c);
    if (c->n_pages < 1 || c->page_size < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 65535) return FCSIM_EINVAL;
    if ((int64_t)c->n_pages * c->page_size > 0x7fffffff) return FCSIM_EINVAL;
    if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim * bytes % 16) return FCSIM_EINVAL;
    if (!good_stride(c->stride_page, bytes) || !good_stride(c->stride_slot, bytes) || !good_stride(c->stride_head, bytes))
        return FCSIM_EINVAL;
    if (!c->k || !c->v || !aligned16(c->k) || !aligned16(c->v) || ((uintptr_t)c->weight & 3)) return FCSIM_ESIZE;
    if (bytes == 1 ? !c->k_scale || !c->v_scale : c->k_scale || c->v_scale) return FCSIM_EINVAL;
    *pool = Pool{(char*)c->k, (char*)c->v, c->weight, c->k_scale, c->v_scale, c->stride_page, c->stride_slot,
                 c->stride_head, c->n_pages, c->page_size, c->n_kv_heads, c->head_dim};
    return FCSIM_OK;
}

// The type of q beside a cache: 16 bits, the cache's own where that has 16 too.
int check_type(const fcsim_kv_cache* c, int dtype) {
    if (dtype != FCSIM_KV_F16 && dtype != FCSIM_KV_BF16) return FCSIM_EINVAL;
    return c->dtype == FCSIM_KV_E4M3 || c->dtype == dtype ? FCSIM_OK : FCSIM_EINVAL;
}

int check_attend(const fcsim_kv_cache* c, const fcsim_kv_attend_args* a, AttendParams* p) {
    int rc = check_cache(c, &p->pool);
    if (rc != FCSIM_OK) return rc;
    if (!a) return FCSIM_EINVAL;
    if ((rc = check_type(c, a->dtype)) != FCSIM_OK) return rc;
    if (a->n_requests < 0 || a->n_requests > 65535 || a->n_heads < 1 || a->n_heads % c->n_kv_heads) return FCSIM_EINVAL;
    if (a->table_cols < 0 || a->max_length < 0 || a->max_length > (int64_t)a->table_cols * c->page_size) return FCSIM_EINVAL;
    if (a->window < 0 || a->table_row < 0 || !isfinite(a->scale)) return FCSIM_EINVAL;
    if (!good_stride(a->q_row, 2) || !good_stride(a->q_head, 2)) return FCSIM_EINVAL;
    if (a->n_requests > 0) {
        if (!a->q || !a->out || !a->lengths || !aligned16(a->q) || !aligned16(a->out)) return FCSIM_ESIZE;
        if (a->max_length > 0 && !a->table) return FCSIM_ESIZE;
        if (a->add_weight && !c->weight) return FCSIM_ESIZE;
    }
    p->q = (const char*)a->q, p->out = (char*)a->out, p->lse = a->lse, p->table = a->table, p->lengths = a->lengths;
    p->status = a->status, p->q_row = a->q_row, p->q_head = a->q_head, p->table_row = a->table_row;
    p->n_requests = a->n_requests, p->n_heads = a->n_heads, p->max_length = a->max_length, p->window = a->window;
    p->add_weight = a->add_weight != 0, p->scale = a->scale;
    return FCSIM_OK;
}

AttendVariant attend_variant(const fcsim_kv_cache* c, const fcsim_kv_attend_args* a) {
    const int group = a->n_heads / c->n_kv_heads;
    if (c->dtype == FCSIM_KV_E4M3)
        return a->dtype == FCSIM_KV_F16 ? attend_variant_f16_e4m3(c->head_dim, group) : attend_variant_bf16_e4m3(c->head_dim, group);
    return a->dtype == FCSIM_KV_F16 ? attend_variant_f16(c->head_dim, group) : attend_variant_bf16(c->head_dim, group);
}

// SMs of the current device (asked once per device).
int sm_count(int* out) {
    static std::atomic<int> known[64];
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return cuda_status(e);
    int n = device < 64 ? known[device].load(std::memory_order_relaxed) : 0;
    if (n == 0) {
        if ((e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device)) != cudaSuccess) return cuda_status(e);
        if (device < 64) known[device].store(n, std::memory_order_relaxed);
    }
    *out = n;
    return FCSIM_OK;
}

// Where things lie in attend's workspace, and its grid.  The counters come first.
struct AttendLayout {
    size_t counters, parts, stats, logits, bytes;
    int64_t logit_tiles;
    int grid, weight_grid;
};

// requests that share no page hold at most the pool's tokens, and each at most one tile that is not full
int64_t logit_tiles(const AttendParams& p) {
    if (!p.add_weight) return 0;
    const int64_t seen = p.window > 0 ? std::min(p.window, p.max_length) : p.max_length;
    return std::min((seen + kTile - 1) / kTile * p.n_requests, (int64_t)p.pool.n_pages * p.pool.page_size / kTile + p.n_requests);
}
// The part of the workspace that does not depend on the device.
size_t attend_kept(const AttendParams& p) {
    return (p.add_weight ? (size_t)p.n_requests * p.n_heads * 16 : 0) + (size_t)logit_tiles(p) * kTile * p.n_heads * 4;
}

int attend_layout(const AttendParams& p, const AttendVariant& v, AttendLayout* l) {
    int sms = 0, per_sm = 0, rc = sm_count(&sms);
    if (rc != FCSIM_OK) return rc;
    if ((rc = v.ctas_per_sm(&per_sm)) != 0) return cuda_status((cudaError_t)rc);
    const int64_t seen = p.window > 0 ? std::min(p.window, p.max_length) : p.max_length;
    const int64_t tiles = (seen + kTile - 1) / kTile, group = p.n_heads / p.pool.n_kv;
    const int64_t most = tiles * p.n_requests * p.pool.n_kv * ((group + v.head_cols - 1) / v.head_cols);
    l->grid = (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)sms * per_sm, (int64_t)kMaxCtas, std::max<int64_t>(most, p.n_requests)}));
    l->counters = (size_t)l->grid * 4;
    l->parts = (l->counters + 15) / 16 * 16;
    l->stats = l->parts + (size_t)2 * l->grid * v.head_cols * (v.width + 2) * 4;
    l->logit_tiles = logit_tiles(p);
    l->logits = l->stats + (p.add_weight ? (size_t)p.n_requests * p.n_heads * 16 : 0);
    l->bytes = l->stats + attend_kept(p);
    l->weight_grid = (int)std::max<int64_t>(1, std::min<int64_t>(sms * 8, l->logit_tiles));
    return FCSIM_OK;
}

int check_evict(const fcsim_kv_cache* c, const fcsim_kv_evict_args* a, EvictParams* p) {
    int rc = check_cache(c, &p->pool);
    if (rc != FCSIM_OK) return rc;
    if (!a || a->n_requests < 0 || a->n_requests > 65535) return FCSIM_EINVAL;
    if (a->table_cols < 0 || a->max_length < 0 || a->max_length > (int64_t)a->table_cols * c->page_size) return FCSIM_EINVAL;
    if (a->new_cols < 0 || a->max_budget < 0 || a->max_budget > (int64_t)a->new_cols * c->page_size) return FCSIM_EINVAL;
    if (a->recent < 0 || a->first < 0 || a->table_row < 0 || a->new_row < 0) return FCSIM_EINVAL;
    if (!c->weight) return FCSIM_ESIZE;
    if (a->n_requests > 0) {
        if (!a->lengths || !a->budget || !a->new_lengths) return FCSIM_ESIZE;
        if ((a->max_length > 0 && !a->table) || (a->max_budget > 0 && (!a->new_table || !a->kept))) return FCSIM_ESIZE;
    }
    p->table = a->table, p->lengths = a->lengths, p->budget = a->budget, p->new_table = a->new_table;
    p->new_lengths = a->new_lengths, p->kept = a->kept, p->status = a->status;
    p->table_row = a->table_row, p->new_row = a->new_row, p->max_length = a->max_length, p->max_budget = a->max_budget;
    p->recent = a->recent, p->first = a->first, p->bytes = cache_bytes(c);
    return FCSIM_OK;
}

}  // namespace

extern "C" int fcsim_kv_append(const fcsim_kv_cache* c, const fcsim_kv_append_args* a, void* cuda_stream) {
    AppendParams p;
    int rc = check_cache(c, &p.pool);
    if (rc != FCSIM_OK) return rc;
    if (!a) return FCSIM_EINVAL;
    if ((rc = check_type(c, a->dtype)) != FCSIM_OK) return rc;
    if (a->n_tokens < 0 || a->n_heads < 0 || !(a->eps >= 0) || !isfinite(a->eps)) return FCSIM_EINVAL;
    if ((int64_t)a->n_heads + 2 * c->n_kv_heads > 1 << 20) return FCSIM_EINVAL;
    if (!good_stride(a->q_row, 2) || !good_stride(a->q_head, 2) || !good_stride(a->k_row, 2) ||
        !good_stride(a->k_head, 2) || !good_stride(a->v_row, 2) || !good_stride(a->v_head, 2))
        return FCSIM_EINVAL;
    if (a->rope) {
        if (a->rope_dim < 2 || a->rope_dim > c->head_dim || a->rope_dim % (a->interleaved ? 2 : 16) || a->n_positions < 1)
            return FCSIM_EINVAL;
        if ((uintptr_t)a->rope & 3) return FCSIM_ESIZE;
    }
    if (a->n_tokens == 0) return FCSIM_OK;
    if (!a->k || !a->v || !a->slots || (a->rope && !a->positions) || (a->n_heads && (!a->q || !a->q_out))) return FCSIM_ESIZE;
    if (!aligned16(a->k) || !aligned16(a->v) || !aligned16(a->q_norm) || !aligned16(a->k_norm)) return FCSIM_ESIZE;
    if (a->n_heads && (!aligned16(a->q) || !aligned16(a->q_out))) return FCSIM_ESIZE;
    p.q = (const char*)a->q, p.k = (const char*)a->k, p.v = (const char*)a->v, p.q_out = (char*)a->q_out;
    p.q_norm = (const char*)a->q_norm, p.k_norm = (const char*)a->k_norm, p.rope = a->rope;
    p.positions = a->positions, p.slots = a->slots, p.status = a->status;
    p.q_row = a->q_row, p.q_head = a->q_head, p.k_row = a->k_row, p.k_head = a->k_head, p.v_row = a->v_row, p.v_head = a->v_head;
    p.n_tokens = a->n_tokens, p.n_heads = a->n_heads, p.rope_dim = a->rope ? a->rope_dim : 0;
    p.n_positions = a->n_positions, p.interleaved = a->interleaved != 0, p.eps = a->eps;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (c->dtype == FCSIM_KV_E4M3)
        return a->dtype == FCSIM_KV_F16 ? launch_append<F16, E4M3>(p, stream) : launch_append<BF16, E4M3>(p, stream);
    return a->dtype == FCSIM_KV_F16 ? launch_append<F16, F16>(p, stream) : launch_append<BF16, BF16>(p, stream);
}

extern "C" int fcsim_kv_attend_workspace(const fcsim_kv_cache* c, const fcsim_kv_attend_args* a, fcsim_kv_workspace* out) {
    AttendParams p;
    int rc = check_attend(c, a, &p);
    if (rc != FCSIM_OK) return rc;
    if (!out) return FCSIM_EINVAL;
    *out = {0, 0};
    if (p.n_requests == 0) return FCSIM_OK;
    AttendLayout l;
    if ((rc = attend_layout(p, attend_variant(c, a), &l)) != FCSIM_OK) return rc;
    *out = {l.bytes, l.counters};
    return FCSIM_OK;
}

extern "C" int fcsim_kv_attend(const fcsim_kv_cache* c, const fcsim_kv_attend_args* a, void* workspace,
                               size_t workspace_bytes, void* cuda_stream) {
    AttendParams p;
    int rc = check_attend(c, a, &p);
    if (rc != FCSIM_OK) return rc;
    if (p.n_requests == 0) return FCSIM_OK;
    if (!workspace || !aligned16(workspace) || workspace_bytes < attend_kept(p)) return FCSIM_ESIZE;
    const AttendVariant v = attend_variant(c, a);
    AttendLayout l;
    if ((rc = attend_layout(p, v, &l)) != FCSIM_OK) return rc;
    if (workspace_bytes < l.bytes) return FCSIM_ESIZE;
    char* ws = (char*)workspace;
    p.counters = (int*)ws, p.parts = (float*)(ws + l.parts), p.stats = (float*)(ws + l.stats), p.logits = (float*)(ws + l.logits);
    p.logit_tiles = l.logit_tiles;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    if ((rc = v.launch(p, l.grid, stream)) != 0) return cuda_status((cudaError_t)rc);
    if (p.add_weight && (rc = launch_weights(p, l.weight_grid, stream)) != 0) return cuda_status((cudaError_t)rc);
    return FCSIM_OK;
}

extern "C" int fcsim_kv_evict_workspace(const fcsim_kv_cache* c, const fcsim_kv_evict_args* a, fcsim_kv_workspace* out) {
    EvictParams p;
    int rc = check_evict(c, a, &p);
    if (rc != FCSIM_OK) return rc;
    if (!out) return FCSIM_EINVAL;
    *out = {0, 0};
    return FCSIM_OK;
}

extern "C" int fcsim_kv_evict(const fcsim_kv_cache* c, const fcsim_kv_evict_args* a, void* workspace,
                              size_t workspace_bytes, void* cuda_stream) {
    EvictParams p;
    int rc = check_evict(c, a, &p);
    if (rc != FCSIM_OK) return rc;
    if (a->n_requests == 0) return FCSIM_OK;
    fcsim_kv_evict_kernel<<<dim3(p.pool.n_kv, a->n_requests), 256, 0, (cudaStream_t)cuda_stream>>>(p);
    return launched();
}

extern "C" int fcsim_kv_last_cuda_error(void) { return g_last_cuda_error; }
