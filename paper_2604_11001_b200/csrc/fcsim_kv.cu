// Paged key-value cache: validation and launches of append, attend and evict.  The C ABI is declared in
// include/fcsim_kv.h.
#include "fcsim_kv.h"

#include <cooperative_groups.h>
#include <math.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "fcsim_kv_attend.cuh"
#include "fcsim_kv_prefill.cuh"

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
    float eps, one_over_dim;
};

// 8 bytes as 4 elements and back.
template <class T>
__device__ __forceinline__ void unpack4(const uint2& w, float* x) {
    const float2 a = T::unpack(w.x), b = T::unpack(w.y);
    x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
}
template <class T>
__device__ __forceinline__ void store4(char* p, const float* x) {
    if constexpr (T::bytes == 2) *reinterpret_cast<uint2*>(p) = make_uint2(T::pack(x[0], x[1]), T::pack(x[2], x[3]));
    else *reinterpret_cast<uint32_t*>(p) = T::pack(x[0], x[1]) | (T::pack(x[2], x[3]) << 16);
}

enum { kQuery, kKey, kValue };

// HPG neighbouring heads of one kind (`n` of them exist) of one token, by a group of LPR lanes: the loads of all first,
// then norm, rotation and store of each.  A lane holds 8 elements of a head, as two runs of 4 at lo and hi.
template <class T, class C, int LPR, int HPG, int KIND>
__device__ __forceinline__ void append_heads(const AppendParams& p, const char* src, int64_t src_head, char* dst, int64_t dst_head, const char* norm,
                                             const float* scale, int n, int lo, int hi, bool mine, bool stored, bool zero, bool pairs,
                                             int neighbours, const float (&cosine)[4], const float (&sine)[4]) {
    using Out = typename std::conditional<KIND == kQuery, T, C>::type;
    uint2 raw[HPG][2];
#pragma unroll
    for (int i = 0; i < HPG; i++) {
        raw[i][0] = raw[i][1] = make_uint2(0, 0);
        if (mine && i < n) {
            raw[i][0] = *reinterpret_cast<const uint2*>(src + lo * 2);
            raw[i][1] = *reinterpret_cast<const uint2*>(src + hi * 2);
        }
        src += src_head;
    }
    float weight[8];
    if (KIND != kValue && norm && mine) {
        unpack4<T>(*reinterpret_cast<const uint2*>(norm + lo * 2), weight);
        unpack4<T>(*reinterpret_cast<const uint2*>(norm + hi * 2), weight + 4);
    }
    char *to_lo = dst + lo * Out::bytes, *to_hi = dst + hi * Out::bytes;
#pragma unroll
    for (int i = 0; i < HPG; i++) {
        if (i >= n) break;
        if (KIND == kValue && C::bytes == 2) {  // as it came
            if (stored) {
                *reinterpret_cast<uint2*>(to_lo) = raw[i][0];
                *reinterpret_cast<uint2*>(to_hi) = raw[i][1];
            }
        } else {
            float x[8];
            unpack4<T>(raw[i][0], x);
            unpack4<T>(raw[i][1], x + 4);
            if (KIND != kValue) {
                if (norm) {
                    float sum = 0;
#pragma unroll
                    for (int e = 0; e < 8; e++) sum += x[e] * x[e];
#pragma unroll
                    for (int m = LPR / 2; m; m >>= 1) sum += __shfl_xor_sync(~0u, sum, m);
                    const float r = rsqrtf(sum * p.one_over_dim + p.eps);
#pragma unroll
                    for (int e = 0; e < 8; e++) x[e] = x[e] * r * weight[e];
                }
                if (pairs) {
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const float a = x[e], b = x[e + 4];
                        x[e] = a * cosine[e] - b * sine[e];
                        x[e + 4] = b * cosine[e] + a * sine[e];
                    }
                } else if (neighbours > 0) {
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        if (e < neighbours) {
                            const float a = x[2 * e], b = x[2 * e + 1];
                            x[2 * e] = a * cosine[e] - b * sine[e];
                            x[2 * e + 1] = b * cosine[e] + a * sine[e];
                        }
                }
                if (zero) {
#pragma unroll
                    for (int e = 0; e < 8; e++) x[e] = 0;
                }
            }
            if (KIND != kQuery && C::bytes == 1) {
                const float s = 1.0f / scale[i];
                if (fabsf(s) < INFINITY) {
#pragma unroll
                    for (int e = 0; e < 8; e++) x[e] *= s;
                } else {  // a scale below 2^-128, or none
#pragma unroll
                    for (int e = 0; e < 8; e++) x[e] /= scale[i];
                }
            }
            if (stored) {
                store4<Out>(to_lo, x);
                store4<Out>(to_hi, x + 4);
            }
        }
        to_lo += dst_head, to_hi += dst_head;
    }
}

// A CTA takes the same HPG heads (of one kind: q, k or v) of 256 / LPR tokens, a group of LPR lanes each, so that every
// branch on the kind is uniform and addresses advance by a stride; the CTAs of a token's other heads are its neighbours.
// The two runs of a lane are a rotation's pairs (i .. i + 3 and i + rope_dim / 2 ..): turning them needs no other lane,
// and half as many cosines and sines as elements, read once for all of the group's heads.  Bound by instructions and
// by the bytes of q, k and v alike when there are many tokens, by latency when few.
template <class T, class C, int LPR, int HPG>
__global__ void __launch_bounds__(256, HPG == 8 ? 4 : HPG == 4 ? 5 : 1) fcsim_kv_append_kernel(const AppendParams p) {
    const int n_kv = p.pool.n_kv, D = p.pool.head_dim;
    const int q_chunks = (p.n_heads + HPG - 1) / HPG, kv_chunks = (n_kv + HPG - 1) / HPG, chunks = q_chunks + 2 * kv_chunks;
    const int block = blockIdx.x / chunks, chunk = blockIdx.x - block * chunks;
    const int kind = chunk < q_chunks ? kQuery : chunk < q_chunks + kv_chunks ? kKey : kValue;
    const int h = (kind == kQuery ? chunk : kind == kKey ? chunk - q_chunks : chunk - q_chunks - kv_chunks) * HPG;
    const int lane = threadIdx.x & (LPR - 1);
    const int at = block * (256 / LPR) + threadIdx.x / LPR;
    const bool there = at < p.n_tokens, mine = there && lane * 8 < D;
    const int64_t token = there ? at : 0;
    const int half = p.rope_dim / 2;
    const bool pairs = p.rope != nullptr && !p.interleaved && lane * 4 < half;
    const int neighbours = p.interleaved ? half - lane * 4 : 0;  // pairs of this lane, if they are neighbours
    const int lo = pairs ? lane * 4 : lane * 8, hi = pairs ? half + lane * 4 : lo + 4;
    bool good = true;
    float cosine[4] = {1, 1, 1, 1}, sine[4] = {0, 0, 0, 0};
    if (p.rope != nullptr) {
        const int position = p.positions[token];
        good = position >= 0 && position < p.n_positions;
        if (!good && there && lane == 0 && chunk == 0) flag(p.status, FCSIM_KV_BAD_POSITION);
        if (kind != kValue) {
            const float* row = p.rope + (int64_t)(good ? position : 0) * p.rope_dim + lane * 4;
            if (pairs) {
                *reinterpret_cast<float4*>(cosine) = *reinterpret_cast<const float4*>(row);
                *reinterpret_cast<float4*>(sine) = *reinterpret_cast<const float4*>(row + half);
            } else {
#pragma unroll
                for (int i = 0; i < 4; i++)
                    if (i < neighbours) cosine[i] = row[i], sine[i] = row[half + i];
            }
        }
    }
    if (kind == kQuery) {
        append_heads<T, C, LPR, HPG, kQuery>(p, p.q + (token * p.q_row + h * p.q_head) * 2, p.q_head * 2, p.q_out + (token * p.n_heads + h) * D * 2, D * 2,
                                             p.q_norm, nullptr, p.n_heads - h, lo, hi, mine, mine, !good, pairs, neighbours, cosine, sine);
        return;
    }
    // the token's place in the cache
    bool stored = mine && good;
    int64_t place = 0;
    if (there && good) {
        const int64_t slot = p.slots[token];
        if (slot < 0 || slot >= (int64_t)p.pool.n_pages * p.pool.page_size) {
            if (slot >= 0 && lane == 0) flag(p.status, FCSIM_KV_BAD_PAGE);
            stored = false;
        } else {
            const int page = page_of(p.pool, (int)slot), in_page = (int)slot - page * p.pool.page_size;
            place = page * p.pool.stride_page + in_page * p.pool.stride_slot + h * p.pool.stride_head;
            if (kind == kKey && p.pool.weight && lane < HPG && h + lane < n_kv)
                p.pool.weight[((int64_t)page * n_kv + h + lane) * p.pool.page_size + in_page] = 0.0f;
        }
    }
    if (kind == kKey)
        append_heads<T, C, LPR, HPG, kKey>(p, p.k + (token * p.k_row + h * p.k_head) * 2, p.k_head * 2, p.pool.k + place * C::bytes,
                                           p.pool.stride_head * C::bytes, p.k_norm, p.pool.k_scale + h, n_kv - h, lo, hi, mine, stored, false, pairs,
                                           neighbours, cosine, sine);
    else
        append_heads<T, C, LPR, HPG, kValue>(p, p.v + (token * p.v_row + h * p.v_head) * 2, p.v_head * 2, p.pool.v + place * C::bytes,
                                             p.pool.stride_head * C::bytes, nullptr, p.pool.v_scale + h, n_kv - h, lo, hi, mine, stored, false, false, 0,
                                             cosine, sine);
}

template <class T, class C, int LPR, int HPG>
int launch_append_as(const AppendParams& p, cudaStream_t stream) {
    const int64_t chunks = (p.n_heads + HPG - 1) / HPG + 2 * ((p.pool.n_kv + HPG - 1) / HPG), tokens = 256 / LPR;
    const int64_t blocks = (p.n_tokens + tokens - 1) / tokens * chunks;
    if (blocks > 0x7fffffff) return FCSIM_EINVAL;
    fcsim_kv_append_kernel<T, C, LPR, HPG><<<(unsigned)blocks, 256, 0, stream>>>(p);
    return launched();
}
template <class T, class C, int LPR>
int launch_append_lanes(const AppendParams& p, cudaStream_t stream) {
    // Heads a group: more share the rotation and the addresses, fewer spread a small call over the SMs.  With 64 + 2 x 8
    // heads of 128 bf16 elements, 1 / 2 / 4 / 8 heads: 64 tokens 3.7 / 3.9 / 4.3 / 5.3 us, 256 tokens 6.1 / 5.0 / 5.0 / 5.8,
    // 1 024 tokens 15.6 / 12.0 / 10.3 / 10.8, 4 096 tokens 55 / 41 / 31 / 29, 16 384 tokens 215 / 158 / 120 / 109.
    const int64_t lanes = (int64_t)p.n_tokens * (p.n_heads + 2 * p.pool.n_kv) * LPR;
    if (lanes < 1 << 17) return launch_append_as<T, C, LPR, 1>(p, stream);
    if (lanes < 1 << 19) return launch_append_as<T, C, LPR, 2>(p, stream);
    if (lanes < 3 << 19) return launch_append_as<T, C, LPR, 4>(p, stream);
    return launch_append_as<T, C, LPR, 8>(p, stream);
}
template <class T, class C>
int launch_append(const AppendParams& p, cudaStream_t stream) {
    const int lanes = p.pool.head_dim / 8;
    if (lanes <= 8) return launch_append_lanes<T, C, 8>(p, stream);
    if (lanes <= 16) return launch_append_lanes<T, C, 16>(p, stream);
    return launch_append_lanes<T, C, 32>(p, stream);
}

// ------------------------------------------------------------------------------------------------ read
struct ReadParams {
    Pool pool;
    const int64_t* slots;
    char *k_out, *v_out;
    int32_t* status;
    int64_t pieces;               // of all tokens: 16 cached bytes each, of k and of v
    int token_pieces, row_pieces; // of a token; of a head
    uint64_t token_magic, row_magic;
};

// x / d for x < 2^31, of magic = ceil(2^63 / d)
__device__ __forceinline__ int divide_by(uint64_t magic, int x) {
    return (int)__umul64hi(magic, (uint64_t)x << 1);
}

// 16 cached bytes as 8 or 16 elements of type T, times `scale` where the cache has scales (in 32 bits: a product of 4 and 24 bits is rounded there, and
// then to T, which near the middle of two values of T may be the other one of them)
template <class T, class C>
__device__ __forceinline__ void convert_piece(const uint4& raw, float scale, char* out) {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    uint32_t y[8];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if constexpr (C::bytes == 1) {
            const float2 a = F16::unpack(E4M3::halves(w[i])), b = F16::unpack(E4M3::halves(w[i] >> 16));
            y[2 * i] = T::pack(a.x * scale, a.y * scale), y[2 * i + 1] = T::pack(b.x * scale, b.y * scale);
        } else if constexpr (std::is_same<T, C>::value) {
            y[i] = w[i];
        } else {
            const float2 a = C::unpack(w[i]);
            y[i] = T::pack(a.x, a.y);
        }
    }
    if (C::bytes == 1 && ((uintptr_t)out & 31) == 0) {  // 32 bytes at once (the output may begin between two such places)
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(out), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]), "r"(y[4]), "r"(y[5]), "r"(y[6]), "r"(y[7])
                     : "memory");
        return;
    }
    __stcs(reinterpret_cast<uint4*>(out), make_uint4(y[0], y[1], y[2], y[3]));
    if constexpr (C::bytes == 1) __stcs(reinterpret_cast<uint4*>(out) + 1, make_uint4(y[4], y[5], y[6], y[7]));
}

// The tokens' rows are cut into pieces of 16 cached bytes, end to end over all tokens, and a thread takes one: neighbouring lanes read and write
// neighbouring bytes whatever the width of a head.  Bound by memory when there are many tokens (131 072 of 8 x 128: bf16 164 us, e4m3 into bf16
// 123 us, 6.55 TB/s both; 16-bit rows of 8-bit ones leave 32 bytes a lane, in two stores of 16 it took 137), by two dependent loads when few (4 us).
// (Four pieces a thread, all asked for before any is used, took 160 us of bf16, but 4 to 14 us more of e4m3.)
template <class T, class C>
__global__ void __launch_bounds__(256) fcsim_kv_read_kernel(const ReadParams p) {
    const int64_t base = (int64_t)blockIdx.x * 256, to = base + threadIdx.x;
    if (to >= p.pieces) return;
    const int64_t token0 = base / p.token_pieces;  // the same for the CTA
    const int x = (int)(base - token0 * p.token_pieces) + threadIdx.x, ahead = divide_by(p.token_magic, x), rest = x - ahead * p.token_pieces;
    const int h = divide_by(p.row_magic, rest), piece = rest - h * p.row_pieces;
    const int64_t slot = p.slots[token0 + ahead];
    float ks = 1, vs = 1;
    if (C::bytes == 1) ks = p.pool.k_scale[h], vs = p.pool.v_scale[h];
    uint4 k = make_uint4(0, 0, 0, 0), v = k;
    if (slot >= (int64_t)p.pool.n_pages * p.pool.page_size) {
        if (h == 0 && piece == 0) flag(p.status, FCSIM_KV_BAD_PAGE);
    } else if (slot >= 0) {
        const int page = page_of(p.pool, (int)slot), place = (int)slot - page * p.pool.page_size;
        const int64_t at = (page * p.pool.stride_page + place * p.pool.stride_slot + h * p.pool.stride_head) * C::bytes + piece * 16;
        k = __ldcs(reinterpret_cast<const uint4*>(p.pool.k + at));
        v = __ldcs(reinterpret_cast<const uint4*>(p.pool.v + at));
    }
    if (slot < 0 || slot >= (int64_t)p.pool.n_pages * p.pool.page_size) ks = vs = 1;  // (zeros, whatever the scale is)
    convert_piece<T, C>(k, ks, p.k_out + to * (16 / C::bytes * 2));
    convert_piece<T, C>(v, vs, p.v_out + to * (16 / C::bytes * 2));
}

template <class T, class C>
int launch_read(const ReadParams& p, cudaStream_t stream) {
    const int64_t blocks = (p.pieces + 255) / 256;
    if (blocks > 0x7fffffff) return FCSIM_EINVAL;
    fcsim_kv_read_kernel<T, C><<<(unsigned)blocks, 256, 0, stream>>>(p);
    return launched();
}
template <class T>
int launch_read_from(int cache_type, const ReadParams& p, cudaStream_t stream) {
    if (cache_type == FCSIM_KV_E4M3) return launch_read<T, E4M3>(p, stream);
    return cache_type == FCSIM_KV_F16 ? launch_read<T, F16>(p, stream) : launch_read<T, BF16>(p, stream);
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

// A weight as an unsigned key of the same order: NaN lowest, -0 as 0.  No weight has key 0.
__device__ __forceinline__ uint32_t order_key(float w) {
    if (w != w) return 1;
    const uint32_t b = __float_as_uint(w + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

constexpr int kSelectThreads = 512, kSelectWarps = kSelectThreads / 32;
constexpr int kMaxCluster = 8;            // CTAs that share a row: the portable size of a cluster
constexpr int64_t kFusedBytes = 128 * 1024;  // what a CTA of the selection copies itself
constexpr int kMaxFours = 12 * 1024;      // fours of keys a CTA keeps in shared memory (192 KB)

// What request r keeps: `keep` tokens, of which [0, lo) and [hi, n) are sure and `places` go to the largest of [lo, hi).
struct Cut {
    int n, keep, lo, hi, places;
};
__device__ __forceinline__ Cut cut_of(const EvictParams& p, int r, int32_t* status) {
    Cut c;
    c.n = length_of(p.lengths, r, p.max_length, status);
    int budget = p.budget[r];
    if (budget < 0 || budget > p.max_budget) {
        flag(status, FCSIM_KV_BAD_BUDGET);
        budget = budget < 0 ? 0 : p.max_budget;
    }
    c.keep = min(c.n, budget);
    const int recent = min(p.recent, budget), first = min(p.first, budget - recent);
    const bool all = c.keep == c.n;
    c.lo = all ? c.n : first;
    c.hi = all ? c.n : c.n - recent;
    c.places = c.keep - (c.n - c.hi) - c.lo;
    return c;
}

// Copies kept rows [row0, row0 + THREADS / LPR) of one kv head of request r: 16 bytes a lane, LPR lanes a row.  A row waits for
// its index and its page before it is read, so more threads hide more than more rows of each (4 requests of 65 536 to 8 192
// tokens, 1, 2, 4, 8 rows a thread: 43, 43, 48, 63 us in all).  Nothing is read twice, so both sides go through the caches
// as streams (64 requests to 1 024 tokens, a call among others 86 -> 82 us).
template <int LPR, int THREADS>
__device__ __forceinline__ void move_rows(const EvictParams& p, int r, int h, int keep, int row0) {
    const int lane = threadIdx.x % LPR, chunks = p.pool.head_dim * p.bytes / 16, size = p.pool.page_size;
    const int row = row0 + threadIdx.x / LPR;
    if (row >= keep) return;
    const int t = p.kept[((int64_t)r * p.pool.n_kv + h) * p.max_budget + row];
    const int from = page_of(p.pool, t), into = page_of(p.pool, row);
    const int page = p.table[r * p.table_row + from], to = p.new_table[r * p.new_row + into];
    const bool there = (unsigned)page < (unsigned)p.pool.n_pages, room = (unsigned)to < (unsigned)p.pool.n_pages;
    if (!there || !room) flag(p.status, FCSIM_KV_BAD_PAGE);
    if (!room) return;
    if (lane < chunks) {
        const int64_t src = (page * p.pool.stride_page + (t - from * size) * p.pool.stride_slot + h * p.pool.stride_head) * p.bytes + lane * 16;
        const int64_t dst = (to * p.pool.stride_page + (row - into * size) * p.pool.stride_slot + h * p.pool.stride_head) * p.bytes + lane * 16;
        uint4 k = make_uint4(0, 0, 0, 0), v = k;  // of a page that does not exist
        if (there) k = __ldcs(reinterpret_cast<const uint4*>(p.pool.k + src)), v = __ldcs(reinterpret_cast<const uint4*>(p.pool.v + src));
        __stcs(reinterpret_cast<uint4*>(p.pool.k + dst), k);
        __stcs(reinterpret_cast<uint4*>(p.pool.v + dst), v);
    }
    if (lane == 0)
        p.pool.weight[((int64_t)to * p.pool.n_kv + h) * size + row - into * size] =
            there ? p.pool.weight[((int64_t)page * p.pool.n_kv + h) * size + t - from * size] : 0.0f;
}

// Which tokens one kv head of one request keeps, by one cluster.  Every CTA takes an equal slice of the candidates and
// keeps their keys in shared memory, so that the weights are read once; four counts by 8 bits each, from the top, give
// the smallest key that is kept and how many of its equals are.  The counts of the CTAs meet over distributed shared
// memory, one cluster barrier for each (every count has a buffer of its own).  Places then follow from running sums in
// the order of the tokens.  A thread holds four neighbouring tokens at a time: they share a page where its size allows,
// and a sum over a warp covers 128 of them.  Bound by the latency of these few passes: a slice is 16 to 32 KB.
// With LPR the same cluster copies what it has selected (its CTAs in turn); without, a second kernel does.
template <int LPR>
__global__ void __launch_bounds__(kSelectThreads, 2) fcsim_kv_select_kernel(const EvictParams p, const int capacity) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    if (LPR == 0) cudaTriggerProgrammaticLaunchCompletion();  // the copies may line up; they wait for this grid's end
    extern __shared__ uint4 keys[];
    __shared__ uint32_t counts[4][256], sums[256];
    __shared__ int warp_sums[kSelectWarps], warp_equals[kSelectWarps], mine, mine_equal, chosen[2];
    const int r = blockIdx.z, h = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = blockIdx.x, ctas = gridDim.x;
    const Cut c = cut_of(p, r, h == 0 && rank == 0 && tid == 0 ? p.status : nullptr);
    int32_t* const kept = p.kept + ((int64_t)r * p.pool.n_kv + h) * p.max_budget;
    for (int i = rank * kSelectThreads + tid; i < p.max_budget; i += ctas * kSelectThreads) {
        if (i < c.lo && i < c.keep) kept[i] = i;
        else if (i >= c.keep) kept[i] = -1;
        else if (i >= c.lo + c.places) kept[i] = c.n - c.keep + i;
    }
    if (h == 0 && rank == 0 && tid == 0) p.new_lengths[r] = c.keep;
    auto copy = [&]() {
        if constexpr (LPR > 0)
            for (int row = rank * (kSelectThreads / LPR); row < c.keep; row += ctas * (kSelectThreads / LPR))
                move_rows<LPR, kSelectThreads>(p, r, h, c.keep, row);
    };
    auto meet = [&]() {  // a barrier of the cluster costs 0.5 us, one of a CTA a tenth of it
        if (ctas > 1) cluster.sync();
        else __syncthreads();
    };
    if (c.places == 0) {  // the same for the whole cluster
        meet();
        copy();
        return;
    }

    // tokens by fours; key 0 for those of the first and last four that are no candidates
    const int four0 = c.lo / 4, fours = (c.hi + 3) / 4 - four0, each = (fours + ctas - 1) / ctas;
    const int begin = four0 + min(fours, rank * each), count = four0 + min(fours, (rank + 1) * each) - begin;
    const bool resident = each <= capacity;
    const float* const weights = p.pool.weight + (int64_t)h * p.pool.page_size;
    const int64_t page_weights = (int64_t)p.pool.n_kv * p.pool.page_size;
    const int32_t* const table = p.table + r * p.table_row;
    auto token_key = [&](int t, int page, float w) {
        if (t < c.lo || t >= c.hi) return 0u;
        if ((unsigned)page >= (unsigned)p.pool.n_pages) {
            flag(p.status, FCSIM_KV_BAD_PAGE);
            return 1u;
        }
        return order_key(w);
    };
    auto read_keys = [&](int i) {
        const int t = (begin + i) * 4;
        uint4 k;
        if (p.pool.page_size % 4 == 0) {  // one page, 16 aligned bytes
            const int index = page_of(p.pool, t), page = table[index];
            float4 w = make_float4(0, 0, 0, 0);
            if ((unsigned)page < (unsigned)p.pool.n_pages)
                w = *reinterpret_cast<const float4*>(weights + page * page_weights + t - index * p.pool.page_size);
            k = make_uint4(token_key(t, page, w.x), token_key(t + 1, page, w.y), token_key(t + 2, page, w.z), token_key(t + 3, page, w.w));
        } else {
            uint32_t x[4];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                int page = 0;
                float w = 0;
                if (t + e >= c.lo && t + e < c.hi) {
                    const int index = page_of(p.pool, t + e);
                    page = table[index];
                    if ((unsigned)page < (unsigned)p.pool.n_pages) w = weights[page * page_weights + t + e - index * p.pool.page_size];
                }
                x[e] = token_key(t + e, page, w);
            }
            k = make_uint4(x[0], x[1], x[2], x[3]);
        }
        return k;
    };
    auto key = [&](int i) { return resident ? keys[i] : read_keys(i); };
    for (int i = tid; i < 4 * 256; i += kSelectThreads) counts[0][i] = 0;
    __syncthreads();
    uint32_t threshold = 0;
    int need = c.places;  // how many of the keys with the digits found so far are kept
#pragma unroll 1
    for (int pass = 0; pass < 4; pass++) {
        const int shift = 24 - 8 * pass;
        if (pass == 0) {
            for (int i0 = tid; i0 < count; i0 += 4 * kSelectThreads) {
                uint4 k[4];
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (i0 + e * kSelectThreads < count) k[e] = read_keys(i0 + e * kSelectThreads);
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (i0 + e * kSelectThreads < count) {
                        if (resident) keys[i0 + e * kSelectThreads] = k[e];
                        atomicAdd(&counts[0][k[e].x >> 24], 1u), atomicAdd(&counts[0][k[e].y >> 24], 1u);
                        atomicAdd(&counts[0][k[e].z >> 24], 1u), atomicAdd(&counts[0][k[e].w >> 24], 1u);
                    }
            }
        } else {
            for (int i = tid; i < count; i += kSelectThreads) {
                const uint4 k = key(i);
                auto add = [&](uint32_t x) {
                    if ((x ^ threshold) >> (shift + 8) == 0) atomicAdd(&counts[pass][(x >> shift) & 255], 1u);
                };
                add(k.x), add(k.y), add(k.z), add(k.w);
            }
        }
        meet();
        if (tid < 256) {
            uint32_t sum = 0;
            for (int i = 0; i < ctas; i++) sum += cluster.map_shared_rank(&counts[pass][0], i)[tid];
            sums[tid] = sum;
        }
        __syncthreads();
        if (warp == 0) {  // lane i has digits 255 - 8 i .. 248 - 8 i
            int own[8], total = 0;
#pragma unroll
            for (int i = 0; i < 8; i++) total += own[i] = (int)sums[255 - 8 * lane - i];
            int upto = total;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int x = __shfl_up_sync(~0u, upto, d);
                if (lane >= d) upto += x;
            }
            int before = upto - total;
            if (before < need && upto >= need) {
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    if (before < need && before + own[i] >= need) chosen[0] = 255 - 8 * lane - i, chosen[1] = need - before;
                    before += own[i];
                }
            }
        }
        __syncthreads();
        threshold |= (uint32_t)chosen[0] << shift;
        need = chosen[1];
    }
    // places: keys above the threshold, and of its equals the first `need`, in order; a warp has a run of the slice
    const int run = ((count + kSelectWarps - 1) / kSelectWarps + 31) / 32 * 32;
    const int from = min(count, warp * run), to = min(count, from + run);
    int above = 0, equal = 0;
    for (int i = from + lane; i < to; i += 32) {
        const uint4 k = key(i);
        above += (k.x > threshold) + (k.y > threshold) + (k.z > threshold) + (k.w > threshold);
        equal += (k.x == threshold) + (k.y == threshold) + (k.z == threshold) + (k.w == threshold);
    }
    above = __reduce_add_sync(~0u, above);
    equal = __reduce_add_sync(~0u, equal);
    if (lane == 0) warp_sums[warp] = above, warp_equals[warp] = equal;
    __syncthreads();
    if (tid == 0) {
        int a = 0, e = 0;
        for (int w = 0; w < kSelectWarps; w++) {
            const int x = warp_sums[w], y = warp_equals[w];
            warp_sums[w] = a, warp_equals[w] = e;
            a += x, e += y;
        }
        mine = a, mine_equal = e;
    }
    meet();
    above = lane < rank ? *cluster.map_shared_rank(&mine, lane) : 0;  // of the CTAs before this one
    equal = lane < rank ? *cluster.map_shared_rank(&mine_equal, lane) : 0;
    above = __reduce_add_sync(~0u, above) + warp_sums[warp];
    equal = __reduce_add_sync(~0u, equal) + warp_equals[warp];
    for (int i0 = from; i0 < to; i0 += 32) {
        const int i = i0 + lane;
        const uint4 k = i < to ? key(i) : make_uint4(0, 0, 0, 0);
        const uint32_t x[4] = {k.x, k.y, k.z, k.w};
        uint32_t own = 0;  // above, and equal in the upper half
#pragma unroll
        for (int e = 0; e < 4; e++) own += (x[e] > threshold) + ((uint32_t)(x[e] == threshold) << 16);
        uint32_t upto = own;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t y = __shfl_up_sync(~0u, upto, d);
            if (lane >= d) upto += y;
        }
        int a = above + (int)((upto - own) & 0xffff), q = equal + (int)((upto - own) >> 16);
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const bool over = x[e] > threshold, same = x[e] == threshold;
            if (over || (same && q < need)) kept[c.lo + a + min(q, need)] = (begin + i) * 4 + e;
            a += over, q += same;
        }
        const uint32_t all = __shfl_sync(~0u, upto, 31);
        above += (int)(all & 0xffff), equal += (int)(all >> 16);
    }
    meet();  // the others may still read this CTA's counts; all of the row's indexes are written
    copy();
}

// The copies as a kernel of their own, bound by memory.
template <int LPR>
__global__ void __launch_bounds__(256) fcsim_kv_move_kernel(const EvictParams p) {
    cudaGridDependencySynchronize();
    const int r = blockIdx.z, h = blockIdx.y;
    move_rows<LPR, 256>(p, r, h, cut_of(p, r, nullptr).keep, blockIdx.x * (256 / LPR));
}

template <int LPR>
int launch_select(const EvictParams& p, dim3 grid, int capacity, int device, cudaStream_t stream) {
    static std::atomic<bool> raised[kMaxDevices];
    if (device >= kMaxDevices || !raised[device].load(std::memory_order_relaxed)) {
        const cudaError_t e = cudaFuncSetAttribute(fcsim_kv_select_kernel<LPR>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxFours * 16);
        if (e != cudaSuccess) return cuda_status(e);
        if (device < kMaxDevices) raised[device].store(true, std::memory_order_relaxed);
    }
    cudaLaunchConfig_t config = {};
    config.gridDim = grid;
    config.blockDim = dim3(kSelectThreads);
    config.dynamicSmemBytes = (size_t)capacity * 16;
    config.stream = stream;
    cudaLaunchAttribute cluster;
    cluster.id = cudaLaunchAttributeClusterDimension;
    cluster.val.clusterDim.x = grid.x, cluster.val.clusterDim.y = 1, cluster.val.clusterDim.z = 1;
    config.attrs = &cluster;
    config.numAttrs = 1;
    return cuda_status(cudaLaunchKernelEx(&config, fcsim_kv_select_kernel<LPR>, (EvictParams)p, (int)capacity));
}
template <int LPR>
int launch_move(const EvictParams& p, int n_requests, cudaStream_t stream) {
    if (p.max_budget == 0) return FCSIM_OK;
    const int rows = 256 / LPR;
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3((p.max_budget + rows - 1) / rows, p.pool.n_kv, n_requests);
    config.blockDim = dim3(256);
    config.stream = stream;
    cudaLaunchAttribute early;  // launched while the selection runs
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    config.attrs = &early;
    config.numAttrs = 1;
    return cuda_status(cudaLaunchKernelEx(&config, fcsim_kv_move_kernel<LPR>, (EvictParams)p));
}

// ------------------------------------------------------------------------------------------------ validation
// Tokens of a call, a request or a budget at most: the kernels count on past the end, by less than 2^16, in 32 bits.
constexpr int kMaxTokens = 0x7fffffff - 0xffff;

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
    if (!c->k || !c->v || !aligned16(c->k) || !aligned16(c->v) || !aligned16(c->weight)) return FCSIM_ESIZE;
    if (bytes == 1 ? !c->k_scale || !c->v_scale : c->k_scale || c->v_scale) return FCSIM_EINVAL;
    *pool = Pool{(char*)c->k, (char*)c->v, c->weight, c->k_scale, c->v_scale, c->stride_page, c->stride_slot,
                 c->stride_head, c->n_pages, c->page_size, c->n_kv_heads, c->head_dim,
                 ((1ull << 63) + c->page_size - 1) / c->page_size};
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
    if (a->max_length > kMaxTokens || (int64_t)a->n_heads * c->head_dim > 0x7fffffff) return FCSIM_EINVAL;
    if (a->window < 0 || a->first < 0 || a->table_row < 0 || !isfinite(a->scale)) return FCSIM_EINVAL;
    if (!good_stride(a->q_row, 2) || !good_stride(a->q_head, 2)) return FCSIM_EINVAL;
    if (a->n_requests > 0) {
        if (!a->q || !a->out || !a->lengths || !aligned16(a->q) || !aligned16(a->out)) return FCSIM_ESIZE;
        if (a->max_length > 0 && !a->table) return FCSIM_ESIZE;
        if (a->add_weight && !c->weight) return FCSIM_ESIZE;
    }
    p->q = (const char*)a->q, p->out = (char*)a->out, p->lse = a->lse, p->table = a->table, p->lengths = a->lengths;
    p->status = a->status, p->q_row = a->q_row, p->q_head = a->q_head, p->table_row = a->table_row;
    p->n_requests = a->n_requests, p->n_heads = a->n_heads, p->max_length = a->max_length;
    const bool all = (int64_t)a->window + a->first >= a->max_length || a->window == 0;  // (of the longest request, and so of all)
    p->most_seen = all ? a->max_length : a->window + a->first, p->first = all ? 0 : a->first;
    p->add_weight = a->add_weight != 0, p->scale = a->scale;
    return FCSIM_OK;
}

AttendVariant attend_variant(const fcsim_kv_cache* c, const AttendParams& p, int dtype) {
    const int group = p.n_heads / c->n_kv_heads;
    const bool first = p.first > 0;
    if (c->dtype == FCSIM_KV_E4M3)
        return dtype == FCSIM_KV_F16 ? attend_variant_f16_e4m3(c->head_dim, group, first) : attend_variant_bf16_e4m3(c->head_dim, group, first);
    return dtype == FCSIM_KV_F16 ? attend_variant_f16(c->head_dim, group, first) : attend_variant_bf16(c->head_dim, group, first);
}

// The current device and its SMs (asked once per device).
int device_and_sms(int* device, int* out) {
    static std::atomic<int> known[kMaxDevices];
    cudaError_t e = cudaGetDevice(device);
    if (e != cudaSuccess) return cuda_status(e);
    int n = *device < kMaxDevices ? known[*device].load(std::memory_order_relaxed) : 0;
    if (n == 0) {
        if ((e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, *device)) != cudaSuccess) return cuda_status(e);
        if (*device < kMaxDevices) known[*device].store(n, std::memory_order_relaxed);
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
    const int64_t tile = 1 << p.tile_bits;
    return std::min((p.most_seen + tile - 1) / tile * p.n_requests, (int64_t)p.pool.n_pages * p.pool.page_size / tile + p.n_requests);
}
// The part of the workspace that does not depend on the device.
size_t attend_kept(const AttendParams& p) {
    return (p.add_weight ? (size_t)p.n_requests * p.n_heads * 16 : 0) + ((size_t)logit_tiles(p) << p.tile_bits) * p.n_heads * 4;
}

int attend_layout(const AttendParams& p, const AttendVariant& v, AttendLayout* l) {
    int device = 0, sms = 0, per_sm = 0, rc = device_and_sms(&device, &sms);
    if (rc != FCSIM_OK) return rc;
    if ((rc = v.ctas_per_sm(device, &per_sm)) != 0) return cuda_status((cudaError_t)rc);
    const int64_t tiles = ((int64_t)p.most_seen + (1 << p.tile_bits) - 1) >> p.tile_bits, group = p.n_heads / p.pool.n_kv;
    const int64_t most = tiles * p.n_requests * p.pool.n_kv * ((group + v.head_cols - 1) / v.head_cols);
    l->grid = (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)sms * per_sm, (int64_t)kMaxCtas, std::max<int64_t>(most + most / 3 + 1, p.n_requests)}));
    // the kernel counts the tiles of all requests, and the work of a CTA, in 32 bits
    if ((tiles + 16) * p.n_requests > 0x7fffffff || (most + (int64_t)p.n_requests * 16 * p.n_heads) / l->grid >= 0x7fffffff) return FCSIM_EINVAL;
    const size_t workers = (size_t)l->grid * (kThreads / 32);
    l->counters = kMaxCtas * (kThreads / 32) * 4;  // the same for every call, so that none finds another's parts there
    l->parts = l->counters;
    l->stats = l->parts + 2 * workers * v.head_cols * (v.width + 2) * 4;
    l->logit_tiles = logit_tiles(p);
    l->logits = l->stats + (p.add_weight ? (size_t)p.n_requests * p.n_heads * 16 : 0);
    l->bytes = l->stats + attend_kept(p);
    l->weight_grid = (int)std::max<int64_t>(1, std::min<int64_t>(sms * kWeightCtas, ((l->logit_tiles << p.tile_bits) * p.pool.n_kv + 4 * kThreads - 1) / (4 * kThreads)));
    return FCSIM_OK;
}

// ------------------------------------------------------------------------------------------------ prefill
PrefillVariant prefill_variant(const fcsim_kv_cache* c, int dtype) {
    if (c->dtype == FCSIM_KV_E4M3) return dtype == FCSIM_KV_F16 ? prefill_variant_f16_e4m3(c->head_dim) : prefill_variant_bf16_e4m3(c->head_dim);
    return dtype == FCSIM_KV_F16 ? prefill_variant_f16(c->head_dim) : prefill_variant_bf16(c->head_dim);
}

int check_prefill(const fcsim_kv_cache* c, const fcsim_kv_prefill_args* a, PrefillParams* p, PrefillVariant* v) {
    int rc = check_cache(c, &p->pool);
    if (rc != FCSIM_OK) return rc;
    if (!a) return FCSIM_EINVAL;
    if ((rc = check_type(c, a->dtype)) != FCSIM_OK) return rc;
    if (a->n_rows < 0 || a->n_rows > kMaxTokens || a->n_requests < 0 || a->n_requests > 65535) return FCSIM_EINVAL;
    if (a->n_heads < 1 || a->n_heads % c->n_kv_heads || (int64_t)a->n_heads * c->head_dim > 0x7fffffff) return FCSIM_EINVAL;
    if (a->table_cols < 0 || a->max_length < 0 || a->max_length > (int64_t)a->table_cols * c->page_size || a->max_length > kMaxTokens)
        return FCSIM_EINVAL;
    if (a->window < 0 || a->first < 0 || a->table_row < 0 || !isfinite(a->scale)) return FCSIM_EINVAL;
    if (!good_stride(a->q_row, 2) || !good_stride(a->q_head, 2)) return FCSIM_EINVAL;
    if (a->n_rows > 0) {
        if (!a->q || !a->out || !aligned16(a->q) || !aligned16(a->out)) return FCSIM_ESIZE;
        if (a->n_requests > 0 && (!a->starts || !a->lengths || (a->max_length > 0 && !a->table))) return FCSIM_ESIZE;
    }
    p->q = (const char*)a->q, p->out = (char*)a->out, p->lse = a->lse, p->starts = a->starts, p->table = a->table;
    p->lengths = a->lengths, p->status = a->status, p->q_row = a->q_row, p->q_head = a->q_head, p->table_row = a->table_row;
    p->n_rows = a->n_rows, p->n_requests = a->n_requests, p->n_heads = a->n_heads, p->max_length = a->max_length;
    const bool all = (int64_t)a->window + a->first >= a->max_length || a->window == 0;  // (of the longest request, and so of all)
    p->window = all ? 0 : a->window, p->first = all ? 0 : a->first;
    p->scale = a->scale;
    // the rows of a block: all heads of a group and as many tokens as there is room for
    *v = prefill_variant(c, a->dtype);
    const int group = a->n_heads / c->n_kv_heads;
    p->head_tiles = (group + v->rows - 1) / v->rows;
    p->heads_a_tile = (group + p->head_tiles - 1) / p->head_tiles;
    p->tokens_a_block = v->rows / p->heads_a_tile;
    // what a block sees at most: with a window, that of all its tokens, the first ones, and what their rounding to whole boxes adds
    const int64_t seen = p->window > 0 ? (int64_t)p->window + p->first + p->tokens_a_block + 2 * v->keys : p->max_length;
    p->aside = std::min<int64_t>(seen, p->max_length) > (int64_t)kAsideTiles * v->keys;
    return FCSIM_OK;
}

// Tensor maps of the cache and of q, for bulk copies, where pages hold whole boxes of 8 tokens or more.  (Other pages and strides are copied row by row.)
using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                 CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
    static std::atomic<void*> known;
    void* f = known.load(std::memory_order_relaxed);
    if (!f) {
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return nullptr;
        }
        known.store(f, std::memory_order_relaxed);
    }
    return (EncodeTiled)f;
}
struct MapDim {
    int64_t size, stride;  // stride in elements; of the first 1
    int box;
};
bool encode(CUtensorMap* map, const void* base, int bytes, int dims, const MapDim* d) {
    const EncodeTiled f = encode_tiled();
    cuuint64_t size[4], stride[4];
    cuuint32_t box[4], ones[4] = {1, 1, 1, 1};
    for (int i = 0; i < dims; i++) {
        size[i] = d[i].size, box[i] = d[i].box;
        if (i == 0) continue;
        stride[i - 1] = (cuuint64_t)d[i].stride * bytes;
        if (d[i].size == 1) stride[i - 1] = std::max<cuuint64_t>(stride[i - 1], 16);  // never taken
        if (stride[i - 1] == 0 || stride[i - 1] >= 1ull << 40) return false;
    }
    return f && f(map, bytes == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16, dims, const_cast<void*>(base), size, stride, box, ones,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
void prefill_maps(PrefillParams* p, const PrefillVariant& v, int bytes) {
    const Pool& c = p->pool;
    p->box = 0, p->kept = p->first;
    if (!v.raw_rows || c.page_size % 8 != 0) return;
    int box = 8;
    while (box * 2 <= v.keys / 2 && c.page_size % (box * 2) == 0) box *= 2;
    p->key_dim = c.stride_slot <= c.stride_head;
    const MapDim slots = {c.page_size, c.stride_slot, box}, heads = {c.n_kv, c.stride_head, 1};
    const MapDim d[4] = {{c.head_dim, 1, 128 / bytes}, p->key_dim ? slots : heads, p->key_dim ? heads : slots, {c.n_pages, c.stride_page, 1}};
    p->query_tokens = 128 % p->heads_a_tile == 0 ? std::min(128 / p->heads_a_tile, p->tokens_a_block) : p->tokens_a_block;
    const MapDim q[3] = {{c.head_dim, 1, 64}, {p->n_heads, p->q_head, p->heads_a_tile}, {p->n_rows, p->q_row, p->query_tokens}};
    if (!encode(&p->k_map, c.k, bytes, 4, d) || !encode(&p->v_map, c.v, bytes, 4, d) || !encode(&p->q_map, p->q, 2, 3, q)) return;
    p->box = box, p->kept = (p->first + box - 1) / box * box;
}

constexpr size_t kPrefillCounters = kMaxCtas * (kThreads / 32) * 4;  // those of attend: one workspace serves both

int prefill_layout(const PrefillParams& p, const PrefillVariant& v, int* device, int* grid, size_t* bytes) {
    int sms = 0, rc = device_and_sms(device, &sms);
    if (rc != FCSIM_OK) return rc;
    // a CTA has an SM to itself; no more of them than tiles that there may be
    const int64_t blocks = (int64_t)p.n_rows / p.tokens_a_block + std::min(p.n_requests, p.n_rows), tiles = (p.max_length + (int64_t)v.keys - 1) / v.keys;
    const int64_t most = std::min<int64_t>(blocks * p.pool.n_kv, 1 << 20) * p.head_tiles * std::max<int64_t>(tiles, 1);
    *grid = (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)sms, (int64_t)kMaxCtas, most}));
    *bytes = kPrefillCounters + (size_t)*grid * (p.aside ? 3 : 2) * (v.rows / 128) * (v.width + 2) * 128 * 4;
    return FCSIM_OK;
}

int check_evict(const fcsim_kv_cache* c, const fcsim_kv_evict_args* a, EvictParams* p) {
    int rc = check_cache(c, &p->pool);
    if (rc != FCSIM_OK) return rc;
    if (!a || a->n_requests < 0 || a->n_requests > 65535) return FCSIM_EINVAL;
    if (a->table_cols < 0 || a->max_length < 0 || a->max_length > (int64_t)a->table_cols * c->page_size) return FCSIM_EINVAL;
    if (a->new_cols < 0 || a->max_budget < 0 || a->max_budget > (int64_t)a->new_cols * c->page_size) return FCSIM_EINVAL;
    if (a->max_length > kMaxTokens || a->max_budget > kMaxTokens) return FCSIM_EINVAL;
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
    if (a->n_tokens < 0 || a->n_tokens > kMaxTokens || a->n_heads < 0 || !(a->eps >= 0) || !isfinite(a->eps)) return FCSIM_EINVAL;
    if ((int64_t)a->n_heads + 2 * c->n_kv_heads > 65535) return FCSIM_EINVAL;
    if (!good_stride(a->q_row, 2) || !good_stride(a->q_head, 2) || !good_stride(a->k_row, 2) ||
        !good_stride(a->k_head, 2) || !good_stride(a->v_row, 2) || !good_stride(a->v_head, 2))
        return FCSIM_EINVAL;
    if (a->rope) {
        if (a->rope_dim < 2 || a->rope_dim > c->head_dim || a->rope_dim % (a->interleaved ? 2 : 16) || a->n_positions < 1)
            return FCSIM_EINVAL;
        if ((uintptr_t)a->rope & (a->interleaved ? 3 : 15)) return FCSIM_ESIZE;
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
    p.n_positions = a->n_positions, p.interleaved = a->rope && a->interleaved, p.eps = a->eps;
    p.one_over_dim = 1.0f / (float)c->head_dim;
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
    const AttendVariant v = attend_variant(c, p, a->dtype);
    p.tile_bits = v.tile_bits;
    AttendLayout l;
    if ((rc = attend_layout(p, v, &l)) != FCSIM_OK) return rc;
    *out = {l.bytes, l.counters};
    return FCSIM_OK;
}

extern "C" int fcsim_kv_attend(const fcsim_kv_cache* c, const fcsim_kv_attend_args* a, void* workspace,
                               size_t workspace_bytes, void* cuda_stream) {
    AttendParams p;
    int rc = check_attend(c, a, &p);
    if (rc != FCSIM_OK) return rc;
    if (p.n_requests == 0) return FCSIM_OK;
    const AttendVariant v = attend_variant(c, p, a->dtype);
    p.tile_bits = v.tile_bits;
    if (!workspace || !aligned16(workspace) || workspace_bytes < attend_kept(p)) return FCSIM_ESIZE;
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
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    int device = 0, sms = 0;
    if ((rc = device_and_sms(&device, &sms)) != FCSIM_OK) return rc;
    // a cluster per (request, kv head), doubled while SMs are idle and a CTA still has two rounds of keys to read
    int ctas = 1;
    while (ctas < kMaxCluster && (int64_t)a->n_requests * p.pool.n_kv * ctas < sms && p.max_length / ctas > 2 * kSelectThreads) ctas *= 2;
    // (and so that the keys fit, whatever the number of rows)
    const int fours = p.max_length / 4 + 2;
    while (ctas < kMaxCluster && (fours + ctas - 1) / ctas > kMaxFours) ctas *= 2;
    const int capacity = std::min((fours + ctas - 1) / ctas, kMaxFours);
    const dim3 grid(ctas, p.pool.n_kv, a->n_requests);
    const int chunks = p.pool.head_dim * p.bytes / 16;
    // One kernel when there is little to copy (4 requests of 515 tokens to 256: 12.1 us a call, with two 13.9); else a second
    // one spreads the copies better (64 requests to 1 024 tokens of 128 elements: 79 us, with one 85).
    const int64_t row_bytes = (int64_t)p.max_budget * p.pool.head_dim * p.bytes * 2;
    if (row_bytes <= kFusedBytes * ctas) {
        if (chunks <= 4) return launch_select<4>(p, grid, capacity, device, stream);
        if (chunks <= 8) return launch_select<8>(p, grid, capacity, device, stream);
        if (chunks <= 16) return launch_select<16>(p, grid, capacity, device, stream);
        return launch_select<32>(p, grid, capacity, device, stream);
    }
    if ((rc = launch_select<0>(p, grid, capacity, device, stream)) != FCSIM_OK) return rc;
    if (chunks <= 4) return launch_move<4>(p, a->n_requests, stream);
    if (chunks <= 8) return launch_move<8>(p, a->n_requests, stream);
    if (chunks <= 16) return launch_move<16>(p, a->n_requests, stream);
    return launch_move<32>(p, a->n_requests, stream);
}

extern "C" int fcsim_kv_prefill_workspace(const fcsim_kv_cache* c, const fcsim_kv_prefill_args* a, fcsim_kv_workspace* out) {
    PrefillParams p;
    PrefillVariant v;
    int rc = check_prefill(c, a, &p, &v);
    if (rc != FCSIM_OK) return rc;
    if (!out) return FCSIM_EINVAL;
    *out = {0, 0};
    if (p.n_rows == 0) return FCSIM_OK;
    int device, grid;
    size_t bytes;
    if ((rc = prefill_layout(p, v, &device, &grid, &bytes)) != FCSIM_OK) return rc;
    *out = {bytes, kPrefillCounters};
    return FCSIM_OK;
}

extern "C" int fcsim_kv_prefill(const fcsim_kv_cache* c, const fcsim_kv_prefill_args* a, void* workspace,
                                size_t workspace_bytes, void* cuda_stream) {
    PrefillParams p;
    PrefillVariant v;
    int rc = check_prefill(c, a, &p, &v);
    if (rc != FCSIM_OK) return rc;
    if (p.n_rows == 0) return FCSIM_OK;
    if (!workspace || !aligned16(workspace) || workspace_bytes < kPrefillCounters) return FCSIM_ESIZE;
    int device, grid;
    size_t bytes;
    if ((rc = prefill_layout(p, v, &device, &grid, &bytes)) != FCSIM_OK) return rc;
    if (workspace_bytes < bytes) return FCSIM_ESIZE;
    p.counters = (int*)workspace, p.parts = (float*)((char*)workspace + kPrefillCounters);
    prefill_maps(&p, v, cache_bytes(c));
    return cuda_status((cudaError_t)v.launch(p, grid, device, (cudaStream_t)cuda_stream));
}

extern "C" int fcsim_kv_read(const fcsim_kv_cache* c, const fcsim_kv_read_args* a, void* cuda_stream) {
    ReadParams p;
    int rc = check_cache(c, &p.pool);
    if (rc != FCSIM_OK) return rc;
    if (!a || (a->dtype != FCSIM_KV_F16 && a->dtype != FCSIM_KV_BF16) || a->n_tokens < 0 || a->n_tokens > kMaxTokens) return FCSIM_EINVAL;
    p.row_pieces = c->head_dim * cache_bytes(c) / 16;
    p.token_pieces = p.row_pieces * c->n_kv_heads;
    p.pieces = (int64_t)p.token_pieces * a->n_tokens;
    if (a->n_tokens == 0) return FCSIM_OK;
    if (!a->slots || !a->k_out || !a->v_out || !aligned16(a->k_out) || !aligned16(a->v_out)) return FCSIM_ESIZE;
    p.slots = a->slots, p.k_out = (char*)a->k_out, p.v_out = (char*)a->v_out, p.status = a->status;
    p.token_magic = ((1ull << 63) + p.token_pieces - 1) / p.token_pieces;
    p.row_magic = ((1ull << 63) + p.row_pieces - 1) / p.row_pieces;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    return a->dtype == FCSIM_KV_F16 ? launch_read_from<F16>(c->dtype, p, stream) : launch_read_from<BF16>(c->dtype, p, stream);
}

extern "C" int fcsim_kv_last_cuda_error(void) { return g_last_cuda_error; }
