// Attention of one query token per request over a paged cache (compiled once per pair of types: FCSIM_KV_TYPES 0..3).
//
//   o_h = sum_t p_t v_t / sum_t p_t,   p_t = exp(c (s_t - m)),   s_t = q_h . k_t,   c = scale,   m = max s_t
//
// Every cached byte is used for 2 * group multiplications (k.q and p.v), so the kernel is bound by the bytes of K and V;
// everything below serves to keep loads in flight on all SMs whatever the lengths are.
//
// * Work is counted in tiles of 64 tokens of one kv head and laid out end to end over all requests; every CTA takes an
//   equal stretch of it (and finds its start by a scan of the lengths), so one request of 131 072 tokens and 500 of a
//   few hundred load the GPU alike and nothing is planned on the host.  A stretch that covers only part of a
//   (request, kv head) leaves its maximum, sum and unnormalised output; the CTA that comes last joins them in a fixed
//   order (no atomics on values: the same call gives the same bits).
// * Each warp copies its own 16 tokens of a tile with cp.async into a ring of its own, and runs ahead over the borders of
//   requests, so the ring never drains at the end of a short one.
// * Both products run on the tensor cores as transposes, tokens (or head_dim) as the 16 rows and the group's query heads
//   as the 8 columns: s^T = K q^T and o^T = V^T p^T, m16n8k16.  A group of 8 heads fills the tile (the other way around
//   half of its 16 rows would be padding), K and V are both read once with ldmatrix, and a column's maximum and sum stay
//   in the lanes that hold it.  The rate needed is two orders below what these instructions give.
// * s, m, the sums and o are 32-bit.  p goes to 16 bits in two parts (p = hi + lo; one where it is f16 and the output
//   bf16), so that rounding it is far below the output's own rounding: one part alone would be as large.  8-bit rows become f16 exactly; a bf16 query beside them is scaled by a
//   power of two per head to lie in f16's range, with at least 38 bits below its largest element.
#include <math.h>

#include <atomic>
#include <type_traits>

#include "fcsim_kv_attend.cuh"

namespace fcsim_kv_dev {
namespace {

__device__ __forceinline__ uint32_t smem_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// 16 bytes global -> shared; with `bytes` = 0 nothing is read and zeros are written
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_group() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void load_matrices(uint32_t a, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void load_matrices_transposed(uint32_t a, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
template <class M>  // M: the type of the tensor-core operands
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same<M, F16>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Two weights in 0 .. 1 as one operand word, and what is left of them as a second.  The first is rounded down and one more
// step below, so that neither is zero unless the weight is nearly (2^-23 for f16): an infinite v then stays infinite.
template <class M>
__device__ __forceinline__ uint32_t below(float a, float b) {
    uint32_t h;
    if constexpr (std::is_same<M, F16>::value)
        asm("cvt.rz.f16x2.f32 %0, %2, %1;" : "=r"(h) : "f"(a), "f"(b));
    else
        h = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
    return __viaddmax_s16x2(h, 0xffffffffu, 0u);
}

template <class T, class C>
struct OperandOf { using type = T; };
template <class T>
struct OperandOf<T, E4M3> { using type = F16; };

// ---------------------------------------------------------------------------------------------- the walk over the work
// A place in the work: request b, head tile r of its `per` (kv head, head tile) pairs, tile j of `tiles`.
struct Place {
    int b, r, j, tiles, start, len;
    int64_t base;  // tiles of the requests before b
};

__device__ __forceinline__ int length_of(const AttendParams& p, int b) {
    const int n = p.lengths[b];
    return n < 0 ? 0 : n > p.max_length ? p.max_length : n;
}
__device__ __forceinline__ int start_of(const AttendParams& p, int len) {
    return p.window > 0 && len > p.window ? len - p.window : 0;
}
__device__ __forceinline__ int tiles_of(const AttendParams& p, int len) {
    return (len - start_of(p, len) + kTile - 1) / kTile;
}
__device__ __forceinline__ void enter(const AttendParams& p, Place& w, int b) {
    w.b = b;
    w.len = length_of(p, b);
    w.start = start_of(p, w.len);
    w.tiles = tiles_of(p, w.len);
}
// The next tile of the work; the caller knows that there is one.
__device__ __forceinline__ void advance(const AttendParams& p, Place& w, int per) {
    if (++w.j < w.tiles) return;
    w.j = 0;
    if (++w.r < per) return;
    w.r = 0;
    w.base += w.tiles;
    do enter(p, w, w.b + 1);
    while (w.tiles == 0);
}

struct Shares {
    int64_t first, end, share;  // this CTA's tiles [first, end); a CTA's share
};

// Divides the tiles of all requests among the CTAs and finds where this CTA's stretch begins.  `per`: how often each
// request's tiles count.  A share is at least `least` tiles, below which joining costs more than it spreads.
__device__ __forceinline__ Shares divide(const AttendParams& p, int per, int least, Place& w) {
    __shared__ int64_t warp_sums[kThreads / 32];
    __shared__ int64_t found_base;
    __shared__ int found_request;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int each = (p.n_requests + kThreads - 1) / kThreads;
    const int b0 = min(tid * each, p.n_requests), b1 = min(b0 + each, p.n_requests);
    int64_t mine = 0;
    for (int b = b0; b < b1; b++) mine += tiles_of(p, length_of(p, b));
    int64_t upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t x = __shfl_up_sync(~0u, upto, d);
        if (lane >= d) upto += x;
    }
    if (lane == 31) warp_sums[warp] = upto;
    __syncthreads();
    int64_t before = 0, total = 0;
#pragma unroll
    for (int i = 0; i < kThreads / 32; i++) {
        if (i < warp) before += warp_sums[i];
        total += warp_sums[i];
    }
    int64_t at = before + upto - mine;  // tiles before this thread's requests
    total *= per;
    Shares s;
    s.share = (total + gridDim.x - 1) / gridDim.x;
    if (s.share < least) s.share = least;
    s.first = min(s.share * (int64_t)blockIdx.x, total);
    s.end = min(s.first + s.share, total);
    if (s.first < s.end && mine > 0 && s.first >= at * per && s.first < (at + mine) * per) {
        int b = b0;
        for (int t; b < b1 && (at + (t = tiles_of(p, length_of(p, b)))) * per <= s.first; b++) at += t;
        found_request = b;
        found_base = at;
    }
    __syncthreads();
    if (s.first < s.end) {
        enter(p, w, found_request);
        w.base = found_base;
        const int64_t in = s.first - w.base * per;
        w.r = (int)(in / w.tiles);
        w.j = (int)(in - (int64_t)w.r * w.tiles);
    }
    return s;
}

// ---------------------------------------------------------------------------------------------- the kernel
// DP: head_dim rounded up to 64, 128 or 256.  NT: column tiles of 8 query heads.
template <class T, class C, int DP, int NT>
struct Shape {
    static constexpr int kRow = DP * C::bytes;                  // bytes of a token's row in shared memory
    static constexpr int kStage = kTile * 2 * kRow;             // K and V of a tile
    static constexpr int kPitch = DP + 4;                       // floats; 4 more: heads fall on different banks
    static constexpr int kMerge = 2 * 8 * NT * kPitch * 4;      // two warps' outputs
    static constexpr int kSmall = 3 * 4 * 8 * NT * 4 + 128;     // statistics of the columns, masks of the ring, a flag
    static constexpr int kTwo = 113 * 1024, kOne = 227 * 1024;  // shared memory of a CTA when two, or one, fit an SM
    static constexpr int kStagesTwo = (kTwo - kMerge - kSmall) / kStage;
    static constexpr int kStagesOne = (kOne - kMerge - kSmall) / kStage;
    // at least three: one in use, two under way
    static constexpr int kStages = kStagesTwo >= 3 ? (kStagesTwo > 6 ? 6 : kStagesTwo) : (kStagesOne > 6 ? 6 : kStagesOne);
    static constexpr int kBytes = kStages * kStage + kMerge + kSmall;
    static_assert(kStages >= 3 && kBytes <= kOne, "shared memory of a CTA");
    // 16-byte chunk c of row t lies at chunk c ^ swizzle(t): eight rows of one column cover all banks
    static __device__ __forceinline__ int swizzle(int t) { return kRow >= 128 ? t & 7 : (t >> 1) & 3; }
};

template <class T, class C, int DP, int NT>
__global__ void __launch_bounds__(kThreads) fcsim_kv_attend_kernel(const AttendParams p) {
    using S = Shape<T, C, DP, NT>;
    using M = typename OperandOf<T, C>::type;
    constexpr bool kNarrow = C::bytes == 1, kRescaled = kNarrow && std::is_same<T, BF16>::value;
    constexpr bool kSplit = !kRescaled;  // f16 weights are 8 times finer than a bf16 output as they are
    constexpr int kCols = 8 * NT, kSteps = DP / 16, kChunks = S::kRow / 16;
    extern __shared__ __align__(128) char smem[];
    float* const merge = reinterpret_cast<float*>(smem + S::kStages * S::kStage);
    float* const warp_m = merge + 2 * kCols * S::kPitch;   // [4][kCols]
    float* const warp_l = warp_m + 4 * kCols;
    float* const col_unit = warp_l + 4 * kCols;            // [kCols]
    int* const last_flag = reinterpret_cast<int*>(col_unit + 4 * kCols);
    uint32_t* const masks = reinterpret_cast<uint32_t*>(last_flag + 1) + (threadIdx.x >> 5) * S::kStages;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int D = p.pool.head_dim, group = p.n_heads / p.pool.n_kv;
    const int head_tiles = (group + kCols - 1) / kCols, per = p.pool.n_kv * head_tiles;

    // requests without tokens
    for (int b = blockIdx.x; b < p.n_requests; b += gridDim.x) {
        const int n = p.lengths[b];
        if ((n < 0 || n > p.max_length) && tid == 0) flag(p.status, FCSIM_KV_BAD_LENGTH);
        if (length_of(p, b) > 0) continue;
        uint4* o = reinterpret_cast<uint4*>(p.out + (int64_t)b * p.n_heads * D * 2);
        for (int i = tid; i < p.n_heads * (D / 8); i += kThreads) o[i] = make_uint4(0, 0, 0, 0);
        if (p.lse)
            for (int i = tid; i < p.n_heads; i += kThreads) p.lse[(int64_t)b * p.n_heads + i] = -INFINITY;
    }

    Place in;  // the tile whose loads are issued next
    const Shares sh = divide(p, per, 4, in);
    int64_t to_load = sh.end - sh.first, to_do = to_load;
    if (to_do == 0) return;
    Place at = in;  // the tile that is computed next

    // columns of a row beyond head_dim are never loaded: zero them once
    const int chunks = D * C::bytes / 16;
    char* const ring = smem + warp * 16 * 2 * S::kRow;  // stage s of this warp: + s * kStage; 16 rows of K, 16 of V
    if (chunks < kChunks) {
        for (int s = 0; s < S::kStages; s++)
            for (int i = lane; i < 32 * kChunks; i += 32) {
                const int t = i / kChunks, c = i % kChunks;
                if (c >= chunks)
                    *reinterpret_cast<uint4*>(ring + s * S::kStage + t * S::kRow + ((c ^ S::swizzle(t & 15)) * 16)) =
                        make_uint4(0, 0, 0, 0);
            }
        __syncwarp();
    }

    // ---- loads: lane i < 16 knows where token i of the warp's 16 lies; the page number is fetched one tile ahead
    int page = -1;
    const int my_token = warp * 16 + (lane & 15);
    auto fetch_page = [&]() {  // for tile `in`
        const int t = in.start + in.j * kTile + my_token;
        page = t < in.len ? p.table[in.b * p.table_row + t / p.pool.page_size] : -1;
    };
    auto issue = [&](int stage) {
        const int t = in.start + in.j * kTile + my_token;
        const bool live = t < in.len, good = live && page >= 0 && page < p.pool.n_pages;
        if (live && !good) flag(p.status, FCSIM_KV_BAD_PAGE);
        const uint32_t mask = __ballot_sync(~0u, good);
        if (lane == 0) masks[stage] = mask;  // tokens that exist, for the computation of this tile
        int64_t offset = -1;
        if (good)
            offset = (page * p.pool.stride_page + (t % p.pool.page_size) * p.pool.stride_slot +
                      (in.r / head_tiles) * p.pool.stride_head) * C::bytes;
        const uint32_t dst = smem_address(ring + stage * S::kStage);
#pragma unroll
        for (int i = 0; i < 16 * kChunks / 32; i++) {
            const int row = (i * 32 + lane) / kChunks, c = lane % kChunks;
            const int64_t o = __shfl_sync(~0u, offset, row);
            if (c < chunks) {
                const uint32_t d = dst + row * S::kRow + ((c ^ S::swizzle(row)) * 16);
                const int64_t src = o < 0 ? 0 : o + c * 16;
                copy16(d, p.pool.k + src, o < 0 ? 0 : 16);
                copy16(d + 16 * S::kRow, p.pool.v + src, o < 0 ? 0 : 16);
            }
        }
    };
    auto load_next = [&](int stage) {
        if (to_load > 0) {
            issue(stage);
            if (--to_load > 0) {
                advance(p, in, per);
                fetch_page();
            }
        }
        commit();
    };
    fetch_page();
#pragma unroll
    for (int s = 0; s < S::kStages - 1; s++) load_next(s);

    uint32_t qf[NT][kSteps][2];  // q^T as the second operand
    float unit[NT][2], m[NT][2], l[NT][2], o[kSteps][NT][4];
    bool fresh = true;
    int stage = 0;
    const float flip = p.scale < 0 ? -1.0f : 1.0f;  // a negative scale turns the order around: turn q instead

    for (int64_t done = 0; done < to_do; done++) {
        const int kv = at.r / head_tiles, col0 = (at.r % head_tiles) * kCols, cols = min(kCols, group - col0);
        if (fresh) {
            fresh = false;
            const float kscale = kNarrow ? p.pool.k_scale[kv] : 1.0f;
#pragma unroll
            for (int nt = 0; nt < NT; nt++) {
                const int col = nt * 8 + lane / 4;
                const char* row = p.q + ((int64_t)at.b * p.q_row + (int64_t)(kv * group + col0 + col) * p.q_head) * 2;
                float big = 0, power = 1;
#pragma unroll
                for (int k = 0; k < kSteps; k++)
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        // 8-bit rows come as four neighbours per lane: the same order for q
                        const int d = kNarrow ? k * 16 + 4 * (lane & 3) + 2 * i : k * 16 + 2 * (lane & 3) + 8 * i;
                        uint32_t x = col < cols && d < D ? *reinterpret_cast<const uint32_t*>(row + d * 2) : 0u;
                        if (flip < 0) x ^= 0x80008000u;
                        qf[nt][k][i] = x;
                        if constexpr (kRescaled) {
                            const float2 f = BF16::unpack(x);
                            big = fmaxf(big, fmaxf(fabsf(f.x), fabsf(f.y)));
                        }
                    }
                if constexpr (kRescaled) {
                    big = fmaxf(big, __shfl_xor_sync(~0u, big, 1));
                    big = fmaxf(big, __shfl_xor_sync(~0u, big, 2));
                    const int e = max((int)(__float_as_uint(big) >> 23), 27);  // biased; infinities stay what they are
                    const float up = e >= 255 ? 1.0f : __uint_as_float((uint32_t)min(127 + 14 + 127 - e, 254) << 23);
                    power = 1.0f / up;  // a power of two: exact
#pragma unroll
                    for (int k = 0; k < kSteps; k++)
#pragma unroll
                        for (int i = 0; i < 2; i++) {
                            const float2 f = BF16::unpack(qf[nt][k][i]);
                            qf[nt][k][i] = F16::pack(f.x * up, f.y * up);
                        }
                }
                const float u = fabsf(p.scale) * kscale * power;
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    unit[nt][i] = __shfl_sync(~0u, u, (2 * (lane & 3) + i) * 4);
                    m[nt][i] = -INFINITY;
                    l[nt][i] = 0;
                }
#pragma unroll
                for (int k = 0; k < kSteps; k++)
#pragma unroll
                    for (int i = 0; i < 4; i++) o[k][nt][i] = 0;
            }
        }

        wait_group<S::kStages - 2>();
        __syncwarp();
        load_next(stage == 0 ? S::kStages - 1 : stage - 1);  // into what the last step has read

        const uint32_t krow = smem_address(ring + stage * S::kStage), vrow = krow + 16 * S::kRow;
        // ---- s^T = K q^T: 16 tokens by 8 heads
        float s[NT][4] = {};
        {
            const int t = (lane & 7) + ((lane >> 3) & 1) * 8;
            const uint32_t row = krow + t * S::kRow;
            if constexpr (!kNarrow) {
#pragma unroll
                for (int k = 0; k < kSteps; k++) {
                    uint32_t a[4];
                    load_matrices(row + (((2 * k + (lane >> 4)) ^ S::swizzle(t)) * 16), a);
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) mma<M>(s[nt], a, qf[nt][k][0], qf[nt][k][1]);
                }
            } else {
#pragma unroll
                for (int k = 0; k < kSteps; k += 2) {
                    uint32_t w[4];
                    load_matrices(row + (((k + (lane >> 4)) ^ S::swizzle(t)) * 16), w);
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        const uint32_t a[4] = {E4M3::halves(w[2 * i] & 0xffff), E4M3::halves(w[2 * i + 1] & 0xffff),
                                               E4M3::halves(w[2 * i] >> 16), E4M3::halves(w[2 * i + 1] >> 16)};
#pragma unroll
                        for (int nt = 0; nt < NT; nt++) mma<M>(s[nt], a, qf[nt][k + i][0], qf[nt][k + i][1]);
                    }
                }
            }
        }
        // ---- softmax: this lane holds tokens lane / 4 and + 8 of heads 2 (lane % 4) and + 1
        const uint32_t live = masks[stage] >> (lane / 4);
        const bool dead[2] = {!(live & 1), !(live & 0x100)};
        uint32_t hi[NT][2], lo[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
            if (p.add_weight && at.base + at.tiles <= p.logit_tiles) {
                float* row = p.logits + (at.base * p.n_heads + (int64_t)(kv * group + col0 + nt * 8) * at.tiles) * kTile +
                             at.j * kTile + warp * 16 + lane / 4;
#pragma unroll
                for (int i = 0; i < 2; i++)
                    if (nt * 8 + 2 * (lane & 3) + i < cols) {
                        float* x = row + (int64_t)(2 * (lane & 3) + i) * at.tiles * kTile;
                        x[0] = s[nt][i];
                        x[8] = s[nt][2 + i];
                    }
            }
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (dead[i >> 1]) s[nt][i] = -INFINITY;
            float shrink[2];
#pragma unroll
            for (int i = 0; i < 2; i++) {
                float top = fmaxf(s[nt][i], s[nt][2 + i]);
                top = fmaxf(top, __shfl_xor_sync(~0u, top, 4));
                top = fmaxf(top, __shfl_xor_sync(~0u, top, 8));
                top = fmaxf(top, __shfl_xor_sync(~0u, top, 16));
                top = fmaxf(top, m[nt][i]);
                const float base = top == -INFINITY ? 0.0f : top, u = unit[nt][i] * 1.4426950408889634f;
                shrink[i] = m[nt][i] == -INFINITY ? 0.0f : exp2f((m[nt][i] - base) * u);
                m[nt][i] = top;
                float sum = 0;
#pragma unroll
                for (int k = 0; k < 2; k++) {
                    const float e = dead[k] ? 0.0f : exp2f((s[nt][2 * k + i] - base) * u);
                    s[nt][2 * k + i] = e;
                    sum += e;
                }
                l[nt][i] = l[nt][i] * shrink[i] + sum;
            }
#pragma unroll
            for (int k = 0; k < 2; k++) {
                const float a = s[nt][2 * k], b = s[nt][2 * k + 1];
                if constexpr (kSplit) {
                    const uint32_t h = below<M>(a, b);
                    const float2 back = M::unpack(h);
                    hi[nt][k] = transpose8x8(h);
                    lo[nt][k] = transpose8x8(M::pack(a - back.x, b - back.y));
                } else
                    hi[nt][k] = transpose8x8(M::pack(a, b));
            }
            if (__any_sync(~0u, shrink[0] != 1.0f || shrink[1] != 1.0f)) {
#pragma unroll
                for (int k = 0; k < kSteps; k++)
#pragma unroll
                    for (int i = 0; i < 4; i++) o[k][nt][i] *= shrink[i & 1];
            }
        }
        // ---- o^T += V^T p^T: 16 elements of head_dim by 8 heads
        {
            const int which = lane >> 3;
            if constexpr (!kNarrow) {
                const int t = (lane & 7) + (which >> 1) * 8;
#pragma unroll
                for (int k = 0; k < kSteps; k++) {
                    uint32_t a[4];
                    load_matrices_transposed(vrow + t * S::kRow + (((2 * k + (which & 1)) ^ S::swizzle(t)) * 16), a);
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) {
                        mma<M>(o[k][nt], a, hi[nt][0], hi[nt][1]);
                        if constexpr (kSplit) mma<M>(o[k][nt], a, lo[nt][0], lo[nt][1]);
                    }
                }
            } else {
                const int t = (lane & 7) + (which & 1) * 8;
#pragma unroll
                for (int k = 0; k < kSteps; k += 2) {
                    // a lane gets bytes 2n, 2n + 1 of two tokens: even and odd elements become rows n and n + 8
                    uint32_t w[4];
                    load_matrices_transposed(vrow + t * S::kRow + (((k + (which >> 1)) ^ S::swizzle(t)) * 16), w);
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        const uint32_t x = w[2 * i], y = w[2 * i + 1];
                        const uint32_t a[4] = {E4M3::halves(__byte_perm(x, 0, 0x4420)), E4M3::halves(__byte_perm(x, 0, 0x4431)),
                                               E4M3::halves(__byte_perm(y, 0, 0x4420)), E4M3::halves(__byte_perm(y, 0, 0x4431))};
#pragma unroll
                        for (int nt = 0; nt < NT; nt++) {
                            mma<M>(o[k + i][nt], a, hi[nt][0], hi[nt][1]);
                            if constexpr (kSplit) mma<M>(o[k + i][nt], a, lo[nt][0], lo[nt][1]);
                        }
                    }
                }
            }
        }
        stage = stage == S::kStages - 1 ? 0 : stage + 1;

        const bool complete = at.j == at.tiles - 1, ends = complete || done + 1 == to_do;
        if (!ends) {
            at.j++;
            continue;
        }
        // ---------------------------------------------------------------- end of this CTA's part of (request, head tile)
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int i = 0; i < 2; i++) {
                float x = l[nt][i];
                x += __shfl_xor_sync(~0u, x, 4);
                x += __shfl_xor_sync(~0u, x, 8);
                x += __shfl_xor_sync(~0u, x, 16);
                l[nt][i] = x;
                if (lane < 4) {
                    const int col = nt * 8 + 2 * lane + i;
                    warp_m[warp * kCols + col] = m[nt][i];
                    warp_l[warp * kCols + col] = x;
                    if (warp == 0) col_unit[col] = unit[nt][i];
                }
            }
        __syncthreads();
        // bring the four warps to one maximum, then add their outputs: 2 and 3 write, 0 and 1 add, all finish
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const int col = nt * 8 + 2 * (lane & 3) + i;
                const float top = fmaxf(fmaxf(warp_m[col], warp_m[kCols + col]), fmaxf(warp_m[2 * kCols + col], warp_m[3 * kCols + col]));
                const float base = top == -INFINITY ? 0.0f : top;
                const float f = m[nt][i] == -INFINITY ? 0.0f : exp2f((m[nt][i] - base) * unit[nt][i] * 1.4426950408889634f);
#pragma unroll
                for (int k = 0; k < kSteps; k++) {
                    o[k][nt][i] *= f;
                    o[k][nt][2 + i] *= f;
                }
            }
        auto element = [&](int k, int nt, int i) {  // where o[k][nt][i] lies in a merge buffer
            const int d = kNarrow ? k * 16 + 2 * (lane / 4) + (i >> 1) : k * 16 + lane / 4 + 8 * (i >> 1);
            return (warp & 1) * kCols * S::kPitch + (nt * 8 + 2 * (lane & 3) + (i & 1)) * S::kPitch + d;
        };
        if (warp >= 2) {
#pragma unroll
            for (int k = 0; k < kSteps; k++)
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int i = 0; i < 4; i++) merge[element(k, nt, i)] = o[k][nt][i];
        }
        __syncthreads();
        if (warp < 2) {
#pragma unroll
            for (int k = 0; k < kSteps; k++)
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int i = 0; i < 4; i++) merge[element(k, nt, i)] += o[k][nt][i];
        }
        __syncthreads();

        // where this (request, head tile) begins and ends in the work, and which CTAs share it
        const int64_t group_first = sh.first + done - at.j, group_end = group_first + at.tiles;
        const int first_cta = (int)(group_first / sh.share), last_cta = (int)((group_end - 1) / sh.share);
        const int parts = last_cta - first_cta + 1;
        const int64_t head0 = (int64_t)at.b * p.n_heads + kv * group + col0;
        const float vscale = kNarrow ? p.pool.v_scale[kv] : 1.0f;
        auto finish = [&](int col, float top, float sum) {  // one lane per head: log-sum-exp and statistics
            const float u = col_unit[col];
            if (p.lse) p.lse[head0 + col] = sum == 0.0f ? -INFINITY : top * u + logf(sum);
            if (p.add_weight)
                *reinterpret_cast<float4*>(p.stats + (head0 + col) * 4) =
                    make_float4(top == -INFINITY ? 0.0f : top, u * 1.4426950408889634f, sum == 0.0f ? 0.0f : 1.0f / sum, 0.0f);
        };
        constexpr int kPartSize = kCols * (DP + 2);
        float* const my_part = p.parts + (2 * (int64_t)blockIdx.x + (first_cta == (int)blockIdx.x ? 1 : 0)) * kPartSize;
        const int per_row = D / 4;
        for (int i = tid; i < cols * per_row; i += kThreads) {
            const int col = i / per_row, d = (i - col * per_row) * 4;
            const float4 x = *reinterpret_cast<const float4*>(merge + col * S::kPitch + d);
            const float4 y = *reinterpret_cast<const float4*>(merge + (kCols + col) * S::kPitch + d);
            const float4 z = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
            float sum = 0, top = -INFINITY;
#pragma unroll
            for (int w = 0; w < 4; w++) top = fmaxf(top, warp_m[w * kCols + col]);
            const float base = top == -INFINITY ? 0.0f : top, u = col_unit[col] * 1.4426950408889634f;
#pragma unroll
            for (int w = 0; w < 4; w++) {
                const float x = warp_m[w * kCols + col];  // -infinity: the sum is 0, or NaN and stays so
                sum += warp_l[w * kCols + col] * (x == -INFINITY ? 0.0f : exp2f((x - base) * u));
            }
            if (parts == 1) {
                const float f = sum == 0.0f ? 0.0f : vscale / sum;
                *reinterpret_cast<uint2*>(p.out + ((head0 + col) * D + d) * 2) =
                    sum == 0.0f ? make_uint2(0, 0) : make_uint2(T::pack(z.x * f, z.y * f), T::pack(z.z * f, z.w * f));
                if (d == 0) finish(col, top, sum);
            } else {
                *reinterpret_cast<float4*>(my_part + col * DP + d) = z;
                if (d == 0) *reinterpret_cast<float2*>(my_part + kCols * DP + col * 2) = make_float2(top, sum);
            }
        }
        if (parts > 1) {
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                const int before = atomicAdd(p.counters + first_cta, 1);
                *last_flag = before == parts - 1;
                if (before == parts - 1) p.counters[first_cta] = 0;
            }
            __syncthreads();
            if (*last_flag) {
                __threadfence();
                auto part = [&](int i) {
                    return p.parts + (2 * (int64_t)(first_cta + i) + (i == 0 ? 1 : 0)) * kPartSize;
                };
                for (int i = tid; i < cols * per_row; i += kThreads) {
                    const int col = i / per_row, d = (i - col * per_row) * 4;
                    const float u = col_unit[col] * 1.4426950408889634f;
                    float top = -INFINITY, sum = 0;
                    for (int k = 0; k < parts; k++) top = fmaxf(top, __ldcg(part(k) + kCols * DP + col * 2));
                    const float base = top == -INFINITY ? 0.0f : top;
                    float4 z = make_float4(0, 0, 0, 0);
#pragma unroll 4
                    for (int k = 0; k < parts; k++) {
                        const float2 ml = __ldcg(reinterpret_cast<const float2*>(part(k) + kCols * DP + col * 2));
                        const float4 x = __ldcg(reinterpret_cast<const float4*>(part(k) + col * DP + d));
                        const float f = ml.x == -INFINITY ? 0.0f : exp2f((ml.x - base) * u);
                        sum += f * ml.y;
                        z.x += f * x.x, z.y += f * x.y, z.z += f * x.z, z.w += f * x.w;
                    }
                    const float f = sum == 0.0f ? 0.0f : vscale / sum;
                    *reinterpret_cast<uint2*>(p.out + ((head0 + col) * D + d) * 2) =
                        sum == 0.0f ? make_uint2(0, 0) : make_uint2(T::pack(z.x * f, z.y * f), T::pack(z.z * f, z.w * f));
                    if (d == 0) finish(col, top, sum);
                }
            }
        }
        __syncthreads();  // the merge buffers and the columns' statistics are free again
        if (done + 1 < to_do) {
            advance(p, at, per);
            fresh = true;
        }
    }
    wait_group<0>();
}

template <class T, class C, int DP, int NT>
int launch(const AttendParams& p, int grid, cudaStream_t stream) {
    using S = Shape<T, C, DP, NT>;
    fcsim_kv_attend_kernel<T, C, DP, NT><<<grid, kThreads, S::kBytes, stream>>>(p);
    return (int)cudaGetLastError();
}
template <class T, class C, int DP, int NT>
int ctas_per_sm(int device, int* out) {
    using S = Shape<T, C, DP, NT>;
    static std::atomic<int> known[kMaxDevices];
    int n = device < kMaxDevices ? known[device].load(std::memory_order_relaxed) : 0;
    if (n == 0) {
        auto* kernel = fcsim_kv_attend_kernel<T, C, DP, NT>;
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kBytes);
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, kThreads, S::kBytes);
        if (e != cudaSuccess) return (int)e;
        if (device < kMaxDevices) known[device].store(n, std::memory_order_relaxed);
    }
    *out = n;
    return 0;
}
template <class T, class C, int DP>
AttendVariant of_group(int group) {
    // more than 8 heads: two column tiles share every load from shared memory; beyond 16 the rows are read again
    if (group <= 8) return {launch<T, C, DP, 1>, ctas_per_sm<T, C, DP, 1>, 8, DP};
    return {launch<T, C, DP, 2>, ctas_per_sm<T, C, DP, 2>, 16, DP};
}
template <class T, class C>
AttendVariant of(int head_dim, int group) {
    return head_dim <= 64 ? of_group<T, C, 64>(group) : head_dim <= 128 ? of_group<T, C, 128>(group) : of_group<T, C, 256>(group);
}

}  // namespace

#if FCSIM_KV_TYPES == 0
AttendVariant attend_variant_f16(int head_dim, int group) { return of<F16, F16>(head_dim, group); }
#elif FCSIM_KV_TYPES == 1
AttendVariant attend_variant_bf16(int head_dim, int group) { return of<BF16, BF16>(head_dim, group); }
#elif FCSIM_KV_TYPES == 2
AttendVariant attend_variant_f16_e4m3(int head_dim, int group) { return of<F16, E4M3>(head_dim, group); }
#else
AttendVariant attend_variant_bf16_e4m3(int head_dim, int group) { return of<BF16, E4M3>(head_dim, group); }
#endif

#if FCSIM_KV_TYPES == 0
// weight[token] += sum over a group's heads of the softmax weights, from the logits that the first kernel left: the final
// maximum and sum of a head are known only when all of its parts are joined.  The same division of the work, a thread
// per token and kv head; the sum over the heads in order.
__global__ void __launch_bounds__(kThreads) fcsim_kv_weight_kernel(const AttendParams p) {
    Place at;
    const Shares sh = divide(p, 1, 1, at);
    const int group = p.n_heads / p.pool.n_kv;
    for (int64_t i = sh.first; i < sh.end; i++) {
        const int in = at.j * kTile + (threadIdx.x & (kTile - 1)), t = at.start + in;
        if (at.base + at.tiles > p.logit_tiles) {
            if (threadIdx.x == 0) flag(p.status, FCSIM_KV_BAD_PAGE);  // more tokens than the pool has: pages are shared
        } else if (t < at.len) {
            const int page = p.table[at.b * p.table_row + t / p.pool.page_size];
            if (page >= 0 && page < p.pool.n_pages) {
                const float* row = p.logits + at.base * p.n_heads * kTile + in;
                const float4* stats = reinterpret_cast<const float4*>(p.stats) + (int64_t)at.b * p.n_heads;
                for (int kv = threadIdx.x / kTile; kv < p.pool.n_kv; kv += kThreads / kTile) {
                    float sum = 0;
                    for (int h = kv * group; h < (kv + 1) * group; h++) {
                        const float4 x = stats[h];
                        sum += exp2f((row[(int64_t)h * at.tiles * kTile] - x.x) * x.y) * x.z;
                    }
                    p.pool.weight[((int64_t)page * p.pool.n_kv + kv) * p.pool.page_size + t % p.pool.page_size] += sum;
                }
            }
        }
        if (i + 1 < sh.end) advance(p, at, 1);
    }
}
int launch_weights(const AttendParams& p, int grid, cudaStream_t stream) {
    fcsim_kv_weight_kernel<<<grid, kThreads, 0, stream>>>(p);
    return (int)cudaGetLastError();
}
#endif

}  // namespace fcsim_kv_dev
