// Attention of one query token per request over a paged cache (compiled once per pair of types: FCSIM_KV_TYPES 0..3).
//
//   o_h = sum_t p_t v_t / sum_t p_t,   p_t = exp(c (s_t - m)),   s_t = q_h . k_t,   c = scale,   m = max s_t
//
// Every cached byte is used for 2 * group multiplications (k.q and p.v), so the kernel is bound by the bytes of K and V;
// everything below serves to keep loads in flight on all SMs whatever the lengths are.
//
// * Work is counted in tiles of one kv head and laid out end to end over all requests; every CTA (every warp, where requests
//   are short) takes an equal stretch of it and finds its start by a scan of the lengths, so one request of 131 072 tokens
//   and 500 of a few hundred load the GPU alike and nothing is planned on the host.  A stretch that covers only part of a
//   (request, kv head) leaves its maximum, sum and unnormalised output; the one that comes last joins them in a fixed
//   order (no atomics on values: the same call gives the same bits).
// * Each warp copies its own 16 or 32 tokens of a tile with cp.async into a ring of its own, and runs ahead over the borders of
//   requests, so the ring never drains at the end of a short one.
// * Both products run on the tensor cores as transposes, tokens (or head_dim) as the 16 rows and the group's query heads
//   as the 8 columns: s^T = K q^T and o^T = V^T p^T, m16n8k16.  A group of 8 heads fills the tile (the other way around
//   half of its 16 rows would be padding), K and V are both read once with ldmatrix, and a column's maximum and sum stay
//   in the lanes that hold it.  The rate needed is two orders below what these instructions give.
// * s, m, the sums and o are 32-bit.  p meets v in 16-bit parts that add up to it, two of f16 (11 bits each) or three of bf16 (8
//   each), so that nothing is lost beside the 32-bit sums: with one part less the output is 1.6e-4 (bf16) or 8.5e-4 (f16 weights of
//   a bf16 output) of its norm from the same sums in 32 bits, with all 4e-5 and 7e-5.  The products cost nothing for bf16 (128
//   requests 189.7 -> 190.0 us), 2 us of 80 over e4m3.  8-bit rows become f16 exactly; a bf16 query beside them is scaled by a
//   power of two per head to lie in f16's range: exact down to 2^-31 of its largest finite element, nothing below 2^-38.  (A
//   second path for such queries, by bands of 30 bits, took 83 -> 90 us from all of them.)
#include <math.h>

#include <atomic>
#include <type_traits>

#include "fcsim_kv_attend.cuh"

namespace fcsim_kv_dev {
namespace {

__device__ __forceinline__ uint32_t smem_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// 16 bytes global -> shared; with `bytes` = 0 nothing is read and zeros are written
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_group() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// 2^x; results below 2^-126 are 0
__device__ __forceinline__ float power2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
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
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
template <class M>  // M: the type of the tensor-core operands
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same<M, F16>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// 64 8-bit elements at `row` (per lane) + 0 .. 63 of 16 tokens, transposed, as the first operand of four products.  A lane gets bytes
// 2n, 2n + 1 of two tokens: even and odd elements become rows n and n + 8.
__device__ __forceinline__ void load_narrow_transposed(uint32_t row, uint32_t (&a)[4][4]) {
    uint32_t w[2][4];
    load_matrices_transposed(row, w[0]);
    load_matrices_transposed(row + 32, w[1]);
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const uint32_t x = w[k / 2][2 * (k & 1)], y = w[k / 2][2 * (k & 1) + 1];
        a[k][0] = E4M3::halves(__byte_perm(x, 0, 0x4420)), a[k][1] = E4M3::halves(__byte_perm(x, 0, 0x4431));
        a[k][2] = E4M3::halves(__byte_perm(y, 0, 0x4420)), a[k][3] = E4M3::halves(__byte_perm(y, 0, 0x4431));
    }
}

// Two weights as one operand word, rounded down and one more step below: what is left of them for the next part is above zero
// then, and no part is zero unless the weight is nearly (2^-23 for f16), so that an infinite v stays infinite.
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
// The work is counted in units: a tile is one, and every (request, kv head, head tile) group counts some more for its start
// and its end (q, the warps' merge, the output), which is what they cost beside a tile.  The units before a group's
// first tile stand for these.  Three ways to divide them, by what the lengths add up to:
//   shares  every CTA an equal stretch of units, a tile at a time by its four warps;
//   cut     few tiles: the groups are cut into equal pieces and each CTA gets one, so that starts, ends and joins do not follow
//           one another (16 requests of 1 024 tokens; 30 of 90 to 300, whole, with their append 22 us, by shares 36);
//   alone   short requests in number: every warp an equal stretch, a tile being its own 16 or 32 tokens: a group of one or two
//           tiles is nearly all start and end, and four at a time hide what one waits for (400 requests of up to 70 tokens,
//           64 heads on 8: 56 -> 32 us; 512 of 300: 130 -> 115).  A short group is the work of the warp in whose stretch its
//           first tile lies, so that it need not be joined.
constexpr int kOverhead = 3;       // units of a group's start and end: shares
constexpr int kOverheadAlone = 3;  // alone
constexpr int kPieceLeast = 4;     // tiles of a piece at least: below that, joining costs more than it spreads
constexpr int kPieceMost = 16;     // tiles of a piece from which equal shares are better
// Warps work alone if they get two groups each of up to kAloneMost tiles on average; if half of them get a group and none is
// longer than kWhole (128 requests of 256 tokens: 38 -> 29 us, 256 of 256: 62 -> 53; with longer ones among them equal shares
// win: 114 requests of 1 to 2 500 tokens, 574 on average, with their append 71 us, alone 85); and if groups have kAloneAlways on average.
constexpr int kAloneMost = 16;
constexpr int kAloneAlways = 2;
// Tiles of a warp up to which a group is not cut for a warp that works alone: all groups whole, or those that change little
// (512 of 600 on average, 8, 16, 32 tiles: 81, 84, 95 us).
constexpr int kWhole = 16;
constexpr int kWholeAmongLonger = 8;

// A place in the work: request b, its group (kv head, head tile), tile j of `tiles`.
struct Place {
    int b, kv, ht, j, tiles, gap, seen;
    int left;              // units from this tile to the end of the worker's stretch; none: the place is beyond it
    int tiles_before;      // tiles (of a CTA) of the requests before b
};

__device__ __forceinline__ int length_of(const AttendParams& p, int b) {
    const int n = p.lengths[b];
    return n < 0 ? 0 : n > p.max_length ? p.max_length : n;
}
// Tokens between the first ones and the window, which are not seen.  What is seen is counted without them: seen token u is token
// u, or behind the first ones u + gap.  (Kernels for calls without first tokens are compiled for themselves: with the comparison, and
// that of the runs of 16 tokens below, in their tile loop too, 64 requests over e4m3 took 83.8 us instead of 82.6, and one of 131 072
// tokens 96.9 instead of 96.0.)
__device__ __forceinline__ int gap_of(const AttendParams& p, int len) { return max(len - p.most_seen, 0); }
template <bool FIRST>
__device__ __forceinline__ int token_of(const AttendParams& p, int gap, int u) {
    return FIRST && u < p.first ? u : u + gap;
}
__device__ __forceinline__ int tiles_of(const AttendParams& p, int len, int bits) {
    return (len - gap_of(p, len) + (1 << bits) - 1) >> bits;
}

// The division of the units [0, total) among the workers (CTAs or warps): worker i has [i * share, (i + 1) * share).  It
// depends on the lengths and the grid alone, so the same call gives the same sums in the same order.
// With `cut`, a unit is a piece of at most `cut` tiles of one group, and a share is one unit.
struct Division {
    int64_t total, share;
    int cut, over, bits;  // bits: of the tokens of a tile
    int most;             // tiles of a group that is not cut (alone; else none)
    bool alone;
    __device__ __forceinline__ int worker(int warp) const { return alone ? blockIdx.x * (kThreads / 32) + warp : blockIdx.x; }
    __device__ __forceinline__ int64_t first(int worker) const { return min(total, worker * share); }
    __device__ __forceinline__ int64_t end(int worker) const { return min(total, (worker + 1) * share); }
    __device__ __forceinline__ bool whole(int tiles) const { return tiles <= most; }
    __device__ __forceinline__ int units(int tiles) const { return cut ? (tiles + cut - 1) / cut : tiles ? tiles + over : 0; }
};

__device__ __forceinline__ void enter(const AttendParams& p, const Division& d, Place& w, int b) {
    w.b = b;
    const int len = length_of(p, b);
    w.gap = gap_of(p, len);
    w.seen = len - w.gap;
    w.tiles = (w.seen + (1 << d.bits) - 1) >> d.bits;
}
// The next group of the work; the caller knows that there is one (the lengths stay as they are during a call; if they do not,
// the results are wrong, but nothing beyond the last request is read).
__device__ __forceinline__ void next_group(const AttendParams& p, const Division& d, Place& w, int n_kv, int head_tiles) {
    w.j = 0;
    if (++w.ht < head_tiles) return;
    w.ht = 0;
    if (++w.kv < n_kv) return;
    w.kv = 0;
    w.tiles_before += (w.seen + (1 << p.tile_bits) - 1) >> p.tile_bits;
    do {
        if (w.b + 1 >= p.n_requests) {
            w.left = 0;
            return;
        }
        enter(p, d, w, w.b + 1);
    } while (w.tiles == 0);
}
// The next tile, if the stretch has one more.  (In a group that is not cut, `left` stays at its first tile.)
__device__ __forceinline__ void advance(const AttendParams& p, const Division& d, Place& w, int n_kv, int head_tiles) {
    const bool whole = d.whole(w.tiles);
    if (!whole) w.left--;
    if (++w.j < w.tiles) return;
    w.left -= d.over + (whole ? w.tiles : 0);
    if (w.left > 0) next_group(p, d, w, n_kv, head_tiles);
}

// What the threads' stretches of the requests add up to before each of them.
struct Before {
    int tiles[kThreads], units[kThreads + 1];  // (tiles of a CTA; units of one of a request's groups)
    int warps[2][kThreads / 32];
    int longest[kThreads / 32];  // tiles of a CTA
};

// Running sums over the threads (exclusive), and the totals.
__device__ __forceinline__ void sums_before(Before& s, int& x, int& y, int& all_x, int& all_y) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int upto_x = x, upto_y = y;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int u = __shfl_up_sync(~0u, upto_x, d), v = __shfl_up_sync(~0u, upto_y, d);
        if (lane >= d) upto_x += u, upto_y += v;
    }
    if (lane == 31) s.warps[0][warp] = upto_x, s.warps[1][warp] = upto_y;
    __syncthreads();
    x = upto_x - x, y = upto_y - y;
    all_x = all_y = 0;
#pragma unroll
    for (int i = 0; i < kThreads / 32; i++) {
        if (i < warp) x += s.warps[0][i], y += s.warps[1][i];
        all_x += s.warps[0][i], all_y += s.warps[1][i];
    }
}

// Adds up the tiles of all requests (less than 2^31: the host refuses more; a request has `per` groups) and divides them.
// `warp_bits`: of a warp's tokens; 0 = equal shares without overhead and no other way.
__device__ __forceinline__ Division divide(const AttendParams& p, int per, int warp_bits, Before& before) {
    const int tid = threadIdx.x;
    const int each = (p.n_requests + kThreads - 1) / kThreads;
    const int b0 = min(tid * each, p.n_requests), b1 = min(b0 + each, p.n_requests);
    int tiles = 0, live = 0, longest = 0, all_tiles, all_live;
    for (int b = b0; b < b1; b++) {
        const int t = tiles_of(p, length_of(p, b), p.tile_bits);
        tiles += t;
        live += t > 0;
        longest = max(longest, t);
    }
    longest = __reduce_max_sync(~0u, longest);
    if ((tid & 31) == 0) before.longest[tid >> 5] = longest;
    sums_before(before, tiles, live, all_tiles, all_live);
#pragma unroll
    for (int i = 0; i < kThreads / 32; i++) longest = max(longest, before.longest[i]);
    const bool longer = longest > kWhole / (kThreads / 32);
    Division d;
    d.cut = 0;
    d.over = warp_bits ? kOverhead : 0;
    d.bits = p.tile_bits;
    d.alone = false;
    d.most = 0;
    const int64_t groups = (int64_t)all_live * per, spare = gridDim.x - groups;
    const int64_t warps = (int64_t)gridDim.x * (kThreads / 32);
    if (warp_bits) {
        if (spare >= 0) {  // so that the pieces fit the grid
            int64_t piece = longest;
            if (spare > 0) piece = min(piece, max((int64_t)kPieceLeast, ((int64_t)all_tiles * per + spare - 1) / spare));
            if (piece <= kPieceMost) d.cut = (int)max((int64_t)kPieceLeast, piece);
        } else if ((groups >= 2 * warps && all_tiles <= (int64_t)kAloneMost * all_live) || (2 * groups >= warps && !longer) ||
                   all_tiles <= (int64_t)kAloneAlways * all_live) {
            d.alone = true;
            d.most = longer ? kWholeAmongLonger : kWhole;
            d.over = kOverheadAlone;
            d.bits = warp_bits;
        }
    }
    int all_units = all_tiles + d.over * all_live, units = tiles + d.over * live;
    if (d.cut || d.alone) {
        int none = 0, all_none;
        units = 0;
        for (int b = b0; b < b1; b++) units += d.units(tiles_of(p, length_of(p, b), d.bits));
        __syncthreads();
        sums_before(before, units, none, all_units, all_none);
    }
    const int workers = d.alone ? gridDim.x * (kThreads / 32) : gridDim.x;
    d.total = (int64_t)all_units * per;
    d.share = d.cut ? 1 : max((int64_t)1, (d.total + workers - 1) / workers);
    before.tiles[tid] = tiles;
    before.units[tid] = units;
    if (tid == 0) before.units[kThreads] = all_units;
    __syncthreads();
    return d;
}

// The first tile of a warp's worker, if it has units (less than 2^31: the host refuses more).
// Pieces that are cut to fit: which of the group's `cuts` this is.
__device__ __forceinline__ void locate(const AttendParams& p, int n_kv, int head_tiles, const Division& d, const Before& before, Place& w,
                                       int& cut, int& cuts) {
    constexpr int kWarps = kThreads / 32;
    __shared__ int64_t found_units[kWarps];
    __shared__ int found_request[kWarps], found_tiles[kWarps];
    const int tid = threadIdx.x, warp = tid >> 5, per = n_kv * head_tiles, each = (p.n_requests + kThreads - 1) / kThreads;
    const int64_t units0 = (int64_t)before.units[tid] * per, units1 = (int64_t)before.units[tid + 1] * per;
    for (int i = 0; i < (d.alone ? kWarps : 1); i++) {
        const int64_t first = d.first(d.worker(i));
        if (first < units0 || first >= units1) continue;
        int64_t units = units0;
        int tiles = before.tiles[tid], b = tid * each;
        for (const int last = min(b + each, p.n_requests) - 1; b < last; b++) {
            const int n = length_of(p, b);
            const int64_t u = (int64_t)d.units(tiles_of(p, n, d.bits)) * per;
            if (units + u > first) break;
            tiles += tiles_of(p, n, p.tile_bits), units += u;
        }
        found_request[i] = b;
        found_tiles[i] = tiles;
        found_units[i] = units;
    }
    __syncthreads();
    const int mine = d.alone ? warp : 0;
    const int64_t first = d.first(d.worker(warp)), end = d.end(d.worker(warp));
    w.left = 0;
    if (first >= end) return;
    enter(p, d, w, min(max(found_request[mine], 0), p.n_requests - 1));
    w.tiles_before = found_tiles[mine];
    const int64_t in = first - found_units[mine];
    const int cost = d.units(w.tiles);
    const int r = cost > 0 ? (int)(in / cost) : -1, x = (int)(in - (int64_t)r * cost);
    if (r < 0 || r >= per) return;  // (lengths that changed since they were added up: see next_group)
    w.kv = r / head_tiles;
    w.ht = r - w.kv * head_tiles;
    if (d.cut) {
        cut = x, cuts = cost;
        w.j = (int)((int64_t)w.tiles * x / cost);
        w.left = (int)((int64_t)w.tiles * (x + 1) / cost) - w.j;
    } else {
        w.j = max(0, x - d.over);
        w.left = (int)(end - first) - max(0, d.over - x);
        if (d.whole(w.tiles) && w.j > 0) {  // the worker before has it all
            w.left = (int)(end - first) - (cost - x) - d.over;
            if (w.left > 0) next_group(p, d, w, n_kv, head_tiles);
        }
    }
}

// ---------------------------------------------------------------------------------------------- the kernel
// DP: head_dim rounded up to 64, 128 or 256.  NT: column tiles of 8 query heads.
template <class T, class C, int DP, int NT>
struct Shape {
    static constexpr int kRow = DP * C::bytes;
    static constexpr int kPitch = kRow + 16;                    // bytes of a row in shared memory: 8 rows of a column cover all banks
    // tokens of a warp: 8-bit rows want twice as many for each tile's fixed work (64 requests over e4m3, 94 -> 83 us; 16-bit rows of
    // 128 bytes lose more by fewer CTAs on an SM: 100 requests in f16, 40.0 -> 42.6)
    static constexpr int kTokens = C::bytes == 1 && kRow == 128 ? 32 : 16;
    static constexpr int kTile = 4 * kTokens, kTileBits = kTokens == 32 ? 7 : 6;
    static constexpr int kStage = kTile * 2 * kPitch;           // K and V of a tile
    static constexpr int kOutPitch = DP + 4;                    // floats; 4 more: heads fall on different banks
    static constexpr int kMerge = 2 * 8 * NT * kOutPitch * 4;   // two warps' outputs
    static constexpr int kSmall = 3 * 4 * 8 * NT * 4 + 128;     // statistics of the columns, masks of the rings, a flag
    static constexpr int kStatic = sizeof(Before) + 64;
    static constexpr int stages(int ctas) { return ((228 / ctas - 1) * 1024 - kMerge - kSmall - kStatic) / kStage; }
    // As many CTAs on an SM (three at most) as registers and two stages each allow, then as many stages as there is room for.  When every SM
    // has work for long, only kFair of them are used: more only queue, SMs differ more in the rate they get, and a call
    // ends with the slowest (131 072 tokens of one request, three stages of 32 KB 100 us, two 96; 128 heavy-tailed requests 196, 190).  When each CTA has one
    // short piece, all: nothing but the loads' latency counts (16 requests of 1 024 tokens 22 -> 18 us).
    static constexpr int kRegisterCtas = DP * NT <= 128 && kRow <= 128 ? 3 : 2;
    static constexpr int kCtas = stages(kRegisterCtas) >= 2 ? kRegisterCtas : stages(2) >= 2 ? 2 : 1;
    static constexpr int kStages = stages(kCtas) < 4 ? stages(kCtas) : 4;
    static constexpr int kFair = kCtas * kStage >= 64 * 1024 || kStages < 3 ? 2 : 3;
    // parts that a join takes at once: as many as the ring holds, and their factors the merge buffers
    static constexpr int kInRing = kStages * kStage / (8 * NT * (DP + 2) * 4), kInMerge = kMerge / (8 * NT * 8);
    static constexpr int kJoined = kInRing < kInMerge ? kInRing : kInMerge;
    static constexpr int kBytes = kStages * kStage + kMerge + kSmall;
    static_assert(kStages >= 2, "shared memory of a CTA");
};

// The exponent of a softmax weight at the reference: those that meet v in f16 use its range up to 2^15, since its steps below are coarse.
template <class M>
constexpr int kRaiseOf = std::is_same<M, F16>::value ? 14 : 0;

// A head's log-sum-exp and what the weights need of it: reference, unit, 1 / sum.
template <class M>
__device__ __forceinline__ void finish(const AttendParams& p, int64_t head, float top, float sum, float unit) {
    sum *= 1.0f / (1 << kRaiseOf<M>);
    const float reference = top == -INFINITY ? 0.0f : top;
    if (p.lse) p.lse[head] = sum == 0.0f ? -INFINITY : reference * (unit * 0.6931471805599453f) + logf(sum);
    if (p.add_weight) *reinterpret_cast<float4*>(p.stats + head * 4) = make_float4(reference, unit, sum == 0.0f ? 0.0f : 1.0f / sum, 0.0f);
}

// Adds up the parts of a group in their order.  They come from L2 while the rest of the GPU keeps memory busy, so every
// dependent load costs a microsecond or two: as many whole parts as the buffer holds are copied at once.  A lone CTA waits
// for its own instructions too, so addresses are constants off one pointer and each factor is computed once.
// `factors`: room for two floats per head of each of those parts.
// (A function of its own, so that it takes no registers from the loop over the tiles.)
template <class T, class M, int DP, int NT>
__device__ __noinline__ void join(const AttendParams& p, char* buffer, int room, float2* factors, int first_worker, int parts, int cols,
                                  int64_t head0, float vscale, const float* col_unit) {
    constexpr int kCols = 8 * NT, kPartSize = kCols * (DP + 2), kOutputs = kCols * (DP / 4) / kThreads, kStats = kCols / 2;
    static_assert(kPartSize % 4 == 0 && kCols * (DP / 4) % kThreads == 0, "part layout");
    const int tid = threadIdx.x, per_row = p.pool.head_dim / 4, my_col = tid % kCols;
    const float* const at = reinterpret_cast<const float*>(buffer);
    float4 z[kOutputs];
    float top[kOutputs], sum[kOutputs];
    int col[kOutputs], d[kOutputs];
#pragma unroll
    for (int i = 0; i < kOutputs; i++) {
        const int x = tid + i * kThreads;
        z[i] = make_float4(0, 0, 0, 0), top[i] = -INFINITY, sum[i] = 0;
        col[i] = x / per_row, d[i] = (x - col[i] * per_row) * 4;
    }
    for (int k0 = 0; k0 < parts; k0 += room) {
        const int n = min(room, parts - k0);
        const uint32_t dst = smem_address(buffer) + tid * 16;
        const float* const src = p.parts + 2 * (int64_t)(first_worker + k0) * kPartSize + tid * 4;  // part k: + 2 k kPartSize
#pragma unroll 8
        for (int k = 0; k < n; k++) {
            const float* const from = src + 2 * k * kPartSize + (k0 + k == 0 ? kPartSize : 0);
#pragma unroll
            for (int i = 0; i < kOutputs; i++) copy16(dst + (k * kPartSize + i * 4 * kThreads) * 4, from + i * 4 * kThreads);
        }
        for (int x = tid; x < n * kStats; x += kThreads) {  // references and sums: the end of each part
            const int k = x / kStats, i = kCols * DP + (x % kStats) * 4;
            copy16(smem_address(buffer) + (k * kPartSize + i) * 4, src - tid * 4 + 2 * k * kPartSize + (k0 + k == 0 ? kPartSize : 0) + i);
        }
        commit();
        wait_group<0>();
        __syncthreads();
        float now = -INFINITY;
        for (int k = 0; k < n; k++) now = fmaxf(now, at[k * kPartSize + kCols * DP + my_col * 2]);
        const float base = now == -INFINITY ? 0.0f : now;
        for (int k = tid / kCols; k < n; k += kThreads / kCols) {
            const float2 ml = *reinterpret_cast<const float2*>(at + k * kPartSize + kCols * DP + my_col * 2);
            const float f = ml.x == -INFINITY ? 0.0f : power2((ml.x - base) * col_unit[my_col]);
            factors[k * kCols + my_col] = make_float2(f, f * ml.y);  // (a NaN without a reference stays)
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kOutputs; i++)
            if (col[i] < cols) {
                // this round's own reference, then the rounds' in turn
                float here = -INFINITY;
                for (int k = 0; k < n; k++) here = fmaxf(here, at[k * kPartSize + kCols * DP + col[i] * 2]);
                float4 y = make_float4(0, 0, 0, 0);
                float all = 0;
#pragma unroll 4
                for (int k = 0; k < n; k++) {
                    const float2 fl = factors[k * kCols + col[i]];
                    const float4 v = *reinterpret_cast<const float4*>(at + k * kPartSize + col[i] * DP + d[i]);
                    all += fl.y;
                    y.x += fl.x * v.x, y.y += fl.x * v.y, y.z += fl.x * v.z, y.w += fl.x * v.w;
                }
                const float most = fmaxf(top[i], here), u = col_unit[col[i]];
                const float old = top[i] == -INFINITY ? 0.0f : power2((top[i] - most) * u), young = here == -INFINITY ? 0.0f : power2((here - most) * u);
                z[i].x = z[i].x * old + y.x * young, z[i].y = z[i].y * old + y.y * young;
                z[i].z = z[i].z * old + y.z * young, z[i].w = z[i].w * old + y.w * young;
                sum[i] = sum[i] * old + all * young;
                top[i] = most;
            }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < kOutputs; i++)
        if (col[i] < cols) {
            const float f = sum[i] == 0.0f ? 0.0f : vscale / sum[i];
            *reinterpret_cast<uint2*>(p.out + ((head0 + col[i]) * p.pool.head_dim + d[i]) * 2) =
                sum[i] == 0.0f ? make_uint2(0, 0) : make_uint2(T::pack(z[i].x * f, z[i].y * f), T::pack(z[i].z * f, z[i].w * f));
            if (d[i] == 0) finish<M>(p, head0 + col[i], top[i], sum[i], col_unit[col[i]]);
        }
}

// The same for one head by one warp: the few groups that lie across the stretches of warps that work alone.
template <class T, class M, int DP, int NT>
__device__ __noinline__ void join_alone(const AttendParams& p, int first_worker, int parts, int col, int64_t head0, float vscale, float unit) {
    constexpr int kCols = 8 * NT, kPartSize = kCols * (DP + 2);
    const int lane = threadIdx.x & 31, D = p.pool.head_dim;
    auto part = [&](int k) { return p.parts + (2 * (int64_t)(first_worker + k) + (k == 0 ? 1 : 0)) * kPartSize; };
    float top = -INFINITY;
    for (int k = 0; k < parts; k++) top = fmaxf(top, __ldcg(part(k) + kCols * DP + col * 2));
    const float base = top == -INFINITY ? 0.0f : top;
    for (int d = lane * 4; d < D; d += 128) {
        float4 z = make_float4(0, 0, 0, 0);
        float sum = 0;
        for (int k = 0; k < parts; k++) {
            const float2 ml = __ldcg(reinterpret_cast<const float2*>(part(k) + kCols * DP + col * 2));
            const float4 v = __ldcg(reinterpret_cast<const float4*>(part(k) + col * DP + d));
            const float f = ml.x == -INFINITY ? 0.0f : power2((ml.x - base) * unit);
            sum += f * ml.y;
            z.x += f * v.x, z.y += f * v.y, z.z += f * v.z, z.w += f * v.w;
        }
        const float f = sum == 0.0f ? 0.0f : vscale / sum;
        *reinterpret_cast<uint2*>(p.out + ((head0 + col) * D + d) * 2) =
            sum == 0.0f ? make_uint2(0, 0) : make_uint2(T::pack(z.x * f, z.y * f), T::pack(z.z * f, z.w * f));
        if (d == 0) finish<M>(p, head0 + col, top, sum, unit);
    }
}

template <class T, class C, int DP, int NT, bool FIRST>
__global__ void __launch_bounds__(kThreads, Shape<T, C, DP, NT>::kCtas) fcsim_kv_attend_kernel(const __grid_constant__ AttendParams p) {
    using S = Shape<T, C, DP, NT>;
    using M = typename OperandOf<T, C>::type;
    constexpr bool kNarrow = C::bytes == 1, kRescaled = kNarrow && std::is_same<T, BF16>::value;
    constexpr int kCols = 8 * NT, kSteps = DP / 16, kTokens = S::kTokens, kSub = kTokens / 16;
    constexpr int kParts = std::is_same<M, F16>::value ? 2 : 3;  // 11 bits each, or 8: of the softmax weights
    constexpr float kLog2e = 1.4426950408889634f;
    // a weight is 2^kRaise at the reference of the exponentials and 2^(kRaise + kLag) at most; see where the reference moves
    constexpr bool kHalf = std::is_same<M, F16>::value;
    constexpr float kRaise = kRaiseOf<M>, kLag = kHalf ? 1.9f : 8, kMost = 36;
    constexpr float kStep = 1.0f / 256, kFiner = 274877906944.0f, kFew = 0.125f, kSlight = 1.0f / 32;  // 2^-8, 2^38, 2^-3, 2^-5: see the end of a tile
    constexpr float kLargest = kNarrow ? 448 : 65504;
    constexpr int kPasses = 3;
    // bf16 weights meet v times 2^-24, so that 2^16 values at the type's end add up whatever their weights are.  (Values below
    // 2^-94 lose bits by it.)
    constexpr float kLowered = 16777216.0f;
    extern __shared__ __align__(128) char smem[];
    float* const merge = reinterpret_cast<float*>(smem + S::kStages * S::kStage);
    float* const warp_m = merge + 2 * kCols * S::kOutPitch;  // [4][kCols]
    float* const warp_l = warp_m + 4 * kCols;
    float* const col_unit = warp_l + 4 * kCols;              // [kCols]
    uint32_t* const masks = reinterpret_cast<uint32_t*>(col_unit + 4 * kCols) + (threadIdx.x >> 5) * S::kStages;
    int* const last_flag = reinterpret_cast<int*>(col_unit + 4 * kCols) + 4 * S::kStages;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int D = p.pool.head_dim, group = p.n_heads / p.pool.n_kv;
    const int head_tiles = (group + kCols - 1) / kCols, n_kv = p.pool.n_kv;

    if (p.add_weight) cudaTriggerProgrammaticLaunchCompletion();  // the weights' kernel may line up; it waits for this grid's end
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

    __shared__ Before before;
    const Division work = divide(p, n_kv * head_tiles, kTokens == 32 ? 5 : 4, before);
    const int worker = work.worker(warp), step = 1 << work.bits, offset = work.alone ? 0 : warp * kTokens;  // tokens: of a tile; of this warp's first
    const int depth = work.cut ? S::kStages : S::kFair;  // stages in use
    Place in = {};  // the tile whose loads are issued next
    Place at = {};  // the tile that is computed next
    int cut = 0, cuts = 1;

    // stage s of this warp: + s * kStage; its tokens' rows of K, then of V
    const uint32_t ring = smem_address(smem + warp * 2 * kTokens * S::kPitch);
    const int chunks = D * C::bytes / 16;

    // ---- loads: a row is kLanes lanes' 16 bytes, kRows rows at once; the page numbers (of token lane % kTokens) are
    // fetched one tile ahead
    constexpr int kLanes = S::kRow / 16, kRows = 32 / kLanes;
    constexpr uint32_t kAll = kTokens == 32 ? ~0u : 0xffffu;
    const int chunk = lane % kLanes, lane_row = lane / kLanes;
    const bool copies = chunk < chunks;
    const int64_t v_from_k = p.pool.v - p.pool.k, slot_bytes = p.pool.stride_slot * C::bytes;
    const uint32_t lane_dst = ring + lane_row * S::kPitch + chunk * 16;
    int page = -1, place = 0;
    auto fetch_page = [&]() {  // for tile `in`
        const int u = in.j * step + offset + lane % kTokens, t = token_of<FIRST>(p, in.gap, u), i = page_of(p.pool, t);
        place = t - i * p.pool.page_size;
        page = u < in.seen ? p.table[in.b * p.table_row + i] : -1;
    };
    auto fetch_queries = [&]() {  // of a group that begins soon, into L2
        const int first = in.ht * kCols, lines = (D + 63) / 64, n = min(kCols, group - first) * lines;
        for (int i = lane; i < n; i += 32) {
            const char* x = p.q + ((int64_t)in.b * p.q_row + (int64_t)(in.kv * group + first + i / lines) * p.q_head + i % lines * 64) * 2;
            asm volatile("prefetch.global.L2 [%0];" ::"l"(x));
        }
    };
    auto load_next = [&](int stage) {
        if (in.left > 0) {
            const bool good = (unsigned)page < (unsigned)p.pool.n_pages;
            const uint32_t mask = __ballot_sync(~0u, good) & kAll;
            if (lane == 0) masks[stage] = mask;  // for the computation of this tile
            if (mask != kAll && !good && in.j * step + offset + lane % kTokens < in.seen) flag(p.status, FCSIM_KV_BAD_PAGE);
            const int64_t head = in.kv * p.pool.stride_head;
#pragma unroll
            for (int b = 0; b < kSub; b++) {
                const uint32_t dst = lane_dst + stage * S::kStage + b * 16 * S::kPitch, half = mask >> (16 * b) & 0xffff;
                const int page0 = __shfl_sync(~0u, page, 16 * b), place0 = __shfl_sync(~0u, place, 16 * b);
                const int before = p.first - (in.j * step + offset + 16 * b);  // first tokens among the 16
                const bool split = FIRST && before > 0 && before < 16 && in.gap > 0;
                if (half == 0xffff && place0 + 16 <= p.pool.page_size && !split) {  // 16 tokens of one page: rows at equal distances
                    const char* src = p.pool.k + (page0 * p.pool.stride_page + (place0 + lane_row) * p.pool.stride_slot + head) * C::bytes + chunk * 16;
                    if (copies) {
#pragma unroll
                        for (int i = 0; i < 16 / kRows; i++) {
                            copy16(dst + i * kRows * S::kPitch, src);
                            copy16(dst + (kTokens + i * kRows) * S::kPitch, src + v_from_k);
                            src += kRows * slot_bytes;
                        }
                    }
                } else if (half) {
                    const int64_t mine = good ? (page * p.pool.stride_page + place * p.pool.stride_slot + head) * C::bytes : -1;
#pragma unroll
                    for (int i = 0; i < 16 / kRows; i++) {
                        const int64_t x = __shfl_sync(~0u, mine, 16 * b + i * kRows + lane_row);
                        const char* src = p.pool.k + (x < 0 ? 0 : x + chunk * 16);
                        if (copies) {  // rows that do not exist: zeros, for weights of zero
                            copy16(dst + i * kRows * S::kPitch, src, x < 0 ? 0 : 16);
                            copy16(dst + (kTokens + i * kRows) * S::kPitch, src + v_from_k, x < 0 ? 0 : 16);
                        }
                    }
                } else if (copies) {  // none of the 16
                    const uint4 none = make_uint4(0, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 16 / kRows; i++) {
                        char* const row = smem + warp * 2 * kTokens * S::kPitch + stage * S::kStage + (b * 16 + lane_row + i * kRows) * S::kPitch + chunk * 16;
                        *reinterpret_cast<uint4*>(row) = none;
                        *reinterpret_cast<uint4*>(row + kTokens * S::kPitch) = none;
                    }
                }
            }
            advance(p, work, in, n_kv, head_tiles);
            if (in.left > 0) {
                fetch_page();
                if (in.j == 0 && (warp == 0 || work.alone)) fetch_queries();
            }
        }
        commit();
    };

    uint32_t qf[NT][kSteps][2];  // q^T as the second operand
    // per head (two a lane): the logits' unit times log2 e, the reference of the exponentials (zero until there is a finite
    // logit), the logit from which it has to move, the sum
    float unit[NT][2], m[NT][2], limit[NT][2], l[NT][2], o[kSteps][NT][4];
    int col0 = 0, cols = 0;
    float* logits = nullptr;  // of this lane's first head and first token of a tile
    int64_t logit_row = 0;
    const int64_t first = work.first(worker), end = work.end(worker);
    locate(p, n_kv, head_tiles, work, before, in, cut, cuts);
    if (in.left <= 0) return;  // a CTA whole, or a warp that works alone and meets no barrier
    at = in;
    bool fresh = true;
    int stage = 0;
    auto start_ring = [&]() {
        if (chunks * 16 < S::kRow)  // elements beyond head_dim are never copied to: zeros
            for (int s = 0; s < depth; s++)
                for (int t = lane; t < 2 * kTokens; t += 32)
                    for (int i = chunks * 16; i < S::kRow; i += 16)
                        *reinterpret_cast<uint4*>(smem + (warp * 2 * kTokens + t) * S::kPitch + s * S::kStage + i) = make_uint4(0, 0, 0, 0);
        stage = 0;
        fetch_page();
#pragma unroll 1
        for (int s = 0; s < depth - 1; s++) load_next(s);
    };
    if (in.left > 0) start_ring();
    while (at.left > 0) {
        const int kv = at.kv;
        if (fresh) {
            fresh = false;
            col0 = at.ht * kCols;
            cols = min(kCols, group - col0);
            logits = nullptr;
            const int cta_tiles = (at.seen + S::kTile - 1) >> S::kTileBits;
            logit_row = (int64_t)cta_tiles * S::kTile;
            if (p.add_weight && at.tiles_before + cta_tiles <= p.logit_tiles)
                logits = p.logits + (int64_t)at.tiles_before * S::kTile * p.n_heads + (kv * group + col0 + 2 * (lane & 3)) * logit_row + offset + lane / 4;
            const float scale = kNarrow ? p.scale * p.pool.k_scale[kv] : p.scale;
            const uint32_t flip = scale < 0 ? 0x80008000u : 0u;  // a negative scale turns the order around: turn q instead
            // logits of bf16 reach the end of fp32, where their differences do not fit: below a scale that makes those vanish
            // as -infinity would, q is halved
            const float half = std::is_same<M, BF16>::value && fabsf(scale) < 1e-36f ? 0.5f : 1.0f;
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
                        x ^= flip;
                        if constexpr (std::is_same<M, BF16>::value)
                            if (half < 1.0f) x = BF16::pack(BF16::unpack(x).x * half, BF16::unpack(x).y * half);
                        qf[nt][k][i] = x;
                        if constexpr (kRescaled) {
                            const float2 f = BF16::unpack(x);
                            big = fmaxf(big, fmaxf(fabsf(f.x), fabsf(f.y)));
                        }
                    }
                if constexpr (kRescaled) {
                    big = fmaxf(big, __shfl_xor_sync(~0u, big, 1));
                    big = fmaxf(big, __shfl_xor_sync(~0u, big, 2));
                    if (__any_sync(~0u, big == INFINITY)) {  // infinities stay what they are: the largest of the rest
                        big = 0;
#pragma unroll
                        for (int k = 0; k < kSteps; k++)
#pragma unroll
                            for (int i = 0; i < 2; i++) {
                                const float2 f = BF16::unpack(qf[nt][k][i]);
                                big = fmaxf(big, fmaxf(fabsf(f.x) < INFINITY ? fabsf(f.x) : 0.0f, fabsf(f.y) < INFINITY ? fabsf(f.y) : 0.0f));
                            }
                        big = fmaxf(big, __shfl_xor_sync(~0u, big, 1));
                        big = fmaxf(big, __shfl_xor_sync(~0u, big, 2));
                    }
                    const int e = max((int)(__float_as_uint(big) >> 23), 27);  // biased
                    const float up = __uint_as_float((uint32_t)(127 + 14 + 127 - e) << 23);
                    power = 1.0f / up;  // a power of two: exact
#pragma unroll
                    for (int k = 0; k < kSteps; k++)
#pragma unroll
                        for (int i = 0; i < 2; i++) {
                            const float2 f = BF16::unpack(qf[nt][k][i]);
                            qf[nt][k][i] = F16::pack(f.x * up, f.y * up);
                        }
                }
                // (never zero: a logit of -infinity must stay without weight.  2^-149 times the largest logit is 5e-7.  A scale that
                // is no number stays none.)
                float u = fabsf(scale) / half * power * kLog2e;
                if (u < 1.4e-45f) u = 1.4e-45f;
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    unit[nt][i] = __shfl_sync(~0u, u, (2 * (lane & 3) + i) * 4);
                    m[nt][i] = l[nt][i] = 0;
                    limit[nt][i] = -INFINITY;
                }
#pragma unroll
                for (int k = 0; k < kSteps; k++)
#pragma unroll
                    for (int i = 0; i < 4; i++) o[k][nt][i] = 0;
            }
        }

        if (depth == 2) wait_group<0>();
        else if (depth == 3) wait_group<1>();
        else wait_group<2>();
        __syncwarp();
        load_next(stage == 0 ? depth - 1 : stage - 1);  // into what the last step has read
        const uint32_t mask = masks[stage];

        if (mask) {  // (a warp may have no token of a request's last tile)
            const uint32_t krow = ring + stage * S::kStage, vrow = krow + kTokens * S::kPitch;
            auto score = [&](float (&s)[kSub][NT][4]) {  // s^T = K q^T: 16 tokens by 8 heads at a time
#pragma unroll
                for (int b = 0; b < kSub; b++) {
                    const uint32_t row = krow + (b * 16 + (lane & 7) + ((lane >> 3) & 1) * 8) * S::kPitch + (lane >> 4) * 16;
                    if constexpr (!kNarrow) {
#pragma unroll
                        for (int k0 = 0; k0 < kSteps; k0 += 4) {
                            uint32_t a[4][4];
#pragma unroll
                            for (int k = 0; k < 4; k++) load_matrices(row + (k0 + k) * 32, a[k]);
#pragma unroll
                            for (int k = 0; k < 4; k++)
#pragma unroll
                                for (int nt = 0; nt < NT; nt++) mma<M>(s[b][nt], a[k], qf[nt][k0 + k][0], qf[nt][k0 + k][1]);
                        }
                    } else {
#pragma unroll
                        for (int k0 = 0; k0 < kSteps; k0 += 4) {
                            uint32_t w[2][4];
                            load_matrices(row + k0 * 16, w[0]);
                            load_matrices(row + k0 * 16 + 32, w[1]);
#pragma unroll
                            for (int k = 0; k < 4; k++) {
                                const uint32_t x = w[k / 2][2 * (k & 1)], y = w[k / 2][2 * (k & 1) + 1];
                                const uint32_t a[4] = {E4M3::halves(x), E4M3::halves(y), E4M3::halves(x >> 16), E4M3::halves(y >> 16)};
#pragma unroll
                                for (int nt = 0; nt < NT; nt++) mma<M>(s[b][nt], a, qf[nt][k0 + k][0], qf[nt][k0 + k][1]);
                            }
                        }
                    }
                }
            };
            auto forget = [&](float (&s)[NT][4], int b, int nt) {  // tokens that do not exist
#pragma unroll
                for (int i = 0; i < 4; i++)
                    if (!(mask >> (16 * b + lane / 4 + 8 * (i >> 1)) & 1)) s[nt][i] = -INFINITY;
            };
            uint32_t part[kParts][kSub][NT][2];
            float s[kSub][NT][4] = {};
            score(s);
            uint32_t least = ~0u;  // of the weights above zero, as bits, less one
            // ---- softmax: this lane holds tokens lane / 4 and + 8 of every 16, of heads 2 (lane % 4) and + 1
#pragma unroll
            for (int nt = 0; nt < NT; nt++) {
                if (logits) {
                    float* x = logits + at.j * step + nt * 8 * logit_row;
#pragma unroll
                    for (int i = 0; i < 2; i++)
                        if (nt * 8 + 2 * (lane & 3) + i < cols) {
#pragma unroll
                            for (int b = 0; b < kSub; b++) {
                                x[16 * b] = s[b][nt][i];
                                x[16 * b + 8] = s[b][nt][2 + i];
                            }
                            x += logit_row;
                        }
                }
                if (mask != kAll) {
#pragma unroll
                    for (int b = 0; b < kSub; b++) forget(s[b], b, nt);
                }
                float most[2];
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    most[i] = fmaxf(s[0][nt][i], s[0][nt][2 + i]);
                    if (kSub == 2) most[i] = fmaxf(most[i], fmaxf(s[kSub - 1][nt][i], s[kSub - 1][nt][2 + i]));
                }
                // The reference moves only when a logit is 2^kLag above it: the weights stay far from f16's and fp32's ends, and
                // the maximum over the lanes is taken a few times in a request instead of in every tile.
                if (__any_sync(~0u, most[0] > limit[nt][0] || most[1] > limit[nt][1])) {
                    float shrink[2];
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        float top = most[i];
#pragma unroll
                        for (int d = 4; d < 32; d *= 2) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
                        const bool first_one = limit[nt][i] == -INFINITY;
                        const float now = first_one ? top : fmaxf(top, m[nt][i]);
                        const float base = now == -INFINITY ? 0.0f : now;
                        shrink[i] = first_one ? 0.0f : power2((m[nt][i] - base) * unit[nt][i]);
                        m[nt][i] = base;
                        limit[nt][i] = now + fminf(kLag / unit[nt][i], 1e30f);
                        l[nt][i] *= shrink[i];
                    }
#pragma unroll
                    for (int k = 0; k < kSteps; k++)
#pragma unroll
                        for (int i = 0; i < 4; i++) o[k][nt][i] *= shrink[i & 1];
                }
#pragma unroll
                for (int b = 0; b < kSub; b++) {
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        s[b][nt][i] = power2(fmaf(s[b][nt][i] - m[nt][i & 1], unit[nt][i & 1], kRaise));
                        l[nt][i & 1] += s[b][nt][i];
                        if constexpr (kHalf) least = __viaddmin_u32(__float_as_uint(s[b][nt][i]), ~0u, least);
                        if constexpr (!kHalf) s[b][nt][i] *= 1 / kLowered;
                    }
#pragma unroll
                    for (int k = 0; k < 2; k++) {
                        const float x = s[b][nt][2 * k], y = s[b][nt][2 * k + 1];
                        float restx = x, resty = y;
#pragma unroll
                        for (int i = 0; i < kParts - 1; i++) {
                            const uint32_t h = below<M>(restx, resty);
                            const float2 back = M::unpack(h);
                            part[i][b][nt][k] = transpose8x8(h);
                            restx -= back.x, resty -= back.y;
                        }
                        part[kParts - 1][b][nt][k] = transpose8x8(M::pack(restx, resty));
                    }
                }
            }
            // ---- o^T += V^T p^T: 16 elements of head_dim by 8 heads
            const int which = lane >> 3;
#pragma unroll
            for (int b = 0; b < kSub; b++) {
                if constexpr (!kNarrow) {
                    const uint32_t row = vrow + (b * 16 + (lane & 7) + (which >> 1) * 8) * S::kPitch + (which & 1) * 16;
#pragma unroll
                    for (int k0 = 0; k0 < kSteps; k0 += 4) {
                        uint32_t a[4][4];
#pragma unroll
                        for (int k = 0; k < 4; k++) load_matrices_transposed(row + (k0 + k) * 32, a[k]);
#pragma unroll
                        for (int i = 0; i < kParts; i++)
#pragma unroll
                            for (int k = 0; k < 4; k++)
#pragma unroll
                                for (int nt = 0; nt < NT; nt++) mma<M>(o[k0 + k][nt], a[k], part[i][b][nt][0], part[i][b][nt][1]);
                    }
                } else {
                    const uint32_t row = vrow + (b * 16 + (lane & 7) + (which & 1) * 8) * S::kPitch + (which >> 1) * 16;
#pragma unroll
                    for (int k0 = 0; k0 < kSteps; k0 += 4) {
                        uint32_t a[4][4];
                        load_narrow_transposed(row + k0 * 16, a);
#pragma unroll
                        for (int k = 0; k < 4; k++)
#pragma unroll
                            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                                for (int i = 0; i < kParts; i++) mma<M>(o[k0 + k][nt], a[k], part[i][b][nt][0], part[i][b][nt][1]);
                    }
                }
            }
            // Weights below kStep are few of f16's steps, too few where those above meet a v of nothing.  So where there are any and an
            // element of the sums is still slight (below kSlight of the tile's largest v, of weights of 2^14 at the reference), what their
            // rounding has lost follows in up to three passes, kFiner times as large in each and added up apart: 22 bits of weights down to
            // 2^-100.  If a head has no others here, its reference moves down for the tiles to come (by 2^22 at most: it has to come back
            // up in one factor).  The parts may be zero or negative, so a tile with a v that is infinite or NaN goes without.  It stands
            // behind the products so that nothing comes between these and the weights.  (Attention alone: 64 requests over e4m3, without
            // any of it 81.3 us, with it 82.8, with logits four times as wide 91, and without the test of the sums 124; 100 requests in f16
            // 41.1, 41.8, and 46.)
            if constexpr (kHalf) {
                bool lost = __any_sync(~0u, least < __float_as_uint(kStep) - 1);
                if (lost) {
                    float slight = INFINITY;
#pragma unroll
                    for (int k = 0; k < kSteps; k++)
#pragma unroll
                        for (int i = 0; i < 4; i++)
                            if (k * 16 + (kNarrow ? 0 : 8 * (i >> 1)) < D) {  // (head_dim is a multiple of 16, or of 8)
#pragma unroll
                                for (int nt = 0; nt < NT; nt++) slight = fminf(slight, fabsf(o[k][nt][i]));
                            }
                    lost = __any_sync(~0u, slight < kSlight * kLargest);
                    if (lost) {  // beside the tile's own largest v
                        uint32_t large = 0;
                        const char* const rows = smem + warp * 2 * kTokens * S::kPitch + stage * S::kStage + kTokens * S::kPitch;
#pragma unroll 4
                        for (int t = lane_row; t < kTokens; t += kRows) {
                            const uint4 x = *reinterpret_cast<const uint4*>(rows + t * S::kPitch + chunk * 16);
                            const uint32_t word[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                            for (int i = 0; i < 4; i++) {
                                if constexpr (kNarrow) large = __vmaxu2(large, __vmaxu2(word[i] << 8 & 0x7f007f00u, word[i] & 0x7f007f00u));
                                else large = __vmaxu2(large, word[i] & 0x7fff7fffu);
                            }
                        }
                        large = __reduce_max_sync(~0u, max(large & 0xffff, large >> 16));
                        float most_v;
                        if constexpr (kNarrow) most_v = M::unpack(E4M3::halves(large >> 8)).x;
                        else most_v = M::unpack(large).x;
                        lost = __any_sync(~0u, slight <= kSlight * most_v) && most_v < INFINITY;  // (NaN: not)
                    }
                }
                if (lost) {
                    float w[kSub][NT][4] = {};
                    score(w);
                    float top[NT][2];
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) {
                        top[nt][0] = top[nt][1] = 0;
#pragma unroll
                        for (int b = 0; b < kSub; b++) {
                            if (mask != kAll) forget(w[b], b, nt);
#pragma unroll
                            for (int i = 0; i < 4; i++) {
                                float& x = w[b][nt][i];
                                x = power2(fmaf(x - m[nt][i & 1], unit[nt][i & 1], kRaise));
                                top[nt][i & 1] = fmaxf(top[nt][i & 1], x);
                                x = x < kStep ? x : 0.0f;
                            }
                        }
                    }
#pragma unroll
                    for (int b = 0; b < kSub; b++)  // what the two parts have left of them
#pragma unroll
                        for (int nt = 0; nt < NT; nt++)
#pragma unroll
                            for (int k = 0; k < 2; k++) {
                                float &x = w[b][nt][2 * k], &y = w[b][nt][2 * k + 1];
                                float2 f = M::unpack(below<M>(x, y));
                                x -= f.x, y -= f.y;
                                f = M::unpack(M::pack(x, y));
                                x -= f.x, y -= f.y;
                            }
                    float lower = 1;
#pragma unroll 1
                    for (int pass = 0; pass < kPasses; pass++) {
                        bool more = false;
#pragma unroll
                        for (int b = 0; b < kSub; b++)
#pragma unroll
                            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                                for (int k = 0; k < 2; k++) {
                                    float &x = w[b][nt][2 * k], &y = w[b][nt][2 * k + 1];
                                    x *= kFiner, y *= kFiner;
                                    const bool few_x = fabsf(x) < kFew, few_y = fabsf(y) < kFew;  // (and few bits again)
                                    more |= (few_x && x != 0.0f) || (few_y && y != 0.0f);
                                    const uint32_t h = M::pack(x, y);
                                    float2 f = M::unpack(h);
                                    x -= f.x, y -= f.y;
                                    const uint32_t g = M::pack(x, y);
                                    f = M::unpack(g);
                                    x = few_x ? x - f.x : 0.0f, y = few_y ? y - f.y : 0.0f;
                                    part[0][b][nt][k] = transpose8x8(h);
                                    part[1][b][nt][k] = transpose8x8(g);
                                }
                        lower /= kFiner;
#pragma unroll
                        for (int k0 = 0; k0 < kSteps; k0 += 4) {
                            float apart[4][NT][4] = {};
#pragma unroll
                            for (int b = 0; b < kSub; b++) {
                                uint32_t a[4][4];
                                if constexpr (kNarrow)
                                    load_narrow_transposed(vrow + (b * 16 + (lane & 7) + (which & 1) * 8) * S::kPitch + (which >> 1) * 16 + k0 * 16, a);
                                else {
#pragma unroll
                                    for (int k = 0; k < 4; k++)
                                        load_matrices_transposed(vrow + (b * 16 + (lane & 7) + (which >> 1) * 8) * S::kPitch + (which & 1) * 16 + (k0 + k) * 32, a[k]);
                                }
#pragma unroll
                                for (int k = 0; k < 4; k++)
#pragma unroll
                                    for (int nt = 0; nt < NT; nt++)
#pragma unroll
                                        for (int i = 0; i < kParts; i++) mma<M>(apart[k][nt], a[k], part[i][b][nt][0], part[i][b][nt][1]);
                            }
#pragma unroll
                            for (int k = 0; k < 4; k++)
#pragma unroll
                                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                                    for (int i = 0; i < 4; i++) o[k0 + k][nt][i] += apart[k][nt][i] * lower;
                        }
                        if (!__any_sync(~0u, more)) break;
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) {
                        float grow[2];
#pragma unroll
                        for (int i = 0; i < 2; i++) {
                            float highest = top[nt][i], most_l = l[nt][i];
#pragma unroll
                            for (int d = 4; d < 32; d *= 2) {
                                highest = fmaxf(highest, __shfl_xor_sync(~0u, highest, d));
                                most_l = fmaxf(most_l, __shfl_xor_sync(~0u, most_l, d));
                            }
                            grow[i] = 1;
                            if (highest > 0.0f && highest < kStep) {
                                const float room = kMost + 126 - (float)(__float_as_uint(most_l) >> 23);  // so that l stays below 2^kMost
                                const float now = m[nt][i] - fmaxf(fminf(kRaise - log2f(highest), room), 0.0f) / unit[nt][i];
                                grow[i] = power2((m[nt][i] - now) * unit[nt][i]);
                                m[nt][i] = now;
                                limit[nt][i] = now + fminf(kLag / unit[nt][i], 1e30f);
                                l[nt][i] *= grow[i];
                            }
                        }
#pragma unroll
                        for (int k = 0; k < kSteps; k++)
#pragma unroll
                            for (int i = 0; i < 4; i++) o[k][nt][i] *= grow[i & 1];
                    }
                }
            }
        }
        if (++stage == depth) stage = 0;

        const bool whole = work.whole(at.tiles);
        if (at.j < at.tiles - 1 && (whole || at.left > 1)) {
            at.j++;
            at.left -= !whole;
            continue;
        }
        // ---------------------------------------------------------------- end of this worker's part of a group
        // the units of the group's tiles, and the workers that have them
        const int64_t group_first = end - at.left - at.j, group_end = group_first + at.tiles;
        int first_worker = worker, last_worker = worker;
        if (work.cut) {
            first_worker -= cut;
            last_worker = first_worker + cuts - 1;
        } else if (!whole) {
            if (group_first < first) first_worker = (int)(group_first / work.share);
            if (group_end > end) last_worker = (int)((group_end - 1) / work.share);
        }
        const int parts = last_worker - first_worker + 1;
        const int64_t head0 = (int64_t)at.b * p.n_heads + kv * group + col0;
        const float vscale = kNarrow ? p.pool.v_scale[kv] : kHalf ? 1.0f : kLowered;
        constexpr int kPartSize = kCols * (DP + 2);
        // a worker leaves at most two parts: of a group that began before it (0), and of one that goes on behind it (1)
        float* const my_part = p.parts + (2 * (int64_t)worker + (first_worker == worker ? 1 : 0)) * kPartSize;
        int* const counter = p.counters + first_worker;
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int i = 0; i < 2; i++) {
                l[nt][i] += __shfl_xor_sync(~0u, l[nt][i], 4);
                l[nt][i] += __shfl_xor_sync(~0u, l[nt][i], 8);
                l[nt][i] += __shfl_xor_sync(~0u, l[nt][i], 16);
            }
        if (work.alone) {
            if (parts == 1) {
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
                    float f[2];
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        const int col = nt * 8 + 2 * (lane & 3) + i;
                        f[i] = vscale / l[nt][i];
                        if (l[nt][i] == 0.0f) {  // zeros, also where a v is infinite
                            f[i] = 0;
#pragma unroll
                            for (int k = 0; k < kSteps; k++) o[k][nt][i] = o[k][nt][2 + i] = 0;
                        }
                        if (lane < 4 && col < cols) finish<M>(p, head0 + col, limit[nt][i] == -INFINITY ? -INFINITY : m[nt][i], l[nt][i], unit[nt][i]);
                    }
                    // two heads a lane become two or four neighbouring elements of one head: lane / 4
                    const bool real = nt * 8 + lane / 4 < cols;
                    char* const row = p.out + (head0 + nt * 8 + lane / 4) * D * 2;
#pragma unroll
                    for (int k = 0; k < kSteps; k++) {
                        const uint32_t x = transpose8x8(T::pack(o[k][nt][0] * f[0], o[k][nt][1] * f[1]));
                        const uint32_t y = transpose8x8(T::pack(o[k][nt][2] * f[0], o[k][nt][3] * f[1]));
                        if constexpr (kNarrow) {
                            const int d = k * 16 + 4 * (lane & 3);
                            if (real && d < D) *reinterpret_cast<uint2*>(row + d * 2) = make_uint2(__byte_perm(x, y, 0x5410), __byte_perm(x, y, 0x7632));
                        } else {
                            const int d = k * 16 + 2 * (lane & 3);
                            if (real && d < D) *reinterpret_cast<uint32_t*>(row + d * 2) = x;
                            if (real && d + 8 < D) *reinterpret_cast<uint32_t*>(row + (d + 8) * 2) = y;
                        }
                    }
                }
            } else {
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const int col = nt * 8 + 2 * (lane & 3) + (i & 1);
                        if (i < 2 && lane < 4)
                            *reinterpret_cast<float2*>(my_part + kCols * DP + col * 2) =
                                make_float2(limit[nt][i] == -INFINITY ? -INFINITY : m[nt][i], l[nt][i]);
#pragma unroll
                        for (int k = 0; k < kSteps; k++)
                            my_part[col * DP + (kNarrow ? k * 16 + 2 * (lane / 4) + (i >> 1) : k * 16 + lane / 4 + 8 * (i >> 1))] = o[k][nt][i];
                    }
                __threadfence();
                __syncwarp();
                int before = 0;
                if (lane == 0) before = atomicAdd(counter, 1);
                if (__shfl_sync(~0u, before, 0) == parts - 1) {
                    if (lane == 0) *counter = 0;
                    __threadfence();
#pragma unroll 1
                    for (int col = 0; col < cols; col++) {
                        float u = 0;
#pragma unroll
                        for (int nt = 0; nt < NT; nt++)
#pragma unroll
                            for (int i = 0; i < 2; i++) {
                                const float x = __shfl_sync(~0u, unit[nt][i], (col & 7) / 2);
                                if (col / 8 == nt && (col & 1) == i) u = x;
                            }
                        join_alone<T, M, DP, NT>(p, first_worker, parts, col, head0, vscale, u);
                    }
                }
            }
            advance(p, work, at, n_kv, head_tiles);
            fresh = true;
            continue;
        }
        bool restart = false;
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int i = 0; i < 2; i++)
                if (lane < 4) {
                    const int col = nt * 8 + 2 * lane + i;
                    warp_m[warp * kCols + col] = limit[nt][i] == -INFINITY ? -INFINITY : m[nt][i];
                    warp_l[warp * kCols + col] = l[nt][i];
                    if (warp == 0) col_unit[col] = unit[nt][i];
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
                const float f = limit[nt][i] == -INFINITY ? 0.0f : power2((m[nt][i] - base) * unit[nt][i]);
#pragma unroll
                for (int k = 0; k < kSteps; k++) {
                    o[k][nt][i] *= f;
                    o[k][nt][2 + i] *= f;
                }
            }
        auto element = [&](int k, int nt, int i) {  // where o[k][nt][i] lies in a merge buffer
            const int d = kNarrow ? k * 16 + 2 * (lane / 4) + (i >> 1) : k * 16 + lane / 4 + 8 * (i >> 1);
            return (warp & 1) * kCols * S::kOutPitch + (nt * 8 + 2 * (lane & 3) + (i & 1)) * S::kOutPitch + d;
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

        const int per_row = D / 4;
        for (int i = tid; i < cols * per_row; i += kThreads) {
            const int col = i / per_row, d = (i - col * per_row) * 4;
            const float4 x = *reinterpret_cast<const float4*>(merge + col * S::kOutPitch + d);
            const float4 y = *reinterpret_cast<const float4*>(merge + (kCols + col) * S::kOutPitch + d);
            const float4 z = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
            float sum = 0, top = -INFINITY;
#pragma unroll
            for (int w = 0; w < 4; w++) top = fmaxf(top, warp_m[w * kCols + col]);
            const float base = top == -INFINITY ? 0.0f : top, u = col_unit[col];
#pragma unroll
            for (int w = 0; w < 4; w++) {
                const float x = warp_m[w * kCols + col];  // -infinity: the sum is 0, or NaN and stays so
                sum += warp_l[w * kCols + col] * (x == -INFINITY ? 0.0f : power2((x - base) * u));
            }
            if (parts == 1) {
                const float f = sum == 0.0f ? 0.0f : vscale / sum;
                *reinterpret_cast<uint2*>(p.out + ((head0 + col) * D + d) * 2) =
                    sum == 0.0f ? make_uint2(0, 0) : make_uint2(T::pack(z.x * f, z.y * f), T::pack(z.z * f, z.w * f));
                if (d == 0) finish<M>(p, head0 + col, top, sum, u);
            } else {
                *reinterpret_cast<float4*>(my_part + col * DP + d) = z;
                if (d == 0) *reinterpret_cast<float2*>(my_part + kCols * DP + col * 2) = make_float2(top, sum);
            }
        }
        if (parts > 1) {
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                const bool last = atomicAdd(counter, 1) == parts - 1;
                *last_flag = last;
                if (last) *counter = 0;
            }
            __syncthreads();
            if (*last_flag) {
                __threadfence();
                wait_group<0>();  // the ring is the buffer: what it holds of the next group is loaded again
                __syncthreads();
                join<T, M, DP, NT>(p, smem, S::kJoined, reinterpret_cast<float2*>(merge), first_worker, parts, cols, head0, vscale, col_unit);
                restart = true;
            }
        }
        __syncthreads();  // the merge buffers and the columns' statistics are free again
        advance(p, work, at, n_kv, head_tiles);
        fresh = true;
        if (restart && at.left > 0) {
            in = at;
            start_ring();
        }
    }
}

template <class T, class C, int DP, int NT, bool FIRST>
int launch(const AttendParams& p, int grid, cudaStream_t stream) {
    using S = Shape<T, C, DP, NT>;
    fcsim_kv_attend_kernel<T, C, DP, NT, FIRST><<<grid, kThreads, S::kBytes, stream>>>(p);
    return (int)cudaGetLastError();
}
template <class T, class C, int DP, int NT, bool FIRST>
int ctas_per_sm(int device, int* out) {
    using S = Shape<T, C, DP, NT>;
    static std::atomic<int> known[kMaxDevices];
    int n = device < kMaxDevices ? known[device].load(std::memory_order_relaxed) : 0;
    if (n == 0) {
        auto* kernel = fcsim_kv_attend_kernel<T, C, DP, NT, FIRST>;
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kBytes);
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, kThreads, S::kBytes);
        if (e != cudaSuccess) return (int)e;
        if (device < kMaxDevices) known[device].store(n, std::memory_order_relaxed);
    }
    *out = n;
    return 0;
}
template <class T, class C, int DP, bool FIRST>
AttendVariant of_group(int group) {
    // more than 8 heads: two column tiles share every load; beyond 16, and for the widest rows (whose registers do not
    // suffice: 32 requests, 16 heads on each kv head of 256, 172 us, rows read twice 136), the rows are read again
    if constexpr (DP <= 128)
        if (group > 8) return {launch<T, C, DP, 2, FIRST>, ctas_per_sm<T, C, DP, 2, FIRST>, 16, DP, Shape<T, C, DP, 2>::kTileBits};
    return {launch<T, C, DP, 1, FIRST>, ctas_per_sm<T, C, DP, 1, FIRST>, 8, DP, Shape<T, C, DP, 1>::kTileBits};
}
template <class T, class C, bool FIRST>
AttendVariant of_width(int head_dim, int group) {
    return head_dim <= 64 ? of_group<T, C, 64, FIRST>(group) : head_dim <= 128 ? of_group<T, C, 128, FIRST>(group) : of_group<T, C, 256, FIRST>(group);
}
template <class T, class C>
AttendVariant of(int head_dim, int group, bool first) {
    return first ? of_width<T, C, true>(head_dim, group) : of_width<T, C, false>(head_dim, group);
}

}  // namespace

#if FCSIM_KV_TYPES == 0
AttendVariant attend_variant_f16(int head_dim, int group, bool first) { return of<F16, F16>(head_dim, group, first); }
#elif FCSIM_KV_TYPES == 1
AttendVariant attend_variant_bf16(int head_dim, int group, bool first) { return of<BF16, BF16>(head_dim, group, first); }
#elif FCSIM_KV_TYPES == 2
AttendVariant attend_variant_f16_e4m3(int head_dim, int group, bool first) { return of<F16, E4M3>(head_dim, group, first); }
#else
AttendVariant attend_variant_bf16_e4m3(int head_dim, int group, bool first) { return of<BF16, E4M3>(head_dim, group, first); }
#endif

#if FCSIM_KV_TYPES == 0
// weight[token] += sum over a group's heads of the softmax weights, from the logits that the first kernel left: the final
// reference and sum of a head are known only when all of its parts are joined.  The same division of the work, without
// overhead: a CTA takes eight tiles (of 64 tokens) of (request, kv head) at a time, four tokens a thread, two
// heads' logits at once and their sum in order.  Bound by the latency of a few dependent loads, so what matters is that
// one round of the grid is all of it, and what does not need the logits is loaded before the first kernel has ended.
template <bool FIRST>
__global__ void __launch_bounds__(kThreads, kWeightCtas) fcsim_kv_weight_kernel(const AttendParams p) {
    constexpr int kAtOnce = 2;
    const int threads = 1 << (p.tile_bits - 2), tiles = kThreads / threads;  // of a tile; at a time
    const int n_kv = p.pool.n_kv, group = p.n_heads / n_kv, mine = threadIdx.x / threads, size = p.pool.page_size;
    __shared__ Before before;
    const Division work = divide(p, n_kv, 0, before);  // (of the lengths alone, which the first kernel does not write)
    Place at = {};
    int cut, cuts;
    locate(p, n_kv, 1, work, before, at, cut, cuts);
    for (int i = 0; i < mine && at.left > 0; i++) advance(p, work, at, n_kv, 1);

    int in;
    bool aligned, room;
    float* weight[4];  // of each token, or none; one page and 16 aligned bytes where the size of a page allows
    float old[4];
    auto load_weights = [&]() {
        in = (at.j << p.tile_bits) + threadIdx.x % threads * 4;
        const int t0 = token_of<FIRST>(p, at.gap, in);
        aligned = size % 4 == 0 && t0 % 4 == 0 && token_of<FIRST>(p, at.gap, in + 3) == t0 + 3;
        room = at.tiles_before + at.tiles <= p.logit_tiles;
        if (!room) flag(p.status, FCSIM_KV_BAD_PAGE);  // more tokens than the pool has: pages are shared
        const int32_t* const table = p.table + at.b * p.table_row;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            weight[i] = nullptr;
            if (room && in + i < at.seen && (i == 0 || !aligned)) {
                const int t = token_of<FIRST>(p, at.gap, in + i), index = page_of(p.pool, t), page = table[index];
                if ((unsigned)page < (unsigned)p.pool.n_pages) weight[i] = p.pool.weight + ((int64_t)page * n_kv + at.kv) * size + t - index * size;
            }
        }
        if (aligned) {
            if (weight[0]) *reinterpret_cast<float4*>(old) = *reinterpret_cast<const float4*>(weight[0]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (weight[i]) old[i] = *weight[i];
        }
    };
    if (at.left > 0) load_weights();
    cudaGridDependencySynchronize();  // (by every CTA: the grid must not end before the first one)
    while (at.left > 0) {
        if (room && in < at.seen) {
            float sum[4] = {0, 0, 0, 0};
            const int64_t step = (int64_t)at.tiles << p.tile_bits;
            const float* logit = p.logits + ((int64_t)at.tiles_before * p.n_heads << p.tile_bits) + at.kv * group * step + in;
            const float4* stats = reinterpret_cast<const float4*>(p.stats) + (int64_t)at.b * p.n_heads + at.kv * group;
            for (int h = 0; h < group; h += kAtOnce, logit += kAtOnce * step, stats += kAtOnce) {
                float4 s[kAtOnce], x[kAtOnce];
#pragma unroll
                for (int i = 0; i < kAtOnce; i++)
                    if (h + i < group) s[i] = *reinterpret_cast<const float4*>(logit + i * step), x[i] = stats[i];
#pragma unroll
                for (int i = 0; i < kAtOnce; i++)
                    if (h + i < group) {
                        sum[0] += power2((s[i].x - x[i].x) * x[i].y) * x[i].z;
                        sum[1] += power2((s[i].y - x[i].x) * x[i].y) * x[i].z;
                        sum[2] += power2((s[i].z - x[i].x) * x[i].y) * x[i].z;
                        sum[3] += power2((s[i].w - x[i].x) * x[i].y) * x[i].z;
                    }
            }
            if (aligned && in + 3 < at.seen) {
                if (weight[0]) *reinterpret_cast<float4*>(weight[0]) = make_float4(old[0] + sum[0], old[1] + sum[1], old[2] + sum[2], old[3] + sum[3]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    float* const w = aligned ? (weight[0] && in + i < at.seen ? weight[0] + i : nullptr) : weight[i];
                    if (w) *w = old[i] + sum[i];
                }
            }
        }
        for (int i = 0; i < tiles && at.left > 0; i++) advance(p, work, at, n_kv, 1);
        if (at.left > 0) load_weights();
    }
}
int launch_weights(const AttendParams& p, int grid, cudaStream_t stream) {
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(grid);
    config.blockDim = dim3(kThreads);
    config.stream = stream;
    cudaLaunchAttribute early;  // launched while the first kernel ends
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    config.attrs = &early;
    config.numAttrs = 1;
    return (int)cudaLaunchKernelEx(&config, p.first ? fcsim_kv_weight_kernel<true> : fcsim_kv_weight_kernel<false>, p);
}
#endif

}  // namespace fcsim_kv_dev
