// Attention of several query tokens per request over a paged cache (compiled once per pair of types: FCSIM_KV_TYPES 0..3).
//
//   o_i = sum_t p_t v_t / sum_t p_t,   p_t = exp(c q_i . k_t - m),   over the tokens t that row i sees:
//   t <= position of i, and with a window also t > position - window or t < first
//
// * The query heads of a kv head and a run of tokens are the rows of a block: one or two tiles of 128 (token, head) pairs, so that
//   few new tokens fill a tile as well as many do, and what is loaded of K and V serves all of them.
// * Both products run on tcgen05: S = Q K^T from shared memory into tensor memory, P back into the columns S had, O += P V with
//   P read from tensor memory.  One thread issues them; two groups of four warps, a row each thread, do the softmax of one tile while the
//   other tile's products run; three warps load.
// * Pages may have any size and strides, so rows come by cp.async, 16 bytes a lane, into the 128-byte swizzled layout that the products
//   read (8-bit rows through registers, as 16 bits, exactly).
// * The work is counted in tiles of keys, laid end to end over all requests, heads and blocks, and every CTA takes an equal stretch (or, where
//   there are few blocks, one piece of one block).  Parts of a block that lies across stretches are joined by the last to come, in
//   their order: the same call gives the same bits.
// * s, m, the sums and o are 32-bit.  p meets v in two 16-bit parts that add up to it to 2^-16 or better.
#include <math.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "fcsim_kv_prefill.cuh"

namespace fcsim_kv_dev {
namespace {

constexpr int kMaxDevices = 64;

// ---------------------------------------------------------------------------------------------- instructions
__device__ __forceinline__ uint32_t smem_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// 16 bytes global -> shared; with `bytes` = 0 nothing is read and zeros are written
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_copies() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void store16(uint32_t a, const uint4& x) {
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
}
__device__ __forceinline__ uint4 load16(uint32_t a) {
    uint4 x;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(a) : "memory");
    return x;
}
// what this thread has written to shared memory, before the tensor core reads it
__device__ __forceinline__ void fence_for_products() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void bar_init(uint32_t bar, int count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
        : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
__device__ __forceinline__ void fence_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_stores() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// all products issued so far by this thread, then one arrival
__device__ __forceinline__ void commit_products(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void product(uint32_t d, uint64_t a, uint64_t b, uint32_t how, uint32_t add) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(how), "r"(add) : "memory");
}
__device__ __forceinline__ void product_from_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t how, uint32_t add) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 ::"r"(d), "r"(a), "l"(b), "r"(how), "r"(add) : "memory");
}
// 32 columns of a warp's 32 lanes of tensor memory
__device__ __forceinline__ void tmem_load(uint32_t at, float (&x)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]), "=f"(x[8]), "=f"(x[9]), "=f"(x[10]),
          "=f"(x[11]), "=f"(x[12]), "=f"(x[13]), "=f"(x[14]), "=f"(x[15]), "=f"(x[16]), "=f"(x[17]), "=f"(x[18]), "=f"(x[19]), "=f"(x[20]),
          "=f"(x[21]), "=f"(x[22]), "=f"(x[23]), "=f"(x[24]), "=f"(x[25]), "=f"(x[26]), "=f"(x[27]), "=f"(x[28]), "=f"(x[29]), "=f"(x[30]),
          "=f"(x[31])
        : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_store(uint32_t at, const uint32_t (&x)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
        ::"r"(at), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]), "r"(x[8]), "r"(x[9]), "r"(x[10]),
          "r"(x[11]), "r"(x[12]), "r"(x[13]), "r"(x[14]), "r"(x[15]), "r"(x[16]), "r"(x[17]), "r"(x[18]), "r"(x[19]), "r"(x[20]), "r"(x[21]),
          "r"(x[22]), "r"(x[23]), "r"(x[24]), "r"(x[25]), "r"(x[26]), "r"(x[27]), "r"(x[28]), "r"(x[29]), "r"(x[30]), "r"(x[31])
        : "memory");
}
// 2^x; results below 2^-126 are 0
__device__ __forceinline__ float power2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Descriptor of an operand in shared memory: rows of 128 bytes (64 elements), swizzled by 128 bytes.  `group`: from 8 rows to the next 8;
// `chunk`: from 64 elements to the next 64 (read only where these are the outer dimension).
__device__ __forceinline__ uint64_t operand(uint32_t address, uint32_t chunk, uint32_t group) {
    return (uint64_t)((address >> 4) & 0x3fff) | (uint64_t)(chunk >> 4) << 16 | (uint64_t)(group >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// What a product is: 32-bit sums, f16 (0) or bf16 (1) operands, B with its rows as the inner dimension or not, sizes.
__device__ __forceinline__ uint32_t instruction(uint32_t type, bool b_across, uint32_t m, uint32_t n) {
    return 1u << 4 | type << 7 | type << 10 | (uint32_t)b_across << 16 | (n >> 3) << 17 | (m >> 4) << 24;
}

// ---------------------------------------------------------------------------------------------- shape
template <class T, class C, int DP>
struct Shape {
    static constexpr int kTiles = DP <= 128 ? 2 : 1;    // of 128 rows: two where their outputs fit tensor memory
    static constexpr int kRows = 128 * kTiles;
    static constexpr int kKeys = DP <= 128 ? 128 : 64;  // of a tile
    static constexpr int kQuery = kRows * DP * 2;       // bytes
    static constexpr int kStage = kKeys * DP * 2;       // of K or V
    static constexpr int kRoom = (227 * 1024 - 2048 - 1024 - kQuery) / kStage;
    static constexpr int kStages = kRoom < 8 ? kRoom : 8;
    static constexpr int kBytes = kQuery + kStages * kStage + 1024;
    static constexpr int kSoftmaxWarps = 4 * kTiles, kLoadWarps = 3;
    static constexpr int kWarps = kSoftmaxWarps + kLoadWarps + 1, kThreads = 32 * kWarps;
    // tensor memory: two areas of kKeys columns for S and P, then O of each tile
    static constexpr int kScore = 0, kOutput = 2 * kKeys, kColumns = 512;
    static_assert(kOutput + kTiles * DP <= kColumns && kStages >= 4, "room");
};

// ---------------------------------------------------------------------------------------------- the walk over the work
// Cost of a block's start and end beside one tile of keys.
constexpr int kOverhead = 2;
constexpr int kPieceLeast = 2;  // tiles of a piece at least, where blocks are cut

// A block of rows: tokens [at, at + tokens) of the new ones of a request, heads of one head tile.
struct Block {
    int r, head, b;              // request, kv head * head tiles + head tile, block
    int row0, rows, position0;   // the request's rows in q; position of the first of them
    int tokens, gap, seen, tiles;
};

__device__ __forceinline__ int request_rows(const PrefillParams& p, int r, int& row0) {
    row0 = min(max(p.starts[r], 0), p.n_rows);
    return max(min(p.starts[r + 1], p.n_rows) - row0, 0);
}
__device__ __forceinline__ int request_length(const PrefillParams& p, int r) { return min(max(p.lengths[r], 0), p.max_length); }

// What a block of tokens sees: all tokens up to its last one, or the first ones and, without the gap behind these, those from the start of
// its first token's window.  Counted without the gap: seen key u is token u, or behind the first ones u + gap.
__device__ __forceinline__ int seen_by(const PrefillParams& p, int position0, int tokens, int& gap) {
    const int64_t low = (int64_t)position0 - p.window + 1;  // (a request of more rows than tokens has positions below 0)
    gap = p.window > 0 && low > p.first ? (int)(low - p.first) : 0;
    return max(position0 + tokens - gap, 0);
}
template <int KEYS>
__device__ __forceinline__ int tiles_of(const PrefillParams& p, int position0, int rows, int b) {
    int gap;
    const int at = b * p.tokens_a_block;
    return max(1, (seen_by(p, position0 + at, min(p.tokens_a_block, rows - at), gap) + KEYS - 1) / KEYS);
}
__device__ __forceinline__ int blocks_of(const PrefillParams& p, int rows) { return (int)(((int64_t)rows + p.tokens_a_block - 1) / p.tokens_a_block); }

template <int KEYS>
__device__ __forceinline__ void enter_block(const PrefillParams& p, Block& x) {
    const int at = x.b * p.tokens_a_block;
    x.tokens = min(p.tokens_a_block, x.rows - at);
    x.seen = seen_by(p, x.position0 + at, x.tokens, x.gap);
    x.tiles = max(1, (x.seen + KEYS - 1) / KEYS);
}
template <int KEYS>
__device__ __forceinline__ void enter_request(const PrefillParams& p, Block& x) {
    x.rows = request_rows(p, x.r, x.row0);
    x.position0 = request_length(p, x.r) - x.rows;
}

// The division of the units among the CTAs, which depends on the lengths and the grid alone.  A unit is a tile of keys (and kOverhead of them
// stand before a block's first tile), or, with `cut`, a piece of a block of at most `cut` tiles.
struct Division {
    int64_t total, share;
    int cut;
    __device__ __forceinline__ int units(int tiles) const { return cut ? (tiles + cut - 1) / cut : tiles + kOverhead; }
};

// Where a CTA's stretch begins.
struct Start {
    Block block;
    int j;               // first tile
    int64_t left;        // units from it to the end of the stretch, or the piece's tiles; none: no work
    int64_t first_unit;  // of the block's first tile (without `cut`)
    int piece, pieces;   // with `cut`
};

__device__ __forceinline__ int64_t warp_sum(int64_t x) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    return x;
}

// Units (or tiles, with `tiles_only`) of one of the heads of request base + lane, and its blocks.  The blocks of long requests are added up by the warp.
template <int KEYS>
__device__ __forceinline__ int64_t units_of_requests(const PrefillParams& p, int r, bool mine, const Division* d, int& blocks) {
    constexpr int kAlone = 4;
    const int lane = threadIdx.x & 31;
    int rows = 0, position0 = 0;
    if (mine) {
        int row0;
        rows = request_rows(p, r, row0);
        position0 = request_length(p, r) - rows;
    }
    blocks = blocks_of(p, rows);
    int64_t own = 0;
    auto cost = [&](int position, int n, int b) {
        const int t = tiles_of<KEYS>(p, position, n, b);
        return d ? d->units(t) : t;
    };
    if (blocks <= kAlone)
        for (int b = 0; b < blocks; b++) own += cost(position0, rows, b);
    uint32_t together = __ballot_sync(~0u, blocks > kAlone);
    while (together) {
        const int src = __ffs(together) - 1;
        together &= together - 1;
        const int n = __shfl_sync(~0u, rows, src), position = __shfl_sync(~0u, position0, src), all = __shfl_sync(~0u, blocks, src);
        int64_t sum = 0;
        for (int b = lane; b < all; b += 32) sum += cost(position, n, b);
        sum = warp_sum(sum);
        if (lane == src) own = sum;
    }
    return own;
}

template <int KEYS, int WARPS>
__device__ __forceinline__ Division plan(const PrefillParams& p, Start& start) {
    __shared__ int64_t sums[2][WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int heads = p.pool.n_kv * p.head_tiles, each = (p.n_requests + WARPS - 1) / WARPS;
    const int r0 = min(warp * each, p.n_requests), r1 = min(r0 + each, p.n_requests);
    auto add_up = [&](const Division* d) {
        int64_t units = 0, blocks = 0;
        for (int base = r0; base < r1; base += 32) {
            int n;
            units += units_of_requests<KEYS>(p, base + lane, base + lane < r1, d, n);
            blocks += n;
        }
        units = warp_sum(units), blocks = warp_sum(blocks);
        __syncthreads();
        if (lane == 0) sums[0][warp] = units, sums[1][warp] = blocks;
        __syncthreads();
    };
    add_up(nullptr);
    int64_t tiles = 0, blocks = 0;
    for (int w = 0; w < WARPS; w++) tiles += sums[0][w], blocks += sums[1][w];
    Division d;
    d.cut = 0;
    if (blocks * heads <= gridDim.x) {  // so that the pieces fit the grid
        const int64_t spare = max((int64_t)1, gridDim.x - blocks * heads);
        d.cut = (int)max((int64_t)kPieceLeast, (tiles * heads + spare - 1) / spare);
        add_up(&d);
        tiles = 0;
        for (int w = 0; w < WARPS; w++) tiles += sums[0][w];
        d.total = tiles * heads;
        d.share = 1;
    } else {
        d.total = (tiles + kOverhead * blocks) * heads;
        d.share = max((int64_t)1, (d.total + gridDim.x - 1) / gridDim.x);
    }
    const int64_t first = min(d.total, (int64_t)blockIdx.x * d.share), end = min(d.total, first + d.share);
    if (threadIdx.x == 0) start.left = 0;
    __syncthreads();
    if (first >= end) return d;
    // the warp whose requests hold the first unit looks for it
    int64_t before = 0;
    for (int w = 0; w < warp; w++) before += (sums[0][w] + (d.cut ? 0 : kOverhead * sums[1][w])) * heads;
    const int64_t mine = (sums[0][warp] + (d.cut ? 0 : kOverhead * sums[1][warp])) * heads;
    if (first >= before && first < before + mine) {
        for (int base = r0; base < r1; base += 32) {
            int n;
            const int64_t own = units_of_requests<KEYS>(p, base + lane, base + lane < r1, &d, n) * heads;
            int64_t upto = own;
#pragma unroll
            for (int i = 1; i < 32; i <<= 1) {
                const int64_t x = __shfl_up_sync(~0u, upto, i);
                if (lane >= i) upto += x;
            }
            const uint32_t found = __ballot_sync(~0u, before + upto > first);
            if (found == 0) {
                before += __shfl_sync(~0u, upto, 31);
                continue;
            }
            const int src = __ffs(found) - 1;
            const int64_t per_head = __shfl_sync(~0u, own, src) / heads;
            int64_t x = first - before - __shfl_sync(~0u, upto - own, src);
            Block k;
            k.r = base + src;
            k.head = (int)(x / per_head);
            x -= k.head * per_head;
            enter_request<KEYS>(p, k);
            const int all = blocks_of(p, k.rows);
            for (int b0 = 0; b0 < all; b0 += 32) {
                const int cost = b0 + lane < all ? d.units(tiles_of<KEYS>(p, k.position0, k.rows, b0 + lane)) : 0;
                int64_t sum = cost;
#pragma unroll
                for (int i = 1; i < 32; i <<= 1) {
                    const int64_t y = __shfl_up_sync(~0u, sum, i);
                    if (lane >= i) sum += y;
                }
                const uint32_t here = __ballot_sync(~0u, sum > x);
                if (here == 0) {
                    x -= __shfl_sync(~0u, sum, 31);
                    continue;
                }
                const int at = __ffs(here) - 1;
                x -= __shfl_sync(~0u, sum - cost, at);
                const int units = __shfl_sync(~0u, cost, at);
                k.b = b0 + at;
                enter_block<KEYS>(p, k);
                if (lane == 0) {
                    start.block = k;
                    if (d.cut) {
                        start.piece = (int)x, start.pieces = units;
                        start.j = (int)((int64_t)k.tiles * x / units);
                        start.left = (int64_t)k.tiles * (x + 1) / units - start.j;
                    } else {
                        start.j = (int)max((int64_t)0, x - kOverhead);
                        start.left = end - first - max((int64_t)0, kOverhead - x);
                        start.first_unit = first - x + kOverhead;
                        start.piece = 0, start.pieces = 1;
                    }
                }
                break;
            }
            break;
        }
    }
    return d;
}

// A run of tiles of one block.
struct Walk {
    Block block;
    int j, j_end;        // tiles
    int64_t left, first_unit;
};

template <int KEYS>
__device__ __forceinline__ bool begin_walk(const Start& s, Walk& w) {
    w.block = s.block, w.j = s.j, w.left = s.left, w.first_unit = s.first_unit;
    if (w.left <= 0) return false;
    w.j_end = (int)min((int64_t)w.block.tiles, w.j + w.left);
    return true;
}
// The next block of the stretch.  (The lengths stay as they are during a call; if they do not, the results are wrong, but nothing beyond the last
// request is read.)
template <int KEYS>
__device__ __forceinline__ bool next_block(const PrefillParams& p, const Division& d, Walk& w) {
    w.left -= w.j_end - w.j + kOverhead;
    if (d.cut || w.left <= 0) return false;
    w.first_unit += w.block.tiles + kOverhead;
    Block& k = w.block;
    if (++k.b >= blocks_of(p, k.rows)) {
        k.b = 0;
        if (++k.head >= p.pool.n_kv * p.head_tiles) {
            k.head = 0;
            do {
                if (++k.r >= p.n_requests) return false;
                enter_request<KEYS>(p, k);
            } while (k.rows == 0);
        }
    }
    enter_block<KEYS>(p, k);
    w.j = 0;
    w.j_end = (int)min((int64_t)k.tiles, w.left);
    return true;
}

// Whether some row of the block does not see some key of a tile: those at or behind `base`.
__device__ __forceinline__ bool partly_seen(const PrefillParams& p, const Block& k, int base, int keys) {
    const int position0 = k.position0 + k.b * p.tokens_a_block - k.gap, position1 = position0 + k.tokens - 1;
    return base + keys - 1 > position0 || (p.window > 0 && max(base, p.first) < min((int64_t)base + keys, (int64_t)position1 - p.window + 1));
}

// the lowest n bits, n of any size
__device__ __forceinline__ uint32_t lowest(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; }

// Where each element type puts p on its scale (the exponent of a weight at the reference) and how far above that weights may come before
// the reference moves.  bf16: 2^16 values at the type's end add up, whatever their weights are (values below 2^-94 lose bits by
// it).  f16: the upper end of its range, since its steps below are coarse.
template <class M>
constexpr float kRaiseOf = std::is_same<M, F16>::value ? 14.0f : -24.0f;
template <class M>
constexpr float kLagOf = std::is_same<M, F16>::value ? 1.9f : 8.0f;

// Two weights as two operand words that add up to them.  The first is rounded down and one more step below, so that the second is above
// zero and an infinite v stays what it is.
template <class M>
__device__ __forceinline__ void split(float a, float b, uint32_t& high, uint32_t& low) {
    uint32_t h;
    if constexpr (std::is_same<M, F16>::value)
        asm("cvt.rz.f16x2.f32 %0, %2, %1;" : "=r"(h) : "f"(a), "f"(b));
    else
        h = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
    h = __viaddmax_s16x2(h, 0xffffffffu, 0u);
    const float2 back = M::unpack(h);
    high = h;
    low = M::pack(a - back.x, b - back.y);
}

// 16 elements of 8 bits as 16 of type T
template <class T>
__device__ __forceinline__ void widen(const uint4& raw, uint4& a, uint4& b) {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    uint32_t y[8];
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const uint32_t h = E4M3::halves(k ? w[i] >> 16 : w[i]);
            if constexpr (std::is_same<T, F16>::value) y[2 * i + k] = h;
            else {
                const float2 f = F16::unpack(h);
                y[2 * i + k] = BF16::pack(f.x, f.y);
            }
        }
    a = make_uint4(y[0], y[1], y[2], y[3]), b = make_uint4(y[4], y[5], y[6], y[7]);
}

// Infinities and NaN among two 16-bit elements become zeros; whether there were any.
template <class T>
__device__ __forceinline__ bool make_finite(uint32_t& w) {
    constexpr uint32_t kEnd = std::is_same<T, F16>::value ? 0x7c00u : 0x7f80u;
    const bool low = (w & kEnd) == kEnd, high = (w >> 16 & kEnd) == kEnd;
    if (low) w &= 0xffff0000u;
    if (high) w &= 0x0000ffffu;
    return low || high;
}
template <class T>
__device__ __forceinline__ bool make_finite(uint4& x) {
    const bool a = make_finite<T>(x.x), b = make_finite<T>(x.y), c = make_finite<T>(x.z), d = make_finite<T>(x.w);
    return a || b || c || d;
}

// ---------------------------------------------------------------------------------------------- the kernel
template <class T, class C, int DP>
__global__ void __launch_bounds__(Shape<T, C, DP>::kThreads, 1) fcsim_kv_prefill_kernel(const __grid_constant__ PrefillParams p) {
    using S = Shape<T, C, DP>;
    constexpr int kTiles = S::kTiles, kKeys = S::kKeys, kStages = S::kStages;
    constexpr bool kNarrow = C::bytes == 1;
    constexpr float kRaise = kRaiseOf<T>, kLag = kLagOf<T>, kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
    constexpr int64_t kPatience = 4000000000ll;  // cycles that a wait may take: seconds, where microseconds are usual
    extern __shared__ char raw_smem[];
    __shared__ __align__(8) uint64_t bars[2 * kStages + 13];
    __shared__ uint32_t tmem_at, valid[8][4];
    __shared__ int stuck, infinite[4][S::kLoadWarps], joins[kTiles];
    __shared__ Start start;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int D = p.pool.head_dim, group = p.n_heads / p.pool.n_kv;
    const uint32_t smem = (smem_address(raw_smem) + 1023) & ~1023u, query = smem, ring = smem + S::kQuery;
    const uint32_t bar0 = smem_address(bars);
    auto full = [&](int s) { return bar0 + s * 8; };
    auto empty = [&](int s) { return bar0 + (kStages + s) * 8; };
    auto score_full = [&](int s) { return bar0 + (2 * kStages + s) * 8; };
    auto weights_ready = [&](int s) { return bar0 + (2 * kStages + 2 + s) * 8; };
    auto output_full = [&](int s) { return bar0 + (2 * kStages + 4 + s) * 8; };
    const uint32_t query_full = bar0 + (2 * kStages + 6) * 8, query_empty = query_full + 8, added = query_full + 16, drained = query_full + 24, both = query_full + 32;
    auto meeting = [&](int i) { return query_full + 40 + i * 8; };

    // A wait that ends: false when the time is up, and then for every other wait of the CTA too.
    auto wait = [&](uint32_t bar, uint32_t parity) {
        if (bar_try(bar, parity)) return true;
        const int64_t began = clock64();
        while (!bar_try(bar, parity)) {
            if (*(volatile int*)&stuck) return false;
            if (clock64() - began > kPatience) {
                *(volatile int*)&stuck = 1;
                flag(p.status, FCSIM_KV_STUCK);
                return false;
            }
        }
        return true;
    };

    if (tid == 0) {
        for (int s = 0; s < kStages; s++) bar_init(full(s), 32), bar_init(empty(s), 1);
        for (int s = 0; s < 2; s++) bar_init(score_full(s), 1), bar_init(weights_ready(s), 128), bar_init(output_full(s), 1);
        bar_init(query_full, 32 * S::kLoadWarps), bar_init(query_empty, 1), bar_init(added, 1), bar_init(drained, 1);
        bar_init(both, 256), bar_init(meeting(0), 128), bar_init(meeting(1), 128);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        stuck = 0;
    }
    // rows that belong to no request, and what is wrong with the requests
    {
        const int n0 = p.n_requests > 0 ? min(max(p.starts[0], 0), p.n_rows) : p.n_rows;
        const int n1 = p.n_requests > 0 ? min(max(p.starts[p.n_requests], n0), p.n_rows) : p.n_rows;
        const int64_t per_row = (int64_t)p.n_heads * (D / 8), none = ((int64_t)p.n_rows - n1 + n0) * per_row;
        for (int64_t i = (int64_t)blockIdx.x * S::kThreads + tid; i < none; i += (int64_t)gridDim.x * S::kThreads)
            reinterpret_cast<uint4*>(p.out)[i < n0 * per_row ? i : i + (n1 - n0) * per_row] = make_uint4(0, 0, 0, 0);
        if (p.lse)
            for (int64_t i = (int64_t)blockIdx.x * S::kThreads + tid; i < ((int64_t)p.n_rows - n1 + n0) * p.n_heads; i += (int64_t)gridDim.x * S::kThreads)
                p.lse[i < (int64_t)n0 * p.n_heads ? i : i + (int64_t)(n1 - n0) * p.n_heads] = -INFINITY;
        for (int r = blockIdx.x * S::kThreads + tid; r < p.n_requests; r += gridDim.x * S::kThreads) {
            const int a = p.starts[r], b = p.starts[r + 1], n = p.lengths[r];
            if (n < 0 || n > p.max_length || a < 0 || b < a || b > p.n_rows || b - a > n) flag(p.status, FCSIM_KV_BAD_LENGTH);
        }
    }
    const Division work = plan<kKeys, S::kWarps>(p, start);
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_address(&tmem_at)), "r"(S::kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (D % 16 != 0) {  // the products read elements by 16: what is beyond head_dim is zero, and stays so
        const int chunk = D / 8;
        auto clear = [&](uint32_t at, int rows, int tall) {
            for (int i = tid; i < rows; i += S::kThreads) {
                const uint32_t tile = at + i / tall * (tall * DP * 2);
                const int row = i % tall;
                store16(tile + chunk / 8 * (tall * 128) + row * 128 + ((chunk % 8) ^ (row % 8)) * 16, make_uint4(0, 0, 0, 0));
            }
        };
        clear(query, S::kRows, 128);
        clear(ring, kStages * kKeys, kKeys);
        fence_for_products();
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = tmem_at;

    Walk w;
    bool more = begin_walk<kKeys>(start, w);
    const int heads_a_tile = p.heads_a_tile;
    auto tiles_in_use = [&](const Block& k) { return kTiles == 2 && k.tokens * heads_a_tile > 128 ? 2 : 1; };

    if (warp >= S::kSoftmaxWarps && warp < S::kSoftmaxWarps + S::kLoadWarps) {
        // ------------------------------------------------------------------------------------------ loads
        // Tiles of K and V in the order in which they are used, one after the other to these warps: a warp waits for its own copies
        // while the others' are on their way.
        const int me = warp - S::kSoftmaxWarps;
        constexpr int kLanes = DP * C::bytes / 16, kAtOnce = 32 / kLanes, kRounds = kKeys / kAtOnce;  // lanes of a row, rows at once
        constexpr int kOffs = kKeys / 32, kBatch = kRounds < 16 ? kRounds : 16;
        const int chunk = lane % kLanes, lane_row = lane / kLanes, chunks = D * C::bytes / 16;
        const bool copies = chunk < chunks;
        int tile0 = 0, step0 = 0, segment = 0;  // tiles and steps of the segments before this one
        bool query_waits = false;               // copies of Q that are not yet told of
        auto tell_query = [&]() {
            if (!query_waits) return;
            fence_for_products();
            bar_arrive(query_full);
            query_waits = false;
        };
        int64_t next_off[kOffs];   // of the rows of this lane's tokens (lane, lane + 32, ..) in the tile that is loaded next, or -1
        uint32_t next_bad = 0;     // which of them are in a page outside the pool
        auto fetch_pages = [&](const Block& k, int j) {
            next_bad = 0;
#pragma unroll
            for (int c = 0; c < kOffs; c++) {
                const int u = j * kKeys + c * 32 + lane;
                next_off[c] = -1;
                if (u < k.seen) {
                    const int t = u + (u >= p.first ? k.gap : 0), i = page_of(p.pool, t), page = p.table[k.r * p.table_row + i];
                    if ((unsigned)page < (unsigned)p.pool.n_pages)
                        next_off[c] = (page * p.pool.stride_page + (t - i * p.pool.page_size) * p.pool.stride_slot + k.head / p.head_tiles * p.pool.stride_head) * C::bytes;
                    else
                        next_bad |= 1u << c;
                }
            }
        };
        // place in a stage of 16 bytes of a row
        auto place = [&](int row, int at) { return (uint32_t)(at / 8 * (kKeys * 128) + row * 128 + ((at % 8) ^ (row % 8)) * 16); };
        bool fine = true;
        while (more && fine) {
            const Block& k = w.block;
            const int steps = w.j_end - w.j;
            // tile x of the segment: which it is (with one tile of rows the scores run a step ahead)
            auto is_key = [&](int x) { return kTiles == 2 ? x % 2 == 0 : x == 0 || (x % 2 == 1 && x < 2 * steps - 1); };
            auto step_of = [&](int x) { return kTiles == 2 || x == 2 * steps - 1 ? x / 2 : is_key(x) ? (x + 1) / 2 : x / 2 - 1; };
            int x = (me + S::kLoadWarps - tile0 % S::kLoadWarps) % S::kLoadWarps;  // this warp's first
            if (x < 2 * steps) fetch_pages(k, w.j + step_of(x));
            if (lane == 0) infinite[segment & 3][me] = 0;
            // this warp's share of the rows of Q
            if (segment > 0 && !wait(query_empty, (segment - 1) & 1)) break;
            {
                constexpr int kQueryLanes = DP / 8, kQueryRows = 32 / kQueryLanes;
                const int at = lane % kQueryLanes, head0 = k.head / p.head_tiles * group, part0 = k.head % p.head_tiles * heads_a_tile;
                const int part = min(heads_a_tile, group - part0);
                for (int r0 = me * 32; r0 < tiles_in_use(k) * 128; r0 += 32 * S::kLoadWarps) {
                    const int row = r0 + lane, token = row / heads_a_tile, g = row - token * heads_a_tile;
                    int64_t off = -1;
                    if (token < k.tokens && g < part)
                        off = ((int64_t)(k.row0 + k.b * p.tokens_a_block + token) * p.q_row + (int64_t)(head0 + part0 + g) * p.q_head) * 2;
#pragma unroll
                    for (int i = 0; i < 32 / kQueryRows; i++) {
                        const int64_t o = __shfl_sync(~0u, off, i * kQueryRows + lane / kQueryLanes);
                        const int y = r0 + i * kQueryRows + lane / kQueryLanes;
                        if (at < D / 8)
                            copy16(query + y / 128 * (128 * DP * 2) + at / 8 * (128 * 128) + y % 128 * 128 + ((at % 8) ^ (y % 8)) * 16,
                                   p.q + (o < 0 ? 0 : o + at * 16), o < 0 ? 0 : 16);
                    }
                }
                commit_copies();
                query_waits = true;
            }
            for (; x < 2 * steps; x += S::kLoadWarps) {
                const int tile = tile0 + x, s = tile % kStages, j = w.j + step_of(x);
                const bool key = is_key(x), edge = !key && partly_seen(p, k, j * kKeys, kKeys);
                const char* const pool = key ? p.pool.k : p.pool.v;
                int64_t off[kOffs];
#pragma unroll
                for (int c = 0; c < kOffs; c++) {
                    off[c] = next_off[c];
                    if (key) {
                        const uint32_t bad = __ballot_sync(~0u, next_bad >> c & 1);
                        if (lane == 0) {
                            valid[(step0 + step_of(x)) & 7][c] = ~bad;  // (what lies behind the last token is no row's)
                            if (bad) flag(p.status, FCSIM_KV_BAD_PAGE);
                        }
                    }
                }
                if (x + S::kLoadWarps < 2 * steps) fetch_pages(k, w.j + step_of(x + S::kLoadWarps));
                if (tile >= kStages && !bar_try(empty(s), (tile / kStages - 1) & 1)) {
                    if (query_waits) {
                        wait_copies<0>();
                        tell_query();
                    }
                    if (!(fine = wait(empty(s), (tile / kStages - 1) & 1))) break;
                }
                const uint32_t to = ring + s * S::kStage;
                bool found = false;
                if constexpr (kNarrow) {
#pragma unroll 1
                    for (int i0 = 0; i0 < kRounds; i0 += kBatch) {
                        uint4 raw[kBatch];
#pragma unroll
                        for (int i = 0; i < kBatch; i++) {
                            const int row = (i0 + i) * kAtOnce + lane_row;
                            int64_t o = __shfl_sync(~0u, off[0], row % 32);
#pragma unroll
                            for (int c = 1; c < kOffs; c++) {
                                const int64_t other = __shfl_sync(~0u, off[c], row % 32);
                                if (row / 32 == c) o = other;
                            }
                            raw[i] = make_uint4(0, 0, 0, 0);
                            if (copies && o >= 0) raw[i] = *reinterpret_cast<const uint4*>(pool + o + chunk * 16);
                        }
                        if (copies) {
#pragma unroll
                            for (int i = 0; i < kBatch; i++) {
                                const int row = (i0 + i) * kAtOnce + lane_row;
                                uint4 a, b;
                                widen<T>(raw[i], a, b);
                                if (edge) found |= make_finite<T>(a) | make_finite<T>(b);
                                store16(to + place(row, 2 * chunk), a);
                                store16(to + place(row, 2 * chunk + 1), b);
                            }
                        }
                    }
                    if (query_waits) {
                        wait_copies<0>();
                        tell_query();
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < kRounds; i++) {
                        const int row = i * kAtOnce + lane_row;
                        const int64_t o = __shfl_sync(~0u, off[i * kAtOnce / 32], row % 32);
                        if (copies) copy16(to + place(row, chunk), pool + (o < 0 ? 0 : o + chunk * 16), o < 0 ? 0 : 16);
                    }
                    commit_copies();
                    if (query_waits) {
                        wait_copies<1>();
                        tell_query();
                    }
                    wait_copies<0>();
                    if (edge && copies) {
                        // what some row does not see must not meet its weight of zero as an infinity or NaN
#pragma unroll 4
                        for (int i = 0; i < kRounds; i++) {
                            const uint32_t at = to + place(i * kAtOnce + lane_row, chunk);
                            uint4 y = load16(at);
                            if (make_finite<T>(y)) {
                                store16(at, y);
                                found = true;
                            }
                        }
                    }
                }
                if (__any_sync(~0u, found) && lane == 0) infinite[segment & 3][me] = 1;
                fence_for_products();
                bar_arrive(full(s));
            }
            if (query_waits) {
                wait_copies<0>();
                tell_query();
            }
            tile0 += 2 * steps, step0 += steps, segment++;
            more = next_block<kKeys>(p, work, w);
        }
        wait_copies<0>();
    } else if (warp == S::kSoftmaxWarps + S::kLoadWarps) {
        // ------------------------------------------------------------------------------------------ products
        if (lane == 0) {
            constexpr uint32_t kType = std::is_same<T, F16>::value ? 0 : 1;
            const uint32_t how_score = instruction(kType, false, 128, kKeys), how_output = instruction(kType, true, 128, (D + 15) / 16 * 16);
            const int depth = (D + 15) / 16;
            int tile = 0, segment = 0, step = 0;
            uint32_t ready[2] = {0, 0};  // parities of the weights
            auto score = [&](int slot, int i, int s) {  // S of row tile i, with K in stage s
                const uint64_t a = operand(query + i * (128 * DP * 2), 16, 1024), b = operand(ring + s * S::kStage, 16, 1024);
                for (int k = 0; k < depth; k++)
                    product(tmem + S::kScore + slot * kKeys, a + ((k / 4 * (128 * 128) + k % 4 * 32) >> 4), b + ((k / 4 * (kKeys * 128) + k % 4 * 32) >> 4),
                            how_score, k > 0);
                commit_products(score_full(slot));
            };
            auto output = [&](int slot, int i, int s, bool add) {  // O of row tile i, with V in stage s
                const uint64_t b = operand(ring + s * S::kStage, kKeys * 128, 1024);
                const uint32_t to = tmem + S::kOutput + i * DP, from = tmem + S::kScore + slot * kKeys;
#pragma unroll
                for (int part = 0; part < 2; part++)
#pragma unroll
                    for (int k = 0; k < kKeys / 16; k++)
                        product_from_tmem(to, from + k / 2 * 32 + part * 16 + k % 2 * 8, b + (k * 2048 >> 4), how_output, add || part > 0 || k > 0);
            };
            auto wait_full = [&](int t) {
                if (!wait(full(t % kStages), (t / kStages) & 1)) return false;
                fence_after_sync();
                return true;
            };
            bool fine = true;
            while (more && fine) {
                const int n = tiles_in_use(w.block), steps = w.j_end - w.j;
                fine = wait(query_full, segment & 1) && wait_full(tile);
                if (!fine) break;
                for (int i = 0; i < n; i++) score(kTiles == 2 ? i : step & 1, i, tile % kStages);
                commit_products(empty(tile % kStages));
                tile++;
                if (steps == 1) commit_products(query_empty);
                for (int j = 0; j < steps && fine; j++) {
                    const bool another = j + 1 < steps;
                    if constexpr (kTiles == 1) {
                        // the next step's scores, then this one's output
                        if (another) {
                            if (!(fine = wait_full(tile))) break;
                            score((step + 1) & 1, 0, tile % kStages);
                            commit_products(empty(tile % kStages));
                            tile++;
                            if (j + 2 == steps) commit_products(query_empty);
                        }
                        const int slot = step & 1;
                        fine = wait_full(tile) && wait(weights_ready(slot), ready[slot]);
                        if (!fine) break;
                        ready[slot] ^= 1;
                        fence_after_sync();
                        output(slot, 0, tile % kStages, j > 0);
                        commit_products(empty(tile % kStages));
                        commit_products(added);
                        if (!another) commit_products(output_full(0));
                        tile++;
                    } else {
                        // tile after tile: the output of this step, then the scores of the next
                        const int v = tile, k = tile + 1;
                        fine = wait_full(v);
                        for (int i = 0; i < n && fine; i++) {
                            if (!(fine = wait(weights_ready(i), ready[i]))) break;
                            ready[i] ^= 1;
                            fence_after_sync();
                            output(i, i, v % kStages, j > 0);
                            if (i == n - 1) commit_products(empty(v % kStages));
                            if (another) {
                                if (i == 0 && !(fine = wait_full(k))) break;
                                score(i, i, k % kStages);
                                if (i == n - 1) {
                                    commit_products(empty(k % kStages));
                                    if (j + 2 == steps) commit_products(query_empty);
                                }
                            } else
                                commit_products(output_full(i));
                        }
                        tile += another ? 2 : 1;
                    }
                    step++;
                }
                segment++;
                more = next_block<kKeys>(p, work, w);
            }
            commit_products(drained);  // nothing is in flight when the CTA ends
            const int64_t began = clock64();
            while (!bar_try(drained, 0) && clock64() - began < kPatience) {}
        }
        __syncwarp();
    } else if (warp < S::kSoftmaxWarps) {
        // ------------------------------------------------------------------------------------------ softmax
        const int i = warp >> 2, row = tid & 127;  // tile; its row
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // this warp's lanes of tensor memory: 32 (warp % 4) << 16
        const uint32_t mine = tmem + S::kOutput + i * DP + lanes;
        const int token = (i * 128 + row) / heads_a_tile, g = i * 128 + row - token * heads_a_tile;
        int step = 0, segment = 0, before_tiles = 0;
        uint32_t score_parity[2] = {0, 0}, output_parity = 0, both_parity = 0, meeting_parity = 0;
        bool fine = true;
        auto meet = [&](uint32_t bar, uint32_t& parity) {
            bar_arrive(bar);
            const bool ok = wait(bar, parity);
            parity ^= 1;
            return ok;
        };
        while (more && fine) {
            const Block& k = w.block;
            const int n = tiles_in_use(k), steps = w.j_end - w.j;
            if (kTiles == 2) {
                // (a group that sits out does not run ahead of one that is at work: flags of a few segments are kept)
                if (before_tiles == 2 && n == 1 && !meet(both, both_parity)) break;
                before_tiles = n;
                if (i >= n) {
                    step += steps, segment++;
                    more = next_block<kKeys>(p, work, w);
                    continue;
                }
            }
            const int kv = k.head / p.head_tiles, head = k.head % p.head_tiles * heads_a_tile + g;
            const bool real = token < k.tokens && head < group && g < heads_a_tile;
            const float unit = (kNarrow ? p.scale * p.pool.k_scale[kv] : p.scale) * kLog2e;
            const bool turned = unit < 0;
            // the last seen key of this row and the first of its window; nothing for rows that are none
            const int position = k.position0 + k.b * p.tokens_a_block + token - k.gap;
            const int last = real ? position : -1, from = p.window > 0 && position >= p.window ? position - p.window + 1 : 0;
            float add = INFINITY, limit = -INFINITY, sum = 0;  // weights are 2^(unit s + add); add is infinite until there is a finite logit
            for (int j = w.j; j < w.j_end; j++, step++) {
                const int slot = kTiles == 2 ? i : step & 1, base = j * kKeys;
                const uint32_t at = tmem + S::kScore + slot * kKeys + lanes;
                if (!(fine = wait(score_full(slot), score_parity[slot]))) break;
                score_parity[slot] ^= 1;
                fence_after_sync();
                uint32_t there = ~0u;
#pragma unroll
                for (int c = 0; c < kKeys / 32; c++) there &= valid[step & 7][c];
                const bool masked = there != ~0u || partly_seen(p, k, base, kKeys);
                uint32_t mask[kKeys / 32];
                if (masked) {
#pragma unroll
                    for (int c = 0; c < kKeys / 32; c++)
                        mask[c] = lowest(last + 1 - base - 32 * c) & (~lowest(from - base - 32 * c) | lowest(p.first - base - 32 * c)) & valid[step & 7][c];
                }
                // the largest logit (with a negative scale: the lowest)
                const float none = turned ? INFINITY : -INFINITY;
                float top = none;
#pragma unroll
                for (int c = 0; c < kKeys / 32; c++) {
                    float s[32];
                    tmem_load(at + 32 * c, s);
                    wait_loads();
                    if (masked) {
#pragma unroll
                        for (int e = 0; e < 32; e++) s[e] = mask[c] >> e & 1 ? s[e] : none;
                    }
                    if (turned) {
#pragma unroll
                        for (int e = 0; e < 32; e++) top = fminf(top, s[e]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; e++) top = fmaxf(top, s[e]);
                    }
                }
                const float most = top == none ? -INFINITY : top * unit;
                // The reference moves only when a logit is 2^kLag above it, so that the output is seldom taken through registers.
                bool moves = most > limit;
                float shrink = 1;
                if (moves) {
                    const bool first_one = limit == -INFINITY;
                    const float now = kRaise - most;
                    shrink = first_one ? 0.0f : power2(now - add);
                    add = now;
                    limit = most + kLag;
                    sum *= shrink;
                }
                if (j > w.j && __any_sync(~0u, moves)) {
                    if (kTiles == 1 && !(fine = wait(added, (step - 1) & 1))) break;
                    fence_after_sync();
#pragma unroll
                    for (int c = 0; c < DP / 32; c++)
                        if (c * 32 < D) {
                            float o[32];
                            uint32_t x[32];
                            tmem_load(mine + 32 * c, o);
                            wait_loads();
#pragma unroll
                            for (int e = 0; e < 32; e++) x[e] = __float_as_uint(o[e] * shrink);
                            tmem_store(mine + 32 * c, x);
                        }
                }
                const float plus = limit == -INFINITY ? 0.0f : add;
                float sums[4] = {0, 0, 0, 0};
#pragma unroll
                for (int c = 0; c < kKeys / 32; c++) {
                    float s[32];
                    uint32_t x[32];
                    tmem_load(at + 32 * c, s);
                    wait_loads();
#pragma unroll
                    for (int e = 0; e < 32; e++) {
                        s[e] = power2(fmaf(s[e], unit, plus));
                    }
                    if (masked) {
#pragma unroll
                        for (int e = 0; e < 32; e++) s[e] = mask[c] >> e & 1 ? s[e] : 0.0f;
                    }
#pragma unroll
                    for (int e = 0; e < 32; e++) sums[e & 3] += s[e];
#pragma unroll
                    for (int e = 0; e < 16; e++) split<T>(s[2 * e], s[2 * e + 1], x[e], x[16 + e]);
                    tmem_store(at + 32 * c, x);
                }
                sum += (sums[0] + sums[1]) + (sums[2] + sums[3]);
                wait_stores();
                fence_before_sync();
                bar_arrive(weights_ready(slot));
            }
            if (!fine) break;
            // -------------------------------------------------------------- end of this CTA's part of a block
            if (!(fine = wait(output_full(i), output_parity))) break;
            output_parity ^= 1;
            fence_after_sync();
            bool poisoned = false;
#pragma unroll
            for (int x = 0; x < S::kLoadWarps; x++) poisoned |= infinite[segment & 3][x] != 0;
            int first_part = blockIdx.x, final_part = blockIdx.x;  // CTAs that have parts of the block
            if (work.cut) {
                first_part -= start.piece;
                final_part = first_part + start.pieces - 1;
            } else {
                first_part = (int)(w.first_unit / work.share);
                final_part = (int)((w.first_unit + k.tiles - 1) / work.share);
            }
            const bool whole = first_part == final_part;
            constexpr int64_t kPart = (int64_t)(DP + 2) * 128;
            auto part_of = [&](int cta) { return p.parts + ((2 * (int64_t)cta + (cta == first_part ? 1 : 0)) * kTiles + i) * kPart; };
            const int64_t out_row = (int64_t)(k.row0 + k.b * p.tokens_a_block + token) * p.n_heads + kv * group + head;
            const float vscale = kNarrow ? p.pool.v_scale[kv] : 1.0f;
            auto store_row = [&](const float (&o)[32], int c, float f, bool none) {  // elements 32 c ..
                char* const to = p.out + (out_row * D + c * 32) * 2;
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (c * 32 + e * 8 < D)
                        *reinterpret_cast<uint4*>(to + e * 16) = none ? make_uint4(0, 0, 0, 0)
                            : make_uint4(T::pack(o[8 * e] * f, o[8 * e + 1] * f), T::pack(o[8 * e + 2] * f, o[8 * e + 3] * f),
                                         T::pack(o[8 * e + 4] * f, o[8 * e + 5] * f), T::pack(o[8 * e + 6] * f, o[8 * e + 7] * f));
            };
            auto finish = [&](float all, float plus) {
                if (p.lse) p.lse[out_row] = all == 0.0f ? -INFINITY : logf(all) - plus * kLn2;
            };
            float* const part = part_of(blockIdx.x);
            const float f = sum == 0.0f ? 0.0f : vscale / sum;
#pragma unroll 1
            for (int c = 0; c < DP / 32; c++) {
                if (c * 32 >= D) break;
                float o[32];
                tmem_load(mine + 32 * c, o);
                wait_loads();
                if (poisoned && real) {
                    // infinite and NaN elements of v in tiles that are not seen whole were left out of the products: those this row sees
                    for (int j = w.j; j < w.j_end; j++) {
                        if (!partly_seen(p, k, j * kKeys, kKeys)) continue;
                        for (int u = j * kKeys; u < min(k.seen, (j + 1) * kKeys); u++) {
                            if (u > position || (u < from && u >= p.first)) continue;
                            const int t = u + (u >= p.first ? k.gap : 0), x = page_of(p.pool, t), page = p.table[k.r * p.table_row + x];
                            if ((unsigned)page >= (unsigned)p.pool.n_pages) continue;
                            const char* const v = p.pool.v + (page * p.pool.stride_page + (t - x * p.pool.page_size) * p.pool.stride_slot + kv * p.pool.stride_head + c * 32) * C::bytes;
#pragma unroll
                            for (int e = 0; e < 16; e++)
                                if (c * 32 + 2 * e < D) {
                                    float2 y;
                                    if constexpr (kNarrow) y = F16::unpack(E4M3::halves(*reinterpret_cast<const uint16_t*>(v + 2 * e)));
                                    else y = C::unpack(*reinterpret_cast<const uint32_t*>(v + 4 * e));
                                    if (!(fabsf(y.x) < INFINITY)) o[2 * e] += y.x;
                                    if (!(fabsf(y.y) < INFINITY)) o[2 * e + 1] += y.y;
                                }
                        }
                    }
                }
                if (!whole) {
#pragma unroll
                    for (int e = 0; e < 32; e++) part[(c * 32 + e) * 128 + row] = o[e];
                } else if (real)
                    store_row(o, c, f, sum == 0.0f);
            }
            fence_before_sync();
            if (whole) {
                if (real) finish(sum, add);
            } else {
                part[DP * 128 + row] = add;
                part[(DP + 1) * 128 + row] = sum;
                __threadfence();
                if (!(fine = meet(meeting(i), meeting_parity))) break;
                if (row == 0) {
                    int* const counter = p.counters + first_part * 2 + i;
                    const bool last_one = atomicAdd(counter, 1) == final_part - first_part;
                    joins[i] = last_one;
                    if (last_one) *counter = 0;
                }
                if (!(fine = meet(meeting(i), meeting_parity))) break;
                if (joins[i]) {
                    __threadfence();
                    float least = INFINITY;  // of add: the highest reference
                    for (int x = first_part; x <= final_part; x++) least = fminf(least, __ldcg(part_of(x) + DP * 128 + row));
                    float all = 0;
                    for (int x = first_part; x <= final_part; x++) {
                        const float* const from_part = part_of(x);
                        const float a = __ldcg(from_part + DP * 128 + row), y = a == INFINITY ? 0.0f : power2(least - a);
                        all += y * __ldcg(from_part + (DP + 1) * 128 + row);
                    }
                    const float g = all == 0.0f ? 0.0f : vscale / all;
#pragma unroll 1
                    for (int c = 0; c < DP / 32; c++) {
                        if (c * 32 >= D) break;
                        float o[32] = {};
                        for (int x = first_part; x <= final_part; x++) {
                            const float* const from_part = part_of(x);
                            const float a = __ldcg(from_part + DP * 128 + row), y = a == INFINITY ? 0.0f : power2(least - a);
#pragma unroll
                            for (int e = 0; e < 32; e++) o[e] += y * __ldcg(from_part + (c * 32 + e) * 128 + row);
                        }
                        if (real) store_row(o, c, g, all == 0.0f);
                    }
                    if (real) finish(all, least);
                }
            }
            segment++;
            more = next_block<kKeys>(p, work, w);
        }
    }
    fence_before_sync();
    __syncthreads();
    if (warp == 0) {
        fence_after_sync();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kColumns) : "memory");
    }
}

template <class T, class C, int DP>
int launch(const PrefillParams& p, int grid, int device, cudaStream_t stream) {
    using S = Shape<T, C, DP>;
    static std::atomic<bool> raised[kMaxDevices];
    if (device >= kMaxDevices || !raised[device].load(std::memory_order_relaxed)) {
        const cudaError_t e = cudaFuncSetAttribute(fcsim_kv_prefill_kernel<T, C, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kBytes);
        if (e != cudaSuccess) return (int)e;
        if (device < kMaxDevices) raised[device].store(true, std::memory_order_relaxed);
    }
    fcsim_kv_prefill_kernel<T, C, DP><<<grid, S::kThreads, S::kBytes, stream>>>(p);
    return (int)cudaGetLastError();
}
template <class T, class C, int DP>
PrefillVariant variant() {
    return {launch<T, C, DP>, Shape<T, C, DP>::kRows, Shape<T, C, DP>::kKeys, DP};
}
template <class T, class C>
PrefillVariant of(int head_dim) {
    return head_dim <= 64 ? variant<T, C, 64>() : head_dim <= 128 ? variant<T, C, 128>() : variant<T, C, 256>();
}

}  // namespace

#if FCSIM_KV_TYPES == 0
PrefillVariant prefill_variant_f16(int head_dim) { return of<F16, F16>(head_dim); }
#elif FCSIM_KV_TYPES == 1
PrefillVariant prefill_variant_bf16(int head_dim) { return of<BF16, BF16>(head_dim); }
#elif FCSIM_KV_TYPES == 2
PrefillVariant prefill_variant_f16_e4m3(int head_dim) { return of<F16, E4M3>(head_dim); }
#else
PrefillVariant prefill_variant_bf16_e4m3(int head_dim) { return of<BF16, E4M3>(head_dim); }
#endif

}  // namespace fcsim_kv_dev
