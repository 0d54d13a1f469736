// Attention of several query tokens per request over a paged cache (compiled once per pair of types: FCSIM_KV_TYPES 0..3).
//
//   o_i = sum_t p_t v_t / sum_t p_t,   p_t = exp(c q_i . k_t - m),   over the tokens t that row i sees:
//   t <= position of i, and with a window also t > position - window or t < first
//
// * The query heads of a kv head and a run of tokens are the rows of a block: one or two tiles of 128 (token, head) pairs, so that
//   few new tokens fill a tile as well as many do, and what is loaded of K and V serves all of them.
// * Both products run on tcgen05: S = Q K^T from shared memory into tensor memory, P back into the columns S had, O += P V with
//   P read from tensor memory.  One thread issues them.  Each tile of rows has a group of four warps, a row a thread, for its softmax, whose
//   time is that of the other tile's products; with one tile of rows the groups take its tiles of keys in turn.
// * Six warps load, half a tile each in turn, into a ring: by bulk copies of the pages' tokens where a page is whole boxes of 8 tokens or
//   more, else 16 bytes a lane (cp.async), both in the 128-byte swizzled layout that the products read.  (8 192 tokens, 32 heads:
//   688 us in boxes when 745 by lanes.)  8-bit rows are turned into 16 bits, exactly, in shared memory.  What some row of a tile does not see is
//   looked over in v: infinities and NaN would reach rows whose weight for them is zero.  One warp walks over the work ahead of the others.
// * The work is counted in tiles of keys, laid end to end over all requests, heads and blocks, and every CTA takes an equal stretch (or, where
//   there are few blocks, one piece of one block).  Parts of a block that lies across stretches are joined by the last to come, in
//   their order: the same call gives the same bits.
// * s, m, the sums and o are 32-bit; a tile's weights are added up by themselves, and what 128 tiles have added to o is put aside, since the tensor core
//   cuts its sums off.  p meets v in two 16-bit parts that add up to it to 2^-14 (bf16) or 2^-20 (f16): with one, its rounding
//   would be as large as the output's own.  The second part is a third of the products: of two tiles of rows and 128 keys the scores take 1 024
//   clocks (64 a product of 128 x 128 x 16), the parts 1 024 each; the exponentials, beside them, 2 050.
//
// Bounds.  Long prompts: the products, three quarters of the 4 200 clocks that such a step takes (8 192 tokens, 32 heads of 128: 660 us, 830 TFLOP/s with p
// counted once, 1 245 of products done); the rest is what one tile's softmax takes longer than the other tile's products.
// Few tokens over a long context: the loads, at 4.6 TB/s (16 x 7 tokens over 8 000, 64 heads: 115 us), and with an 8-bit cache the instructions that turn
// them (197 us; 8 192 tokens 904 to 985 us by the GPU).  Widths over 128, with one tile of rows, one group for the softmax and 64 keys a tile: products, 68 and
// 59 % of their rate (4 096 tokens, 32 heads of 256: 370 us, 744 TFLOP/s with p counted once; of 192 321; over 8 bits 671 and 636).  Small calls: latency, 10 us.
// With the shared memory that this kernel takes there is next to no L1 cache, so what lies in local memory (spilled registers, structs whose address is
// taken) is at L2's distance: hence the registers' split by role, and values in place of references.
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
// and with as many bytes of bulk copies to come
__device__ __forceinline__ void bar_expect(uint32_t bar, int bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// as many bytes of bulk copies to come, the arrival itself being still to come too
__device__ __forceinline__ void bar_bytes(uint32_t bar, int bytes) {
    asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// whether the phase of this parity is over; the thread sleeps for up to so many nanoseconds
__device__ __forceinline__ bool bar_sleep(uint32_t bar, uint32_t parity, uint32_t ns) {
    uint32_t done;
    asm volatile(
        "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}"
        : "=r"(done) : "r"(bar), "r"(parity), "r"(ns) : "memory");
    return done != 0;
}
// a box of a tensor of 4 or 3 dimensions into shared memory, rows of 128 bytes swizzled by 128 bytes
__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
}
__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
        : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
__device__ __forceinline__ void fence_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// What was loaded from tensor memory is there.  (`x`: where it was loaded to.  Nothing else says that it changes here, and the compiler is free to
// move what reads a register to before a wait that does not name it.)
template <int N>
__device__ __forceinline__ void loaded(float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; i++) asm volatile("" : "+f"(x[i])::"memory");
}
template <int... N>
__device__ __forceinline__ void wait_loads(float (&... x)[N]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
    (loaded(x), ...);
}
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
__device__ __forceinline__ void tmem_load16(uint32_t at, float (&x)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]), "=f"(x[8]), "=f"(x[9]), "=f"(x[10]),
          "=f"(x[11]), "=f"(x[12]), "=f"(x[13]), "=f"(x[14]), "=f"(x[15])
        : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t (&x)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(at), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]), "r"(x[8]), "r"(x[9]),
                   "r"(x[10]), "r"(x[11]), "r"(x[12]), "r"(x[13]), "r"(x[14]), "r"(x[15]) : "memory");
}
// two 32-bit values at once
__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t x;
    asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(a), "f"(b));
    return x;
}
__device__ __forceinline__ float2 unpair(uint64_t x) {
    float2 y;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(y.x), "=f"(y.y) : "l"(x));
    return y;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
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

// whichever of the warp's lanes, for numbers that are the same in all: in a register of the warp, as what issues products needs them
__device__ __forceinline__ uint32_t uni(uint32_t x) { return __reduce_max_sync(~0u, x); }
__device__ __forceinline__ bool elected() {
    uint32_t x;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(x));
    return x != 0;
}

// ---------------------------------------------------------------------------------------------- shape
template <class T, class C, int DP>
struct Shape {
    static constexpr int kTiles = DP <= 128 ? 2 : 1;    // of 128 rows: two where their outputs fit tensor memory
    static constexpr int kRows = 128 * kTiles;
    static constexpr int kKeys = DP <= 128 ? 128 : 64;  // of a tile
    static constexpr int kQuery = kRows * DP * 2;       // bytes
    static constexpr int kStage = kKeys * DP * 2;       // of K or V
    static constexpr int kRoom = (224 * 1024 - kQuery) / kStage;  // (of 227 KB, 3 for what the kernel keeps itself)
    static constexpr int kStages = kRoom < 8 ? kRoom : 8;
    static constexpr int kBytes = kQuery + kStages * kStage;
    static constexpr int kSoftmaxWarps = 4 * kTiles, kLoadWarps = 6;
    static constexpr int kWarps = kSoftmaxWarps + kLoadWarps + 2, kThreads = 32 * kWarps;
    // With two tiles the kernel starts with 128 registers a thread, and the loads' warps leave some of theirs to the softmax's: fewer where they turn
    // 8-bit rows (8 192 tokens, 32 heads, 8-bit cache: 144 and 112 take 1 065 us, 160 and 96 1 155; a 16-bit one 718 and 682), and at width 64, where
    // more is spilled otherwise (2 048 tokens: 72 us, 76).
    static constexpr int kSoftmaxRegisters = C::bytes == 1 || DP == 64 ? 144 : 160, kOtherRegisters = 256 - kSoftmaxRegisters;
    // A warp loads half a tile at a time.  It waits for the place of a tile by the parity of one barrier, so the tile that was there two rounds before
    // has to be gone: it is, as what the warp has loaded last waited for a later one.
    static_assert(kLoadWarps <= 2 * kStages, "parities");
    static_assert(kTiles == 1 || 256 * kSoftmaxRegisters + 256 * kOtherRegisters <= 128 * kThreads, "a split beyond the launch's total waits for good");
    // tensor memory: two areas of kKeys columns for S and P, then O of each tile
    static constexpr int kScore = 0, kOutput = 2 * kKeys, kColumns = 512;
    static_assert(kOutput + kTiles * DP <= kColumns && kStages >= 4, "room");
};

// ---------------------------------------------------------------------------------------------- the walk over the work
// Cost of a block's start and end beside one tile of keys (4 096 tokens, 32 heads: 221 us, without it 256; 12 x 200 tokens, 64 heads: 72, 94).
constexpr int kOverhead = 2;
constexpr int kPieceLeast = 2;  // tiles of a piece at least, where blocks are cut
// Tiles by which the longest piece may exceed an equal share: what the joins of shares cost more than those of pieces.  (Always pieces: a request of 60 000 tokens beside 16
// of 50, 8 new ones each, takes 340 us instead of 84.  Pieces where whole blocks are as few tiles longer: 400 tokens 27.3 us instead of 19.7.  Always shares: 16 tokens over 60 000 take 90 us instead of 88, 50 x 20 over 2 000 122 and 121.)
constexpr int kShareCost = 4;
// And by which whole blocks, one a CTA, may exceed it, since they need no join: fewer where 8-bit rows are turned, which doubles a tile's time.  (16 x 7
// tokens, whole and in shares: over 6 000 of 16 bits 89 and 95 us, over 24 000 302 and 290; over 3 000 of 8 bits 93 and 97, over 16 000 392 and 350.
// Lengths from 1 000 to 16 000: 194 and 124 us of 16 bits, 397 and 180 of 8.)
template <class C, int DP>
constexpr int kWholeGain = C::bytes == 1 && DP > 64 ? 5 : 11;
// So many requests are planned for by one warp, a lane each, without barriers, while the others set up; with more every warp takes part.  (18 x 30 tokens,
// whole blocks: 23.5 us, by all warps 25.6.  32 x 8 tokens, more blocks than CTAs: 30, of 33 by all warps 28.)
constexpr int kOneWarpPlans = 32;
// A block with one tile of rows is shared by the two groups of warps from so many tiles of keys on: each takes every other one, and the first
// adds up what both have (16 x 7 tokens over 8 000: 113 us, by one group alone 174).
constexpr int kSharedLeast = 2;

// A block of rows: tokens [b * tokens_a_block, + tokens) of the new ones of a request, heads of one head tile.
struct Block {
    int r, kv, ht, b;
    int row0, rows, position0;   // the request's rows in q; position of the first of them
    int tokens, gap, seen, tiles;
};

__device__ __forceinline__ int request_rows(const PrefillParams& p, int r, int& row0) {
    row0 = min(max(p.starts[r], 0), p.n_rows);
    return max(min(p.starts[r + 1], p.n_rows) - row0, 0);
}
__device__ __forceinline__ int request_length(const PrefillParams& p, int r) { return min(max(p.lengths[r], 0), p.max_length); }

// What a block of tokens sees: all tokens up to its last one, or the first ones and, without the gap behind these, those from the start of
// its first token's window.  Counted without the gap: seen key u is token u, or behind the first ones u + gap.  (Both ends of the gap are rounded
// so that what one bulk copy brings lies on one side of it.)
__device__ __forceinline__ int seen_by(const PrefillParams& p, int position0, int tokens, int& gap) {
    gap = 0;
    if (p.window > 0) {
        const int64_t low = (int64_t)position0 - p.window + 1;  // (a request of more rows than tokens has positions below 0)
        if (low > p.kept) gap = (int)(low - p.kept) & -max(p.box, 1);
    }
    return max(position0 + tokens - gap, 0);
}
template <int KEYS>
__device__ __forceinline__ int tiles_of(const PrefillParams& p, int position0, int rows, int b) {
    int gap;
    const int at = b * p.tokens_a_block;
    return max(1, (int)((unsigned)(seen_by(p, position0 + at, min(p.tokens_a_block, rows - at), gap) + KEYS - 1) / KEYS));
}
__device__ __forceinline__ int blocks_of(const PrefillParams& p, int rows) { return (unsigned)(rows + p.tokens_a_block - 1) / (unsigned)p.tokens_a_block; }

template <int KEYS>
__device__ __forceinline__ void enter_block(const PrefillParams& p, Block& x) {
    const int at = x.b * p.tokens_a_block;
    x.tokens = min(p.tokens_a_block, x.rows - at);
    x.seen = seen_by(p, x.position0 + at, x.tokens, x.gap);
    x.tiles = max(1, (int)((unsigned)(x.seen + KEYS - 1) / KEYS));
}
__device__ __forceinline__ void enter_request(const PrefillParams& p, Block& x) {
    x.rows = request_rows(p, x.r, x.row0);
    x.position0 = request_length(p, x.r) - x.rows;
}

__device__ __noinline__ int64_t divide_wide(int64_t a, int64_t b) { return a / b; }
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {  // neither below 0
    return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : divide_wide(a, b);
}

// The division of the units among the CTAs, which depends on the lengths and the grid alone.  A unit is a tile of keys (and kOverhead of them
// stand before a block's first tile), or, with `cut`, a piece of a block of at most `cut` tiles.
struct Division {
    int64_t first, end, share;  // of this CTA
    int cut;
    __device__ __forceinline__ int units(int tiles) const { return cut ? (unsigned)(tiles + cut - 1) / (unsigned)cut : tiles + kOverhead; }
};

// The work of one warp's walk: a block and tiles j .. j_end of it.
struct Walk {
    Block block;
    int j, j_end;
    int64_t left;        // units from j to the end of the stretch, or the piece's tiles; none: no work
    int64_t first_unit;  // of the block's first tile (without `cut`)
    int piece, pieces;   // with `cut`
};

__device__ __forceinline__ int64_t warp_sum(int64_t x) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    return x;
}

// Tiles of one of the heads of a lane's request (`rows` of them from position0 on), with `cut` its pieces of so many tiles, `over` more for each block.
// Long requests are added up by the warp.
template <int KEYS>
__device__ __forceinline__ int64_t add_blocks(const PrefillParams& p, int rows, int position0, int cut, int over) {
    // A lane adds up to two blocks itself, or where several requests have more, up to 24: the warp takes as long for a request as a lane for six
    // (12 requests of 200 tokens, 64 heads: 56.5 us a call, with two always 61.4; one of 400: 27.4, with 24 always 28.3).
    const int lane = threadIdx.x & 31, blocks = blocks_of(p, rows), alone = __popc(__ballot_sync(~0u, blocks > 2)) > 2 ? 24 : 2;
    int64_t own = 0;
    auto cost = [&](int position, int n, int b) {
        const int t = tiles_of<KEYS>(p, position, n, b);
        return cut ? (unsigned)(t + cut - 1) / (unsigned)cut : t + over;
    };
    if (blocks <= alone)
#pragma unroll 1
        for (int b = 0; b < blocks; b++) own += cost(position0, rows, b);
    uint32_t together = __ballot_sync(~0u, blocks > alone);
#pragma unroll 1
    while (together) {
        const int src = __ffs(together) - 1;
        together &= together - 1;
        const int n = __shfl_sync(~0u, rows, src), position = __shfl_sync(~0u, position0, src), all = __shfl_sync(~0u, blocks, src);
        int64_t sum = 0;
#pragma unroll 1
        for (int b = lane; b < all; b += 32) sum += cost(position, n, b);
        sum = warp_sum(sum);
        if (lane == src) own = sum;
    }
    return own;
}

// The division of the work, and where this CTA's part begins.  Warps 0 .. warps - 1 take part, each with a stretch of the requests; one of them
// finds the start and leaves it in `start`.
template <int KEYS>
__device__ __forceinline__ Division plan(const PrefillParams& p, Walk& start, int64_t (*sums)[16], int me, int warps, int whole_gain) {
    const int lane = threadIdx.x & 31;
    const int heads = p.pool.n_kv * p.head_tiles, each = (unsigned)(p.n_requests + warps - 1) / (unsigned)warps;
    const int r0 = min(me * each, p.n_requests), r1 = min(r0 + each, p.n_requests);
    int rows = 0, position0 = 0;
    auto enter = [&](int r) {  // this lane's request
        int row0;
        rows = position0 = 0;
        if (r < r1) {
            rows = request_rows(p, r, row0);
            position0 = request_length(p, r) - rows;
        }
    };
    Division d;
    d.cut = 0, d.share = 1;
    int64_t all[2], total = 0;  // tiles and blocks, of one head
#pragma unroll 1
    for (int pass = 0; pass < 2; pass++) {  // tiles; with `cut` also pieces
        int64_t units = 0, blocks = 0;
        int longest = 0;
#pragma unroll 1
        for (int base = r0; base < r1; base += 32) {
            enter(base + lane);
            units += add_blocks<KEYS>(p, rows, position0, pass ? d.cut : 0, 0);
            const int n = blocks_of(p, rows);
            blocks += n;
            if (n > 0) longest = max(longest, tiles_of<KEYS>(p, position0, rows, n - 1));
        }
        units = warp_sum(units), blocks = warp_sum(blocks), longest = __reduce_max_sync(~0u, longest);
        all[0] = units, all[1] = blocks;
        if (warps > 1) {
            __syncthreads();
            if (lane == 0) sums[0][me] = units, sums[1][me] = blocks, sums[2][me] = longest;
            __syncthreads();
            all[0] = all[1] = 0;
#pragma unroll 1
            for (int w = 0; w < warps; w++) all[0] += sums[0][w], all[1] += sums[1][w], longest = max(longest, (int)sums[2][w]);
        }
        if (pass) {
            total = all[0] * heads;
            break;
        }
        // Whole blocks, or pieces that fit the grid, if there are as few blocks and that leaves none much longer than an equal share.
        if (all[1] * heads <= gridDim.x) {
            const int64_t spare = max((int64_t)1, gridDim.x - all[1] * heads), equal = divide(all[0] * heads, gridDim.x);
            d.cut = (int)min((int64_t)1 << 30, max((int64_t)kPieceLeast, divide(all[0] * heads + spare - 1, spare)));
            if (longest <= d.cut + kShareCost) d.cut = max(d.cut, longest);  // whole, if a join costs more
            const bool whole = d.cut >= longest, pieces = whole ? longest <= equal + whole_gain : d.cut <= equal + kShareCost;
            if (whole && pieces && warps == 1) {
                // Every block whole, one a CTA: few numbers, all small.  (The general way takes 4 us, as long as the rest of a small call.)
                const int own = blocks_of(p, rows) * heads;
                int upto = own;
#pragma unroll
                for (int i = 1; i < 32; i <<= 1) {
                    const int x = __shfl_up_sync(~0u, upto, i);
                    if (lane >= i) upto += x;
                }
                const int me_first = blockIdx.x;
                const uint32_t found = __ballot_sync(~0u, upto > me_first);
                d.first = d.end = 0;
                if (found && lane == __ffs(found) - 1) {
                    Block k;
                    const int x = me_first - (upto - own), n = blocks_of(p, rows), head = (unsigned)x / (unsigned)n;
                    k.r = lane, k.b = x - head * n;
                    k.kv = (unsigned)head / (unsigned)p.head_tiles, k.ht = head - k.kv * p.head_tiles;
                    k.rows = request_rows(p, lane, k.row0), k.position0 = position0;
                    enter_block<KEYS>(p, k);
                    start.block = k;
                    start.j = 0, start.left = k.tiles, start.first_unit = 0, start.piece = 0, start.pieces = 1;
                }
                return d;
            }
            if (pieces) continue;
            d.cut = 0;
        }
        total = (all[0] + kOverhead * all[1]) * heads;
        d.share = max((int64_t)1, divide(total + gridDim.x - 1, gridDim.x));
        break;
    }
    const int over = d.cut ? 0 : kOverhead;
    d.first = min(total, (int64_t)blockIdx.x * d.share), d.end = min(total, d.first + d.share);
    if (d.first >= d.end) return d;
    // the warp whose requests hold the first unit looks for it
    int64_t before = 0;
    if (warps > 1) {
#pragma unroll 1
        for (int w = 0; w < me; w++) before += (sums[0][w] + over * sums[1][w]) * heads;
        if (d.first < before || d.first >= before + (sums[0][me] + over * sums[1][me]) * heads) return d;
    }
#pragma unroll 1
    for (int base = r0; base < r1; base += 32) {
        enter(base + lane);
        const int64_t own = add_blocks<KEYS>(p, rows, position0, d.cut, over) * heads;
        int64_t upto = own;
#pragma unroll 1
        for (int i = 1; i < 32; i <<= 1) {
            const int64_t x = __shfl_up_sync(~0u, upto, i);
            if (lane >= i) upto += x;
        }
        const uint32_t found = __ballot_sync(~0u, before + upto > d.first);
        if (found == 0) {
            before += __shfl_sync(~0u, upto, 31);
            continue;
        }
        const int src = __ffs(found) - 1;
        const int64_t per_head = divide(__shfl_sync(~0u, own, src), heads);
        int64_t x = d.first - before - __shfl_sync(~0u, upto - own, src);
        Block k;
        k.r = base + src;
        const int head = (int)divide(x, per_head);
        k.kv = (unsigned)head / (unsigned)p.head_tiles, k.ht = head - k.kv * p.head_tiles;
        x -= head * per_head;
        enter_request(p, k);
        const int blocks = blocks_of(p, k.rows);
#pragma unroll 1
        for (int b0 = 0; b0 < blocks; b0 += 32) {
            const int cost = b0 + lane < blocks ? d.units(tiles_of<KEYS>(p, k.position0, k.rows, b0 + lane)) : 0;
            int64_t sum = cost;
#pragma unroll 1
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
                start.piece = 0, start.pieces = 1;
                if (d.cut) {
                    start.piece = (int)x, start.pieces = units;
                    start.j = (int)divide((int64_t)k.tiles * x, units);
                    start.left = divide((int64_t)k.tiles * (x + 1), units) - start.j;
                    start.first_unit = 0;
                } else {
                    start.j = (int)max((int64_t)0, x - kOverhead);
                    start.left = d.end - d.first - max((int64_t)0, kOverhead - x);
                    start.first_unit = d.first - x + kOverhead;
                }
            }
            return d;
        }
        return d;
    }
    return d;
}

// The next block of the stretch.  (The lengths stay as they are during a call; if they do not, the results are wrong, but nothing beyond the last
// request is read.)
template <int KEYS>
__device__ __forceinline__ bool next_block(const PrefillParams& p, const Division& d, Walk& w) {
    w.left -= w.j_end - w.j + kOverhead;
    if (d.cut || w.left <= 0) return false;
    w.first_unit += w.block.tiles + kOverhead;
    Block& k = w.block;
    if (++k.b * (int64_t)p.tokens_a_block >= k.rows) {
        k.b = 0;
        if (++k.ht >= p.head_tiles) {
            k.ht = 0;
            if (++k.kv >= p.pool.n_kv) {
                k.kv = 0;
                do {
                    if (++k.r >= p.n_requests) return false;
                    enter_request(p, k);
                } while (k.rows == 0);
            }
        }
    }
    enter_block<KEYS>(p, k);
    w.j = 0;
    w.j_end = (int)min((int64_t)k.tiles, w.left);
    return true;
}

// What the warps are told of a run of tiles of one block.
struct Segment {
    int r, kv, ht, row, tokens;      // request, heads, first row in q and how many tokens follow it
    int position, gap, seen;         // of the first row, counted without the gap; the gap; keys
    int j, steps;                    // the first tile, and how many; no steps: the end
    int tiles_in_use;                // tiles of rows
    bool shared, whole;              // one tile of rows, whose tiles of keys the groups of warps take in turn; no other CTA has a part
    int first_part, final_part;      // the CTAs that have
};

// Whether some row of the block does not see some key of a tile: those at or behind `base`.
__device__ __forceinline__ bool partly_seen(const PrefillParams& p, const Segment& k, int base, int keys) {
    const int last = k.position + k.tokens - 1;
    return base + keys - 1 > k.position || (p.window > 0 && max(base, p.first) < min((int64_t)base + keys, (int64_t)last - p.window + 1));
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
    const float2 rest = unpair(add2(pair(a, b), pair(-back.x, -back.y)));
    low = M::pack(rest.x, rest.y);
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

// Whether there are any among eight: bits of the result.
template <class T>
__device__ __forceinline__ uint32_t infinite_among(const uint4& x) {
    constexpr uint32_t kStep = std::is_same<T, F16>::value ? 0x04000400u : 0x00800080u;  // carries into the sign where the exponent is all ones
    return (((x.x & 0x7fff7fffu) + kStep) | ((x.y & 0x7fff7fffu) + kStep) | ((x.z & 0x7fff7fffu) + kStep) | ((x.w & 0x7fff7fffu) + kStep)) & 0x80008000u;
}
// The same as the first for NaN among sixteen 8-bit elements.
__device__ __forceinline__ bool make_finite8(uint4& x) {
    uint32_t* const w = &x.x;
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const uint32_t nan = __vcmpeq4(w[i] & 0x7f7f7f7fu, 0x7f7f7f7fu);
        w[i] &= ~nan;
        any |= nan;
    }
    return any != 0;
}

// ---------------------------------------------------------------------------------------------- the end of a block
// What a row's thread needs to leave its output.
struct Row {
    uint32_t at;       // tensor memory: O of the row
    int row;           // of its tile
    int64_t out;       // row of the output (token and head)
    bool real;         // it is one
    int position, from;  // the last seen key, the first of the window (counted without the gap)
};

// 32 bytes at once where the rows of the output lie so
__device__ __forceinline__ void store32(char* to, const uint32_t (&y)[8], bool aligned) {
    if (aligned)
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(to), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]), "r"(y[4]), "r"(y[5]), "r"(y[6]), "r"(y[7]) : "memory");
    else {
        reinterpret_cast<uint4*>(to)[0] = make_uint4(y[0], y[1], y[2], y[3]);
        reinterpret_cast<uint4*>(to)[1] = make_uint4(y[4], y[5], y[6], y[7]);
    }
}
template <class T>
__device__ __forceinline__ void store_columns(char* out, int D, int64_t out_row, int c, const float (&o)[32], float f, bool none, bool wide = true) {
    char* const to = out + (out_row * D + c * 32) * 2;
    const bool aligned = wide && D % 16 == 0 && ((uintptr_t)out & 31) == 0;
#pragma unroll
    for (int e = 0; e < 2; e++) {
        uint32_t y[8];
#pragma unroll
        for (int i = 0; i < 8; i++) y[i] = none ? 0u : T::pack(o[16 * e + 2 * i] * f, o[16 * e + 2 * i + 1] * f);
        if (c * 32 + e * 16 + 8 < D) store32(to + e * 32, y, aligned);
        else if (c * 32 + e * 16 < D) *reinterpret_cast<uint4*>(to + e * 32) = make_uint4(y[0], y[1], y[2], y[3]);
    }
}

// Tiles that are not seen whole had infinite or NaN elements of v, which were left out of the products: those that this row sees are added to
// its O (tiles t0, t0 + by, .. of the segment).
template <class C, int KEYS>
__device__ __noinline__ void add_infinite(const PrefillParams& p, Row x, const Segment& k, int t0, int by) {
    const int D = p.pool.head_dim;
#pragma unroll 1
    for (int c = 0; c * 16 < D; c++) {
        float o[16];
        tmem_load16(x.at + 16 * c, o);
        wait_loads(o);
        if (x.real)
#pragma unroll 1
            for (int j = k.j + t0; j < k.j + k.steps; j += by) {
                if (!partly_seen(p, k, j * KEYS, KEYS)) continue;
#pragma unroll 1
                for (int u = j * KEYS; u < min(k.seen, (j + 1) * KEYS); u++) {
                    if (u > x.position || (u < x.from && u >= p.first)) continue;
                    const int t = u + (u >= p.kept ? k.gap : 0), i = page_of(p.pool, t), page = p.table[k.r * p.table_row + i];
                    if ((unsigned)page >= (unsigned)p.pool.n_pages) continue;
                    const char* const v = p.pool.v + (page * p.pool.stride_page + (t - i * p.pool.page_size) * p.pool.stride_slot + k.kv * p.pool.stride_head + c * 16) * C::bytes;
#pragma unroll
                    for (int e = 0; e < 8; e++)
                        if (c * 16 + 2 * e < D) {
                            float2 y;
                            if constexpr (C::bytes == 1) y = F16::unpack(E4M3::halves(*reinterpret_cast<const uint16_t*>(v + 2 * e)));
                            else y = C::unpack(*reinterpret_cast<const uint32_t*>(v + 4 * e));
                            if (!(fabsf(y.x) < INFINITY)) o[2 * e] += y.x;
                            if (!(fabsf(y.y) < INFINITY)) o[2 * e + 1] += y.y;
                        }
                }
            }
        __syncwarp();  // (lanes that are not here yet would lose registers to the next load from tensor memory)
        uint32_t y[16];
#pragma unroll
        for (int e = 0; e < 16; e++) y[e] = __float_as_uint(o[e]);
        tmem_store16(x.at + 16 * c, y);
    }
    wait_stores();
}

// What a row's O has summed up goes to `aside`, laid out like a part, and O begins again at zero; `again`: onto what is there already, which stands for
// the reference that it had.  (A row without a finite logit so far keeps its O.)
template <int DP>
__device__ __forceinline__ void put_aside_here(uint32_t at, float* aside, int row, int D, float add, bool again) {
    float* const reference = aside + DP * 128 + row;
    const float before = again ? *reference : INFINITY, f = before == INFINITY ? 0.0f : power2(add - before);
#pragma unroll 1
    for (int c = 0; c * 16 < D; c++) {
        float o[16];
        tmem_load16(at + 16 * c, o);
        wait_loads(o);
        uint32_t y[16];
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            float4* const to = reinterpret_cast<float4*>(aside) + (c * 4 + e / 4) * 128 + row;
            float4 z = make_float4(0, 0, 0, 0);
            if (before != INFINITY) z = *to;
            *to = make_float4(z.x * f + o[e], z.y * f + o[e + 1], z.z * f + o[e + 2], z.w * f + o[e + 3]);
        }
        __syncwarp();  // (as above)
#pragma unroll
        for (int e = 0; e < 16; e++) y[e] = add == INFINITY ? __float_as_uint(o[e]) : 0u;
        tmem_store16(at + 16 * c, y);
    }
    *reference = add;
    wait_stores();
}
template <int DP>
__device__ __noinline__ void put_aside(uint32_t at, float* aside, int row, int D, float add, bool again) { put_aside_here<DP>(at, aside, row, D, add, again); }
// And back again, at the end of the walk.
template <int DP>
__device__ __noinline__ void take_back(uint32_t at, const float* aside, int row, int D, float add) {
    const float before = aside[DP * 128 + row], f = before == INFINITY ? 0.0f : power2(add - before);
#pragma unroll 1
    for (int c = 0; c * 16 < D; c++) {
        float o[16];
        tmem_load16(at + 16 * c, o);
        wait_loads(o);
        uint32_t y[16];
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            float4 z = make_float4(0, 0, 0, 0);
            if (before != INFINITY) z = reinterpret_cast<const float4*>(aside)[(c * 4 + e / 4) * 128 + row];
            y[e] = __float_as_uint(z.x * f + o[e]), y[e + 1] = __float_as_uint(z.y * f + o[e + 1]);
            y[e + 2] = __float_as_uint(z.z * f + o[e + 2]), y[e + 3] = __float_as_uint(z.w * f + o[e + 3]);
        }
        __syncwarp();  // (as above)
        tmem_store16(at + 16 * c, y);
    }
    wait_stores();
}

// O of a row, 32 columns of tensor memory at a time, to the output or to a part.  `with`: columns from there to a second O, or none; the sum
// of both, times f1 and f2, is what leaves (either may be anything where its factor is zero).
template <class T>
__device__ __forceinline__ void leave(const PrefillParams& p, const Row& x, float* part, float f, bool none, int with, float f1, float f2) {
#pragma unroll 1
    for (int c = 0; c * 32 < p.pool.head_dim; c++) {
        float o[32];
        tmem_load(x.at + 32 * c, o);
        wait_loads(o);
        if (with)
#pragma unroll
            for (int h = 0; h < 2; h++) {
                float y[16];
                tmem_load16(x.at + with + 32 * c + 16 * h, y);
                wait_loads(y);
#pragma unroll
                for (int e = 0; e < 16; e++) o[16 * h + e] = (f1 == 0.0f ? 0.0f : o[16 * h + e] * f1) + (f2 == 0.0f ? 0.0f : y[e] * f2);
            }
        if (part) {  // fours of columns
#pragma unroll
            for (int e = 0; e < 32; e += 4) reinterpret_cast<float4*>(part)[(c * 8 + e / 4) * 128 + x.row] = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
        } else if (x.real)
            store_columns<T>(p.out, p.pool.head_dim, x.out, c, o, f, none);
        __syncwarp();  // (as above)
    }
}

// A row's log-sum-exp from the sum of its weights 2^(logit + add).
__device__ __forceinline__ void leave_lse(float* lse, int64_t out, float sum, float add) {
    if (lse) lse[out] = sum == 0.0f ? -INFINITY : logf(sum) - add * 0.6931471805599453f;
}

// Adds up the parts of a block's tile, in their order: references, sums and outputs of each; of row `at` a thread, 32 columns of every `by` times 32, from
// `c0` times 32 on (few rows are shared by the warps).  The first is at `first`, the others of
// `n` from `rest` on, `stride` floats apart.  (All that it is told comes in registers.  What is passed by its address lies in memory, and with the shared memory that this kernel takes there is next to no
// cache before L2: a join of 16 parts took 70 us that way.)
template <class T, int DP>
__device__ __noinline__ void join(char* out, float* lse, int D, int at, int64_t out_row, bool real, const float* first, const float* rest, int64_t stride, int n, int c0,
                                  int by, float vscale) {
    auto part = [&](int x) { return x == 0 ? first : rest + (x - 1) * stride; };
    // What can be asked for at once is.
    constexpr int kMost = 8;
    float add[kMost], least = INFINITY, all = 0;  // references as numbers to add; the least is the highest reference
#pragma unroll 1
    for (int x0 = 0; x0 < n; x0 += kMost) {
        float sum[kMost];
#pragma unroll
        for (int x = 0; x < kMost; x++) {
            const float* const from = part(min(x0 + x, n - 1)) + DP * 128 + at;
            add[x] = __ldcg(from), sum[x] = __ldcg(from + 128);
        }
        const float before = least;
#pragma unroll
        for (int x = 0; x < kMost; x++) {
            if (x0 + x >= n) add[x] = INFINITY, sum[x] = 0;
            least = fminf(least, add[x]);
        }
        all *= before == INFINITY ? 0.0f : power2(least - before);
#pragma unroll
        for (int x = 0; x < kMost; x++) all += (add[x] == INFINITY ? 0.0f : power2(least - add[x])) * sum[x];
    }
    const float f = all == 0.0f ? 0.0f : vscale / all;
    if (n <= kMost) {
#pragma unroll
        for (int x = 0; x < kMost; x++) add[x] = add[x] == INFINITY ? 0.0f : power2(least - add[x]);  // now factors
    }
#pragma unroll 1
    for (int c = c0; c * 32 < D; c += by) {
        float o[32] = {};
#pragma unroll 1
        for (int x0 = 0; x0 < n; x0 += kMost) {
            if (n > kMost) {
#pragma unroll
                for (int x = 0; x < kMost; x++) {
                    const float a = x0 + x < n ? __ldcg(part(x0 + x) + DP * 128 + at) : INFINITY;
                    add[x] = a == INFINITY ? 0.0f : power2(least - a);
                }
            }
#pragma unroll
            for (int x1 = 0; x1 < kMost; x1 += 2) {
                if (x0 + x1 >= n) break;
                float4 z[2][8];
#pragma unroll
                for (int x = 0; x < 2; x++) {
                    const float4* const from = reinterpret_cast<const float4*>(part(min(x0 + x1 + x, n - 1))) + c * 1024 + at;
#pragma unroll
                    for (int e = 0; e < 8; e++) z[x][e] = __ldcg(from + e * 128);
                }
#pragma unroll
                for (int x = 0; x < 2; x++) {
                    const float y = add[x1 + x];
                    if (y == 0.0f) continue;  // (a part without a tile has no output, but what was there before)
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        float* const to = o + 4 * e;
                        to[0] += y * z[x][e].x, to[1] += y * z[x][e].y, to[2] += y * z[x][e].z, to[3] += y * z[x][e].w;
                    }
                }
            }
        }
        // (16 bytes at once: of 32, in a function that two kernels call, this compiler (12.9.86) stores the first 4)
        if (real) store_columns<T>(out, D, out_row, c, o, f, all == 0.0f, false);
    }
    if (real && c0 == 0) leave_lse(lse, out_row, all, least);
}

// A wait of a warp that ends: false when the time is up, and then for every other wait of the CTA too.  (One function for each side of the kernel:
// they have different numbers of registers.)
template <int SIDE>
__device__ __noinline__ bool wait_long(uint32_t bar, uint32_t parity, volatile int* stuck, int32_t* status) {
    constexpr int64_t kPatience = 4000000000ll;  // cycles: seconds, where microseconds are usual
    const int64_t began = clock64();
    bool done = false;
    while (!(done = bar_sleep(bar, parity, 100000))) {
        if (*stuck) break;
        if (clock64() - began > kPatience) {
            *stuck = 1;
            flag(status, FCSIM_KV_STUCK);
            break;
        }
    }
    return (bool)__all_sync(~0u, done);
}

// ---------------------------------------------------------------------------------------------- the kernel
// LONG: walks of more than kAsideTiles tiles.  (Kernels of their own, so that other calls take what they took: 8 192 tokens of width 64 574 us with it and 561
// without.  Width 128: 661 and 691 of 16 bits, 985 and 924 of 8, within what repeats differ by; there a call of the function costs 2 % more than the
// function in place, with 16 bits it is the other way around.)
template <class T, class C, int DP, bool LONG>
__global__ void __launch_bounds__(Shape<T, C, DP>::kThreads, 1) fcsim_kv_prefill_kernel(const __grid_constant__ PrefillParams p) {
    using S = Shape<T, C, DP>;
    constexpr int kTiles = S::kTiles, kKeys = S::kKeys, kStages = S::kStages, kSegments = 4;
    constexpr bool kNarrow = C::bytes == 1;
    constexpr float kRaise = kRaiseOf<T>, kLag = kLagOf<T>, kLog2e = 1.4426950408889634f;
    extern __shared__ __align__(1024) char raw_smem[];
    __shared__ __align__(8) uint64_t bars[2 * kStages + 2 * kSegments + 14 + 2 * S::kLoadWarps];
    __shared__ float2 others[kTiles == 2 ? 128 : 1];
    __shared__ uint32_t tmem_at, valid[8][4];
    __shared__ int stuck, infinite[kSegments], joins[kTiles];
    __shared__ Walk start;
    __shared__ Segment segments[kSegments];
    __shared__ int64_t sums[3][16];

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int D = p.pool.head_dim, group = p.n_heads / p.pool.n_kv;
    const uint32_t smem = smem_address(raw_smem), query = smem, ring = smem + S::kQuery;
    const uint32_t bar0 = smem_address(bars);
    auto full = [&](int s) { return bar0 + s * 8; };
    auto empty = [&](int s) { return bar0 + (kStages + s) * 8; };
    auto told_of = [&](int s) { return bar0 + (2 * kStages + s) * 8; };               // of a segment
    auto done_with = [&](int s) { return bar0 + (2 * kStages + kSegments + s) * 8; };
    const uint32_t rest = bar0 + (2 * kStages + 2 * kSegments) * 8;
    auto score_full = [&](int s) { return rest + s * 8; };
    auto weights_ready = [&](int s) { return rest + 16 + s * 8; };
    auto output_full = [&](int s) { return rest + 32 + s * 8; };
    auto meeting = [&](int i) { return rest + 48 + i * 8; };
    auto landed = [&](int me, int turn) { return rest + 112 + (me * 2 + turn) * 8; };  // a warp's bulk copies that it looks over
    const uint32_t query_full = rest + 64, query_empty = rest + 72, added = rest + 80, drained = rest + 88;
    const uint32_t other_ready = rest + 96, other_taken = rest + 104;  // the second group's output of a tile that both have, for the first
    auto wait_on = [&](auto side, uint32_t bar, uint32_t parity) {
        return __all_sync(~0u, bar_try(bar, parity)) || wait_long<decltype(side)::value>(bar, parity, &stuck, p.status);
    };

    constexpr int kProductWarp = S::kWarps - 2, kPlanWarp = S::kWarps - 1;
    {
        // how many arrivals each of the barriers, in the order in which they lie, waits for
        constexpr int kBars = 2 * kStages + 2 * kSegments + 14 + 2 * S::kLoadWarps;
        if (tid < kBars) {
            const int i = tid - 2 * kStages - 2 * kSegments;
            int count = 1;
            if (tid < kStages) count = 64;                                                        // full
            else if (tid >= 2 * kStages + kSegments && i < 0) count = S::kWarps - 1;              // done_with
            else if ((i >= 2 && i < 4) || (i >= 6 && i < 8) || (i >= 12 && i < 14)) count = 128;  // weights_ready, meeting, other_ready, other_taken
            else if (i == 8) count = p.box ? 1 : 32 * S::kLoadWarps;                              // query_full
            bar_init(bar0 + tid * 8, count);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        if (tid == 0) stuck = 0, start.left = 0;
    }
    if (warp == kProductWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_address(&tmem_at)), "r"(S::kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (D % 16 != 0) {  // the products read elements by 16: what is beyond head_dim is zero, and stays so
        const int chunk = D / 8;
        auto clear = [&](uint32_t at, int rows, int tall) {
#pragma unroll 1
            for (int i = tid; i < rows; i += S::kThreads) {
                const uint32_t tile = at + i / tall * (tall * DP * 2);
                const int row = i % tall;
                store16(tile + chunk / 8 * (tall * 128) + row * 128 + ((chunk % 8) ^ (row % 8)) * 16, make_uint4(0, 0, 0, 0));
            }
        };
        clear(query, S::kRows, S::kRows);
        clear(ring, kStages * kKeys, kKeys);
        fence_for_products();
    }
    Division work;
    if (p.n_requests > kOneWarpPlans) {
        __syncthreads();  // (start.left)
        work = plan<kKeys>(p, start, sums, warp, S::kWarps, kWholeGain<C, DP>);
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = tmem_at;
    const int heads_a_tile = p.heads_a_tile;
    int segment = 0;
    bool fine = true;
    // the next segment; false at the end
    auto next_segment = [&](auto& wait) {
        if (!(fine = wait(told_of(segment % kSegments), segment / kSegments & 1))) return false;
        return segments[segment % kSegments].steps > 0;
    };
    auto leave_segment = [&]() {
        __syncwarp();
        if (lane == 0) bar_arrive(done_with(segment % kSegments));
        segment++;
    };

    // (each side leaves or takes its registers in a branch of its own: what comes before both is compiled for the fewer)
    if (warp < S::kSoftmaxWarps) {
        if constexpr (kTiles == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::kSoftmaxRegisters));
        auto wait = [&](uint32_t bar, uint32_t parity) { return wait_on(std::integral_constant<int, 0>(), bar, parity); };
        // ------------------------------------------------------------------------------------------ softmax
        // rows that belong to no request, and what is wrong with the requests
        {
            constexpr int kHere = 32 * S::kSoftmaxWarps;
            const int n0 = p.n_requests > 0 ? min(max(p.starts[0], 0), p.n_rows) : p.n_rows;
            const int n1 = p.n_requests > 0 ? min(max(p.starts[p.n_requests], n0), p.n_rows) : p.n_rows, none = p.n_rows - n1 + n0;
            if (none > 0) {
                const int64_t per_row = (int64_t)p.n_heads * (D / 8);
#pragma unroll 1
                for (int64_t i = (int64_t)blockIdx.x * kHere + tid; i < none * per_row; i += (int64_t)gridDim.x * kHere)
                    reinterpret_cast<uint4*>(p.out)[i < n0 * per_row ? i : i + (n1 - n0) * per_row] = make_uint4(0, 0, 0, 0);
                if (p.lse)
#pragma unroll 1
                    for (int64_t i = (int64_t)blockIdx.x * kHere + tid; i < (int64_t)none * p.n_heads; i += (int64_t)gridDim.x * kHere)
                        p.lse[i < (int64_t)n0 * p.n_heads ? i : i + (int64_t)(n1 - n0) * p.n_heads] = -INFINITY;
            }
#pragma unroll 1
            for (int r = blockIdx.x * kHere + tid; r < p.n_requests; r += gridDim.x * kHere) {
                const int a = p.starts[r], b = p.starts[r + 1], n = p.lengths[r];
                if (n < 0 || n > p.max_length || a < 0 || b < a || b > p.n_rows || b - a > n) flag(p.status, FCSIM_KV_BAD_LENGTH);
            }
        }
        const int i = warp >> 2;  // tile
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // this warp's lanes of tensor memory: 32 (warp % 4) << 16
        Row x;
        x.row = tid & 127;
        x.at = tmem + S::kOutput + i * DP + lanes;
        // token and head of the row, in a tile of its own or where both groups have the first
        const int token_own = (uint32_t)tid / (uint32_t)heads_a_tile, g_own = tid - token_own * heads_a_tile;
        const int token_first = (uint32_t)x.row / (uint32_t)heads_a_tile, g_first = x.row - token_first * heads_a_tile;
        int step0 = 0;
        uint32_t score_parity[2] = {0, 0}, output_parity = 0, meeting_parity = 0, other_parity = 0;
        auto meet = [&]() {
            bar_arrive(meeting(i));
            const bool ok = wait(meeting(i), meeting_parity);
            meeting_parity ^= 1;
            return ok;
        };
        constexpr int64_t kPart = (int64_t)(DP + 2) * 128;
        auto aside = [&]() { return p.parts + ((2 * (int64_t)gridDim.x + blockIdx.x) * kTiles + i) * kPart; };  // (there is room where a walk may be so long)
        while (next_segment(wait)) {
            const Segment& k = segments[segment % kSegments];
            const int steps = k.steps;
            const bool shared = k.shared, whole = k.whole;
            const int step_first = shared ? i : i >= k.tiles_in_use ? steps : 0, step_by = shared ? 2 : 1;
            const bool worked = step_first < steps;
            if (worked || shared) {
                const int token = shared ? token_first : token_own, head = k.ht * heads_a_tile + (shared ? g_first : g_own);
                x.real = token < k.tokens && head < group;
                x.out = (int64_t)(k.row + token) * p.n_heads + k.kv * group + head;
                // A warp without a real row leaves the scores as they are for its weights: what becomes of them is nobody's output.
                const bool idle = !__any_sync(~0u, x.real);
                // (never zero, so that what is not seen, a logit of -infinity, stays without weight: 2^-149 times the largest logit is 5e-7)
                float unit = fabsf(kNarrow ? p.scale * p.pool.k_scale[k.kv] : p.scale) * kLog2e;
                if (unit < 1.4e-45f) unit = 1.4e-45f;
                // the last seen key of this row and the first of its window; nothing for rows that are none
                x.position = x.real ? k.position + token : -1;
                x.from = p.window > 0 && x.position >= p.window ? x.position - p.window + 1 : 0;
                float add = INFINITY, limit = -INFINITY, sum = 0;  // weights are 2^(unit s + add); add is infinite until there is a finite logit
                int t0 = step_first;
                do {
                    if (LONG && t0 >= kAsideTiles) {
                        const int slot = kTiles == 2 ? i : t0 & 1;
                        if (!(fine = wait(score_full(slot), score_parity[slot]) && (kTiles == 2 || wait(added, (step0 + t0 - 1) & 1)))) break;
                        fence_after_sync();
                        if (!idle) {
                            if constexpr (kNarrow) put_aside_here<DP>(x.at, aside(), x.row, D, add, t0 >= 2 * kAsideTiles);
                            else put_aside<DP>(x.at, aside(), x.row, D, add, t0 >= 2 * kAsideTiles);
                        }
                    }
                    const int t_end = LONG ? min(steps, t0 + kAsideTiles) : steps;
#pragma unroll 1
                    for (int t = t0; t < t_end; t += step_by) {
                        const int slot = kTiles == 2 ? i : t & 1, tile_base = (k.j + t) * kKeys;
                        const uint32_t at = tmem + S::kScore + slot * kKeys + lanes;
                        const bool edge = partly_seen(p, k, tile_base, kKeys);
                        if (!(fine = wait(score_full(slot), score_parity[slot]))) break;
                        score_parity[slot] ^= 1;
                        fence_after_sync();
                        if (idle) {
                            fence_before_sync();
                            bar_arrive(weights_ready(slot));
                            continue;
                        }
                        const uint32_t* const there = valid[(step0 + t) & 7];
                        uint32_t some = ~0u;
#pragma unroll
                        for (int c = 0; c < kKeys / 32; c++) some &= there[c];
                        const bool masked = edge || some != ~0u;
                        auto load = [&](int c, float (&s)[4][16]) {  // 64 logits; those that are not seen are -infinity
#pragma unroll
                            for (int e = 0; e < 4; e++) tmem_load16(at + c * 64 + 16 * e, s[e]);
                            wait_loads(s[0], s[1], s[2], s[3]);
                            if (masked) {
#pragma unroll
                                for (int y = 0; y < 2; y++) {
                                    const int b = tile_base + 64 * c + 32 * y;
                                    const uint32_t mask = lowest(x.position + 1 - b) & (~lowest(x.from - b) | lowest(p.first - b)) & there[2 * c + y];
#pragma unroll
                                    for (int e = 0; e < 32; e++) s[2 * y + e / 16][e % 16] = mask >> e & 1 ? s[2 * y + e / 16][e % 16] : -INFINITY;
                                }
                            }
                        };
                        float top = -INFINITY;
#pragma unroll 1
                        for (int c = 0; c < kKeys / 64; c++) {
                            float s[4][16];
                            load(c, s);
                            float tops[4] = {top, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                            for (int e = 0; e < 64; e += 2) tops[e / 2 % 4] = fmaxf(fmaxf(tops[e / 2 % 4], s[e / 16][e % 16]), s[e / 16][e % 16 + 1]);
                            top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
                        }
                        const float most = top * unit;
                        // The reference moves only when a logit is 2^kLag above it, so that the output is seldom taken through registers.
                        const bool moves = most > limit;
                        if (__any_sync(~0u, moves)) {
                            float shrink = 1;
                            if (moves) {
                                const float now = kRaise - most;
                                shrink = limit == -INFINITY ? 0.0f : power2(now - add);
                                add = now;
                                limit = most + kLag;
                                sum *= shrink;
                            }
                            __syncwarp();  // (a warp that has come apart must not load from tensor memory: what comes is written to all lanes' registers)
                            if (t > step_first) {
                                if (kTiles == 1 && !(fine = wait(added, (step0 + t - 1) & 1))) break;
                                fence_after_sync();
#pragma unroll 1
                                for (int c = 0; c * 32 < D; c++) {
                                    float o[2][16];
                                    tmem_load16(x.at + 32 * c, o[0]);
                                    tmem_load16(x.at + 32 * c + 16, o[1]);
                                    wait_loads(o[0], o[1]);
#pragma unroll
                                    for (int h = 0; h < 2; h++) {
                                        uint32_t y[16];
#pragma unroll
                                        for (int e = 0; e < 16; e++) y[e] = __float_as_uint(o[h][e] * shrink);
                                        tmem_store16(x.at + 32 * c + 16 * h, y);
                                    }
                                }
                            }
                        }
                        const float plus = limit == -INFINITY ? 0.0f : add;
                        const uint64_t unit2 = pair(unit, unit), plus2 = pair(plus, plus);
                        uint64_t sums2[2] = {pair(0.0f, 0.0f), pair(0.0f, 0.0f)};  // of this tile: the row's total takes one rounding of each
#pragma unroll 1
                        for (int c = 0; c < kKeys / 64; c++) {
                            float s[4][16];
                            load(c, s);
#pragma unroll
                            for (int h = 0; h < 4; h++) {
                                uint32_t y[16];
#pragma unroll
                                for (int e = 0; e < 8; e++) {
                                    const float2 z = unpair(fma2(pair(s[h][2 * e], s[h][2 * e + 1]), unit2, plus2));
                                    const float a = power2(z.x), b = power2(z.y);
                                    sums2[e & 1] = add2(sums2[e & 1], pair(a, b));
                                    split<T>(a, b, y[e], y[8 + e]);
                                }
                                tmem_store16(at + c * 64 + 16 * h, y);
                            }
                        }
                        const float2 z = unpair(add2(sums2[0], sums2[1]));
                        sum += z.x + z.y;
                        wait_stores();
                        fence_before_sync();
                        bar_arrive(weights_ready(slot));
                    }
                    t0 += kAsideTiles;
                } while (LONG && fine && t0 < steps);
                if (!fine) break;
                // -------------------------------------------------------------- end of this CTA's part of a block
                if (worked) {
                    if (!(fine = wait(output_full(i), output_parity))) break;
                    output_parity ^= 1;
                    fence_after_sync();
                }
                if (LONG && step_first + kAsideTiles < steps && !idle) take_back<DP>(x.at, aside(), x.row, D, add);
                if (worked && !idle && infinite[segment % kSegments]) add_infinite<C, kKeys>(p, x, k, step_first, step_by);
                float f1 = 1, f2 = 0;
                if (kTiles == 2 && shared) {
                    if (i == 1) {  // the first group takes this one's output with its own
                        others[x.row] = make_float2(add, sum);
                        fence_before_sync();
                        bar_arrive(other_ready);
                        if (!(fine = wait(other_taken, other_parity))) break;
                    } else {
                        if (!(fine = wait(other_ready, other_parity))) break;
                        const float2 other = others[x.row];
                        const float least = fminf(add, other.x);
                        f1 = add == INFINITY ? 0.0f : power2(least - add), f2 = other.x == INFINITY ? 0.0f : power2(least - other.x);
                        sum = f1 * sum + f2 * other.y, add = least;  // (NaN stays NaN)
                    }
                    other_parity ^= 1;
                    fence_after_sync();
                }
                if (!(kTiles == 2 && shared && i == 1)) {
                    const float vscale = kNarrow ? p.pool.v_scale[k.kv] : 1.0f, f = sum == 0.0f ? 0.0f : vscale / sum;
                    // this CTA's part is the first of its two, unless the block begins here
                    float* const part = whole ? nullptr : p.parts + ((2 * (int64_t)blockIdx.x + (k.first_part == (int)blockIdx.x ? 1 : 0)) * kTiles + i) * kPart;
                    if (!idle) leave<T>(p, x, part, f, sum == 0.0f, kTiles == 2 && shared ? DP : 0, f1, f2);
                    fence_before_sync();
                    if (kTiles == 2 && shared) bar_arrive(other_taken);
                    if (whole) {
                        if (x.real) leave_lse(p.lse, x.out, sum, add);
                    } else {
                        if (!idle) {
                            part[DP * 128 + x.row] = add;
                            part[(DP + 1) * 128 + x.row] = sum;
                            __threadfence();
                        }
                        if (!(fine = meet())) break;
                        if (x.row == 0) {
                            int* const counter = p.counters + k.first_part * 2 + i;
                            const bool last = atomicAdd(counter, 1) == k.final_part - k.first_part;
                            joins[i] = last;
                            if (last) *counter = 0;
                        }
                        if (!(fine = meet())) break;
                        if (joins[i]) {
                            __threadfence();
                            const float* const first = p.parts + ((2 * (int64_t)k.first_part + 1) * kTiles + i) * kPart;
                            // one, two or four warps for the rows, and so four, two or one for the columns
                            const int rows = k.tokens * heads_a_tile - 128 * i, row_warps = rows <= 32 ? 1 : rows <= 64 ? 2 : 4, w = warp & 3;
                            const int at = w % row_warps * 32 + lane, token = (uint32_t)(at + 128 * i) / (uint32_t)heads_a_tile;
                            const int head = k.ht * heads_a_tile + at + 128 * i - token * heads_a_tile;
                            const bool real = token < k.tokens && head < group;
                            if (__any_sync(~0u, real))
                                join<T, DP>(p.out, p.lse, D, at, (int64_t)(k.row + token) * p.n_heads + k.kv * group + head, real, first, first + kTiles * kPart, 2 * kTiles * kPart,
                                            k.final_part - k.first_part + 1, w / row_warps, 4 / row_warps, vscale);
                        }
                    }
                }
            }
            step0 += steps;
            leave_segment();
        }
    } else {
        if constexpr (kTiles == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::kOtherRegisters));
        auto wait = [&](uint32_t bar, uint32_t parity) { return wait_on(std::integral_constant<int, 1>(), bar, parity); };
        if (warp == kPlanWarp) {
            // ------------------------------------------------------------------------------------------ the walk
            if (p.n_requests <= kOneWarpPlans) work = plan<kKeys>(p, start, sums, 0, 1, kWholeGain<C, DP>);
            __syncwarp();
            Walk w = start;
            bool more = w.left > 0;
            if (more) w.j_end = (int)min((int64_t)w.block.tiles, w.j + w.left);
            while (true) {
                const int s = segment % kSegments;
                if (segment >= kSegments && !wait(done_with(s), (segment / kSegments - 1) & 1)) break;
                if (lane == 0) {
                    Segment& k = segments[s];
                    k.steps = 0;
                    if (more) {
                        const Block& b = w.block;
                        const int at = b.b * p.tokens_a_block;
                        k.r = b.r, k.kv = b.kv, k.ht = b.ht, k.row = b.row0 + at, k.tokens = b.tokens;
                        k.position = b.position0 + at - b.gap, k.gap = b.gap, k.seen = b.seen;
                        k.j = w.j, k.steps = w.j_end - w.j;
                        k.tiles_in_use = kTiles == 2 && b.tokens * heads_a_tile > 128 ? 2 : 1;
                        k.whole = w.j == 0 && w.j_end == b.tiles;
                        k.shared = kTiles == 2 && k.tiles_in_use == 1 && (!k.whole || k.steps >= kSharedLeast);
                        k.first_part = k.final_part = blockIdx.x;
                        if (!k.whole) {
                            if (work.cut) {
                                k.first_part -= w.piece;
                                k.final_part = k.first_part + w.pieces - 1;
                            } else {
                                if (w.first_unit < work.first) k.first_part = (int)divide(w.first_unit, work.share);
                                if (w.first_unit + b.tiles > work.end) k.final_part = (int)divide(w.first_unit + b.tiles - 1, work.share);
                            }
                        }
                    }
                    infinite[s] = 0;
                    bar_arrive(told_of(s));
                }
                segment++;
                if (!more) break;
                more = next_block<kKeys>(p, work, w);
            }
        } else if (warp == kProductWarp) {
            // ------------------------------------------------------------------------------------------ products
            constexpr uint32_t kType = std::is_same<T, F16>::value ? 0 : 1;
            const uint32_t depth = uni((D + 15) / 16), base = uni(tmem);
            const uint32_t how_output = instruction(kType, true, 128, depth * 16);
            const uint64_t query_operand = operand(uni(query), 16, 1024), key_operand = operand(uni(ring), 16, 1024), value_operand = operand(uni(ring), kKeys * 128, 1024);
            // What decides the way through the loop is in registers of the warp, and few instructions stand between a wait and the products that
            // it lets go: with 200 clocks of them for each tile the tensor core stood idle 40 % of the time.
            uint32_t stage = 0, phase = 0, ready = 0;  // of the ring: the next tile; parities of the weights, a bit each
            uint32_t key_stage = 0, value_stage = 0;
            auto next_tile = [&](uint32_t& at) {  // the next tile of the ring is there
                if (!wait(full(stage), phase)) return false;
                fence_after_sync();
                at = stage;
                if (++stage == kStages) stage = 0, phase ^= 1;
                return true;
            };
            while (next_segment(wait)) {
                const Segment& k = segments[segment % kSegments];
                const uint32_t steps = uni(k.steps), n = uni(k.tiles_in_use);
                // With two tiles of rows, tile after tile: the output of a step, then the scores of the next (K0 V0 K1 V1 ..).  With one, the scores
                // run a step ahead, in the two areas in turn (K0 K1 V0 K2 V1 ..).  Both are a row of outputs, each followed by the scores of the
                // output `lead` later.
                const uint32_t ahead = kTiles == 1 ? 1u : uni(k.shared), both = 1 - ahead & n - 1;
                const uint32_t outputs = steps << both, lead = ahead ? min(2u, steps) : n;
                // a negative scale turns the order of the logits around: Q is taken as -Q instead
                const float scale = kNarrow ? p.scale * p.pool.k_scale[k.kv] : p.scale;
                const uint32_t how_score = instruction(kType, false, 128, kKeys) | uni(scale < 0) << 13;
                if (!(fine = wait(query_full, segment & 1))) break;
#pragma unroll 1
                for (uint32_t q = 0; q < outputs + lead; q++) {  // scores of output q, behind the products of output q - lead
                    if (q >= lead) {
                        const uint32_t w = q - lead, i = ahead ? w & 1 : w & both;
                        if ((!both || i == 0) && !(fine = next_tile(value_stage))) break;
                        const uint32_t o = kTiles == 1 ? 0 : i, j = w >> both, more_of = j >= (kTiles == 2 && ahead ? 2 : 1);
                        const uint32_t to = base + S::kOutput + o * DP, from = base + S::kScore + i * kKeys;
                        const uint64_t b = value_operand + value_stage * (S::kStage >> 4);
                        if (!(fine = wait(weights_ready(i), ready >> i & 1))) break;
                        ready ^= 1u << i;
                        fence_after_sync();
                        if (elected()) {
#pragma unroll
                            for (int y = 0; y < kKeys / 16; y++)
#pragma unroll
                                for (int part = 0; part < 2; part++)
                                    product_from_tmem(to, from + y * 16 + part * 8, b + (y * 2048 >> 4), how_output, part > 0 || y > 0 ? 1u : more_of);
                            if (!both || i == 1) commit_products(empty(value_stage));
                            if (kTiles == 1) commit_products(added);
                            if (kTiles == 2 && ahead ? w + 2 >= outputs : j + 1 == steps) commit_products(output_full(o));
                        }
                    }
                    if (q < outputs) {
                        const uint32_t i = ahead ? q & 1 : q & both;
                        if ((!both || i == 0) && !(fine = next_tile(key_stage))) break;
                        const uint32_t to = base + S::kScore + i * kKeys;
                        const uint64_t a = query_operand + (ahead ? 0 : i) * (128 * 128 >> 4), b = key_operand + key_stage * (S::kStage >> 4);
                        if (elected()) {
#pragma unroll
                            for (int y = 0; y < DP / 16; y++)
                                if (y < depth) product(to, a + ((y / 4 * (S::kRows * 128) + y % 4 * 32) >> 4), b + ((y / 4 * (kKeys * 128) + y % 4 * 32) >> 4), how_score, y > 0);
                            commit_products(score_full(i));
                            if (!both || i == 1) commit_products(empty(key_stage));
                            if (q + 1 == outputs) commit_products(query_empty);
                        }
                    }
                }
                if (!fine) break;
                leave_segment();
            }
            if (elected()) commit_products(drained);  // nothing is in flight when the CTA ends
            const int64_t began = clock64();
            while (!bar_try(drained, 0) && clock64() - began < 4000000000ll) {}
        } else if (warp >= S::kSoftmaxWarps) {
            // ------------------------------------------------------------------------------------------ loads
            // Halves of the tiles of K and V in the order in which they are used, one after the other to these warps.  A warp keeps two on their
            // way: it waits for the copies of one when those of the next are asked for, unless there is no place yet for the next.
            const int me = warp - S::kSoftmaxWarps;
            constexpr int kLanes = DP * C::bytes / 16, kAtOnce = 32 / kLanes, kHalf = kKeys / 2, kRounds = kHalf / kAtOnce;  // lanes of a row, rows at once
            constexpr int kOffs = kHalf / 32;
            const int chunk = lane % kLanes, lane_row = lane / kLanes, chunks = D * C::bytes / 16;
            const bool copies = chunk < chunks;
            const uint32_t token_magic = (65536 + heads_a_tile - 1) / heads_a_tile;  // row / heads_a_tile for rows below 256
            int tile0 = 0, step0 = 0;  // tiles and steps of the segments before this one
            // Place in a stage of 16 bytes of a row.  8-bit rows come into the upper half of the place of a row, 16 bytes to where 8 elements will be, and become
            // 16-bit ones from there.
            auto place = [&](int row, int at) { return (uint32_t)(at / 8 * (kKeys * 128) + row * 128 + ((at % 8) ^ (row % 8)) * 16); };
            constexpr int kRaw = kNarrow ? DP / 16 : 0;
            uint32_t landed_parity = 0, turn = 0;  // of the two barriers, a bit each; the next
            // 8-bit rows are turned by eight lanes that take four pieces each of rows r and r ^ 5: so both what they read and what they write lies in all
            // banks.  The places of a lane's pieces, as they were and as they will be, for the first rows; the others follow 8 rows apart.
            constexpr int kGroups = kLanes < 4 ? 1 : kLanes / 4, kPairs = 4 / kGroups, kBases = kGroups;
            const int turned_chunk = (lane >> 3) % kGroups * 4 + (lane & 3), swap = lane & 4 ? 5 : 0;
            auto turned_row = [&](int i) {
                const int pair = i * kPairs + (lane >> 3) / kGroups;
                return pair / 4 * 8 + (pair % 4 ^ swap);
            };
            uint32_t place_raw[kBases], place_low[kBases], place_high[kBases];
            if constexpr (kNarrow)
#pragma unroll
                for (int i = 0; i < kBases; i++) {
                    place_raw[i] = place(turned_row(i), kRaw + turned_chunk);
                    place_low[i] = place(turned_row(i), 2 * turned_chunk), place_high[i] = place(turned_row(i), 2 * turned_chunk + 1);
                }
            while (next_segment(wait)) {
                const Segment& k = segments[segment % kSegments];
                const int steps = k.steps, halves = 4 * steps, gap = k.gap, seen = k.seen;
                const int32_t* const table = p.table + k.r * p.table_row;
                const int64_t head = k.kv * p.pool.stride_head;
                // tile x of the segment
                const bool ahead = kTiles == 1 || k.shared;
                auto is_key = [&](int x) { return !ahead ? x % 2 == 0 : x == 0 || (x % 2 == 1 && x < 2 * steps - 1); };
                auto step_of = [&](int x) { return !ahead || x == 2 * steps - 1 ? x / 2 : is_key(x) ? (x + 1) / 2 : x / 2 - 1; };
                // Bulk copies: a lane has a box of `box` tokens by 128 bytes of a half.  Otherwise a lane has tokens lane and lane + 32.
                constexpr int kAcross = kNarrow ? (DP + 127) / 128 : DP / 64;
                const int across = kNarrow ? (D + 127) / 128 : (D + 63) / 64, my_box = lane / kAcross * p.box, my_part = lane % kAcross;
                const bool in_boxes = p.box > 0, has_box = in_boxes && my_box < kHalf && my_part < across;
                // pages of this lane's tokens: asked for long before they are used
                int pages[kOffs];
                auto fetch_pages = [&](int h) {
                    if (in_boxes) {
                        const int u = (k.j + step_of(h / 2)) * kKeys + h % 2 * kHalf + my_box;
                        pages[0] = 0;
                        if (has_box && u < seen) pages[0] = table[page_of(p.pool, u + (u >= p.kept ? gap : 0))];
                        return;
                    }
#pragma unroll
                    for (int c = 0; c < kOffs; c++) {
                        const int u = (k.j + step_of(h / 2)) * kKeys + h % 2 * kHalf + c * 32 + lane;
                        pages[c] = 0;
                        if (u < seen) pages[c] = table[page_of(p.pool, u + (u >= p.kept ? gap : 0))];
                    }
                };
                // A half whose copies are on their way and which is looked over, or turned into 16 bits, when they are there: which, on what barrier, and
                // rows whose page is in the pool.
                int pending = -1, pending_turn = 0;
                uint32_t pending_rows[kOffs];
                int h = (me + S::kLoadWarps - 2 * tile0 % S::kLoadWarps) % S::kLoadWarps;  // this warp's first half
                if (h < halves) fetch_pages(h);
                // The first two tiles do not wait for the rows of Q, which wait for the end of the last block's scores.  (The places of these two
                // are left by tiles of blocks before.)  The first warp brings them in bulk; else each brings some.
                bool query_due = !in_boxes || me == 0;
                // (Each step stands here once: the instructions of all roles have to come through one cache.)
#pragma unroll 1
                while (query_due || h < halves || pending >= 0) {
                    int issued = -1, issued_turn = 0;
                    uint32_t rows_there[kOffs];
                    if (h < (query_due ? min(4, halves) : halves)) {
                        const int x = h / 2, tile = tile0 + x, s = tile % kStages, u0 = (k.j + step_of(x)) * kKeys + h % 2 * kHalf;
                        bool room = tile < kStages || __all_sync(~0u, bar_try(empty(s), (tile / kStages - 1) & 1));
                        if (!room && pending < 0 && !query_due) {  // (nothing else to do)
                            if (!(fine = wait(empty(s), (tile / kStages - 1) & 1))) break;
                            room = true;
                        }
                        if (room) {
                            const bool key = is_key(x);
                            const uint32_t to = ring + s * S::kStage + h % 2 * kHalf * 128;
                            if (in_boxes) {
                                const int u = u0 + my_box, t = u + (u >= p.kept ? gap : 0), page = pages[0];
                                const bool bad = has_box && u < seen && (unsigned)page >= (unsigned)p.pool.n_pages, issue = has_box && u < seen && !bad;
                                const int slot = t - page_of(p.pool, t) * p.pool.page_size;
                                const uint32_t any_bad = __ballot_sync(~0u, bad), issues = __ballot_sync(~0u, issue);
#pragma unroll
                                for (int c = 0; c < kOffs; c++)
                                    rows_there[c] = any_bad ? ~__reduce_or_sync(~0u, bad ? lowest(my_box + p.box - c * 32) & ~lowest(my_box - c * 32) : 0u) : ~0u;
                                const bool looks = kNarrow || (!key && (any_bad || partly_seen(p, k, u0 - h % 2 * kHalf, kKeys)));
                                const uint32_t bar = looks ? landed(me, turn) : full(s);
                                if (lane == 0) {
                                    if (looks) bar_expect(bar, __popc(issues) * p.box * 128);
                                    else bar_bytes(bar, __popc(issues) * p.box * 128);
                                }
                                __syncwarp();
                                if (issue)
                                    copy_box(to + (my_part + (kNarrow ? kAcross : 0)) * (kKeys * 128) + my_box * 128, key ? &p.k_map : &p.v_map, my_part * (kNarrow ? 128 : 64),
                                             p.key_dim ? slot : k.kv, p.key_dim ? k.kv : slot, page, bar);
                                if (looks) issued = h, issued_turn = turn, turn ^= 1;
                            } else {
                                int64_t off[kOffs];  // of the rows of this lane's tokens, or -1
#pragma unroll
                                for (int c = 0; c < kOffs; c++) {
                                    const int u = u0 + c * 32 + lane, t = u + (u >= p.kept ? gap : 0);
                                    const bool there = (unsigned)pages[c] < (unsigned)p.pool.n_pages;
                                    off[c] = u < seen && there ? (pages[c] * p.pool.stride_page + (t - page_of(p.pool, t) * p.pool.page_size) * p.pool.stride_slot + head) * C::bytes : -1;
                                    rows_there[c] = ~__ballot_sync(~0u, u < seen && !there);
                                }
                                const char* const pool = (key ? p.pool.k : p.pool.v) + chunk * 16;
                                constexpr int kBatch = kRounds / kOffs < 8 ? kRounds / kOffs : 8;
#pragma unroll
                                for (int c = 0; c < kOffs; c++) {
#pragma unroll 1
                                    for (int i0 = 0; i0 < kRounds / kOffs; i0 += kBatch) {
#pragma unroll
                                        for (int i = 0; i < kBatch; i++) {
                                            const int row = (i0 + i) * kAtOnce + lane_row;
                                            const int64_t o = __shfl_sync(~0u, off[c], row);
                                            if (copies) copy16(to + place(c * 32 + row, kRaw + chunk), pool + (o < 0 ? 0 : o), o < 0 ? 0 : 16);
                                        }
                                    }
                                }
                                commit_copies();
                                issued = h;
                            }
                            if (lane == 0) {
                                bool any_bad = false;
#pragma unroll
                                for (int c = 0; c < kOffs; c++) {
                                    if (key) valid[(step0 + step_of(x)) & 7][h % 2 * kOffs + c] = rows_there[c];  // (what lies behind the last token is no row's)
                                    any_bad |= rows_there[c] != ~0u;
                                }
                                if (any_bad) flag(p.status, FCSIM_KV_BAD_PAGE);
                            }
                            __syncwarp();
                            // (Behind `valid`: who waits for the tile reads that too, and where no page of it is in the pool no copy is waited for.)
                            if (in_boxes && issued < 0) bar_arrive(full(s));
                            h += S::kLoadWarps;
                            if (h < halves) fetch_pages(h);
                        }
                    }
                    if (query_due) {
                        if (segment > 0 && !(fine = wait(query_empty, (segment - 1) & 1))) break;
                        if (in_boxes) {
                            // all rows of the block, or tile after tile; what lies behind the request's rows is no row of the block
                            const int boxes = p.query_tokens == p.tokens_a_block ? 1 : k.tiles_in_use, rows = p.query_tokens * heads_a_tile;
                            if (lane == 0) bar_expect(query_full, boxes * (DP / 64) * rows * 128);
                            __syncwarp();
                            if (lane < boxes * (DP / 64))
                                copy_box(query + lane / (DP / 64) * (128 * 128) + lane % (DP / 64) * (S::kRows * 128), &p.q_map, lane % (DP / 64) * 64,
                                         k.kv * group + k.ht * heads_a_tile, k.row + lane / (DP / 64) * p.query_tokens, query_full);
                        } else {
                            constexpr int kQueryLanes = DP / 8, kQueryRows = 32 / kQueryLanes;
                            const int at = lane % kQueryLanes, head0 = k.kv * group + k.ht * heads_a_tile, part = min(heads_a_tile, group - k.ht * heads_a_tile);
#pragma unroll 1
                            for (int r0 = me * 16; r0 < k.tiles_in_use * 128; r0 += 16 * S::kLoadWarps) {
                                const int row = r0 + lane % 16, token = row * token_magic >> 16, g = row - token * heads_a_tile;
                                int64_t off = -1;
                                if (token < k.tokens && g < part) off = ((int64_t)(k.row + token) * p.q_row + (int64_t)(head0 + g) * p.q_head) * 2;
#pragma unroll
                                for (int i = 0; i < 16 / kQueryRows; i++) {
                                    const int64_t o = __shfl_sync(~0u, off, i * kQueryRows + lane / kQueryLanes);
                                    const int y = r0 + i * kQueryRows + lane / kQueryLanes;
                                    if (at < D / 8)
                                        copy16(query + at / 8 * (S::kRows * 128) + y * 128 + ((at % 8) ^ (y % 8)) * 16, p.q + (o < 0 ? 0 : o + at * 16), o < 0 ? 0 : 16);
                                }
                            }
                            commit_copies();
                            wait_copies<0>();
                            fence_for_products();
                            bar_arrive(query_full);
                        }
                        query_due = false;
                    }
                    // The half before this one, whose copies had the time of this one's.  (One by one they take longer than to arrive: then it is this one.)
                    bool pending_now = pending >= 0;
                    if (!in_boxes && !kNarrow && issued >= 0) {
                        pending_now = true, pending = issued, issued = -1;
#pragma unroll
                        for (int c = 0; c < kOffs; c++) pending_rows[c] = rows_there[c];
                    }
                    if (pending_now) {
                        if (in_boxes) {
                            if (!(fine = wait(landed(me, pending_turn), landed_parity >> pending_turn & 1))) break;
                            landed_parity ^= 1u << pending_turn;
                        } else if (issued >= 0)
                            wait_copies<1>();
                        else
                            wait_copies<0>();
                        const int x = pending / 2, s = (tile0 + x) % kStages, u0 = (k.j + step_of(x)) * kKeys + pending % 2 * kHalf;
                        const uint32_t to = ring + s * S::kStage + pending % 2 * kHalf * 128;
                        uint32_t gone[kOffs];  // rows without a token, or of pages outside the pool
                        bool edge = partly_seen(p, k, u0 - pending % 2 * kHalf, kKeys);
#pragma unroll
                        for (int c = 0; c < kOffs; c++) {
                            gone[c] = ~lowest(seen - u0 - c * 32) | ~pending_rows[c];
                            edge |= gone[c] != 0;
                        }
                        // What some row does not see must not meet its weight of zero as an infinity or NaN.
                        edge = edge && !is_key(x);
                        auto is_gone = [&](int row) { return (row < 32 || kOffs == 1 ? gone[0] : gone[kOffs - 1]) >> row % 32 & 1; };
                        bool found = false;
                        if constexpr (kNarrow) {
                            constexpr int kBatch = 4;  // rows a lane reads before the first is written over
                            const bool turns = turned_chunk < chunks;
                            auto rows_on = [&](int i0, int i) { return to + (i0 / kBases + i / kBases) * 1024; };
#pragma unroll 1
                            for (int i0 = 0; i0 < kRounds; i0 += kBatch) {
                                uint4 raw[kBatch];
                                __syncwarp();
#pragma unroll
                                for (int i = 0; i < kBatch; i++) {
                                    raw[i] = make_uint4(0, 0, 0, 0);
                                    if (turns) raw[i] = load16(rows_on(i0, i) + place_raw[i % kBases]);
                                }
                                if (edge) {
#pragma unroll 1
                                    for (int i = 0; i < kBatch; i++) {
                                        uint4 y = raw[0];
                                        if (i == 1) y = raw[1];
                                        if (i == 2) y = raw[2];
                                        if (i == 3) y = raw[3];
                                        if (is_gone(turned_row(i0 + i))) y = make_uint4(0, 0, 0, 0);
                                        else found |= make_finite8(y);
                                        if (i == 0) raw[0] = y;
                                        if (i == 1) raw[1] = y;
                                        if (i == 2) raw[2] = y;
                                        if (i == 3) raw[3] = y;
                                    }
                                }
                                __syncwarp();
#pragma unroll
                                for (int i = 0; i < kBatch; i++) {
                                    uint4 a, b;
                                    widen<T>(raw[i], a, b);
                                    if (turns) {
                                        store16(rows_on(i0, i) + place_low[i % kBases], a);
                                        store16(rows_on(i0, i) + place_high[i % kBases], b);
                                    }
                                }
                            }
                        } else if (edge && copies) {
                            uint32_t any = 0;
#pragma unroll 8
                            for (int i = 0; i < kRounds; i++) any |= infinite_among<T>(load16(to + place(i * kAtOnce + lane_row, chunk)));
                            uint32_t none = 0;
#pragma unroll
                            for (int c = 0; c < kOffs; c++) none |= gone[c];
                            if (any | none) {
#pragma unroll 1
                                for (int i = 0; i < kRounds; i++) {
                                    const uint32_t at = to + place(i * kAtOnce + lane_row, chunk);
                                    uint4 y = load16(at);
                                    if (is_gone(i * kAtOnce + lane_row)) store16(at, make_uint4(0, 0, 0, 0));
                                    else if (any && make_finite<T>(y)) {
                                        store16(at, y);
                                        found = true;
                                    }
                                }
                            }
                        }
                        if (found) infinite[segment % kSegments] = 1;
                        fence_for_products();
                        bar_arrive(full(s));
                    }
                    pending = issued, pending_turn = issued_turn;
#pragma unroll
                    for (int c = 0; c < kOffs; c++) pending_rows[c] = rows_there[c];
                }
                if (!fine) {  // what is on its way arrives before the CTA ends
                    const int64_t began = clock64();
                    while (clock64() - began < 4000000) {}
                    break;
                }
                tile0 += 2 * steps, step0 += steps;
                leave_segment();
            }
            wait_copies<0>();
        }
    }
    fence_before_sync();
    __syncthreads();
    if (warp == kProductWarp) {
        fence_after_sync();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kColumns) : "memory");
    }
}

template <class T, class C, int DP, bool LONG>
int launch_walks(const PrefillParams& p, int grid, int device, cudaStream_t stream) {
    using S = Shape<T, C, DP>;
    static std::atomic<bool> raised[kMaxDevices];
    if (device >= kMaxDevices || !raised[device].load(std::memory_order_relaxed)) {
        auto* kernel = fcsim_kv_prefill_kernel<T, C, DP, LONG>;
        cudaFuncAttributes a;
        cudaError_t e = cudaFuncGetAttributes(&a, kernel);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kBytes);
        if (e != cudaSuccess) return (int)e;
        if (S::kTiles == 2 && a.numRegs * S::kThreads < 256 * (S::kSoftmaxRegisters + S::kOtherRegisters)) return (int)cudaErrorLaunchOutOfResources;
        if (device < kMaxDevices) raised[device].store(true, std::memory_order_relaxed);
    }
    fcsim_kv_prefill_kernel<T, C, DP, LONG><<<grid, S::kThreads, S::kBytes, stream>>>(p);
    return (int)cudaGetLastError();
}
template <class T, class C, int DP>
int launch(const PrefillParams& p, int grid, int device, cudaStream_t stream) {
    return p.aside ? launch_walks<T, C, DP, true>(p, grid, device, stream) : launch_walks<T, C, DP, false>(p, grid, device, stream);
}
template <class T, class C, int DP>
PrefillVariant variant() {
    return {launch<T, C, DP>, Shape<T, C, DP>::kRows, Shape<T, C, DP>::kKeys, DP, C::bytes == 2 || DP > 64};
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
