// attend_tc.cu -- attention of drafted tokens over the paged bf16 cache on the
// tensor cores.
//
// One CTA an SM, twelve warps:
//   warps 0-3, 4-7   two softmax groups, one a stream; thread = query row
//   warps 8, 11      load key tiles and value tiles (TMA) into two rings of shared memory
//   warps 9, 10      issue the score products and the products with the values
// A stream holds up to 128 query rows (token, head of the key/value head): its
// scores S = Q K^T (two buffers of 128 x 64 fp32) and sums O (128 x D fp32) lie in
// tensor memory.  Per 64 keys: S by tcgen05.mma from shared memory; the group
// reads its rows, computes p = 2^(s - m) and writes them (bf16) over S; O += P V
// by tcgen05.mma with P from tensor memory, which frees the buffer for the scores
// after next.  So the next scores are there when a group has written its weights,
// and both groups compute exponentials all the time.
//   PAIR:   an item has up to 256 rows, each stream takes 128 of them and all
//           keys: a tile crosses HBM once for all heads and tokens;
//   !PAIR:  up to 128 rows (single tokens, short chains): stream 0 takes the
//           first 64 keys of every tile, stream 1 the others, and their sums are
//           joined at the end.
// A parity tells a phase only from its neighbours, so a phase may be waited for only
// when the one before it has ended.  The loading and issuing warps meet every phase of
// their barriers in turn, the softmax groups those of the scores, the queries and the
// items' starts.  The groups skip phases of pv_done and of full_v: what has ended by
// then is said at these waits.
// The reference m of a row follows its largest score only when that has grown by
// more than kSlack in log2 units: then O is multiplied in place (rare after the
// first tiles); until then p <= 2^kSlack, which bf16 and the fp32 sums hold with
// the same relative error.
//
// Places that a token does not see: their scores become -inf before the maximum
// (tiles that reach past the cached tokens only).  Rows of V that nobody may see
// (the rest of the last page) are zeroed in shared memory, and so are elements
// of drafted tokens' V that are not finite (0 * inf would spoil every row); the
// rows that do see such a token get the element added at the end.
//
// What bounds it.  32 single tokens, 32 query and 8 key/value heads of 128, contexts
// to 16,201: 166 to 169 us, 6.3 TB/s (93 % of a copy's rate).  64 trees of 61 tokens over
// contexts to 8,101: 241 to 264 us on several GB300s, 4.4 to 4.9 TB/s, 1.0 to 1.1
// PFLOP/s: 64 keys of 256 rows need 1,400 cycles of HBM, 1,280 of shared memory (the
// queries are read again for each score product), 1,050 of the tensor cores and 800 of
// issue slots, and take 1,970, the chain of a softmax warp's steps.  One tree of 61 over
// 1,911: 19 us with the join, dependent latencies.  Measured against this layout: keys in
// units of 64 in the rings 185 / 389 / 29 us where this took 193 / 367 / 24, scores of
// 128 keys at a time (no second buffer) 196 / 404 / 23.
// With windows: the 64 trees and 2,048 positions 155 us (floor 84), two prompt pieces of 2,000 tokens and 1,024 positions
// 107 (34), 32 single tokens 43.5 (19): items of ten to twenty tiles, whose starts and ends take as long as four.  Over packed
// pages the 64 trees take 326 us (floor 142, the products): tensor cores 37 %, instructions 57 % of what can be issued, HBM
// 16 %; the softmax warps' chain, and instruction fetch, as the roles' loops share the instruction cache.  32 trees of 17
// (68 rows, one stream a half) take 154 to 158 us (floor 24), hardly less with half the rows: a fixed time a tile.
#include <cuda.h>
#include <cuda_bf16.h>

#include "attend.cuh"
#include "packed.cuh"
#include "rheo_kernels.h"

namespace rheo {
namespace {

constexpr int kTile = 128;                   // keys a tile: what is loaded at a time
constexpr int kSub = 64;                     // keys of a score product: half a tile
constexpr int kScores = 2;                   // score buffers of a stream
constexpr int kTcThreads = 12 * 32, kTcPackedThreads = 16 * 32;
__host__ __device__ constexpr int tc_threads(int kind) { return kind == 2 ? kTcPackedThreads : kTcThreads; }
// Registers a thread where sixteen warps share them: softmax groups, warps that load and issue, warps that expand packed
// tiles.  64 trees of 61 tokens: 367, 341, 328 us with 160, 168, 176 for the softmax groups, 327 with 184 (the issuing warps spill).
constexpr int kSoftmaxRegs = 176, kIssueRegs = 80, kExpandRegs = 80, kPackedLaunchRegs = 128;
static_assert(2 * kSoftmaxRegs + kIssueRegs + kExpandRegs <= 4 * kPackedLaunchRegs);
constexpr float kSlack = 8.0f;
constexpr int kWaitLimit = 1 << 23;          // polls of a wait before the kernel gives up
constexpr int kDrainLimit = 1 << 16;         // and of a drain after that

template <int D, bool PAIR, int KIND> struct TcShape {
    static constexpr int kUnit = kTile * D * 2;  // bytes of a key or value tile
    static constexpr int kHalves = D / 64;       // 128-byte wide parts of a line
    static constexpr int kK = D == 128 ? 2 : KIND == 2 ? 4 : 5;                   // slots of the key ring
    static constexpr int kV = D == 128 ? (KIND == 2 ? 2 : 3) : KIND == 2 ? 4 : 5;  // and of the value ring, which is read later
    // Packed tiles on their way: 64 places' codes and scales of the keys, or the values, a slot.
    static constexpr int kRawK = 4, kRawV = 3;
    static constexpr int kRawUnit = KIND == 2 ? 36 * D : 0;  // four blocks of 16 tokens: the most
    static constexpr int kRawScales = 32 * D;                // where the scales lie, behind the codes
    static constexpr int kQ = 128 * D * 2;       // bytes of 128 rows of queries
    static constexpr int kQueries = PAIR ? 2 * kQ : kQ;
    static constexpr int kMerge = PAIR ? 0 : 16384;
    // Tensor memory: stream s has two buffers of scores at columns 128 s and 128 s + 64, whose first 32 columns take
    // the weights (bf16 pairs), and its sums at kO + s D.
    static constexpr int kO = 256;
    // A softmax group that waits for the values of tile u knows that those of tile u - 2 have come (the reason is at clean(),
    // and rests on the order of tc_scores).
    static_assert(kV >= kScores);
};

struct TcControl {
    unsigned long long full_k[5], empty_k[5], full_v[5], empty_v[5];
    unsigned long long s_full[2][kScores], p_ready[2][kScores], pv_done[2][kScores], drained[2], q_ready, q_taken, all_sync;
    uint32_t tmem;
    int abort;
    int any_odd;          // some drafted value is not finite
    union {
        uint32_t odd[128];  // kWhole: which drafted tokens'
        struct {            // kPacked: packed halves on their way, keys and values, and which of their blocks are there
            unsigned long long raw_full[2][4], raw_empty[2][4];
            uint32_t raw_have[2][4];
        };
    };
    float2 ml[128];       // !PAIR: stream 1's reference and sum, then the weights of both streams
    AttendCut cut;
};

template <int D, bool PAIR, int KIND> constexpr size_t tc_smem_bytes() {
    using S = TcShape<D, PAIR, KIND>;
    return 1024 + S::kQueries + (size_t)(S::kK + S::kV) * S::kUnit + S::kMerge + (S::kRawK + S::kRawV) * S::kRawUnit + sizeof(TcControl);
}

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(unsigned long long* b, int count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(unsigned long long* b) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(b)) : "memory");
}
// One arrival for a warp, after all its lanes' accesses.
__device__ __forceinline__ void bar_arrive_warp(unsigned long long* b) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) bar_arrive(b);
}
__device__ __forceinline__ void bar_expect(unsigned long long* b, int bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(b)), "r"(bytes) : "memory");
}
// Waits for the phase of this parity to end (called by whole warps); false, for all lanes, after kWaitLimit polls or
// where another warp gave up.  A drain (the last waits before the CTA ends) goes on where another warp gave up.
template <bool DRAIN = false>
__device__ __forceinline__ bool bar_wait(unsigned long long* b, uint32_t parity, TcControl& c) {
    const uint32_t at = smem_u32(b);
    uint32_t done = 0;
    for (int i = 0; i < kWaitLimit; ++i) {
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(done)
            : "r"(at), "r"(parity)
            : "memory");
        if (done || (!DRAIN && (i & 255) == 255 && *(volatile int*)&c.abort)) break;
        if (DRAIN && i > kDrainLimit && *(volatile int*)&c.abort) break;
    }
    if (__all_sync(0xffffffffu, done)) return true;
    *(volatile int*)&c.abort = 1;
    return false;
}

__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// True in one lane of the warp, always the same one.  Products and commits are issued under it, with operands that the
// compiler knows to be uniform; a branch on the lane instead cost 110 cycles a product.
__device__ __forceinline__ bool elect_one() {
    uint32_t e;
    asm volatile(
        "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\tselp.u32 %0, 1, 0, e;\n\t}"
        : "=r"(e)::"memory");
    return e != 0;
}
__device__ __forceinline__ void tc_commit_at(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_commit(unsigned long long* b) { tc_commit_at(smem_u32(b)); }
// A value that is the same in all lanes, in a register that the compiler knows to be.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __reduce_or_sync(0xffffffffu, x); }

#define RHEO_R32(M) M(0), M(1), M(2), M(3), M(4), M(5), M(6), M(7), M(8), M(9), M(10), M(11), M(12), M(13), M(14), M(15), \
    M(16), M(17), M(18), M(19), M(20), M(21), M(22), M(23), M(24), M(25), M(26), M(27), M(28), M(29), M(30), M(31)
#define RHEO_R16(M) M(0), M(1), M(2), M(3), M(4), M(5), M(6), M(7), M(8), M(9), M(10), M(11), M(12), M(13), M(14), M(15)

// Columns of this thread's row.  These are .sync.aligned: callers come with the whole warp together (after a bar_wait,
// which ends in a vote, or a __syncwarp where lanes took different ways before).
__device__ __forceinline__ void tmem_ld32(uint32_t (&r)[32], uint32_t at) {
#define OUT(i) "=r"(r[i])
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : RHEO_R32(OUT)
        : "r"(at));
#undef OUT
}
__device__ __forceinline__ void tmem_st32(uint32_t at, const uint32_t (&r)[32]) {
#define IN(i) "r"(r[i])
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::RHEO_R32(IN),
        "r"(at)
        : "memory");
#undef IN
}
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t (&r)[16]) {
#define IN(i) "r"(r[i])
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::RHEO_R16(IN),
        "r"(at)
        : "memory");
#undef IN
}

// Shared-memory operand in 128-byte swizzle: start, leading and stride byte offsets.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lead, uint32_t stride) {
    return (uint64_t)((addr & 0x3FFFF) >> 4) | ((uint64_t)(lead >> 4) << 16) | ((uint64_t)(stride >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}
// bf16 x bf16 -> fp32, M = 128; B along K, or along N.
__device__ __forceinline__ constexpr uint32_t mma_desc(int n, bool b_along_n) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (b_along_n ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | (8u << 24);
}
constexpr uint32_t kNegateA = 1u << 13;
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(desc), "r"((uint32_t)add)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t desc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(desc), "r"((uint32_t)add)
        : "memory");
}
__device__ __forceinline__ void tma_tile(uint32_t dst, const CUtensorMap* map, int x, int head, int page,
                                         unsigned long long* bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
        "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(0), "r"(head), "r"(page)
        : "memory");
}

__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, int bytes, unsigned long long* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}

using TcWalk = AttendWalk<kTile>;

// kWhole: a class is a request, and an item walks all its places.  kWindow, kPacked: classes and tiles of LongItem.
enum { kWhole, kWindow, kPacked };

// One item: request, key/value head, first query row, lengths (ctx: all cached tokens), and its tiles.
template <int KIND> struct TcItem {
    int b, h, r0;
    AttendSpan s;
    LongItem<kTile> it;
    __device__ __forceinline__ TcItem() {}
    __device__ __forceinline__ TcItem(int request, int item, int groups, int item_rows, const AttendSpan& span)
        : b(request), h(item / groups), r0(item % groups * item_rows), s(span) {}
    __device__ __forceinline__ TcItem(const AttendArgs& a, int cls, int item, int groups, int item_rows) {
        if constexpr (KIND == kWhole) {
            b = cls;
            h = item / groups;
            r0 = item % groups * item_rows;
            s = attend_span(a, b);
        } else {
            b = cls / groups;
            h = item;
            r0 = cls % groups * item_rows;
            it = LongItem<kTile>(a, b, r0, item_rows);
            s = AttendSpan{it.s.ctx, it.s.add, it.s.bad};
        }
    }
    __device__ __forceinline__ void open(TcWalk& w) const {
        if constexpr (KIND == kWhole) w.open(s.len());
        else w.open_tiles(it.n);
    }
    // of the item's i-th tile
    __device__ __forceinline__ int begin(int i) const { return KIND == kWhole ? i * kTile : it.begin(it.number(i)); }
    __device__ __forceinline__ int end(int i) const { return KIND == kWhole ? s.len() : it.end(it.number(i)); }
    __device__ __forceinline__ bool packed(int i) const { return KIND == kPacked && it.is_packed(it.number(i)); }
    // score products: the second half only where it has a place
    __device__ __forceinline__ int subs(int i) const { return end(i) - begin(i) > kSub ? 2 : 1; }
    // LONG: whether a tile of 16 bits has places that not all of the item's tokens see (or nobody); of those from lo_most
    // on they all see the ones below `upto`.
    __device__ __forceinline__ bool unclear(int upto, int place, int end) const {
        return place + kTile > min(end, upto) || place < it.lo_most;
    }
    // Whether some of n tiles from the i-th on has a second half: only the last ones of the sinks and of both parts may lack it.
    __device__ __forceinline__ bool second(int i, int n) const {
        if constexpr (KIND == kWhole) return n > 1 || subs(i) == 2;
        bool any = false;
        for (int k = 0; k < min(n, 4); ++k) any |= subs(i + k) == 2;
        return any;
    }
};
template <int KIND> __device__ __forceinline__ int tc_per(const AttendArgs& a, int groups) {
    return KIND == kWhole ? a.H * groups : a.H;
}

__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Elements of a pair that are not finite.
__device__ __forceinline__ uint32_t odd_mask(uint32_t w) {
    return ((w & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((w & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
}

// This thread's share of the copies of an item's query rows into the swizzled operand (asynchronous).  Rows that the
// item does not have keep what is there: they only reach their own, unused, rows of the products.
template <int D>
__device__ __forceinline__ void tc_queries(const AttendArgs& a, int b, int h, int first, int count, char* to, int tid,
                                           int threads) {
    constexpr int C = D / 8;  // 16-byte pieces of a row
    const char* q = static_cast<const char*>(a.io.q) + (int64_t)b * a.io.q_batch * 2;
    for (int i = tid; i < count * C; i += threads) {
        const int r = i / C, p = i % C, row = first + r, t = row / a.G;
        const char* src = q + (t * a.io.q_token + (h * a.G + row - t * a.G) * a.io.q_head + p * 8) * 2;
        const uint32_t dst = smem_u32(to + (p >> 3) * 16384 + r * 128 + (((p & 7) ^ (r & 7)) << 4));
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    }
}

// Which of the 64 places from the j0-th drafted token on the tokens tt0 .. t_last see, a vote a word; the lane of token t
// keeps its words.  TOKENS at a time, so that as many loads are under way.
template <int TOKENS, int KIND>
__device__ __forceinline__ void tc_votes(const AttendArgs& a, const TcItem<KIND>& item, int j0, int tt0, int t_last, int t,
                                         uint32_t (&words)[2]) {
    const int lane = threadIdx.x & 31, b = item.b;
    const AttendSpan span = item.s;
    for (int tt = tt0; tt <= t_last; tt += TOKENS) {
        bool sees[TOKENS][2];
#pragma unroll
        for (int u = 0; u < TOKENS; ++u) {
            const int tok = min(tt + u, t_last);
            const uint8_t* mrow = a.mask ? a.mask + ((int64_t)b * a.T + tok) * a.T : nullptr;
            const int first = KIND == kWhole ? 0 : long_first(a, item.it.s, long_depth(a, b, tok));
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                const int place = span.ctx + j0 + 32 * v + lane;
                if constexpr (KIND == kWhole) sees[u][v] = tt + u < span.add && attend_sees(span, mrow, tt + u, place);
                else sees[u][v] = tt + u < span.add && place >= span.ctx && item.it.sees(a, b, mrow, tt + u, first, place);
            }
        }
#pragma unroll
        for (int u = 0; u < TOKENS; ++u)
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                const uint32_t bits = __ballot_sync(0xffffffffu, sees[u][v]);
                if (tt + u == t) words[v] = bits;
            }
    }
}

// The n lowest of 64 bits.
__device__ __forceinline__ unsigned long long low_bits(int n) {
    return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1;
}

// The softmax group of stream `st`.
template <int D, bool PAIR, int KIND>
__device__ __forceinline__ void tc_softmax(const AttendArgs& a, TcControl& c, char* q_smem, char* v_ring, char* merge, int st) {
    using S = TcShape<D, PAIR, KIND>;
    const int tid = threadIdx.x & 127, lane = tid & 31, warp = tid >> 5;
    const int rows = a.T * a.G, item_rows = PAIR ? 256 : 128, groups = (rows + item_rows - 1) / item_rows,
              per = tc_per<KIND>(a, groups);
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    const uint32_t t_s = c.tmem + lanes + st * 128, t_o = c.tmem + lanes + S::kO + st * D;
    const float sc = fmaxf(fabsf(a.scale_log2), 1e-30f);  // above 0, so that hidden places stay at -inf
    uint32_t items = 0, products = 0, syncs = 0, tile0 = 0;
    unsigned long long seen = 0;  // T <= 64: drafted tokens that this row sees, of request seen_b's rows from seen_r0
    int seen_b = -1, seen_r0 = -1;
    auto sync_all = [&]() -> bool {
        bar_arrive_warp(&c.all_sync);
        return bar_wait(&c.all_sync, syncs++ & 1, c);
    };
    // queries of an item: each stream's group fetches its own rows (PAIR), or stream 0's all of them
    auto fetch = [&](int cls, int item) {
        const int h = KIND == kWhole ? item / groups : item, b = KIND == kWhole ? cls : cls / groups;
        const int first = (KIND == kWhole ? item : cls) % groups * item_rows + (PAIR ? st * 128 : 0);
        tc_queries<D>(a, b, h, first, min(128, rows - first), q_smem + (PAIR ? st * S::kQ : 0), tid, 128);
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    TcWalk w(c.cut);
    AttendSpan next_span{0, 0, false};
    if (w.more()) {
        if (KIND == kWhole) next_span = attend_span(a, w.b);
        if (PAIR || st == 0) fetch(w.b, w.item);
    }
    while (w.more()) {
        TcItem<KIND> item;
        if constexpr (KIND == kWhole) item = TcItem<KIND>(w.b, w.item, groups, item_rows, next_span);
        else item = TcItem<KIND>(a, w.b, w.item, groups, item_rows);
        const AttendSpan span = item.s;
        item.open(w);
        const int n = w.n, b = item.b, h = item.h, r0 = item.r0;
        if (span.bad && threadIdx.x == 0) atomicOr(a.status, kStBadLength);
        if (!sync_all()) return;  // both streams are through with the last item
        // and the scores' warp has seen its start (it has to meet every phase of q_ready)
        if (items > 0 && !bar_wait(&c.q_taken, (items - 1) & 1, c)) return;
        if (KIND == kWhole && threadIdx.x < 128) c.odd[threadIdx.x] = 0;
        if (threadIdx.x == 0) c.any_odd = 0;
        asm volatile("cp.async.wait_all;" ::: "memory");
        fence_async();
        tc_fence_before();
        bar_arrive_warp(&c.q_ready);
        const bool last = w.last();
        const int next_b = w.item + 1 == per ? w.b + 1 : w.b, next_item = w.item + 1 == per ? 0 : w.item + 1;
        if (KIND == kWhole && !last) next_span = attend_span(a, next_b);
        ++items;

        const int row = r0 + (PAIR ? st * 128 : 0) + tid, t = row / a.G;
        const bool live = row < rows && t < span.add;
        const bool warp_live = __any_sync(0xffffffffu, live);
        const bool stream_live = PAIR ? r0 + st * 128 < rows : true;
        if (PAIR && !stream_live && !last) fetch(next_b, next_item);
        const int t_first = (row - lane) / a.G, t_last = min(min(row - lane + 31, rows - 1) / a.G, a.T - 1);  // of the warp
        // LONG: what a row sees is places [first, upto) and those below the sinks' end, without a mask and depths of its own
        // also among the drafted tokens; the warp's rows all see places [all_from, all_to)
        const bool chain = KIND != kWhole && !a.mask && (!a.depth || !a.window);
        int first = 0, upto = 0, all_from = 0, all_to = 0, clear_to = 0;
        if constexpr (KIND != kWhole) {
            if (live) first = long_first(a, item.it.s, long_depth(a, b, t));
            upto = chain ? span.ctx + t + 1 : span.ctx;
            all_to = chain ? span.ctx + t_first + 1 : span.ctx;
            clear_to = chain ? span.ctx + r0 / a.G + 1 : span.ctx;
            all_from = a.depth ? item.it.lo_most : long_first(a, item.it.s, t_last);
        }
        if (a.T <= 64 && !chain && (b != seen_b || r0 != seen_r0) && warp_live) {
            // which drafted tokens the row sees: once for all heads of a request
            uint32_t x[2] = {0u, 0u};
            tc_votes<8>(a, item, 0, t_first, t_last, t, x);
            seen = ((unsigned long long)x[1] << 32) | x[0];
            seen_b = b;
            seen_r0 = r0;
        }
        // Values of the tile at place k0 (tile u of this CTA) before a product of this stream reads them: nothing behind
        // the request's places, and no element that is not finite among the drafted tokens'.  PAIR: a thread a line;
        // !PAIR: the stream's half of the lines, two threads a line.
        // Called with a product of this stream's scores at hand, the only waits for full_v here, and not for each tile.  The
        // phase before, tile u - kV, has ended:
        // PAIR: a stream with rows has a product in every tile of the item, so its product two before this one (whose
        // buffer these scores took: they were issued after it) read tile u - 2 or a later one, or is of an earlier item.
        // !PAIR: stream 1 has no product in a tile without a second half, which LONG has in the middle of items (the last
        // tiles of the sinks and of the packed part), so its product two before may be of tile u - 3 or u - 4.  Stream 0 has
        // one in every tile, and tc_scores issues its scores of tile u before stream 1's: after stream 0's product with the
        // values of tile u - 2, or of an earlier item's last tile.
        // Where tile u - 2 is of an earlier item: stream 0, which reads every tile, has waited for that item's last product
        // before this item began.
        // The phase after needs this stream's product with tile u, which waits for what follows here.
        // LONG: nothing that no token of the item sees, and no element that is not finite where some may not see the place.
        auto clean = [&](int k0, int end, uint32_t u) -> bool {
            if (!bar_wait(&c.full_v[u % S::kV], (u / S::kV) & 1, c)) return false;
            constexpr int pieces = PAIR ? D / 8 : D / 16;
            const int r = PAIR ? tid : st * kSub + tid / 2, p0 = PAIR ? 0 : tid % 2 * pieces, place = k0 + r;
            char* line = v_ring + (u % S::kV) * S::kUnit + r * 128;
            auto piece = [&](int i) {
                const int p = p0 + i;
                return reinterpret_cast<uint4*>(line + (p >> 3) * 16384 + (((p & 7) ^ (r & 7)) << 4));
            };
            if (place >= end || (KIND != kWhole && !item.it.wanted(place, 1))) {
#pragma unroll
                for (int i = 0; i < pieces; ++i) *piece(i) = make_uint4(0, 0, 0, 0);
            } else if (place >= span.ctx || (KIND != kWhole && place < item.it.lo_most)) {
                // 0 * v summed over the line is NaN exactly if some element is not finite
                const __nv_bfloat162 zero = __floats2bfloat162_rn(0.0f, 0.0f);
                __nv_bfloat162 acc = zero;
#pragma unroll
                for (int i = 0; i < pieces; ++i) {
                    const uint4 x = *piece(i);
                    acc = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&x.x), zero, acc);
                    acc = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&x.y), zero, acc);
                    acc = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&x.z), zero, acc);
                    acc = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&x.w), zero, acc);
                }
                if (!(__low2float(acc) == 0.0f && __high2float(acc) == 0.0f)) {
                    const int j = place - span.ctx;
                    if (KIND == kWhole) atomicOr(&c.odd[j >> 5], 1u << (j & 31));
                    c.any_odd = 1;
                    __threadfence_block();  // the other stream's group finds either the elements or the mark
#pragma unroll 1
                    for (int i = 0; i < pieces; ++i) {
                        const uint4 x = *piece(i);
                        *piece(i) = make_uint4(x.x & ~odd_mask(x.x), x.y & ~odd_mask(x.y), x.z & ~odd_mask(x.z),
                                               x.w & ~odd_mask(x.w));
                    }
                }
            }
            fence_async();
            return true;
        };
        float m = -INFINITY, l = 0.0f;
        int mine = 0;  // score products of this stream in this item so far
        for (int q = 0; q < n && stream_live; ++q) {
            const int tile_k0 = item.begin(w.tile + q), end = item.end(w.tile + q), subs = item.subs(w.tile + q);
            // places that not all of the item's tokens see, in 16 bits
            const bool to_clean = KIND == kWhole ? tile_k0 + kTile > span.ctx
                                                 : !item.packed(w.tile + q) && item.unclear(clear_to, tile_k0, end);
            for (int sub = PAIR ? 0 : st; sub < subs; sub += PAIR ? 1 : 2) {
                const int k0 = tile_k0 + sub * kSub;
                const bool tail = KIND == kWhole ? k0 + kSub > span.ctx : k0 + kSub > min(end, all_to) || k0 < all_from;
                uint32_t vis[2] = {0xffffffffu, 0xffffffffu};
                if (KIND != kWhole && tail && warp_live) {
                    unsigned long long x = low_bits(min(end, upto) - k0) & (~low_bits(first - k0) | low_bits(item.it.sinks - k0));
                    const int off = k0 - span.ctx;
                    if (!chain && off > -kSub && !item.packed(w.tile + q)) {
                        // drafted tokens by the mask, their depths and the window
                        if (a.T <= 64) {
                            x |= off >= 0 ? (off < 64 ? seen >> off : 0ull) : seen << -off;
                        } else {
                            uint32_t y[2] = {0u, 0u};
                            tc_votes<8>(a, item, off, t_first, t_last, t, y);
                            x |= ((unsigned long long)y[1] << 32) | y[0];
                        }
                    }
                    vis[0] = (uint32_t)x;
                    vis[1] = (uint32_t)(x >> 32);
                } else if (tail && warp_live) {
                    if (a.T <= 64) {
                        // seen: bit j is drafted token j; bits below it are the cached places
                        const int off = k0 - span.ctx;
                        const unsigned long long x = off >= 0 ? (off < 64 ? seen >> off : 0ull)
                                                              : (seen << -off) | ((1ull << -off) - 1);
                        vis[0] = (uint32_t)x;
                        vis[1] = (uint32_t)(x >> 32);
                    } else {
                        tc_votes<8>(a, item, k0 - span.ctx, t_first, t_last, t, vis);
                    }
                }
                const uint32_t buf = products & 1, t_b = t_s + 64 * buf;
                if (!bar_wait(&c.s_full[st][buf], (products / 2) & 1, c)) return;
                tc_fence_after();
                // the item's last scores are there: this stream's queries have been read
                if (PAIR && q == n - 1 && sub == subs - 1 && !last) fetch(next_b, next_item);
                __syncwarp();
                if (warp_live) {
                    uint32_t s[2][32];
                    tmem_ld32(s[0], t_b);
                    tmem_ld32(s[1], t_b + 32);
                    tc_wait_ld();
                    if (KIND == kWhole && a.scale_log2 < 0.0f) {
#pragma unroll
                        for (int v = 0; v < 2; ++v)
#pragma unroll
                            for (int i = 0; i < 32; ++i) s[v][i] ^= 0x80000000u;
                    }
                    if (tail) {
#pragma unroll
                        for (int v = 0; v < 2; ++v)
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (!((vis[v] >> i) & 1u)) s[v][i] = 0xFF800000u;
                    }
                    float tops[4];
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const uint32_t* x = s[v / 2] + v % 2 * 16;
                        tops[v] = max3(__uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(x[2]));
#pragma unroll
                        for (int i = 3; i + 1 < 16; i += 2)
                            tops[v] = max3(tops[v], __uint_as_float(x[i]), __uint_as_float(x[i + 1]));
                        tops[v] = fmaxf(tops[v], __uint_as_float(x[15]));
                    }
                    const float top = fmaxf(max3(tops[0], tops[1], tops[2]), tops[3]) * sc;
                    if (mine == 0) {
                        m = top;
                    } else {
                        const bool grow = top > m + kSlack || (m == -INFINITY && top > m);
                        if (__any_sync(0xffffffffu, grow)) {
                            // the sums so far move to the new reference; the phase before of the last product's barrier has
                            // ended, as these scores were issued after the product before that one, and products end in order
                            if (!bar_wait(&c.pv_done[st][buf ^ 1], ((products - 1) / 2) & 1, c)) return;
                            tc_fence_after();
                            const float f = !grow || m == -INFINITY ? 1.0f : fast_exp2(m - top);
#pragma unroll 1
                            for (int d = 0; d < D; d += 32) {
                                uint32_t o[32];
                                __syncwarp();
                                tmem_ld32(o, t_o + d);
                                tc_wait_ld();
#pragma unroll
                                for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                                tmem_st32(t_o + d, o);
                            }
                            l *= f;
                            if (grow) m = top;
                        }
                    }
                    const float ref = m == -INFINITY ? 0.0f : m;
                    const unsigned long long sc2 = f2_pack(sc, sc), ref2 = f2_pack(-ref, -ref);
                    unsigned long long sum[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
                    for (int v = 0; v < 2; ++v) {
                        uint32_t p[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const unsigned long long x = f2_exp2(
                                f2_fma(f2_pack(__uint_as_float(s[v][2 * i]), __uint_as_float(s[v][2 * i + 1])), sc2, ref2));
                            sum[i & 3] = f2_add(sum[i & 3], x);
                            p[i] = pack_bf16(__uint_as_float((uint32_t)x), __uint_as_float((uint32_t)(x >> 32)));
                        }
                        if (v == 0) __syncwarp();
                        tmem_st16(t_b + 16 * v, p);  // over scores that are in registers by now
                    }
                    l += f2_fold(f2_add(f2_add(sum[0], sum[1]), f2_add(sum[2], sum[3])));
                    tc_wait_st();
                }
                if ((!PAIR || sub == 0) && to_clean) {
                    if (!clean(tile_k0, end, tile0 + q)) return;
                }
                tc_fence_before();
                bar_arrive_warp(&c.p_ready[st][buf]);
                ++products;
                ++mine;
            }
        }
        tile0 += n;

        // ---- the item's sums
        // both buffers' last products (the last scores were issued after the product before them, so the phases before
        // these have ended)
        if (mine > 0) {
            const uint32_t x = products - 1;
            if (x > 0 && !bar_wait(&c.pv_done[st][(x - 1) & 1], ((x - 1) / 2) & 1, c)) return;
            if (!bar_wait(&c.pv_done[st][x & 1], (x / 2) & 1, c)) return;
            tc_fence_after();
        }
        const bool whole = n == w.all;
        const int64_t part = attend_part(blockIdx.x, w.tile == 0);
        const int r_in = (PAIR ? st * 128 : 0) + tid, head = h * a.G + row - t * a.G;
        const bool both = !PAIR && item.second(w.tile, n);               // stream 1 has a share of the sums
        float f0 = 1.0f, f1 = 0.0f;                                      // the weights of the two streams
        int columns = D;             // that the streams exchange at a time
        const int kept = PAIR ? 128 : min(128, (rows + 31) / 32 * 32);  // rows of an item, to whole warps
        if (both) {
            columns = min(D, 4096 / kept / 32 * 32);
            if (st == 1) c.ml[tid] = make_float2(m, l);
        } else if (!PAIR && st == 1) {
            columns = 0;
        }
        if (!PAIR && !both && st == 0 && !last) fetch(next_b, next_item);
        float4* pass = reinterpret_cast<float4*>(merge);  // [columns / 4][kept]
        float ll = live ? l : 0.0f;
        for (int d0 = 0; d0 < D && columns > 0; d0 += columns) {
            if (both) {
                if (st == 1 && warp_live) {
                    for (int d = d0; d < d0 + columns; d += 32) {
                        uint32_t x[32];
                        __syncwarp();
                        tmem_ld32(x, t_o + d);
                        tc_wait_ld();
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            pass[((d - d0) / 4 + i) * kept + tid] =
                                make_float4(__uint_as_float(x[4 * i]), __uint_as_float(x[4 * i + 1]),
                                            __uint_as_float(x[4 * i + 2]), __uint_as_float(x[4 * i + 3]));
                    }
                }
                if (!sync_all()) return;
                if (st == 0 && d0 == 0) {
                    if (!last) fetch(next_b, next_item);  // both streams are through with the queries
                    const float2 x = c.ml[tid];
                    const float mm = fmaxf(m, x.x), ref = mm == -INFINITY ? 0.0f : mm;
                    f0 = fast_exp2(m - ref);
                    f1 = fast_exp2(x.x - ref);
                    l = l * f0 + x.y * f1;
                    m = mm;
                    ll = live ? l : 0.0f;
                }
            }
            if (PAIR || st == 0) {
                __threadfence_block();
                const bool odd = *(volatile int*)&c.any_odd != 0;
                const float inv = ll == 0.0f ? 0.0f : 1.0f / ll;
#pragma unroll 1
                for (int d = d0; d < d0 + columns; d += 32) {
                    float o[32];
                    __syncwarp();
                    if (warp_live) {
                        uint32_t x[32];
                        tmem_ld32(x, t_o + d);
                        tc_wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __uint_as_float(x[i]);
                        if (both) {
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const float4 y = pass[((d - d0) / 4 + i) * kept + tid];
                                o[4 * i] = o[4 * i] * f0 + y.x * f1;
                                o[4 * i + 1] = o[4 * i + 1] * f0 + y.y * f1;
                                o[4 * i + 2] = o[4 * i + 2] * f0 + y.z * f1;
                                o[4 * i + 3] = o[4 * i + 3] * f0 + y.w * f1;
                            }
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = 0.0f;
                    }
                    if (odd && live) {
                        // values that are not finite, for the rows that see their places
                        const uint8_t* mrow = a.mask ? a.mask + ((int64_t)b * a.T + t) * a.T : nullptr;
                        auto add_odd = [&](int x) {  // place x in the pages of 16 bits
                            const int64_t page = a.block_table[(int64_t)b * a.max_pages + (x >> a.page_shift)];
                            if (page < 0 || page >= a.pages) return;
                            const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(a.kv.value) + page * a.kv.value_page +
                                                     h * a.kv.value_head + (x & (a.P - 1)) * a.kv.value_token + d;
#pragma unroll
                            for (int i = 0; i < 32; ++i) {
                                const float y = __bfloat162float(v[i]);
                                if (!(fabsf(y) < INFINITY)) o[i] += y;
                            }
                        };
                        if constexpr (KIND == kWhole) {
                            for (int word = 0; word < (span.add + 31) / 32; ++word) {
                                for (uint32_t bits = c.odd[word]; bits; bits &= bits - 1) {
                                    const int j = word * 32 + __ffs(bits) - 1;
                                    if (mrow ? mrow[j] != 0 : j <= t) add_odd(span.ctx + j);
                                }
                            }
                        } else {
                            for (int i = w.tile; i < w.tile + n; ++i) {
                                if (item.packed(i) || !item.unclear(clear_to, item.begin(i), item.end(i))) continue;
                                for (int l0 = item.begin(i); l0 < item.end(i); ++l0)
                                    if ((l0 >= span.ctx || l0 < item.it.lo_most) && item.it.wanted(l0, 1) &&
                                        item.it.sees(a, b, mrow, t, first, l0))
                                        add_odd(l0 - item.it.s.pk);
                            }
                        }
                    }
                    // (no lane leaves the iteration early: the next one begins with a warp-wide load)
                    if (row < rows && whole) {
                        uint4* out = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.io.out) + b * a.io.out_batch +
                                                              t * a.io.out_token + head * a.io.out_head + d);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint4 y = make_uint4(0, 0, 0, 0);
                            if (ll != 0.0f) {
                                y.x = pack_bf16(o[8 * i] * inv, o[8 * i + 1] * inv);
                                y.y = pack_bf16(o[8 * i + 2] * inv, o[8 * i + 3] * inv);
                                y.z = pack_bf16(o[8 * i + 4] * inv, o[8 * i + 5] * inv);
                                y.w = pack_bf16(o[8 * i + 6] * inv, o[8 * i + 7] * inv);
                            }
                            out[i] = y;
                        }
                    } else if (row < rows) {
                        float4* po = reinterpret_cast<float4*>(a.part_o) + attend_part_at(a, part, r_in, d / 4);
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            po[i * a.part_rows] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                    }
                }
            }
            // stream 1 writes the next columns when stream 0 has read these
            if (both && d0 + columns < D && !sync_all()) return;
        }
        if ((PAIR || st == 0) && row < rows) {
            if (whole) {
                if (a.io.lse) a.io.lse[((int64_t)b * a.T + t) * a.H * a.G + head] = attend_lse(m, ll);
            } else {
                // a row past the request's tokens follows its query, whatever that holds: its reference is not kept
                *reinterpret_cast<float2*>(a.part_ml + (part * a.part_rows + r_in) * 2) = make_float2(live ? m : -INFINITY, ll);
            }
        }
        if (!whole && w.tile == 0 && threadIdx.x == 0)
            a.join[blockIdx.x] = make_int4(b, h * groups + r0 / item_rows, w.segments(c.cut, blockIdx.x), 0);
        w.next(per);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// A place in a ring: slot and the parity of its phase, one step at a time.
struct TcSlot {
    uint32_t slot = 0, parity = 0;
    __device__ __forceinline__ void next(uint32_t slots) {
        if (++slot == slots) {
            slot = 0;
            parity ^= 1;
        }
    }
};

// Key tiles, or value tiles, into their ring: lane = (page, half) of a tile.  Packed ones go to a ring of their own, 64
// places at a time, from which tc_expand fills the other; lane = block.
template <int D, bool PAIR, int KIND>
__device__ __forceinline__ void tc_load(const AttendArgs& a, TcControl& c, bool keys, const CUtensorMap* map, char* ring, char* raw) {
    using S = TcShape<D, PAIR, KIND>;
    unsigned long long* const full = keys ? c.full_k : c.full_v;
    unsigned long long* const empty = keys ? c.empty_k : c.empty_v;
    unsigned long long* const raw_full = c.raw_full[keys ? 0 : 1];
    unsigned long long* const raw_empty = c.raw_empty[keys ? 0 : 1];
    uint32_t* const raw_have = c.raw_have[keys ? 0 : 1];
    const uint32_t slots = keys ? S::kK : S::kV, raws = keys ? S::kRawK : S::kRawV;
    const int lane = threadIdx.x & 31;
    const int rows = a.T * a.G, item_rows = PAIR ? 256 : 128, groups = (rows + item_rows - 1) / item_rows,
              per = tc_per<KIND>(a, groups);
    const int boxes = kTile / a.P * S::kHalves;
    const int pi = lane / S::kHalves, half = lane % S::kHalves;
    const int N = packed_tokens(a.P), codes = N * D / 2, marks = keys ? D : N * D / 32;  // bytes of a block's codes, scales
    // this lane's block of a packed tile: which half it is of, its place there, where it lies in its page
    const int my_half = lane / (64 / N), my_place = lane % (64 / N);
    const int my_block = (lane & (a.P / N - 1)) * packed_block_bytes(N, D) + (keys ? 0 : codes);
    const int my_marks = 2 * codes + (keys ? 0 : D - codes);  // its scales behind its codes
    const uint32_t raw_to = smem_u32(raw);
    TcSlot at;
    uint32_t u = 0, copied = 0, seen = 0;  // tiles; packed halves copied, and known to have been expanded
    // Packed halves before the `to`-th have been expanded.
    auto expanded = [&](uint32_t to) {
        for (; seen < to; ++seen)
            if (!bar_wait(&raw_empty[seen % raws], (seen / raws) & 1, c)) return false;
        return true;
    };
    for (TcWalk w(c.cut); w.more();) {
        const TcItem<KIND> item(a, w.b, w.item, groups, item_rows);
        const int h = item.h;
        item.open(w);
        const int n = w.n;
        const int32_t* table = a.block_table + (int64_t)item.b * a.max_pages;
        // whether a token may see some of this lane's places of the tile, which begin at l0
        auto wants = [&](int i, int& l0) {
            if (KIND == kPacked && item.packed(i)) {
                l0 = item.begin(i) + lane * N;
                return lane < kTile / N && l0 < item.end(i) && item.it.wanted(l0, N);
            }
            l0 = item.begin(i) + pi * a.P;
            return lane < boxes && l0 < item.end(i) && (KIND == kWhole || item.it.wanted(l0, a.P));
        };
        auto page_of = [&](int q) {
            int page = -1, l0;
            if (KIND == kPacked && q < n && item.packed(w.tile + q)) {
                if (wants(w.tile + q, l0)) page = a.table4[(int64_t)item.b * a.max_pages4 + (l0 >> a.page_shift)];
            } else {
                page = a.pages;  // past the pool: reads as zeros
                if (q < n && wants(w.tile + q, l0)) page = table[(KIND == kWhole ? l0 : l0 - item.it.s.pk) >> a.page_shift];
            }
            return page;
        };
        int page = page_of(0);
        for (int q = 0; q < n; ++q, ++u, at.next(slots)) {
            const int next = page_of(q + 1);
            int l0;
            if (KIND == kPacked && item.packed(w.tile + q)) {
                const bool wanted = wants(w.tile + q, l0), good = wanted && page >= 0 && page < a.pages4;
                if (keys && wanted && !good) atomicOr(a.status, kStBadIndex);
                const uint32_t have = __ballot_sync(0xffffffffu, good);
                const uint32_t subs = item.subs(w.tile + q);
                copied += subs;
                if (copied > raws && !expanded(copied - raws)) goto out;
                if (lane < subs) {
                    const uint32_t mine = have >> (lane * (64 / N)) & ((1u << (64 / N)) - 1), rs = (copied - subs + lane) % raws;
                    raw_have[rs] = mine;
                    bar_expect(&raw_full[rs], __popc(mine) * (codes + marks));
                }
                __syncwarp();
                if (good) {
                    const uint32_t rs = (copied - subs + my_half) % raws, to = raw_to + rs * S::kRawUnit;
                    const uint8_t* src = a.packed.data + page * a.packed.page + h * a.packed.head + my_block;
                    bulk_copy(to + my_place * codes, src, codes, &raw_full[rs]);
                    bulk_copy(to + S::kRawScales + my_place * marks, src + my_marks, marks, &raw_full[rs]);
                }
                __syncwarp();
                page = next;
                continue;
            }
            // (a phase of `empty` may be waited for only when the one before it has ended: the warps that expanded the tiles
            // up to here have met it)
            if (KIND == kPacked && !expanded(copied)) goto out;
            if (u >= slots && !bar_wait(&empty[at.slot], at.parity ^ 1, c)) goto out;
            if (lane == 0) bar_expect(&full[at.slot], S::kUnit);
            __syncwarp();
            if (page < 0 || page > a.pages) {
                if (keys) atomicOr(a.status, kStBadIndex);
                page = a.pages;
            }
            if (lane < boxes) {
                if (keys && page == a.pages && wants(w.tile + q, l0)) atomicOr(a.status, kStBadIndex);
                tma_tile(smem_u32(ring + at.slot * S::kUnit + half * 16384 + pi * a.P * 128), map, half * 64, h, page, &full[at.slot]);
            }
            page = next;
        }
        w.next(per);
    }
out:
    // no copy is in flight when the CTA ends, and no arrival of a product that read one
    for (; seen < copied; ++seen) bar_wait<true>(&raw_empty[seen % raws], (seen / raws) & 1, c);
    for (uint32_t x = u > slots ? u - slots : 0; x < u; ++x) {
        bar_wait<true>(&full[x % slots], (x / slots) & 1, c);
        bar_wait<true>(&empty[x % slots], (x / slots) & 1, c);
    }
}

// Products of a tile in the issuing warps' code: how many of the four stand one behind the other, the rest a loop, because
// the loops of all roles together have to stay in the instruction cache.  64 trees of 61 tokens with 1, 2, 4: over packed
// pages 388, 367 and 438 us, in windows 169, 163 and 158; 32 single tokens in a window, where a stream has one
// half of a tile, 43.5, 45.2 and 45.7.
template <int KIND, bool PAIR> constexpr int kProductUnroll = KIND == kWhole ? 4 : KIND == kPacked ? 2 : PAIR ? 4 : 1;

// Which streams have a product with half `sub` of a tile that has `subs` halves.
template <bool PAIR> __device__ __forceinline__ bool tc_has(int st, int sub, int subs, bool second) {
    return PAIR ? sub < subs && (st == 0 || second) : st == sub && sub < subs;
}

// The score products of both streams, tile after tile.
template <int D, bool PAIR, int KIND>
__device__ __forceinline__ void tc_scores(const AttendArgs& a, TcControl& c, char* q_smem, char* k_ring) {
    using S = TcShape<D, PAIR, KIND>;
    const int lane = threadIdx.x & 31;
    const int rows = a.T * a.G, item_rows = PAIR ? 256 : 128, groups = (rows + item_rows - 1) / item_rows,
              per = tc_per<KIND>(a, groups);
    const uint32_t t_s = uniform(c.tmem), q_at = uniform(smem_u32(q_smem)), ring = uniform(smem_u32(k_ring));
    uint32_t items = 0, done0 = 0, done1 = 0;  // products of both streams
    // windows and packed pages: a scale below 0 turns the queries' signs here, not those of the scores in the softmax groups,
    // which need the room in the instruction cache (64 trees in windows 158 us, two prompt pieces 111, so 155 and 107; without
    // windows or packed pages 241 as it is, so 245)
    const uint32_t s_desc =
        KIND == kWhole ? mma_desc(kSub, false) : uniform(mma_desc(kSub, false) | (a.scale_log2 < 0.0f ? kNegateA : 0u));
    TcSlot at;
    for (TcWalk w(c.cut); w.more(); ++items) {
        const TcItem<KIND> item(a, w.b, w.item, groups, item_rows);
        item.open(w);
        const int n = w.n;
        const bool second = PAIR && item.r0 + 128 < rows;  // stream 1 has rows
        if (!bar_wait(&c.q_ready, items & 1, c)) goto out;
        tc_fence_after();
        if (lane == 0) bar_arrive(&c.q_taken);
        for (int q = 0; q < n; ++q, at.next(S::kK)) {
            const int subs = item.subs(w.tile + q);
            if (!bar_wait(&c.full_k[at.slot], at.parity, c)) goto out;
            // (stream 0's scores of a tile before stream 1's: stream 1's waits for values at clean() rest on it)
#pragma unroll (kProductUnroll<KIND, PAIR>)
            for (int x = 0; x < 4; ++x) {
                const int sub = x >> 1, st = x & 1;
                if (!tc_has<PAIR>(st, sub, subs, second)) continue;
                // the buffer's last weights have been read
                const uint32_t d = st ? done1 : done0, buf = d & 1;
                if (d > 1 && !bar_wait(&c.pv_done[st][buf], (d / 2 - 1) & 1, c)) goto out;
                if (st) ++done1;
                else ++done0;
                tc_fence_after();
                const uint32_t s_at = uniform(t_s + st * 128 + 64 * buf);
                const uint64_t q_desc = smem_desc(uniform(q_at + (PAIR ? st * S::kQ : 0)), 16, 1024);
                const uint64_t k_desc = smem_desc(uniform(ring + at.slot * S::kUnit + sub * kSub * 128), 16, 1024);
                const uint32_t bar = uniform(smem_u32(&c.s_full[st][buf]));
                if (elect_one()) {
#pragma unroll (KIND == kWhole ? D / 64 : 1)
                    for (int z = 0; z < D / 64; ++z)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t off = (z * 16384 + i * 32) / 16;  // (addresses count 16 bytes, in the low bits)
                            mma_ss(s_at, q_desc + off, k_desc + off, s_desc, z + i > 0);
                        }
                    tc_commit_at(bar);
                }
                __syncwarp();
            }
            if (elect_one()) tc_commit(&c.empty_k[at.slot]);
            __syncwarp();
        }
        w.next(per);
    }
out:
    // nothing is in flight when the CTA ends
    __syncwarp();
    if (elect_one()) tc_commit(&c.drained[0]);
    __syncwarp();
    bar_wait<true>(&c.drained[0], 0, c);
}

// The products of weights and values of both streams.
template <int D, bool PAIR, int KIND>
__device__ __forceinline__ void tc_sums(const AttendArgs& a, TcControl& c, char* v_ring) {
    using S = TcShape<D, PAIR, KIND>;
    const int rows = a.T * a.G, item_rows = PAIR ? 256 : 128, groups = (rows + item_rows - 1) / item_rows,
              per = tc_per<KIND>(a, groups);
    const uint32_t t_s = uniform(c.tmem), ring = uniform(smem_u32(v_ring));
    uint32_t done0 = 0, done1 = 0;
    TcSlot at;
    for (TcWalk w(c.cut); w.more();) {
        const TcItem<KIND> item(a, w.b, w.item, groups, item_rows);
        item.open(w);
        const int n = w.n;
        const bool second = PAIR && item.r0 + 128 < rows;
        uint32_t begun = 0;  // streams with sums
        for (int q = 0; q < n; ++q, at.next(S::kV)) {
            const int subs = item.subs(w.tile + q);
            // 16 bits: a line a token, the second half's lines behind the first's; packed: a line a channel, the second half of
            // the tokens behind the first
            const bool packed = KIND == kPacked && item.packed(w.tile + q);
            const uint32_t half_bytes = KIND == kPacked ? uniform(packed ? D * 128 : kSub * 128) : kSub * 128;
            const uint32_t step = KIND == kPacked ? uniform(packed ? 32 / 16 : 2048 / 16) : 2048 / 16;
            const uint32_t lead = KIND == kPacked ? uniform(packed ? 16 : 16384) : 16384;
            const uint32_t desc = KIND == kPacked ? uniform(packed ? mma_desc(D, false) : mma_desc(D, true)) : mma_desc(D, true);
            if (!bar_wait(&c.full_v[at.slot], at.parity, c)) goto out;
#pragma unroll (kProductUnroll<KIND, PAIR>)
            for (int x = 0; x < 4; ++x) {
                const int sub = x >> 1, st = x & 1;
                if (!tc_has<PAIR>(st, sub, subs, second)) continue;
                const uint32_t d = st ? done1 : done0, buf = d & 1;
                if (!bar_wait(&c.p_ready[st][buf], (d / 2) & 1, c)) goto out;
                if (st) ++done1;
                else ++done0;
                tc_fence_after();
                const uint32_t p_at = uniform(t_s + st * 128 + 64 * buf), o_at = uniform(t_s + S::kO + st * D);
                const uint64_t v_desc = smem_desc(uniform(ring + at.slot * S::kUnit + sub * half_bytes), lead, 1024);
                const uint32_t add = uniform(begun >> st & 1);  // the first of an item starts the sums
                const uint32_t bar = uniform(smem_u32(&c.pv_done[st][buf]));
                begun |= 1u << st;
                if (elect_one()) {
#pragma unroll
                    for (int i = 0; i < kSub / 16; ++i) mma_ts(o_at, p_at + 8 * i, v_desc + i * step, desc, i > 0 || add);
                    tc_commit_at(bar);
                }
                __syncwarp();
            }
            if (elect_one()) tc_commit(&c.empty_v[at.slot]);
            __syncwarp();
        }
        w.next(per);
    }
out:
    __syncwarp();
    if (elect_one()) tc_commit(&c.drained[1]);
    __syncwarp();
    bar_wait<true>(&c.drained[1], 0, c);
}

// Packed tiles into both rings, as the products read them: two warps the keys (a line a token), two the values (a
// line a channel, so that the tokens, whose pairs share a word, lie side by side).  A warp takes every second pair of
// patches of 32 tokens and 32 channels; lanes of even r take the first patch of a pair first, the others the second,
// which keeps the stores of eight lanes in different banks.  Rolled loops: with all patches of a tile unrolled the code was
// longer than what the instruction caches hold beside the other warps' (64 trees of 61 tokens: 927 us), and with the look-ups
// and copies in these warps they held the products up (835 us).
template <int D, bool PAIR>
__device__ __forceinline__ void tc_expand(const AttendArgs& a, TcControl& c, bool keys, char* ring, const char* raw) {
    using S = TcShape<D, PAIR, kPacked>;
    constexpr int X = D / 32;
    unsigned long long* const full = keys ? c.full_k : c.full_v;
    unsigned long long* const empty = keys ? c.empty_k : c.empty_v;
    unsigned long long* const raw_full = c.raw_full[keys ? 0 : 1];
    unsigned long long* const raw_empty = c.raw_empty[keys ? 0 : 1];
    const uint32_t* const raw_have = c.raw_have[keys ? 0 : 1];
    const uint32_t slots = keys ? S::kK : S::kV, raws = keys ? S::kRawK : S::kRawV;
    const int lane = threadIdx.x & 31, r = lane >> 2, t4 = lane & 3, half = threadIdx.x >> 5 & 1;
    const int rows = a.T * a.G, item_rows = PAIR ? 256 : 128, groups = (rows + item_rows - 1) / item_rows,
              per = tc_per<kPacked>(a, groups);
    const int N = packed_tokens(a.P), codes = N * D / 2, marks = keys ? D : N * D / 32;  // bytes of a block's codes, scales
    // the lane's place in the codes and scales of a run of 32 tokens (two blocks of 16, or one), its first patch of 32 channels
    const int sub = N == 16 ? (keys ? r >> 2 : t4 >> 1) : 0, in_run = 32 / N;
    const int code_at = sub * codes + (keys ? ((N == 16 ? r & 3 : r) * 4 + t4) * 16
                                            : (r * (N / 8) + (N == 16 ? t4 & 1 : t4)) * 16);
    const int scale_at = S::kRawScales + sub * marks + (keys ? 8 * t4 : 8 * (N == 16 ? t4 & 1 : t4));
    TcSlot at, from_at;  // of the tiles' ring, and of the packed halves'
    uint32_t u = 0;
    for (TcWalk w(c.cut); w.more(); w.next(per)) {
        const TcItem<kPacked> item(a, w.b, w.item, groups, item_rows);
        item.open(w);
        for (int q = 0; q < w.n; ++q, ++u, at.next(slots)) {
            if (u >= slots && !bar_wait(&empty[at.slot], at.parity ^ 1, c)) return;
            const bool packed = item.packed(w.tile + q);
            const int halves = packed ? item.subs(w.tile + q) : 0;
#pragma unroll 1
            for (int hf = 0; hf < halves; ++hf, from_at.next(raws)) {
                const uint32_t rs = from_at.slot;
                if (!bar_wait(&raw_full[rs], from_at.parity, c)) return;
                const uint32_t have = raw_have[rs];
                const char* from = raw + rs * S::kRawUnit;
                char* tile = ring + at.slot * S::kUnit;
#pragma unroll 1
                for (int i = 0; i < X; ++i) {
                    // keys: neighbouring patches of channels, values: of tokens
                    const int second = (i ^ r) & 1, pair = 2 * (i / 2) + half;
                    const int run = keys ? pair / (X / 2) : second, x = keys ? 2 * (pair % (X / 2)) + second : pair;
                    uint4 words = *reinterpret_cast<const uint4*>(from + run * in_run * codes + code_at + N * 16 * x);
                    uint2 bytes = *reinterpret_cast<const uint2*>(from + run * in_run * marks + scale_at + (keys ? 32 : N) * x);
                    if (!((have >> (run * in_run + sub)) & 1)) {
                        words = make_uint4(kPackedZero, kPackedZero, kPackedZero, kPackedZero);
                        bytes = make_uint2(0, 0);
                    }
                    uint32_t s[4], o[4], d[4][4];
                    packed_scales(bytes, s, o);
                    packed_words(words, s, o, d);
                    // rows: the tile's tokens, or the channels; octets of the other
                    const int row0 = (keys ? 64 * hf + 32 * run : 32 * x) + 8 * (r >> 1) + (r & 1);
                    const int octet = keys ? 4 * x + t4 : 4 * run + t4;
                    char* line = tile + (keys ? (octet >> 3) * 16384 : hf * D * 128) + row0 * 128;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        *reinterpret_cast<uint4*>(line + 256 * k + (((octet & 7) ^ ((row0 + 2 * k) & 7)) << 4)) =
                            make_uint4(d[k][0], d[k][1], d[k][2], d[k][3]);
                }
                bar_arrive_warp(&raw_empty[rs]);
            }
            if (packed) {
                fence_async();
                if (half == 0) bar_arrive_warp(&full[at.slot]);  // in the loading warp's place
            }
            bar_arrive_warp(&full[at.slot]);
        }
    }
}

template <int D, bool PAIR, int KIND>
__global__ void __launch_bounds__(tc_threads(KIND), 1)
    attend_tc_kernel(const AttendArgs a, const __grid_constant__ CUtensorMap key, const __grid_constant__ CUtensorMap value) {
    using S = TcShape<D, PAIR, KIND>;
    extern __shared__ char raw[];
    char* base = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
    char* q_smem = base;
    char* k_ring = q_smem + S::kQueries;
    char* v_ring = k_ring + S::kK * S::kUnit;
    char* merge = v_ring + S::kV * S::kUnit;
    char* raw_ring = merge + S::kMerge;
    TcControl& c = *reinterpret_cast<TcControl*>(raw_ring + (S::kRawK + S::kRawV) * S::kRawUnit);
    const int warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        constexpr int fill = KIND == kPacked ? 3 : 1;  // the loading warp, and two that expand
        for (int i = 0; i < S::kK; ++i) {
            bar_init(&c.full_k[i], fill);
            bar_init(&c.empty_k[i], 1);
        }
        for (int i = 0; i < S::kV; ++i) {
            bar_init(&c.full_v[i], fill);
            bar_init(&c.empty_v[i], 1);
        }
        for (int i = 0; KIND == kPacked && i < 8; ++i) {
            bar_init(&c.raw_full[i / 4][i % 4], 1);
            bar_init(&c.raw_empty[i / 4][i % 4], 2);
        }
        for (int i = 0; i < 2; ++i) {
            for (int buf = 0; buf < 2; ++buf) {
                bar_init(&c.s_full[i][buf], 1);
                bar_init(&c.p_ready[i][buf], 4);
                bar_init(&c.pv_done[i][buf], 1);
            }
            bar_init(&c.drained[i], 1);
        }
        bar_init(&c.q_ready, 8);
        bar_init(&c.q_taken, 1);
        bar_init(&c.all_sync, 8);
        c.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    grid_dependency_begin();
    if (warp == 8) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&c.tmem)), "r"(512)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (warp == 9) {
        const int rows = a.T * a.G, item_rows = PAIR ? 256 : 128, groups = (rows + item_rows - 1) / item_rows;
        AttendCut cut;
        if constexpr (KIND == kWhole)
            cut = attend_cut<kTile>(a, a.H * groups, blockIdx.x);
        else
            cut = attend_cut_over(a, a.B * groups, a.H, blockIdx.x, [&](int i) {
                return LongItem<kTile>(a, i / groups, i % groups * item_rows, item_rows).n;
            });
        if ((threadIdx.x & 31) == 0) c.cut = cut;
    }
    if (threadIdx.x == 0) a.join[blockIdx.x] = make_int4(0, 0, 0, 0);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp < 8) {
        if (KIND == kPacked) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        tc_softmax<D, PAIR, KIND>(a, c, q_smem, v_ring, merge, warp >> 2);
    } else if (warp < 12) {
        if (KIND == kPacked) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kIssueRegs));
        char* raw_values = raw_ring + S::kRawK * S::kRawUnit;
        if (KIND == kWhole && warp == 8) {  // (code of its own: 32 single tokens 168 us, with the other's 171)
            tc_load<D, PAIR, KIND>(a, c, true, &key, k_ring, raw_ring);
        } else if (warp == 8 || warp == 11) {
            const bool keys = KIND != kWhole && warp == 8;
            tc_load<D, PAIR, KIND>(a, c, keys, keys ? &key : &value, keys ? k_ring : v_ring, keys ? raw_ring : raw_values);
        } else if (warp == 9) tc_scores<D, PAIR, KIND>(a, c, q_smem, k_ring);
        else tc_sums<D, PAIR, KIND>(a, c, v_ring);
    } else if constexpr (KIND == kPacked) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kExpandRegs));
        const bool keys = warp < 14;
        tc_expand<D, PAIR>(a, c, keys, keys ? k_ring : v_ring, keys ? raw_ring : raw_ring + S::kRawK * S::kRawUnit);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 8) {
        tc_fence_after();
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(c.tmem), "r"(512));
        if (c.abort && (threadIdx.x & 31) == 0) atomicOr(a.status, kStInternal);
    }
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encode_fn() {
    static const EncodeFn fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult how;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &how) != cudaSuccess ||
            how != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeFn>(p);
    }();
    return fn;
}

// [page][head][token][D] with any strides, a page of one head and 64 elements a box.
bool encode(CUtensorMap* map, const AttendArgs& a, void* base, int64_t page, int64_t head, int64_t token) {
    const EncodeFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)a.D, (cuuint64_t)a.P, (cuuint64_t)a.H, (cuuint64_t)a.pages};
    const cuuint64_t strides[3] = {(cuuint64_t)token * 2, a.H == 1 ? 16 : (cuuint64_t)head * 2,
                                   a.pages == 1 ? 16 : (cuuint64_t)page * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)a.P, 1, 1}, one[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, base, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool PAIR, int KIND> cudaError_t launch_tc(const AttendArgs& a, cudaStream_t s) {
    CUtensorMap key, value;
    if (!encode_fn()) return cudaErrorNotSupported;
    if (!encode(&key, a, a.kv.key, a.kv.key_page, a.kv.key_head, a.kv.key_token) ||
        !encode(&value, a, a.kv.value, a.kv.value_page, a.kv.value_head, a.kv.value_token))
        return cudaErrorInvalidValue;
    constexpr size_t smem = tc_smem_bytes<D, PAIR, KIND>();
    static_assert(smem <= 227 * 1024);
    if (KIND == kPacked) {
        // the groups' registers are taken from what the block was launched with: less would leave a group waiting
        static const int regs = [] {
            cudaFuncAttributes f;
            return cudaFuncGetAttributes(&f, attend_tc_kernel<D, PAIR, KIND>) == cudaSuccess ? f.numRegs : 0;
        }();
        if (regs < kPackedLaunchRegs) return cudaErrorNotSupported;
    }
    cudaError_t err = cudaFuncSetAttribute(attend_tc_kernel<D, PAIR, KIND>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (err != cudaSuccess) return err;
    return launch_dependent(attend_tc_kernel<D, PAIR, KIND>, dim3(a.ctas), dim3(tc_threads(KIND)), smem, s, a, key, value);
}

template <int KIND> cudaError_t launch_tc_kind(const AttendArgs& a, cudaStream_t s) {
    const bool pair = (int64_t)a.T * a.G > 128;
    if (a.D == 64) return pair ? launch_tc<64, true, KIND>(a, s) : launch_tc<64, false, KIND>(a, s);
    return pair ? launch_tc<128, true, KIND>(a, s) : launch_tc<128, false, KIND>(a, s);
}

}  // namespace

cudaError_t launch_attend_tc(const AttendArgs& a, cudaStream_t s) { return launch_tc_kind<kWhole>(a, s); }
cudaError_t launch_window_tc(const AttendArgs& a, cudaStream_t s) { return launch_tc_kind<kWindow>(a, s); }
cudaError_t launch_packed_tc(const AttendArgs& a, cudaStream_t s) { return launch_tc_kind<kPacked>(a, s); }

}  // namespace rheo
