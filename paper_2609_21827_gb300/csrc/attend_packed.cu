// attend_packed.cu -- attention of few query rows over packed pages and the 16-bit
// ones behind them.
//
// An item is up to 8 NT query rows (token, head of the key/value head) of a request and
// its tiles of 32 places.  A CTA is four warps, of which each takes every fourth tile, with running maxima,
// sums and outputs of its own; they are joined in shared memory at the item's end.  Three or four
// CTAs an SM, so that the others have work where one begins or ends an item.  A warp looks
// up 32 of its packed tiles at a time (a lane each) and has the next one copied (a bulk copy, as a
// block is contiguous) while it works on one.
// Both products are taken with the cache as the first operand of m16n8k16, so
// that the few query rows fill its 8 columns: S^T = K Q^T (16 places x 8 rows), O^T = V^T P^T
// (16 channels x 8 rows).  A lane's 16 bytes of a packed block are four rows of that
// operand, and become bf16 in its registers, never in memory (packed.cuh).  The weights
// turn from accumulators into the second operand by an 8 x 8 transposition (movmatrix).
// Places in 16 bits are read straight into the same registers, values by the same transposition.
// The reference m of a row follows its largest score when that has grown by more than kSlack in
// log2 units; p <= 2^kSlack until then.
//
// Places that a row does not see get -inf before the maximum.  16-bit values that are
// not finite count as 0 where some row may not see their place (0 * inf would
// spoil it) and are added at the item's end for the rows that see them.
//
// What bounds it: instructions.  32 single tokens, contexts to 16,201, 32 query and 8 key/value heads of 128: 75 us,
// 3.9 TB/s (57 % of a copy's rate), some 730 instructions a tile, 51 % of what the SMs can issue in that time, more than half
// of which turn numbers into bf16 (a shift, a logic operation and a multiply-add a pair, on pipes of half rate).  48 chains
// of three tokens, heads of 64, a window of 8,192: 51 us.  With the tensor cores' kernel, whose tiles have 128 rows, these
// take 251 and 142 us.  Items of 16 rows spill registers (256 bytes of stores a thread with heads of 64, 360 with heads of 128,
// which single tokens do not but for 24): chains of 5 and 8, four rows each, 32 requests, contexts to 8,201: 110 and 116 us.
// (Over 16 bits alone the tensor cores' kernel is quicker, as nothing is to be turned: 32 single tokens in a window of 1,024
// take it 43 us, this one 53.)
#include <cuda_bf16.h>

#include "attend.cuh"
#include "packed.cuh"
#include "rheo_kernels.h"

namespace rheo {
namespace {

constexpr int kTile = 32;            // places a tile
constexpr int kWarps = 4;            // of a CTA
constexpr int kThreads = 32 * kWarps;
constexpr int kSlots = 2;            // of a warp
constexpr float kSlack = 8.0f;
constexpr int kWaitLimit = 1 << 22;  // polls of a wait before the kernel gives up

template <int D, int NT> struct Few {
    static constexpr int kPerSm = few_per_sm(D);
    static constexpr int kX = D / 32;
    static constexpr int kRows = 8 * NT;
    static constexpr int kSlot = packed_block_bytes(16, D) * 2;  // the larger of one block of 32 tokens and two of 16
    static constexpr int kLine = D + 1;                          // floats of a row in a warp's sums: no bank twice
    static_assert(packed_block_bytes(32, D) <= kSlot && kSlot % 16 == 0);
};

template <int D, int NT> struct FewSmem {
    using F = Few<D, NT>;
    alignas(16) unsigned char slot[kWarps][kSlots][F::kSlot];
    float o[kWarps][F::kRows * F::kLine];
    float2 ml[kWarps][F::kRows];
    unsigned long long full[kWarps][kSlots];
    AttendCut cut;
    int abort;
    int odd[2];  // some value that is not finite was left out, of items in turn
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(unsigned long long* b, int count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(unsigned long long* b, int bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(b)), "r"(bytes) : "memory");
}
// Waits for the phase of this parity to end (whole warps); false, for all lanes, after kWaitLimit polls or where another
// warp gave up.  A drain (DRAIN) goes on where another warp gave up.
template <bool DRAIN = false> __device__ __forceinline__ bool bar_wait(unsigned long long* b, uint32_t parity, int* abort) {
    uint32_t done = 0;
    for (int i = 0; i < kWaitLimit && !done; ++i) {
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(done)
            : "r"(smem_u32(b)), "r"(parity)
            : "memory");
        if (!DRAIN && (i & 255) == 255 && *(volatile int*)abort) break;
    }
    if (__all_sync(0xffffffffu, done)) return true;
    *(volatile int*)abort = 1;
    return false;
}
__device__ __forceinline__ void bulk_copy(void* dst, const void* src, int bytes, unsigned long long* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
                 "l"(src), "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Elements of a pair that are not finite.
__device__ __forceinline__ uint32_t odd_mask(uint32_t w) {
    return ((w & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((w & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
}
// Part i (row f(r, i)) and pair p (elements 2p, 2p + 1 of the lane's eight) of a 32 x 32 operand: two products of 16
// rows, two steps of 16 along the sum.
__device__ __forceinline__ void feed(float (&c0)[4], float (&c1)[4], const uint32_t (&d)[4][4], const uint32_t (&b)[4]) {
    mma(c0, d[0][0], d[1][0], d[0][1], d[1][1], b[0], b[1]);
    mma(c1, d[2][0], d[3][0], d[2][1], d[3][1], b[0], b[1]);
    mma(c0, d[0][2], d[1][2], d[0][3], d[1][3], b[2], b[3]);
    mma(c1, d[2][2], d[3][2], d[2][3], d[3][3], b[2], b[3]);
}
__device__ __forceinline__ int quad_row(int r, int i) { return 8 * (r >> 1) + (r & 1) + 2 * i; }

template <int D, int NT>
__global__ void __launch_bounds__(kThreads, Few<D, NT>::kPerSm) packed_few_kernel(const AttendArgs a) {
    using F = Few<D, NT>;
    extern __shared__ __align__(128) unsigned char raw_smem[];
    FewSmem<D, NT>& sm = *reinterpret_cast<FewSmem<D, NT>*>(raw_smem);
    const int tid = threadIdx.x, lane = tid & 31, r = lane >> 2, t4 = lane & 3;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);  // (known to be the same in all lanes)
    const int rows = a.T * a.G, groups = (rows + F::kRows - 1) / F::kRows;
    if (tid == 0) {
        for (int i = 0; i < kWarps * kSlots; ++i) bar_init(&sm.full[0][i], 1);
        sm.abort = sm.odd[0] = sm.odd[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    grid_dependency_begin();
    if (warp == 0) {
        const AttendCut cut = attend_cut_over(a, a.B * groups, a.H, blockIdx.x, [&](int c) {
            return LongItem<kTile>(a, c / groups, c % groups * F::kRows, F::kRows).n;
        });
        if (lane == 0) {
            sm.cut = cut;
            a.join[blockIdx.x] = make_int4(0, 0, 0, 0);
        }
    }
    __syncthreads();
    const int N = packed_tokens(a.P), block_bytes = packed_block_bytes(N, D);
    // where this lane's pieces of a tile lie: its keys' block and its values' one (two blocks of 16 tokens, or the same of 32)
    const int k_block = N == 16 ? (r >> 2) * block_bytes : 0, v_block = N == 16 ? (t4 >> 1) * block_bytes : 0;
    const int k_at = k_block + ((N == 16 ? r & 3 : r) * 4 + t4) * 16, k_step = N * 16;  // from 32 channels to the next
    const int v_at = v_block + N * D / 2 + (r * (N / 8) + (N == 16 ? t4 & 1 : t4)) * 16, v_step = N * 16;
    const int ks_at = k_block + N * D + 8 * t4, vs_at = v_block + N * D + D + 8 * (N == 16 ? t4 & 1 : t4);
    const int blocks = kTile / N;
    uint32_t items = 0, ahead = 0, done = 0;  // items, copies begun and waited for; the k-th copy goes to slot k % kSlots
    // Copies of one tile's blocks, which lie at src0 and src1 (of 32 tokens: one); 0: not there, zeros
    auto copy = [&](unsigned long long src0, unsigned long long src1) {
        const uint32_t k = ahead++ % kSlots;
        unsigned char* to = sm.slot[warp][k];
        if (src0 == 0 || (blocks == 2 && src1 == 0)) {
            for (int z = 0; z < blocks; ++z)
                for (int j = lane * 16; (z == 0 ? src0 : src1) == 0 && j < block_bytes; j += 512)
                    *reinterpret_cast<uint4*>(to + z * block_bytes + j) = make_uint4(kPackedZero, kPackedZero, kPackedZero, kPackedZero);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        __syncwarp();
        if (lane == 0) {
            const int n0 = src0 != 0, n1 = blocks == 2 && src1 != 0;
            bar_expect(&sm.full[warp][k], (n0 + n1) * block_bytes);
            if (n0) bulk_copy(to, reinterpret_cast<const void*>(src0), block_bytes, &sm.full[warp][k]);
            if (n1) bulk_copy(to + block_bytes, reinterpret_cast<const void*>(src1), block_bytes, &sm.full[warp][k]);
        }
        __syncwarp();
    };

    for (AttendWalk<kTile> w(sm.cut); w.more(); w.next(a.H)) {
        const int b = w.b / groups, g = w.b % groups, h = w.item, r0 = g * F::kRows;
        const LongItem<kTile> it(a, b, r0, F::kRows);
        w.open_tiles(it.n);
        if (it.s.bad && tid == 0) atomicOr(a.status, kStBadLength);
        const int to = w.tile + w.n, packed_to = min(to, it.packed_tiles());
        const int32_t* table = a.block_table + (int64_t)b * a.max_pages;

        // this warp's tiles: every kWarps-th from `at` on; the packed ones come first
        const int at = w.tile + warp;
        const bool mine = at < to;
        const int turns = at < packed_to ? (packed_to - at + kWarps - 1) / kWarps : 0;
        unsigned long long src[2] = {0, 0};  // where this lane's one of 32 packed tiles lies
        int asked = 0;                       // packed tiles of this item whose copies have begun
        auto copy_next = [&] {
            if (asked >= turns) return;
            if (asked % 32 == 0) {
                const int i = at + (asked + lane) * kWarps;
                src[0] = src[1] = 0;
                if (i < packed_to) {
                    const int place = it.number(i) * kTile;
                    const int32_t* table4 = a.table4 + (int64_t)b * a.max_pages4;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int l0 = place + k * N;
                        if (k >= blocks || l0 >= it.s.pk || !it.wanted(l0, N)) continue;
                        const int page = table4[l0 >> a.page_shift];
                        if (page < 0 || page >= a.pages4) atomicOr(a.status, kStBadIndex);
                        else
                            src[k] = (unsigned long long)(a.packed.data + page * a.packed.page + h * a.packed.head +
                                                          (l0 & (a.P - 1)) / N * block_bytes);
                    }
                }
                __syncwarp();
            }
            const unsigned long long src0 = __shfl_sync(0xffffffffu, src[0], asked & 31);
            copy(src0, blocks == 2 ? __shfl_sync(0xffffffffu, src[1], asked & 31) : 0);
            ++asked;
        };
        for (int k = 0; k < kSlots; ++k) copy_next();

        // queries: column r of the products
        uint32_t q[NT][F::kX][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int row = r0 + 8 * n + r, t = row / a.G;
            const bool live = row < rows && t < it.s.add;
            const char* src = static_cast<const char*>(a.io.q) +
                              (b * a.io.q_batch + t * a.io.q_token + (h * a.G + row - t * a.G) * a.io.q_head + 8 * t4) * 2;
#pragma unroll
            for (int x = 0; x < F::kX; ++x) {
                uint4 y = make_uint4(0, 0, 0, 0);
                if (live) y = *reinterpret_cast<const uint4*>(src + 64 * x);
                q[n][x][0] = y.x, q[n][x][1] = y.y, q[n][x][2] = y.z, q[n][x][3] = y.w;
            }
        }
        // rows 2 t4 and 2 t4 + 1 of the accumulators: token (below 0: none), first place of its window
        int token[NT][2], first[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int row = r0 + 8 * n + 2 * t4 + e, t = row / a.G;
                const bool live = row < rows && t < it.s.add;
                token[n][e] = live ? t : -1;
                first[n][e] = live && a.window ? long_first(a, it.s, long_depth(a, b, t)) : 0;
            }
        float o[NT][F::kX][2][4], m[NT][2], l[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m[n][0] = m[n][1] = -INFINITY;
            l[n][0] = l[n][1] = 0.0f;
#pragma unroll
            for (int x = 0; x < F::kX; ++x)
#pragma unroll
                for (int k = 0; k < 8; ++k) o[n][x][k / 4][k % 4] = 0.0f;
        }
        // Scores (of places f(r, k), rows 8 n + 2 t4 + e at s[n][k / 2][2 (k % 2) + e]) to weights, the second operand of the
        // values' product.
        auto weigh = [&](float (&s)[NT][2][4], uint32_t (&p)[NT][4], int place, int end, bool masked) {
            bool grow = false;
            float top[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int k = 0; k < 8; ++k) s[n][k / 4][k % 4] *= a.scale_log2;
            if (masked) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int l0 = place + quad_row(r, k / 2), t = token[n][k % 2];
                        const uint8_t* mrow = a.mask ? a.mask + ((int64_t)b * a.T + max(t, 0)) * a.T : nullptr;
                        if (t < 0 || l0 >= end || !it.sees(a, b, mrow, t, first[n][k % 2], l0)) s[n][k / 4][k % 4] = -INFINITY;
                    }
                __syncwarp();
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    top[n][e] = fmaxf(fmaxf(s[n][0][e], s[n][0][2 + e]), fmaxf(s[n][1][e], s[n][1][2 + e]));
                    // (a reference of -inf: the comparison holds for anything above it)
                    grow |= top[n][e] > m[n][e] + kSlack;
                }
            if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float y = fmaxf(top[n][e], m[n][e]);
#pragma unroll
                        for (int z = 4; z < 32; z <<= 1) y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, z));
                        const float f = m[n][e] == -INFINITY ? 1.0f : fast_exp2(m[n][e] - y);
                        m[n][e] = y;
                        l[n][e] *= f;
#pragma unroll
                        for (int x = 0; x < F::kX; ++x)
#pragma unroll
                            for (int k = 0; k < 2; ++k) o[n][x][k][e] *= f, o[n][x][k][2 + e] *= f;
                    }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float ref0 = m[n][0] == -INFINITY ? 0.0f : m[n][0], ref1 = m[n][1] == -INFINITY ? 0.0f : m[n][1];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float p0 = fast_exp2(s[n][k / 2][2 * (k % 2)] - ref0), p1 = fast_exp2(s[n][k / 2][2 * (k % 2) + 1] - ref1);
                    l[n][0] += p0;
                    l[n][1] += p1;
                    p[n][k] = transposed(pack_bf16(p0, p1));
                }
            }
        };
        // ---- in 16 bits: first, as their loads wait for one another
        for (int i = at + turns * kWarps; i < to; i += kWarps) {
            const int number = it.number(i), place = it.begin(number), end = it.end(number);
            const bool masked = place + kTile > min(end, it.s.ctx) || place < it.lo_most;
            int page[4];  // of this lane's places; -1 where there is none to read
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int l0 = place + quad_row(r, k);
                page[k] = l0 < end && it.wanted(l0, 1) ? table[(l0 - it.s.pk) >> a.page_shift] : -1;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int l0 = place + quad_row(r, k);
                if (l0 < end && it.wanted(l0, 1) && (page[k] < 0 || page[k] >= a.pages)) {
                    atomicOr(a.status, kStBadIndex);
                    page[k] = -1;
                }
            }
            __syncwarp();
            // 32 channels of the places' lines (a load under a condition would wait for the one before: what is not there is
            // read from page 0)
            auto line = [&](const void* base, int64_t page_stride, int64_t head_stride, int64_t token_stride, int k, int x) {
                const int row = (place + quad_row(r, k) - it.s.pk) & (a.P - 1);
                const uint4 y = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(base) +
                                                                max(page[k], 0) * page_stride + h * head_stride +
                                                                row * token_stride + 8 * t4 + 32 * x);
                return page[k] < 0 ? make_uint4(0, 0, 0, 0) : y;
            };
            float s[NT][2][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int k = 0; k < 8; ++k) s[n][k / 4][k % 4] = 0.0f;
#pragma unroll
            for (int x = 0; x < F::kX; ++x) {
                uint32_t d[4][4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint4 y = line(a.kv.key, a.kv.key_page, a.kv.key_head, a.kv.key_token, k, x);
                    d[k][0] = y.x, d[k][1] = y.y, d[k][2] = y.z, d[k][3] = y.w;
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) feed(s[n][0], s[n][1], d, q[n][x]);
            }
            uint32_t p[NT][4];
            weigh(s, p, place, end, masked);
            bool odd = false;
#pragma unroll
            for (int x = 0; x < F::kX; ++x) {
                uint32_t d[4][4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint4 y = line(a.kv.value, a.kv.value_page, a.kv.value_head, a.kv.value_token, k, x);
                    if (masked) {
                        const uint32_t z[4] = {odd_mask(y.x), odd_mask(y.y), odd_mask(y.z), odd_mask(y.w)};
                        odd |= (z[0] | z[1] | z[2] | z[3]) != 0;
                        y = make_uint4(y.x & ~z[0], y.y & ~z[1], y.z & ~z[2], y.w & ~z[3]);
                    }
                    d[0][k] = transposed(y.x), d[1][k] = transposed(y.y), d[2][k] = transposed(y.z), d[3][k] = transposed(y.w);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) feed(o[n][x][0], o[n][x][1], d, p[n]);
            }
            if (odd) sm.odd[items & 1] = 1;
        }

        // ---- packed
        for (int i = at; i < packed_to; i += kWarps) {
            const int number = it.number(i), place = number * kTile;
            const uint32_t k = done % kSlots;
            const unsigned char* from = sm.slot[warp][k];
            bar_wait(&sm.full[warp][k], (done / kSlots) & 1, &sm.abort);  // (where it fails the results do not count)
            float s[NT][2][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int z = 0; z < 8; ++z) s[n][z / 4][z % 4] = 0.0f;
#pragma unroll
            for (int x = 0; x < F::kX; ++x) {
                uint32_t sc[4], so[4], d[4][4];
                packed_scales(*reinterpret_cast<const uint2*>(from + ks_at + 32 * x), sc, so);
                packed_words(*reinterpret_cast<const uint4*>(from + k_at + k_step * x), sc, so, d);
#pragma unroll
                for (int n = 0; n < NT; ++n) feed(s[n][0], s[n][1], d, q[n][x]);
            }
            uint32_t p[NT][4];
            weigh(s, p, place, it.end(number), place + kTile > it.s.pk || place < it.lo_most);
#pragma unroll
            for (int x = 0; x < F::kX; ++x) {
                uint32_t sc[4], so[4], d[4][4];
                packed_scales(*reinterpret_cast<const uint2*>(from + vs_at + N * x), sc, so);
                packed_words(*reinterpret_cast<const uint4*>(from + v_at + v_step * x), sc, so, d);
#pragma unroll
                for (int n = 0; n < NT; ++n) feed(o[n][x][0], o[n][x][1], d, p[n]);
            }
            ++done;
            __syncwarp();
            copy_next();
        }

        // ---- the item's sums: every warp's into shared memory, then a thread four columns of a row
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int z = 4; z < 32; z <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], z);
                if (r == 0) sm.ml[warp][8 * n + 2 * t4 + e] = make_float2(mine ? m[n][e] : -INFINITY, l[n][e]);
                if (mine) {
                    float* to_row = &sm.o[warp][(8 * n + 2 * t4 + e) * F::kLine];
#pragma unroll
                    for (int x = 0; x < F::kX; ++x)
#pragma unroll
                        for (int k = 0; k < 4; ++k) to_row[32 * x + quad_row(r, k)] = o[n][x][k / 2][2 * (k % 2) + e];
                }
            }
        __syncthreads();
        const bool left_out = *(volatile int*)&sm.odd[items & 1] != 0;
        if (tid == 0) sm.odd[~items & 1] = 0;  // the next item's, read last before the sums of this one
        ++items;
        const bool whole = w.n == w.all;
        const int64_t part = attend_part(blockIdx.x, w.tile == 0);
        const int filled = min((int)kWarps, w.n);
        for (int k = tid; k < F::kRows * (D / 4); k += kThreads) {
            const int rr = k / (D / 4), c4 = k % (D / 4), row = r0 + rr, t = row / a.G, head = h * a.G + row - t * a.G;
            if (row >= rows) continue;
            float mm = -INFINITY, ll = 0.0f, y[4] = {0, 0, 0, 0};
            for (int z = 0; z < filled; ++z) mm = fmaxf(mm, sm.ml[z][rr].x);
            const float ref = mm == -INFINITY ? 0.0f : mm;
            for (int z = 0; z < filled; ++z) {
                const float2 x = sm.ml[z][rr];
                const float f = fast_exp2(x.x - ref);
                ll += f * x.y;
                const float* src = &sm.o[z][rr * F::kLine + 4 * c4];
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] += f * src[e];
            }
            if (t >= it.s.add) mm = -INFINITY, ll = 0.0f;
            if (left_out && t < it.s.add) {
                // values that are not finite, of the tiles at hand, for the rows that see them
                const uint8_t* mrow = a.mask ? a.mask + ((int64_t)b * a.T + t) * a.T : nullptr;
                const int first_place = a.window ? long_first(a, it.s, long_depth(a, b, t)) : 0;
                for (int i = max(w.tile, packed_to); i < to; ++i) {
                    const int number = it.number(i), place = it.begin(number), end = it.end(number);
                    if (!(place + kTile > min(end, it.s.ctx) || place < it.lo_most)) continue;  // nothing was left out there
                    for (int l0 = place; l0 < end; ++l0) {
                        if (!it.wanted(l0, 1) || !it.sees(a, b, mrow, t, first_place, l0)) continue;
                        const int x = l0 - it.s.pk, page = table[x >> a.page_shift];
                        if (page < 0 || page >= a.pages) continue;
                        const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(a.kv.value) + page * a.kv.value_page +
                                                 h * a.kv.value_head + (x & (a.P - 1)) * a.kv.value_token + 4 * c4;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float z = __bfloat162float(v[e]);
                            if (!(fabsf(z) < INFINITY)) y[e] += z;
                        }
                    }
                }
            }
            if (whole) {
                const float inv = ll == 0.0f ? 0.0f : 1.0f / ll;
                uint2 z = make_uint2(0, 0);
                if (ll != 0.0f) z = make_uint2(pack_bf16(y[0] * inv, y[1] * inv), pack_bf16(y[2] * inv, y[3] * inv));
                *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.io.out) + b * a.io.out_batch + t * a.io.out_token +
                                          head * a.io.out_head + 4 * c4) = z;
                if (a.io.lse && c4 == 0) a.io.lse[((int64_t)b * a.T + t) * a.H * a.G + head] = attend_lse(mm, ll);
            } else {
                reinterpret_cast<float4*>(a.part_o)[attend_part_at(a, part, rr, c4)] = make_float4(y[0], y[1], y[2], y[3]);
                if (c4 == 0) *reinterpret_cast<float2*>(a.part_ml + (part * a.part_rows + rr) * 2) = make_float2(mm, ll);
            }
        }
        if (!whole && w.tile == 0 && tid == 0)
            a.join[blockIdx.x] = make_int4(b, h * groups + g, w.segments(sm.cut, blockIdx.x), 0);
        __syncthreads();
    }
    // no copy is in flight when the CTA ends (all have been waited for, but where a wait failed)
    for (; done < ahead; ++done) bar_wait<true>(&sm.full[warp][done % kSlots], (done / kSlots) & 1, &sm.abort);
    if (tid == 0 && *(volatile int*)&sm.abort) atomicOr(a.status, kStInternal);
}

template <int D, int NT> cudaError_t launch_few(const AttendArgs& a, cudaStream_t s) {
    constexpr size_t smem = sizeof(FewSmem<D, NT>);
    static_assert((smem + 1024) * Few<D, NT>::kPerSm <= 228 * 1024);
    const cudaError_t err = cudaFuncSetAttribute(packed_few_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (err != cudaSuccess) return err;
    return launch_dependent(packed_few_kernel<D, NT>, dim3(a.ctas), dim3(kThreads), smem, s, a);
}

}  // namespace

cudaError_t launch_packed_attend(const AttendArgs& in, cudaStream_t s) {
    AttendArgs a = in;
    const int rows = a.T * a.G;
    if (rows > kFewRows) {
        const cudaError_t err = launch_packed_tc(a, s);
        return err != cudaSuccess ? err : launch_attend_join(a, 1, s);
    }
    const bool one = rows <= 8;
    a.item_rows = a.part_rows = few_item_rows(rows);
    a.ctas = kAttendCtas * few_per_sm(a.D);
    // What an item's start and end cost in tiles (32 single tokens, contexts to 16,201: 99.7, 89.7, 80.7, 80.9 us with 6, 12,
    // 24, 32), and the tiles of a part at least where few items are cut by themselves (one token over 16,201: 28.1, 26.1,
    // 25.6 us with 4, 8, 16).
    a.lead = 24;
    a.least = 16;
    const cudaError_t err = a.D == 64 ? (one ? launch_few<64, 1>(a, s) : launch_few<64, 2>(a, s))
                                      : (one ? launch_few<128, 1>(a, s) : launch_few<128, 2>(a, s));
    return err != cudaSuccess ? err : launch_attend_join(a, 1, s);
}

}  // namespace rheo
