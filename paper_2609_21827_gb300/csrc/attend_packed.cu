// attend_packed.cu -- attention of few query rows over packed pages and the 16-bit
// ones behind them.
//
// An item is up to 8 NT query rows (token, head of the key/value head) of a request and
// its tiles of 32 places.  A CTA an SM; one warp copies packed blocks into a ring of
// shared memory (one bulk copy each, a page of a head is contiguous), the others take
// every kWarps-th tile, each with running maxima, sums and outputs of its own, and are
// joined in shared memory at the item's end.
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
#include <cuda_bf16.h>

#include "attend.cuh"
#include "packed.cuh"
#include "rheo_kernels.h"

namespace rheo {
namespace {

constexpr int kTile = 32;            // places a tile
constexpr int kSlots = 32;           // of the ring
constexpr float kSlack = 8.0f;
constexpr int kWaitLimit = 1 << 22;  // polls of a wait before the kernel gives up

template <int D, int NT> struct Few {
    // Warps that take tiles: with the copying one 16, which leaves a thread 128 registers, or 8.
    static constexpr int kWarps = NT == 1 ? 15 : 7;
    static constexpr int kThreads = 32 * (kWarps + 1);
    static constexpr int kX = D / 32;
    static constexpr int kRows = 8 * NT;
    static constexpr int kSlot = packed_block_bytes(16, D) * 2;  // the larger of one block of 32 tokens and two of 16
    static constexpr int kLine = D + 1;                          // floats of a row in a warp's sums: no bank twice
    static_assert(packed_block_bytes(32, D) <= kSlot && kSlot % 16 == 0);
};

template <int D, int NT> struct FewSmem {
    using F = Few<D, NT>;
    alignas(16) unsigned char ring[kSlots][F::kSlot];
    float o[F::kWarps][F::kRows * F::kLine];
    float2 ml[F::kWarps][F::kRows];
    unsigned long long full[kSlots], empty[kSlots];
    AttendCut cut;
    int abort;
    int odd[2];  // some value that is not finite was left out, of items in turn
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(unsigned long long* b, int count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(unsigned long long* b) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(b)) : "memory");
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
    asm volatile(
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

// Copies the packed tiles of this CTA's items into the ring, in order; lane = tile of 32 at a time.
template <int D, int NT> __device__ __forceinline__ void few_load(const AttendArgs& a, FewSmem<D, NT>& sm) {
    using F = Few<D, NT>;
    const int lane = threadIdx.x & 31, N = packed_tokens(a.P), block_bytes = packed_block_bytes(N, D), blocks = kTile / N;
    const int rows = a.T * a.G, groups = (rows + F::kRows - 1) / F::kRows;
    uint32_t u = 0;
    bool fine = true;
    for (AttendWalk<kTile> w(sm.cut); w.more() && fine; w.next(a.H)) {
        const int b = w.b / groups, r0 = w.b % groups * F::kRows;
        const LongItem<kTile> it(a, b, r0, F::kRows);
        w.open_tiles(it.n);
        const int to = min(w.tile + w.n, it.packed_tiles());
        const int32_t* table = a.table4 + (int64_t)b * a.max_pages4;
        for (int i0 = w.tile; i0 < to && fine; i0 += 32) {
            // this lane's tile: where its blocks lie (null: not wanted, or a bad page)
            const uint8_t* src[2] = {nullptr, nullptr};
            if (i0 + lane < to) {
                const int place = it.begin(it.number(i0 + lane));
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int at = place + k * N;
                    if (k >= blocks || at >= it.s.pk || !it.wanted(at, N)) continue;
                    const int page = table[at >> a.page_shift];
                    if (page < 0 || page >= a.pages4) {
                        atomicOr(a.status, kStBadIndex);
                        continue;
                    }
                    src[k] = a.packed.data + page * a.packed.page + w.item * a.packed.head + (at & (a.P - 1)) / N * block_bytes;
                }
            }
            const uint32_t gone = __ballot_sync(0xffffffffu, !src[0] || (blocks == 2 && !src[1]));
            const int count = min(32, to - i0);
            for (int l = 0; l < count; ++l, ++u) {
                const uint32_t slot = u % kSlots;
                if (u >= kSlots && !bar_wait(&sm.empty[slot], (u / kSlots - 1) & 1, &sm.abort)) {
                    fine = false;
                    break;
                }
                if ((gone >> l) & 1) {  // blocks that are not there are zeros
                    const uint32_t has = __shfl_sync(0xffffffffu, (src[0] ? 1 : 0) | (src[1] ? 2 : 0), l);
                    for (int k = 0; k < blocks; ++k)
                        for (int j = lane * 16; !((has >> k) & 1) && j < block_bytes; j += 512)
                            *reinterpret_cast<uint4*>(&sm.ring[slot][k * block_bytes + j]) =
                                make_uint4(kPackedZero, kPackedZero, kPackedZero, kPackedZero);
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                }
                if (lane == l) {
                    bar_expect(&sm.full[slot], ((src[0] ? 1 : 0) + (src[1] ? 1 : 0)) * block_bytes);
                    if (src[0]) bulk_copy(&sm.ring[slot][0], src[0], block_bytes, &sm.full[slot]);
                    if (src[1]) bulk_copy(&sm.ring[slot][block_bytes], src[1], block_bytes, &sm.full[slot]);
                }
                __syncwarp();
            }
        }
    }
    // no copy is in flight when the CTA ends
    for (uint32_t x = u > kSlots ? u - kSlots : 0; x < u; ++x) bar_wait<true>(&sm.full[x % kSlots], (x / kSlots) & 1, &sm.abort);
}

template <int D, int NT>
__global__ void __launch_bounds__(Few<D, NT>::kThreads, 1) packed_few_kernel(const AttendArgs a) {
    using F = Few<D, NT>;
    extern __shared__ __align__(128) unsigned char raw_smem[];
    FewSmem<D, NT>& sm = *reinterpret_cast<FewSmem<D, NT>*>(raw_smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = lane >> 2, t4 = lane & 3;
    const int rows = a.T * a.G, groups = (rows + F::kRows - 1) / F::kRows;
    if (tid == 0) {
        for (int i = 0; i < kSlots; ++i) {
            bar_init(&sm.full[i], 1);
            bar_init(&sm.empty[i], 1);
        }
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
    if (warp == F::kWarps) {
        few_load<D, NT>(a, sm);
        return;
    }
    auto sync = [] { asm volatile("bar.sync 1, %0;" ::"n"(32 * F::kWarps) : "memory"); };

    const int N = packed_tokens(a.P), block_bytes = packed_block_bytes(N, D);
    // where this lane's pieces of a tile lie: its keys' block and its values' one (two blocks of 16 tokens, or the same of 32)
    const int k_block = N == 16 ? (r >> 2) * block_bytes : 0, v_block = N == 16 ? (t4 >> 1) * block_bytes : 0;
    const int k_at = k_block + ((N == 16 ? r & 3 : r) * 4 + t4) * 16, k_step = N * 16;  // from 32 channels to the next
    const int v_at = v_block + N * D / 2 + (r * (N / 8) + (N == 16 ? t4 & 1 : t4)) * 16, v_step = N * 16;
    const int ks_at = k_block + N * D + 8 * t4, vs_at = v_block + N * D + D + 8 * (N == 16 ? t4 & 1 : t4);
    uint32_t seq = 0, seq4 = 0, items = 0;  // tiles, packed tiles, items of this CTA before the item at hand

    for (AttendWalk<kTile> w(sm.cut); w.more(); w.next(a.H)) {
        const int b = w.b / groups, g = w.b % groups, h = w.item, r0 = g * F::kRows;
        const LongItem<kTile> it(a, b, r0, F::kRows);
        w.open_tiles(it.n);
        if (it.s.bad && tid == 0) atomicOr(a.status, kStBadLength);
        const int to = w.tile + w.n, packed_to = min(to, it.packed_tiles());
        const int32_t* table = a.block_table + (int64_t)b * a.max_pages;

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
        bool mine = false;
        for (int i = w.tile + (int)((warp + F::kWarps - seq % F::kWarps) % F::kWarps); i < to; i += F::kWarps) {
            mine = true;
            const int number = it.number(i), place = it.begin(number), end = it.end(number);
            const bool packed = i < packed_to;
            const uint32_t u = seq4 + (i - w.tile), slot = u % kSlots;
            const unsigned char* ring = sm.ring[slot];
            float s[NT][2][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int k = 0; k < 8; ++k) s[n][k / 4][k % 4] = 0.0f;
            const char* near_value[4];  // 16 bits: this lane's places' values; null where there is none to read
            if (packed) {
                bar_wait(&sm.full[slot], (u / kSlots) & 1, &sm.abort);  // (where it fails the results do not count)
#pragma unroll
                for (int x = 0; x < F::kX; ++x) {
                    uint32_t sc[4], so[4], d[4][4];
                    packed_scales(*reinterpret_cast<const uint2*>(ring + ks_at + 32 * x), sc, so);
                    packed_words(*reinterpret_cast<const uint4*>(ring + k_at + k_step * x), sc, so, d);
#pragma unroll
                    for (int n = 0; n < NT; ++n) feed(s[n][0], s[n][1], d, q[n][x]);
                }
            } else {
                const char* key[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int l0 = place + quad_row(r, k), x = l0 - it.s.pk;
                    key[k] = near_value[k] = nullptr;
                    if (l0 >= end || !it.wanted(l0, 1)) continue;
                    const int page = table[x >> a.page_shift];
                    if (page < 0 || page >= a.pages) {
                        atomicOr(a.status, kStBadIndex);
                        continue;
                    }
                    key[k] = static_cast<const char*>(a.kv.key) +
                             (page * a.kv.key_page + h * a.kv.key_head + (x & (a.P - 1)) * a.kv.key_token + 8 * t4) * 2;
                    near_value[k] = static_cast<const char*>(a.kv.value) +
                                    (page * a.kv.value_page + h * a.kv.value_head + (x & (a.P - 1)) * a.kv.value_token + 8 * t4) * 2;
                }
                __syncwarp();
#pragma unroll
                for (int x = 0; x < F::kX; ++x) {
                    uint32_t d[4][4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint4 y = make_uint4(0, 0, 0, 0);
                        if (key[k]) y = *reinterpret_cast<const uint4*>(key[k] + 64 * x);
                        d[k][0] = y.x, d[k][1] = y.y, d[k][2] = y.z, d[k][3] = y.w;
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) feed(s[n][0], s[n][1], d, q[n][x]);
                }
            }
            // s[n][k / 2][2 (k % 2) + e]: place f(r, k), row 8 n + 2 t4 + e
            const bool masked = place + kTile > min(end, it.s.ctx) || place < it.lo_most;
            uint32_t p[NT][4];
            bool grow = false;
            float top[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    top[n][e] = -INFINITY;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        float& y = s[n][k / 2][2 * (k % 2) + e];
                        y *= a.scale_log2;
                        if (masked) {
                            const int l0 = place + quad_row(r, k), t = token[n][e];
                            const uint8_t* mrow = a.mask ? a.mask + ((int64_t)b * a.T + max(t, 0)) * a.T : nullptr;
                            if (t < 0 || l0 >= end || !it.sees(a, b, mrow, t, first[n][e], l0)) y = -INFINITY;
                        }
                        top[n][e] = fmaxf(top[n][e], y);
                    }
                    grow |= top[n][e] > m[n][e] + kSlack || (m[n][e] == -INFINITY && top[n][e] > m[n][e]);
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
            if (packed) {
#pragma unroll
                for (int x = 0; x < F::kX; ++x) {
                    uint32_t sc[4], so[4], d[4][4];
                    packed_scales(*reinterpret_cast<const uint2*>(ring + vs_at + N * x), sc, so);
                    packed_words(*reinterpret_cast<const uint4*>(ring + v_at + v_step * x), sc, so, d);
#pragma unroll
                    for (int n = 0; n < NT; ++n) feed(o[n][x][0], o[n][x][1], d, p[n]);
                }
                __syncwarp();
                if (lane == 0) bar_arrive(&sm.empty[slot]);
            } else {
                bool odd = false;
#pragma unroll
                for (int x = 0; x < F::kX; ++x) {
                    uint32_t d[4][4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint4 y = make_uint4(0, 0, 0, 0);
                        if (near_value[k]) y = *reinterpret_cast<const uint4*>(near_value[k] + 64 * x);
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
        }
        seq += w.n;
        seq4 += max(0, packed_to - w.tile);

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
        sync();
        const bool left_out = *(volatile int*)&sm.odd[items & 1] != 0;
        if (tid == 0) sm.odd[~items & 1] = 0;  // the next item's, read last before the sums of this one
        ++items;
        const bool whole = w.n == w.all;
        const int64_t part = attend_part(blockIdx.x, w.tile == 0);
        const int filled = min((int)F::kWarps, w.n);  // warps that had a tile: seq - w.n .. on
        for (int k = tid; k < F::kRows * (D / 4); k += 32 * F::kWarps) {
            const int rr = k / (D / 4), c4 = k % (D / 4), row = r0 + rr, t = row / a.G, head = h * a.G + row - t * a.G;
            if (row >= rows) continue;
            float mm = -INFINITY, ll = 0.0f, y[4] = {0, 0, 0, 0};
            for (int z = 0; z < filled; ++z) mm = fmaxf(mm, sm.ml[(seq - w.n + z) % F::kWarps][rr].x);
            const float ref = mm == -INFINITY ? 0.0f : mm;
            for (int z = 0; z < filled; ++z) {
                const int from = (seq - w.n + z) % F::kWarps;
                const float2 x = sm.ml[from][rr];
                const float f = fast_exp2(x.x - ref);
                ll += f * x.y;
                const float* src = &sm.o[from][rr * F::kLine + 4 * c4];
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
        sync();
    }
    if (tid == 0 && *(volatile int*)&sm.abort) atomicOr(a.status, kStInternal);
}

template <int D, int NT> cudaError_t launch_few(const AttendArgs& a, cudaStream_t s) {
    constexpr size_t smem = sizeof(FewSmem<D, NT>);
    static_assert(smem <= 227 * 1024);
    const cudaError_t err = cudaFuncSetAttribute(packed_few_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (err != cudaSuccess) return err;
    return launch_dependent(packed_few_kernel<D, NT>, dim3(a.ctas), dim3(Few<D, NT>::kThreads), smem, s, a);
}

}  // namespace

cudaError_t launch_packed_attend(const AttendArgs& in, cudaStream_t s) {
    AttendArgs a = in;
    const int rows = a.T * a.G;
    if (rows > 16) {
        const cudaError_t err = launch_packed_tc(a, s);
        return err != cudaSuccess ? err : launch_attend_join(a, 1, s);
    }
    const bool one = rows <= 8;
    a.item_rows = one ? 8 : 16;
    a.part_rows = a.item_rows;
    a.lead = 8;
    a.least = 16;
    const cudaError_t err = a.D == 64 ? (one ? launch_few<64, 1>(a, s) : launch_few<64, 2>(a, s))
                                      : (one ? launch_few<128, 1>(a, s) : launch_few<128, 2>(a, s));
    return err != cudaSuccess ? err : launch_attend_join(a, 1, s);
}

}  // namespace rheo
