// attend_simt.cu -- attention of drafted tokens over a paged fp32 cache on the
// fp32 units, and the join of partial sums of either type.
//
// For an item of R query rows and its key tiles of 64: scores s = q k (fp32 FMA
// on register tiles of R/16 x 4 a thread), running maximum m and sum l a row in
// log2 units, p = 2^(s - m), O = 2^(m_old - m) O + p V.  Half a warp owns R/16
// rows, so the row statistics are four shuffles and p passes through shared
// memory without a block barrier.
// Four trees of up to 17 tokens over up to 733 places (8 query, 4 key/value heads of
// 64): 15 to 17.5 us with the join, 0.2 TB/s: bound by dependent latencies (lengths, table, keys, two
// products, join), as its few bytes come from L2.  The fp32 units, because tf32
// products would round what an fp32 cache is kept for.
#include <cuda_bf16.h>

#include <type_traits>

#include "attend.cuh"
#include "rheo_kernels.h"

namespace rheo {

constexpr int kSimtThreads = 256;
constexpr int kSimtTile = 64;

__device__ __forceinline__ void cp_async16(void* dst, const void* src, bool valid) {
    const unsigned d = (unsigned)__cvta_generic_to_shared(dst);
    const int n = valid ? 16 : 0;  // 0: the 16 bytes are zeroed
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

template <int D, int R> struct SimtSmem {
    float q[R][D + 4];
    float k[2][kSimtTile][D + 4];
    float v[2][kSimtTile][D];
    float p[R][kSimtTile + 4];
};

template <int D, int R>
__global__ void __launch_bounds__(kSimtThreads, 1) attend_simt_kernel(const AttendArgs a) {
    grid_dependency_begin();
    extern __shared__ __align__(16) unsigned char raw_smem[];
    SimtSmem<D, R>& sm = *reinterpret_cast<SimtSmem<D, R>*>(raw_smem);
    __shared__ AttendCut cut_s;
    constexpr int RT = R / 16, DJ = D / 64, ES = 4;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int rows = a.T * a.G, groups = (rows + R - 1) / R, per = a.H * groups;
    if (tid < 32) {
        const AttendCut c = attend_cut<kSimtTile>(a, per, blockIdx.x);
        if (tid == 0) cut_s = c;
    }
    __syncthreads();
    const AttendCut cut = cut_s;
    if (tid == 0) a.join[blockIdx.x] = make_int4(0, 0, 0, 0);

    for (AttendWalk<kSimtTile> walk(cut); walk.more(); walk.next(per)) {
        const int b = walk.b;
        const AttendSpan span = attend_span(a, b);
        if (span.bad && tid == 0) atomicOr(a.status, kStBadLength);
        const int len = span.len();
        walk.open(len);
        const int tile = walk.tile, n = walk.n, h = walk.item / groups, r0 = (walk.item % groups) * R;
        const int32_t* table = a.block_table + (int64_t)b * a.max_pages;

        auto load = [&](int tl, int buf) {
            constexpr int C = D * ES / 16;  // 16-byte pieces of a line
            for (int i = tid; i < kSimtTile * C; i += kSimtThreads) {
                const int kr = i / C, c = i % C, l = tl * kSimtTile + kr;
                bool ok = l < len;
                int64_t page = 0;
                if (ok) {
                    page = table[l >> a.page_shift];
                    if (page < 0 || page >= a.pages) {
                        atomicOr(a.status, kStBadIndex);
                        ok = false;
                        page = 0;
                    }
                }
                const int64_t row = l & (a.P - 1);
                const char* ks = static_cast<const char*>(a.kv.key) +
                                 (page * a.kv.key_page + h * a.kv.key_head + row * a.kv.key_token) * ES + c * 16;
                const char* vs = static_cast<const char*>(a.kv.value) +
                                 (page * a.kv.value_page + h * a.kv.value_head + row * a.kv.value_token) * ES + c * 16;
                cp_async16(&sm.k[buf][kr][c * 4], ks, ok);
                cp_async16(&sm.v[buf][kr][c * 4], vs, ok);
            }
            cp_async_commit();
        };

        __syncthreads();  // the last item's tiles and queries have been read
        load(tile, 0);
        for (int i = tid; i < R * (D / 4); i += kSimtThreads) {
            const int r = i / (D / 4), d = i % (D / 4) * 4, row = r0 + r, t = row / a.G;
            float4 x = make_float4(0, 0, 0, 0);
            if (row < rows && t < span.add) {
                const char* src = static_cast<const char*>(a.io.q) +
                                  (b * a.io.q_batch + t * a.io.q_token + (h * a.G + row % a.G) * a.io.q_head + d) * ES;
                x = *reinterpret_cast<const float4*>(src);
            }
            *reinterpret_cast<float4*>(&sm.q[r][d]) = x;
        }

        float m[RT], l[RT], o[RT][DJ * 4];
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            m[i] = -INFINITY;
            l[i] = 0.0f;
#pragma unroll
            for (int d = 0; d < DJ * 4; ++d) o[i][d] = 0.0f;
        }
        for (int q = 0; q < n; ++q) {
            const int buf = q & 1, k0 = (tile + q) * kSimtTile;
            if (q + 1 < n) load(tile + q + 1, buf ^ 1);
            if (q + 1 < n) cp_async_wait<1>();
            else cp_async_wait<0>();
            __syncthreads();

            float s[RT][4];
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[i][j] = 0.0f;
#pragma unroll 4
            for (int d = 0; d < D; d += 4) {
                float4 kk[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) kk[j] = *reinterpret_cast<const float4*>(&sm.k[buf][tx + 16 * j][d]);
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    const float4 qq = *reinterpret_cast<const float4*>(&sm.q[ty * RT + i][d]);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        s[i][j] += qq.x * kk[j].x + qq.y * kk[j].y + qq.z * kk[j].z + qq.w * kk[j].w;
                }
            }
            const bool tail = k0 + kSimtTile > span.ctx;  // places that not every token sees
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const int row = r0 + ty * RT + i, t = row / a.G;
                const uint8_t* mrow = a.mask ? a.mask + ((int64_t)b * a.T + min(t, a.T - 1)) * a.T : nullptr;
                unsigned hidden = 0;
                float top = -INFINITY;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s[i][j] *= a.scale_log2;
                    if (tail && !(t < span.add && attend_sees(span, mrow, t, k0 + tx + 16 * j))) {
                        s[i][j] = -INFINITY;
                        hidden |= 1u << j;
                    }
                    top = fmaxf(top, s[i][j]);
                }
#pragma unroll
                for (int w = 8; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
                const float mn = fmaxf(m[i], top), ref = mn == -INFINITY ? 0.0f : mn;
                const float keep = fast_exp2(m[i] - ref);
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float p = fast_exp2(s[i][j] - ref);
                    // a hidden place is marked by the sign of its zero, so that V's NaN and infinities there are skipped
                    if ((hidden >> j) & 1u) p = -0.0f;
                    sum += p;
                    sm.p[ty * RT + i][tx + 16 * j] = p;
                }
#pragma unroll
                for (int w = 8; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
                l[i] = l[i] * keep + sum;
                m[i] = mn;
#pragma unroll
                for (int d = 0; d < DJ * 4; ++d) o[i][d] *= keep;
            }
            __syncwarp();
            auto times_v = [&](auto skip) {
#pragma unroll 2
                for (int k = 0; k < kSimtTile; k += 4) {
                    float4 pp[RT];
#pragma unroll
                    for (int i = 0; i < RT; ++i) pp[i] = *reinterpret_cast<const float4*>(&sm.p[ty * RT + i][k]);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
#pragma unroll
                        for (int c = 0; c < DJ; ++c) {
                            const float4 vv = *reinterpret_cast<const float4*>(&sm.v[buf][k + u][tx * 4 + 64 * c]);
#pragma unroll
                            for (int i = 0; i < RT; ++i) {
                                const float p = u == 0 ? pp[i].x : u == 1 ? pp[i].y : u == 2 ? pp[i].z : pp[i].w;
                                if (decltype(skip)::value && __float_as_uint(p) == 0x80000000u) continue;
                                o[i][4 * c] += p * vv.x;
                                o[i][4 * c + 1] += p * vv.y;
                                o[i][4 * c + 2] += p * vv.z;
                                o[i][4 * c + 3] += p * vv.w;
                            }
                        }
                    }
                }
            };
            if (tail) times_v(std::true_type{});
            else times_v(std::false_type{});
            __syncthreads();  // the buffer is free for the tile after the next
        }

        const bool whole = n == walk.all;
        const int64_t part = attend_part(blockIdx.x, tile == 0);
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int r = ty * RT + i, row = r0 + r;
            if (row >= rows) continue;
            const int t = row / a.G, head = h * a.G + row % a.G;
            const float ll = t < span.add ? l[i] : 0.0f;
            if (!whole) {
#pragma unroll
                for (int c = 0; c < DJ; ++c)
                    reinterpret_cast<float4*>(a.part_o)[attend_part_at(a, part, r, tx + 16 * c)] =
                        make_float4(o[i][4 * c], o[i][4 * c + 1], o[i][4 * c + 2], o[i][4 * c + 3]);
                if (tx == 0) {
                    a.part_ml[(part * a.part_rows + r) * 2] = m[i];
                    a.part_ml[(part * a.part_rows + r) * 2 + 1] = ll;
                }
                continue;
            }
            const float inv = ll == 0.0f ? 0.0f : 1.0f / ll;
#pragma unroll
            for (int c = 0; c < DJ; ++c) {
                float4 y = make_float4(0, 0, 0, 0);
                if (ll != 0.0f)
                    y = make_float4(o[i][4 * c] * inv, o[i][4 * c + 1] * inv, o[i][4 * c + 2] * inv,
                                    o[i][4 * c + 3] * inv);
                *reinterpret_cast<float4*>(static_cast<float*>(a.io.out) + b * a.io.out_batch + t * a.io.out_token +
                                           head * a.io.out_head + tx * 4 + 64 * c) = y;
            }
            if (a.io.lse && tx == 0) a.io.lse[((int64_t)b * a.T + t) * a.H * a.G + head] = attend_lse(m[i], ll);
        }
        if (!whole && tile == 0 && tid == 0)
            a.join[blockIdx.x] = make_int4(b, walk.item, walk.segments(cut, blockIdx.x), 0);
    }
}

// Joins the parts of an item that several CTAs summed, in the order of its keys.  A
// thread takes eight columns of a row; neighbouring threads take neighbouring
// rows, as the parts lie.  Grid (CTAs of the sums, pieces of 256 threads).
// One pass: the parts' references are not known beforehand, so the sums follow the
// largest so far, four parts at a time.
// A second launch, although it costs 2 to 3 us: the last warp to add a part (a ticket an
// item) joining its rows was slower even where they are few (17.0 us for 15.8 with four short fp32
// trees, 23.2 for 19.9 with one token over 16,000), as what one warp reads
// is on its way for longer, and the last CTA alone would read up to 2.4 MB.
constexpr int kJoinBatch = 4;  // parts under way

template <int DT, int D>
__global__ void __launch_bounds__(256) attend_join_kernel(const AttendArgs a) {
    grid_dependency_begin();
    const int4 rec = a.join[blockIdx.x];
    const int segments = rec.z, i = blockIdx.y * 256 + threadIdx.x;
    const int c8 = i / a.part_rows, r = i - c8 * a.part_rows;
    if (segments == 0 || c8 >= D / 8) return;
    const int b = rec.x, rows = a.T * a.G, groups = (rows + a.item_rows - 1) / a.item_rows;
    const int h = rec.y / groups, row = rec.y % groups * a.item_rows + r;
    if (row >= rows) return;
    const int t = row / a.G, head = h * a.G + row % a.G;
    float m = -INFINITY, l = 0.0f, x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int s0 = 0; s0 < segments; s0 += kJoinBatch) {
        float2 ml[kJoinBatch];
        float4 u[kJoinBatch], v[kJoinBatch];
#pragma unroll
        for (int k = 0; k < kJoinBatch; ++k) {
            ml[k] = make_float2(-INFINITY, 0.0f);
            u[k] = v[k] = make_float4(0, 0, 0, 0);
            if (s0 + k < segments) {
                const int64_t part = attend_part(blockIdx.x + s0 + k, s0 + k == 0);
                const float4* po = reinterpret_cast<const float4*>(a.part_o) + attend_part_at(a, part, r, 2 * c8);
                ml[k] = *reinterpret_cast<const float2*>(a.part_ml + (part * a.part_rows + r) * 2);
                u[k] = po[0];
                v[k] = po[a.part_rows];
            }
        }
        float top = m;
#pragma unroll
        for (int k = 0; k < kJoinBatch; ++k) top = fmaxf(top, ml[k].x);
        const float ref = top == -INFINITY ? 0.0f : top, f = fast_exp2(m - ref);
        m = top;
        l *= f;
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] *= f;
#pragma unroll
        for (int k = 0; k < kJoinBatch; ++k) {
            const float w = fast_exp2(ml[k].x - ref);
            l += w * ml[k].y;
            x[0] += w * u[k].x;
            x[1] += w * u[k].y;
            x[2] += w * u[k].z;
            x[3] += w * u[k].w;
            x[4] += w * v[k].x;
            x[5] += w * v[k].y;
            x[6] += w * v[k].z;
            x[7] += w * v[k].w;
        }
    }
    const float inv = 1.0f / l;
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = l == 0.0f ? 0.0f : x[k] * inv;
    const int64_t e = b * a.io.out_batch + t * a.io.out_token + head * a.io.out_head + 8 * c8;
    if (DT == 0) {
        float4* out = reinterpret_cast<float4*>(static_cast<float*>(a.io.out) + e);
        out[0] = make_float4(x[0], x[1], x[2], x[3]);
        out[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        uint32_t y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const __nv_bfloat162 z = __floats2bfloat162_rn(x[2 * k], x[2 * k + 1]);
            y[k] = *reinterpret_cast<const uint32_t*>(&z);
        }
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.io.out) + e) = make_uint4(y[0], y[1], y[2], y[3]);
    }
    if (a.io.lse && c8 == 0) a.io.lse[((int64_t)b * a.T + t) * a.H * a.G + head] = attend_lse(m, l);
}

// fp32: 16 rows an item where that holds them all (single tokens and short
// chains: the products are few and the bytes count), else 64.  bf16: the 128 rows
// of one stream, or the 256 of two.
int attend_item_rows(int dtype, int T, int G) {
    const int64_t rows = (int64_t)T * G;
    return dtype == 1 ? (rows <= 128 ? 128 : 256) : (rows <= 16 ? 16 : 64);
}
int attend_part_rows(int dtype, int T, int G) {
    const int64_t rows = ((int64_t)T * G + 7) / 8 * 8, most = attend_item_rows(dtype, T, G);
    return (int)(rows < most ? rows : most);
}

// An item's start and end against a tile's time: queries, masks and results take as long as four tiles of the tensor
// cores' kernel (64 trees of 61 tokens: 262, 253, 247, 250, 253 us with 2, 3, 4, 6, 8), less than one of the fp32 kernel's.
int attend_lead(int dtype) { return dtype == 1 ? 4 : 1; }
// One tree of 61 tokens over 1,911 cached ones (bf16): 22.0, 19.7, 21.1, 21.3 us with chunks of 1, 2, 3, 4 tiles at
// least; four short fp32 trees: 18.1, 22.0, 26.6, 31.4.
int attend_least(int dtype) { return dtype == 1 ? 2 : 1; }

template <int DT, int D> static cudaError_t launch_join(const AttendArgs& a, cudaStream_t s) {
    return launch_dependent(attend_join_kernel<DT, D>, dim3(a.ctas, (a.part_rows * (D / 8) + 255) / 256), dim3(256), 0, s, a);
}

template <int D, int R> static cudaError_t launch_simt(const AttendArgs& a, cudaStream_t s) {
    const size_t smem = sizeof(SimtSmem<D, R>);
    cudaError_t err = cudaFuncSetAttribute(attend_simt_kernel<D, R>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                           (int)smem);
    if (err != cudaSuccess) return err;
    return launch_dependent(attend_simt_kernel<D, R>, dim3(a.ctas), dim3(kSimtThreads), smem, s, a);
}

cudaError_t launch_attend(const AttendArgs& a, int dtype, cudaStream_t s) {
    cudaError_t err;
    if (dtype == 1) {
        err = launch_attend_tc(a, s);
        if (err != cudaSuccess) return err;
        return a.D == 64 ? launch_join<1, 64>(a, s) : launch_join<1, 128>(a, s);
    }
    if (a.item_rows == 16) err = a.D == 64 ? launch_simt<64, 16>(a, s) : launch_simt<128, 16>(a, s);
    else err = a.D == 64 ? launch_simt<64, 64>(a, s) : launch_simt<128, 64>(a, s);
    if (err != cudaSuccess) return err;
    return a.D == 64 ? launch_join<0, 64>(a, s) : launch_join<0, 128>(a, s);
}

}  // namespace rheo
