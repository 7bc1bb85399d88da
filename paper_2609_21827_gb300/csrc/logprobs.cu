// logprobs.cu -- log probabilities of given tokens with rank, entropy and the
// top alternatives, in one pass over each row's logits.
//
// With a running reference m (the largest logit that the thread's warp has met: one
// for all its lanes, so that it moves a handful of times a row), c = log2(e)/T and
// d = (l - m) c, a thread keeps Z = sum 2^d and W = sum 2^d d; a new reference m'
// with D = (m - m') c turns them into 2^D Z and 2^D (W + D Z).  Then, in log2 units,
//   log p(t) = (l_t - m) c - log2 Z,   H = log2 Z - W / Z.
// The difference is taken before the product, so that logits near the type's
// lowest value (a common mask) neither overflow nor lose their order.
// The rank counts l > l_t, and l = l_t at smaller ids.
// Top alternatives: the k-th largest of the maxima of 128 groups of four threads
// bounds the row's k-th largest from below, so the stream needs nothing but each
// thread's maximum and where it was; afterwards only the stripes of the k groups at
// or above the bound are read again (from L2), and the few logits found there are
// ranked.  Keys are (logit, -id) in 64 bits, all different, so ties need no care.
// A row is cut into segments where there are fewer rows than SMs; the last CTA of
// a row joins them.
// 144 rows of 151,936 in bf16 take 26.6 us (1.6 TB/s; their loads alone 13.5), 576 rows 71
// us (2.5 TB/s), four rows of 1,024 5.7 us in a captured graph.  288 rows: 19.5 instructions an
// element (maximum, two sums, count, and the ends of rows), issue slots 53 % busy: a CTA
// reads while the other one of its SM ranks.
#include <cuda_bf16.h>

#include "cache_kernels.h"
#include "rheo_device.cuh"
#include "rheo_kernels.h"

namespace rheo {

constexpr int kLpThreads = 512;
constexpr int kLpWarps = kLpThreads / 32;
constexpr int kLpBatch = 2;       // vectors of a thread in work, and as many on their way
constexpr int kLpCand = 2048;     // candidates ranked at a time
constexpr int kLpGroups = kLpThreads / 4;
constexpr int kLpMaxSegments = kLpCand / kMaxTop;
constexpr float kLpFloor = -10000.0f;  // 2^floor = 0: keeps (-inf) * 0 out of W

struct LpSums {
    float m, z, w;  // reference (a logit; -inf: nothing yet), Z, W
};

__device__ __forceinline__ LpSums lp_join(LpSums a, LpSums b, float c) {
    const float m = fmaxf(a.m, b.m);
    if (m == -INFINITY) return LpSums{m, a.z + b.z, a.w + b.w};  // zeros, or a NaN to keep
    const float da = fmaxf((a.m - m) * c, kLpFloor), db = fmaxf((b.m - m) * c, kLpFloor);
    const float ea = fast_exp2(da), eb = fast_exp2(db);
    return LpSums{m, ea * a.z + eb * b.z, ea * (a.w + da * a.z) + eb * (b.w + db * b.z)};
}

__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Counts logits above a cut.  The cut for vectors before the token's is the type's
// next value below its logit, so that equal ones count there; NaN for -inf, above
// which (unordered) everything counts.
__device__ __forceinline__ uint32_t below_bits(uint32_t u, uint32_t sign, uint32_t neg_inf, uint32_t nan) {
    if (u == neg_inf) return nan;
    if ((u & ~sign) == 0) return sign | 1u;  // either zero
    return u & sign ? u + 1 : u - 1;
}
template <int DT> struct LpAbove;
template <> struct LpAbove<0> {
    unsigned long long n = 0ull;
    __device__ static __forceinline__ uint32_t cut(float l, bool before) {
        const uint32_t u = __float_as_uint(l);
        return before ? below_bits(u, 0x80000000u, 0xFF800000u, 0x7FC00000u) : u;
    }
    __device__ static __forceinline__ float one(uint32_t l, uint32_t cut) {
        float r;
        asm("set.gtu.f32.f32 %0, %1, %2;" : "=f"(r) : "f"(__uint_as_float(l)), "f"(__uint_as_float(cut)));
        return r;
    }
    __device__ __forceinline__ void add(const uint4& x, uint32_t cut) {
        n = f2_add(n, f2_add(f2_pack(one(x.x, cut), one(x.y, cut)), f2_pack(one(x.z, cut), one(x.w, cut))));
    }
    __device__ __forceinline__ void flush(int& count) {
        count += (int)f2_fold(n);
        n = 0ull;
    }
};
template <> struct LpAbove<1> {
    __nv_bfloat162 n = __floats2bfloat162_rn(0.0f, 0.0f);  // whole numbers to 256
    __device__ static __forceinline__ uint32_t cut(float l, bool before) {
        const uint32_t h = __float_as_uint(l) >> 16, u = before ? below_bits(h, 0x8000u, 0xFF80u, 0x7FC0u) : h;
        return u | (u << 16);
    }
    __device__ static __forceinline__ __nv_bfloat162 two(uint32_t l, uint32_t cut) {
        uint32_t r;
        asm("set.gtu.bf16x2.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(l), "r"(cut));
        return *reinterpret_cast<const __nv_bfloat162*>(&r);
    }
    __device__ __forceinline__ void add(const uint4& x, uint32_t cut) {
        n = __hadd2(n, __hadd2(__hadd2(two(x.x, cut), two(x.y, cut)), __hadd2(two(x.z, cut), two(x.w, cut))));
    }
    __device__ __forceinline__ void flush(int& count) {
        count += (int)(__low2float(n) + __high2float(n));
        n = __floats2bfloat162_rn(0.0f, 0.0f);
    }
};

// Larger for larger logits, then for smaller ids; 0 for -inf.
__device__ __forceinline__ unsigned long long lp_key(float v, int id) {
    if (v == -INFINITY) return 0ull;
    return ((unsigned long long)ord_f32(v) << 32) | (0xFFFFFFFFu - (uint32_t)id);
}
__device__ __forceinline__ int lp_id(unsigned long long key) { return (int)(0xFFFFFFFFu - (uint32_t)key); }
__device__ __forceinline__ float lp_value(unsigned long long key) { return Elem<0>::value_of_key((uint32_t)(key >> 32)); }

// The largest (NaN if there is one) and the smallest logit of a vector.
template <int DT> struct LpVec;
template <> struct LpVec<0> {
    __device__ static __forceinline__ float largest(const uint4& x) {
        return max_nan(max_nan(__uint_as_float(x.x), __uint_as_float(x.y)), max_nan(__uint_as_float(x.z), __uint_as_float(x.w)));
    }
    __device__ static __forceinline__ float smallest(const uint4& x) {
        return fminf(fminf(__uint_as_float(x.x), __uint_as_float(x.y)), fminf(__uint_as_float(x.z), __uint_as_float(x.w)));
    }
};
template <> struct LpVec<1> {
    __device__ static __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    __device__ static __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    __device__ static __forceinline__ float largest(const uint4& x) {
        const uint32_t r = max2(max2(x.x, x.y), max2(x.z, x.w));
        return max_nan(bf_lo(r), bf_hi(r));
    }
    __device__ static __forceinline__ float smallest(const uint4& x) {
        const uint32_t r = min2(min2(x.x, x.y), min2(x.z, x.w));
        return fminf(bf_lo(r), bf_hi(r));
    }
};

struct LpShared {
    unsigned long long cand[kLpCand];
    unsigned long long best[kLpGroups];
    unsigned long long top[kMaxTop];
    unsigned long long red[kLpWarps];
    LpSums sums[kLpWarps];
    int count[kLpWarps];
    int group[kMaxTop];
    int n_group, n_cand, last;
    unsigned long long floor;
};

// Ranks sm.cand[0..n) and leaves the k first in sm.top (0 where there are fewer).
__device__ __forceinline__ void lp_rank(LpShared& sm, int n, int k) {
    const int tid = threadIdx.x;
    if (tid < k) sm.top[tid] = 0ull;
    __syncthreads();
    for (int i = tid; i < n; i += kLpThreads) {
        const unsigned long long mine = sm.cand[i];
        if (mine == 0ull) continue;
        int above = 0;
        for (int j = 0; j < n; ++j) above += sm.cand[j] > mine;
        if (above < k) sm.top[above] = mine;
    }
    __syncthreads();
}

template <int DT, bool ALIGNED>
__global__ void __launch_bounds__(kLpThreads) logprob_kernel(const LogprobArgs a) {
    grid_dependency_begin();
    using E = Elem<DT>;
    constexpr int VEC = E::VEC;
    __shared__ LpShared sm;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int i = blockIdx.x / a.segments, seg = blockIdx.x % a.segments;
    const int V = a.V, k = a.k;

    int64_t r = a.row_index ? a.row_index[i] : i;
    if (r < -1 || r >= a.logit_rows) {
        if (tid == 0) atomicOr(a.status, kStBadIndex);
        r = -1;
    }
    if (r < 0) {
        if (seg == 0) {
            if (tid == 0) {
                a.out.logprob[i] = 0.0f;
                a.out.rank[i] = -1;
                a.out.entropy[i] = 0.0f;
            }
            if (tid < k) {
                a.out.top_ids[(int64_t)i * k + tid] = -1;
                a.out.top_logprobs[(int64_t)i * k + tid] = -INFINITY;
            }
        }
        return;
    }
    int tk = a.token[i];
    if (tk < -1 || tk >= V) {
        if (tid == 0) atomicOr(a.status, kStBadIndex);
        tk = -1;
    }
    float T = a.temperature ? a.temperature[i / a.per_t] : 1.0f;
    if (!(T > 0.0f && T < INFINITY)) {
        if (tid == 0) atomicOr(a.status, kStBadTemperature);
        T = 1.0f;
    }
    const float c = fminf(1.4426950408889634f / T, 3.0e38f);
    const char* row = a.logits + r * a.row_stride_bytes;
    const float lt = tk >= 0 ? E::value(E::load_scalar(row, tk)) : INFINITY;
    const int tv = tk >= 0 ? tk / VEC : -1;  // the vector that holds the token
    const int vectors = (V + VEC - 1) / VEC;
    const int v0 = (int)((int64_t)seg * vectors / a.segments), v1 = (int)((int64_t)(seg + 1) * vectors / a.segments);

    float m = -INFINITY, mx = -INFINITY;       // reference, largest logit
    unsigned long long z2 = 0ull, w2 = 0ull;   // sums of the even and of the odd elements
    int mv = -1, count = 0;                    // the vector in which the largest was met first
    const unsigned long long c2 = f2_pack(c, c);
    LpAbove<DT> above;
    const uint32_t before = LpAbove<DT>::cut(lt, true), after = LpAbove<DT>::cut(lt, false);
    auto take = [&](const uint4& x, int v) {
        const int own_tv = v < v1 ? tv : -1;
        const float vm = LpVec<DT>::largest(x), vn = LpVec<DT>::smallest(x);
        mv = vm > mx ? v : mv;
        mx = max_nan(mx, vm);
        if (__any_sync(0xffffffffu, !(vm <= m))) {
            float top = max_nan(m, vm);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
            const float d = fmaxf((m - top) * c, kLpFloor), f = fast_exp2(d);
            const unsigned long long f2 = f2_pack(f, f), d2 = f2_pack(d, d);
            w2 = f2_mul(f2, f2_fma(d2, z2, w2));
            z2 = f2_mul(f2, z2);
            m = top;
        }
        if (m > -INFINITY || m != m) {  // nothing but -inf so far adds nothing
            const unsigned long long m2 = f2_pack(-m, -m);
            if ((vn - m) * c > kLpFloor) {
#pragma unroll
                for (int e = 0; e < VEC; e += 2) {
                    const unsigned long long d =
                        f2_mul(f2_add(f2_pack(E::value(E::raw(x, e)), E::value(E::raw(x, e + 1))), m2), c2);
                    const unsigned long long p = f2_exp2(d);
                    z2 = f2_add(z2, p);
                    w2 = f2_fma(p, d, w2);
                }
            } else {
                // logits so far below the reference (masked ones) that 0 * d may not be 0
#pragma unroll
                for (int e = 0; e < VEC; e += 2) {
                    const float d0 = max_nan((E::value(E::raw(x, e)) - m) * c, kLpFloor);
                    const float d1 = max_nan((E::value(E::raw(x, e + 1)) - m) * c, kLpFloor);
                    const unsigned long long d = f2_pack(d0, d1), p = f2_exp2(d);
                    z2 = f2_add(z2, p);
                    w2 = f2_fma(p, d, w2);
                }
            }
        }
        above.add(x, v < own_tv ? before : after);
        if (v == own_tv) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) count += E::value(E::raw(x, e)) == lt && v * VEC + e < tk;
        }
    };
    // (lanes past the segment take an empty vector, which no cut but NaN counts)
    // a batch is taken while the next one is on its way
    uint4 now[kLpBatch], next[kLpBatch];
    const uint32_t low = DT == 1 ? 0xFF80FF80u : 0xFF800000u;
    const uint4 none = make_uint4(low, low, low, low);  // -inf: adds nothing
    auto fetch = [&](uint4 (&x)[kLpBatch], int base) {
#pragma unroll
        for (int u = 0; u < kLpBatch; ++u)
            x[u] = base + u * kLpThreads < v1 ? load_vec<DT, ALIGNED>(row, (int64_t)(base + u * kLpThreads) * VEC, V) : none;
    };
    fetch(now, v0 + tid);
    for (int base = v0 + warp * 32; base < v1; base += kLpThreads * kLpBatch) {  // the same for the whole warp
        fetch(next, base + lane + kLpThreads * kLpBatch);
#pragma unroll
        for (int u = 0; u < kLpBatch; ++u)
            if (base + u * kLpThreads < v1) take(now[u], base + u * kLpThreads + lane);
        above.flush(count);
#pragma unroll
        for (int u = 0; u < kLpBatch; ++u) now[u] = next[u];
    }
    LpSums s{m, f2_fold(z2), f2_fold(w2)};

    // sums and count over the block
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        LpSums t{__shfl_xor_sync(0xffffffffu, s.m, o), __shfl_xor_sync(0xffffffffu, s.z, o),
                 __shfl_xor_sync(0xffffffffu, s.w, o)};
        s = lp_join(s, t, c);
    }
    count = __reduce_add_sync(0xffffffffu, count);
    if (lane == 0) {
        sm.sums[warp] = s;
        sm.count[warp] = count;
    }
    if (k > 0) {
        // no larger than the key of the thread's first largest logit
        unsigned long long key = mv >= 0 && mx > -INFINITY ? lp_key(mx, mv * VEC + VEC - 1) : 0ull;
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
            const unsigned long long y = __shfl_xor_sync(0xffffffffu, key, o);
            key = y > key ? y : key;
        }
        if ((tid & 3) == 0) sm.best[tid >> 2] = key;
        if (tid == 0) {
            sm.n_group = sm.n_cand = 0;
            sm.floor = 1ull;
        }
        __syncthreads();
        if (tid < kLpGroups && (key = sm.best[tid]) != 0ull) {
            int above_me = 0;
#pragma unroll 8
            for (int j = 0; j < kLpGroups; ++j) above_me += sm.best[j] > key;
            if (above_me < k) sm.group[atomicAdd(&sm.n_group, 1)] = tid;
            if (above_me == k - 1) sm.floor = key;
        }
        __syncthreads();
        const unsigned long long floor = sm.floor;
        const int n_group = sm.n_group;
        // a group's stripes by a warp: four neighbouring vectors a quarter of eight lanes, four rounds under way
        auto each = [&](auto&& f) {
            constexpr int step = 8 * kLpThreads;
            for (int q = warp; q < n_group; q += kLpWarps) {
                for (int v = v0 + sm.group[q] * 4 + (lane & 3) + (lane >> 2) * kLpThreads; v < v1; v += 4 * step) {
                    uint4 x[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (v + u * step < v1) x[u] = load_vec<DT, ALIGNED>(row, (int64_t)(v + u * step) * VEC, V);
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (v + u * step < v1)
#pragma unroll
                            for (int e = 0; e < VEC; ++e)
                                f(lp_key(E::value(E::raw(x[u], e)), (v + u * step) * VEC + e));
                }
            }
        };
        each([&](unsigned long long y) {
            if (y >= floor) {
                const int at = atomicAdd(&sm.n_cand, 1);
                if (at < kLpCand) sm.cand[at] = y;
            }
        });
        __syncthreads();
        const int n = sm.n_cand;
        if (n <= kLpCand) {
            lp_rank(sm, n, k);
        } else {
            // more than the buffer holds (stripes full of large logits): one round of maxima an alternative
            unsigned long long last = ~0ull;
            for (int round = 0; round < k; ++round) {
                unsigned long long top = 0ull;
                each([&](unsigned long long y) {
                    if (y < last && y > top) top = y;
                });
                top = warp_max_u64(top);
                if (lane == 0) sm.red[warp] = top;
                __syncthreads();
                top = sm.red[0];
                for (int w = 1; w < kLpWarps; ++w) top = sm.red[w] > top ? sm.red[w] : top;
                if (tid == 0) sm.top[round] = top;
                last = top;
                __syncthreads();
            }
        }
    }
    __syncthreads();
    if (a.segments > 1) {
        const int64_t part = (int64_t)i * a.segments + seg;
        if (tid < k) a.part_key[part * kMaxTop + tid] = sm.top[tid];
        if (tid == 0) {
            s = sm.sums[0];
            count = sm.count[0];
            for (int w = 1; w < kLpWarps; ++w) {
                s = lp_join(s, sm.sums[w], c);
                count += sm.count[w];
            }
            *reinterpret_cast<float4*>(a.part + part * 4) = make_float4(s.m, s.z, s.w, __int_as_float(count));
        }
        __threadfence();
        __syncthreads();
        if (tid == 0) sm.last = atomicAdd(&a.ticket[i], 1u) == (unsigned)a.segments - 1;
        __syncthreads();
        if (!sm.last) return;
        __threadfence();
        if (tid == 0) a.ticket[i] = 0;
        const int64_t first = (int64_t)i * a.segments;
        if (k > 0) {
            for (int j = tid; j < a.segments * k; j += kLpThreads)
                sm.cand[j] = __ldcg(a.part_key + (first + j / k) * kMaxTop + j % k);
            __syncthreads();
            lp_rank(sm, a.segments * k, k);
        }
    }
    if (tid < 32) {
        // the sums once more, by one warp in a fixed order
        LpSums t{-INFINITY, 0.0f, 0.0f};
        int n = 0;
        if (a.segments > 1) {
            for (int j = lane; j < a.segments; j += 32) {
                const float4 x = __ldcg(reinterpret_cast<const float4*>(a.part + ((int64_t)i * a.segments + j) * 4));
                t = lp_join(t, LpSums{x.x, x.y, x.z}, c);
                n += __float_as_int(x.w);
            }
        } else if (lane < kLpWarps) {
            t = sm.sums[lane];
            n = sm.count[lane];
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            t = lp_join(t, LpSums{__shfl_xor_sync(0xffffffffu, t.m, o), __shfl_xor_sync(0xffffffffu, t.z, o),
                                  __shfl_xor_sync(0xffffffffu, t.w, o)}, c);
        n = __reduce_add_sync(0xffffffffu, n);
        const float lz = log2f(t.z);
        constexpr float kLn2 = 0.69314718055994531f;
        if (lane == 0) {
            if (!(t.z == t.z) || t.m == INFINITY) atomicOr(a.status, kStBadLogit);
            else if (t.m == -INFINITY) atomicOr(a.status, kStEmptyRow);
            a.out.logprob[i] = tk >= 0 ? (lt - t.m) / T - lz * kLn2 : 0.0f;
            a.out.rank[i] = tk >= 0 ? n : -1;
            a.out.entropy[i] = (lz - t.w / t.z) * kLn2;
        }
        if (lane < k) {
            const unsigned long long y = sm.top[lane];
            a.out.top_ids[(int64_t)i * k + lane] = y ? lp_id(y) : -1;
            a.out.top_logprobs[(int64_t)i * k + lane] = y ? (lp_value(y) - t.m) / T - lz * kLn2 : -INFINITY;
        }
    }
}

// CTAs a row: about two an SM in all, so that one reads while the other ranks, with
// four vectors a thread at least (144 rows of 151,936 in bf16: 33.8, 24.4, 32.7 us
// with one, two, three an SM, measured with a reference per thread, which took 2 us
// less than the warp's and was less exact for peaked rows).
int logprob_segments(int rows, int vocab, int dtype) {
    const int vec = dtype == 1 ? 8 : 4, vectors = (vocab + vec - 1) / vec;
    int n = kLogprobParts / rows, most = vectors / (4 * kLpThreads);
    n = n < most ? n : most;
    n = n < kLpMaxSegments ? n : kLpMaxSegments;
    return n < 1 ? 1 : n;
}

template <int DT, bool ALIGNED> static cudaError_t launch_lp(const LogprobArgs& a, cudaStream_t s) {
    return launch_dependent(logprob_kernel<DT, ALIGNED>, dim3((unsigned)a.R * a.segments), dim3(kLpThreads), 0, s, a);
}

cudaError_t launch_logprobs(const LogprobArgs& a, int dtype, bool aligned, cudaStream_t s) {
    if (dtype == 1) return aligned ? launch_lp<1, true>(a, s) : launch_lp<1, false>(a, s);
    return aligned ? launch_lp<0, true>(a, s) : launch_lp<0, false>(a, s);
}

}  // namespace rheo
