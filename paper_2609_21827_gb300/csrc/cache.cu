// cache.cu -- the paged cache beside the attention: block tables and slots from
// lengths (reserve), norms and rotation of queries and keys with the store into
// the cache (qk_norm_rope), and the accepted path's move into place (commit).
#include <cuda_bf16.h>

#include "cache_kernels.h"
#include "rheo_device.cuh"
#include "rheo_kernels.h"

namespace rheo {

// ---------------------------------------------------------------------------
// reserve.  One launch of up to two CTAs per SM.  Every CTA derives the whole
// plan itself: pages to give back and to take of all B requests (three ints a
// request, read from L2), and their exclusive prefix sums in shared memory.
// From these each request's pages follow without any order between CTAs: the
// i-th page taken in the call is entry F-1-i of the stack as it stands after
// all releases, which is an old entry of the free list or, past the old top, a
// page that some request releases, found by a binary search over the release
// sums and read from that request's row.  Released and taken entries never
// overlap, so the tables may be updated in place; the counts, which every CTA
// reads, are written by the last CTA to have read them (a ticket).
// Latency bound: three dependent rounds of loads, a scan and the stores.  One request
// takes 4.2 us in a captured graph, 256 of 129 tokens into new tables 6.1; from Python
// both take 10, which the call's checks bound.  (256 from a Python call of 6.6 us that
// checked less: 10.3 with one CTA an SM and a load at a time.)
// ---------------------------------------------------------------------------
constexpr int kReserveThreads = 256;
constexpr int kReserveBad = (int)0x80000000u;  // mark of a request that keeps what it holds

// A thread's share of a copy: places at, at + step, ... below `to`, four loads under way.
__device__ __forceinline__ void copy_ints(int32_t* out, const int32_t* in, int64_t at, int64_t to, int64_t step) {
    for (; at < to; at += 4 * step) {
        int32_t x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (at + i * step < to) x[i] = in[at + i * step];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (at + i * step < to) out[at + i * step] = x[i];
    }
}

// Inclusive sums of both components over the block.
__device__ __forceinline__ int2 block_scan_pair(int2 v, int2* warp_sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, v.x, o), y = __shfl_up_sync(0xffffffffu, v.y, o);
        if (lane >= o) {
            v.x += x;
            v.y += y;
        }
    }
    if (lane == 31) warp_sums[warp] = v;
    __syncthreads();
    for (int w = 0; w < warp; ++w) {
        v.x += warp_sums[w].x;
        v.y += warp_sums[w].y;
    }
    __syncthreads();
    return v;
}

__global__ void __launch_bounds__(kReserveThreads) reserve_kernel(const ReserveArgs a) {
    grid_dependency_begin();
    extern __shared__ int rsm[];
    __shared__ int2 warp_sums[kReserveThreads / 32];
    __shared__ int2 carry;
    __shared__ int s_last;
    int* back_at = rsm;                // [B+1] pages given back before request b
    int* take_at = back_at + a.B + 1;  // [B+1] pages asked for before request b
    int* held = take_at + a.B + 1;     // [B] pages held, kReserveBad set where lengths are bad
    const int tid = threadIdx.x;
    const int64_t capacity = (int64_t)a.max_pages * a.P;

    int free0 = *a.before.n_free;
    if (free0 < 0 || free0 > a.pages) {
        if (tid == 0) atomicOr(a.status, kStInternal);
        free0 = free0 < 0 ? 0 : a.pages;
    }
    if (tid == 0) {
        carry = make_int2(0, 0);
        back_at[0] = take_at[0] = 0;
    }
    __syncthreads();
    for (int b0 = 0; b0 < a.B; b0 += kReserveThreads) {
        const int b = b0 + tid;
        int2 v = make_int2(0, 0);
        if (b < a.B) {
            const int64_t ctx = a.ctx_len[b], add = a.new_len ? a.new_len[b] : a.T;
            int own = a.before.n_pages[b];
            if (own < 0 || own > a.max_pages) {
                atomicOr(a.status, kStInternal);
                own = own < 0 ? 0 : a.max_pages;
            }
            const bool bad = ctx < 0 || add < 0 || add > a.T || ctx + add > capacity;
            if (bad) {
                atomicOr(a.status, kStBadLength);
                held[b] = own | kReserveBad;
            } else {
                const int need = (int)((ctx + add + a.P - 1) / a.P);
                v = make_int2(max(own - need, 0), max(need - own, 0));
                held[b] = own;
            }
        }
        v = block_scan_pair(v, warp_sums);
        const int2 c = carry;
        if (b < a.B) {
            back_at[b + 1] = c.x + v.x;
            take_at[b + 1] = c.y + v.y;
        }
        __syncthreads();
        if (tid == kReserveThreads - 1) carry = make_int2(c.x + v.x, c.y + v.y);
        __syncthreads();
    }
    const int have = free0 + back_at[a.B];  // the stack's height after all releases
    if (have > a.pages && tid == 0) atomicOr(a.status, kStInternal);
    if (tid == 0) {
        __threadfence();
        s_last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();

    // page i (0 = first) of those that request b takes
    auto taken = [&](int b, int i) -> int {
        const int at = have - 1 - (take_at[b] + i);
        if (at < free0) return a.before.free_list[at];
        const int r = at - free0;
        int lo = 0, hi = a.B - 1;  // the request with back_at[lo] <= r < back_at[lo + 1]
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (back_at[mid] <= r) lo = mid;
            else hi = mid - 1;
        }
        const int keep = (held[lo] & ~kReserveBad) - (back_at[lo + 1] - back_at[lo]);
        return a.before.block_table[(int64_t)lo * a.max_pages + keep + (r - back_at[lo])];
    };

    for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
        const int64_t row = (int64_t)b * a.max_pages;
        const bool bad = held[b] & kReserveBad;
        const int own = held[b] & ~kReserveBad;
        const int back = back_at[b + 1] - back_at[b], want = take_at[b + 1] - take_at[b];
        const bool served = !bad && (want == 0 || take_at[b + 1] <= have);
        if (!bad && !served && tid == 0) atomicOr(a.status, kStNoPages);
        const int take = served ? want : 0;
        const int32_t* in = a.before.block_table + row;
        int32_t* out = a.after.block_table + row;
        if (!a.in_place) {
            copy_ints(out, in, tid, own, kReserveThreads);
            copy_ints(out, in, own + take + tid, a.max_pages, kReserveThreads);
        }
        for (int j = own + tid; j < own + take; j += kReserveThreads) out[j] = taken(b, j - own);
        for (int r = tid; r < back; r += kReserveThreads) {
            const int at = free0 + back_at[b] + r;
            if (at < a.pages) a.after.free_list[at] = in[own - back + r];
        }
        const int ctx = a.ctx_len[b];
        const int add = !served ? 0 : a.new_len ? a.new_len[b] : a.T;
        for (int t = tid; t < a.T; t += kReserveThreads) {
            int64_t slot = -1;
            int pos = -1;
            if (t < add) {
                const int x = ctx + t, j = x / a.P;
                const int page = j < own ? in[j] : taken(b, j - own);
                if (page < 0 || page >= a.pages) {
                    atomicOr(a.status, kStBadIndex);
                } else {
                    slot = (int64_t)page * a.P + x % a.P;
                    pos = ctx + (a.depth ? a.depth[(int64_t)b * a.T + t] : t);
                }
            }
            a.slot[(int64_t)b * a.T + t] = slot;
            a.position[(int64_t)b * a.T + t] = pos;
        }
    }
    if (!a.in_place) {
        const int64_t at = (int64_t)blockIdx.x * kReserveThreads + tid, step = (int64_t)gridDim.x * kReserveThreads;
        copy_ints(a.after.free_list, a.before.free_list, at, free0, step);
        copy_ints(a.after.free_list, a.before.free_list, have + at, a.pages, step);
    }

    if (s_last) {
        // every CTA has its copy of the counts: they may change now
        int most = 0;  // pages taken: the last prefix that the stack could give
        for (int b = tid; b < a.B; b += kReserveThreads) {
            const bool bad = held[b] & kReserveBad;
            const int want = take_at[b + 1] - take_at[b];
            const bool served = !bad && take_at[b + 1] <= have;
            if (served) most = max(most, take_at[b + 1]);
            a.after.n_pages[b] = (held[b] & ~kReserveBad) - (back_at[b + 1] - back_at[b]) + (served ? want : 0);
        }
        most = __reduce_max_sync(0xffffffffu, most);
        if ((tid & 31) == 0) warp_sums[tid >> 5].x = most;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kReserveThreads / 32; ++w) most = max(most, warp_sums[w].x);
            *a.after.n_free = min(have, a.pages) - most;
            *a.ticket = 0;
        }
    }
}

cudaError_t launch_reserve(const ReserveArgs& a, int sms, cudaStream_t s) {
    const size_t smem = sizeof(int) * (3 * (size_t)a.B + 2);
    if (smem > 47 * 1024) {  // the kernel's static 80 bytes count towards the 48 KB that need no leave
        const cudaError_t err = cudaFuncSetAttribute(reserve_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (err != cudaSuccess) return err;
    }
    return launch_dependent(reserve_kernel, dim3(a.B < 2 * sms ? a.B : 2 * sms), dim3(kReserveThreads), smem, s, a);
}

// ---------------------------------------------------------------------------
// qk_norm_rope.  An item is one token and a run of its query heads, its key heads
// or its value heads; a warp takes items at a stride of all warps of the grid, and
// has the next one's slot and position on their way while it works on one.  A lane
// holds 16 bytes of a head (VEC elements; 8 bytes where the rotated part does not
// divide into pieces of 16), so 16 lanes hold a bf16 head of 128.  The loads of a
// run are issued first.  With w the weights, c and s the turn, x an element and y its
// pair, the result is (x (w c) + y (w' s)) / rms(x), in packed fp32 arithmetic: the
// two factors of a lane's elements are made once for the run, the sum of squares is
// a butterfly over the head's lanes, and the pair is in the same lane (interleaved) or
// rot / (2 VEC) lanes away (a shuffle of the raw elements).
// HBM bound: each input and output element crosses once.  33,024 tokens of 32 query
// and 8 key/value heads of 128 in bf16 take 140 us, 5.8 TB/s; what counts is bytes under way: 153, 149
// and 155 us with 8 (spills), 6 and 5 CTAs an SM; one item a warp 154; runs of 16
// heads with the next loads under way 158 to 185 (fewer warps); two loads a lane 176.
// ---------------------------------------------------------------------------
constexpr int kRopeThreads = 128;
constexpr int kRopeCtas = 7;  // resident on an SM

using F2 = unsigned long long;  // two floats for the packed fp32 instructions
__device__ __forceinline__ float f2_lo(F2 x) { return __uint_as_float((uint32_t)x); }
__device__ __forceinline__ float f2_hi(F2 x) { return __uint_as_float((uint32_t)(x >> 32)); }
__device__ __forceinline__ F2 f2_swap(F2 x) { return f2_pack(f2_hi(x), f2_lo(x)); }

template <int DT, int VEC> struct Piece;  // VEC neighbouring elements
template <> struct Piece<0, 4> {
    using Raw = float4;
    __device__ static __forceinline__ void wide(float4 r, F2 (&x)[2]) { x[0] = f2_pack(r.x, r.y), x[1] = f2_pack(r.z, r.w); }
    __device__ static __forceinline__ float4 narrow(const F2 (&x)[2]) {
        return make_float4(f2_lo(x[0]), f2_hi(x[0]), f2_lo(x[1]), f2_hi(x[1]));
    }
    __device__ static __forceinline__ float4 zero() { return make_float4(0, 0, 0, 0); }
};
__device__ __forceinline__ F2 bf16_wide(uint32_t x) { return f2_pack(bf_lo(x), bf_hi(x)); }
__device__ __forceinline__ uint32_t bf16_narrow(F2 x) {
    const __nv_bfloat162 y = __floats2bfloat162_rn(f2_lo(x), f2_hi(x));
    return *reinterpret_cast<const uint32_t*>(&y);
}
template <> struct Piece<1, 4> {
    using Raw = uint2;
    __device__ static __forceinline__ void wide(uint2 r, F2 (&x)[2]) { x[0] = bf16_wide(r.x), x[1] = bf16_wide(r.y); }
    __device__ static __forceinline__ uint2 narrow(const F2 (&x)[2]) { return make_uint2(bf16_narrow(x[0]), bf16_narrow(x[1])); }
    __device__ static __forceinline__ uint2 zero() { return make_uint2(0, 0); }
};
template <> struct Piece<1, 8> {
    using Raw = uint4;
    __device__ static __forceinline__ void wide(uint4 r, F2 (&x)[4]) {
        x[0] = bf16_wide(r.x), x[1] = bf16_wide(r.y), x[2] = bf16_wide(r.z), x[3] = bf16_wide(r.w);
    }
    __device__ static __forceinline__ uint4 narrow(const F2 (&x)[4]) {
        return make_uint4(bf16_narrow(x[0]), bf16_narrow(x[1]), bf16_narrow(x[2]), bf16_narrow(x[3]));
    }
    __device__ static __forceinline__ uint4 zero() { return make_uint4(0, 0, 0, 0); }
};

constexpr int kRopeRounds = 4;  // loads a lane has under way
template <int D, int VEC> __host__ __device__ constexpr int rope_heads() { return kRopeRounds * (32 * VEC / D); }

__device__ __forceinline__ uint32_t shfl_raw(uint32_t x, int from) { return __shfl_sync(0xffffffffu, x, from); }
__device__ __forceinline__ uint2 shfl_raw(uint2 x, int from) { return make_uint2(shfl_raw(x.x, from), shfl_raw(x.y, from)); }
__device__ __forceinline__ uint4 shfl_raw(uint4 x, int from) {
    return make_uint4(shfl_raw(x.x, from), shfl_raw(x.y, from), shfl_raw(x.z, from), shfl_raw(x.w, from));
}
__device__ __forceinline__ float4 shfl_raw(float4 x, int from) {
    return make_float4(__shfl_sync(0xffffffffu, x.x, from), __shfl_sync(0xffffffffu, x.y, from),
                       __shfl_sync(0xffffffffu, x.z, from), __shfl_sync(0xffffffffu, x.w, from));
}

template <int DT, int D, int VEC, bool INTERLEAVED>
__global__ void __launch_bounds__(kRopeThreads, kRopeCtas) rope_kernel(const RopeArgs a) {
    grid_dependency_begin();
    using Q = Piece<DT, VEC>;
    using Raw = typename Q::Raw;
    constexpr int LPH = D / VEC, HPW = 32 / LPH, HEADS = rope_heads<D, VEC>();
    constexpr int ES = DT == 1 ? 2 : 4;
    const int lane = threadIdx.x & 31, ci = lane & (LPH - 1), sub = lane / LPH, e = ci * VEC;
    const int q_runs = (a.Hq + HEADS - 1) / HEADS, kv_runs = (a.H + HEADS - 1) / HEADS, runs = q_runs + 2 * kv_runs;

    // items (token, run) at a stride of all warps, advanced without a division
    const int64_t item = (int64_t)blockIdx.x * (kRopeThreads / 32) + (threadIdx.x >> 5);
    const int64_t stride = (int64_t)gridDim.x * (kRopeThreads / 32), skip = stride / runs;
    const int skip_run = (int)(stride - skip * runs), skip_t = (int)(skip % a.T), skip_b = (int)(skip / a.T);
    const int64_t first_token = item / runs;
    int at = (int)(item - first_token * runs), t = (int)(first_token % a.T), b = (int)(first_token / a.T);
    int64_t slot_ahead = -1;
    int pos_ahead = 0;
    if (b < a.B) {
        slot_ahead = a.slot[first_token];
        pos_ahead = a.position[first_token];
    }
    while (b < a.B) {
        const int64_t slot = slot_ahead;
        const int pos = pos_ahead;
        // which: 0 queries, 1 keys, 2 values; the same for the whole warp
        const int which = at < q_runs ? 0 : at < q_runs + kv_runs ? 1 : 2;
        const int run = which == 0 ? at : which == 1 ? at - q_runs : at - q_runs - kv_runs;
        const int h0 = run * HEADS + sub, heads = which == 0 ? a.Hq : a.H;
        const char* in = static_cast<const char*>(which == 0 ? a.in.q : which == 1 ? a.in.k : a.in.v);
        const int64_t in_batch = which == 0 ? a.in.q_batch : which == 1 ? a.in.k_batch : a.in.v_batch;
        const int64_t in_token = which == 0 ? a.in.q_token : which == 1 ? a.in.k_token : a.in.v_token;
        const int64_t in_head = which == 0 ? a.in.q_head : which == 1 ? a.in.k_head : a.in.v_head;
        in += (b * in_batch + t * in_token + h0 * in_head + e) * ES;
        Raw raw[kRopeRounds];
#pragma unroll
        for (int r = 0; r < kRopeRounds; ++r)
            raw[r] = h0 + r * HPW < heads ? *reinterpret_cast<const Raw*>(in + r * HPW * in_head * ES) : Q::zero();
        char* const q_out = static_cast<char*>(a.q_out) + (b * a.o_batch + t * a.o_token) * ES;

        at += skip_run;
        const int carry = at >= runs;
        if (carry) at -= runs;
        t += skip_t + carry;
        b += skip_b;
        if (t >= a.T) t -= a.T, ++b;
        if (b < a.B) {
            const int64_t token = (int64_t)b * a.T + t;
            slot_ahead = a.slot[token];
            pos_ahead = a.position[token];
        }

        const bool inside = slot < a.slots && (a.rot == 0 || (pos >= 0 && pos < a.max_position));
        if (slot >= 0 && !inside && lane == 0) atomicOr(a.status, kStBadIndex);
        const bool live = slot >= 0 && inside;
        char* out = q_out;
        int64_t out_head = a.o_head;
        if (which != 0) {
            if (!live) continue;
            const int64_t page = slot >> a.page_shift, row = slot & ((1 << a.page_shift) - 1);
            out = static_cast<char*>(which == 1 ? a.kv.key : a.kv.value) +
                  (page * (which == 1 ? a.kv.key_page : a.kv.value_page) +
                   row * (which == 1 ? a.kv.key_token : a.kv.value_token)) * ES;
            out_head = which == 1 ? a.kv.key_head : a.kv.value_head;
        }
        out += (h0 * out_head + e) * ES;
        if (which == 2 || !live) {
#pragma unroll
            for (int r = 0; r < kRopeRounds; ++r)
                if (h0 + r * HPW < heads) *reinterpret_cast<Raw*>(out + r * HPW * out_head * ES) = live ? raw[r] : Q::zero();
            continue;
        }

        // factors of an element and of its pair
        const char* weight = static_cast<const char*>(which == 0 ? a.q_weight : a.k_weight);
        F2 fx[VEC / 2], fy[VEC / 2];
        int pair = lane;  // the lane that holds the pairs of this lane's elements
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) fx[i] = f2_pack(1.0f, 1.0f), fy[i] = 0ull;
        const bool turns = e < a.rot;
        if (weight) Q::wide(*reinterpret_cast<const Raw*>(weight + e * ES), fx);
        if (turns) {
            const float* cs = a.cos_sin + (int64_t)pos * a.rot;
            if (INTERLEAVED) {
#pragma unroll
                for (int i = 0; i < VEC / 2; i += 2) {
                    const float2 c2 = *reinterpret_cast<const float2*>(cs + e / 2 + i);
                    const float2 s2 = *reinterpret_cast<const float2*>(cs + a.rot / 2 + e / 2 + i);
                    fy[i] = f2_mul(f2_pack(-s2.x, s2.x), f2_swap(fx[i]));
                    fy[i + 1] = f2_mul(f2_pack(-s2.y, s2.y), f2_swap(fx[i + 1]));
                    fx[i] = f2_mul(fx[i], f2_pack(c2.x, c2.x));
                    fx[i + 1] = f2_mul(fx[i + 1], f2_pack(c2.y, c2.y));
                }
            } else {
                const bool first = e < a.rot / 2;
                const int from = first ? e : e - a.rot / 2;
                const float sign = first ? -1.0f : 1.0f;
                F2 w[VEC / 2];
#pragma unroll
                for (int i = 0; i < VEC / 2; ++i) w[i] = f2_pack(1.0f, 1.0f);
                if (weight) Q::wide(*reinterpret_cast<const Raw*>(weight + (first ? e + a.rot / 2 : from) * ES), w);
#pragma unroll
                for (int i = 0; i < VEC / 2; i += 2) {
                    const float4 c4 = *reinterpret_cast<const float4*>(cs + from + 2 * i);
                    const float4 s4 = *reinterpret_cast<const float4*>(cs + a.rot / 2 + from + 2 * i);
                    fx[i] = f2_mul(fx[i], f2_pack(c4.x, c4.y)), fx[i + 1] = f2_mul(fx[i + 1], f2_pack(c4.z, c4.w));
                    fy[i] = f2_mul(f2_pack(sign * s4.x, sign * s4.y), w[i]);
                    fy[i + 1] = f2_mul(f2_pack(sign * s4.z, sign * s4.w), w[i + 1]);
                }
                pair = first ? lane + a.rot / (2 * VEC) : lane - a.rot / (2 * VEC);
            }
        }
#pragma unroll
        for (int r = 0; r < kRopeRounds; ++r) {
            if (h0 - sub + r * HPW >= heads) break;  // the same for the whole warp
            F2 x[VEC / 2], y[VEC / 2];
            Q::wide(raw[r], x);
            // what does not turn has no pair: zeros, as 0 * inf is none of it
            if (INTERLEAVED) {
#pragma unroll
                for (int i = 0; i < VEC / 2; ++i) y[i] = turns ? f2_swap(x[i]) : 0ull;
            } else {
                const Raw other = shfl_raw(raw[r], pair);
                Q::wide(turns ? other : Q::zero(), y);
            }
            F2 inv = f2_pack(1.0f, 1.0f);
            if (weight) {
                F2 squares = f2_mul(x[0], x[0]);
#pragma unroll
                for (int i = 1; i < VEC / 2; ++i) squares = f2_fma(x[i], x[i], squares);
                float ss = f2_fold(squares);
#pragma unroll
                for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
                ss = rsqrtf(ss * (1.0f / D) + a.eps);
                inv = f2_pack(ss, ss);
            }
#pragma unroll
            for (int i = 0; i < VEC / 2; ++i) x[i] = f2_mul(f2_fma(y[i], fy[i], f2_mul(x[i], fx[i])), inv);
            if (h0 + r * HPW < heads) *reinterpret_cast<Raw*>(out + r * HPW * out_head * ES) = Q::narrow(x);
        }
    }
}

template <int DT, int D, int VEC, bool I>
static cudaError_t launch_rope_t(const RopeArgs& a, int sms, cudaStream_t s) {
    constexpr int heads = rope_heads<D, VEC>();
    const int runs = (a.Hq + heads - 1) / heads + 2 * ((a.H + heads - 1) / heads);
    const int64_t per = kRopeThreads / 32, ctas = ((int64_t)a.B * a.T * runs + per - 1) / per, most = (int64_t)sms * kRopeCtas;
    return launch_dependent(rope_kernel<DT, D, VEC, I>, dim3((unsigned)(ctas < most ? ctas : most)), dim3(kRopeThreads), 0,
                            s, a);
}
template <int DT, int D, int VEC>
static cudaError_t launch_rope_i(const RopeArgs& a, bool interleaved, int sms, cudaStream_t s) {
    return interleaved ? launch_rope_t<DT, D, VEC, true>(a, sms, s) : launch_rope_t<DT, D, VEC, false>(a, sms, s);
}

cudaError_t launch_rope(const RopeArgs& a, int dtype, int D, bool interleaved, int sms, cudaStream_t s) {
    const bool wide = D == 128;
    if (dtype == 0) return wide ? launch_rope_i<0, 128, 4>(a, interleaved, sms, s) : launch_rope_i<0, 64, 4>(a, interleaved, sms, s);
    if (a.rot % 16 == 0)
        return wide ? launch_rope_i<1, 128, 8>(a, interleaved, sms, s) : launch_rope_i<1, 64, 8>(a, interleaved, sms, s);
    return wide ? launch_rope_i<1, 128, 4>(a, interleaved, sms, s) : launch_rope_i<1, 64, 4>(a, interleaved, sms, s);
}

// ---------------------------------------------------------------------------
// commit.  A thread owns one 16-byte column of (layer, key or value, head) and
// moves it for all nodes of a request's path.  Places are written in ascending
// order and node k lies at or behind place k+1, so a batch of loads followed by
// its stores never overwrites a line that a later batch reads.  Lines already
// in place are left alone.  The bytes are few: bound by launch and by two
// dependent rounds of loads (path, table), then HBM.  A path of six in 32 layers,
// and 64 paths in 16 layers (25 MB): 3.0 and 6.4 us in a captured graph, 8.5 each from
// Python, which the call bounds.
// ---------------------------------------------------------------------------
constexpr int kCommitThreads = 256;
constexpr int kCommitBatch = 8;
constexpr int kMaxPath = 128;

__global__ void __launch_bounds__(kCommitThreads) commit_kernel(const CommitArgs a, int cols) {
    grid_dependency_begin();
    __shared__ int2 src[kMaxPath], dst[kMaxPath];  // page, row
    const int tid = threadIdx.x, b = blockIdx.y;
    const int ctx = a.ctx_len[b], n = a.accepted_len[b];
    const int64_t capacity = (int64_t)a.max_pages * a.P;
    unsigned bad = 0;
    if (n < 0 || n > a.depth) bad = kStBadIndex;
    if (ctx < 0 || ctx + (int64_t)1 + (n > 0 ? n : 0) > capacity) bad |= kStBadLength;
    int moves = 0;
    if (!bad && tid < n) {
        const int32_t* path = a.accepted_nodes + (int64_t)b * a.depth;
        const int node = path[tid], before = tid > 0 ? path[tid - 1] : 0;
        const int64_t from = (int64_t)ctx + node, to = (int64_t)ctx + tid + 1;
        if (node <= before || node < tid + 1 || node >= a.T) {
            bad = kStBadIndex;
        } else if (from >= capacity) {
            bad = kStBadLength;
        } else {
            const int32_t* table = a.block_table + (int64_t)b * a.max_pages;
            src[tid] = make_int2(table[from / a.P], (int)(from % a.P));
            dst[tid] = make_int2(table[to / a.P], (int)(to % a.P));
            if (src[tid].x < 0 || src[tid].x >= a.pages || dst[tid].x < 0 || dst[tid].x >= a.pages) bad = kStBadIndex;
            moves = from != to;
        }
    }
    if (bad) atomicOr(a.status, bad);
    const int any_bad = __syncthreads_or(bad != 0);
    const int any_move = __syncthreads_or(moves);
    if (blockIdx.x == 0 && tid == 0) a.next_len[b] = any_bad ? ctx : ctx + 1 + n;
    if (any_bad || !any_move) return;

    const int64_t i = (int64_t)blockIdx.x * kCommitThreads + tid;
    const int col = (int)(i % cols);
    const int64_t line = i / cols;
    const int h = (int)(line % a.H), which = (int)(line / a.H % 2);
    const int64_t layer = line / a.H / 2;
    if (layer >= a.layers) return;
    const int es = a.kv_elem_bytes;
    char* base = which ? static_cast<char*>(a.kv.value) + (layer * a.value_layer + h * a.kv.value_head) * es
                       : static_cast<char*>(a.kv.key) + (layer * a.key_layer + h * a.kv.key_head) * es;
    const int64_t page_stride = (which ? a.kv.value_page : a.kv.key_page) * es;
    const int64_t row_stride = (which ? a.kv.value_token : a.kv.key_token) * es;
    base += col * 16;
    for (int k0 = 0; k0 < n; k0 += kCommitBatch) {
        uint4 x[kCommitBatch];
#pragma unroll
        for (int u = 0; u < kCommitBatch; ++u)
            if (k0 + u < n)
                x[u] = *reinterpret_cast<const uint4*>(base + src[k0 + u].x * page_stride + src[k0 + u].y * row_stride);
#pragma unroll
        for (int u = 0; u < kCommitBatch; ++u)
            if (k0 + u < n && (src[k0 + u].x != dst[k0 + u].x || src[k0 + u].y != dst[k0 + u].y))
                *reinterpret_cast<uint4*>(base + dst[k0 + u].x * page_stride + dst[k0 + u].y * row_stride) = x[u];
    }
}

cudaError_t launch_commit(const CommitArgs& a, int line_bytes, cudaStream_t s) {
    const int cols = line_bytes / 16;
    const int64_t threads = (int64_t)a.layers * 2 * a.H * cols;
    return launch_dependent(commit_kernel, dim3((unsigned)((threads + kCommitThreads - 1) / kCommitThreads), a.B),
                            dim3(kCommitThreads), 0, s, a, cols);
}

}  // namespace rheo
