// pack.cu -- whole pages of the 16-bit cache into 4 bits (cache_pack) and back
// (cache_unpack).
//
// A warp takes 32 tokens of 64 channels of a head (two pages where a page has 16
// tokens): lane (o, j) has the tokens 8j .. 8j + 7 of the channels 8o .. 8o + 7, eight
// loads of 16 bytes.  Keys: the largest magnitude of a channel over the lane's tokens,
// then over the lanes j; values: of a token over the lane's channels, then over four
// lanes o.  The codes that a lane makes are two whole words of 16 bytes of either kind.
//
// Rounding without divisions: magnitudes have 8 significant bits and scales 4, so
// max / 7 is a scale, or at least 2^-8 of it away from one, and x / s is half-way between two
// codes, or at least 2^-9 away.  So the reciprocals are taken 2^-20 to one side: max / 7 a little low, so
// that a maximum of exactly 7 s gets s; x / s a little high, so that a half goes away from 0.
// A fused multiply-add with 1.5 * 2^23 + 8 leaves n + 8 in the low bits of the sum.
//
// What bounds it: HBM, sixteen loads of 16 bytes a lane under way.  The prompts of 16 requests (503 to 9,001 tokens, 4 layers, 8
// heads of 128) packed and unpacked again 521 us, 5.8 TB/s (86 % of a copy's rate); three prefixes of 4,099 to 12,001 tokens in 8
// layers unpacked 174 us, 5.7 TB/s.  A page of each of 32 layers: a launch for the pages and one for the tables, dependent latencies.
#include <cuda_bf16.h>

#include "cache_kernels.h"
#include "packed.cuh"
#include "rheo_device.cuh"
#include "rheo_kernels.h"

namespace rheo {
namespace {

constexpr int kPackThreads = 256;
constexpr int kPackBad = 1 << 30;      // mark of a request whose numbers are bad
constexpr uint32_t kPackMost = 0x4752u;  // 53760 in bf16: 7 times the largest scale

// Where the lanes of a warp stand in a run of 32 tokens and 64 channels.
struct PackLane {
    int o, j;  // octet of channels, octet of tokens
    __device__ __forceinline__ PackLane() : o(threadIdx.x & 7), j((threadIdx.x & 31) >> 3) {}
};

// Offsets of lane (octet og of the head's channels, token octet jn of the block) in a block.
__device__ __forceinline__ int pack_key_at(int N, int og, int jn, int part) {
    return (((og >> 2) * (N / 4) + 2 * jn + part) * 4 + (og & 3)) * 16;
}
__device__ __forceinline__ int pack_value_at(int N, int D, int og, int jn, int part) {
    return N * D / 2 + (((og >> 2) * 8 + 2 * (og & 3) + part) * (N / 8) + jn) * 16;
}
__device__ __forceinline__ int pack_key_scale_at(int N, int D, int og) { return N * D + 8 * og; }
__device__ __forceinline__ int pack_value_scale_at(int N, int D, int og, int jn) {
    return N * D + D + (og >> 2) * N + 8 * jn;
}

__device__ __forceinline__ uint32_t max_abs(uint32_t a, uint32_t b) {  // of pairs; NaN stays
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b & 0x7FFF7FFFu));
    return r;
}
__device__ __forceinline__ bool past_most(uint32_t pair) {  // a magnitude that no scale reaches, or none at all
    return (pair & 0xFFFFu) > kPackMost || (pair >> 16) > kPackMost;
}
// Numbers outside +-7 s of the largest scale become its ends, NaN 0.
__device__ __forceinline__ uint32_t to_range(uint32_t pair) {
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t x = pair >> (16 * i) & 0xFFFFu, m = x & 0x7FFFu;
        r |= (m > 0x7F80u ? 0u : m > kPackMost ? (x & 0x8000u) | kPackMost : x) << (16 * i);
    }
    return r;
}
// The scale byte for a largest magnitude.
__device__ __forceinline__ uint32_t scale_byte(float top) {
    const float s = top * (0.14285714f * (1.0f - 0x1p-20f));
    return (uint32_t)min(max((int)((__float_as_uint(s) + 0xFFFFFu) >> 20) - 108 * 8, 0), 255);
}
__device__ __forceinline__ float scale_inverse(uint32_t byte) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(__uint_as_float((byte + 108 * 8) << 20)));
    return r * (1.0f + 0x1p-20f);
}
__device__ __forceinline__ uint32_t code_of(float x, float inverse) { return __float_as_uint(fmaf(x, inverse, 12582920.0f)); }
// Eight codes (n + 8 in the low 16 bits) as a word.
__device__ __forceinline__ uint32_t word_of(const uint32_t (&n)[8]) {
    uint32_t u = 0;
#pragma unroll
    for (int p = 0; p < 4; ++p) u += __byte_perm(n[2 * p], n[2 * p + 1], 0x5410) << (4 * p);
    return __funnelshift_l(u, u, 3);
}
__device__ __forceinline__ uint32_t part(const uint4& x, int i) { return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w; }
__device__ __forceinline__ float element(const uint4& x, int c) {
    const uint32_t w = part(x, c / 2);
    return c % 2 ? bf_hi(w) : bf_lo(w);
}
__device__ __forceinline__ uint2 eight_bytes(const uint32_t (&b)[8]) {
    return make_uint2(b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24, b[4] | b[5] << 8 | b[6] << 16 | b[7] << 24);
}
__device__ __forceinline__ void to_range_all(uint4 (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = make_uint4(to_range(x[i].x), to_range(x[i].y), to_range(x[i].z), to_range(x[i].w));
}

// Both halves of a warp's run: x[i] is token i of the lane's octet.  True where a number was not in range.
template <bool KEYS>
__device__ __forceinline__ bool pack_run(uint4 (&x)[8], int N, uint4 (&words)[2], uint2& scales) {
    uint32_t tops[4];  // keys: pairs of channels; values: pairs of tokens
    bool odd = false;
#pragma unroll 1
    for (int round = 0; round < 2; ++round) {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            if (KEYS) {
                tops[p] = part(x[0], p) & 0x7FFF7FFFu;
#pragma unroll
                for (int i = 1; i < 8; ++i) tops[p] = max_abs(tops[p], part(x[i], p));
            } else {
                uint32_t two[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint4& y = x[2 * p + e];
                    two[e] = max_abs(max_abs(max_abs(y.x & 0x7FFF7FFFu, y.y), y.z), y.w);
                }
                tops[p] = max_abs(__byte_perm(two[0], two[1], 0x5410), __byte_perm(two[0], two[1], 0x7632));
            }
            if (KEYS) {
                tops[p] = max_abs(tops[p], __shfl_xor_sync(0xffffffffu, tops[p], 8));
                if (N == 32) tops[p] = max_abs(tops[p], __shfl_xor_sync(0xffffffffu, tops[p], 16));
            } else {
                tops[p] = max_abs(tops[p], __shfl_xor_sync(0xffffffffu, tops[p], 1));
                tops[p] = max_abs(tops[p], __shfl_xor_sync(0xffffffffu, tops[p], 2));
            }
        }
        const bool past = past_most(tops[0]) || past_most(tops[1]) || past_most(tops[2]) || past_most(tops[3]);
        if (!__any_sync(0xffffffffu, past)) break;
        odd |= past;
        to_range_all(x);
    }
    uint32_t bytes[8];
    float inverse[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        bytes[e] = scale_byte(e % 2 ? bf_hi(tops[e / 2]) : bf_lo(tops[e / 2]));
        inverse[e] = scale_inverse(bytes[e]);
    }
    scales = eight_bytes(bytes);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t n[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)  // keys: the token h + 2i, its channels; values: the channel h + 2i, its tokens
                n[e] = code_of(KEYS ? element(x[h + 2 * i], e) : element(x[e], h + 2 * i), inverse[e]);
            w[i] = word_of(n);
        }
        words[h] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return odd;
}

// Inclusive sum over the block, in units that every thread adds to.
__device__ __forceinline__ int block_scan(int v, int* warp_sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += x;
    }
    if (lane == 31) warp_sums[warp] = v;
    __syncthreads();
    for (int w = 0; w < warp; ++w) v += warp_sums[w];
    __syncthreads();
    return v;
}

// How many pages request b is to have packed; kPackBad where its numbers are bad.
__device__ __forceinline__ int pack_wants(const PackArgs& a, int b) {
    const int ctx = a.ctx_len[b], n = a.before.n_pages[b], n4 = a.before4.n_pages[b];
    if (n < 0 || n > a.max_pages || n4 < 0 || n4 > a.max_pages4 || ctx < 0 || ctx > (int64_t)n * a.P) return kPackBad;
    const int k = ctx > a.keep ? (ctx - a.keep) / a.P : 0;
    return n4 + k > a.max_pages4 ? kPackBad : k;
}

__device__ __forceinline__ int stack_height(const int32_t* n_free, int pages) { return min(max(*n_free, 0), pages); }

// Every CTA derives the plan by itself (pages that each request packs, and their sums
// before it, in shared memory), and its warps take runs of 32 tokens at a stride of
// the grid.  CTA 0 leaves the plan for the tables' launch.  The first requests, as far as the
// stack of 4-bit pages reaches, are served: sums only grow.
__global__ void __launch_bounds__(kPackThreads) pack_kernel(const PackArgs a) {
    grid_dependency_begin();
    extern __shared__ int page_at[];  // [B + 1] pages packed before request b
    __shared__ int warp_sums[kPackThreads / 32];
    __shared__ int carry;
    const int tid = threadIdx.x;
    const int free4 = stack_height(a.before4.n_free, a.pages4);
    if (tid == 0) carry = page_at[0] = 0;
    __syncthreads();
    unsigned bad = 0;
    for (int b0 = 0; b0 < a.B; b0 += kPackThreads) {
        const int b = b0 + tid;
        int k = b < a.B ? pack_wants(a, b) : 0;
        if (k == kPackBad) bad |= kStBadLength, k = 0;
        const int upto = carry + block_scan(k, warp_sums);  // (ends in a barrier after the reads of carry)
        if (b < a.B) {
            page_at[b + 1] = upto;
            if (k > 0 && upto > free4) bad |= kStNoPages;
        }
        __syncthreads();
        if (tid == kPackThreads - 1) carry = upto;
        __syncthreads();
    }
    if (blockIdx.x == 0) {
        if (tid == 0 && (*a.before4.n_free != free4 || *a.before.n_free != stack_height(a.before.n_free, a.pages))) bad |= kStInternal;
        for (int b = tid; b <= a.B; b += kPackThreads) a.plan[b] = page_at[b];
        if (tid == 0) a.plan[a.B + 1] = stack_height(a.before.n_free, a.pages), a.plan[a.B + 2] = free4;
        if (bad) atomicOr(a.status, bad);
    }
    // the last request that is served, and the pages up to it
    int lo = 0, hi = a.B;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (page_at[mid] <= free4) lo = mid;
        else hi = mid - 1;
    }
    // runs of 32 tokens over all pages in order: where a page has 16 tokens a run is two of them, of any requests
    const int total = page_at[lo], N = packed_tokens(a.P), halves = a.D / 64;
    const int64_t runs = ((int64_t)total * a.P + 31) / 32, units = runs * a.H * halves * a.layers;
    const int64_t stride = (int64_t)gridDim.x * (kPackThreads / 32);
    const PackLane at;
    for (int64_t u = (int64_t)blockIdx.x * (kPackThreads / 32) + (tid >> 5); u < units; u += stride) {
        const int half = (int)(u % halves), h = (int)(u / halves % a.H);
        const int64_t run = u / halves / a.H % runs, layer = u / halves / a.H / runs;
        const int64_t token = run * 32 + 8 * at.j;
        const int i = (int)(token / a.P), row = (int)(token % a.P);  // page of the call, token in it
        int page = -1, page4 = -1;
        if (i < total) {
            int first = 0, last = lo - 1;  // the request with page_at[first] <= i < page_at[first + 1]
            while (first < last) {
                const int mid = (first + last + 1) >> 1;
                if (page_at[mid] <= i) first = mid;
                else last = mid - 1;
            }
            page = a.before.block_table[(int64_t)first * a.max_pages + i - page_at[first]];
            page4 = a.before4.free_list[free4 - 1 - i];
            if (page < 0 || page >= a.pages || page4 < 0 || page4 >= a.pages4) {
                atomicOr(a.status, kStBadIndex);
                page = -1;
            }
        }
        const int og = half * 8 + at.o;
        const char* key = static_cast<const char*>(a.kv.key) +
                          (layer * a.key_layer + page * a.kv.key_page + h * a.kv.key_head + row * a.kv.key_token + og * 8) * 2;
        const char* value = static_cast<const char*>(a.kv.value) + (layer * a.value_layer + page * a.kv.value_page +
                                                                    h * a.kv.value_head + row * a.kv.value_token + og * 8) * 2;
        uint4 x[8], y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = y[e] = make_uint4(0, 0, 0, 0);
            if (page >= 0) {
                x[e] = *reinterpret_cast<const uint4*>(key + e * a.kv.key_token * 2);
                y[e] = *reinterpret_cast<const uint4*>(value + e * a.kv.value_token * 2);
            }
        }
        uint4 kw[2], vw[2];
        uint2 ks, vs;
        bool odd = pack_run<true>(x, N, kw, ks);
        odd |= pack_run<false>(y, N, vw, vs);
        if (odd) atomicOr(a.status, kStBadValue);
        if (page >= 0) {
            const int jn = at.j & (N / 8 - 1);
            uint8_t* block = a.packed.data + layer * a.packed_layer + page4 * a.packed.page + h * a.packed.head +
                             row / N * packed_block_bytes(N, a.D);
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                *reinterpret_cast<uint4*>(block + pack_key_at(N, og, jn, p)) = kw[p];
                *reinterpret_cast<uint4*>(block + pack_value_at(N, a.D, og, jn, p)) = vw[p];
            }
            if (jn == 0) *reinterpret_cast<uint2*>(block + pack_key_scale_at(N, a.D, og)) = ks;
            if ((og & 3) == 0) *reinterpret_cast<uint2*>(block + pack_value_scale_at(N, a.D, og, jn)) = vs;
        }
        __syncwarp();
    }
}

// The tables after that: a CTA a request, from the plan alone and the request's own entries, so that it may
// be done in place.
__global__ void __launch_bounds__(kPackThreads) pack_tables_kernel(const PackArgs a) {
    grid_dependency_begin();
    const int tid = threadIdx.x;
    const int free0 = a.plan[a.B + 1], free4 = a.plan[a.B + 2];
    for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
        const int first = a.plan[b], upto = a.plan[b + 1];
        const int k = upto <= free4 ? upto - first : 0;
        const int64_t row = (int64_t)b * a.max_pages, row4 = (int64_t)b * a.max_pages4;
        const int32_t* in = a.before.block_table + row;
        int32_t* out = a.after.block_table + row;
        const int n = a.before.n_pages[b], n4 = a.before4.n_pages[b], ctx = a.ctx_len[b];
        for (int j = tid; j < k; j += kPackThreads)
            if (free0 + first + j < a.pages) a.after.free_list[free0 + first + j] = in[j];
        __syncthreads();  // these entries have been read
        const int most = a.in_place ? n : a.max_pages;
        for (int j0 = 0; j0 < most && (k > 0 || !a.in_place); j0 += kPackThreads) {
            const int j = j0 + tid;
            int page = 0;
            if (j < most) page = in[j + k < n ? j + k : j];
            __syncthreads();  // a place is written after the places up to k before it were read
            if (j < most && (!a.in_place || j + k < n)) out[j] = page;
        }
        for (int j = tid; j < a.max_pages4; j += kPackThreads) {
            const bool fresh = j >= n4 && j < n4 + k;
            if (fresh || !a.in_place)
                a.after4.block_table[row4 + j] = fresh ? a.before4.free_list[free4 - 1 - (first + j - n4)] : a.before4.block_table[row4 + j];
        }
        __syncthreads();  // the counts have been read
        if (tid == 0) {
            a.after.n_pages[b] = n - k;
            a.after4.n_pages[b] = n4 + k;
            a.ctx_out[b] = ctx - k * a.P;
        }
    }
    // the stacks: what is not put on them now keeps its value
    int lo = 0, hi = a.B;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.plan[mid] <= free4) lo = mid;
        else hi = mid - 1;
    }
    const int total = a.plan[lo], have = min(free0 + total, a.pages);
    if (!a.in_place) {
        const int64_t at = (int64_t)blockIdx.x * kPackThreads + tid, step = (int64_t)gridDim.x * kPackThreads;
        for (int64_t i = at; i < a.pages; i += step)
            if (i < free0 || i >= have) a.after.free_list[i] = a.before.free_list[i];
        for (int64_t i = at; i < a.pages4; i += step) a.after4.free_list[i] = a.before4.free_list[i];
    }
    if (blockIdx.x == 0 && tid == 0) {
        if (free0 + total > a.pages) atomicOr(a.status, kStInternal);
        *a.after.n_free = have;
        *a.after4.n_free = free4 - total;
    }
}

// The other way, page by page of a list: the same lanes, words to rows of 16 bytes.
__global__ void __launch_bounds__(kPackThreads) unpack_kernel(const UnpackArgs a) {
    grid_dependency_begin();
    const int tid = threadIdx.x, N = packed_tokens(a.P), halves = a.D / 64;
    const int64_t runs = ((int64_t)a.n * a.P + 31) / 32, units = runs * a.H * halves * a.layers;
    const int64_t stride = (int64_t)gridDim.x * (kPackThreads / 32);
    const PackLane at;
    for (int64_t u = (int64_t)blockIdx.x * (kPackThreads / 32) + (tid >> 5); u < units; u += stride) {
        const int half = (int)(u % halves), h = (int)(u / halves % a.H);
        const int64_t run = u / halves / a.H % runs, layer = u / halves / a.H / runs;
        const int64_t token = run * 32 + 8 * at.j, i = token / a.P;
        const int row = (int)(token % a.P);
        if (i >= a.n) continue;
        const int page4 = a.src[i], page = a.dst[i];
        if (page4 == -1 || page == -1) continue;
        if (page < 0 || page >= a.pages || page4 < 0 || page4 >= a.pages4) {
            atomicOr(a.status, kStBadIndex);
            continue;
        }
        const int og = half * 8 + at.o, jn = at.j & (N / 8 - 1);
        const uint8_t* block = a.packed.data + layer * a.packed_layer + page4 * a.packed.page + h * a.packed.head +
                               row / N * packed_block_bytes(N, a.D);
        uint4 kw[2], vw[2];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            kw[p] = *reinterpret_cast<const uint4*>(block + pack_key_at(N, og, jn, p));
            vw[p] = *reinterpret_cast<const uint4*>(block + pack_value_at(N, a.D, og, jn, p));
        }
        const uint2 ks = *reinterpret_cast<const uint2*>(block + pack_key_scale_at(N, a.D, og));
        const uint2 vs = *reinterpret_cast<const uint2*>(block + pack_value_scale_at(N, a.D, og, jn));
        char* key = static_cast<char*>(a.kv.key) +
                    (layer * a.key_layer + page * a.kv.key_page + h * a.kv.key_head + row * a.kv.key_token + og * 8) * 2;
        char* value = static_cast<char*>(a.kv.value) +
                      (layer * a.value_layer + page * a.kv.value_page + h * a.kv.value_head + row * a.kv.value_token + og * 8) * 2;
        uint32_t s[4], c[4];
        packed_scales(ks, s, c);
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            uint32_t d[4][4];  // token p + 2i, its channels
            packed_words(kw[p], s, c, d);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<uint4*>(key + (p + 2 * q) * a.kv.key_token * 2) = make_uint4(d[q][0], d[q][1], d[q][2], d[q][3]);
        }
        packed_scales(vs, s, c);
        uint32_t even[4][4], uneven[4][4];  // channels 2i and 2i + 1: pairs of tokens
        packed_words(vw[0], s, c, even);
        packed_words(vw[1], s, c, uneven);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint32_t w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) w[q] = __byte_perm(even[q][e / 2], uneven[q][e / 2], e % 2 ? 0x7632 : 0x5410);
            *reinterpret_cast<uint4*>(value + e * a.kv.value_token * 2) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

// CTAs for `units` warps' worth of work at most, `per` resident on an SM.
int pack_grid(int64_t units, int sms, int per) {
    const int64_t ctas = (units + kPackThreads / 32 - 1) / (kPackThreads / 32);
    return (int)(ctas < (int64_t)sms * per ? (ctas > 0 ? ctas : 1) : (int64_t)sms * per);
}

}  // namespace

cudaError_t launch_pack(const PackArgs& a, int sms, cudaStream_t s) {
    const int64_t pages = (int64_t)a.B * a.max_pages < a.pages4 ? (int64_t)a.B * a.max_pages : a.pages4;
    const int64_t units = (pages * a.P + 31) / 32 * a.H * (a.D / 64) * a.layers;
    cudaError_t err = launch_dependent(pack_kernel, dim3(pack_grid(units, sms, 2)), dim3(kPackThreads),
                                       sizeof(int) * ((size_t)a.B + 1), s, a);
    if (err != cudaSuccess) return err;
    return launch_dependent(pack_tables_kernel, dim3(a.B < 2 * sms ? a.B : 2 * sms), dim3(kPackThreads), 0, s, a);
}

cudaError_t launch_unpack(const UnpackArgs& a, int sms, cudaStream_t s) {
    const int64_t units = ((int64_t)a.n * a.P + 31) / 32 * a.H * (a.D / 64) * a.layers;
    return launch_dependent(unpack_kernel, dim3(pack_grid(units, sms, 4)), dim3(kPackThreads), 0, s, a);
}

}  // namespace rheo
