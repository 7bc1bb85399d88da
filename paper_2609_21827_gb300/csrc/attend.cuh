// attend.cuh -- what the attention kernels share: how the key tiles of all
// requests are cut over the CTAs, and which places a token sees.
//
// An item is (request, key/value head, group of query rows): the rows of a
// group are consecutive (token, query head of the key/value head) pairs, so
// that one read of a key tile serves all query heads that share it.  An item of
// request b has ceil((ctx + new) / tile) key tiles, one at least.
//
// Many items: all of them lie on one line, each as `lead` units for its start
// and end and one unit a tile; CTA i of n takes the units [i total / n, (i+1)
// total / n), whatever the lengths are, so ragged contexts keep every SM as busy
// as equal ones.  Few items (a quarter of the CTAs at most): each is cut by
// itself, into chunks of at most the least size (from `least` on: smaller ones
// cost more in their join than they save) with which the chunks of all items fit
// the CTAs, so that no CTA pays for the start of two.
// An item cut by a boundary leaves partial sums: CTA i keeps at most two, slot
// 2i for one that began in an earlier CTA and slot 2i+1 for one that goes on in
// a later CTA.
#pragma once

#include "cache_kernels.h"
#include "rheo_device.cuh"

namespace rheo {

struct AttendSpan {  // a request's lengths, checked
    int ctx, add;    // cached tokens, new tokens; both 0 where a length is bad
    bool bad;
    __device__ __forceinline__ int len() const { return ctx + add; }
};

__device__ __forceinline__ AttendSpan attend_span(const AttendArgs& a, int b) {
    const int ctx = a.ctx_len[b], add = a.new_len ? a.new_len[b] : a.T;
    const bool bad = ctx < 0 || add < 0 || add > a.T || (int64_t)ctx + add > (int64_t)a.max_pages * a.P;
    return bad ? AttendSpan{0, 0, true} : AttendSpan{ctx, add, false};
}

template <int TILE> __device__ __forceinline__ int attend_tiles(const AttendArgs& a, int b) {
    const int n = (attend_span(a, b).len() + TILE - 1) / TILE;
    return n > 0 ? n : 1;
}

struct AttendCut {      // one CTA's range of units, and where it starts
    int64_t total;
    int n;              // CTAs that take part
    int lead;           // units before an item's first tile
    int chunks;         // CTAs of this CTA's only item; 0: the items lie on the line
    int64_t begin, end;
    int b, item, unit;  // request, item within it, unit within that
    __device__ __forceinline__ int owner(int64_t t) const { return (int)((t * n + n - 1) / total); }
};

// Computed by one warp; `per` items a request.
template <int TILE> __device__ __forceinline__ AttendCut attend_cut(const AttendArgs& a, int per, int cta) {
    const int lane = threadIdx.x & 31;
    AttendCut c;
    if (a.B <= 32 && 4 * (int64_t)a.B * per <= a.ctas) {
        const int tiles = lane < a.B ? attend_tiles<TILE>(a, lane) : 0;
        int hi = __reduce_max_sync(0xffffffffu, tiles), lo = min(a.least, hi);  // the least size of a chunk that fits
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (__reduce_add_sync(0xffffffffu, (tiles + mid - 1) / mid) * per <= a.ctas) hi = mid;
            else lo = mid + 1;
        }
        const int mine = (tiles + lo - 1) / lo;  // chunks of an item of this lane's request
        int upto = mine * per;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        const unsigned past = __ballot_sync(0xffffffffu, upto > cta);
        c.lead = 0;
        c.chunks = 1;
        c.n = c.b = c.item = c.unit = 0;
        c.total = c.begin = c.end = 0;
        if (past) {
            const int l = __ffs(past) - 1;
            const int at = cta - __shfl_sync(0xffffffffu, upto - mine * per, l), t = __shfl_sync(0xffffffffu, tiles, l);
            c.chunks = __shfl_sync(0xffffffffu, mine, l);
            c.b = l;
            c.item = at / c.chunks;
            const int k = at % c.chunks;
            c.unit = (int)((int64_t)k * t / c.chunks);
            c.end = (int)((int64_t)(k + 1) * t / c.chunks) - c.unit;
        }
        return c;
    }
    int64_t sum = 0;
    for (int b = lane; b < a.B; b += 32) sum += attend_tiles<TILE>(a, b) + a.lead;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    c.total = sum * per;
    c.n = c.total < a.ctas ? (int)c.total : a.ctas;
    c.lead = a.lead;
    c.chunks = 0;
    c.begin = cta < c.n ? (int64_t)cta * c.total / c.n : c.total;
    c.end = cta < c.n ? (int64_t)(cta + 1) * c.total / c.n : c.total;
    c.b = a.B;
    c.item = c.unit = 0;
    int64_t before = 0;  // units of the requests before this round of 32
    for (int b0 = 0; b0 < a.B; b0 += 32) {
        const int b = b0 + lane;
        const int64_t mine = b < a.B ? (int64_t)(attend_tiles<TILE>(a, b) + a.lead) * per : 0;
        int64_t upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        const unsigned past = __ballot_sync(0xffffffffu, before + upto > c.begin);
        if (past) {
            const int l = __ffs(past) - 1;
            const int64_t first = __shfl_sync(0xffffffffu, before + upto - mine, l);
            const int units = (int)(__shfl_sync(0xffffffffu, mine, l) / per);
            c.b = b0 + l;
            c.item = (int)((c.begin - first) / units);
            c.unit = (int)((c.begin - first) % units);
            break;
        }
        before += __shfl_sync(0xffffffffu, upto, 31);
    }
    return c;
}

// One CTA's run through its items, the same in every warp: `tile` and `n` are
// the first tile and the tiles of the item at hand, set by open().
template <int TILE> struct AttendWalk {
    int b, item, unit, lead, tile, n, all, took;
    int64_t at, end;
    __device__ __forceinline__ explicit AttendWalk(const AttendCut& c)
        : b(c.b), item(c.item), unit(c.unit), lead(c.lead), at(c.begin), end(c.end) {}
    // whether a tile is left (the units before an item's first tile are none)
    __device__ __forceinline__ bool more() const { return at + max(0, lead - unit) < end; }
    __device__ __forceinline__ void open(int len) {
        all = max(1, (len + TILE - 1) / TILE);
        took = (int)min((int64_t)(all + lead - unit), end - at);
        tile = max(0, unit - lead);
        n = unit + took - lead - tile;
    }
    __device__ __forceinline__ bool last() const { return at + took + lead >= end; }
    __device__ __forceinline__ void next(int per) {
        at += took;
        unit = 0;
        if (++item == per) {
            item = 0;
            ++b;
        }
    }
    // CTAs that sum the item at hand, of which this one has the first tile
    __device__ __forceinline__ int segments(const AttendCut& c, int cta) const {
        return c.chunks ? c.chunks : c.owner(at - unit + lead + all - 1) - cta + 1;
    }
};

// Whether new token t (of `add`) sees place l of its request.
__device__ __forceinline__ bool attend_sees(const AttendSpan& s, const uint8_t* mask_row, int t, int l) {
    const int j = l - s.ctx;
    if (j < 0) return true;
    if (j >= s.add) return false;
    return mask_row ? mask_row[j] != 0 : j <= t;
}

// The slot of a.part_o / a.part_ml for CTA `cta`'s part of an item that it does not hold whole.
__device__ __forceinline__ int64_t attend_part(int cta, bool starts_here) { return 2 * (int64_t)cta + (starts_here ? 1 : 0); }

// Four columns (group c4) of row r of a part: rows side by side, as the threads that write and read them are.
__device__ __forceinline__ int64_t attend_part_at(const AttendArgs& a, int64_t part, int r, int c4) {
    return (part * (a.D / 4) + c4) * a.part_rows + r;
}

__device__ __forceinline__ float attend_lse(float m, float l) {
    return l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

}  // namespace rheo
