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
    int b, item, unit;  // class, item within it, unit within that
    __device__ __forceinline__ int owner(int64_t t) const { return (int)((t * n + n - 1) / total); }
};

// Computed by one warp, over `classes` (requests, or their groups of query rows) of `per` items each, which have
// tiles_of(class) tiles.
template <class F>
__device__ __forceinline__ AttendCut attend_cut_over(const AttendArgs& a, int classes, int per, int cta, F tiles_of) {
    const int lane = threadIdx.x & 31;
    AttendCut c;
    if (classes <= 32 && 4 * (int64_t)classes * per <= a.ctas) {
        const int tiles = lane < classes ? tiles_of(lane) : 0;
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
    for (int b = lane; b < classes; b += 32) sum += tiles_of(b) + a.lead;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    c.total = sum * per;
    c.n = c.total < a.ctas ? (int)c.total : a.ctas;
    c.lead = a.lead;
    c.chunks = 0;
    c.begin = cta < c.n ? (int64_t)cta * c.total / c.n : c.total;
    c.end = cta < c.n ? (int64_t)(cta + 1) * c.total / c.n : c.total;
    c.b = classes;
    c.item = c.unit = 0;
    int64_t before = 0;  // units of the classes before this round of 32
    for (int b0 = 0; b0 < classes; b0 += 32) {
        const int b = b0 + lane;
        const int64_t mine = b < classes ? (int64_t)(tiles_of(b) + a.lead) * per : 0;
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

// Every request a class of `per` items that walk all its places.
template <int TILE> __device__ __forceinline__ AttendCut attend_cut(const AttendArgs& a, int per, int cta) {
    return attend_cut_over(a, a.B, per, cta, [&](int b) { return attend_tiles<TILE>(a, b); });
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
    __device__ __forceinline__ void open(int len) { open_tiles(max(1, (len + TILE - 1) / TILE)); }
    __device__ __forceinline__ void open_tiles(int tiles) {
        all = tiles;
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

// ---------------------------------------------------------------------------
// Windows and packed pages.  A class is (request, group of query rows), an item one
// key/value head of it.  Places 0 .. pk-1 are packed, the others lie in 16 bits; the tiles
// of the two parts are numbered one part behind the other, each part from its first place, so no tile
// is of both kinds.  An item's tiles are the first `sinks` ones and those from w0 on.
// ---------------------------------------------------------------------------
struct LongSpan {
    int pk, ctx, add;  // packed tokens, all cached ones, new ones; all 0 where a number is bad
    bool bad;
    __device__ __forceinline__ int len() const { return ctx + add; }
};

__device__ __forceinline__ LongSpan long_span(const AttendArgs& a, int b) {
    const int near = a.ctx_len[b], add = a.new_len ? a.new_len[b] : a.T, n4 = a.packed.data ? a.n_pages4[b] : 0;
    const bool bad = near < 0 || add < 0 || add > a.T || (int64_t)near + add > (int64_t)a.max_pages * a.P || n4 < 0 ||
                     n4 > a.max_pages4;
    return bad ? LongSpan{0, 0, 0, true} : LongSpan{n4 * a.P, n4 * a.P + near, add, false};
}

// Depth of new token t, and the first place of its window (0: from the start).
__device__ __forceinline__ int long_depth(const AttendArgs& a, int b, int t) {
    return a.depth ? min(max(a.depth[(int64_t)b * a.T + t], 0), a.T - 1) : t;
}
__device__ __forceinline__ int long_first(const AttendArgs& a, const LongSpan& s, int depth) {
    return a.window ? max(0, s.ctx + depth - a.window + 1) : 0;
}

template <int TILE> struct LongItem {
    LongSpan s;
    int np;            // tiles of the packed part
    int ns, w0, n;     // tiles of the sinks, first one of the window, all of the item
    int lo, lo_most;   // first place of the window of any of the item's tokens, and the last such first place
    int sinks;         // places below it are seen whatever the window (0 without one)
    int sinks_end;     // where the sinks' tiles end: at the last sink, if the window begins behind them
    __device__ __forceinline__ LongItem() {}
    // Rows r0 .. r0 + count - 1 of request b's (token, query head) pairs.
    __device__ __forceinline__ LongItem(const AttendArgs& a, int b, int r0, int count) {
        s = long_span(a, b);
        np = (s.pk + TILE - 1) / TILE;
        const int t0 = r0 / a.G, t1 = min((min(r0 + count, a.T * a.G) - 1) / a.G, s.add - 1);
        ns = n = 1;
        w0 = sinks = 0;
        lo = lo_most = sinks_end = INT32_MAX;
        if (t0 >= s.add) return;  // no row is of a token: one tile, of which nothing is seen or read
        lo = lo_most = 0;
        const int hi = a.mask ? s.len() : s.ctx + t1 + 1;
        ns = 0;
        if (a.window) {
            lo = long_first(a, s, a.depth ? 0 : t0);
            lo_most = long_first(a, s, a.depth ? a.T - 1 : t1);
            sinks = a.sinks;
            if (sinks > 0) ns = index(min(sinks, hi) - 1) + 1;
        }
        const int from = index(min(lo, hi - 1));
        w0 = max(ns, from);
        sinks_end = from >= ns ? sinks : INT32_MAX;
        n = ns + index(hi - 1) + 1 - w0;
    }
    __device__ __forceinline__ int index(int place) const {
        return place < s.pk ? place / TILE : np + (place - s.pk) / TILE;
    }
    __device__ __forceinline__ int number(int i) const { return i < ns ? i : i - ns + w0; }  // of the item's i-th tile
    __device__ __forceinline__ bool is_packed(int number) const { return number < np; }
    __device__ __forceinline__ int begin(int number) const { return number < np ? number * TILE : s.pk + (number - np) * TILE; }
    __device__ __forceinline__ int end(int number) const {
        const int e = number < np ? min(number * TILE + TILE, s.pk) : min(s.pk + (number - np + 1) * TILE, s.len());
        return number < ns ? min(e, sinks_end) : e;
    }
    __device__ __forceinline__ int packed_tiles() const { return np <= ns ? np : ns + max(0, min(np, w0 - ns + n) - w0); }
    // whether some token of the item may see one of `count` places from `place` on
    __device__ __forceinline__ bool wanted(int place, int count) const { return place < sinks || place + count > lo; }
    // Whether a token, with its depth's first place, sees place l; row_mask: its row of the mask.
    __device__ __forceinline__ bool sees(const AttendArgs& a, int b, const uint8_t* row_mask, int t, int first, int l) const {
        const int j = l - s.ctx;
        int position = l;
        if (j >= 0) {
            if (j >= s.add || !(row_mask ? row_mask[j] != 0 : j <= t)) return false;
            position = s.ctx + long_depth(a, b, j);
        }
        return position >= first || position < sinks;
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
