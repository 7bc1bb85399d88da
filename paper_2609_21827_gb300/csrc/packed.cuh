// packed.cuh -- pages held in 4 bits: where a page's numbers lie, and how they
// become bf16.
//
// A page of one head is P / N blocks, one behind the other; a block holds N =
// min(P, 32) tokens of D channels as n s with n in -7 .. 7:
//   key codes     [D/32][N/4][4] words of 16 bytes: word (x, r, t) has the tokens f(r, 0..3), channels 32x + 8t + (0..7)
//   value codes   [D/32][8][N/8]                    word (x, r, t) has the channels 32x + f(r, 0..3), tokens 8t + (0..7)
//   key scales    [D]        one byte a channel, for the block's tokens
//   value scales  [D/32][N]  one byte a token, for 32 channels
// with f(r, i) = 8 (r / 2) + r % 2 + 2i.  So lane (r, t) = (lane / 4, lane % 4) of a
// warp reads 16 bytes that are its operands of an m16n8k16 product over 32 tokens or 32
// channels: part i of the 16 bytes is row f(r, i), its eight codes are neighbours
// in the summed direction.
// Keys share a scale along the tokens because single channels are large in every
// token; values along the channels, as their weighted sum runs over tokens.
//
// Scale byte c: s = (1 + (c & 7) / 8) 2^((c >> 3) - 19), the smallest with 7 s >= max
// |x|.  Four significant bits, so that n s has seven and bf16 holds it exactly.
// The 32 bits of part i: n + 8 of element 2p at bit 3 + 4p, of 2p + 1 at bit 19 + 4p
// (modulo 32).  A pair under the mask 0x00780078 with 16 (0x4180) above it is 16 + n + 8
// in bf16, and one fused multiply-add with s and -24 s gives n s: exact, as 24 s has six
// significant bits.
#pragma once

#include <stdint.h>

namespace rheo {

__host__ __device__ constexpr int packed_tokens(int P) { return P < 32 ? P : 32; }
__host__ __device__ constexpr int packed_block_bytes(int N, int D) { return N * D + D + N * D / 32; }
__host__ __device__ constexpr int packed_page_bytes(int P, int D) {
    return P / packed_tokens(P) * packed_block_bytes(packed_tokens(P), D);
}
constexpr uint32_t kPackedZero = 0x44444444u;  // eight codes of 0: n + 8 = 8 in each

// The pairs of scales s and of -24 s of eight scale bytes.
__device__ __forceinline__ void packed_scales(uint2 bytes, uint32_t (&s)[4], uint32_t (&c)[4]) {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const uint32_t two = __byte_perm(p < 2 ? bytes.x : bytes.y, 0, p % 2 == 0 ? 0x4140 : 0x4342);
        s[p] = two * 16 + 0x36003600u;  // exponents move by 127 - 19 = 108
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(c[p]) : "r"(s[p]), "r"(0xC1C0C1C0u));
    }
}
// The four bf16 pairs of a word.  (One lop3 a pair: written in C++ it became two, 1,150 instructions a tile for 1,020.)
__device__ __forceinline__ void packed_word(uint32_t w, const uint32_t (&s)[4], const uint32_t (&c)[4], uint32_t (&out)[4]) {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const uint32_t x = p == 0 ? w : p == 3 ? __funnelshift_r(w, w, 12) : w >> (4 * p);
        uint32_t n;
        asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(n) : "r"(x), "r"(0x00780078u), "r"(0x41804180u));  // (x & mask) | sixteens
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(out[p]) : "r"(n), "r"(s[p]), "r"(c[p]));
    }
}
__device__ __forceinline__ void packed_words(uint4 w, const uint32_t (&s)[4], const uint32_t (&c)[4], uint32_t (&out)[4][4]) {
    packed_word(w.x, s, c, out[0]);
    packed_word(w.y, s, c, out[1]);
    packed_word(w.z, s, c, out[2]);
    packed_word(w.w, s, c, out[3]);
}

}  // namespace rheo
