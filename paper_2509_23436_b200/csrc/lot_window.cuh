// Device helpers of window attention and the 4-bit cache: what a query sees, the stored rows' layout.
#pragma once

#include "lot_common.cuh"
#include "lot_window.h"

namespace lot {
namespace window {

// ---- two float32 numbers an instruction ------------------------------------------------------------------------------------
typedef unsigned long long f2;
__device__ __forceinline__ f2 pack2(float a, float b)
{
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(f2 x, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ f2 add2(f2 a, f2 b)
{
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b)
{
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c)
{
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// Keys of one batch row: query i stands at p = pos + i and sees [max(p - left, 0), hi(p)] and the first `sinks` keys up to hi(p).
struct Row {
    int pos, len;                          // len: keys that exist and that some query of the row may see
    int left, right, sinks, first;         // first: no query sees a key before it but the sinks
    __device__ __forceinline__ int hi(int p) const { return min(p + right, len - 1); }
    __device__ __forceinline__ int lo(int p) const { return max(p - left, 0); }
    __device__ __forceinline__ bool sees(int p, int j) const { return j <= hi(p) && (j >= p - left || j < sinks); }
    __device__ __forceinline__ bool used(int j) const { return j < len && (j >= first || j < sinks); }
};

__device__ __forceinline__ Row row_of(const Band &b, int batch)
{
    Row r;
    r.left = b.left;
    r.right = b.right;
    r.sinks = b.sinks;
    int len = b.nk;
    if (b.key_len != nullptr) len = min(max(b.key_len[batch], 0), b.nk);
    r.pos = b.q_start != nullptr ? min(max(b.q_start[batch], -kMaxPos), kMaxPos) : b.nk - b.nq;
    r.first = max(r.pos - r.left, 0);
    r.len = max(min(len, r.pos + b.nq + r.right), 0);
    return r;
}

// ---- the 4-bit cache ---------------------------------------------------------------------------------------------------
// A page's area of one head and side: d / 2 bytes of codes a token, then a word (scale, least value; bf16 each) for each group of 32
// channels of a token.  The codes stand in the order in which the attention's 16 x 8 x 16 products take them, W = d / 32 groups:
//   keys    a token's d / 2 bytes after the other's; 32-bit word t W + w (t < 4): channels 32 w + 8 t .. + 7, lowest nibble first:
//           lane (g, t) of a product finds its channels of key g, all groups, in W neighbouring words
//   values  blocks of 16 tokens; the half of channels 32 w + g, + 8, + 16, + 24 (lowest nibble first, g < 8) of token j is half
//           ((j / 8 * 32 + 4 g + j / 2 % 4) W + w) * 2 + j % 2 of the block: lane (g, t) finds its channels of keys 2 t and 2 t + 1 side by
//           side in a word, so that one mask gives both entries of an operand register, and all groups in W neighbouring words
constexpr int kGroup = 32, kBlockTokens = 16;
__host__ __device__ inline size_t side_bytes(int page_size, int d) { return (size_t)page_size * (d / 2 + d / 8); }

__device__ __forceinline__ uint8_t *side_base(const Cache4 &c, int page, int head, int side)
{
    return c.base + (((size_t)page * c.Hkv + head) * 2 + side) * side_bytes(c.page_size, c.d);
}
// byte of half (g, w) of the values of the page's token `at`
__device__ __forceinline__ int value_half(int at, int g, int w, int W)
{
    const int j = at & 15;
    return (at >> 4) * (kBlockTokens * 16 * W) + ((((j >> 3) * 32 + 4 * g + ((j >> 1) & 3)) * W + w) * 2 + (j & 1)) * 2;
}
__device__ __forceinline__ float param_scale(uint32_t p) { return __uint_as_float(p << 16); }
__device__ __forceinline__ float param_least(uint32_t p) { return __uint_as_float(p & 0xffff0000u); }

} // namespace window
} // namespace lot
