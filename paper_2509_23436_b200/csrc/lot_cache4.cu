// The 4-bit cache: tokens quantised as they are written, and read back.
//
// A group of 32 channels of a token and head is held as s = bf16((hi - lo) / 15), z = bf16(lo) and codes round((x - z) / s), half to even.
// The quotients are taken in float32; where one comes so near to the border between two results that its rounding could fall on the
// other side, it is taken in float64, so that what is stored depends on the definition alone.
// A warp takes a block of 16 places of one head and side, which lies in one page: a lane eight channels of every group of two tokens, so that
// rows are read and written in 64-byte pieces and codes in whole words; the values' codes change from the tokens' order to the operands'
// by three exchanges between lanes.
#include "lot_window.cuh"

#include <type_traits>

namespace lot {
namespace window {
namespace {

constexpr int kThreads = 256;

// What float32 cannot decide, out of line: only groups next to a border of the scale, or of magnitudes near the type's ends, come here.
__device__ __noinline__ float exact_scale(float lo, float hi) { return (float)(((double)hi - (double)lo) / 15.0); }
__device__ __noinline__ uint32_t exact_code(float x, float z, float s) { return (uint32_t)fmin(fmax(rint(((double)x - (double)z) / (double)s), 0.0), 15.0); }

// scale of a group: ((hi - lo) / 15) rounded to float32 and then to bf16, as the bits of the bf16
__device__ __forceinline__ uint32_t scale_bits(float lo, float hi)
{
    const float q = (hi - lo) * (1.f / 15.f);
    uint32_t u = __float_as_uint(q);
    const uint32_t low = u & 0xffffu;
    // q is within 3 ulp of the exact quotient: only next to the middle between two bf16 numbers can that matter
    if ((low >= 0x7ff8u && low <= 0x8008u) || !(q < 1e30f) || (q < 1e-30f && hi != lo)) u = __float_as_uint(exact_scale(lo, hi));
    return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}
// The code of x when (x - z) / s is next to h = below + 1/2: the sign of x - z - h s.  d + e is x - z exactly, h s (13 bits) is exact and so is
// its difference with d, which it nearly equals.  bf16 tensors, whose differences and scales have few bits, come exactly between two
// codes in one of 500 channels.
__device__ __forceinline__ uint32_t border_code(float x, float z, float s, float below)
{
    const float hs = (below + 0.5f) * s, d = x - z, b = d - x, e = (x - (d - b)) - (z + b), t = (d - hs) + e;
    const uint32_t n = (uint32_t)below;
    return t > 0.f ? n + 1u : t < 0.f ? n : n + (n & 1u);
}
// Codes of eight channels; s > 0.  clamp: quotients may lie outside 0 .. 15.5 (a least value that was rounded to bf16).
template <bool CLAMP> __device__ __forceinline__ uint32_t codes_of(const float (&x)[8], float z, float s)
{
    constexpr float kWhole = 12582912.f;                       // 1.5 x 2^23: adding it rounds to a whole number, half to even
    constexpr float kNear = 0.5f - 6e-6f;                      // three roundings and an approximate reciprocal: within 15.1 x 4 x 2^-24 = 3.6e-6
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
    const f2 inv2 = pack2(inv, inv), z2 = pack2(-z, -z), whole = pack2(kWhole, kWhole), back = pack2(-kWhole, -kWhole), minus = pack2(-1.f, -1.f);
    f2 n[4], off[4];                                           // channels c and c + 4
    float near = 0.f;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        f2 r = mul2(add2(pack2(x[c], x[c + 4]), z2), inv2);
        if (CLAMP) {
            float u, v;
            unpack2(r, u, v);
            r = pack2(fminf(fmaxf(u, 0.f), 15.f), fminf(fmaxf(v, 0.f), 15.f));
        }
        n[c] = add2(add2(r, whole), back);
        off[c] = fma2(n[c], minus, r);
        float u, v;
        unpack2(off[c], u, v);
        near = fmaxf(near, fmaxf(fabsf(u), fabsf(v)));
    }
    // four codes in one number below 2^16, exactly
    const f2 by16 = pack2(16.f, 16.f), word = add2(fma2(fma2(n[3], by16, n[2]), pack2(256.f, 256.f), fma2(n[1], by16, n[0])), pack2(8388608.f, 8388608.f));
    float lo, hi;
    unpack2(word, lo, hi);
    uint32_t codes = __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x5410);
    if (s < 1e-30f || s > 1e30f) {
        codes = 0;
#pragma unroll
        for (int c = 0; c < 8; ++c) codes |= exact_code(x[c], z, s) << (4 * c);
    } else if (near > kNear) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            float u, v, m, w;
            unpack2(off[c], u, v);
            unpack2(n[c], m, w);
            if (fabsf(u) > kNear) codes = (codes & ~(15u << (4 * c))) | border_code(x[c], z, s, u > 0.f ? m : m - 1.f) << (4 * c);
            if (fabsf(v) > kNear) codes = (codes & ~(15u << (4 * c + 16))) | border_code(x[c + 4], z, s, v > 0.f ? w : w - 1.f) << (4 * c + 16);
        }
    }
    return codes;
}

// The same for bf16 channels, in fewer instructions.  d = x - z is exact where adding z gives x back; then a quotient corrected by its exact
// remainder is the quotient of d and s to half an ulp: a quotient half way between two codes (one channel in 500) comes out as exactly
// that, any other is a 2^-17th or more away from it (d has 17 bits at most, s 8), and adding 1.5 x 2^23 rounds half to even.
__device__ __forceinline__ uint32_t codes_of_bf16(const float (&x)[8], float z, float s)
{
    constexpr float kWhole = 12582912.f;
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
    const f2 inv2 = pack2(inv, inv), z2 = pack2(z, z), whole = pack2(kWhole, kWhole), back = pack2(-kWhole, -kWhole), minus = pack2(-z, -z), s2 = pack2(-s, -s);
    f2 n[4];
    uint32_t lost = 0;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const f2 v = pack2(x[c], x[c + 4]), d = add2(v, minus), r = mul2(d, inv2), q = fma2(fma2(r, s2, d), inv2, r);
        lost |= (uint32_t)(add2(d, z2) ^ v) | (uint32_t)((add2(d, z2) ^ v) >> 32);
        n[c] = add2(add2(q, whole), back);
    }
    if ((lost & 0x7fffffffu) != 0 || s < 1e-30f || s > 1e30f) return codes_of<false>(x, z, s);
    const f2 by16 = pack2(16.f, 16.f), word = add2(fma2(fma2(n[3], by16, n[2]), pack2(256.f, 256.f), fma2(n[1], by16, n[0])), pack2(8388608.f, 8388608.f));
    float lo, hi;
    unpack2(word, lo, hi);
    return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x5410);
}

// least and largest of eight channels; NaN if one is
__device__ __forceinline__ float min_nan(float a, float b)
{
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint32_t min_nan2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_nan2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// Eight channels of a lane as they were loaded, and the least and largest of its group (lanes 4 and 8 apart).
template <typename T> struct Eight;
template <> struct Eight<float> {
    float x[8];
    __device__ __forceinline__ void load(const float *p)
    {
        const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int c = 0; c < 8; ++c) x[c] = 0.f;
    }
    __device__ __forceinline__ void range(float &lo, float &hi) const
    {
        lo = min_nan(min_nan(min_nan(x[0], x[1]), min_nan(x[2], x[3])), min_nan(min_nan(x[4], x[5]), min_nan(x[6], x[7])));
        hi = max_nan(max_nan(max_nan(x[0], x[1]), max_nan(x[2], x[3])), max_nan(max_nan(x[4], x[5]), max_nan(x[6], x[7])));
#pragma unroll
        for (int o = 4; o < 16; o <<= 1) {
            lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
            hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        }
    }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
#pragma unroll
        for (int c = 0; c < 8; ++c) v[c] = x[c];
    }
};
template <> struct Eight<__nv_bfloat16> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const __nv_bfloat16 *p)
    {
        const uint4 a = *reinterpret_cast<const uint4 *>(p);
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
    }
    __device__ __forceinline__ void clear() { w[0] = w[1] = w[2] = w[3] = 0u; }
    __device__ __forceinline__ void range(float &lo, float &hi) const
    {
        uint32_t a = min_nan2(min_nan2(w[0], w[1]), min_nan2(w[2], w[3])), b = max_nan2(max_nan2(w[0], w[1]), max_nan2(w[2], w[3]));
        a = min_nan2(a, __byte_perm(a, a, 0x1032));
        b = max_nan2(b, __byte_perm(b, b, 0x1032));
        a = __byte_perm(a, b, 0x5410);                         // least below, largest above: both cross the lanes in one word
#pragma unroll
        for (int o = 4; o < 16; o <<= 1) {
            const uint32_t y = __shfl_xor_sync(0xffffffffu, a, o);
            a = __byte_perm(min_nan2(a, y), max_nan2(a, y), 0x7610);
        }
        lo = __uint_as_float(a << 16);
        hi = __uint_as_float(a & 0xffff0000u);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
};
__device__ __forceinline__ void store8(float *p, const float (&v)[8])
{
    *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float (&v)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&t);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

struct Rows {
    Cache4 c;
    const int32_t *start, *count;
    int m, shift;                          // shift: log2 of the page size where that is whole, else -1
    int *status;
};

// A warp's block of 16 places.
struct Block {
    int first, m, at, page;                // first: the call's token at the block's first place (may be negative); m tokens in all; page < 0: none
    __device__ __forceinline__ bool has(int j) const { return first + j >= 0 && first + j < m; }
};
__device__ __forceinline__ Block block_of(const Rows &r, int b, int n, int lane)
{
    Block k;
    const int start = r.start[b];
    k.m = r.count != nullptr ? min(max(r.count[b], 0), r.m) : r.m;
    k.first = n * kBlockTokens - (start & 15);
    k.at = 0;
    k.page = -1;
    if (k.first >= k.m) { k.m = 0; return k; }
    const uint32_t pos = (uint32_t)start + (uint32_t)k.first;       // places before the first wrap round to beyond the last
    if (pos < (uint32_t)(r.c.max_pages * r.c.page_size)) {
        const uint32_t page = r.shift >= 0 ? pos >> r.shift : pos / (uint32_t)r.c.page_size;
        k.at = (int)(pos - page * r.c.page_size);
        k.page = r.c.pages[(size_t)b * r.c.max_pages + page];
        if (k.page >= r.c.num_pages) k.page = -1;
    }
    if (k.page < 0 && lane == 0 && r.status != nullptr) atomicOr(r.status, 32 /* LOT_DEV_PAGE */);
    return k;
}

// Lane 4 x + t, x = 4 e + i, holds words of eight nibbles: token 2 t + e, channels 8 i .. 8 i + 7 of a group.  Afterwards it holds the same
// group's stored word of lane (g, t), g = x: nibble 4 e + i is token 2 t + e's channel 8 i + g.  Three exchanges, each of one bit of x with
// one bit of the nibble's number; its own inverse.
__device__ __forceinline__ uint32_t exchange(uint32_t w, int lane)
{
    const uint32_t a = __shfl_xor_sync(0xffffffffu, w, 4);
    w = lane & 4 ? (w & 0xf0f0f0f0u) | ((a >> 4) & 0x0f0f0f0fu) : (w & 0x0f0f0f0fu) | ((a << 4) & 0xf0f0f0f0u);
    const uint32_t b = __shfl_xor_sync(0xffffffffu, w, 8);
    w = lane & 8 ? (w & 0xff00ff00u) | ((b >> 8) & 0x00ff00ffu) : (w & 0x00ff00ffu) | ((b << 8) & 0xff00ff00u);
    const uint32_t c = __shfl_xor_sync(0xffffffffu, w, 16);
    return lane & 16 ? (w & 0xffff0000u) | (c >> 16) : (w & 0x0000ffffu) | (c << 16);
}

template <int W> struct Words;
template <> struct Words<1> { typedef uint32_t T; };
template <> struct Words<2> { typedef uint2 T; };
template <> struct Words<4> { typedef uint4 T; };
template <int W> __device__ __forceinline__ void store_words(void *p, const uint32_t (&w)[W])
{
    typename Words<W>::T v;
    memcpy(&v, w, sizeof v);
    *static_cast<typename Words<W>::T *>(p) = v;
}
template <int W> __device__ __forceinline__ void load_words(const void *p, uint32_t (&w)[W])
{
    const typename Words<W>::T v = __ldg(static_cast<const typename Words<W>::T *>(p));
    memcpy(w, &v, sizeof v);
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) write_kernel(const __grid_constant__ Rows r, const T *k, const T *v)
{
    constexpr int W = D / kGroup;
    const int lane = threadIdx.x & 31, b = blockIdx.z, head = blockIdx.y >> 1, side = blockIdx.y & 1, t = lane & 3, i = (lane >> 2) & 3, e = lane >> 4;
    const Block blk = block_of(r, b, (int)(blockIdx.x * (blockDim.x / 32) + (threadIdx.x >> 5)), lane);
    if (blk.m == 0 || blk.page < 0) return;
    const T *x0 = (side ? v : k) + ((size_t)b * r.c.Hkv + head) * r.m * D + (long long)blk.first * D + i * 8;
    Eight<T> x[2][W];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int j = 8 * u + 2 * t + e;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            if (blk.has(j)) x[u][w].load(x0 + j * D + w * kGroup);
            else x[u][w].clear();
        }
    }
    uint8_t *base = side_base(r.c, blk.page, head, side);
    uint32_t *params = reinterpret_cast<uint32_t *>(base + (size_t)r.c.page_size * (D / 2));
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int j = 8 * u + 2 * t + e;
        uint32_t codes[W], param[W];
#pragma unroll
        for (int w = 0; w < W; ++w) {
            float lo, hi;
            x[u][w].range(lo, hi);
            codes[w] = 0;
            param[w] = 0x7fc07fc0u;                            // a value that is not finite: NaN for the group
            if (fmaxf(fabsf(lo), fabsf(hi)) < __int_as_float(0x7f800000) && lo == lo) {
                const uint32_t sb = scale_bits(lo, hi), zb = __float_as_uint(lo), zr = (zb + 0x7fffu + ((zb >> 16) & 1u)) & 0xffff0000u;
                const float s = __uint_as_float(sb << 16), z = __uint_as_float(zr);
                param[w] = sb | zr;
                if (s > 0.f) {
                    float y[8];
                    x[u][w].get(y);
                    // bf16 tensors: z is the least value itself and (hi - z) / s at most 15 (1 + 2^-8)
                    codes[w] = sizeof(T) == 4 ? codes_of<true>(y, z, s) : codes_of_bf16(y, z, s);
                }
            }
        }
        if (blk.has(j) && i == 0) store_words(params + (size_t)(blk.at + j) * W, param);
        if (side == 0) {
            if (blk.has(j)) store_words(base + (size_t)(blk.at + j) * (D / 2) + i * 4 * W, codes);
            continue;
        }
#pragma unroll
        for (int w = 0; w < W; ++w) codes[w] = exchange(codes[w], lane);
        uint8_t *o = base + value_half(blk.at + 8 * u + 2 * t, lane >> 2, 0, W);
        const bool even = blk.has(8 * u + 2 * t), odd = blk.has(8 * u + 2 * t + 1);
        if (even && odd) {
            store_words(o, codes);
        } else if (even || odd) {
#pragma unroll
            for (int w = 0; w < W; ++w) *reinterpret_cast<uint16_t *>(o + 4 * w + (odd ? 2 : 0)) = (uint16_t)(odd ? codes[w] >> 16 : codes[w]);
        }
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) read_kernel(const __grid_constant__ Rows r, T *k, T *v)
{
    constexpr int W = D / kGroup;
    const int lane = threadIdx.x & 31, b = blockIdx.z, head = blockIdx.y >> 1, side = blockIdx.y & 1, t = lane & 3, i = (lane >> 2) & 3, e = lane >> 4;
    const Block blk = block_of(r, b, (int)(blockIdx.x * (blockDim.x / 32) + (threadIdx.x >> 5)), lane);
    if (blk.m == 0) return;
    uint32_t codes[2][W], param[2][W];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int j = 8 * u + 2 * t + e;
#pragma unroll
        for (int w = 0; w < W; ++w) codes[u][w] = param[u][w] = 0;
        if (blk.page < 0) continue;                            // a token whose page is missing reads as zeros
        const uint8_t *base = side_base(r.c, blk.page, head, side);
        load_words(reinterpret_cast<const uint32_t *>(base + (size_t)r.c.page_size * (D / 2)) + (size_t)(blk.at + j) * W, param[u]);
        load_words(side ? base + value_half(blk.at + 8 * u + 2 * t, lane >> 2, 0, W) : base + (size_t)(blk.at + j) * (D / 2) + i * 4 * W, codes[u]);
    }
    T *x0 = (side ? v : k) + ((size_t)b * r.c.Hkv + head) * r.m * D + (long long)blk.first * D + i * 8;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int j = 8 * u + 2 * t + e;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            if (side) codes[u][w] = exchange(codes[u][w], lane);
            if (!blk.has(j)) continue;
            const float s = param_scale(param[u][w]), z = param_least(param[u][w]);
            float x[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) x[c] = fmaf(s, (float)((codes[u][w] >> (4 * c)) & 15u), z);
            store8(x0 + j * D + w * kGroup, x);
        }
    }
}

template <typename F> cudaError_t by_width(int dtype, int d, F f)
{
    if (dtype == 0) return d == 32 ? f(float{}, std::integral_constant<int, 32>{}) : d == 64 ? f(float{}, std::integral_constant<int, 64>{}) : f(float{}, std::integral_constant<int, 128>{});
    return d == 32 ? f(__nv_bfloat16{}, std::integral_constant<int, 32>{}) : d == 64 ? f(__nv_bfloat16{}, std::integral_constant<int, 64>{}) : f(__nv_bfloat16{}, std::integral_constant<int, 128>{});
}
// Blocks of 16 places that m tokens may touch, up to eight in a thread block.
struct Shape {
    dim3 grid;
    unsigned threads;
    int shift;
};
Shape shape_of(const Cache4 &c, int B, int m)
{
    const int blocks = (int)(((long long)m + 2 * (kBlockTokens - 1)) / kBlockTokens), warps = blocks < kThreads / 32 ? blocks : kThreads / 32;
    int shift = -1;
    for (int i = 4; i < 29; ++i)
        if (c.page_size == 1 << i) shift = i;
    return Shape{dim3((unsigned)((blocks + warps - 1) / warps), 2 * c.Hkv, B), 32u * warps, shift};
}

} // namespace

cudaError_t launch_write4(const Cache4 &c, const void *k, const void *v, const int32_t *start, const int32_t *count, int dtype, int B, int m, int *status,
                          cudaStream_t st)
{
    return by_width(dtype, c.d, [&](auto t, auto width) {
        using T = decltype(t);
        const Shape s = shape_of(c, B, m);
        write_kernel<T, decltype(width)::value><<<s.grid, s.threads, 0, st>>>(Rows{c, start, count, m, s.shift, status}, static_cast<const T *>(k), static_cast<const T *>(v));
        return cudaGetLastError();
    });
}
cudaError_t launch_read4(const Cache4 &c, void *k, void *v, const int32_t *start, const int32_t *count, int dtype, int B, int m, int *status,
                         cudaStream_t st)
{
    return by_width(dtype, c.d, [&](auto t, auto width) {
        using T = decltype(t);
        const Shape s = shape_of(c, B, m);
        read_kernel<T, decltype(width)::value><<<s.grid, s.threads, 0, st>>>(Rows{c, start, count, m, s.shift, status}, static_cast<T *>(k), static_cast<T *>(v));
        return cudaGetLastError();
    });
}

} // namespace window
} // namespace lot
