// The 4-bit cache: tokens quantised as they are written, and read back.
//
// A group of 32 channels of a token and head is held as s = bf16((hi - lo) / 15), z = bf16(lo) and codes round((x - z) / s), half to even.
// Four lanes share a group, eight channels each.  The quotients are taken in float32; where one comes so near to the border between two
// results that its rounding could fall on the other side, it is taken in float64, so that what is stored depends on the definition alone.
// Both kernels are bound by what they read and write; a warp takes neighbouring tokens (by their place in the cache, so that the two
// tokens whose value codes share words are neighbours in it) and stores whole words.
#include "lot_window.cuh"

#include <type_traits>

namespace lot {
namespace window {
namespace {

constexpr int kThreads = 256;

// scale of a group: ((hi - lo) / 15) rounded to float32 and then to bf16, as the bits of the bf16
__device__ __forceinline__ uint32_t scale_bits(float lo, float hi)
{
    const float q = __fdiv_rn(hi - lo, 15.f);
    uint32_t u = __float_as_uint(q);
    const uint32_t low = u & 0xffffu;
    // q is within 2 ulp of the exact quotient: only next to the middle between two bf16 numbers can that matter
    if ((low >= 0x7ffcu && low <= 0x8004u) || !(q < 1e30f) || q < 1e-30f) u = __float_as_uint((float)(((double)hi - (double)lo) / 15.0));
    return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}
__device__ __forceinline__ uint32_t code_of(float x, float z, float s, float inv)
{
    const float r = (x - z) * inv;                             // within 1e-5 of the exact quotient where s is in the ordinary range
    float n = rintf(r);
    if (fabsf(fabsf(r - n) - 0.5f) < 1e-4f || s < 1e-30f || s > 1e30f) n = (float)rint(((double)x - (double)z) / (double)s);
    return (uint32_t)fminf(fmaxf(n, 0.f), 15.f);
}

__device__ __forceinline__ void load8(const float *p, float (&v)[8])
{
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16 *p, float (&v)[8])
{
    const uint4 a = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
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
    int m;
    int *status;
};

// The token of this thread: its index in the call (or -1: none here), page and place.  Threads of a token and of its pair agree.
struct Token {
    int i, page, at;
};
__device__ __forceinline__ Token token_of(const Rows &r, int b, int slot)
{
    const int start = r.start[b], m = r.count != nullptr ? min(max(r.count[b], 0), r.m) : r.m;
    const long long pos = (long long)start - (start & 1) + slot;      // pairs of places begin at even ones
    Token t{(int)(pos - start), 0, 0};
    if (pos < start || t.i >= m) { t.i = -1; return t; }
    if (pos < 0 || pos >= (long long)r.c.max_pages * r.c.page_size) {
        if (r.status != nullptr) atomicOr(r.status, 32 /* LOT_DEV_PAGE */);
        t.i = -1;
        return t;
    }
    t.page = r.c.pages[(size_t)b * r.c.max_pages + (int)pos / r.c.page_size];
    t.at = (int)pos % r.c.page_size;
    if (t.page < 0 || t.page >= r.c.num_pages) {
        if (r.status != nullptr) atomicOr(r.status, 32);
        t.page = -1;
    }
    return t;
}

// The four lanes of a group hold 32-bit words of eight nibbles, nibble x of lane t for channel 8 t + x; back come the halves of g = 2 t
// (low) and 2 t + 1 (high), whose nibble i is the one of lane i.  Its own inverse up to the roles of the words.
__device__ __forceinline__ uint32_t across(uint32_t w, int t)
{
    uint32_t lo = 0, hi = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t y = __shfl_sync(0xffffffffu, w, i, 4) >> (8 * t);
        lo |= (y & 15u) << (4 * i);
        hi |= ((y >> 4) & 15u) << (4 * i);
    }
    return lo | (hi << 16);
}
// nibble x of lane t from the halves of across(): half g stands in lane g / 2
__device__ __forceinline__ uint32_t back(uint32_t h, int t)
{
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t y = __shfl_sync(0xffffffffu, h, i, 4) >> (4 * t);
        w |= ((y & 15u) | ((y >> 16) & 15u) << 4) << (8 * i);
    }
    return w;
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) write_kernel(const __grid_constant__ Rows r, const T *k, const T *v)
{
    constexpr int W = D / kGroup, LANES = D / 8;               // lanes of a token
    const int head = blockIdx.y, b = blockIdx.z >> 1, side = blockIdx.z & 1;
    const int slot = (int)((blockIdx.x * kThreads + threadIdx.x) / LANES), lane = threadIdx.x % LANES, w = lane >> 2, t = lane & 3;
    const Token tok = token_of(r, b, slot);
    const bool here = tok.i >= 0 && tok.page >= 0;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
    if (here) load8((side ? v : k) + (((size_t)b * r.c.Hkv + head) * r.m + tok.i) * D + lane * 8, x);
    float lo = x[0], hi = x[0];
    uint32_t big = __float_as_uint(x[0]) & 0x7fffffffu;
#pragma unroll
    for (int e = 1; e < 8; ++e) {
        lo = fminf(lo, x[e]);
        hi = fmaxf(hi, x[e]);
        big = max(big, __float_as_uint(x[e]) & 0x7fffffffu);
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        big = max(big, __shfl_xor_sync(0xffffffffu, big, o));
    }
    uint32_t param = 0x7fc07fc0u, codes = 0;                   // a value that is not finite: NaN for the group
    if (big < 0x7f800000u) {
        const uint32_t sb = scale_bits(lo, hi);
        const float s = __uint_as_float(sb << 16);
        const uint32_t zb = __float_as_uint(lo), zr = (zb + 0x7fffu + ((zb >> 16) & 1u)) & 0xffff0000u;
        const float z = __uint_as_float(zr);
        param = sb | zr;
        if (s > 0.f) {
            const float inv = __frcp_rn(s);
#pragma unroll
            for (int e = 0; e < 8; ++e) codes |= code_of(x[e], z, s, inv) << (4 * e);
        }
    }
    uint8_t *base = side_base(r.c, here ? tok.page : 0, head, side);
    if (here && t == 0) reinterpret_cast<uint32_t *>(base + (size_t)r.c.page_size * (D / 2))[(size_t)tok.at * W + w] = param;
    if (side == 0) {
        if (here) *reinterpret_cast<uint32_t *>(base + (size_t)tok.at * (D / 2) + (t * W + w) * 4) = codes;
        return;
    }
    const uint32_t halves = across(codes, t), other = __shfl_xor_sync(0xffffffffu, halves, LANES);       // the pair's token
    const int pair = __shfl_xor_sync(0xffffffffu, here ? 1 : 0, LANES);
    if (!here) return;
    const int odd = slot & 1;
    if (pair) {                                                // the even token's lanes store g = 2 t of both, the odd one's 2 t + 1
        const uint32_t word = odd ? (other >> 16) | (halves & 0xffff0000u) : (halves & 0xffffu) | (other << 16);
        *reinterpret_cast<uint32_t *>(base + value_half(tok.at & ~1, 2 * t + odd, w, W)) = word;
    } else {
        *reinterpret_cast<uint16_t *>(base + value_half(tok.at, 2 * t, w, W)) = (uint16_t)halves;
        *reinterpret_cast<uint16_t *>(base + value_half(tok.at, 2 * t + 1, w, W)) = (uint16_t)(halves >> 16);
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) read_kernel(const __grid_constant__ Rows r, T *k, T *v)
{
    constexpr int W = D / kGroup, LANES = D / 8;
    const int head = blockIdx.y, b = blockIdx.z >> 1, side = blockIdx.z & 1;
    const int slot = (int)((blockIdx.x * kThreads + threadIdx.x) / LANES), lane = threadIdx.x % LANES, w = lane >> 2, t = lane & 3;
    const int start = r.start[b], m = r.count != nullptr ? min(max(r.count[b], 0), r.m) : r.m;
    const int i = slot - (start & 1);
    const Token tok = token_of(r, b, slot);
    const bool here = tok.i >= 0 && tok.page >= 0;
    const uint8_t *base = side_base(r.c, here ? tok.page : 0, head, side);
    uint32_t param = 0, codes = 0;
    if (here) {
        param = __ldg(reinterpret_cast<const uint32_t *>(base + (size_t)r.c.page_size * (D / 2)) + (size_t)tok.at * W + w);
        if (side == 0) {
            codes = __ldg(reinterpret_cast<const uint32_t *>(base + (size_t)tok.at * (D / 2) + (t * W + w) * 4));
        } else {                                               // words of g = 2 t, 2 t + 1 hold both tokens of the pair
            const uint32_t p = __ldg(reinterpret_cast<const uint32_t *>(base + value_half(tok.at & ~1, 2 * t, w, W)));
            const uint32_t q = __ldg(reinterpret_cast<const uint32_t *>(base + value_half(tok.at & ~1, 2 * t + 1, w, W)));
            codes = (tok.at & 1) ? (p >> 16) | (q & 0xffff0000u) : (p & 0xffffu) | (q << 16);
        }
    }
    if (side == 1) codes = back(codes, t);
    if (i < 0 || i >= m) return;                               // a token whose page is missing reads as zeros
    const float s = param_scale(param), z = param_least(param);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = fmaf(s, (float)((codes >> (4 * e)) & 15u), z);
    store8((side ? v : k) + (((size_t)b * r.c.Hkv + head) * r.m + i) * D + lane * 8, x);
}

template <typename F> cudaError_t by_width(int dtype, int d, F f)
{
    if (dtype == 0) return d == 32 ? f(float{}, std::integral_constant<int, 32>{}) : d == 64 ? f(float{}, std::integral_constant<int, 64>{}) : f(float{}, std::integral_constant<int, 128>{});
    return d == 32 ? f(__nv_bfloat16{}, std::integral_constant<int, 32>{}) : d == 64 ? f(__nv_bfloat16{}, std::integral_constant<int, 64>{}) : f(__nv_bfloat16{}, std::integral_constant<int, 128>{});
}
dim3 grid_of(const Cache4 &c, int B, int m) { return dim3((unsigned)(((long long)m + 1) * (c.d / 8) + kThreads - 1) / kThreads, c.Hkv, 2 * B); }

} // namespace

cudaError_t launch_write4(const Cache4 &c, const void *k, const void *v, const int32_t *start, const int32_t *count, int dtype, int B, int m, int *status,
                          cudaStream_t st)
{
    return by_width(dtype, c.d, [&](auto t, auto width) {
        using T = decltype(t);
        write_kernel<T, decltype(width)::value><<<grid_of(c, B, m), kThreads, 0, st>>>(Rows{c, start, count, m, status}, static_cast<const T *>(k), static_cast<const T *>(v));
        return cudaGetLastError();
    });
}
cudaError_t launch_read4(const Cache4 &c, void *k, void *v, const int32_t *start, const int32_t *count, int dtype, int B, int m, int *status,
                         cudaStream_t st)
{
    return by_width(dtype, c.d, [&](auto t, auto width) {
        using T = decltype(t);
        read_kernel<T, decltype(width)::value><<<grid_of(c, B, m), kThreads, 0, st>>>(Rows{c, start, count, m, status}, static_cast<T *>(k), static_cast<T *>(v));
        return cudaGetLastError();
    });
}

} // namespace window
} // namespace lot
