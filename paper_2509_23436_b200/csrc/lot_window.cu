// Window attention with sinks of float32 tensors: forward and backward on warp-level tensor-core products.
//
// float32 accuracy from tf32 products: x = hi + lo, hi rounded to tf32's eleven bits, x y = hi hi + hi lo + lo hi up to 2^-22 (three products for one).  On
// float32 multiply-adds the same kernels took 62 us where these take 27 (32 sequences of 197 tokens, 3 heads of 64
// channels, windows of 32 keys on either side), and 311 where they take 116 (forward and backward of 2 x 1001 tokens, 8 heads of 32 channels, 255 keys back).  Three bf16 terms and six products of half the time
// each took 31 and 133: splitting an operand costs more than its products.
// A block takes 64 rows, a warp 16 of them with all columns, so that the softmax stays inside lane quads and weights become operands of the next
// product as they lie (a lane's two neighbouring columns are entries t and t + 4 of an operand whose columns are counted accordingly).
// Forward: 64 queries go over the 64-key tiles that any of them sees, first those of the sinks, then the window's, in one pass with the running
// maximum and sum.  Backward: P = exp(S - lse) again, D_i = <dout_i, out_i>, dS = P (dP - D): a block of 64 queries gathers dq over its keys, a
// block of 64 keys gathers dk and dv over the query heads and the queries that see them, so nothing is added by atomics.
#include "lot_window.cuh"

#include <mutex>

namespace lot {
int device_sm_count();
namespace window {
namespace {

constexpr int kT = 64, kThreads = 128, kN = 4, kPart = 8 * kN;       // columns are worked on in parts of kN pieces of 8; a part that none of a warp's rows sees is left out

// rows of a tile in shared memory: 8 numbers of padding, so that four rows' 32-byte pieces, and four rows' 8 neighbours, lie in different banks
template <int DP> struct Dim {
    static constexpr int LD = DP + 8, NT = DP / 8;             // NT: 8-channel pieces
};

// ROWS rows of x (from `first`, below n; channels below d) into s[ROWS][LD]; rows for which keep(row) fails become zeros
template <int DP, int ROWS = kT, typename F>
__device__ __forceinline__ void stage(float *s, const float *x, int first, int n, int d, F keep)
{
    for (int idx = threadIdx.x; idx < ROWS * (DP / 4); idx += kThreads) {
        const int r = idx / (DP / 4), c = (idx % (DP / 4)) * 4, row = first + r;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (row < n && c < d && keep(row)) v = __ldg(reinterpret_cast<const float4 *>(x + (size_t)row * d + c));
        *reinterpret_cast<float4 *>(s + r * Dim<DP>::LD + c) = v;
    }
}
struct All {
    __device__ __forceinline__ bool operator()(int) const { return true; }
};

__device__ __forceinline__ void halves(float x, uint32_t &hi, uint32_t &lo)
{
    hi = (__float_as_uint(x) + 0x1000u) & 0xffffe000u;
    lo = __float_as_uint(x - __uint_as_float(hi));
}
__device__ __forceinline__ void mma_tf32(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// d += a b of 16 x 8 and 8 x 8 numbers; a's entries (row g, k t), (row g + 8, k t), (row g, k t + 4), (row g + 8, k t + 4), b's (k t, n g), (k t + 4, n g)
struct Frag {
    uint32_t hi[4], lo[4];
    __device__ __forceinline__ Frag(float a0, float a1, float a2, float a3)
    {
        halves(a0, hi[0], lo[0]);
        halves(a1, hi[1], lo[1]);
        halves(a2, hi[2], lo[2]);
        halves(a3, hi[3], lo[3]);
    }
};
// d[n] += hi hi, e[n] += lo hi + hi lo of a b[n] for N independent sums: a term of all of them before the next, for a warp waits for a sum that it adds
// to again.  The instruction rounds its sums towards zero, so a sum is kept short, and apart from the small terms: into one long sum the error was 1.2e-6
// (windows of 65 keys) to 4.9e-6 (of 256, gradients) of the outputs' norm, now it is 3.5e-7 and 5e-7.
template <int N> __device__ __forceinline__ void mma3(float (*d)[4], float (*e)[4], const Frag &a, const float2 (&b)[N])
{
    uint32_t h[N][2], l[N][2];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        halves(b[n].x, h[n][0], l[n][0]);
        halves(b[n].y, h[n][1], l[n][1]);
    }
#pragma unroll
    for (int n = 0; n < N; ++n) mma_tf32(e[n], a.lo, h[n][0], h[n][1]);
#pragma unroll
    for (int n = 0; n < N; ++n) mma_tf32(d[n], a.hi, h[n][0], h[n][1]);
#pragma unroll
    for (int n = 0; n < N; ++n) mma_tf32(e[n], a.hi, l[n][0], l[n][1]);
}
template <int N> __device__ __forceinline__ void clear(float (&x)[N][4])
{
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[n][e] = 0.f;
}

// acc[n] (16 rows x 8) = <row of a, row 8 n + .. of b> for this warp's rows a[0 .. 15][LD] and 8 N rows of b; channels are taken in pairs
template <int DP, int N> __device__ __forceinline__ void scores(const float *a, const float *b, float (&acc)[N][4])
{
    constexpr int LD = Dim<DP>::LD;
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    float small[N][4];
    clear(acc);
    clear(small);
#pragma unroll 2
    for (int k = 0; k < DP; k += 8) {
        const float2 x = *reinterpret_cast<const float2 *>(a + g * LD + k + 2 * t), y = *reinterpret_cast<const float2 *>(a + (g + 8) * LD + k + 2 * t);
        float2 z[N];
#pragma unroll
        for (int n = 0; n < N; ++n) z[n] = *reinterpret_cast<const float2 *>(b + (8 * n + g) * LD + k + 2 * t);
        mma3<N>(acc, small, Frag(x.x, y.x, x.y, y.y), z);
    }
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[n][e] += small[n][e];
}
// o[c] (16 rows x 8 channels) += w x, w this warp's 16 x 8 N weights as scores() leaves them, x 8 N rows
template <int DP, int N> __device__ __forceinline__ void apply(const float (&w)[N][4], const float *x, float (&o)[Dim<DP>::NT][4])
{
    constexpr int LD = Dim<DP>::LD, C = 4;
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const float *p = x + 2 * t * LD + g;
#pragma unroll
    for (int c = 0; c < Dim<DP>::NT; c += C) {
        float sum[C][4], small[C][4];
        clear(sum);
        clear(small);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float2 z[C];
#pragma unroll
            for (int u = 0; u < C; ++u) z[u] = make_float2(p[8 * n * LD + 8 * (c + u)], p[(8 * n + 1) * LD + 8 * (c + u)]);
            mma3<C>(sum, small, Frag(w[n][0], w[n][2], w[n][1], w[n][3]), z);      // columns 2 t and 2 t + 1 as entries t and t + 4
        }
#pragma unroll
        for (int u = 0; u < C; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[c + u][e] += sum[u][e] + small[u][e];
    }
}
// one row of the sums: channels 8 c + 2 t, + 1
template <int DP> __device__ __forceinline__ void store_sums(float *row, int d, const float (&o)[Dim<DP>::NT][4], int lower, float f)
{
    const int t = threadIdx.x & 3;
#pragma unroll
    for (int c = 0; c < Dim<DP>::NT; ++c)
        if (8 * c < d) *reinterpret_cast<float2 *>(row + 8 * c + 2 * t) = make_float2(o[c][2 * lower] * f, o[c][2 * lower + 1] * f);
}

// Key tiles that queries at positions p0 .. p1 see: those of the sinks below the window's first, then the window's.
struct Tiles {
    int sink, first, last;                 // sink tiles 0 .. sink - 1, window tiles first .. last
    __device__ __forceinline__ int count() const { return sink + max(last - first + 1, 0); }
    __device__ __forceinline__ int at(int i) const { return i < sink ? i : first + i - sink; }
};
__device__ __forceinline__ Tiles tiles_of(const Row &R, int p0, int p1)
{
    Tiles t;
    const int hi = R.hi(p1);
    t.last = hi < 0 ? -1 : hi / kT;
    t.first = R.lo(p0) / kT;
    const int s = min(R.sinks, hi + 1);
    t.sink = min((s + kT - 1) / kT, t.first);
    if (t.sink < 0) t.sink = 0;
    return t;
}

// do queries at positions pa .. pb see any of the keys j .. j + kPart - 1
__device__ __forceinline__ bool touches(const Row &R, int pa, int pb, int j) { return j <= R.hi(pb) && (j + kPart - 1 >= pa - R.left || j < R.sinks); }

template <int DP>
__global__ void __launch_bounds__(kThreads) fwd_kernel(const __grid_constant__ Fwd a)
{
    extern __shared__ __align__(16) float sm[];
    constexpr int LD = Dim<DP>::LD, NT = Dim<DP>::NT;
    float *sQ = sm, *sK = sQ + kT * LD, *sV = sK + kT * LD;
    const int b = blockIdx.z, h = blockIdx.y, q0 = ((int)gridDim.x - 1 - (int)blockIdx.x) * kT, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int nq = a.band.nq, nk = a.band.nk, d = a.d;
    const Row R = row_of(a.band, b);
    const size_t qrow = ((size_t)b * a.H + h) * nq, krow = ((size_t)b * a.Hkv + h / (a.H / a.Hkv)) * nk;
    const float *k = static_cast<const float *>(a.k) + krow * d, *v = static_cast<const float *>(a.v) + krow * d;
    stage<DP>(sQ, static_cast<const float *>(a.q) + qrow * d, q0, nq, d, All{});
    const Tiles tiles = tiles_of(R, R.pos + q0, R.pos + min(q0 + kT, nq) - 1);
    const float c = a.scale * kLog2e;
    const int row[2] = {q0 + 16 * warp + g, q0 + 16 * warp + g + 8};
    float m[2] = {neg_inf(), neg_inf()}, l[2] = {0.f, 0.f}, o[NT][4];
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[u][e] = 0.f;
    for (int it = 0; it < tiles.count(); ++it) {
        const int j0 = tiles.at(it) * kT;
        __syncthreads();
        auto used = [&](int j) { return R.used(j); };
        stage<DP>(sK, k, j0, nk, d, used);
        stage<DP>(sV, v, j0, nk, d, used);
        __syncthreads();
        const int pa = R.pos + q0 + 16 * warp, pb = pa + 15;
#pragma unroll 1
        for (int n0 = 0; n0 < kT; n0 += kPart) {
            const int j = j0 + n0;
            if (q0 + 16 * warp >= nq || !touches(R, pa, pb, j)) continue;
            float s[kN][4];
            scores<DP, kN>(sQ + 16 * warp * LD, sK + n0 * LD, s);
            if (!(j + kPart - 1 <= R.hi(pa) && j >= pb - R.left)) {
#pragma unroll
                for (int n = 0; n < kN; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (!R.sees(R.pos + row[e >> 1], j + 8 * n + 2 * t + (e & 1))) s[n][e] = neg_inf();
            }
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float top = neg_inf();
#pragma unroll
                for (int n = 0; n < kN; ++n) top = fmaxf(top, fmaxf(s[n][2 * r], s[n][2 * r + 1]));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(m[r], c * fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2)));
                const float ref = top == neg_inf() ? 0.f : top, old = ex2(m[r] - ref);       // nothing visible so far: 0
                m[r] = top;
                float sum = 0.f;
#pragma unroll
                for (int n = 0; n < kN; ++n) {
                    s[n][2 * r] = ex2(fmaf(s[n][2 * r], c, -ref));
                    s[n][2 * r + 1] = ex2(fmaf(s[n][2 * r + 1], c, -ref));
                    sum += s[n][2 * r] + s[n][2 * r + 1];
                }
                l[r] = l[r] * old + sum;
#pragma unroll
                for (int u = 0; u < NT; ++u) { o[u][2 * r] *= old; o[u][2 * r + 1] *= old; }
            }
            apply<DP, kN>(s, sV + n0 * LD, o);
        }
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
        if (row[r] >= nq) continue;
        store_sums<DP>(static_cast<float *>(a.out) + (qrow + row[r]) * d, d, o, r, l[r] > 0.f ? 1.f / l[r] : 0.f);
        if (a.lse != nullptr && t == 0) a.lse[qrow + row[r]] = l[r] > 0.f ? m[r] * kLn2 + logf(l[r]) : neg_inf();
    }
}

// ---- few queries: sixteen rows of a key head (its query heads times the queries, which lie in a row) a block, which goes over a part of the key tiles;
// a warp takes sixteen keys of each.  The warps join in shared memory, the blocks of a row tile in few_join_kernel.  8 x 16 heads on 4, 8192 keys of 128
// channels, one query: 142 us, 1.9 TB/s (a block waits for its tile, then works on it; two blocks an SM overlap). ----
constexpr int kFewRows = 16, kFewKeys = kT / (kThreads / 32);

struct Few {
    Fwd a;
    int G, splits, each;                   // key tiles of a split
    float *part;                           // splits > 1: [B Hkv][row tile][split][kFewRows][DP + 2]
};

template <int DP>
__global__ void __launch_bounds__(kThreads) few_kernel(const __grid_constant__ Few f)
{
    extern __shared__ __align__(16) float sm[];
    constexpr int LD = Dim<DP>::LD, NT = Dim<DP>::NT, N = kFewKeys / 8, OWN = kFewRows * DP + 2 * kFewRows;
    static_assert(4 * OWN <= 2 * kT * LD, "the warps' sums take the tiles' place");
    const Fwd &a = f.a;
    float *sQ = sm, *sK = sQ + kFewRows * LD, *sV = sK + kT * LD;
    const int split = blockIdx.x % f.splits, r0 = blockIdx.x / f.splits * kFewRows, hk = blockIdx.y, b = blockIdx.z;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3, nq = a.band.nq, nk = a.band.nk, d = a.d, rows = f.G * nq;
    const Row R = row_of(a.band, b);
    const size_t qrow = ((size_t)b * a.H + (size_t)hk * f.G) * nq, krow = ((size_t)b * a.Hkv + hk) * nk;
    const float *k = static_cast<const float *>(a.k) + krow * d, *v = static_cast<const float *>(a.v) + krow * d;
    stage<DP, kFewRows>(sQ, static_cast<const float *>(a.q) + qrow * d, r0, rows, d, All{});
    const int p0 = R.pos, p1 = R.pos + nq - 1, pos[2] = {p0 + min(r0 + g, rows - 1) % nq, p0 + min(r0 + g + 8, rows - 1) % nq};
    const Tiles tiles = tiles_of(R, p0, p1);
    const int to = min(tiles.count(), (split + 1) * f.each);
    const float c = a.scale * kLog2e;
    float m[2] = {neg_inf(), neg_inf()}, l[2] = {0.f, 0.f}, o[NT][4];
    clear(o);
    for (int it = split * f.each; it < to; ++it) {
        const int j0 = tiles.at(it) * kT, j = j0 + kFewKeys * warp;
        __syncthreads();
        auto used = [&](int i) { return R.used(i); };
        stage<DP>(sK, k, j0, nk, d, used);
        stage<DP>(sV, v, j0, nk, d, used);
        __syncthreads();
        if (j > R.hi(p1) || (j + kFewKeys - 1 < p0 - R.left && j >= R.sinks)) continue;
        float s[N][4];
        scores<DP, N>(sQ, sK + kFewKeys * warp * LD, s);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float top = neg_inf();
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int e = 2 * r; e < 2 * r + 2; ++e) {
                    if (!R.sees(pos[r], j + 8 * n + 2 * t + (e & 1))) s[n][e] = neg_inf();
                    top = fmaxf(top, s[n][e]);
                }
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(m[r], c * fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2)));
            const float ref = top == neg_inf() ? 0.f : top, old = ex2(m[r] - ref);
            m[r] = top;
            float sum = 0.f;
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int e = 2 * r; e < 2 * r + 2; ++e) {
                    s[n][e] = ex2(fmaf(s[n][e], c, -ref));
                    sum += s[n][e];
                }
            l[r] = l[r] * old + sum;
#pragma unroll
            for (int u = 0; u < NT; ++u) { o[u][2 * r] *= old; o[u][2 * r + 1] *= old; }
        }
        apply<DP, N>(s, sV + kFewKeys * warp * LD, o);
    }
    __syncthreads();                                       // every warp has left the tiles
    float *own = sK + warp * OWN;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
        store_sums<DP>(own + (g + 8 * r) * DP, DP, o, r, 1.f);
        if (t == 0) { own[kFewRows * DP + g + 8 * r] = m[r]; own[kFewRows * DP + kFewRows + g + 8 * r] = l[r]; }
    }
    __syncthreads();
    for (int idx = threadIdx.x; idx < kFewRows * DP; idx += kThreads) {
        const int r = idx / DP, col = idx % DP;
        if (r0 + r >= rows) break;
        float top = neg_inf(), sum = 0.f, x = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, sK[w * OWN + kFewRows * DP + r]);
        const float at = top == neg_inf() ? 0.f : top;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float e = ex2(sK[w * OWN + kFewRows * DP + r] - at);
            sum += e * sK[w * OWN + kFewRows * DP + kFewRows + r];
            x += e * sK[w * OWN + idx];
        }
        if (f.splits > 1) {
            float *p = f.part + ((((size_t)b * a.Hkv + hk) * (gridDim.x / f.splits) + blockIdx.x / f.splits) * f.splits + split) * (kFewRows * (DP + 2)) + r * (DP + 2);
            p[col] = x;
            if (col == 0) { p[DP] = top; p[DP + 1] = sum; }
            continue;
        }
        if (col < d) static_cast<float *>(a.out)[(qrow + r0 + r) * d + col] = sum > 0.f ? x / sum : 0.f;
        if (col == 0 && a.lse != nullptr) a.lse[qrow + r0 + r] = sum > 0.f ? top * kLn2 + logf(sum) : neg_inf();
    }
}
// a block joins the splits of one row, a thread a channel
template <int DP>
__global__ void __launch_bounds__(DP) few_join_kernel(const __grid_constant__ Few f)
{
    const Fwd &a = f.a;
    const int r = blockIdx.x, hk = blockIdx.y, b = blockIdx.z, col = threadIdx.x, rows = f.G * a.band.nq;
    constexpr size_t STEP = kFewRows * (DP + 2);
    const float *p = f.part + (((size_t)b * a.Hkv + hk) * ((rows + kFewRows - 1) / kFewRows) + r / kFewRows) * f.splits * STEP + r % kFewRows * (DP + 2);
    float top = neg_inf(), sum = 0.f, x = 0.f;
    for (int i = 0; i < f.splits; ++i) top = fmaxf(top, p[i * STEP + DP]);
    const float at = top == neg_inf() ? 0.f : top;
    for (int i = 0; i < f.splits; ++i) {
        const float e = ex2(p[i * STEP + DP] - at);
        sum += e * p[i * STEP + DP + 1];
        x += e * p[i * STEP + col];
    }
    const size_t row = ((size_t)b * a.H + (size_t)hk * f.G) * a.band.nq + r;
    if (col < a.d) static_cast<float *>(a.out)[row * a.d + col] = sum > 0.f ? x / sum : 0.f;
    if (col == 0 && a.lse != nullptr) a.lse[row] = sum > 0.f ? top * kLn2 + logf(sum) : neg_inf();
}
// two waves of blocks, of two tiles at least
Few few_of(const Fwd &a)
{
    Few f{a, a.H / a.Hkv, 1, 1, static_cast<float *>(a.ws)};
    const Band &n = a.band;
    const long long tiles = (f.G * n.nq + kFewRows - 1) / kFewRows, blocks = tiles * a.B * a.Hkv, slots = (a.d <= 64 ? 8ll : 4ll) * device_sm_count();
    const long long run = (long long)(n.left < n.nk ? n.left : n.nk) + (n.right < n.nk ? n.right : n.nk) + n.nq, all = (n.nk + kT - 1) / kT;
    const long long touched = (run + 2 * (kT - 1)) / kT + (n.sinks + kT - 1) / kT, len = touched < all ? touched : all, parts = slots / blocks > 1 ? slots / blocks : 1;
    const long long each = (len + parts - 1) / parts;
    f.each = (int)(each > 2 ? each : 2);
    f.splits = len > f.each ? (int)((len + f.each - 1) / f.each) : 1;
    return f;
}

// delta = <dout, out> of every row: a warp each
__global__ void __launch_bounds__(256) delta_kernel(const float *out, const float *dout, float *delta, long long rows, int d)
{
    const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (row >= rows) return;
    const int c = (threadIdx.x & 31) * 4;
    float s = 0.f;
    if (c < d) {
        float x[4], y[4];
        load4(out + row * d + c, x);
        load4(dout + row * d + c, y);
        s = x[0] * y[0] + x[1] * y[1] + (x[2] * y[2] + x[3] * y[3]);
    }
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) s += __shfl_xor_sync(0xffffffffu, s, w);
    if ((threadIdx.x & 31) == 0) delta[row] = s;
}

template <int DP>
__global__ void __launch_bounds__(kThreads) dq_kernel(const __grid_constant__ Bwd a)
{
    extern __shared__ __align__(16) float sm[];
    constexpr int LD = Dim<DP>::LD, NT = Dim<DP>::NT;
    float *sQ = sm, *sO = sQ + kT * LD, *sK = sO + kT * LD, *sV = sK + kT * LD;
    const int b = blockIdx.z, h = blockIdx.y, q0 = ((int)gridDim.x - 1 - (int)blockIdx.x) * kT, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int nq = a.band.nq, nk = a.band.nk, d = a.d;
    const Row R = row_of(a.band, b);
    const size_t qrow = ((size_t)b * a.H + h) * nq, krow = ((size_t)b * a.Hkv + h / (a.H / a.Hkv)) * nk;
    const float *k = static_cast<const float *>(a.k) + krow * d, *v = static_cast<const float *>(a.v) + krow * d;
    stage<DP>(sQ, static_cast<const float *>(a.q) + qrow * d, q0, nq, d, All{});
    stage<DP>(sO, static_cast<const float *>(a.dout) + qrow * d, q0, nq, d, All{});
    const Tiles tiles = tiles_of(R, R.pos + q0, R.pos + min(q0 + kT, nq) - 1);
    const float c = a.scale * kLog2e;
    const int row[2] = {q0 + 16 * warp + g, q0 + 16 * warp + g + 8};
    float lse2[2], dl[2], o[NT][4];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        lse2[r] = a.lse[qrow + min(row[r], nq - 1)] * kLog2e;
        dl[r] = a.delta[qrow + min(row[r], nq - 1)];
    }
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[u][e] = 0.f;
    for (int it = 0; it < tiles.count(); ++it) {
        const int j0 = tiles.at(it) * kT;
        __syncthreads();
        auto used = [&](int j) { return R.used(j); };
        stage<DP>(sK, k, j0, nk, d, used);
        stage<DP>(sV, v, j0, nk, d, used);
        __syncthreads();
#pragma unroll 1
        for (int n0 = 0; n0 < kT; n0 += kPart) {
            if (!touches(R, R.pos + q0 + 16 * warp, R.pos + q0 + 16 * warp + 15, j0 + n0)) continue;
            float s[kN][4], dp[kN][4];
            scores<DP, kN>(sQ + 16 * warp * LD, sK + n0 * LD, s);
            scores<DP, kN>(sO + 16 * warp * LD, sV + n0 * LD, dp);
#pragma unroll
            for (int n = 0; n < kN; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool seen = R.sees(R.pos + row[e >> 1], j0 + n0 + 8 * n + 2 * t + (e & 1));
                    s[n][e] = seen ? ex2(fmaf(s[n][e], c, -lse2[e >> 1])) * (dp[n][e] - dl[e >> 1]) : 0.f;
                }
            apply<DP, kN>(s, sK + n0 * LD, o);
        }
    }
#pragma unroll
    for (int r = 0; r < 2; ++r)
        if (row[r] < nq) store_sums<DP>(static_cast<float *>(a.dq) + (qrow + row[r]) * d, d, o, r, a.scale);
}

size_t delta_bytes(int B, int H, int nq) { return ((size_t)B * H * nq * 4 + 255) & ~(size_t)255; }

// How key tiles are cut: a tile's list (the query tiles of all its query heads that see it) in parts of at most `most` tiles, whose sums merge_kernel adds
// in order.  Parts of the tiles with sinks (every later query sees them) first, then the others'.
struct Cut {
    int tiles, sink_tiles, sink_parts, key_parts;
    __host__ __device__ int works(int sinks) const { return sinks ? sink_tiles * sink_parts : (tiles - sink_tiles) * key_parts; }
    __host__ __device__ int all() const { return works(1) + works(0); }
    __host__ __device__ bool whole() const { return (sink_tiles == 0 || sink_parts == 1) && (tiles == sink_tiles || key_parts == 1); }
};
Cut cut_of(int B, int H, int Hkv, int nq, int nk, int left, int right, int sinks)
{
    Cut c;
    c.tiles = (nk + kT - 1) / kT;
    c.sink_tiles = ((sinks < nk ? sinks : nk) + kT - 1) / kT;
    const long long qtiles = (nq + kT - 1) / kT, span = ((long long)left + right + kT - 1) / kT + 2, G = H / Hkv;
    const long long sink_len = G * qtiles, key_len = G * (span < qtiles ? span : qtiles), heads = (long long)B * Hkv;
    // three blocks an SM: no part longer than a third of a block's share, nor of more than four tiles where that leaves enough of them
    const long long share = heads * (c.sink_tiles * sink_len + (c.tiles - c.sink_tiles) * key_len) / (9ll * device_sm_count()), most = share > 4 ? share : 4;
    c.sink_parts = (int)((sink_len + most - 1) / most);
    c.key_parts = (int)((key_len + most - 1) / most);
    if (c.sink_parts < 1) c.sink_parts = 1;
    if (c.key_parts < 1) c.key_parts = 1;
    return c;
}
struct BwdCut {
    Bwd a;
    Cut cut;
    float *part;                           // [B Hkv][part][dk, dv][64][DP], or nullptr: every tile whole
};
size_t part_floats(const Cut &c, int B, int Hkv, int DP) { return c.whole() ? 0 : (size_t)B * Hkv * c.all() * 2 * kT * DP; }

template <int DP>
__global__ void __launch_bounds__(kThreads) dkv_kernel(const __grid_constant__ BwdCut c)
{
    extern __shared__ __align__(16) float sm[];
    constexpr int LD = Dim<DP>::LD, NT = Dim<DP>::NT;
    const Bwd &a = c.a;
    float *sQ = sm, *sO = sQ + kT * LD, *sK = sO + kT * LD, *sV = sK + kT * LD, *sL = sV + kT * LD;
    const int b = blockIdx.z, hk = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3, G = a.H / a.Hkv;
    const bool has_sinks = (int)blockIdx.x < c.cut.works(1);
    const int work = blockIdx.x - (has_sinks ? 0 : c.cut.works(1)), parts = has_sinks ? c.cut.sink_parts : c.cut.key_parts, part = work % parts;
    const int j0 = (work / parts + (has_sinks ? 0 : c.cut.sink_tiles)) * kT;
    const int nq = a.band.nq, nk = a.band.nk, d = a.d;
    const Row R = row_of(a.band, b);
    const size_t krow = ((size_t)b * a.Hkv + hk) * nk;
    auto used = [&](int j) { return R.used(j); };
    stage<DP>(sK, static_cast<const float *>(a.k) + krow * d, j0, nk, d, used);
    stage<DP>(sV, static_cast<const float *>(a.v) + krow * d, j0, nk, d, used);
    // queries that see a key of the tile: positions j0 - right .. j0 + 63 + left, all later ones if the tile holds a sink
    const int i0 = max(j0 - R.right - R.pos, 0), i1 = j0 < R.sinks ? nq - 1 : (int)min((long long)nq - 1, (long long)j0 + kT - 1 + R.left - R.pos);
    const float sc = a.scale * kLog2e;
    const int row[2] = {j0 + 16 * warp + g, j0 + 16 * warp + g + 8};
    float dk[NT][4], dv[NT][4];
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) dk[u][e] = dv[u][e] = 0.f;
    const int first = i0 / kT, per = j0 < R.len && i1 >= i0 ? i1 / kT - first + 1 : 0;
    const int from = (int)((long long)per * G * part / parts), to = (int)((long long)per * G * (part + 1) / parts);
    for (int u = from; u < to; ++u) {
        const size_t qrow = ((size_t)b * a.H + hk * G + u / per) * nq;
        const int q0 = (first + u % per) * kT;
        __syncthreads();
        stage<DP>(sQ, static_cast<const float *>(a.q) + qrow * d, q0, nq, d, All{});
        stage<DP>(sO, static_cast<const float *>(a.dout) + qrow * d, q0, nq, d, All{});
        if (threadIdx.x < kT) {
            const int i = min(q0 + (int)threadIdx.x, nq - 1);
            sL[threadIdx.x] = a.lse[qrow + i] * kLog2e;
            sL[kT + threadIdx.x] = a.delta[qrow + i];
        }
        __syncthreads();
#pragma unroll 1
        for (int n0 = 0; n0 < kT; n0 += kPart) {
            // do the queries q0 + n0 .. + kPart - 1 see any of the warp's keys
            const int pa = R.pos + q0 + n0, ja = j0 + 16 * warp;
            if (ja > R.hi(pa + kPart - 1) || (ja + 15 < pa - R.left && ja >= R.sinks)) continue;
            float s[kN][4], dp[kN][4];
            scores<DP, kN>(sK + 16 * warp * LD, sQ + n0 * LD, s);
            scores<DP, kN>(sV + 16 * warp * LD, sO + n0 * LD, dp);
#pragma unroll
            for (int n = 0; n < kN; ++n) {
                const int col = n0 + 8 * n + 2 * t;
                const float2 ls = *reinterpret_cast<const float2 *>(sL + col), dl = *reinterpret_cast<const float2 *>(sL + kT + col);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = q0 + col + (e & 1);
                    const bool seen = i < nq && R.sees(R.pos + i, row[e >> 1]);
                    s[n][e] = seen ? ex2(fmaf(s[n][e], sc, -(e & 1 ? ls.y : ls.x))) : 0.f;
                    dp[n][e] = seen ? s[n][e] * (dp[n][e] - (e & 1 ? dl.y : dl.x)) : 0.f;
                }
            }
            apply<DP, kN>(s, sO + n0 * LD, dv);
            apply<DP, kN>(dp, sQ + n0 * LD, dk);
        }
    }
    if (c.part != nullptr) {
        float *o = c.part + (((size_t)b * a.Hkv + hk) * c.cut.all() + blockIdx.x) * (2 * kT * DP);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            store_sums<DP>(o + (16 * warp + g + 8 * r) * DP, DP, dk, r, a.scale);
            store_sums<DP>(o + (kT + 16 * warp + g + 8 * r) * DP, DP, dv, r, 1.f);
        }
        return;
    }
#pragma unroll
    for (int r = 0; r < 2; ++r)
        if (row[r] < nk) {
            store_sums<DP>(static_cast<float *>(a.dk) + (krow + row[r]) * d, d, dk, r, a.scale);
            store_sums<DP>(static_cast<float *>(a.dv) + (krow + row[r]) * d, d, dv, r, 1.f);
        }
}

// dk (side 0) and dv of a key tile from its parts, in order
template <int DP>
__global__ void __launch_bounds__(kThreads) merge_kernel(const __grid_constant__ BwdCut c)
{
    const Bwd &a = c.a;
    const int tile = blockIdx.x >> 1, side = blockIdx.x & 1, hk = blockIdx.y, b = blockIdx.z, d = a.d;
    const bool has_sinks = tile < c.cut.sink_tiles;
    const int parts = has_sinks ? c.cut.sink_parts : c.cut.key_parts, first = has_sinks ? tile * parts : c.cut.works(1) + (tile - c.cut.sink_tiles) * parts;
    const float *p = c.part + (((size_t)b * a.Hkv + hk) * c.cut.all() + first) * (2 * kT * DP) + side * (kT * DP);
    float *out = static_cast<float *>(side ? a.dv : a.dk) + ((size_t)b * a.Hkv + hk) * a.band.nk * d;
    for (int idx = threadIdx.x; idx < kT * (DP / 4); idx += kThreads) {
        const int r = idx / (DP / 4), ch = idx % (DP / 4) * 4, row = tile * kT + r;
        if (row >= a.band.nk || ch >= d) continue;
        float o[4] = {0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < parts; ++k) {
            const float4 x = *reinterpret_cast<const float4 *>(p + (size_t)k * (2 * kT * DP) + r * DP + ch);
            o[0] += x.x; o[1] += x.y; o[2] += x.z; o[3] += x.w;
        }
        store4(out + (size_t)row * d + ch, o);
    }
}

// Dynamic shared memory above 48 KB is asked for once per kernel and device.
template <auto KERN> cudaError_t allow_smem(int bytes)
{
    static std::mutex mu;
    static bool set[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(mu);
    if (!set[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(KERN, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != cudaSuccess) return e;
        set[dev] = true;
    }
    return cudaSuccess;
}
template <auto KERN, typename A> cudaError_t launch(const A &a, dim3 grid, int bytes, cudaStream_t st)
{
    const cudaError_t e = allow_smem<KERN>(bytes);
    if (e != cudaSuccess) return e;
    KERN<<<grid, kThreads, bytes, st>>>(a);
    return cudaGetLastError();
}

// Few queries: up to 32, and up to 64 of few heads.  A block of fwd_kernel would leave rows empty, not share a key head's keys, and go over all of its keys
// by itself.  32 heads on 4 key heads of 128 channels, 16384 keys: one query 45 us against 2540, 32 380 against 2610, 64 790 against 2400; 8 x 16 heads on
// 4, 8192 keys: 33 queries 967 against 1620.
bool few_f32(int B, int H, int nq) { return nq <= 32 || (nq <= 64 && (long long)B * H * nq <= 32ll * device_sm_count()); }

template <int DP> cudaError_t fwd_t(const Fwd &a, cudaStream_t st)
{
    if (few_f32(a.B, a.H, a.band.nq)) {
        const Few f = few_of(a);
        const cudaError_t e = launch<few_kernel<DP>>(f, dim3((f.G * a.band.nq + kFewRows - 1) / kFewRows * f.splits, a.Hkv, a.B), (kFewRows + 2 * kT) * Dim<DP>::LD * 4, st);
        if (e != cudaSuccess || f.splits == 1) return e;
        few_join_kernel<DP><<<dim3(f.G * a.band.nq, a.Hkv, a.B), DP, 0, st>>>(f);
        return cudaGetLastError();
    }
    return launch<fwd_kernel<DP>>(a, dim3((a.band.nq + kT - 1) / kT, a.H, a.B), 3 * kT * Dim<DP>::LD * 4, st);
}
template <int DP> cudaError_t bwd_t(const Bwd &a, cudaStream_t st)
{
    const long long rows = (long long)a.B * a.H * a.band.nq;
    if (rows > 0) {
        delta_kernel<<<(unsigned)((rows + 7) / 8), 256, 0, st>>>(static_cast<const float *>(a.out), static_cast<const float *>(a.dout), a.delta, rows, a.d);
        cudaError_t e = cudaGetLastError();
        if (e == cudaSuccess) e = launch<dq_kernel<DP>>(a, dim3((a.band.nq + kT - 1) / kT, a.H, a.B), 4 * kT * Dim<DP>::LD * 4, st);
        if (e != cudaSuccess) return e;
    }
    if (a.band.nk == 0) return cudaSuccess;
    BwdCut c{a, cut_of(a.B, a.H, a.Hkv, a.band.nq, a.band.nk, a.band.left, a.band.right, a.band.sinks), nullptr};
    if (!c.cut.whole()) c.part = reinterpret_cast<float *>(reinterpret_cast<char *>(a.delta) + delta_bytes(a.B, a.H, a.band.nq));
    cudaError_t e = launch<dkv_kernel<DP>>(c, dim3(c.cut.all(), a.Hkv, a.B), (4 * kT * Dim<DP>::LD + 2 * kT) * 4, st);
    if (e != cudaSuccess || c.part == nullptr) return e;
    return launch<merge_kernel<DP>>(c, dim3(2 * c.cut.tiles, a.Hkv, a.B), 0, st);
}

} // namespace

cudaError_t launch_fwd(const Fwd &a, cudaStream_t st)
{
    if (a.dtype == 0) return a.d <= 32 ? fwd_t<32>(a, st) : a.d <= 64 ? fwd_t<64>(a, st) : fwd_t<128>(a, st);
    return few_supported(a.B, a.H, a.Hkv, a.band.nq, a.band.nk) ? launch_few(a, st) : launch_fwd_tc(a, st);
}
size_t fwd_workspace(int dtype, int B, int H, int Hkv, const Band &band, int d)
{
    if (dtype != 0) return few_supported(B, H, Hkv, band.nq, band.nk) ? few_workspace(B, H, Hkv, band, d) : 0;
    if (!few_f32(B, H, band.nq)) return 0;
    Fwd a{};
    a.band = band;
    a.B = B; a.H = H; a.Hkv = Hkv; a.d = d;
    const Few f = few_of(a);
    const size_t rows = (f.G * band.nq + kFewRows - 1) / kFewRows * kFewRows, DP = d <= 32 ? 32 : d <= 64 ? 64 : 128;
    return f.splits == 1 ? 0 : ((size_t)B * Hkv * rows * f.splits * (DP + 2) * 4 + 255) & ~(size_t)255;
}
size_t bwd_f32_workspace(int B, int H, int Hkv, int nq, int nk, int d, int left, int right, int sinks)
{
    const Cut c = cut_of(B, H, Hkv, nq, nk, left, right, sinks);
    return delta_bytes(B, H, nq) + ((part_floats(c, B, Hkv, d <= 32 ? 32 : d <= 64 ? 64 : 128) * 4 + 255) & ~(size_t)255);
}

cudaError_t launch_bwd(const Bwd &a, cudaStream_t st)
{
    if (a.dtype == 0) return a.d <= 32 ? bwd_t<32>(a, st) : a.d <= 64 ? bwd_t<64>(a, st) : bwd_t<128>(a, st);
    return launch_bwd_tc(a, st);
}

} // namespace window
} // namespace lot
