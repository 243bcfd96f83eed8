// Window attention with sinks on float32 multiply-adds: forward and backward of float32 tensors.
//
// Forward: a block takes 64 queries of a head and goes over the 64-key tiles that any of them sees, first those of the sinks, then the
// window's, in one pass with the running maximum and sum of the softmax.  Backward: P = exp(S - lse) again, D_i = <dout_i, out_i>,
// dS = P (dP - D): a block of 64 queries gathers dq over its keys, a block of 64 keys gathers dk and dv over the query heads and the
// queries that see them, so nothing is added by atomics.
// A thread holds 4 x 4 scores (rows in sixteen-lane groups) and 4 rows of d / 16 channels of the sums.
#include "lot_window.cuh"

#include <mutex>

namespace lot {
int device_sm_count();
namespace window {
namespace {

constexpr int kT = 64, kThreads = 256;

template <int DP> struct Dim {
    static constexpr int LD = DP + 4, NC = DP / 16;            // padded row of a tile; channels a thread sums
};

// 64 rows of x (rows first .. first + 63 below n, channels below d) into s[64][LD]; rows for which keep(row) fails become zeros
template <int DP, typename T, typename F>
__device__ __forceinline__ void stage(float *s, const T *x, int first, int n, int d, F keep)
{
    for (int idx = threadIdx.x; idx < kT * (DP / 4); idx += kThreads) {
        const int r = idx / (DP / 4), c = (idx % (DP / 4)) * 4, row = first + r;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        if (row < n && c < d && keep(row)) load4(x + (size_t)row * d + c, v);
        *reinterpret_cast<float4 *>(s + r * Dim<DP>::LD + c) = make_float4(v[0], v[1], v[2], v[3]);
    }
}
struct All {
    __device__ __forceinline__ bool operator()(int) const { return true; }
};

// acc[i][j] = <a row 4 ty + i, b row tx + 16 j>
template <int DP> __device__ __forceinline__ void scores(const float *a, const float *b, int ty, int tx, float (&acc)[4][4])
{
    constexpr int LD = Dim<DP>::LD;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
#pragma unroll 4
    for (int k = 0; k < DP; k += 4) {
        float4 x[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const float4 *>(a + (4 * ty + i) * LD + k);
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const float4 *>(b + (tx + 16 * j) * LD + k);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                acc[i][j] = fmaf(x[i].w, y[j].w, fmaf(x[i].z, y[j].z, fmaf(x[i].y, y[j].y, fmaf(x[i].x, y[j].x, acc[i][j]))));
    }
}

// channel u of a thread's sums: 4 neighbours of every 64, or DP / 16 neighbours below that
template <int DP> __device__ __forceinline__ int channel(int tx, int u) { return DP >= 64 ? (u >> 2) * 64 + tx * 4 + (u & 3) : tx * Dim<DP>::NC + u; }

// o[i][u] += sum_k w[4 ty + i][k] x[k][channel u], w with rows of kT + 4
template <int DP> __device__ __forceinline__ void apply(const float *w, const float *x, int ty, int tx, float (&o)[4][Dim<DP>::NC])
{
    constexpr int LD = Dim<DP>::LD, NC = Dim<DP>::NC;
#pragma unroll 2
    for (int k = 0; k < kT; k += 4) {
        float p[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 t = *reinterpret_cast<const float4 *>(w + (4 * ty + i) * (kT + 4) + k);
            p[i][0] = t.x; p[i][1] = t.y; p[i][2] = t.z; p[i][3] = t.w;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float y[NC];
#pragma unroll
            for (int u = 0; u < NC; ++u) y[u] = x[(k + e) * LD + channel<DP>(tx, u)];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int u = 0; u < NC; ++u) o[i][u] = fmaf(p[i][e], y[u], o[i][u]);
        }
    }
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

template <typename T, int DP>
__global__ void __launch_bounds__(kThreads) fwd_kernel(const __grid_constant__ Fwd a)
{
    extern __shared__ __align__(16) float sm[];
    constexpr int LD = Dim<DP>::LD, NC = Dim<DP>::NC;
    float *sQ = sm, *sK = sQ + kT * LD, *sV = sK + kT * LD, *sP = sV + kT * LD;
    const int b = blockIdx.z, h = blockIdx.y, q0 = ((int)gridDim.x - 1 - (int)blockIdx.x) * kT, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int nq = a.band.nq, nk = a.band.nk, d = a.d;
    const Row R = row_of(a.band, b);
    const size_t qrow = ((size_t)b * a.H + h) * nq, krow = ((size_t)b * a.Hkv + h / (a.H / a.Hkv)) * nk;
    const T *k = static_cast<const T *>(a.k) + krow * d, *v = static_cast<const T *>(a.v) + krow * d;
    stage<DP>(sQ, static_cast<const T *>(a.q) + qrow * d, q0, nq, d, All{});
    const Tiles t = tiles_of(R, R.pos + q0, R.pos + min(q0 + kT, nq) - 1);
    const float c = a.scale * kLog2e;
    float m[4], l[4], o[4][NC];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = neg_inf(); l[i] = 0.f;
#pragma unroll
        for (int u = 0; u < NC; ++u) o[i][u] = 0.f;
    }
    for (int it = 0; it < t.count(); ++it) {
        const int j0 = t.at(it) * kT;
        __syncthreads();
        auto used = [&](int j) { return R.used(j); };
        stage<DP>(sK, k, j0, nk, d, used);
        stage<DP>(sV, v, j0, nk, d, used);
        __syncthreads();
        float s[4][4];
        scores<DP>(sQ, sK, ty, tx, s);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = R.pos + q0 + 4 * ty + i;
            float top = neg_inf();
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[i][j] = R.sees(p, j0 + tx + 16 * j) ? s[i][j] * c : neg_inf();
                top = fmaxf(top, s[i][j]);
            }
#pragma unroll
            for (int w = 1; w < 16; w <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
            top = fmaxf(top, m[i]);
            const float ref = top == neg_inf() ? 0.f : top, old = ex2(m[i] - ref);       // nothing visible so far: 0
            m[i] = top;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[i][j] = ex2(s[i][j] - ref);
                sum += s[i][j];
                sP[(4 * ty + i) * (kT + 4) + tx + 16 * j] = s[i][j];
            }
#pragma unroll
            for (int w = 1; w < 16; w <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
            l[i] = l[i] * old + sum;
#pragma unroll
            for (int u = 0; u < NC; ++u) o[i][u] *= old;
        }
        __syncwarp();                      // a row's weights are written and read by one half warp
        apply<DP>(sP, sV, ty, tx, o);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = q0 + 4 * ty + i;
        if (row >= nq) break;
        const float inv = l[i] > 0.f ? 1.f / l[i] : 0.f;
        T *out = static_cast<T *>(a.out) + (qrow + row) * d;
#pragma unroll
        for (int u = 0; u < NC; ++u)
            if (channel<DP>(tx, u) < d) Elem<T>::store(out + channel<DP>(tx, u), o[i][u] * inv);
        if (a.lse != nullptr && tx == 0) a.lse[qrow + row] = l[i] > 0.f ? m[i] * kLn2 + logf(l[i]) : neg_inf();
    }
}

// delta = <dout, out> of every row: a warp each
template <typename T>
__global__ void __launch_bounds__(256) delta_kernel(const T *out, const T *dout, float *delta, long long rows, int d)
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

// P and dS of one query and key; both zero where the query does not see the key
__device__ __forceinline__ void weights(bool seen, float s, float dp, float c, float scale, float lse2, float delta, float &p, float &ds)
{
    p = seen ? ex2(fmaf(s, c, -lse2)) : 0.f;
    ds = seen ? p * (dp - delta) * scale : 0.f;
}

template <typename T, int DP>
__global__ void __launch_bounds__(kThreads) dq_kernel(const __grid_constant__ Bwd a)
{
    extern __shared__ __align__(16) float sm[];
    constexpr int LD = Dim<DP>::LD, NC = Dim<DP>::NC;
    float *sQ = sm, *sO = sQ + kT * LD, *sK = sO + kT * LD, *sV = sK + kT * LD, *sW = sV + kT * LD;
    const int b = blockIdx.z, h = blockIdx.y, q0 = ((int)gridDim.x - 1 - (int)blockIdx.x) * kT, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int nq = a.band.nq, nk = a.band.nk, d = a.d;
    const Row R = row_of(a.band, b);
    const size_t qrow = ((size_t)b * a.H + h) * nq, krow = ((size_t)b * a.Hkv + h / (a.H / a.Hkv)) * nk;
    const T *k = static_cast<const T *>(a.k) + krow * d, *v = static_cast<const T *>(a.v) + krow * d;
    stage<DP>(sQ, static_cast<const T *>(a.q) + qrow * d, q0, nq, d, All{});
    stage<DP>(sO, static_cast<const T *>(a.dout) + qrow * d, q0, nq, d, All{});
    const Tiles t = tiles_of(R, R.pos + q0, R.pos + min(q0 + kT, nq) - 1);
    const float c = a.scale * kLog2e;
    float lse2[4], dl[4], o[4][NC];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = min(q0 + 4 * ty + i, nq - 1);
        lse2[i] = a.lse[qrow + row] * kLog2e;
        dl[i] = a.delta[qrow + row];
#pragma unroll
        for (int u = 0; u < NC; ++u) o[i][u] = 0.f;
    }
    for (int it = 0; it < t.count(); ++it) {
        const int j0 = t.at(it) * kT;
        __syncthreads();
        auto used = [&](int j) { return R.used(j); };
        stage<DP>(sK, k, j0, nk, d, used);
        stage<DP>(sV, v, j0, nk, d, used);
        __syncthreads();
        float s[4][4], dp[4][4];
        scores<DP>(sQ, sK, ty, tx, s);
        scores<DP>(sO, sV, ty, tx, dp);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float p, ds;
                weights(R.sees(R.pos + q0 + 4 * ty + i, j0 + tx + 16 * j), s[i][j], dp[i][j], c, a.scale, lse2[i], dl[i], p, ds);
                sW[(4 * ty + i) * (kT + 4) + tx + 16 * j] = ds;
            }
        __syncwarp();
        apply<DP>(sW, sK, ty, tx, o);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = q0 + 4 * ty + i;
        if (row >= nq) break;
        T *out = static_cast<T *>(a.dq) + (qrow + row) * d;
#pragma unroll
        for (int u = 0; u < NC; ++u)
            if (channel<DP>(tx, u) < d) Elem<T>::store(out + channel<DP>(tx, u), o[i][u]);
    }
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

template <typename T, int DP>
__global__ void __launch_bounds__(kThreads) dkv_kernel(const __grid_constant__ BwdCut c)
{
    const Bwd &a = c.a;
    extern __shared__ __align__(16) float sm[];
    constexpr int LD = Dim<DP>::LD, NC = Dim<DP>::NC;
    float *sQ = sm, *sO = sQ + kT * LD, *sK = sO + kT * LD, *sV = sK + kT * LD, *sP = sV + kT * LD, *sW = sP + kT * (kT + 4), *sL = sW + kT * (kT + 4);
    const int b = blockIdx.z, hk = blockIdx.y, tx = threadIdx.x & 15, ty = threadIdx.x >> 4, G = a.H / a.Hkv;
    const bool has_sinks = (int)blockIdx.x < c.cut.works(1);
    const int work = blockIdx.x - (has_sinks ? 0 : c.cut.works(1)), parts = has_sinks ? c.cut.sink_parts : c.cut.key_parts, part = work % parts;
    const int j0 = (work / parts + (has_sinks ? 0 : c.cut.sink_tiles)) * kT;
    const int nq = a.band.nq, nk = a.band.nk, d = a.d;
    const Row R = row_of(a.band, b);
    const size_t krow = ((size_t)b * a.Hkv + hk) * nk;
    auto used = [&](int j) { return R.used(j); };
    stage<DP>(sK, static_cast<const T *>(a.k) + krow * d, j0, nk, d, used);
    stage<DP>(sV, static_cast<const T *>(a.v) + krow * d, j0, nk, d, used);
    // queries that see a key of the tile: positions j0 - right .. j0 + 63 + left, all later ones if the tile holds a sink
    const int i0 = max(j0 - R.right - R.pos, 0), i1 = j0 < R.sinks ? nq - 1 : (int)min((long long)nq - 1, (long long)j0 + kT - 1 + R.left - R.pos);
    const float sc = a.scale * kLog2e;
    float dk[4][NC], dv[4][NC];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int u = 0; u < NC; ++u) dk[i][u] = dv[i][u] = 0.f;
    const int first = i0 / kT, per = j0 < R.len && i1 >= i0 ? i1 / kT - first + 1 : 0;
    const int from = (int)((long long)per * G * part / parts), to = (int)((long long)per * G * (part + 1) / parts);
    for (int u = from; u < to; ++u) {
        const size_t qrow = ((size_t)b * a.H + hk * G + u / per) * nq;
        const int q0 = (first + u % per) * kT;
        __syncthreads();
        stage<DP>(sQ, static_cast<const T *>(a.q) + qrow * d, q0, nq, d, All{});
        stage<DP>(sO, static_cast<const T *>(a.dout) + qrow * d, q0, nq, d, All{});
        if (threadIdx.x < kT) {
            const int row = min(q0 + (int)threadIdx.x, nq - 1);
            sL[threadIdx.x] = a.lse[qrow + row] * kLog2e;
            sL[kT + threadIdx.x] = a.delta[qrow + row];
        }
        __syncthreads();
        float s[4][4], dp[4][4];
        scores<DP>(sK, sQ, ty, tx, s);
        scores<DP>(sV, sO, ty, tx, dp);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = tx + 16 * j, at = (4 * ty + i) * (kT + 4) + row;
                const bool seen = q0 + row < nq && R.sees(R.pos + q0 + row, j0 + 4 * ty + i);
                weights(seen, s[i][j], dp[i][j], sc, a.scale, sL[row], sL[kT + row], sP[at], sW[at]);
            }
        __syncwarp();
        apply<DP>(sP, sO, ty, tx, dv);
        apply<DP>(sW, sQ, ty, tx, dk);
    }
    if (c.part != nullptr) {
        float *o = c.part + (((size_t)b * a.Hkv + hk) * c.cut.all() + blockIdx.x) * (2 * kT * DP);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int u = 0; u < NC; ++u) {
                o[(4 * ty + i) * DP + channel<DP>(tx, u)] = dk[i][u];
                o[(kT + 4 * ty + i) * DP + channel<DP>(tx, u)] = dv[i][u];
            }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = j0 + 4 * ty + i;
        if (row >= nk) break;
        T *ok = static_cast<T *>(a.dk) + (krow + row) * d, *ov = static_cast<T *>(a.dv) + (krow + row) * d;
#pragma unroll
        for (int u = 0; u < NC; ++u)
            if (channel<DP>(tx, u) < d) {
                Elem<T>::store(ok + channel<DP>(tx, u), dk[i][u]);
                Elem<T>::store(ov + channel<DP>(tx, u), dv[i][u]);
            }
    }
}

// dk (side 0) and dv of a key tile from its parts, in order
template <typename T, int DP>
__global__ void __launch_bounds__(kThreads) merge_kernel(const __grid_constant__ BwdCut c)
{
    const Bwd &a = c.a;
    const int tile = blockIdx.x >> 1, side = blockIdx.x & 1, hk = blockIdx.y, b = blockIdx.z, d = a.d;
    const bool has_sinks = tile < c.cut.sink_tiles;
    const int parts = has_sinks ? c.cut.sink_parts : c.cut.key_parts, first = has_sinks ? tile * parts : c.cut.works(1) + (tile - c.cut.sink_tiles) * parts;
    const float *p = c.part + (((size_t)b * a.Hkv + hk) * c.cut.all() + first) * (2 * kT * DP) + side * (kT * DP);
    T *out = static_cast<T *>(side ? a.dv : a.dk) + ((size_t)b * a.Hkv + hk) * a.band.nk * d;
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

template <typename T, int DP> cudaError_t fwd_t(const Fwd &a, cudaStream_t st)
{
    return launch<fwd_kernel<T, DP>>(a, dim3((a.band.nq + kT - 1) / kT, a.H, a.B), (3 * kT * Dim<DP>::LD + kT * (kT + 4)) * 4, st);
}
template <typename T, int DP> cudaError_t bwd_t(const Bwd &a, cudaStream_t st)
{
    const long long rows = (long long)a.B * a.H * a.band.nq;
    if (rows > 0) {
        delta_kernel<T><<<(unsigned)((rows + 7) / 8), 256, 0, st>>>(static_cast<const T *>(a.out), static_cast<const T *>(a.dout), a.delta, rows, a.d);
        cudaError_t e = cudaGetLastError();
        if (e == cudaSuccess)
            e = launch<dq_kernel<T, DP>>(a, dim3((a.band.nq + kT - 1) / kT, a.H, a.B), (4 * kT * Dim<DP>::LD + kT * (kT + 4)) * 4, st);
        if (e != cudaSuccess) return e;
    }
    if (a.band.nk == 0) return cudaSuccess;
    BwdCut c{a, cut_of(a.B, a.H, a.Hkv, a.band.nq, a.band.nk, a.band.left, a.band.right, a.band.sinks), nullptr};
    if (!c.cut.whole()) c.part = reinterpret_cast<float *>(reinterpret_cast<char *>(a.delta) + delta_bytes(a.B, a.H, a.band.nq));
    cudaError_t e = launch<dkv_kernel<T, DP>>(c, dim3(c.cut.all(), a.Hkv, a.B), (4 * kT * Dim<DP>::LD + 2 * kT * (kT + 4) + 2 * kT) * 4, st);
    if (e != cudaSuccess || c.part == nullptr) return e;
    return launch<merge_kernel<T, DP>>(c, dim3(2 * c.cut.tiles, a.Hkv, a.B), 0, st);
}

} // namespace

cudaError_t launch_fwd(const Fwd &a, cudaStream_t st)
{
    if (a.dtype == 0) return a.d <= 32 ? fwd_t<float, 32>(a, st) : a.d <= 64 ? fwd_t<float, 64>(a, st) : fwd_t<float, 128>(a, st);
    return few_supported(a.dtype, a.H, a.Hkv, a.band.nq, a.band.nk) ? launch_few(a, st) : launch_fwd_tc(a, st);
}
size_t bwd_f32_workspace(int B, int H, int Hkv, int nq, int nk, int d, int left, int right, int sinks)
{
    const Cut c = cut_of(B, H, Hkv, nq, nk, left, right, sinks);
    return delta_bytes(B, H, nq) + ((part_floats(c, B, Hkv, d <= 32 ? 32 : d <= 64 ? 64 : 128) * 4 + 255) & ~(size_t)255);
}

cudaError_t launch_bwd(const Bwd &a, cudaStream_t st)
{
    if (a.dtype == 0) return a.d <= 32 ? bwd_t<float, 32>(a, st) : a.d <= 64 ? bwd_t<float, 64>(a, st) : bwd_t<float, 128>(a, st);
    return launch_bwd_tc(a, st);
}

} // namespace window
} // namespace lot
