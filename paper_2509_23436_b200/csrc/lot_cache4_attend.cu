// Attention of few queries over the 4-bit cache (lot_cache4_attention).
//
// Bound by the bytes of the cache, if the instructions that take four-bit codes to operands can be kept below: 1.25 bytes a pair of
// channels, so at the copy rate an SM has about 110 clocks for 16 tokens of 128 channels, keys and values.  Hence
//   - the queries are the narrow side of the products (16 x 8 x 16: sixteen tokens by eight query rows), the codes the wide one, and one
//     masked shift makes two entries of an operand: 0x4300 | code is the bf16 number 128 + code.  The query rows of a key head (its query
//     heads times the new tokens) share its codes.
//   - scale and least value never touch the codes: S = s (sum q (128 + n) - 128 sum q) + z sum q for each group of 32 channels, and
//     sum_j p_j v_j = sum (p_j s_j) (n_j - 8) + sum p_j (z_j + 8 s_j); the latter product's weights p_j s_j are rounded to bf16, so the
//     codes are centred for it (n - 8 is exact): the rounding counts for no more than it would on the values themselves.
//   - float32 queries: three bf16 terms that sum to the number exactly; weights likewise.
// A warp goes over chunks of 32 tokens by itself: its lanes fetch them with bulk copies into a ring of its own.  Running maximum and sum
// per warp (the maximum moves only when a score passes it by 2^8), warps and blocks of a split join at the end.
#include "lot_chain.cuh"
#include "lot_sm100.cuh"
#include "lot_window.cuh"

#include <mutex>

namespace lot {
int device_sm_count();
namespace window {
namespace {

using namespace sm100;

constexpr int kWarps = 4, kThreads = kWarps * 32, kChunk = 32, kStages = 3, kRows = 8;
constexpr float kLift = 8.f;               // log2 of how far a weight may pass 1 before the reference moves

template <int D> struct Lay {
    static constexpr int W = D / kGroup, CODES = kChunk * D / 2, PARAMS = kChunk * D / 8, STAGE = 2 * (CODES + PARAMS);
    static constexpr int RING = kStages * STAGE, MERGE = kRows * D * 4 + 2 * kRows * 4;      // of a warp
    static constexpr int WARP = RING > MERGE ? RING : MERGE, TOTAL = kWarps * WARP + kWarps * kStages * 8 + 16;
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, const float (&c)[4])
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
// codes i and i + 4 of a word as bf16 128 + code
__device__ __forceinline__ uint32_t lifted(uint32_t w, int i)
{
    uint32_t r;
    asm("lop3.b32 %0, %1, 0x000f000f, 0x43004300, 0xea;" : "=r"(r) : "r"(w >> (4 * i)));
    return r;
}
__device__ __forceinline__ uint32_t centred(uint32_t w, int i)                   // code - 8, exactly
{
    const uint32_t x = lifted(w, i), c = 0x43084308u;                           // 136
    const __nv_bfloat162 y = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&x), *reinterpret_cast<const __nv_bfloat162 *>(&c));
    return *reinterpret_cast<const uint32_t *>(&y);
}
__device__ __forceinline__ uint32_t flip(uint32_t x)                            // 8 x 8 transposed across the warp
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ uint32_t pack(float lo, float hi)
{
    const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&t);
}
// a pair as TERMS bf16 pairs, largest first: what is left over is less than 2^-8 of the term before
template <int TERMS> __device__ __forceinline__ void terms(float a, float b, uint32_t (&o)[TERMS])
{
#pragma unroll
    for (int i = 0; i < TERMS; ++i) {
        o[i] = pack(a, b);
        a -= __uint_as_float(o[i] << 16);
        b -= __uint_as_float(o[i] & 0xffff0000u);
    }
}

struct Args {
    Attend4 a;
    int splits, row_tiles, G;
    float *part;                           // splits > 1: [row tile][B Hkv][split][kRows][D + 2]: sums, maximum (base 2), weight
};

// chunks of 32 tokens that the rows at positions p0 .. p1 see: those of the sinks, then the window's
struct Chunks {
    int sink, first, last;
    __device__ __forceinline__ int count() const { return sink + max(last - first + 1, 0); }
    __device__ __forceinline__ int at(int i) const { return i < sink ? i : first + i - sink; }
};

template <int D, typename T>
__global__ void __launch_bounds__(kThreads, 3) attend_kernel(const __grid_constant__ Args A)
{
    extern __shared__ __align__(128) uint8_t smem[];
    using L = Lay<D>;
    constexpr int W = L::W, TERMS = sizeof(T) == 4 ? 3 : 1;
    const Attend4 &a = A.a;
    const Cache4 &c = a.cache;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int split = blockIdx.x % A.splits, tile = blockIdx.x / A.splits, hk = blockIdx.y, b = blockIdx.z;
    const int rows = A.G * a.band.nq, r0 = tile * kRows;
    const int len = min(max(a.band.key_len[b], 0), a.band.nk), pos = len - a.band.nq;
    // row r of the key head: query head hk G + r / nq, query r % nq
    auto position = [&](int r) { return pos + r % a.band.nq; };
    int p0 = pos, p1 = len - 1;
    if (a.band.nq == 1) p0 = p1;
    Chunks ch;
    {
        const int lo = max(p0 - a.band.left, 0);
        ch.last = p1 < 0 ? -1 : p1 / kChunk;
        ch.first = lo / kChunk;
        ch.sink = min((min(a.band.sinks, p1 + 1) + kChunk - 1) / kChunk, ch.first);
        if (ch.sink < 0) ch.sink = 0;
    }
    const int wfirst = max(p0 - a.band.left, 0);           // no row sees a token before it but the sinks
    const int total = ch.count(), step = A.splits * kWarps, mine = split * kWarps + warp;
    const int turns = mine < total ? (total - mine + step - 1) / step : 0;

    uint8_t *ring = smem + warp * L::WARP;
    const uint32_t ring_s = smem_u32(ring), bars = smem_u32(smem) + kWarps * L::WARP + warp * kStages * 8;
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + kWarps * L::WARP + kWarps * kStages * 8);
    if (lane == 0)
        for (int s = 0; s < kStages; ++s) mbar_init(bars + 8 * s, 1);
    if (tid == 0) *abort_flag = 0;
    fence_barrier_init();
    __syncthreads();

    // A chunk's two blocks of 16 tokens may lie in different pages: lanes 0 .. 7 copy (block, codes or parameters, side).  Blocks that no row
    // sees are not read, nor are their page entries.  Returns the blocks that came (bit k).
    auto fetch = [&](int turn) -> uint32_t {
        const int s = turn % kStages, tok = ch.at(mine + turn * step) * kChunk + (lane & 1) * kBlockTokens;
        const bool want = tok <= p1 && (tok + kBlockTokens > wfirst || tok < a.band.sinks);
        int page = -1;
        if (want) {
            page = __ldg(c.pages + (size_t)b * c.max_pages + tok / c.page_size);
            if (page < 0 || page >= c.num_pages) {
                if (a.status != nullptr && lane < 2) atomicOr(a.status, 32 /* LOT_DEV_PAGE */);
                page = -1;
            }
        }
        const uint32_t got = __ballot_sync(0xffffffffu, page >= 0) & 3u;
        if (lane == 0) mbar_arrive_expect_tx(bars + 8 * s, __popc(got) * (L::STAGE / 2));
        __syncwarp();
        if (lane < 8 && page >= 0) {
            const int side = (lane >> 1) & 1, par = lane >> 2, blk = lane & 1, at = tok % c.page_size;
            const uint8_t *base = side_base(c, page, hk, side);
            const uint32_t dst = ring_s + s * L::STAGE + side * (L::CODES + L::PARAMS);
            if (par == 0) bulk_load(dst + blk * (L::CODES / 2), base + (size_t)at * (D / 2), L::CODES / 2, bars + 8 * s);
            else bulk_load(dst + L::CODES + blk * (L::PARAMS / 2), base + (size_t)c.page_size * (D / 2) + (size_t)at * (D / 8), L::PARAMS / 2, bars + 8 * s);
        }
        return got;
    };
    uint32_t present = 0;                                  // two bits a stage
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s)
        if (s < turns) present |= fetch(s) << (2 * s);

    // queries: this lane's channels of query row g as B operands, and the rows' sums over each group
    uint32_t qf[TERMS][W][2][2];
    float qsum[W][2];
    {
        const int r = r0 + g;
        const T *q = static_cast<const T *>(a.q) + (((size_t)b * a.H + hk * A.G + (r < rows ? r / a.band.nq : 0)) * a.band.nq + (r < rows ? r % a.band.nq : 0)) * D;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            float x[8];
            {
                float y[4];
                load4(q + 32 * w + 8 * t, y);
                x[0] = y[0]; x[1] = y[1]; x[2] = y[2]; x[3] = y[3];
                load4(q + 32 * w + 8 * t + 4, y);
                x[4] = y[0]; x[5] = y[1]; x[6] = y[2]; x[7] = y[3];
            }
            if (r >= rows) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = 0.f;
            }
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += x[e];
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            qsum[w][0] = __shfl_sync(0xffffffffu, sum, 8 * t);             // of row 2 t
            qsum[w][1] = __shfl_sync(0xffffffffu, sum, 8 * t + 4);         // of row 2 t + 1
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t o[TERMS];
                terms<TERMS>(x[e], x[e + 4], o);
#pragma unroll
                for (int m = 0; m < TERMS; ++m) qf[m][w][e >> 1][e & 1] = o[m];
            }
        }
    }
    const float scale = a.scale * kLog2e;
    float o[2 * W][4], zs[W][2], ref[2] = {neg_inf(), neg_inf()}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int m = 0; m < 2 * W; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[m][e] = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) zs[w][0] = zs[w][1] = 0.f;
    const int prow[2] = {position(min(r0 + 2 * t, rows - 1)), position(min(r0 + 2 * t + 1, rows - 1))};

    for (int turn = 0; turn < turns; ++turn) {
        const int s = turn % kStages, tok0 = ch.at(mine + turn * step) * kChunk;
        if (turn + kStages - 1 < turns) {
            const int sn = (turn + kStages - 1) % kStages;
            __syncwarp();                                  // the stage's readers are done
            present = (present & ~(3u << (2 * sn))) | (fetch(turn + kStages - 1) << (2 * sn));
        }
        if (!mbar_wait(bars + 8 * s, (turn / kStages) & 1, abort_flag, a.status != nullptr ? a.status : const_cast<int *>(abort_flag))) {
            for (int u = turn + 1; u < turns && u < turn + kStages; ++u)           // copies on their way, before the block may end
                for (int it = 0; it < 4096 && !mbar_try_wait(bars + 8 * (u % kStages), (u / kStages) & 1); ++it) {}
            break;
        }
        const uint32_t got = (present >> (2 * s)) & 3u;
        uint8_t *st = ring + s * L::STAGE;
        uint32_t *kp = reinterpret_cast<uint32_t *>(st + L::CODES), *vp = reinterpret_cast<uint32_t *>(st + 2 * L::CODES + L::PARAMS);
        const bool whole = got == 3u && tok0 >= wfirst && tok0 + kChunk - 1 <= p1 && (p1 == p0 || (tok0 + kChunk - 1 <= p0 && tok0 >= p1 - a.band.left));
        if (!whole) {
            // tokens that no row sees: parameters of zero, whatever is there
            const int j = tok0 + lane;
            const bool there = ((got >> (lane >> 4)) & 1u) && j <= p1 && (j >= wfirst || j < a.band.sinks);
            if (!there) {
#pragma unroll
                for (int w = 0; w < W; ++w) kp[lane * W + w] = vp[lane * W + w] = 0u;
                fence_proxy_async_smem();                  // before a later copy writes there
            }
            __syncwarp();
        }
        float S[2][4];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const uint32_t *k0 = reinterpret_cast<const uint32_t *>(st + (kb * 16 + g) * (D / 2) + t * 4 * W), *k1 = k0 + 8 * (D / 8);
            uint32_t ka[W], kc[W], pa[W], pc[W];
#pragma unroll
            for (int w = 0; w < W; ++w) {
                ka[w] = k0[w]; kc[w] = k1[w];
                pa[w] = kp[(kb * 16 + g) * W + w]; pc[w] = kp[(kb * 16 + g + 8) * W + w];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) S[kb][e] = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                // bf16 queries: the products' 128 is taken out beforehand; float32 ones: of the codes, 128 sums would cost five bits
                constexpr float kOff = TERMS == 1 ? 128.f : 0.f;
                float x[4] = {-kOff * qsum[w][0], -kOff * qsum[w][1], -kOff * qsum[w][0], -kOff * qsum[w][1]};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t f[4];
                    f[0] = TERMS == 1 ? lifted(ka[w], 2 * h) : centred(ka[w], 2 * h);
                    f[1] = TERMS == 1 ? lifted(kc[w], 2 * h) : centred(kc[w], 2 * h);
                    f[2] = TERMS == 1 ? lifted(ka[w], 2 * h + 1) : centred(ka[w], 2 * h + 1);
                    f[3] = TERMS == 1 ? lifted(kc[w], 2 * h + 1) : centred(kc[w], 2 * h + 1);
#pragma unroll
                    for (int m = TERMS - 1; m >= 0; --m) mma(x, f, qf[m][w][h][0], qf[m][w][h][1], x);
                }
                const float s0 = param_scale(pa[w]), s1 = param_scale(pc[w]);
                const float z0 = fmaf(TERMS == 1 ? 0.f : 8.f, s0, param_least(pa[w])), z1 = fmaf(TERMS == 1 ? 0.f : 8.f, s1, param_least(pc[w]));
                S[kb][0] = fmaf(s0, x[0], fmaf(z0, qsum[w][0], S[kb][0]));
                S[kb][1] = fmaf(s0, x[1], fmaf(z0, qsum[w][1], S[kb][1]));
                S[kb][2] = fmaf(s1, x[2], fmaf(z1, qsum[w][0], S[kb][2]));
                S[kb][3] = fmaf(s1, x[3], fmaf(z1, qsum[w][1], S[kb][3]));
            }
        }
        if (!whole) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = tok0 + kb * 16 + g + (e >> 1) * 8, p = prow[e & 1];
                    const bool seen = ((got >> kb) & 1u) && j <= p && (j >= p - a.band.left || j < a.band.sinks);
                    S[kb][e] = seen ? S[kb][e] : neg_inf();
                }
        }
        float top[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) top[q] = scale * fmaxf(fmaxf(S[0][q], S[0][q + 2]), fmaxf(S[1][q], S[1][q + 2]));
        if (__any_sync(0xffffffffu, top[0] > ref[0] + kLift || top[1] > ref[1] + kLift)) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float m = fmaxf(top[q], ref[q]);
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                const float f = m == neg_inf() ? 1.f : ex2(ref[q] - m);
                ref[q] = m;
                l[q] *= f;
#pragma unroll
                for (int w = 0; w < W; ++w) zs[w][q] *= f;
#pragma unroll
                for (int m2 = 0; m2 < 2 * W; ++m2) { o[m2][q] *= f; o[m2][q + 2] *= f; }
            }
        }
        const float r0v = ref[0] == neg_inf() ? 0.f : ref[0], r1v = ref[1] == neg_inf() ? 0.f : ref[1];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            S[kb][0] = ex2(fmaf(S[kb][0], scale, -r0v));
            S[kb][1] = ex2(fmaf(S[kb][1], scale, -r1v));
            S[kb][2] = ex2(fmaf(S[kb][2], scale, -r0v));
            S[kb][3] = ex2(fmaf(S[kb][3], scale, -r1v));
            l[0] += S[kb][0] + S[kb][2];
            l[1] += S[kb][1] + S[kb][3];
            const uint8_t *vb = st + L::CODES + L::PARAMS + kb * (L::CODES / 2);
            const uint32_t *v0 = reinterpret_cast<const uint32_t *>(vb) + lane * W, *v1 = v0 + 32 * W;
            uint32_t va[W], vc[W], pa[W], pc[W];
#pragma unroll
            for (int w = 0; w < W; ++w) {
                va[w] = v0[w]; vc[w] = v1[w];
                pa[w] = vp[(kb * 16 + g) * W + w]; pc[w] = vp[(kb * 16 + g + 8) * W + w];
            }
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float s0 = param_scale(pa[w]), s1 = param_scale(pc[w]);
                const float z0 = fmaf(8.f, s0, param_least(pa[w])), z1 = fmaf(8.f, s1, param_least(pc[w]));
                zs[w][0] = fmaf(S[kb][0], z0, fmaf(S[kb][2], z1, zs[w][0]));
                zs[w][1] = fmaf(S[kb][1], z0, fmaf(S[kb][3], z1, zs[w][1]));
                uint32_t x0[TERMS], x1[TERMS];
                terms<TERMS>(S[kb][0] * s0, S[kb][1] * s0, x0);
                terms<TERMS>(S[kb][2] * s1, S[kb][3] * s1, x1);
#pragma unroll
                for (int m = 0; m < TERMS; ++m) { x0[m] = flip(x0[m]); x1[m] = flip(x1[m]); }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t f[4];
                    f[0] = centred(va[w], 2 * h);
                    f[1] = centred(va[w], 2 * h + 1);
                    f[2] = centred(vc[w], 2 * h);
                    f[3] = centred(vc[w], 2 * h + 1);
#pragma unroll
                    for (int m = TERMS - 1; m >= 0; --m) mma(o[2 * w + h], f, x0[m], x1[m], o[2 * w + h]);
                }
            }
        }
    }
    // the lanes of a row's tokens together
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) {
            l[q] += __shfl_xor_sync(0xffffffffu, l[q], x);
#pragma unroll
            for (int w = 0; w < W; ++w) zs[w][q] += __shfl_xor_sync(0xffffffffu, zs[w][q], x);
        }
    __syncthreads();                                       // every warp has left its ring
    float *mo = reinterpret_cast<float *>(ring), *mm = mo + kRows * D;
#pragma unroll
    for (int m = 0; m < 2 * W; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) mo[(2 * t + (e & 1)) * D + 16 * m + g + (e >> 1) * 8] = o[m][e] + zs[m >> 1][e & 1];
    if (g == 0) {
        mm[2 * t] = ref[0]; mm[2 * t + 1] = ref[1];
        mm[kRows + 2 * t] = l[0]; mm[kRows + 2 * t + 1] = l[1];
    }
    __syncthreads();
    const bool failed = *abort_flag != 0;
    for (int idx = tid; idx < kRows * D; idx += kThreads) {
        const int r = idx / D, ch_ = idx % D;
        if (r0 + r >= rows) break;
        float top = neg_inf();
#pragma unroll
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, reinterpret_cast<const float *>(smem + w * L::WARP)[kRows * D + r]);
        const float at = top == neg_inf() ? 0.f : top;
        float sum = 0.f, x = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float *p = reinterpret_cast<const float *>(smem + w * L::WARP);
            const float f = ex2(p[kRows * D + r] - at);
            sum += f * p[kRows * D + kRows + r];
            x += f * p[r * D + ch_];
        }
        if (failed) sum = x = __int_as_float(0x7fc00000);
        if (A.splits > 1) {
            float *part = A.part + ((((size_t)tile * a.B + b) * c.Hkv + hk) * A.splits + split) * (kRows * (D + 2)) + r * (D + 2);
            part[ch_] = x;
            if (ch_ == 0) { part[D] = top; part[D + 1] = sum; }
        } else {
            const size_t row = ((size_t)b * a.H + hk * A.G + (r0 + r) / a.band.nq) * a.band.nq + (r0 + r) % a.band.nq;
            Elem<T>::store(static_cast<T *>(a.out) + row * D + ch_, sum > 0.f ? x / sum : failed ? x : 0.f);
            if (ch_ == 0 && a.lse != nullptr) a.lse[row] = sum > 0.f ? top * kLn2 + logf(sum) : failed ? x : neg_inf();
        }
    }
    chain_next();
}

// a block joins the splits of one row
template <int D, typename T>
__global__ void __launch_bounds__(D) join_kernel(const __grid_constant__ Args A)
{
    const Attend4 &a = A.a;
    const int r = blockIdx.x, hk = blockIdx.y, b = blockIdx.z, ch = threadIdx.x;
    const float *part = A.part + ((((size_t)(r / kRows) * a.B + b) * a.cache.Hkv + hk) * A.splits) * (kRows * (D + 2)) + (r % kRows) * (D + 2);
    chain_wait();
    float top = neg_inf();
    for (int s = 0; s < A.splits; ++s) top = fmaxf(top, chain_ld(part + (size_t)s * kRows * (D + 2) + D));
    const float at = top == neg_inf() ? 0.f : top;
    float sum = 0.f, x = 0.f;
    for (int s = 0; s < A.splits; ++s) {
        const float *p = part + (size_t)s * kRows * (D + 2);
        const float f = ex2(chain_ld(p + D) - at);
        sum += f * chain_ld(p + D + 1);
        x += f * chain_ld(p + ch);
    }
    const size_t row = ((size_t)b * a.H + hk * A.G + r / a.band.nq) * a.band.nq + r % a.band.nq;
    const bool nothing = sum == 0.f;
    Elem<T>::store(static_cast<T *>(a.out) + row * D + ch, nothing ? 0.f : x / sum);
    if (ch == 0 && a.lse != nullptr) a.lse[row] = nothing ? neg_inf() : top * kLn2 + logf(sum);
}

// Splits of a sequence's chunks: enough blocks for two waves of three an SM, and no warp with less than two chunks.
int splits_of(int sms, int B, int Hkv, int tiles, int nk, int nq, int left, int sinks)
{
    const long long seen = (left < nk ? left + 1ll : nk) + nq - 1 + sinks, chunks = ((seen < nk ? seen : nk) + kChunk - 1) / kChunk + 1;
    const long long blocks = (long long)B * Hkv * tiles, want = (6ll * sms + blocks - 1) / blocks, most = (chunks + 2 * kWarps - 1) / (2 * kWarps);
    const long long s = want < most ? want : most;
    return s < 1 ? 1 : s > 512 ? 512 : (int)s;
}

template <int D, typename T> cudaError_t run(const Args &A, cudaStream_t st)
{
    static std::mutex mu;
    static bool set[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!set[dev]) {
            const cudaError_t e = cudaFuncSetAttribute(attend_kernel<D, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, Lay<D>::TOTAL);
            if (e != cudaSuccess) return e;
            set[dev] = true;
        }
    }
    attend_kernel<D, T><<<dim3(A.splits * A.row_tiles, A.a.cache.Hkv, A.a.B), kThreads, Lay<D>::TOTAL, st>>>(A);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || A.splits == 1) return e;
    return chain_launch(join_kernel<D, T>, dim3(A.G * A.a.band.nq, A.a.cache.Hkv, A.a.B), D, 0, st, A);
}

} // namespace

size_t attend4_workspace(int dtype, int B, int H, int Hkv, int nq, int d, int nk, int left, int sinks)
{
    (void)dtype;
    const int tiles = (H / Hkv * nq + kRows - 1) / kRows, s = splits_of(device_sm_count(), B, Hkv, tiles, nk, nq, left, sinks);
    if (s == 1) return 0;
    return ((size_t)tiles * B * Hkv * s * kRows * (d + 2) * 4 + 255) & ~(size_t)255;
}

cudaError_t launch_attend4(const Attend4 &a, cudaStream_t st)
{
    Args A;
    A.a = a;
    A.G = a.H / a.cache.Hkv;
    A.row_tiles = (A.G * a.band.nq + kRows - 1) / kRows;
    A.splits = splits_of(device_sm_count(), a.B, a.cache.Hkv, A.row_tiles, a.band.nk, a.band.nq, a.band.left, a.band.sinks);
    A.part = static_cast<float *>(a.ws);
    const int d = a.cache.d;
    if (a.dtype == 0) return d == 32 ? run<32, float>(A, st) : d == 64 ? run<64, float>(A, st) : run<128, float>(A, st);
    return d == 32 ? run<32, __nv_bfloat16>(A, st) : d == 64 ? run<64, __nv_bfloat16>(A, st) : run<128, __nv_bfloat16>(A, st);
}

} // namespace window
} // namespace lot
