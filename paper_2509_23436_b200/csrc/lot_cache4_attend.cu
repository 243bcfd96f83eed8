// Attention of few queries over the 4-bit cache (lot_cache4_attention).
//
// Bound by the bytes of the cache, if the instructions that take four-bit codes to operands can be kept below: 1.25 bytes a pair of
// channels, so at the copy rate an SM has about 110 clocks for 16 tokens of 128 channels, keys and values.  Hence
//   - the queries are the narrow side of the products (16 x 8 x 16: sixteen tokens by eight query rows), the codes the wide one, and one
//     shift and mask make two entries of an operand: 0x4300 | code is the bf16 number 128 + code.  (0x6400 | code << 4 k, f16 numbers, would
//     save two shifts of a word's three, but sums that begin at 1024 times the queries lose four digits of a score in the tensor cores.)
//     The query rows of a key head (its query heads times the new tokens) share its codes.
//   - scale and least value never touch the codes: S = s (sum q n) + z sum q for each group of 32 channels, and
//     sum_j p_j v_j = sum (p_j s_j) (n_j - 8) + sum p_j (z_j + 8 s_j).  The values' 136 goes off the operands (one subtraction a pair, exact), so that the
//     rounding of the weights p_j s_j to bf16 counts for no more than it would on the values themselves; off the sums, by a product of the same
//     weights with a constant, it took 162 us where this takes 150.  The keys' 128 goes off the sums:
//   - (z - 128 s) sum q of all groups is two more products, the sums as three bf16 terms.
//   - float32 queries: everything as three bf16 terms that sum to the number exactly, and centred codes.
// A warp goes over chunks of 32 tokens by itself: its lanes fetch them with bulk copies into a ring of its own.  Running maximum and sum
// per warp (the maximum moves only when a score passes it by 2^8), warps and blocks of a split join at the end: the blocks of few
// sequences through a cluster's shared memory (one launch, latency), of many through memory and join_kernel.
// 32 sequences of up to 16384 tokens, 32 heads on 8 of 128 channels: 150 us, 3.4 TB/s.  At 166 us issue slots were 60 % used and the ALU
// pipe 55 %, and three blocks an SM with three stages took 175, five of 96 registers 190.
#include "lot_chain.cuh"
#include "lot_sm100.cuh"
#include "lot_window.cuh"

#include <mutex>

namespace lot {
int device_sm_count();
namespace window {
namespace {

using namespace sm100;

constexpr int kWarps = 4, kThreads = kWarps * 32, kChunk = 32, kStages = 2, kRows = 8, kBlocks = 4;      // kBlocks: on an SM at once
constexpr float kLift = 8.f;               // log2 of how far a weight may pass 1 before the reference moves

template <int D> struct Lay {
    static constexpr int W = D / kGroup, CODES = kChunk * D / 2, PARAMS = kChunk * D / 8, STAGE = 2 * (CODES + PARAMS);
    static constexpr int RING = kStages * STAGE, MERGE = kRows * D * 4 + 2 * kRows * 4;      // of a warp
    static constexpr int WARP = RING > MERGE ? RING : MERGE, OWN = kWarps * WARP + kWarps * kStages * 8 + 16, TOTAL = OWN + (kRows * D + 2 * kRows) * 4;
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
    int splits, each, row_tiles, G, shift; // each: chunks of a split; shift: log2 of the page size where that is whole, else -1
    int clustered;                         // the splits are the blocks of a cluster
    float *part;                           // else, splits > 1: [row tile][B Hkv][split][kRows][D + 2]: sums, maximum (base 2), weight
};

// chunks of 32 tokens that the rows at positions p0 .. p1 see: those of the sinks, then the window's
struct Chunks {
    int sink, first, last;
    __device__ __forceinline__ int count() const { return sink + max(last - first + 1, 0); }
    __device__ __forceinline__ int at(int i) const { return i < sink ? i : first + i - sink; }
};

template <int W> __device__ __forceinline__ void words(const void *p, uint32_t (&w)[W])
{
    if constexpr (W == 4) {
        const uint4 v = *static_cast<const uint4 *>(p);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else if constexpr (W == 2) {
        const uint2 v = *static_cast<const uint2 *>(p);
        w[0] = v.x; w[1] = v.y;
    } else {
        w[0] = *static_cast<const uint32_t *>(p);
    }
}

template <int D, typename T>
__global__ void __launch_bounds__(kThreads, kBlocks) attend_kernel(const __grid_constant__ Args A)
{
    extern __shared__ __align__(128) uint8_t smem[];
    using L = Lay<D>;
    constexpr int W = L::W, TERMS = sizeof(T) == 4 ? 3 : 1;
    constexpr bool kLifted = TERMS == 1;                   // keys: products of 128 + code, the 128 taken out of the sums
    const Attend4 &a = A.a;
    const Cache4 &c = a.cache;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int split = blockIdx.x % A.splits, tile = blockIdx.x / A.splits, hk = blockIdx.y, b = blockIdx.z;
    const int rows = A.G * a.band.nq, r0 = tile * kRows;
    const int len = min(max(a.band.key_len[b], 0), a.band.nk), p0 = len - a.band.nq, p1 = len - 1;     // positions of the first and last query
    // row r of the key head: query head hk G + r / nq, query r % nq
    Chunks ch;
    const int wfirst = max(p0 - a.band.left, 0);           // no row sees a token before it but the sinks
    ch.last = p1 < 0 ? -1 : p1 / kChunk;
    ch.first = wfirst / kChunk;
    ch.sink = max(min((min(a.band.sinks, p1 + 1) + kChunk - 1) / kChunk, ch.first), 0);
    const int total = min(ch.count(), (split + 1) * A.each), mine = split * A.each + warp;      // this split's chunks, every fourth
    const int turns = mine < total ? (total - mine + kWarps - 1) / kWarps : 0;

    uint8_t *ring = smem + warp * L::WARP;
    const uint32_t ring_s = smem_u32(ring), bars = smem_u32(smem) + kWarps * L::WARP + warp * kStages * 8;
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + kWarps * L::WARP + kWarps * kStages * 8);
    if (lane == 0)
        for (int s = 0; s < kStages; ++s) mbar_init(bars + 8 * s, 1);
    if (tid == 0) *abort_flag = 0;
    fence_barrier_init();
    __syncthreads();

    // A chunk's two blocks of 16 tokens may lie in different pages: lanes 0 .. 7 copy (block, side, codes or parameters).  Blocks that no row
    // sees are not read, nor are their page entries.
    const int blk = lane & 1, side = (lane >> 1) & 1, par = (lane >> 2) & 1;
    const uint32_t dst0 = ring_s + side * (L::CODES + L::PARAMS) + (par ? L::CODES + blk * (L::PARAMS / 2) : blk * (L::CODES / 2));
    const uint32_t piece = par ? L::PARAMS / 2 : L::CODES / 2;
    const size_t page_bytes = side_bytes(c.page_size, D) * 2 * c.Hkv;
    const uint32_t unit = par ? D / 8 : D / 2;
    const uint8_t *lane_base = side_base(c, 0, hk, side) + (par ? (size_t)c.page_size * (D / 2) : 0);
    const int32_t *table = c.pages + (size_t)b * c.max_pages;
    auto token = [&](int turn) { return ch.at(mine + turn * kWarps) * kChunk + blk * kBlockTokens; };
    auto page_of = [&](int tok) { return A.shift >= 0 ? tok >> A.shift : tok / c.page_size; };
    auto entry = [&](int turn) -> int {                    // page of this lane's block, -1: none, -2: not there
        if (turn >= turns) return -1;
        const int tok = token(turn);
        if (!(tok <= p1 && (tok + kBlockTokens > wfirst || tok < a.band.sinks))) return -1;
        const int page = __ldg(table + page_of(tok));
        return page >= 0 && page < c.num_pages ? page : -2;
    };
    auto fetch = [&](int turn, int page) -> uint32_t {     // the blocks that come (bit k)
        const int s = turn % kStages;
        const uint32_t got = __ballot_sync(0xffffffffu, page >= 0) & 3u;
        if (lane == 0) mbar_arrive_expect_tx(bars + 8 * s, __popc(got) * (L::STAGE / 2));
        __syncwarp();
        const bool both = got == 3u && c.page_size % kChunk == 0;                       // neighbours: one copy for both (162 us, two 166)
        if (lane < 8 && page >= 0 && !(both && blk)) {
            const int tok = token(turn), at = tok - page_of(tok) * c.page_size;
            bulk_load(dst0 + s * L::STAGE, lane_base + page * page_bytes + (uint32_t)at * unit, both ? 2 * piece : piece, bars + 8 * s);
        }
        if (page == -2 && lane < 2 && a.status != nullptr) atomicOr(a.status, 32 /* LOT_DEV_PAGE */);
        return got;
    };
    uint32_t present = 0;                                  // two bits a stage
    int page[kStages];
#pragma unroll
    for (int s = 0; s < kStages; ++s) page[s] = entry(s);
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s)
        if (s < turns) present |= fetch(s, page[s]) << (2 * s);
    int ahead = page[kStages - 1];                         // page of the next chunk to fetch, asked for a turn before

    // queries: this lane's channels of query row g as B operands, and the rows' sums over each group
    uint32_t qf[TERMS][W][2][2], zb[2], sb[2];
    float qsum[W][2];
    {
        const int r = r0 + g;
        const T *q = static_cast<const T *>(a.q) + (((size_t)b * a.H + hk * A.G + (r < rows ? r / a.band.nq : 0)) * a.band.nq + (r < rows ? r % a.band.nq : 0)) * D;
        float mine_sum[W];
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
            float sum = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            mine_sum[w] = sum;
            qsum[w][0] = __shfl_sync(0xffffffffu, sum, 8 * t);                                         // of row 2 t
            qsum[w][1] = __shfl_sync(0xffffffffu, sum, 8 * t + 4);                                     // of row 2 t + 1
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t o[TERMS];
                terms<TERMS>(x[e], x[e + 4], o);
#pragma unroll
                for (int m = 0; m < TERMS; ++m) qf[m][w][e >> 1][e & 1] = o[m];
            }
        }
        // row g's sums as the operand of the least values: entries 0 .. 3 the first term of groups 0 .. 3, 4 .. 7 the second, 8 .. 11 the third
        uint32_t z3[2][3];
        terms<3>(mine_sum[0], W > 1 ? mine_sum[W > 1 ? 1 : 0] : 0.f, z3[0]);
        terms<3>(W > 2 ? mine_sum[W > 2 ? 2 : 0] : 0.f, W > 2 ? mine_sum[W > 2 ? 3 : 0] : 0.f, z3[1]);
        zb[0] = t == 0 ? z3[0][0] : t == 1 ? z3[1][0] : t == 2 ? z3[0][1] : z3[1][1];
        zb[1] = t == 0 ? z3[0][2] : t == 1 ? z3[1][2] : 0u;
        // -128 times as much, for the scales
#pragma unroll
        for (int e = 0; e < 2; ++e) sb[e] = pack(-128.f * __uint_as_float(zb[e] << 16), -128.f * __uint_as_float(zb[e] & 0xffff0000u));
    }
    const float scale = a.scale * kLog2e;
    float o[2 * W][4], zs[W][2], ref[2] = {neg_inf(), neg_inf()}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int m = 0; m < 2 * W; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[m][e] = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) zs[w][0] = zs[w][1] = 0.f;
    const int prow[2] = {p0 + min(r0 + 2 * t, rows - 1) % a.band.nq, p0 + min(r0 + 2 * t + 1, rows - 1) % a.band.nq};

    for (int turn = 0; turn < turns; ++turn) {
        const int s = turn % kStages, tok0 = ch.at(mine + turn * kWarps) * kChunk;
        if (turn + kStages - 1 < turns) {
            const int sn = (turn + kStages - 1) % kStages;
            __syncwarp();                                  // the stage's readers are done
            present = (present & ~(3u << (2 * sn))) | (fetch(turn + kStages - 1, ahead) << (2 * sn));
            ahead = entry(turn + kStages);
        }
        if (!mbar_wait(bars + 8 * s, (turn / kStages) & 1, abort_flag, a.status != nullptr ? a.status : const_cast<int *>(abort_flag))) {
            for (int u = turn + 1; u < turns && u < turn + kStages; ++u)           // copies on their way, before the block may end
                for (int it = 0; it < 4096 && !mbar_try_wait(bars + 8 * (u % kStages), (u / kStages) & 1); ++it) {}
            break;
        }
        const uint32_t got = (present >> (2 * s)) & 3u;
        uint8_t *st = ring + s * L::STAGE;
        uint32_t *kp = reinterpret_cast<uint32_t *>(st + L::CODES), *vp = reinterpret_cast<uint32_t *>(st + 2 * L::CODES + L::PARAMS);
        const bool whole = got == 3u && tok0 >= max(p1 - a.band.left, 0) && tok0 + kChunk - 1 <= p0;      // every row sees every token
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
            uint32_t ka[W], kc[W], pa[W], pc[W];
            words<W>(st + (kb * 16 + g) * (D / 2) + t * 4 * W, ka);
            words<W>(st + (kb * 16 + g + 8) * (D / 2) + t * 4 * W, kc);
            words<W>(kp + (kb * 16 + g) * W, pa);
            words<W>(kp + (kb * 16 + g + 8) * W, pc);
            if (kLifted) {
                // least values and scales: rows g, g + 8 by groups 2 (t % 2), 2 (t % 2) + 1
                uint32_t f[4], h[4];
                const bool up = t & 1;
                if (W == 4) {
                    const uint32_t a0 = up ? pa[W / 2] : pa[0], a1 = up ? pa[W - 1] : pa[W > 1], c0 = up ? pc[W / 2] : pc[0], c1 = up ? pc[W - 1] : pc[W > 1];
                    f[0] = __byte_perm(a0, a1, 0x7632);
                    f[1] = __byte_perm(c0, c1, 0x7632);
                    h[0] = __byte_perm(a0, a1, 0x5410);
                    h[1] = __byte_perm(c0, c1, 0x5410);
                } else {
                    const uint32_t a1 = W > 1 ? pa[W - 1] : 0u, c1 = W > 1 ? pc[W - 1] : 0u;
                    f[0] = up ? 0u : __byte_perm(pa[0], a1, 0x7632);
                    f[1] = up ? 0u : __byte_perm(pc[0], c1, 0x7632);
                    h[0] = up ? 0u : __byte_perm(pa[0], a1, 0x5410);
                    h[1] = up ? 0u : __byte_perm(pc[0], c1, 0x5410);
                }
                f[2] = f[0];
                f[3] = f[1];
                h[2] = h[0];
                h[3] = h[1];
                const float none[4] = {0.f, 0.f, 0.f, 0.f};
                mma(S[kb], f, zb[0], zb[1], none);
                mma(S[kb], h, sb[0], sb[1], S[kb]);
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    float x[4];
                    const uint32_t lo[4] = {lifted(ka[w], 0), lifted(kc[w], 0), lifted(ka[w], 1), lifted(kc[w], 1)};
                    mma(x, lo, qf[0][w][0][0], qf[0][w][0][1], none);
                    const uint32_t hi[4] = {lifted(ka[w], 2), lifted(kc[w], 2), lifted(ka[w], 3), lifted(kc[w], 3)};
                    mma(x, hi, qf[0][w][1][0], qf[0][w][1][1], x);
                    const float s0 = param_scale(pa[w]), s1 = param_scale(pc[w]);
                    S[kb][0] = fmaf(s0, x[0], S[kb][0]);
                    S[kb][1] = fmaf(s0, x[1], S[kb][1]);
                    S[kb][2] = fmaf(s1, x[2], S[kb][2]);
                    S[kb][3] = fmaf(s1, x[3], S[kb][3]);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) S[kb][e] = 0.f;
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    float x[4] = {0.f, 0.f, 0.f, 0.f}, y[4] = {0.f, 0.f, 0.f, 0.f};      // y: the small terms
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t f[4] = {centred(ka[w], 2 * h), centred(kc[w], 2 * h), centred(ka[w], 2 * h + 1), centred(kc[w], 2 * h + 1)};
#pragma unroll
                        for (int m = TERMS - 1; m > 0; --m) mma(y, f, qf[m][w][h][0], qf[m][w][h][1], y);
                        mma(x, f, qf[0][w][h][0], qf[0][w][h][1], x);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] += y[e];
                    const float s0 = param_scale(pa[w]), s1 = param_scale(pc[w]);
                    const float z0 = fmaf(8.f, s0, param_least(pa[w])), z1 = fmaf(8.f, s1, param_least(pc[w]));
                    S[kb][0] = fmaf(s0, x[0], fmaf(z0, qsum[w][0], S[kb][0]));
                    S[kb][1] = fmaf(s0, x[1], fmaf(z0, qsum[w][1], S[kb][1]));
                    S[kb][2] = fmaf(s1, x[2], fmaf(z1, qsum[w][0], S[kb][2]));
                    S[kb][3] = fmaf(s1, x[3], fmaf(z1, qsum[w][1], S[kb][3]));
                }
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
        const float top[2] = {scale * fmaxf(fmaxf(S[0][0], S[0][2]), fmaxf(S[1][0], S[1][2])), scale * fmaxf(fmaxf(S[0][1], S[0][3]), fmaxf(S[1][1], S[1][3]))};
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
            const uint8_t *vb = st + L::CODES + L::PARAMS + kb * (L::CODES / 2) + lane * 4 * W;
            uint32_t va[W], vc[W], pa[W], pc[W];
            words<W>(vb, va);
            words<W>(vb + 128 * W, vc);
            words<W>(vp + (kb * 16 + g) * W, pa);
            words<W>(vp + (kb * 16 + g + 8) * W, pc);
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
                    const uint32_t f[4] = {centred(va[w], 2 * h), centred(va[w], 2 * h + 1), centred(vc[w], 2 * h), centred(vc[w], 2 * h + 1)};
                    if (TERMS == 1) {
                        mma(o[2 * w + h], f, x0[0], x1[0], o[2 * w + h]);
                    } else {                               // products round their sums towards zero: short ones for float32
                        float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int m = TERMS - 1; m >= 0; --m) mma(y, f, x0[m], x1[m], y);
#pragma unroll
                        for (int n = 0; n < 4; ++n) o[2 * w + h][n] += y[n];
                    }
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
    const float nan = __int_as_float(0x7fc00000);
    const bool failed = *abort_flag != 0;
    // one row and channel of this block's warps: maximum, weight, sum
    auto of_block = [&](int r, int col, float &top, float &sum, float &x) {
        top = neg_inf();
#pragma unroll
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, reinterpret_cast<const float *>(smem + w * L::WARP)[kRows * D + r]);
        const float at = top == neg_inf() ? 0.f : top;
        sum = x = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float *p = reinterpret_cast<const float *>(smem + w * L::WARP);
            const float f = ex2(p[kRows * D + r] - at);
            sum += f * p[kRows * D + kRows + r];
            x += f * p[r * D + col];
        }
        if (failed) sum = x = nan;
    };
    auto write = [&](int r, int col, float top, float sum, float x) {
        const size_t row = ((size_t)b * a.H + hk * A.G + (r0 + r) / a.band.nq) * a.band.nq + (r0 + r) % a.band.nq;
        const bool nothing = sum == 0.f;
        Elem<T>::store(static_cast<T *>(a.out) + row * D + col, nothing ? 0.f : x / sum);
        if (col == 0 && a.lse != nullptr) a.lse[row] = nothing ? neg_inf() : top * kLn2 + logf(sum);
    };
    if (A.clustered) {
        // every block leaves its rows in its own shared memory (behind the warps' parts) and takes every splits-th number of all blocks'
        float *own = reinterpret_cast<float *>(smem + L::OWN);
        for (int idx = tid; idx < kRows * D; idx += kThreads) {
            float top, sum, x;
            of_block(idx / D, idx % D, top, sum, x);
            own[idx] = x;
            if (idx % D == 0) { own[kRows * D + idx / D] = top; own[kRows * D + kRows + idx / D] = sum; }
        }
        asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
        const uint32_t base = smem_u32(own);
        auto of = [&](int rank, int at) {
            uint32_t addr;
            float v;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(base + 4u * at), "r"(rank));
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr));
            return v;
        };
        for (int idx = split * kThreads + tid; idx < kRows * D; idx += A.splits * kThreads) {
            const int r = idx / D;
            if (r0 + r >= rows) break;
            float top = neg_inf(), sum = 0.f, x = 0.f;
            for (int k = 0; k < A.splits; ++k) top = fmaxf(top, of(k, kRows * D + r));
            const float at = top == neg_inf() ? 0.f : top;
            for (int k = 0; k < A.splits; ++k) {
                const float f = ex2(of(k, kRows * D + r) - at);
                sum += f * of(k, kRows * D + kRows + r);
                x += f * of(k, idx);
            }
            write(r, idx % D, top, sum, x);
        }
        asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");      // no block ends while another reads it
    } else {
        for (int idx = tid; idx < kRows * D; idx += kThreads) {
            const int r = idx / D, col = idx % D;
            if (r0 + r >= rows) break;
            float top, sum, x;
            of_block(r, col, top, sum, x);
            if (A.splits > 1) {
                float *part = A.part + ((((size_t)tile * a.B + b) * c.Hkv + hk) * A.splits + split) * (kRows * (D + 2)) + r * (D + 2);
                part[col] = x;
                if (col == 0) { part[D] = top; part[D + 1] = sum; }
            } else {
                write(r, col, top, sum, x);
            }
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

Split attend_split(int B, int H, int Hkv, int nq, int nk, int left, int sinks)
{
    const int tiles = (H / Hkv * nq + kRows - 1) / kRows;
    return split_of(device_sm_count(), (long long)B * Hkv * tiles, nk, (long long)(left < nk ? left : nk) + nq, sinks, kChunk, kWarps, kBlocks);
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
    const dim3 grid(A.splits * A.row_tiles, A.a.cache.Hkv, A.a.B);
    if (A.clustered) return cluster_launch(attend_kernel<D, T>, grid, kThreads, Lay<D>::TOTAL, A.splits, st, A);
    attend_kernel<D, T><<<grid, kThreads, Lay<D>::TOTAL, st>>>(A);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || A.splits == 1) return e;
    return chain_launch(join_kernel<D, T>, dim3(A.G * A.a.band.nq, A.a.cache.Hkv, A.a.B), D, 0, st, A);
}

} // namespace

size_t attend4_workspace(int dtype, int B, int H, int Hkv, int nq, int d, int nk, int left, int sinks)
{
    (void)dtype;
    const size_t tiles = (H / Hkv * nq + kRows - 1) / kRows;
    const Split s = attend_split(B, H, Hkv, nq, nk, left, sinks);
    if (s.splits == 1 || s.clustered) return 0;
    return (tiles * B * Hkv * s.splits * kRows * (d + 2) * 4 + 255) & ~(size_t)255;
}

cudaError_t launch_attend4(const Attend4 &a, cudaStream_t st)
{
    Args A;
    A.a = a;
    A.G = a.H / a.cache.Hkv;
    A.row_tiles = (A.G * a.band.nq + kRows - 1) / kRows;
    const Split s = attend_split(a.B, a.H, a.cache.Hkv, a.band.nq, a.band.nk, a.band.left, a.band.sinks);
    A.splits = s.splits;
    A.each = s.each;
    A.clustered = s.clustered;
    A.shift = -1;
    for (int i = 4; i < 29; ++i)
        if (a.cache.page_size == 1 << i) A.shift = i;
    A.part = static_cast<float *>(a.ws);
    const int d = a.cache.d;
    if (a.dtype == 0) return d == 32 ? run<32, float>(A, st) : d == 64 ? run<64, float>(A, st) : run<128, float>(A, st);
    return d == 32 ? run<32, __nv_bfloat16>(A, st) : d == 64 ? run<64, __nv_bfloat16>(A, st) : run<128, __nv_bfloat16>(A, st);
}

} // namespace window
} // namespace lot
