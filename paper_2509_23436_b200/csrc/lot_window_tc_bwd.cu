// Window attention backward of bf16 tensors on tcgen05.
//
// P = 2^(c S - lse2), D_i = <dout_i, out_i>, dS = P (dP - D): dq = scale dS K, dk = scale dS^T Q, dv = P^T dO.  Nothing is added by atomics:
// one persistent launch goes through two kinds of items,
//   queries  128 queries of a head gather dq over the key tiles they see: S = Q K^T, dP = dO V^T, dq += dS K
//   keys     128 keys of a key head gather dk, dv over its query heads' query tiles that see them: S^T = K Q^T, dP^T = V dO^T,
//            dv += P^T dO, dk += dS^T Q
// (seven products of a pair of tiles where one pass with sums shared by atomics or in memory takes five; with a window those sums would be
// written and read once for every key tile, several times what the two products cost).  Both kinds are the same loop: a standing pair of
// tiles X1, X2, a stream of pairs Y1, Y2, S = X1 Y1^T, dP = X2 Y2^T, weights as first operand from tensor memory: [+= P Y2], += dS Y1.
// Eight warps make the weights (a thread: a row, half the columns), one loads, one issues the products.  P takes the columns of S that its
// own warps have read, dS those of dP, so the products of one and the exponentials of the other run side by side:
//   products   P Y2 (i), S (i+1) | dS Y1 (i), dP (i+1) | ..        weights   dS (i)         | P (i+1)          | ..
// A key tile whose list is long (sinks: every later query; few key heads) is cut into parts of a fixed length, whose float32 sums
// merge_kernel adds in order.
#include "lot_chain.cuh"
#include "lot_window_tc.cuh"

#include <mutex>

namespace lot {
namespace window {
namespace {

constexpr int kThreads = 320, kMmaWarp = 8, kLoadWarp = 9;
constexpr float kNever = 1e30f;            // lse2 of rows that see nothing or do not exist: their weights are zero

template <int DP> struct Plan {
    static constexpr int kXStages = DP == 64 ? 2 : 1, kYStages = DP == 64 ? 4 : 2, kStat = 2 * kTile * 4;
    static constexpr int kX = 0, kY = kXStages * 2 * kTileBytes<DP>, kYBytes = 2 * kTileBytes<DP>, kS = kY + kYStages * kYBytes, kBars = kS + kYStages * kStat;
    static constexpr int bXFull = kBars, bXEmpty = bXFull + 8 * kXStages, bYFull = bXEmpty + 8 * kXStages, bYEmpty = bYFull + 8 * kYStages,
                         bS = bYEmpty + 8 * kYStages, bDP = bS + 8, bW1 = bDP + 8, bW2 = bW1 + 8, bAcc = bW2 + 8, kAbort = bAcc + 8, kTmem = kAbort + 8,
                         kTotal = kTmem + 8;
    static constexpr int cS = 0, cDP = 128, cV = 256, cK = 256 + DP;
};

struct Args {
    Bwd a;
    CUtensorMap q, k, v, dout;
    const float *stat;                     // [B H][query tiles][2][128]: lse2, D
    float *part;                           // parts of key tiles: [part][2][128][DP]
    int G, qtiles, ktiles, sink_tiles;     // of a head
    int sink_parts, key_parts;             // parts of a key tile with and without sinks
    int sink_items, key_items, items;      // sink tiles' parts first, then the other key tiles', then the queries
};

struct Item {
    Row R;
    bool keys;                             // which kind
    int b, h, x0, part;                    // h: key head, or query head; x0: first row of X; part: of the float32 sums, or -1
    int first, per, from, n;               // Y tiles: keys: number u = from .. from + n - 1 is head u / per, query tile first + u % per
    KeyTiles tiles;                        // queries: the key tiles
};
__device__ __forceinline__ Item item_of(const Args &A, int i)
{
    Item it;
    const Band &B = A.a.band;
    if (i < A.sink_items + A.key_items) {
        it.keys = true;
        const bool sink = i < A.sink_items;
        const int parts = sink ? A.sink_parts : A.key_parts, y = sink ? i : i - A.sink_items, heads = A.a.B * A.a.Hkv, p = y % parts, x = y / parts;
        const int kt = (sink ? 0 : A.sink_tiles) + x / heads;
        it.b = x % heads / A.a.Hkv;
        it.h = x % heads % A.a.Hkv;
        it.x0 = kt * kTile;
        it.part = parts == 1 ? -1 : sink || A.sink_parts == 1 ? y : A.sink_items + y;
        it.R = row_of(B, it.b);
        // queries that see a key of the tile: positions x0 - right .. x0 + 127 + left, and all later ones where there are sinks
        const int i0 = max(it.x0 - it.R.right - it.R.pos, 0);
        const int i1 = it.x0 < it.R.sinks ? B.nq - 1 : (int)min((long long)B.nq - 1, (long long)it.x0 + kTile - 1 + it.R.left - it.R.pos);
        it.first = i0 / kTile;
        it.per = it.x0 < it.R.len && i1 >= i0 ? i1 / kTile - it.first + 1 : 0;
        const int all = it.per * A.G;
        it.from = (int)((long long)all * p / parts);
        it.n = (int)((long long)all * (p + 1) / parts) - it.from;
    } else {
        it.keys = false;
        const int y = i - A.sink_items - A.key_items, heads = A.a.B * A.a.H, x = y % heads;
        it.b = x / A.a.H;
        it.h = x % A.a.H;
        it.x0 = (A.qtiles - 1 - y / heads) * kTile;
        it.part = -1;
        it.R = row_of(B, it.b);
        it.tiles = key_tiles(it.R, it.R.pos + it.x0, it.R.pos + min(it.x0 + kTile, B.nq) - 1);
        it.n = it.tiles.n;
    }
    return it;
}
struct Y {
    int outer, row;                        // head (of all batch rows') and first row
};
__device__ __forceinline__ Y stream_of(const Args &A, const Item &it, int n)
{
    if (!it.keys) return Y{it.b * A.a.Hkv + it.h / A.G, it.tiles.at(n) * kTile};
    const int u = it.from + n;
    return Y{it.b * A.a.H + it.h * A.G + u / it.per, (it.first + u % it.per) * kTile};
}
// The Y tiles of all items of this block, one after the other; items without any are left out.
struct Walk {
    Item it;
    int i, tile, count;
    __device__ __forceinline__ void begin(const Args &A)
    {
        i = blockIdx.x;
        tile = count = 0;
        find(A);
    }
    __device__ __forceinline__ void find(const Args &A)
    {
        for (; i < A.items; i += gridDim.x) {
            it = item_of(A, i);
            if (it.n > 0) return;
        }
    }
    __device__ __forceinline__ bool more(const Args &A) const { return i < A.items; }
    __device__ __forceinline__ bool last() const { return tile == it.n - 1; }
    __device__ __forceinline__ void next(const Args &A)
    {
        if (++tile < it.n) return;
        tile = 0;
        ++count;
        i += gridDim.x;
        find(A);
    }
};

// D (128 x DP) += W Y: the weights' columns 0 .. 63 at w, 64 .. 127 at w + 64 (each in what its warps had read)
template <int DP> __device__ __forceinline__ void product_halves(uint32_t d, uint32_t w, uint32_t y, bool accumulate)
{
    constexpr uint32_t idesc = make_idesc_bf16(128, DP, 0, 1);
    const uint64_t dy = make_smem_desc(y, kTile * 128, 1024);
#pragma unroll
    for (int ks = 0; ks < kTile / 16; ++ks) umma_bf16_ts(d, w + (ks >> 2) * 64 + (ks & 3) * 8, dy + ks * 128, idesc, accumulate || ks != 0);
}

template <int DP>
__global__ void __launch_bounds__(kThreads, 1) bwd_tc_kernel(const __grid_constant__ Args A)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    using P = Plan<DP>;
    constexpr int TB = kTileBytes<DP>;
    const uint32_t sbase = smem_u32(smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + P::kAbort);
    const Waits wait{abort_flag, A.a.status != nullptr ? A.a.status : reinterpret_cast<int *>(smem + P::kAbort + 4)};
    if (tid == 0) {
        for (int s = 0; s < P::kXStages; ++s) { mbar_init(sbase + P::bXFull + 8 * s, 1); mbar_init(sbase + P::bXEmpty + 8 * s, 1); }
        for (int s = 0; s < P::kYStages; ++s) { mbar_init(sbase + P::bYFull + 8 * s, 1); mbar_init(sbase + P::bYEmpty + 8 * s, 1); }
        mbar_init(sbase + P::bS, 1);
        mbar_init(sbase + P::bDP, 1);
        mbar_init(sbase + P::bW1, 8);
        mbar_init(sbase + P::bW2, 8);
        mbar_init(sbase + P::bAcc, 1);
        abort_flag[0] = abort_flag[1] = 0;
        fence_barrier_init();
    }
    if (warp == kMmaWarp) { tmem_alloc(sbase + P::kTmem, 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(smem + P::kTmem);
    chain_wait();                                          // the row statistics

    if (warp == kLoadWarp) {
        Walk w;
        uint32_t n = 0;
        for (w.begin(A); w.more(A); w.next(A), ++n) {
            const Item &it = w.it;
            if (w.tile == 0) {
                const int s = w.count % P::kXStages;
                const uint32_t turn = w.count / P::kXStages, bar = sbase + P::bXFull + 8 * s, dst = sbase + P::kX + 2 * s * TB;
                if (turn > 0 && !wait(sbase + P::bXEmpty + 8 * s, turn - 1)) break;
                if (elect_one()) {
                    mbar_arrive_expect_tx(bar, 2 * TB);
                    const int outer = it.b * (it.keys ? A.a.Hkv : A.a.H) + it.h;
                    load_tile<DP>(dst, it.keys ? &A.k : &A.q, bar, it.x0, outer);
                    load_tile<DP>(dst + TB, it.keys ? &A.v : &A.dout, bar, it.x0, outer);
                }
                __syncwarp();
            }
            const uint32_t s = n % P::kYStages, turn = n / P::kYStages, bar = sbase + P::bYFull + 8 * s, dst = sbase + P::kY + s * P::kYBytes;
            if (turn > 0 && !wait(sbase + P::bYEmpty + 8 * s, turn - 1)) break;
            const Y y = stream_of(A, it, w.tile);
            if (elect_one()) {
                mbar_arrive_expect_tx(bar, 2 * TB + (it.keys ? P::kStat : 0));
                load_tile<DP>(dst, it.keys ? &A.q : &A.k, bar, y.row, y.outer);
                load_tile<DP>(dst + TB, it.keys ? &A.dout : &A.v, bar, y.row, y.outer);
                if (it.keys) {
                    const float *st = A.stat + ((size_t)y.outer * A.qtiles + y.row / kTile) * (2 * kTile);
                    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                                 ::"r"(sbase + P::kS + s * P::kStat), "l"(st), "r"(P::kStat), "r"(bar) : "memory");
                }
            }
            __syncwarp();
        }
        if (*abort_flag) {                                 // copies still on their way land before the block ends
            for (uint32_t u = n > P::kYStages ? n - P::kYStages : 0; u < n; ++u)
                for (int x = 0; x < 4096 && !mbar_try_wait(sbase + P::bYFull + 8 * (u % P::kYStages), (u / P::kYStages) & 1); ++x) {}
        }
    } else if (warp == kMmaWarp) {
        Walk w, ahead;
        w.begin(A);
        ahead = w;
        uint32_t g = 0;
        bool ok = true;
        auto operands = [&](uint32_t at) {                 // X and Y of the tile `ahead` stands at, number `at` of this block's
            if (ahead.tile == 0 && !wait(sbase + P::bXFull + 8 * (ahead.count % P::kXStages), ahead.count / P::kXStages)) return false;
            const uint32_t s = at % P::kYStages;
            if (!wait(sbase + P::bYFull + 8 * s, at / P::kYStages)) return false;
            if (!ahead.it.keys) {                          // keys that no query sees are multiplied by zero: they must be numbers
                const int j0 = ahead.it.tiles.at(ahead.tile) * kTile;
                if (!all_used(ahead.it.R, j0)) clear_unused<DP>(smem + P::kY + s * P::kYBytes, ahead.it.R, j0, lane);
            }
            return true;
        };
        auto product = [&](uint32_t at, int side) {        // S (side 0) or dP (1) of that tile
            if (elect_one()) {
                product_rows<DP>(tmem + (side ? P::cDP : P::cS), sbase + P::kX + (2 * (ahead.count % P::kXStages) + side) * TB,
                                 sbase + P::kY + (at % P::kYStages) * P::kYBytes + side * TB);
                umma_commit(sbase + (side ? P::bDP : P::bS));
                if (side && ahead.last()) umma_commit(sbase + P::bXEmpty + 8 * (ahead.count % P::kXStages));
            }
            __syncwarp();
        };
        if (w.more(A)) {
            ok = operands(0);
            if (ok) { product(0, 0); product(0, 1); ahead.next(A); }
        }
        for (; ok && w.more(A); w.next(A), ++g) {
            const bool follow = ahead.more(A);
            const uint32_t y = sbase + P::kY + (g % P::kYStages) * P::kYBytes;
            ok = wait(sbase + P::bW1, g);
            if (!ok) break;
            tc_fence_after();
            if (w.it.keys) {
                if (elect_one()) product_halves<DP>(tmem + P::cV, tmem + P::cS, y + TB, w.tile > 0);
                __syncwarp();
            }
            if (follow) {
                ok = operands(g + 1);
                if (!ok) break;
                product(g + 1, 0);
            }
            ok = wait(sbase + P::bW2, g);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
                product_halves<DP>(tmem + P::cK, tmem + P::cDP, y, w.tile > 0);
                umma_commit(sbase + P::bYEmpty + 8 * (g % P::kYStages));
                if (w.last()) umma_commit(sbase + P::bAcc);
            }
            __syncwarp();
            if (follow) {
                product(g + 1, 1);
                ahead.next(A);
            }
        }
        if (*abort_flag) {                                 // products on their way end before tensor memory is given back
            for (int x = 0; x < 4096; ++x) (void)mbar_try_wait(sbase + P::bAcc, (w.count & 1) ^ 1);
        }
    } else {
        const int half = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const float c = A.a.scale * kLog2e;
        uint32_t g = 0, count = 0;
        bool ok = true;
        for (int i = blockIdx.x; i < A.items; i += gridDim.x) {
            const Item it = item_of(A, i);
            const Row &R = it.R;
            float lse2 = kNever, dl = 0.f;
            if (!it.keys && it.n > 0) {
                const float *st = A.stat + ((size_t)(it.b * A.a.H + it.h) * A.qtiles + it.x0 / kTile) * (2 * kTile) + row;
                lse2 = chain_ld(st);
                dl = chain_ld(st + kTile);
            }
            for (int n = 0; ok && n < it.n; ++n, ++g) {
                const Y y = stream_of(A, it, n);
                const uint32_t s = g % P::kYStages;
                const float *st = reinterpret_cast<const float *>(smem + P::kS + s * P::kStat) + 64 * half;
                float p[2][32];
                ok = wait(sbase + P::bS, g);
                if (!ok) break;
                tc_fence_after();
                tmem_ld32(lanes + P::cS + 64 * half, p[0]);
                tmem_ld32(lanes + P::cS + 64 * half + 32, p[1]);
                uint32_t seen[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int y0 = y.row + 64 * half + 32 * k;
                    seen[k] = it.keys ? seeing(R, R.pos + y0, it.x0 + row) : seen_keys(R, R.pos + it.x0 + row, y0);
                }
                if (it.keys) {
                    ok = wait(sbase + P::bYFull + 8 * s, g / P::kYStages);      // the columns' statistics
                    if (!ok) break;
                }
                settle(p[0]);
                settle(p[1]);
                tc_fence_before();
                __syncwarp();
                if (!it.keys && lane == 0) mbar_arrive(sbase + P::bW1);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if (it.keys) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            const float4 x = *reinterpret_cast<const float4 *>(st + 32 * k + e);
                            p[k][e] = ex2(fmaf(p[k][e], c, -x.x));
                            p[k][e + 1] = ex2(fmaf(p[k][e + 1], c, -x.y));
                            p[k][e + 2] = ex2(fmaf(p[k][e + 2], c, -x.z));
                            p[k][e + 3] = ex2(fmaf(p[k][e + 3], c, -x.w));
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) p[k][e] = ex2(fmaf(p[k][e], c, -lse2));
                    }
                    if (__any_sync(0xffffffffu, seen[k] != 0xffffffffu)) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) p[k][e] = (seen[k] >> e) & 1u ? p[k][e] : 0.f;
                    }
                    if (it.keys) {
                        uint32_t x[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[e] = tile::pack_bf16(p[k][2 * e], p[k][2 * e + 1]);
                        tmem_st16(lanes + P::cS + 64 * half + 16 * k, x);
                    }
                }
                if (it.keys) {
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(sbase + P::bW1);
                }
                ok = wait(sbase + P::bDP, g);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float dp[32];
                    uint32_t x[16];
                    tmem_ld32(lanes + P::cDP + 64 * half + 32 * k, dp);
                    settle(dp);
                    if (it.keys) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            const float4 z = *reinterpret_cast<const float4 *>(st + kTile + 32 * k + e);
                            p[k][e] *= dp[e] - z.x;
                            p[k][e + 1] *= dp[e + 1] - z.y;
                            p[k][e + 2] *= dp[e + 2] - z.z;
                            p[k][e + 3] *= dp[e + 3] - z.w;
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) p[k][e] *= dp[e] - dl;
                    }
                    if (__any_sync(0xffffffffu, seen[k] != 0xffffffffu)) {      // not a product with what may be no number
#pragma unroll
                        for (int e = 0; e < 32; ++e) p[k][e] = (seen[k] >> e) & 1u ? p[k][e] : 0.f;
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[e] = tile::pack_bf16(p[k][2 * e], p[k][2 * e + 1]);
                    tmem_st16(lanes + P::cDP + 64 * half + 16 * k, x);
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(sbase + P::bW2);
            }
            if (ok && it.n > 0) {
                ok = wait(sbase + P::bAcc, count++);
                tc_fence_after();
            }
            // keys: the first four warps have dv, the others dk; queries: half of dq's channels each
            const float nan = __int_as_float(0x7fc00000), f = !ok ? nan : it.keys && half == 0 ? 1.f : A.a.scale;
            const int r = it.x0 + row, d = A.a.d, rows = it.keys ? A.a.band.nk : A.a.band.nq;
            const size_t at = (size_t)(it.b * (it.keys ? A.a.Hkv : A.a.H) + it.h) * rows + r;
            __nv_bfloat16 *out = static_cast<__nv_bfloat16 *>(it.keys ? (half ? A.a.dk : A.a.dv) : A.a.dq) + at * d;
            float *part = A.part + ((size_t)max(it.part, 0) * 2 + half) * (kTile * DP) + (size_t)row * DP;
            const int from = it.keys ? 0 : half * (DP / 2), to = it.keys ? DP : from + DP / 2, acc = it.keys && half == 0 ? P::cV : P::cK;
            for (int col = from; col < to; col += 32) {
                float x[32];
                if (it.n > 0) {
                    tmem_ld32(lanes + acc + col, x);
                    settle(x);
                }
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] = it.n > 0 || !ok ? x[e] * f : 0.f;
                if (it.part >= 0) {
#pragma unroll
                    for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4 *>(part + col + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
                } else if (r < rows) {
                    store_row32(out, col, d, x);
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    chain_next();
    if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
}

// lse2 and D of every row, in tiles of 128 (rows beyond the last: weights of zero).  LANES threads a row, eight channels each.
template <int LANES>
__global__ void __launch_bounds__(256) stat_kernel(const __nv_bfloat16 *out, const __nv_bfloat16 *dout, const float *lse, float *stat, int nq, int tiles, int d)
{
    chain_next();
    const long long x = ((long long)blockIdx.x * 256 + threadIdx.x) / LANES, head = x / (tiles * kTile);
    const int r = (int)(x % (tiles * kTile)), c = (threadIdx.x % LANES) * 8;
    float s = 0.f, l = neg_inf();
    if (r < nq) {
        const size_t row = (size_t)head * nq + r;
        if (c < d) {
            const uint4 a = *reinterpret_cast<const uint4 *>(out + row * d + c), b = *reinterpret_cast<const uint4 *>(dout + row * d + c);
            const uint32_t u[4] = {a.x, a.y, a.z, a.w}, v[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 p = tile::unpack_bf16(u[e]), q = tile::unpack_bf16(v[e]);
                s = fmaf(p.x, q.x, fmaf(p.y, q.y, s));
            }
        }
        l = lse[row];
    }
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (threadIdx.x % LANES == 0) {
        float *o = stat + ((size_t)head * tiles + r / kTile) * (2 * kTile) + r % kTile;
        const bool none = l == neg_inf();
        o[0] = none ? kNever : l * kLog2e;
        o[kTile] = none ? 0.f : s;
    }
    chain_wait();
}

// dk and dv of key tiles that came in parts: a block a tile's quarter (32 rows) and side
template <int DP>
__global__ void __launch_bounds__(256) merge_kernel(const __grid_constant__ Args A)
{
    const int heads = A.a.B * A.a.Hkv, sink_work = A.sink_parts > 1 ? A.sink_tiles * heads : 0, x = blockIdx.x, quarter = blockIdx.y & 3, side = blockIdx.y >> 2;
    const bool sink = x < sink_work;
    const int parts = sink ? A.sink_parts : A.key_parts, y = sink ? x : x - sink_work;
    const int first = sink ? y * parts : (A.sink_parts > 1 ? A.sink_items : 0) + y * parts;
    const int kt = (sink ? 0 : A.sink_tiles) + y / heads, head = y % heads;
    chain_wait();
    for (int idx = threadIdx.x; idx < 32 * (DP / 4); idx += 256) {
        const int r = quarter * 32 + idx / (DP / 4), c = idx % (DP / 4) * 4, row = kt * kTile + r;
        if (row >= A.a.band.nk || c >= A.a.d) continue;
        float o[4] = {0.f, 0.f, 0.f, 0.f};
        for (int p = 0; p < parts; ++p) {
            const float4 z = chain_ld4(A.part + ((size_t)(first + p) * 2 + side) * (kTile * DP) + (size_t)r * DP + c);
            o[0] += z.x; o[1] += z.y; o[2] += z.z; o[3] += z.w;
        }
        store4(static_cast<__nv_bfloat16 *>(side ? A.a.dk : A.a.dv) + ((size_t)head * A.a.band.nk + row) * A.a.d + c, o);
    }
}

// How key tiles are cut: no part longer than a third of a block's share of all the work, or 16 tiles.
struct Cut {
    int qtiles, ktiles, sink_tiles, sink_parts, key_parts;
    long long parts;                       // whose sums are kept
};
Cut cut_of(int B, int H, int Hkv, int nq, int nk, int left, int right, int sinks)
{
    Cut c;
    c.qtiles = (nq + kTile - 1) / kTile;
    c.ktiles = (nk + kTile - 1) / kTile;
    if (sinks > nk) sinks = nk;
    c.sink_tiles = (sinks + kTile - 1) / kTile;
    const long long G = H / Hkv, heads = (long long)B * Hkv, span = ((long long)left + right + kTile - 1) / kTile + 2;
    const long long sink_len = G * c.qtiles, key_len = G * (span < c.qtiles ? span : c.qtiles);
    const long long all = heads * (c.sink_tiles * sink_len + (c.ktiles - c.sink_tiles) * key_len), share = all / (3ll * device_sm_count());
    const long long most = share > 16 ? share : 16;
    c.sink_parts = c.sink_tiles > 0 ? (int)((sink_len + most - 1) / most) : 1;
    c.key_parts = (int)((key_len + most - 1) / most);
    if (c.sink_parts < 1) c.sink_parts = 1;
    if (c.key_parts < 1) c.key_parts = 1;
    c.parts = heads * ((c.sink_parts > 1 ? (long long)c.sink_tiles * c.sink_parts : 0) + (c.key_parts > 1 ? (long long)(c.ktiles - c.sink_tiles) * c.key_parts : 0));
    return c;
}
inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
size_t stat_bytes(int B, int H, int qtiles) { return up256((size_t)B * H * qtiles * 2 * kTile * 4); }

template <int DP> cudaError_t launch_t(const Args &A, bool merge, cudaStream_t st)
{
    static std::mutex mu;
    static bool set[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!set[dev]) {
            const cudaError_t e = cudaFuncSetAttribute(bwd_tc_kernel<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, Plan<DP>::kTotal);
            if (e != cudaSuccess) return e;
            set[dev] = true;
        }
    }
    const long long rows = (long long)A.a.B * A.a.H * A.qtiles * kTile;
    cudaError_t e = cudaSuccess;
    if (rows > 0) {
        stat_kernel<DP / 8><<<(unsigned)(rows * (DP / 8) / 256), 256, 0, st>>>(static_cast<const __nv_bfloat16 *>(A.a.out), static_cast<const __nv_bfloat16 *>(A.a.dout),
                                                                              A.a.lse, const_cast<float *>(A.stat), A.a.band.nq, A.qtiles, A.a.d);
        e = cudaGetLastError();
    }
    const int sms = device_sm_count();
    if (e == cudaSuccess) e = chain_launch(bwd_tc_kernel<DP>, dim3(A.items < sms ? A.items : sms), kThreads, Plan<DP>::kTotal, st, A);
    if (e != cudaSuccess || !merge) return e;
    const int heads = A.a.B * A.a.Hkv;
    const int work = (A.sink_parts > 1 ? A.sink_tiles * heads : 0) + (A.key_parts > 1 ? (A.ktiles - A.sink_tiles) * heads : 0);
    return chain_launch(merge_kernel<DP>, dim3(work, 8), 256, 0, st, A);
}

} // namespace

size_t bwd_tc_workspace(int B, int H, int Hkv, int nq, int nk, int d, int left, int right, int sinks)
{
    const Cut c = cut_of(B, H, Hkv, nq, nk, left, right, sinks);
    return stat_bytes(B, H, c.qtiles) + up256((size_t)c.parts * 2 * kTile * (d <= 64 ? 64 : 128) * 4);
}

cudaError_t launch_bwd_tc(const Bwd &a, cudaStream_t st)
{
    const Cut c = cut_of(a.B, a.H, a.Hkv, a.band.nq, a.band.nk, a.band.left, a.band.right, a.band.sinks);
    Args A;
    A.a = a;
    A.G = a.H / a.Hkv;
    A.qtiles = c.qtiles;
    A.ktiles = c.ktiles;
    A.sink_tiles = c.sink_tiles;
    A.sink_parts = c.sink_parts;
    A.key_parts = c.key_parts;
    A.sink_items = a.B * a.Hkv * c.sink_tiles * c.sink_parts;
    A.key_items = a.B * a.Hkv * (c.ktiles - c.sink_tiles) * c.key_parts;
    A.items = A.sink_items + A.key_items + a.B * a.H * c.qtiles;
    A.stat = a.delta;
    A.part = reinterpret_cast<float *>(reinterpret_cast<char *>(a.delta) + stat_bytes(a.B, a.H, c.qtiles));
    const void *any = a.band.nq > 0 ? a.q : a.k;           // without queries or keys no item has tiles
    const int rows = a.band.nq > 0 ? a.band.nq : a.band.nk;
    const long long outer = (long long)a.B * (a.band.nq > 0 ? a.H : a.Hkv);
    if (!make_tile_map(&A.q, any, outer, rows, a.d)) return cudaErrorInvalidValue;
    A.k = A.v = A.dout = A.q;
    if (a.band.nq > 0 && !make_tile_map(&A.dout, a.dout, outer, rows, a.d)) return cudaErrorInvalidValue;
    if (a.band.nk > 0 && (!make_tile_map(&A.k, a.k, (long long)a.B * a.Hkv, a.band.nk, a.d) || !make_tile_map(&A.v, a.v, (long long)a.B * a.Hkv, a.band.nk, a.d)))
        return cudaErrorInvalidValue;
    return a.d <= 64 ? launch_t<64>(A, c.parts > 0, st) : launch_t<128>(A, c.parts > 0, st);
}

} // namespace window
} // namespace lot
