// Window attention backward of bf16 tensors on tcgen05.
//
// P = 2^(c S - lse2), D_i = sum_j P_ij dP_ij = <dout_i, o_i>, dS = P (dP - D): dq = scale dS K, dk = scale dS^T Q, dv = P^T dO.  Nothing is added
// by atomics: persistent launches go through two kinds of items, first
//   queries  128 queries of a head gather dq over the key tiles they see: S = Q K^T, dP = dO V^T, dq += dS K
// then
//   keys     128 keys of a key head gather dk, dv over its query heads' query tiles that see them: S^T = K Q^T, dP^T = V dO^T,
//            dv += P^T dO, dk += dS^T Q
// (eight products of a pair of tiles where one pass with sums shared by atomics or in memory takes five; with a window those sums would be
// written and read once for every key tile, several times what the other products cost).
// D~ = <dout, out> of the rounded output is off by up to 2^-8 |dout| |out|, with few visible keys as much as dS itself: the gradients had three times
// the error of their own rounding.  With any D~, sum_j P (dP - D~) = D - D~ =: e, so the queries' items sum their float32 score gradients, take
// e P K off (one more product, which e makes small) and leave the exact D to the keys' items.  For dq e is the sum of the score gradients as they
// were rounded for the product: that takes the part of their roundings' error along the keys' mean off too.
// Both kinds are the same loop: a standing pair of
// tiles X1, X2, a stream of pairs Y1, Y2, S = X1 Y1^T, dP = X2 Y2^T, weights as first operand from tensor memory: += P Y2 (queries: Y1), += dS Y1.
// Sixteen warps make the weights (a thread: a row, a quarter of the columns), one loads, one clears keys that no query sees, two issue the
// products.  P takes the columns of S that its own warps have read, dS those of dP, so the products of one and the exponentials of the other
// run side by side:
//   products   P Y2 (i), S (i+1) by one warp | dS Y1 (i), dP (i+1) by the other | ..        weights   dS (i)  | P (i+1)  | ..
// A key tile whose list is long (sinks: every later query; few key heads) is cut into parts of a fixed length, whose float32 sums
// merge_kernel adds in order.
#include "lot_chain.cuh"
#include "lot_window_tc.cuh"

#include <mutex>

namespace lot {
namespace window {
namespace {

constexpr int kThreads = 640, kMmaWarp = 16, kLoadWarp = 18, kClearWarp = 19;
constexpr float kNever = -1e30f;           // -lse2 of rows that see nothing or do not exist: their weights are zero

template <int DP> struct Plan {
    static constexpr int kXStages = DP == 64 ? 2 : 1, kYStages = DP == 64 ? 4 : 2, kStat = 2 * kTile * 4;
    static constexpr int kX = 0, kY = kXStages * 2 * kTileBytes<DP>, kYBytes = 2 * kTileBytes<DP>, kS = kY + kYStages * kYBytes, kBars = kS + kYStages * kStat;
    static constexpr int bXFull = kBars, bXEmpty = bXFull + 8 * kXStages, bYFull = bXEmpty + 8 * kXStages, bYEmpty = bYFull + 8 * kYStages,
                         bS = bYEmpty + 8 * kYStages, bDP = bS + 8, bW1 = bDP + 8, bW2 = bW1 + 8, bAcc = bW2 + 8, bClear = bAcc + 8, kAbort = bClear + 8 * kYStages, kTmem = kAbort + 8,
                         kSum = kTmem + 8, kTotal = kSum + 8 * kTile * 4;
    static constexpr int cS = 0, cDP = 128, cV = 256, cK = 256 + DP;
};

struct Args {
    Bwd a;
    CUtensorMap q, k, v, dout;
    const float *stat;                     // [B H][query tiles][2][128]: -lse2, -D
    float *part;                           // parts of key tiles: [part][2][128][DP]
    int G, qtiles, ktiles, sink_tiles;     // of a head
    FastDiv kheads, qheads, Hkv, H, group, sink_cut, key_cut;      // heads of all batch rows, of one; query heads of a key head; parts of a tile
    int sink_parts, key_parts;             // parts of a key tile with and without sinks
    int sink_items, key_items, begin, items;               // sink tiles' parts first, then the other key tiles', then the queries; this launch's: begin .. items - 1
};

struct Item {
    Row R;
    int b, h, x0, part;                    // h: key head, or query head; x0: first row of X; part: of the float32 sums, or -1
    int first, per, from, n;               // Y tiles: keys: number u = from .. from + n - 1 is head u / per, query tile first + u % per
    KeyTiles tiles;                        // queries: the key tiles
};
template <bool KEYS> __device__ __forceinline__ Item item_of(const Args &A, int i)
{
    Item it;
    const Band &B = A.a.band;
    if constexpr (KEYS) {
        const bool sink = i < A.sink_items;
        const int parts = sink ? A.sink_parts : A.key_parts, y = sink ? i : i - A.sink_items;
        int p, z;
        const int x = sink ? A.sink_cut.divmod(y, p) : A.key_cut.divmod(y, p), kt = (sink ? 0 : A.sink_tiles) + A.kheads.divmod(x, z);
        it.b = A.Hkv.divmod(z, it.h);
        it.x0 = kt * kTile;
        it.part = parts == 1 ? -1 : sink || A.sink_parts == 1 ? y : A.sink_items + y;
        it.R = row_of(B, it.b);
        // queries that see a key of the tile: positions x0 - right .. x0 + 127 + left, and all later ones where there are sinks
        const int i0 = max(it.x0 - it.R.right - it.R.pos, 0);
        const int i1 = it.x0 < it.R.sinks ? B.nq - 1 : (int)min((long long)B.nq - 1, (long long)it.x0 + kTile - 1 + it.R.left - it.R.pos);
        it.first = i0 / kTile;
        it.per = it.x0 < it.R.len && i1 >= i0 ? i1 / kTile - it.first + 1 : 0;
        const int all = it.per * A.G;
        it.from = parts == 1 ? 0 : (int)((long long)all * p / parts);
        it.n = parts == 1 ? all : (int)((long long)all * (p + 1) / parts) - it.from;
    } else {
        int x;
        it.x0 = (A.qtiles - 1 - A.qheads.divmod(i - A.sink_items - A.key_items, x)) * kTile;
        it.b = A.H.divmod(x, it.h);
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
template <bool KEYS> __device__ __forceinline__ Y stream_of(const Args &A, const Item &it, int n)
{
    if constexpr (!KEYS) return Y{it.b * A.a.Hkv + A.group.div(it.h), it.tiles.at(n) * kTile};
    const int u = it.from + n, g = A.G == 1 ? 0 : u / it.per;
    return Y{it.b * A.a.H + it.h * A.G + g, (it.first + u - g * it.per) * kTile};
}
// four numbers of shared memory; stays where it stands, so that they do not all come at once
__device__ __forceinline__ void lds2(uint32_t at, f2 &a, f2 &b) { asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(a), "=l"(b) : "r"(at)); }
// The Y tiles of all items of this block, one after the other; items without any are left out.
template <bool KEYS> struct Walk {
    Item it;
    int i, tile, count;
    __device__ __forceinline__ void begin(const Args &A)
    {
        i = A.begin + blockIdx.x;
        tile = count = 0;
        find(A);
    }
    __device__ __forceinline__ void find(const Args &A)
    {
        for (; i < A.items; i += gridDim.x) {
            it = item_of<KEYS>(A, i);
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

template <int DP, bool KEYS>
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
        for (int s = 0; s < P::kXStages; ++s) { mbar_init(sbase + P::bXFull + 8 * s, 1); mbar_init(sbase + P::bXEmpty + 8 * s, 2); }
        for (int s = 0; s < P::kYStages; ++s) { mbar_init(sbase + P::bYFull + 8 * s, 1); mbar_init(sbase + P::bYEmpty + 8 * s, 3); mbar_init(sbase + P::bClear + 8 * s, 1); }
        mbar_init(sbase + P::bS, 1);
        mbar_init(sbase + P::bDP, 1);
        mbar_init(sbase + P::bW1, 16);
        mbar_init(sbase + P::bW2, 16);
        mbar_init(sbase + P::bAcc, 2);
        abort_flag[0] = abort_flag[1] = 0;
        fence_barrier_init();
    }
    if (warp == kMmaWarp) { tmem_alloc(sbase + P::kTmem, 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // all columns are this block's, so they begin at 0, which the products' addresses take for granted
    constexpr uint32_t tmem = 0;
    if (tid == 0 && *reinterpret_cast<volatile uint32_t *>(smem + P::kTmem) != tmem) {
        *abort_flag = 1;
        atomicOr(wait.status, 4 /* LOT_DEV_TIMEOUT */);
    }
    chain_wait();                                          // the row statistics

    if (warp == kLoadWarp) {
        Walk<KEYS> w;
        uint32_t n = 0;
        for (w.begin(A); w.more(A); w.next(A), ++n) {
            const Item &it = w.it;
            if (w.tile == 0) {
                const int s = w.count % P::kXStages;
                const uint32_t turn = w.count / P::kXStages, bar = sbase + P::bXFull + 8 * s, dst = sbase + P::kX + 2 * s * TB;
                if (turn > 0 && !wait(sbase + P::bXEmpty + 8 * s, turn - 1)) break;
                if (elect_one()) {
                    mbar_arrive_expect_tx(bar, 2 * TB);
                    const int outer = it.b * (KEYS ? A.a.Hkv : A.a.H) + it.h;
                    load_tile<DP>(dst, KEYS ? &A.k : &A.q, bar, it.x0, outer);
                    load_tile<DP>(dst + TB, KEYS ? &A.v : &A.dout, bar, it.x0, outer);
                }
                __syncwarp();
            }
            const uint32_t s = n % P::kYStages, turn = n / P::kYStages, bar = sbase + P::bYFull + 8 * s, dst = sbase + P::kY + s * P::kYBytes;
            if (turn > 0 && !wait(sbase + P::bYEmpty + 8 * s, turn - 1)) break;
            const Y y = stream_of<KEYS>(A, it, w.tile);
            if (elect_one()) {
                mbar_arrive_expect_tx(bar, 2 * TB + (KEYS ? P::kStat : 0));
                load_tile<DP>(dst, KEYS ? &A.q : &A.k, bar, y.row, y.outer);
                load_tile<DP>(dst + TB, KEYS ? &A.dout : &A.v, bar, y.row, y.outer);
                if (KEYS) {
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
    } else if (warp == kClearWarp) {
        // Keys that no query of the batch row sees are multiplied by score gradients of zero: they must be numbers.  This warp passes every stage in
        // turn and gives it free like the products' warps, so that none of its waits is a whole turn ahead or behind.
        Walk<KEYS> w;
        uint32_t n = 0;
        for (w.begin(A); w.more(A); w.next(A), ++n) {
            const uint32_t s = n % P::kYStages;
            if (!wait(sbase + P::bYFull + 8 * s, n / P::kYStages)) break;
            if (!KEYS) {
                const int j0 = w.it.tiles.at(w.tile) * kTile;
                if (!all_used(w.it.R, j0)) {
                    clear_unused<DP>(smem + P::kY + s * P::kYBytes, w.it.R, j0, lane);
                    if (lane == 0) mbar_arrive(sbase + P::bClear + 8 * s);
                }
            }
            if (lane == 0) mbar_arrive(sbase + P::bYEmpty + 8 * s);
        }
    } else if (warp >= kMmaWarp) {
        const int side = warp - kMmaWarp;                  // 0: S and the products with P; 1: dP and the products with dS
        const uint32_t leader = elect_one(), tile = tmem + (side ? P::cDP : P::cS), acc = tmem + (side ? P::cK : P::cV), ready = sbase + (side ? P::bW2 : P::bW1);
        Walk<KEYS> w, ahead;
        w.begin(A);
        ahead = w;
        uint32_t g = 0, cleared = 0;                       // cleared: for each stage, whether its keys were cleared an odd number of times
        auto product = [&](uint32_t at) {                  // S or dP of the tile `ahead` stands at, number `at` of this block's
            const uint32_t x = ahead.count % P::kXStages, y = at % P::kYStages;
            if (ahead.tile == 0 && !wait(sbase + P::bXFull + 8 * x, ahead.count / P::kXStages)) return false;
            if (!wait(sbase + P::bYFull + 8 * y, at / P::kYStages)) return false;
            product_rows<DP>(leader, tile, sbase + P::kX + (2 * x + side) * TB, sbase + P::kY + y * P::kYBytes + side * TB);
            commit_to(leader, sbase + (side ? P::bDP : P::bS));
            if (ahead.last()) commit_to(leader, sbase + P::bXEmpty + 8 * x);
            return true;
        };
        bool ok = !w.more(A) || product(0);
        if (w.more(A)) ahead.next(A);
        for (; ok && w.more(A); w.next(A), ++g) {
            const uint32_t s = g % P::kYStages;
            if (!KEYS && !all_used(w.it.R, w.it.tiles.at(w.tile) * kTile)) {
                ok = wait(sbase + P::bClear + 8 * s, cleared >> s);
                if (!ok) break;
                cleared ^= 1u << s;
            }
            ok = wait(ready, g);
            if (!ok) break;
            tc_fence_after();
            product_weights<DP, 4>(leader, acc, tile, sbase + P::kY + s * P::kYBytes + (side || !KEYS ? 0 : TB), w.tile > 0);
            commit_to(leader, sbase + P::bYEmpty + 8 * s);
            if (w.last()) commit_to(leader, sbase + P::bAcc);
            if (ahead.more(A)) {
                ok = product(g + 1);
                if (!ok) break;
                ahead.next(A);
            }
        }
        if (*abort_flag) {                                 // products on their way end before tensor memory is given back
            for (int x = 0; x < 4096; ++x) (void)mbar_try_wait(sbase + P::bAcc, (w.count & 1) ^ 1);
        }
    } else {
        const int part4 = warp >> 2, row = (warp & 3) * 32 + lane, col0 = 32 * part4;
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const float c = A.a.scale * kLog2e;
        const f2 c2 = pack2(c, c);
        uint32_t g = 0, count = 0;
        bool ok = true;
        for (int i = A.begin + blockIdx.x; i < A.items; i += gridDim.x) {
            // What the loop needs of the item, and no more: registers.  This row sees the rows lo .. hi and 0 .. sk of Y; Y's tiles go up by one from yt,
            // and at wrap_at back (or on) to wrap_to.
            int left, lo, hi, sk, yt, wrap_at, wrap_to;
            float lse2 = kNever, dl = 0.f;
            {
                const Item it = item_of<KEYS>(A, i);
                const Row &R = it.R;
                left = it.n;
                if (KEYS) {
                    const int j = it.x0 + row;
                    lo = j - R.right - R.pos;
                    hi = j >= R.len ? -1 : j < R.sinks ? kFar : j + R.left - R.pos;
                    sk = -1;
                    wrap_to = it.first;
                    wrap_at = it.first + it.per;
                    yt = it.first + (it.n > 0 ? it.from % it.per : 0);
                } else {
                    const int p = R.pos + it.x0 + row;
                    lo = p - R.left;
                    hi = R.hi(p);
                    sk = min(hi, R.sinks - 1);
                    wrap_to = it.tiles.first;
                    wrap_at = it.tiles.sink;
                    yt = it.tiles.at(0);
                    if (it.n > 0) {
                        const float *st = A.stat + ((size_t)(it.b * A.a.H + it.h) * A.qtiles + it.x0 / kTile) * (2 * kTile) + row;
                        lse2 = chain_ld(st);
                        dl = chain_ld(st + kTile);
                    }
                }
            }
            const bool some = left > 0;
            const f2 l2 = pack2(lse2, lse2), d2 = pack2(dl, dl);
            float sum = 0.f, rounded = 0.f;                // queries: of this row's score gradients, and of what the products take for them
            for (; ok && left > 0; --left, ++g) {
                const int y0 = yt * kTile + col0;
                if (++yt == wrap_at) yt = wrap_to;
                const uint32_t s = g % P::kYStages;
                const uint32_t st = sbase + P::kS + s * P::kStat + 4 * col0;
                float p[32];
                ok = wait(sbase + P::bS, g);
                if (!ok) break;
                tc_fence_after();
                tmem_ld32(lanes + P::cS + col0, p);
                const uint32_t seen = bits_between(lo - y0, hi - y0) | bits_between(-y0, sk - y0);
                const bool part = __any_sync(0xffffffffu, seen != 0xffffffffu);
                if constexpr (KEYS) {
                    ok = wait(sbase + P::bYFull + 8 * s, g / P::kYStages);      // the columns' statistics
                    if (!ok) break;
                }
                settle(p);
                if constexpr (!KEYS) {
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float u, v;
                        unpack2(fma2(pack2(p[e], p[e + 1]), c2, l2), u, v);
                        p[e] = ex2(u);
                        p[e + 1] = ex2(v);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        f2 x, y;
                        float u, v;
                        lds2(st + 4 * e, x, y);
                        unpack2(fma2(pack2(p[e], p[e + 1]), c2, x), u, v);
                        p[e] = ex2(u);
                        p[e + 1] = ex2(v);
                        unpack2(fma2(pack2(p[e + 2], p[e + 3]), c2, y), u, v);
                        p[e + 2] = ex2(u);
                        p[e + 3] = ex2(v);
                    }
                }
                if (part) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) p[e] = (seen >> e) & 1u ? p[e] : 0.f;
                }
                {
                    uint32_t x[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[e] = tile::pack_bf16(p[2 * e], p[2 * e + 1]);
                    tmem_st16(lanes + P::cS + col0, x);
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(sbase + P::bW1);
                }
                ok = wait(sbase + P::bDP, g);
                if (!ok) break;
                tc_fence_after();
                // dP sixteen columns at a time, the next on their way: registers
                float dp[2][16];
                tmem_ld16(lanes + P::cDP + col0, dp[0]);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    uint32_t x[8];
                    settle(dp[k]);
                    if (k == 0) tmem_ld16(lanes + P::cDP + col0 + 16, dp[1]);
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        const int at = 16 * k + e;
                        f2 u = d2, v = d2;
                        if constexpr (KEYS) lds2(st + 4 * (kTile + at), u, v);
                        u = mul2(pack2(p[at], p[at + 1]), add2(pack2(dp[k][e], dp[k][e + 1]), u));
                        v = mul2(pack2(p[at + 2], p[at + 3]), add2(pack2(dp[k][e + 2], dp[k][e + 3]), v));
                        unpack2(u, p[at], p[at + 1]);
                        unpack2(v, p[at + 2], p[at + 3]);
                    }
                    if (part) {                        // not a product with what may be no number
#pragma unroll
                        for (int e = 16 * k; e < 16 * k + 16; ++e) p[e] = (seen >> e) & 1u ? p[e] : 0.f;
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        x[e] = tile::pack_bf16(p[16 * k + 2 * e], p[16 * k + 2 * e + 1]);
                        if (!KEYS) {
                            sum += p[16 * k + 2 * e] + p[16 * k + 2 * e + 1];
                            rounded += __uint_as_float(x[e] << 16) + __uint_as_float(x[e] & 0xffff0000u);
                        }
                    }
                    tmem_st8(lanes + P::cDP + col0 + 8 * k, x);
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(sbase + P::bW2);
            }
            if (ok && some) {
                ok = wait(sbase + P::bAcc, count++);
                tc_fence_after();
            }
            int again = i;
            asm volatile("" : "+r"(again));                // not kept over the loop
            const Item it = item_of<KEYS>(A, again);
            const int r = it.x0 + row, d = A.a.d, rows = KEYS ? A.a.band.nk : A.a.band.nq;
            const size_t at = (size_t)(it.b * (KEYS ? A.a.Hkv : A.a.H) + it.h) * rows + r;
            float e_row = 0.f;
            if (!KEYS && some) {
                float *sums = reinterpret_cast<float *>(smem + P::kSum);
                sums[part4 * kTile + row] = sum;
                sums[(4 + part4) * kTile + row] = rounded;
                named_bar_sync(1, 512);
                if (part4 == 0)
                    const_cast<float *>(A.stat)[((size_t)(it.b * A.a.H + it.h) * A.qtiles + it.x0 / kTile) * (2 * kTile) + kTile + row] =
                        dl - ((sums[row] + sums[kTile + row]) + (sums[2 * kTile + row] + sums[3 * kTile + row]));
                sums += 4 * kTile;
                e_row = (sums[row] + sums[kTile + row]) + (sums[2 * kTile + row] + sums[3 * kTile + row]);
            }
            // sixteen channels at a time: keys: eight warps dv, the others dk; queries: dq
            const float nan = __int_as_float(0x7fc00000);
#pragma unroll 1
            for (int n = part4; n < (KEYS ? 2 : 1) * (DP / 16); n += 4) {
                const int which = KEYS ? n / (DP / 16) : 1, col = n % (DP / 16) * 16;              // 0: dv, 1: dk or dq
                const float f = !ok ? nan : which ? A.a.scale : 1.f;
                float x[16];
                if (some) {
                    tmem_ld16(lanes + (which ? P::cK : P::cV) + col, x);
                    settle(x);
                    if (!KEYS) {
                        float y[16];
                        tmem_ld16(lanes + P::cV + col, y);
                        settle(y);
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[e] = fmaf(-e_row, y[e], x[e]);
                    }
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] = some || !ok ? x[e] * f : 0.f;
                if (it.part >= 0) {
                    float *part = A.part + ((size_t)it.part * 2 + which) * (kTile * DP) + (size_t)row * DP;
#pragma unroll
                    for (int e = 0; e < 16; e += 4) *reinterpret_cast<float4 *>(part + col + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
                } else if (r < rows) {
                    store_row(static_cast<__nv_bfloat16 *>(KEYS ? (which ? A.a.dk : A.a.dv) : A.a.dq) + at * d, col, d, x);
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

// -lse2 and -D of every row, in tiles of 128 (rows beyond the last: weights of zero).  LANES threads a row, eight channels each.
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
        o[0] = none ? kNever : -l * kLog2e;
        o[kTile] = none ? 0.f : -s;
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

template <int DP, bool KEYS> cudaError_t launch_kind(Args A, int begin, int end, cudaStream_t st)
{
    static std::mutex mu;
    static bool set[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!set[dev]) {
            const cudaError_t e = cudaFuncSetAttribute(bwd_tc_kernel<DP, KEYS>, cudaFuncAttributeMaxDynamicSharedMemorySize, Plan<DP>::kTotal);
            if (e != cudaSuccess) return e;
            set[dev] = true;
        }
    }
    if (begin == end) return cudaSuccess;
    A.begin = begin;
    A.items = end;
    const int sms = device_sm_count();
    return chain_launch(bwd_tc_kernel<DP, KEYS>, dim3(end - begin < sms ? end - begin : sms), kThreads, Plan<DP>::kTotal, st, A);
}

template <int DP> cudaError_t launch_t(const Args &A, bool merge, cudaStream_t st)
{
    const long long rows = (long long)A.a.B * A.a.H * A.qtiles * kTile;
    cudaError_t e = cudaSuccess;
    if (rows > 0) {
        stat_kernel<DP / 8><<<(unsigned)(rows * (DP / 8) / 256), 256, 0, st>>>(static_cast<const __nv_bfloat16 *>(A.a.out), static_cast<const __nv_bfloat16 *>(A.a.dout),
                                                                              A.a.lse, const_cast<float *>(A.stat), A.a.band.nq, A.qtiles, A.a.d);
        e = cudaGetLastError();
    }
    const int keys = A.sink_items + A.key_items;
    if (e == cudaSuccess) e = launch_kind<DP, false>(A, keys, A.items, st);
    if (e == cudaSuccess) e = launch_kind<DP, true>(A, 0, keys, st);
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
    A.kheads = fast_div(a.B * a.Hkv);
    A.qheads = fast_div(a.B * a.H);
    A.Hkv = fast_div(a.Hkv);
    A.H = fast_div(a.H);
    A.group = fast_div(A.G);
    A.sink_cut = fast_div(c.sink_parts);
    A.key_cut = fast_div(c.key_parts);
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
