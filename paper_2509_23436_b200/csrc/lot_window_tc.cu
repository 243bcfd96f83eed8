// Window attention forward of bf16 tensors on tcgen05.
//
// A persistent block per SM goes through items of two 128-query tiles that read the same keys: two query heads of a key head, or two
// neighbouring tiles of one head.  Roles: two groups of eight softmax warps (one a query tile; a warp 16 rows, whose 128 columns lie in lane quads),
// for each group a warp that issues its products (one for both was busy all the time), a warp that loads tiles (TMA) and one that clears
// values no query sees.  For each 128-key tile
//   S = Q K^T in tensor memory -> the group's rows: maximum, exponentials, sum -> P (bf16) back into tensor memory, where it is the first
//   operand of O += P V -> O stays in tensor memory over the item's tiles.
// The running maximum moves only when a score passes it by 2^8 (weights up to 2^8 lose nothing in float32 sums or bf16 weights), so O is
// hardly ever rescaled, and the quads' maxima need not be joined to see that nothing passes it.
// Bound by the exponentials (16 a clock and SM: 2048 clocks for both tiles) and, at 128 channels, as much by the products.  With eight softmax warps (a thread a
// row) a warp's waits, loads and loop around 2000 clocks of exponentials took as long again: two warps a scheduler did not hide them.
// Key tiles outside a block's window are never visited, 64-column halves outside a warp's never worked on.
#include "lot_chain.cuh"
#include "lot_window_tc.cuh"

#include <mutex>

namespace lot {
namespace window {
namespace {

constexpr int kThreads = 640, kMmaWarp = 16, kLoadWarp = 18, kClearWarp = 19, kGroup8 = 256;
constexpr float kLift = 8.f;

template <int DP> struct Plan {
    static constexpr bool kApart = DP == 64;               // P has columns of its own: the next S may be written while P is made
    static constexpr int kQStages = DP == 64 ? 2 : 1, kSlots = DP == 64 ? 8 : 4;
    static constexpr int kQ = 0, kKV = kQStages * 2 * kTileBytes<DP>, kBars = kKV + kSlots * kTileBytes<DP>;
    // q_full, q_empty [stages]; kv_full, kv_empty [slots]; s_full, s_free, p_full, o_done [2]; clear [slots]
    static constexpr int bQFull = kBars, bQEmpty = bQFull + 8 * kQStages, bFull = bQEmpty + 8 * kQStages, bEmpty = bFull + 8 * kSlots, bS = bEmpty + 8 * kSlots,
                         bSFree = bS + 16, bP = bSFree + 16, bO = bP + 16, bClear = bO + 16, kAbort = bClear + 8 * kSlots, kTmem = kAbort + 8, kInv = kTmem + 8, kTotal = kInv + 2 * kTile * 4;
    static constexpr int cS = 0, cP = kApart ? 128 : 0, cO = kApart ? 192 : 128, kCols = 256;      // columns of a tile's half of tensor memory
};

struct Args {
    Fwd a;
    CUtensorMap q, k, v;
    int paired, steps, items;                              // paired: two heads of a key head; steps: items of a head or pair
    FastDiv per, heads, group;                             // items of a step; heads or pairs of a batch row; query heads of a key head
};

struct Item {
    Row R;
    int b, h0, row0, hk, hstep, rstep;                     // head and first query of the two tiles
    KeyTiles keys;
    __device__ __forceinline__ int head(int t) const { return h0 + (t ? hstep : 0); }
    __device__ __forceinline__ int row(int t) const { return row0 + (t ? rstep : 0); }
    // the last key tile first: with right = 0 every row sees its own key in it, so that the maximum is near its place from the start
    __device__ __forceinline__ int tile(int n) const { return keys.at(keys.n - 1 - n); }
};
__device__ __forceinline__ Item item_of(const Args &A, int i)
{
    Item it;
    // last query tiles first: with a window that is not limited to the left they are the longest
    int x, y;
    const int t = A.steps - 1 - A.per.divmod(i, x);
    it.b = A.heads.divmod(x, y);
    it.h0 = A.paired ? 2 * y : y;
    it.hstep = A.paired ? 1 : 0;
    it.row0 = A.paired ? t * kTile : 2 * t * kTile;
    it.rstep = A.paired ? 0 : kTile;
    it.hk = A.group.div(it.h0);
    it.R = row_of(A.a.band, it.b);
    it.keys = key_tiles(it.R, it.R.pos + it.row0, it.R.pos + min(it.row0 + it.rstep + kTile, A.a.band.nq) - 1);
    return it;
}
// The key tiles of all items of this block, one after the other; items that see nothing have none.
struct Walk {
    Item it;
    int i, tile, count;                                    // count: items with tiles so far
    __device__ __forceinline__ void begin(const Args &A)
    {
        i = blockIdx.x;
        tile = 0;
        count = 0;
        settle_on(A);
    }
    __device__ __forceinline__ void settle_on(const Args &A)
    {
        while (i < A.items) {
            it = item_of(A, i);
            if (it.keys.n > 0) return;
            i += gridDim.x;
        }
    }
    __device__ __forceinline__ bool more(const Args &A) const { return i < A.items; }
    __device__ __forceinline__ void next(const Args &A)
    {
        if (++tile < it.keys.n) return;
        tile = 0;
        ++count;
        i += gridDim.x;
        settle_on(A);
    }
};

// how many of the columns 0, 1, 8, 9, 16, 17, .. 57 a quad's thread has lie before column n
__device__ __forceinline__ int columns(int n)
{
    n = min(max(n, 0), 64);
    return 2 * (n >> 3) + min(n & 7, 2);
}

template <int DP>
__global__ void __launch_bounds__(kThreads, 1) fwd_tc_kernel(const __grid_constant__ Args A)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    using P = Plan<DP>;
    constexpr int TB = kTileBytes<DP>;
    const uint32_t sbase = smem_u32(smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + P::kAbort);
    const Waits wait{abort_flag, A.a.status != nullptr ? A.a.status : reinterpret_cast<int *>(smem + P::kAbort + 4)};
    if (tid == 0) {
        for (int s = 0; s < P::kQStages; ++s) { mbar_init(sbase + P::bQFull + 8 * s, 1); mbar_init(sbase + P::bQEmpty + 8 * s, 2); }
        for (int s = 0; s < P::kSlots; ++s) { mbar_init(sbase + P::bFull + 8 * s, 1); mbar_init(sbase + P::bEmpty + 8 * s, 3); mbar_init(sbase + P::bClear + 8 * s, 1); }
        for (int t = 0; t < 2; ++t) {
            mbar_init(sbase + P::bS + 8 * t, 1);
            mbar_init(sbase + P::bSFree + 8 * t, 8);
            mbar_init(sbase + P::bP + 8 * t, 8);
            mbar_init(sbase + P::bO + 8 * t, 1);
        }
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

    if (warp == kLoadWarp) {
        Walk w;
        uint32_t n = 0;                                    // tiles loaded, keys and values counted apart
        bool ok = true;
        for (w.begin(A); ok && w.more(A); w.next(A)) {
            const int j0 = w.it.tile(w.tile) * kTile, kv = w.it.b * A.a.Hkv + w.it.hk;
            if (w.tile == 0) {
                const int s = w.count % P::kQStages;
                const uint32_t turn = w.count / P::kQStages;
                if (turn > 0 && !wait(sbase + P::bQEmpty + 8 * s, turn - 1)) break;
                if (elect_one()) {
                    mbar_arrive_expect_tx(sbase + P::bQFull + 8 * s, 2 * TB);
                    for (int t = 0; t < 2; ++t)
                        load_tile<DP>(sbase + P::kQ + (2 * s + t) * TB, &A.q, sbase + P::bQFull + 8 * s, w.it.row(t), w.it.b * A.a.H + w.it.head(t));
                }
                __syncwarp();
            }
            for (int side = 0; ok && side < 2; ++side, ++n) {
                const uint32_t s = n % P::kSlots, turn = n / P::kSlots;
                if (turn > 0 && !wait(sbase + P::bEmpty + 8 * s, turn - 1)) { ok = false; break; }
                if (elect_one()) {
                    mbar_arrive_expect_tx(sbase + P::bFull + 8 * s, TB);
                    load_tile<DP>(sbase + P::kKV + s * TB, side ? &A.v : &A.k, sbase + P::bFull + 8 * s, j0, kv);
                }
                __syncwarp();
            }
        }
        if (*abort_flag) {                                 // copies still on their way land before the block ends
            for (uint32_t u = n > P::kSlots ? n - P::kSlots : 0; u < n; ++u)
                for (int x = 0; x < 4096 && !mbar_try_wait(sbase + P::bFull + 8 * (u % P::kSlots), (u / P::kSlots) & 1); ++x) {}
        }
    } else if (warp == kClearWarp) {
        // Values that no query of the batch row sees are multiplied by weights of zero: they must be numbers.  This warp passes every tile in turn and
        // gives its slot free like the products' warps, so that none of its waits is a whole turn ahead or behind.
        Walk w;
        uint32_t n = 0;
        bool ok = true;
        for (w.begin(A); ok && w.more(A); w.next(A)) {
            const int j0 = w.it.tile(w.tile) * kTile;
            for (int side = 0; ok && side < 2; ++side, ++n) {
                const uint32_t s = n % P::kSlots;
                ok = wait(sbase + P::bFull + 8 * s, n / P::kSlots);
                if (!ok) break;
                if (side && !all_used(w.it.R, j0)) {
                    clear_unused<DP>(smem + P::kKV + s * TB, w.it.R, j0, lane);
                    if (lane == 0) mbar_arrive(sbase + P::bClear + 8 * s);
                }
                if (lane == 0) mbar_arrive(sbase + P::bEmpty + 8 * s);
            }
        }
    } else if (warp >= kMmaWarp) {
        const int t = warp - kMmaWarp;
        const uint32_t leader = elect_one();
        Walk w, ahead;
        w.begin(A);
        ahead = w;
        uint32_t g = 0, cleared = 0;                       // tiles done; for each slot, whether its values were cleared an odd number of times
        // S of the tile `ahead` stands at, number `at` of this block's: its queries and keys have come
        auto scores = [&](uint32_t at) {
            const uint32_t s = 2 * at % P::kSlots, q = ahead.count % P::kQStages;
            if (ahead.tile == 0 && !wait(sbase + P::bQFull + 8 * q, ahead.count / P::kQStages)) return false;
            if (!wait(sbase + P::bFull + 8 * s, 2 * at / P::kSlots)) return false;
            product_rows<DP>(leader, tmem + t * P::kCols + P::cS, sbase + P::kQ + (2 * q + t) * TB, sbase + P::kKV + s * TB);
            commit_to(leader, sbase + P::bS + 8 * t);
            commit_to(leader, sbase + P::bEmpty + 8 * s);
            if (ahead.tile == ahead.it.keys.n - 1) commit_to(leader, sbase + P::bQEmpty + 8 * q);
            return true;
        };
        bool ok = !w.more(A) || scores(0);
        if (w.more(A)) ahead.next(A);
        for (; ok && w.more(A); w.next(A), ++g) {
            const bool follow = ahead.more(A);
            const uint32_t vs = (2 * g + 1) % P::kSlots;
            if (P::kApart && follow) {
                ok = wait(sbase + P::bSFree + 8 * t, g);
                if (!ok) break;
                tc_fence_after();
                ok = scores(g + 1);
                if (!ok) break;
            }
            ok = wait(sbase + P::bFull + 8 * vs, (2 * g + 1) / P::kSlots);
            if (!ok) break;
            if (!all_used(w.it.R, w.it.tile(w.tile) * kTile)) {
                ok = wait(sbase + P::bClear + 8 * vs, cleared >> vs);
                if (!ok) break;
                cleared ^= 1u << vs;
            }
            ok = wait(sbase + P::bP + 8 * t, g);
            if (!ok) break;
            tc_fence_after();
            product_weights<DP, 1>(leader, tmem + t * P::kCols + P::cO, tmem + t * P::kCols + P::cP, sbase + P::kKV + vs * TB, w.tile > 0);
            commit_to(leader, sbase + P::bO + 8 * t);
            commit_to(leader, sbase + P::bEmpty + 8 * vs);
            if (follow) {
                if (!P::kApart && !(ok = scores(g + 1))) break;
                ahead.next(A);
            }
        }
        if (*abort_flag) {                                 // products on their way end before tensor memory is given back
            for (int x = 0; x < 4096; ++x) (void)mbar_try_wait(sbase + P::bO + 8 * t, (g & 1) ^ 1);
        }
    } else {
        const int t = warp >> 3, half = (warp >> 2) & 1, first = (warp & 3) * 32 + half * 16, quad = lane & 3;
        // a warp's 16 rows as lanes of tensor memory; this thread has rows first + lane / 4 (A) and 8 further (B), columns 8 i + 2 quad, + 1
        const uint32_t rows16 = tmem + ((uint32_t)first << 16) + t * P::kCols, rows32 = tmem + ((uint32_t)((warp & 3) * 32) << 16) + t * P::kCols;
        float *inv = reinterpret_cast<float *>(smem + P::kInv) + t * kTile;
        const float c = A.a.scale * kLog2e;
        const f2 c2 = pack2(c, c);
        uint32_t g = 0;
        bool ok = true;
        for (int i = blockIdx.x; i < A.items; i += gridDim.x) {
            // what the loop needs of the item, and no more: registers
            int n_tiles, sink, first_tile, ha, la_, hb, lb_, ns, full_hi, any_hi, full_lo, any_lo;
            {
                const Item it = item_of(A, i);
                const Row &R = it.R;
                const int pw0 = R.pos + it.row(t) + first, pw1 = pw0 + 15, pa = pw0 + (lane >> 2), pb = pa + 8;
                n_tiles = it.keys.n; sink = it.keys.sink; first_tile = it.keys.first;
                ha = R.hi(pa) - 2 * quad; la_ = pa - R.left - 2 * quad; hb = R.hi(pb) - 2 * quad; lb_ = pb - R.left - 2 * quad; ns = R.sinks - 2 * quad;
                full_hi = R.hi(pw0); any_hi = R.hi(pw1); full_lo = pw1 - R.left; any_lo = pw0 - R.left;
            }
            float ma = neg_inf(), mb = neg_inf(), la = 0.f, lb = 0.f;
            for (int n = n_tiles - 1; ok && n >= 0; --n, ++g) {             // last key tile first
                const int j0 = (n < sink ? n : first_tile + n - sink) * kTile;
                float x[2][32];
                ok = wait(sbase + P::bS + 8 * t, g);
                if (!ok) break;
                tc_fence_after();
                tile::tmem_ld_acc<8>(rows16 + P::cS, x[0]);
                tile::tmem_ld_acc<8>(rows16 + P::cS + 64, x[1]);
                settle(x[0]);
                settle(x[1]);
                if (P::kApart) {                           // S may be written again
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(sbase + P::bSFree + 8 * t);
                }
                int kind[2];                               // of 64 columns, for the warp: 0 nothing seen, 1 a part, 2 all
                float ta = neg_inf(), tb = neg_inf();
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int a = j0 + 64 * k, b = a + 63;
                    kind[k] = a > any_hi || (b < any_lo && a - 2 * quad >= ns) ? 0 : b <= full_hi && (a >= full_lo || b - 2 * quad < ns) ? 2 : 1;
                    if (kind[k] == 0) continue;
                    if (kind[k] == 1) {
                        // a row's sixteen columns of the half as bits
                        const int to_a = columns(ha - a + 1), to_b = columns(hb - a + 1), s = columns(ns - a);
                        const uint32_t sa = ((1u << to_a) - 1u) & (~((1u << columns(la_ - a)) - 1u) | ((1u << s) - 1u));
                        const uint32_t sb = ((1u << to_b) - 1u) & (~((1u << columns(lb_ - a)) - 1u) | ((1u << s) - 1u));
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            const int bit = 2 * (e >> 2) + (e & 1);
                            x[k][e] = ((e & 2 ? sb : sa) >> bit) & 1u ? x[k][e] : neg_inf();
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        ta = tile::max3(ta, x[k][e], x[k][e + 1]);
                        tb = tile::max3(tb, x[k][e + 2], x[k][e + 3]);
                    }
                }
                ta *= c;
                tb *= c;
                float fa = 1.f, fb = 1.f;
                const bool lift = __any_sync(0xffffffffu, ta > ma + kLift || tb > mb + kLift);
                if (lift) {
                    ta = fmaxf(ta, __shfl_xor_sync(0xffffffffu, ta, 1));
                    tb = fmaxf(tb, __shfl_xor_sync(0xffffffffu, tb, 1));
                    ta = fmaxf(ma, fmaxf(ta, __shfl_xor_sync(0xffffffffu, ta, 2)));
                    tb = fmaxf(mb, fmaxf(tb, __shfl_xor_sync(0xffffffffu, tb, 2)));
                    fa = ta == neg_inf() ? 1.f : ex2(ma - ta);
                    fb = tb == neg_inf() ? 1.f : ex2(mb - tb);
                    ma = ta;
                    mb = tb;
                    la *= fa;
                    lb *= fb;
                }
                const float ra = ma == neg_inf() ? 0.f : -ma, rb = mb == neg_inf() ? 0.f : -mb;
                const f2 ra2 = pack2(ra, ra), rb2 = pack2(rb, rb);
                f2 sa = pack2(la, 0.f), sb = pack2(lb, 0.f);
                uint32_t w[2][16];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if (kind[k] == 0) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) w[k][e] = 0u;
                        continue;
                    }
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        float u, v;
                        unpack2(fma2(pack2(x[k][e], x[k][e + 1]), c2, ra2), u, v);
                        u = ex2(u);
                        v = ex2(v);
                        sa = add2(sa, pack2(u, v));
                        w[k][e / 2] = tile::pack_bf16(u, v);
                        unpack2(fma2(pack2(x[k][e + 2], x[k][e + 3]), c2, rb2), u, v);
                        u = ex2(u);
                        v = ex2(v);
                        sb = add2(sb, pack2(u, v));
                        w[k][e / 2 + 1] = tile::pack_bf16(u, v);
                    }
                }
                {
                    float u, v;
                    unpack2(sa, u, v);
                    la = u + v;
                    unpack2(sb, u, v);
                    lb = u + v;
                }
                if (g > 0) {                               // P is free, O may be touched
                    ok = wait(sbase + P::bO + 8 * t, g - 1);
                    if (!ok) break;
                    tc_fence_after();
                }
                tile::tmem_st_pk<8>(rows16 + P::cP, w[0]);
                tile::tmem_st_pk<8>(rows16 + P::cP + 32, w[1]);
                if (lift && n < n_tiles - 1) {
#pragma unroll 1
                    for (int k = 0; k < DP; k += 32) {
                        uint32_t o[16];
                        tile::tmem_ld_pk<8>(rows16 + P::cO + k, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 16; ++e) asm volatile("mul.f32 %0, %0, %1;" : "+r"(o[e]) : "f"(e & 1 ? fb : fa));
                        tile::tmem_st_pk<8>(rows16 + P::cO + k, o);
                    }
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(sbase + P::bP + 8 * t);
            }
            // the rows' weights for whoever reads them: a warp takes all 32 rows of its lanes of tensor memory and half of the channels
            int again = i;
            asm volatile("" : "+r"(again));                // not kept over the loop
            const Item it = item_of(A, again);
            const int q0 = it.row(t), q = q0 + (warp & 3) * 32 + lane;
            const size_t head = ((size_t)it.b * A.a.H + it.head(t)) * A.a.band.nq;
            __nv_bfloat16 *out = static_cast<__nv_bfloat16 *>(A.a.out) + (head + q) * A.a.d;
            if (it.keys.n > 0) {
                if (ok) ok = wait(sbase + P::bO + 8 * t, g - 1);
                tc_fence_after();
                const float nan = __int_as_float(0x7fc00000);
                la += __shfl_xor_sync(0xffffffffu, la, 1);
                lb += __shfl_xor_sync(0xffffffffu, lb, 1);
                la += __shfl_xor_sync(0xffffffffu, la, 2);
                lb += __shfl_xor_sync(0xffffffffu, lb, 2);
                if (quad < 2) {
                    const int r = first + (lane >> 2) + 8 * quad;
                    const float l = quad ? lb : la, m = quad ? mb : ma;
                    inv[r] = !ok ? nan : l == 0.f ? 0.f : 1.f / l;
                    if (A.a.lse != nullptr && q0 + r < A.a.band.nq) A.a.lse[head + q0 + r] = !ok ? nan : l == 0.f ? neg_inf() : m * kLn2 + logf(l);
                }
                named_bar_sync(1 + t, kGroup8);
                const float f = inv[(warp & 3) * 32 + lane];
#pragma unroll
                for (int k = half * (DP / 2); k < half * (DP / 2) + DP / 2; k += 32) {
                    float o[32];
                    tmem_ld32(rows32 + P::cO + k, o);
                    settle(o);
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = f == 0.f ? 0.f : o[e] * f;
                    if (q < A.a.band.nq) store_row(out, k, A.a.d, o);
                }
            } else if (q < A.a.band.nq) {
                const float o[32] = {};
                for (int k = half * (DP / 2); k < half * (DP / 2) + DP / 2; k += 32) store_row(out, k, A.a.d, o);
                if (half == 0 && A.a.lse != nullptr) A.a.lse[head + q] = neg_inf();
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
}

template <int DP> cudaError_t launch_t(const Args &A, cudaStream_t st)
{
    static std::mutex mu;
    static bool set[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!set[dev]) {
            const cudaError_t e = cudaFuncSetAttribute(fwd_tc_kernel<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, Plan<DP>::kTotal);
            if (e != cudaSuccess) return e;
            set[dev] = true;
        }
    }
    const int sms = device_sm_count();
    fwd_tc_kernel<DP><<<A.items < sms ? A.items : sms, kThreads, Plan<DP>::kTotal, st>>>(A);
    return cudaGetLastError();
}

} // namespace

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                  const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

bool make_tile_map(CUtensorMap *m, const void *base, long long outer, int rows, int cols, int box_rows)
{
    static EncodeTiledFn fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) == cudaSuccess && found == cudaDriverEntryPointSuccess
                   ? reinterpret_cast<EncodeTiledFn>(p) : nullptr;
    }();
    if (fn == nullptr) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)outer}, strides[2] = {(cuuint64_t)cols * 2, (cuuint64_t)rows * cols * 2};
    const cuuint32_t box[3] = {64u, (cuuint32_t)box_rows, 1u}, es[3] = {1u, 1u, 1u};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t launch_fwd_tc(const Fwd &a, cudaStream_t st)
{
    Args A;
    A.a = a;
    const int G = a.H / a.Hkv, tiles = (a.band.nq + kTile - 1) / kTile;
    A.paired = G % 2 == 0;
    A.steps = A.paired ? tiles : (tiles + 1) / 2;
    const int heads = A.paired ? a.H / 2 : a.H;
    A.items = A.steps * a.B * heads;
    A.per = fast_div(a.B * heads);
    A.heads = fast_div(heads);
    A.group = fast_div(G);
    if (!make_tile_map(&A.q, a.q, (long long)a.B * a.H, a.band.nq, a.d)) return cudaErrorInvalidValue;
    A.k = A.v = A.q;                                       // without keys no item has tiles
    if (a.band.nk > 0 && (!make_tile_map(&A.k, a.k, (long long)a.B * a.Hkv, a.band.nk, a.d) ||
                          !make_tile_map(&A.v, a.v, (long long)a.B * a.Hkv, a.band.nk, a.d)))
        return cudaErrorInvalidValue;
    return a.d <= 64 ? launch_t<64>(A, st) : launch_t<128>(A, st);
}

} // namespace window
} // namespace lot
