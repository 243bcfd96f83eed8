// What the tcgen05 kernels of window attention share: tiles of 128 rows in shared memory, key tiles a block of queries sees, products with the
// first operand in tensor memory, bounded waits.
#pragma once

#include "lot_sm100.cuh"
#include "lot_tile.cuh"
#include "lot_window.cuh"

namespace lot {
int device_sm_count();
namespace window {

using namespace sm100;

constexpr int kTile = 128;

// Key tiles that queries at positions p0 .. p1 see: those of the sinks below the window's first, then the window's.
struct KeyTiles {
    int sink, first, n;                    // tiles 0 .. sink - 1, then first ..; n in all
    __device__ __forceinline__ int at(int i) const { return i < sink ? i : first + i - sink; }
};
__device__ __forceinline__ KeyTiles key_tiles(const Row &R, int p0, int p1)
{
    KeyTiles t;
    const int hi = R.hi(p1), last = hi < 0 ? -1 : hi / kTile;
    t.first = R.lo(p0) / kTile;
    t.sink = max(min((min(R.sinks, hi + 1) + kTile - 1) / kTile, t.first), 0);
    t.n = t.sink + max(last - t.first + 1, 0);
    return t;
}

__device__ __forceinline__ uint32_t bits_between(int a, int b)      // bits a .. b (clamped to 0 .. 31)
{
    a = max(a, 0);
    b = min(b, 31);
    return a > b ? 0u : (0xffffffffu >> (31 - b)) & (0xffffffffu << a);
}

// ---- shared memory: a tile is DP / 64 panels of 128 rows x 128 bytes, 16-byte chunks permuted by the row (128-byte swizzle) ----
template <int DP> constexpr int kTileBytes = kTile * DP * 2;

template <int DP> __device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap *map, uint32_t bar, int row, int outer)
{
#pragma unroll
    for (int p = 0; p < DP / 64; ++p) tma_load_3d(dst + p * kTile * 128, map, bar, p * 64, row, outer);
}
// rows of a tile of keys or values that no query sees: whatever they hold, zeros take part in the products (whole warp)
template <int DP> __device__ __forceinline__ void clear_unused(uint8_t *tile, const Row &R, int j0, int lane)
{
    for (int r = lane; r < kTile; r += 32) {
        if (R.used(j0 + r)) continue;
#pragma unroll
        for (int p = 0; p < DP / 64; ++p) {
            uint4 *x = reinterpret_cast<uint4 *>(tile + p * kTile * 128 + r * 128);
#pragma unroll
            for (int c = 0; c < 8; ++c) x[c] = make_uint4(0, 0, 0, 0);
        }
    }
    fence_proxy_async_smem();
    __syncwarp();
}
template <int ROWS = kTile> __device__ __forceinline__ bool all_used(const Row &R, int j0)
{
    return R.used(j0) && j0 + ROWS <= R.len && (j0 >= R.first || j0 + ROWS <= R.sinks);
}

// ---- products ---------------------------------------------------------------------------------------------------------------
// The whole warp computes the descriptors; the lane with `leader` set, always the same one, issues: its products and the commit behind them stay in order.
// D (tensor memory, 128 x N) = or += A B; descriptors as low word (address) and high word
__device__ __forceinline__ void issue_ss(uint32_t leader, uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b64 a, b;\n\t"
                 "setp.ne.b32 p, %5, 0;\n\t"
                 "setp.ne.b32 q, %6, 0;\n\t"
                 "mov.b64 a, {%1, %3};\n\t"
                 "mov.b64 b, {%2, %3};\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, p;\n\t}"
                 ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate), "r"(leader) : "memory");
}
// A (tensor memory, 128 x 16 bf16: two to a column)
__device__ __forceinline__ void issue_ts(uint32_t leader, uint32_t d, uint32_t a, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b64 b;\n\t"
                 "setp.ne.b32 p, %5, 0;\n\t"
                 "setp.ne.b32 q, %6, 0;\n\t"
                 "mov.b64 b, {%2, %3};\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate), "r"(leader) : "memory");
}
__device__ __forceinline__ void commit_to(uint32_t leader, uint32_t bar)
{
    asm volatile("{\n\t.reg .pred q;\n\t"
                 "setp.ne.b32 q, %1, 0;\n\t"
                 "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(leader) : "memory");
}
// descriptor words (make_smem_desc): rows of 64 channels, K-major; and the same rows as the K of an MN-major operand, panels of 64 channels apart
constexpr uint32_t kDescRows = (1024u >> 4) | (1u << 14) | (2u << 29), kDescRowsLo = (16u >> 4) << 16, kDescColsLo = ((kTile * 128u) >> 4) << 16;
// D = X Y^T over DP channels, both tiles with 64 channels a panel row
template <int DP> __device__ __forceinline__ void product_rows(uint32_t leader, uint32_t d, uint32_t x, uint32_t y)
{
    constexpr uint32_t idesc = make_idesc_bf16(128, kTile, 0, 0);
    const uint32_t lx = (x >> 4) | kDescRowsLo, ly = (y >> 4) | kDescRowsLo;
#pragma unroll
    for (int ks = 0; ks < DP / 16; ++ks) {
        const uint32_t off = (ks >> 2) * (kTile * 128 / 16) + (ks & 3) * 2;
        issue_ss(leader, d, lx + off, ly + off, kDescRows, idesc, ks != 0);
    }
}
// D (128 x DP) += W Y: W 128 x 128 bf16 in tensor memory, 64 / PARTS neighbouring columns at w, w + 32, .. each; Y's 128 rows
template <int DP, int PARTS> __device__ __forceinline__ void product_weights(uint32_t leader, uint32_t d, uint32_t w, uint32_t y, bool accumulate)
{
    constexpr uint32_t idesc = make_idesc_bf16(128, DP, 0, 1);
    constexpr int RUN = kTile / 16 / PARTS;                // products to a part
    const uint32_t ly = (y >> 4) | kDescColsLo;
#pragma unroll
    for (int ks = 0; ks < kTile / 16; ++ks)
        issue_ts(leader, d, w + ks / RUN * 32 + ks % RUN * 8, ly + ks * 128, kDescRows, idesc, accumulate || ks != 0);
}

// ---- tensor memory ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
                 "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                   "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
// Behind it the columns just requested may be used.
__device__ __forceinline__ void settle(float (&v)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]),
                   "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15])::"memory");
}
// Behind it the 32 columns just requested may be used.
__device__ __forceinline__ void settle(float (&v)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]),
                   "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15])::"memory");
    asm volatile("" : "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]), "+f"(v[25]),
                   "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])::"memory");
}

// N numbers of one row as bf16 to columns col .. col + N - 1 of a [rows][d] tensor; d is a multiple of 8
template <int N> __device__ __forceinline__ void store_row(__nv_bfloat16 *row, int col, int d, const float (&v)[N])
{
#pragma unroll
    for (int c = 0; c < N; c += 8)
        if (col + c < d)
            *reinterpret_cast<uint4 *>(row + col + c) = make_uint4(tile::pack_bf16(v[c], v[c + 1]), tile::pack_bf16(v[c + 2], v[c + 3]),
                                                                    tile::pack_bf16(v[c + 4], v[c + 5]), tile::pack_bf16(v[c + 6], v[c + 7]));
}

// Division of numbers below 2^31 by a number fixed at the launch: q = (n + high half of n mul) >> shift.
struct FastDiv {
    uint32_t mul, shift, by;
    __device__ __forceinline__ int div(int n) const { return (int)((__umulhi((uint32_t)n, mul) + (uint32_t)n) >> shift); }
    __device__ __forceinline__ int divmod(int n, int &rest) const
    {
        const int q = div(n);
        rest = n - q * (int)by;
        return q;
    }
};
inline FastDiv fast_div(int d)
{
    FastDiv f;
    f.by = (uint32_t)d;
    f.shift = 0;
    while ((1ull << f.shift) < (uint64_t)d) ++f.shift;
    f.mul = (uint32_t)(((1ull << 32) * ((1ull << f.shift) - (uint64_t)d)) / (uint64_t)d + 1);
    return f;
}

// ---- barriers -------------------------------------------------------------------------------------------------------------
// A try suspends the warp for up to kNap nanoseconds, so that a waiting warp is not counted among those that could issue.
constexpr uint32_t kNap = 100000;
__device__ __forceinline__ bool try_nap(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity), "r"(kNap) : "memory");
    return ok != 0;
}
struct Waits {                             // bounded waits of one block: the first that gives up ends them all
    volatile int *abort_flag;
    int *status;
    __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t phase) const
    {
        if (try_nap(bar, phase & 1u)) return true;
        return slow(bar, phase & 1u, abort_flag, status);
    }
    static __device__ __noinline__ bool slow(uint32_t bar, uint32_t parity, volatile int *abort_flag, int *status)
    {
        const uint64_t t0 = global_timer_ns();
        for (;;) {
            if (try_nap(bar, parity)) return true;
            if (*abort_flag) return false;
            if (global_timer_ns() - t0 > kWaitLimitNs) break;
        }
        *abort_flag = 1;
        atomicOr(status, 4 /* LOT_DEV_TIMEOUT */);
        return false;
    }
};

// host: bf16 tensor [outer][rows][cols], box 64 columns x `box` rows; columns and rows beyond the tensor read as zeros
bool make_tile_map(CUtensorMap *m, const void *base, long long outer, int rows, int cols, int box = kTile);

} // namespace window
} // namespace lot
