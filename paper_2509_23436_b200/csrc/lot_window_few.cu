// Window attention forward of few bf16 queries (a decoder's next tokens): bound by reading the visible keys and values once per key head.
//
// The query rows of a key head (its query heads times the queries) are the narrow side of warp-level products (16 x 8 x 16: sixteen keys by eight rows).  A warp
// goes over chunks of 16 keys by itself, which TMA brings into a ring of its own (128-byte swizzle: the reads below meet no bank twice): eight warps an
// SM with two chunks each on their way.  A key's 16 bytes are two operands of the scores' products as they lie; of the values a byte permutation of two keys'
// words makes an operand.  The running maximum moves only when a score passes it by 2^8.  Blocks share a sequence's chunks: the blocks of a
// cluster join in shared memory (one launch), those of many through memory and a second kernel.
// B = 64, H = 16, 4 key heads of 128, 4100 visible keys of up to 8192: 90 us, 0.92 of the
// copy rate.
#include "lot_chain.cuh"
#include "lot_window_tc.cuh"

#include <mutex>

namespace lot {
namespace window {
namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32, kChunk = 16, kStages = 3, kRows = 8;
constexpr float kLift = 8.f;

template <int D> struct Lay {
    static constexpr int SIDE = kChunk * D * 2, STAGE = 2 * SIDE, RING = kStages * STAGE, WARP = RING;       // of a warp; the join takes less
    static constexpr int OWN = kWarps * WARP, BARS = OWN + (kRows * D + 2 * kRows) * 4, TOTAL = BARS + kWarps * kStages * 8 + 16;
    static constexpr int kBlocks = D == 64 ? 4 : 2;        // on an SM at once
    static_assert(WARP % 1024 == 0 && (kRows * D + 2 * kRows) * 4 <= WARP, "ring");
};

struct Args {
    Fwd a;
    CUtensorMap k, v;
    int splits, each, row_tiles, G, clustered;
    float *part;                           // splits > 1, not clustered: [row tile][B Hkv][split][kRows][D + 2]
};

__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t flip(uint32_t x)      // 8 x 8 transposed across the warp
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
// 16-byte chunk c of row r of a panel [16 rows][128 bytes]
__device__ __forceinline__ uint4 piece(const uint8_t *panel, int r, int c) { return *reinterpret_cast<const uint4 *>(panel + r * 128 + ((c ^ (r & 7)) << 4)); }

template <int D>
__global__ void __launch_bounds__(kThreads, Lay<D>::kBlocks) few_kernel(const __grid_constant__ Args A)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    using L = Lay<D>;
    constexpr int PANELS = D / 64, PANEL = kChunk * 128;
    typedef __nv_bfloat16 T;
    const Fwd &a = A.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int split = blockIdx.x % A.splits, tile = blockIdx.x / A.splits, hk = blockIdx.y, b = blockIdx.z;
    const int nq = a.band.nq, rows = A.G * nq, r0 = tile * kRows, d = a.d;
    const Row R = row_of(a.band, b);
    const int p0 = R.pos, p1 = R.pos + nq - 1;
    // chunks that some row sees: those of the sinks, then the window's
    const int any_hi = R.hi(p1), all_hi = R.hi(p0), all_lo = max(p1 - R.left, 0);
    const int first = R.lo(p0) / kChunk, last = any_hi < 0 ? -1 : any_hi / kChunk, sink = max(min((min(R.sinks, any_hi + 1) + kChunk - 1) / kChunk, first), 0);
    const int count = sink + max(last - first + 1, 0), total = min(count, (split + 1) * A.each), mine = split * A.each + warp;
    const int turns = mine < total ? (total - mine + kWarps - 1) / kWarps : 0;

    uint8_t *ring = smem + warp * L::WARP;
    const uint32_t ring_s = smem_u32(ring), bars = smem_u32(smem) + L::BARS + warp * kStages * 8;
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + L::BARS + kWarps * kStages * 8);
    const Waits wait{abort_flag, a.status != nullptr ? a.status : const_cast<int *>(abort_flag) + 1};
    if (lane == 0)
        for (int s = 0; s < kStages; ++s) mbar_init(bars + 8 * s, 1);
    if (tid == 0) abort_flag[0] = abort_flag[1] = 0;
    fence_barrier_init();
    __syncthreads();
    auto chunk = [&](int turn) {
        const int n = mine + turn * kWarps;
        return (n < sink ? n : first + n - sink) * kChunk;
    };
    auto fetch = [&](int turn) {
        const uint32_t s = turn % kStages, bar = bars + 8 * s, dst = ring_s + s * L::STAGE;
        if (lane == 0) {
            const int j = chunk(turn), head = b * a.Hkv + hk;
            mbar_arrive_expect_tx(bar, L::STAGE);
#pragma unroll
            for (int p = 0; p < PANELS; ++p) {
                tma_load_3d(dst + p * PANEL, &A.k, bar, p * 64, j, head);
                tma_load_3d(dst + L::SIDE + p * PANEL, &A.v, bar, p * 64, j, head);
            }
        }
    };
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s)
        if (s < turns) fetch(s);

    // row r of the key head: query head hk G + r / nq, query r % nq; lane (g, t) holds of row g channels 8 (4 i + t) .. + 7 of every 32
    uint32_t qf[D / 32][4];
    {
        const int r = r0 + g;
        const T *q = static_cast<const T *>(a.q) + (((size_t)b * a.H + hk * A.G + (r < rows ? r / nq : 0)) * nq + (r < rows ? r % nq : 0)) * d;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            const int c = 8 * (4 * i + t);
            const uint4 x = r < rows && c < d ? *reinterpret_cast<const uint4 *>(q + c) : make_uint4(0, 0, 0, 0);
            qf[i][0] = x.x; qf[i][1] = x.y; qf[i][2] = x.z; qf[i][3] = x.w;
        }
    }
    const float scale = a.scale * kLog2e;
    // sums of channel 64 i + 8 g + 2 w + e / 2 by row 2 t + e % 2 in o[4 i + w][e]
    float o[D / 16][4], ref[2] = {neg_inf(), neg_inf()}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int m = 0; m < D / 16; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[m][e] = 0.f;
    const int prow[2] = {p0 + min(r0 + 2 * t, rows - 1) % nq, p0 + min(r0 + 2 * t + 1, rows - 1) % nq};

    for (int turn = 0; turn < turns; ++turn) {
        const uint32_t s = turn % kStages;
        const int j0 = chunk(turn);
        if (turn + kStages - 1 < turns) {
            __syncwarp();                                  // the stage's readers are done
            fetch(turn + kStages - 1);
        }
        if (!wait(bars + 8 * s, turn / kStages)) {
            for (int u = turn + 1; u < turns && u < turn + kStages; ++u)           // copies on their way, before the block may end
                for (int it = 0; it < 4096 && !mbar_try_wait(bars + 8 * (u % kStages), (u / kStages) & 1); ++it) {}
            break;
        }
        uint8_t *kp = ring + s * L::STAGE, *vp = kp + L::SIDE;
        const bool whole = j0 + kChunk - 1 <= all_hi && j0 >= all_lo;
        if (!whole && !all_used<kChunk>(R, j0)) {
            // values that no query sees are multiplied by zero: they must be numbers
            if (lane < kChunk && !R.used(j0 + lane)) {
#pragma unroll
                for (int p = 0; p < PANELS; ++p)
#pragma unroll
                    for (int c = 0; c < 8; ++c) *reinterpret_cast<uint4 *>(vp + p * PANEL + lane * 128 + c * 16) = make_uint4(0, 0, 0, 0);
                fence_proxy_async_smem();                  // before a later copy writes there
            }
            __syncwarp();
        }
        float S[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            const uint4 x = piece(kp + (i >> 1) * PANEL, g, 4 * (i & 1) + t), y = piece(kp + (i >> 1) * PANEL, g + 8, 4 * (i & 1) + t);
            const uint32_t f[4] = {x.x, y.x, x.y, y.y}, h[4] = {x.z, y.z, x.w, y.w};
            mma(S, f, qf[i][0], qf[i][1]);
            mma(S, h, qf[i][2], qf[i][3]);
        }
        if (!whole) {
#pragma unroll
            for (int e = 0; e < 4; ++e) S[e] = R.sees(prow[e & 1], j0 + g + (e >> 1) * 8) ? S[e] : neg_inf();
        }
        const float top[2] = {scale * fmaxf(S[0], S[2]), scale * fmaxf(S[1], S[3])};
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
                for (int m2 = 0; m2 < D / 16; ++m2) { o[m2][q] *= f; o[m2][q + 2] *= f; }
            }
        }
        const float ra = ref[0] == neg_inf() ? 0.f : ref[0], rb = ref[1] == neg_inf() ? 0.f : ref[1];
        S[0] = ex2(fmaf(S[0], scale, -ra));
        S[1] = ex2(fmaf(S[1], scale, -rb));
        S[2] = ex2(fmaf(S[2], scale, -ra));
        S[3] = ex2(fmaf(S[3], scale, -rb));
        l[0] += S[0] + S[2];
        l[1] += S[1] + S[3];
        const uint32_t x0 = flip(tile::pack_bf16(S[0], S[1])), x1 = flip(tile::pack_bf16(S[2], S[3]));
#pragma unroll
        for (int i = 0; i < PANELS; ++i) {
            const uint4 va = piece(vp + i * PANEL, 2 * t, g), vb = piece(vp + i * PANEL, 2 * t + 1, g), vc = piece(vp + i * PANEL, 2 * t + 8, g),
                        ve = piece(vp + i * PANEL, 2 * t + 9, g);
            const uint32_t wa[4] = {va.x, va.y, va.z, va.w}, wb[4] = {vb.x, vb.y, vb.z, vb.w}, wc[4] = {vc.x, vc.y, vc.z, vc.w}, we[4] = {ve.x, ve.y, ve.z, ve.w};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t f[4] = {__byte_perm(wa[w], wb[w], 0x5410), __byte_perm(wa[w], wb[w], 0x7632), __byte_perm(wc[w], we[w], 0x5410),
                                       __byte_perm(wc[w], we[w], 0x7632)};
                mma(o[4 * i + w], f, x0, x1);
            }
        }
    }
    // the lanes of a row's keys together
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[q] += __shfl_xor_sync(0xffffffffu, l[q], x);
    __syncthreads();                                       // every warp has left its ring
    float *mo = reinterpret_cast<float *>(ring), *mm = mo + kRows * D;
#pragma unroll
    for (int m = 0; m < D / 16; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) mo[(2 * t + (e & 1)) * D + 64 * (m >> 2) + 8 * g + 2 * (m & 3) + (e >> 1)] = o[m][e];
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
        const size_t row = ((size_t)b * a.H + hk * A.G + (r0 + r) / nq) * nq + (r0 + r) % nq;
        const bool nothing = sum == 0.f;
        if (col < d) Elem<T>::store(static_cast<T *>(a.out) + row * d + col, nothing ? 0.f : x / sum);
        if (col == 0 && a.lse != nullptr) a.lse[row] = nothing ? neg_inf() : top * kLn2 + logf(sum);
    };
    if (A.clustered) {
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
                float *part = A.part + ((((size_t)tile * a.B + b) * a.Hkv + hk) * A.splits + split) * (kRows * (D + 2)) + r * (D + 2);
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
template <int D>
__global__ void __launch_bounds__(D) join_kernel(const __grid_constant__ Args A)
{
    const Fwd &a = A.a;
    const int nq = a.band.nq, r = blockIdx.x, hk = blockIdx.y, b = blockIdx.z, ch = threadIdx.x;
    const float *part = A.part + ((((size_t)(r / kRows) * a.B + b) * a.Hkv + hk) * A.splits) * (kRows * (D + 2)) + (r % kRows) * (D + 2);
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
    const size_t row = ((size_t)b * a.H + hk * A.G + r / nq) * nq + r % nq;
    const bool nothing = sum == 0.f;
    if (ch < a.d) Elem<__nv_bfloat16>::store(static_cast<__nv_bfloat16 *>(a.out) + row * a.d + ch, nothing ? 0.f : x / sum);
    if (ch == 0 && a.lse != nullptr) a.lse[row] = nothing ? neg_inf() : top * kLn2 + logf(sum);
}

template <int D> cudaError_t run(const Args &A, cudaStream_t st)
{
    static std::mutex mu;
    static bool set[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!set[dev]) {
            const cudaError_t e = cudaFuncSetAttribute(few_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Lay<D>::TOTAL);
            if (e != cudaSuccess) return e;
            set[dev] = true;
        }
    }
    const dim3 grid(A.splits * A.row_tiles, A.a.Hkv, A.a.B);
    if (A.clustered) return cluster_launch(few_kernel<D>, grid, kThreads, Lay<D>::TOTAL, A.splits, st, A);
    few_kernel<D><<<grid, kThreads, Lay<D>::TOTAL, st>>>(A);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || A.splits == 1) return e;
    return chain_launch(join_kernel<D>, dim3(A.G * A.a.band.nq, A.a.Hkv, A.a.B), D, 0, st, A);
}

Split few_split(int B, int H, int Hkv, const Band &b, int d)
{
    const int tiles = (H / Hkv * b.nq + kRows - 1) / kRows;
    // keys the rows may touch: left + nq + right in a row (positions are on the device), and the sinks
    const long long run = (long long)(b.left < b.nk ? b.left : b.nk) + (b.right < b.nk ? b.right : b.nk) + b.nq;
    return split_of(device_sm_count(), (long long)B * Hkv * tiles, b.nk, run, b.sinks, kChunk, kWarps, d <= 64 ? Lay<64>::kBlocks : Lay<128>::kBlocks);
}

} // namespace

// Few queries: while the row tiles (eight rows; each reads the keys again, by then from the L2) are no more than two blocks an SM for each round of the
// other kernel's blocks (256 rows, not split along the keys).  32 heads on 4 key heads of 128 channels, 16384 keys: 17 queries 68 us against 293, 64 209
// against 295; 8 x 16 heads on 4, 8192 keys: 17 queries 119 against 154 (24, which do not count as few, would take some 165).
bool few_supported(int B, int H, int Hkv, int nq, int nk)
{
    if (nk == 0 || nq > 64) return false;
    const long long sms = device_sm_count(), G = H / Hkv, tiles = (G * nq + kRows - 1) / kRows * B * Hkv;
    const long long items = (long long)B * (G % 2 ? H : H / 2), rounds = (items + sms - 1) / sms;
    return tiles <= 2 * sms * rounds;
}

size_t few_workspace(int B, int H, int Hkv, const Band &b, int d)
{
    const Split s = few_split(B, H, Hkv, b, d);
    if (s.splits == 1 || s.clustered) return 0;
    const size_t D = d <= 64 ? 64 : 128, tiles = (H / Hkv * b.nq + kRows - 1) / kRows;
    return (tiles * B * Hkv * s.splits * kRows * (D + 2) * 4 + 255) & ~(size_t)255;
}

cudaError_t launch_few(const Fwd &a, cudaStream_t st)
{
    const Split s = few_split(a.B, a.H, a.Hkv, a.band, a.d);
    Args A;
    A.a = a;
    A.G = a.H / a.Hkv;
    A.row_tiles = (A.G * a.band.nq + kRows - 1) / kRows;
    A.splits = s.splits;
    A.each = s.each;
    A.clustered = s.clustered;
    A.part = static_cast<float *>(a.ws);
    if (!make_tile_map(&A.k, a.k, (long long)a.B * a.Hkv, a.band.nk, a.d, kChunk) || !make_tile_map(&A.v, a.v, (long long)a.B * a.Hkv, a.band.nk, a.d, kChunk))
        return cudaErrorInvalidValue;
    return a.d <= 64 ? run<64>(A, st) : run<128>(A, st);
}

} // namespace window
} // namespace lot
