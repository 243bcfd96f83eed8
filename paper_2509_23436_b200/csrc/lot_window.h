// Internal launch interface of window attention (lot_window_fwd, lot_window_bwd) and of the 4-bit cache.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace lot {
namespace window {

constexpr int kFar = 1 << 30;              // left, right without limit: positions stay below 2^29, sums inside 32 bits
constexpr int kMaxPos = 1 << 29;

struct Band {                              // which keys a query sees
    const int32_t *key_len;                // [B] or nullptr (nk)
    const int32_t *q_start;                // [B] or nullptr (nk - nq)
    int nq, nk, left, right, sinks;        // left, right <= kFar, sinks <= nk
};

struct Fwd {
    Band band;
    const void *q, *k, *v;                 // [B][H][nq][d], [B][Hkv][nk][d]
    void *out;                             // [B][H][nq][d]
    float *lse;                            // [B][H][nq] or nullptr
    int dtype, B, H, Hkv, d;
    float scale;
    int *status;                           // or nullptr
    void *ws;                              // few_workspace bytes where that kernel is taken
};

struct Bwd {
    Band band;
    const void *q, *k, *v, *out, *dout;
    const float *lse;
    void *dq, *dk, *dv;
    float *delta;                          // the workspace: <dout, out> of every row, and what bf16 tensors need besides
    int dtype, B, H, Hkv, d;
    float scale;
    int *status;
};

struct Cache4 {                            // [num_pages][Hkv][2][page_size * (d/2 + d/8)] bytes
    uint8_t *base;
    const int32_t *pages;                  // [B][max_pages]
    int num_pages, max_pages, page_size, Hkv, d;
};

struct Attend4 {
    Cache4 cache;
    Band band;                             // key_len = length, nk = capacity of the page table, q_start unused (length - nq)
    const void *q;
    void *out;
    float *lse;
    int dtype, B, H;
    float scale;
    int *status;
    void *ws;                              // attend4_workspace bytes
};

cudaError_t launch_fwd(const Fwd &a, cudaStream_t st);
cudaError_t launch_fwd_tc(const Fwd &a, cudaStream_t st);      // bf16 tensors (lot_window_tc.cu)
cudaError_t launch_bwd(const Bwd &a, cudaStream_t st);
size_t fwd_workspace(int dtype, int B, int H, int Hkv, const Band &band, int d);
size_t bwd_f32_workspace(int B, int H, int Hkv, int nq, int nk, int d, int left, int right, int sinks);
cudaError_t launch_bwd_tc(const Bwd &a, cudaStream_t st);      // bf16 tensors (lot_window_tc_bwd.cu)
size_t bwd_tc_workspace(int B, int H, int Hkv, int nq, int nk, int d, int left, int right, int sinks);
size_t attend4_workspace(int dtype, int B, int H, int Hkv, int nq, int d, int nk, int left, int sinks);
cudaError_t launch_attend4(const Attend4 &a, cudaStream_t st);
cudaError_t launch_write4(const Cache4 &c, const void *k, const void *v, const int32_t *start, const int32_t *count, int dtype, int B, int m, int *status,
                          cudaStream_t st);
cudaError_t launch_read4(const Cache4 &c, void *k, void *v, const int32_t *start, const int32_t *count, int dtype, int B, int m, int *status,
                         cudaStream_t st);

// ---- few queries: how the keys of a sequence are split over blocks ----
// The lengths are on the device, so a split is a number of chunks (`each`), counted for the longest sequence there may be; a shorter one leaves
// its last splits nothing to do.
struct Split {
    int splits, each, clustered;           // clustered: the splits are the blocks of a cluster
};
// blocks: without splits; run, sinks: neighbouring keys, and first keys, that the rows of one may see; at_once: blocks on an SM.
// A round is a chunk for each of a block's warps.  Few blocks: up to eight splits of up to 16 rounds, one launch.  Else so many that the blocks
// fill the SMs four times over, which evens out sequences of different lengths, but none of less than four rounds (a block's beginning and end
// cost as much as two).
inline Split split_of(int sms, long long blocks, int nk, long long run, int sinks, int chunk, int warps, int at_once)
{
    const long long all = ((long long)nk + chunk - 1) / chunk, touched = (run + 2 * (chunk - 1)) / chunk + (sinks + chunk - 1) / chunk;
    const long long rounds = ((touched < all ? touched : all) + warps - 1) / warps, slots = (long long)at_once * sms;
    Split s{1, (int)rounds * warps, 0};
    if (rounds <= 1) return s;
    if (blocks * 2 <= slots) {
        const long long room = slots / blocks, n = rounds < room ? rounds : room, m = n < 8 ? n : 8, per = (rounds + m - 1) / m;
        if (per <= 16) return Split{(int)((rounds + per - 1) / per), (int)per * warps, (rounds + per - 1) / per > 1};
    }
    const long long n = (4 * slots + blocks - 1) / blocks;
    long long per = (rounds + n - 1) / n;
    if (per < 4) per = 4;
    if ((rounds + per - 1) / per > 512) per = (rounds + 511) / 512;
    s.splits = (int)((rounds + per - 1) / per);
    s.each = (int)per * warps;
    return s;
}

bool few_supported(int B, int H, int Hkv, int nq, int nk);         // lot_window_few.cu
size_t few_workspace(int B, int H, int Hkv, const Band &b, int d);
cudaError_t launch_few(const Fwd &a, cudaStream_t st);

} // namespace window
} // namespace lot
