// C entry points of window attention and of the 4-bit cache (see include/lot.h): argument checks, workspaces, launches.
#include "../../include/lot.h"
#include "lot_window.h"

#include <math.h>

namespace {

using namespace lot::window;

inline bool aligned(const void *p, unsigned by) { return (reinterpret_cast<uintptr_t>(p) & (by - 1)) == 0; }

int check_sizes(int dtype, int B, int H, int Hkv, int nq, int nk, int d, int sinks)
{
    if (dtype != LOT_F32 && dtype != LOT_BF16) return LOT_ERR_INVALID_ARG;
    if (B < 0 || H < 1 || Hkv < 1 || H % Hkv != 0 || nq < 0 || nk < 0 || d < 1 || sinks < 0) return LOT_ERR_INVALID_ARG;
    if (d > 128 || d % 8 != 0 || (long long)B * H > 32767) return LOT_ERR_UNSUPPORTED_SHAPE;
    if ((long long)nq * d >= (1ll << 31) || (long long)nk * d >= (1ll << 31)) return LOT_ERR_UNSUPPORTED_SHAPE;
    return LOT_OK;
}
bool bad_scale(float scale) { return !(scale > 0.f) || !isfinite(scale); }

Band band_of(const int32_t *key_len, const int32_t *q_start, int nq, int nk, int left, int right, int sinks)
{
    return Band{key_len, q_start, nq, nk, left < 0 || left > kFar ? kFar : left, right < 0 || right > kFar ? kFar : right, sinks < nk ? sinks : nk};
}

int check_cache(int B, int Hkv, int d, int page_size, int max_pages, int num_pages)
{
    if (B < 0 || Hkv < 1 || d < 1 || page_size < 1 || max_pages < 1 || num_pages < 1) return LOT_ERR_INVALID_ARG;
    if ((d != 32 && d != 64 && d != 128) || page_size % 16 != 0) return LOT_ERR_UNSUPPORTED_SHAPE;
    if ((long long)max_pages * page_size > (1ll << 28) || (long long)B * Hkv > 32767) return LOT_ERR_UNSUPPORTED_SHAPE;
    return LOT_OK;
}

int done(cudaError_t e) { return e == cudaSuccess ? LOT_OK : LOT_ERR_CUDA; }

} // namespace

extern "C" {

size_t lot_window_fwd_workspace_bytes(int dtype, int B, int H, int Hkv, int nq, int nk, int d, int left, int right, int sinks)
{
    if (check_sizes(dtype, B, H, Hkv, nq, nk, d, sinks) != LOT_OK || B == 0 || nq == 0) return 0;
    return fwd_workspace(dtype, B, H, Hkv, band_of(nullptr, nullptr, nq, nk, left, right, sinks), d);
}

int lot_window_fwd(const void *q, const void *k, const void *v, const int32_t *key_len, const int32_t *q_start,
                   int dtype, int B, int H, int Hkv, int nq, int nk, int d, int left, int right, int sinks, float scale,
                   void *out, float *lse, int32_t *status, void *ws, size_t ws_bytes, lot_stream_t stream)
{
    const int st = check_sizes(dtype, B, H, Hkv, nq, nk, d, sinks);
    if (st != LOT_OK) return st;
    if (bad_scale(scale)) return LOT_ERR_INVALID_ARG;
    if (B == 0 || nq == 0) return LOT_OK;
    if (!q || !out || (nk > 0 && (!k || !v))) return LOT_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(lse, 16) || !aligned(key_len, 4) ||
        !aligned(q_start, 4) || !aligned(status, 4))
        return LOT_ERR_INVALID_ARG;
    const size_t need = lot_window_fwd_workspace_bytes(dtype, B, H, Hkv, nq, nk, d, left, right, sinks);
    if (need > 0 && (!ws || !aligned(ws, 256) || ws_bytes < need)) return LOT_ERR_WORKSPACE;
    const Fwd a{band_of(key_len, q_start, nq, nk, left, right, sinks), q, k, v, out, lse, dtype, B, H, Hkv, d, scale, status, ws};
    return done(launch_fwd(a, (cudaStream_t)stream));
}

size_t lot_window_bwd_workspace_bytes(int dtype, int B, int H, int Hkv, int nq, int nk, int d, int left, int right, int sinks)
{
    if (check_sizes(dtype, B, H, Hkv, nq, nk, d, sinks) != LOT_OK || B == 0) return 0;
    const Band b = band_of(nullptr, nullptr, nq, nk, left, right, sinks);
    return (dtype == LOT_F32 ? bwd_f32_workspace : bwd_tc_workspace)(B, H, Hkv, nq, nk, d, b.left, b.right, b.sinks);
}

int lot_window_bwd(const void *q, const void *k, const void *v, const void *out, const float *lse, const void *dout,
                   const int32_t *key_len, const int32_t *q_start,
                   int dtype, int B, int H, int Hkv, int nq, int nk, int d, int left, int right, int sinks, float scale,
                   void *dq, void *dk, void *dv, int32_t *status, void *ws, size_t ws_bytes, lot_stream_t stream)
{
    const int st = check_sizes(dtype, B, H, Hkv, nq, nk, d, sinks);
    if (st != LOT_OK) return st;
    if (bad_scale(scale)) return LOT_ERR_INVALID_ARG;
    if (B == 0 || (nq == 0 && nk == 0)) return LOT_OK;
    if ((nq > 0 && (!q || !out || !lse || !dout || !dq)) || (nk > 0 && (!k || !v || !dk || !dv))) return LOT_ERR_INVALID_ARG;
    for (const void *p : {q, k, v, out, static_cast<const void *>(lse), dout, static_cast<const void *>(dq), static_cast<const void *>(dk), static_cast<const void *>(dv)})
        if (!aligned(p, 16)) return LOT_ERR_INVALID_ARG;
    if (!aligned(key_len, 4) || !aligned(q_start, 4) || !aligned(status, 4)) return LOT_ERR_INVALID_ARG;
    const size_t need = lot_window_bwd_workspace_bytes(dtype, B, H, Hkv, nq, nk, d, left, right, sinks);
    if (need > 0 && (!ws || !aligned(ws, 256) || ws_bytes < need)) return LOT_ERR_WORKSPACE;
    const Bwd a{band_of(key_len, q_start, nq, nk, left, right, sinks), q, k, v, out, dout, lse, dq, dk, dv, static_cast<float *>(ws), dtype, B, H, Hkv, d,
                scale, status};
    return done(launch_bwd(a, (cudaStream_t)stream));
}

size_t lot_cache4_bytes(int num_pages, int Hkv, int page_size, int d)
{
    if (check_cache(1, Hkv, d, page_size, 1, num_pages) != LOT_OK) return 0;
    return (size_t)num_pages * Hkv * 2 * page_size * (d / 2 + d / 8);
}

static int check_rows(const void *k, const void *v, const void *cache, const int32_t *pages, const int32_t *start, const int32_t *count, int dtype, int B,
                      int Hkv, int m, int d, int page_size, int max_pages, int num_pages, const int32_t *status)
{
    if ((dtype != LOT_F32 && dtype != LOT_BF16) || m < 0) return LOT_ERR_INVALID_ARG;
    const int st = check_cache(B, Hkv, d, page_size, max_pages, num_pages);
    if (st != LOT_OK) return st;
    if ((long long)m * d >= (1ll << 31)) return LOT_ERR_UNSUPPORTED_SHAPE;
    if (B == 0 || m == 0) return LOT_OK;
    if (!k || !v || !cache || !pages || !start) return LOT_ERR_INVALID_ARG;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(cache, 16) || !aligned(pages, 4) || !aligned(start, 4) || !aligned(count, 4) || !aligned(status, 4))
        return LOT_ERR_INVALID_ARG;
    return LOT_OK;
}

int lot_cache4_write(const void *k, const void *v, const int32_t *pages, const int32_t *start, const int32_t *count,
                     int dtype, int B, int Hkv, int m, int d, int page_size, int max_pages, int num_pages,
                     void *cache, int32_t *status, lot_stream_t stream)
{
    const int st = check_rows(k, v, cache, pages, start, count, dtype, B, Hkv, m, d, page_size, max_pages, num_pages, status);
    if (st != LOT_OK || B == 0 || m == 0) return st;
    const Cache4 c{static_cast<uint8_t *>(cache), pages, num_pages, max_pages, page_size, Hkv, d};
    return done(launch_write4(c, k, v, start, count, dtype, B, m, status, (cudaStream_t)stream));
}

int lot_cache4_read(const void *cache, const int32_t *pages, const int32_t *start, const int32_t *count,
                    int dtype, int B, int Hkv, int m, int d, int page_size, int max_pages, int num_pages,
                    void *k, void *v, int32_t *status, lot_stream_t stream)
{
    const int st = check_rows(k, v, cache, pages, start, count, dtype, B, Hkv, m, d, page_size, max_pages, num_pages, status);
    if (st != LOT_OK || B == 0 || m == 0) return st;
    const Cache4 c{static_cast<uint8_t *>(const_cast<void *>(cache)), pages, num_pages, max_pages, page_size, Hkv, d};
    return done(launch_read4(c, k, v, start, count, dtype, B, m, status, (cudaStream_t)stream));
}

static int check_attention4(int dtype, int B, int H, int Hkv, int nq, int d, int page_size, int max_pages, int num_pages, int sinks)
{
    const int st = check_cache(B, Hkv, d, page_size, max_pages, num_pages);
    return st != LOT_OK ? st : check_sizes(dtype, B, H, Hkv, nq, 1, d, sinks);
}

size_t lot_cache4_attention_workspace_bytes(int dtype, int B, int H, int Hkv, int nq, int d, int page_size, int max_pages, int left, int sinks)
{
    if (check_attention4(dtype, B, H, Hkv, nq, d, page_size, max_pages, 1, sinks) != LOT_OK || B == 0 || nq == 0) return 0;
    return attend4_workspace(dtype, B, H, Hkv, nq, d, max_pages * page_size, left < 0 || left > kFar ? kFar : left, sinks);
}

int lot_cache4_attention(const void *q, const void *cache, const int32_t *pages, const int32_t *length,
                         int dtype, int B, int H, int Hkv, int nq, int d, int page_size, int max_pages, int num_pages,
                         int left, int sinks, float scale,
                         void *out, float *lse, int32_t *status, void *ws, size_t ws_bytes, lot_stream_t stream)
{
    const int st = check_attention4(dtype, B, H, Hkv, nq, d, page_size, max_pages, num_pages, sinks);
    if (st != LOT_OK) return st;
    if (bad_scale(scale)) return LOT_ERR_INVALID_ARG;
    if (B == 0 || nq == 0) return LOT_OK;
    if (!q || !cache || !pages || !length || !out) return LOT_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(cache, 16) || !aligned(out, 16) || !aligned(lse, 16) || !aligned(pages, 4) || !aligned(length, 4) || !aligned(status, 4))
        return LOT_ERR_INVALID_ARG;
    const size_t need = lot_cache4_attention_workspace_bytes(dtype, B, H, Hkv, nq, d, page_size, max_pages, left, sinks);
    if (need > 0 && (!ws || !aligned(ws, 256) || ws_bytes < need)) return LOT_ERR_WORKSPACE;
    Attend4 a;
    a.cache = Cache4{static_cast<uint8_t *>(const_cast<void *>(cache)), pages, num_pages, max_pages, page_size, Hkv, d};
    a.band = band_of(length, nullptr, nq, max_pages * page_size, left, 0, sinks);
    a.q = q; a.out = out; a.lse = lse; a.dtype = dtype; a.B = B; a.H = H; a.scale = scale; a.status = status; a.ws = ws;
    return done(launch_attend4(a, (cudaStream_t)stream));
}

} // extern "C"
