"""Window attention in 64 bits, with the bounds of what its roundings may cost, and the 4-bit cache's definition in numpy: shared by the
tests of lot_window_fwd, lot_window_bwd and lot_cache4_*."""
import math

import numpy as np
import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}           # half a step, relative: what one rounding may cost


def visible(nq, nk, start, length, left, right, sinks, device="cpu"):
    """[nq, nk] truth values of one batch row."""
    p = (start + torch.arange(nq, device=device)).unsqueeze(1)
    j = torch.arange(nk, device=device).unsqueeze(0)
    ok = j < min(max(length, 0), nk)
    if right >= 0:
        ok = ok & (j <= p + right)
    if left >= 0:
        ok = ok & ((j >= p - left) | (j < sinks))
    return ok.expand(nq, nk)


def reference(q, k, v, starts, lengths, left, right, sinks, scale, dout=None, centre=None):
    """Outputs, lse, gradients in float64 and, for each, how far a correct implementation of q's dtype may be off.

    Counted: scores as sums of d float32 products and the exponent's own error (e, relative error of a weight); sums of up to nk terms in
    float32; for bf16 tensors one rounding of a weight or score gradient before its product; the rounding of the result; for the gradients
    the error of <dout, out> that comes with the rounded output.
    centre (like v, float64): weights are rounded for their product with v - centre, and the product with centre is exact:
    sum_j p_j (1 + r_j) (v_j - c_j) + sum_j p_j c_j is off by sum_j p_j r_j (v_j - c_j), |r_j| at most half a step."""
    half, eps = HALF[q.dtype], 2.0 ** -24
    B, H, nq, d = q.shape
    G, nk = H // k.shape[1], k.shape[2]
    Q, K, V = q.double(), k.double(), v.double()
    w = half if q.dtype == torch.bfloat16 else 0.0                                # rounding of an operand of the second products
    res = {n: torch.zeros_like(Q) for n in ("out", "dq")}
    res.update({n: torch.zeros_like(K) for n in ("dk", "dv")})
    tol = {n: torch.zeros_like(x) for n, x in res.items()}
    res["lse"] = torch.full((B, H, nq), -math.inf, device=q.device, dtype=torch.float64)
    tol["lse"] = torch.zeros_like(res["lse"])
    for b in range(B):
        ok = visible(nq, nk, int(starts[b]), int(lengths[b]), left, right, sinks, q.device)
        used = ok.any(0).unsqueeze(1)
        for h in range(H):
            kk, vv = torch.where(used, K[b, h // G], 0.0), torch.where(used, V[b, h // G], 0.0)
            s = (Q[b, h] @ kk.T * scale).masked_fill(~ok, -math.inf)
            lse = torch.logsumexp(s, 1) if nk else torch.full((nq,), -math.inf, device=q.device, dtype=torch.float64)
            ref = torch.where(torch.isfinite(lse), lse, 0.0).unsqueeze(1)
            p = torch.exp(s - ref).masked_fill(~ok, 0.0)
            out = p @ vv
            # a score's error in units of its exponent: its sum, its scaling, the exponent's argument and the exponential (2 ulp)
            big = (Q[b, h].abs() @ kk.abs().T * scale * ((d + 4) * eps) + (s.masked_fill(~ok, 0.0) - ref).abs() * 4 * eps + 8 * eps).masked_fill(~ok, 0.0)
            e = big + (p * big).sum(1, keepdim=True) + (nk + 8) * eps * 0.5                 # of a normalised weight
            by = vv if centre is None else torch.where(used, V[b, h // G] - centre[b, h // G], 0.0)
            t_out = (p * e) @ vv.abs() + w * (p @ by.abs()) + (half + (nk + 8) * eps) * (p @ vv.abs())
            res["out"][b, h], res["lse"][b, h] = out, lse
            tol["out"][b, h] = t_out
            tol["lse"][b, h] = (p * big).sum(1) + (nk + 8) * eps * 0.5 + lse.abs().masked_fill(~torch.isfinite(lse), 0.0) * 4 * eps
            if dout is None:
                continue
            do = torch.where(ok.any(1, keepdim=True), dout[b, h].double(), 0.0)
            dp, dl = do @ vv.T, (do * out).sum(1, keepdim=True)
            ds = p * (dp - dl) * scale
            t_dl = (t_out * do.abs()).sum(1, keepdim=True) + (d + 4) * eps * (do * out).abs().sum(1, keepdim=True)
            # lse comes rounded to float32 from the forward
            t_p = p * (big + (tol["lse"][b, h].unsqueeze(1) + 4 * eps * (1 + ref.abs())))
            t_ds = scale * (t_p * (dp - dl).abs() + p * (t_dl + (d + 4) * eps * (do.abs() @ vv.abs().T)) + 4 * eps * p * (dp - dl).abs())
            res["dq"][b, h] = ds @ kk
            more = half + (nk + nq * G + 8) * eps
            tol["dq"][b, h] = (t_ds + (w + 8 * eps) * ds.abs()) @ kk.abs() + more * (ds.abs() @ kk.abs())
            res["dk"][b, h // G] += ds.T @ Q[b, h]
            tol["dk"][b, h // G] += (t_ds + (w + 8 * eps) * ds.abs()).T @ Q[b, h].abs() + more * (ds.abs().T @ Q[b, h].abs())
            res["dv"][b, h // G] += p.T @ do
            tol["dv"][b, h // G] += (t_p + (w + 8 * eps) * p).T @ do.abs() + more * (p.T @ do.abs())
    return res, tol


def check(name, got, ref, tol):
    got = got.double()
    assert got.shape == ref.shape
    fin = torch.isfinite(ref)
    assert torch.equal(torch.isfinite(got), fin), f"{name}: finite where it should not be, or the reverse"
    assert torch.equal(got[~fin], ref[~fin]), name
    over = ((got - ref).abs() - tol - 1e-30)[fin]
    if over.numel():
        assert float(over.max()) <= 0, f"{name}: {float((got - ref)[fin].abs().max()):.3e} off, {float(over.max()):.3e} over its bound"


# ---- the cache ------------------------------------------------------------------------------------------------------------


def quantise(x):
    """Values a cache holds of rows x [.., d] (float32 or bf16 tensor): float64 numpy array; and (codes, scale, least)."""
    x = x.detach().float().cpu().numpy().astype(np.float64)
    g = x.reshape(*x.shape[:-1], -1, 32)

    def bf16(a):
        return torch.from_numpy(np.ascontiguousarray(a.astype(np.float32))).to(torch.bfloat16).double().numpy()

    bad = ~np.isfinite(g).all(-1, keepdims=True)
    g0 = np.where(bad, 0.0, g)
    lo, hi = g0.min(-1, keepdims=True), g0.max(-1, keepdims=True)
    s, z = bf16((hi - lo) / 15.0), bf16(lo)
    code = np.where(s > 0, np.clip(np.rint((g0 - z) / np.where(s > 0, s, 1.0)), 0, 15), 0)
    val = np.where(bad, np.nan, z + s * code)
    return val.reshape(x.shape), (code, s, z)


def centres(cache, pages, page, d):
    """least + 8 scale of every value's group, [B, Hkv, tokens, d] float64: the stored word of a token's group is (scale, least)."""
    raw = cache[pages.long()].permute(0, 2, 3, 1, 4)[:, :, 1, :, page * (d // 2):]                # [B, Hkv, pages, page * d / 8]
    par = raw.unflatten(-1, (page, -1)).flatten(2, 3).contiguous().view(torch.bfloat16).double()  # [B, Hkv, tokens, d / 16]
    return (par[..., 1::2] + 8 * par[..., 0::2]).repeat_interleave(32, -1)
