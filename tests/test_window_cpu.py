"""Refusals of window attention and of the 4-bit cache: before any device work, through the C ABI and through the binding."""
import ctypes

import pytest
import torch

from paper_2509_23436_b200 import binding as lot
from paper_2509_23436_b200 import build as lot_build

INVALID, SHAPE, WORKSPACE = 1, 2, 3


@pytest.fixture(scope="module")
def L():
    lot_build.build_lib()
    return lot.lib()


P, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(4100)          # never dereferenced on these paths
BIG = 1 << 40


def fwd(L, q=P, k=P, v=P, key_len=None, q_start=None, dtype=0, B=1, H=2, Hkv=1, nq=4, nk=4, d=64, left=1, right=0, sinks=0, scale=0.1, out=P, lse=None,
        status=None, ws=P, ws_bytes=BIG):
    return L.lot_window_fwd(q, k, v, key_len, q_start, dtype, B, H, Hkv, nq, nk, d, left, right, sinks, scale, out, lse, status, ws, ws_bytes, None)


def bwd(L, q=P, k=P, v=P, out=P, lse=P, dout=P, key_len=None, q_start=None, dtype=0, B=1, H=2, Hkv=1, nq=4, nk=4, d=64, left=1, right=0, sinks=0,
        scale=0.1, dq=P, dk=P, dv=P, status=None, ws=P, ws_bytes=BIG):
    return L.lot_window_bwd(q, k, v, out, lse, dout, key_len, q_start, dtype, B, H, Hkv, nq, nk, d, left, right, sinks, scale, dq, dk, dv, status, ws,
                            ws_bytes, None)


def write(L, k=P, v=P, pages=P, start=P, count=None, dtype=1, B=1, Hkv=1, m=1, d=64, page=16, max_pages=4, num=4, cache=P, status=None):
    return L.lot_cache4_write(k, v, pages, start, count, dtype, B, Hkv, m, d, page, max_pages, num, cache, status, None)


def attend(L, q=P, cache=P, pages=P, length=P, dtype=1, B=1, H=2, Hkv=1, nq=1, d=64, page=16, max_pages=4, num=4, left=-1, sinks=0, scale=0.1, out=P,
           lse=None, status=None, ws=P, ws_bytes=BIG):
    return L.lot_cache4_attention(q, cache, pages, length, dtype, B, H, Hkv, nq, d, page, max_pages, num, left, sinks, scale, out, lse, status, ws,
                                  ws_bytes, None)


BAD_BAND = [(dict(dtype=2), INVALID), (dict(H=3, Hkv=2), INVALID), (dict(Hkv=0), INVALID), (dict(nq=-1), INVALID), (dict(nk=-1), INVALID),
            (dict(sinks=-1), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
            (dict(scale=float("inf")), INVALID), (dict(d=0), INVALID), (dict(d=4), SHAPE), (dict(d=60), SHAPE), (dict(d=136), SHAPE),
            (dict(B=32768, H=1), SHAPE), (dict(nk=1 << 26), SHAPE), (dict(nq=1 << 26), SHAPE), (dict(q=None), INVALID), (dict(q=ODD), INVALID),
            (dict(k=None), INVALID), (dict(v=ODD), INVALID), (dict(key_len=ctypes.c_void_p(4097)), INVALID), (dict(status=ctypes.c_void_p(4098)), INVALID)]


@pytest.mark.parametrize("args,code", BAD_BAND)
def test_window_refuses(L, args, code):
    assert fwd(L, **args) == code
    assert bwd(L, **args) == code


def test_window_refuses_its_own(L):
    assert fwd(L, out=None) == INVALID and fwd(L, lse=ODD) == INVALID
    for name in ("out", "lse", "dout", "dq", "dk", "dv"):
        assert bwd(L, **{name: None}) == INVALID and bwd(L, **{name: ODD}) == INVALID
    need = L.lot_window_bwd_workspace_bytes(0, 1, 2, 1, 4, 4, 64, 1, 0, 0)
    assert need > 0 and need % 256 == 0
    assert bwd(L, ws=None) == WORKSPACE and bwd(L, ws_bytes=need - 1) == WORKSPACE and bwd(L, ws=ODD) == WORKSPACE
    assert fwd(L, B=0) == 0 and fwd(L, nq=0) == 0 and bwd(L, B=0) == 0
    assert L.lot_window_fwd_workspace_bytes(0, 1, 2, 1, 4, 4, 60, 1, 0, 0) == 0
    assert L.lot_window_bwd_workspace_bytes(7, 1, 2, 1, 4, 4, 64, 1, 0, 0) == 0


@pytest.mark.parametrize("args,code", [(dict(dtype=3), INVALID), (dict(d=48), SHAPE), (dict(d=256), SHAPE), (dict(page=8), SHAPE), (dict(page=0), INVALID),
                                       (dict(page=24), SHAPE), (dict(max_pages=0), INVALID), (dict(num=0), INVALID), (dict(max_pages=1 << 25), SHAPE),
                                       (dict(B=-1), INVALID), (dict(Hkv=0), INVALID), (dict(cache=None), INVALID), (dict(cache=ODD), INVALID),
                                       (dict(pages=None), INVALID), (dict(status=ctypes.c_void_p(4098)), INVALID)])
def test_cache_refuses(L, args, code):
    assert write(L, **args) == code
    assert attend(L, **args) == code


def test_cache_refuses_its_own(L):
    assert write(L, m=-1) == INVALID and write(L, k=None) == INVALID and write(L, v=ODD) == INVALID and write(L, start=None) == INVALID
    assert write(L, B=0) == 0 and write(L, m=0) == 0 and write(L, m=1 << 25) == SHAPE
    assert attend(L, H=3, Hkv=2) == INVALID and attend(L, sinks=-1) == INVALID and attend(L, scale=0.0) == INVALID and attend(L, length=None) == INVALID
    assert attend(L, out=ODD) == INVALID and attend(L, B=0) == 0 and attend(L, nq=0) == 0
    need = L.lot_cache4_attention_workspace_bytes(1, 1, 2, 1, 1, 64, 16, 4096, -1, 0)
    assert need > 0
    assert attend(L, max_pages=4096, num=4096, ws=None) == WORKSPACE and attend(L, max_pages=4096, num=4096, ws_bytes=need - 1) == WORKSPACE
    assert L.lot_cache4_bytes(10, 2, 16, 64) == 10 * 2 * 2 * 16 * 40
    assert L.lot_cache4_bytes(10, 2, 16, 48) == 0 and L.lot_cache4_bytes(10, 2, 20, 64) == 0


def test_binding_refuses():
    q, k = torch.zeros(1, 2, 8, 64), torch.zeros(1, 1, 8, 64)
    with pytest.raises(lot.LotError, match="CUDA"):
        lot.lot_window_fwd(q, k, k, left=1)
    with pytest.raises(lot.LotError, match="dtype"):
        lot.lot_window_fwd(q, k.to(torch.bfloat16), k, left=1)
    with pytest.raises(lot.LotError, match="unsupported tensor dtype"):
        lot.lot_window_fwd(q.double(), k.double(), k.double(), left=1)
    with pytest.raises(lot.LotError, match="key_len"):
        lot.lot_window_fwd(q, k, k, left=1, key_len=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(lot.LotError, match="lse"):
        lot.lot_window_bwd(q, k, k, q, torch.zeros(1, 2, 7), q, left=1)
    cache, pages = torch.zeros(3, 1, 2, 16 * 40, dtype=torch.uint8), torch.zeros(1, 2, dtype=torch.int32)
    one = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(lot.LotError, match="cache rows"):
        lot.lot_cache4_read(cache, pages, one, 4, d=128 + 64)
    with pytest.raises(lot.LotError, match="start"):
        lot.lot_cache4_write(cache, pages, k, k, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(lot.LotError, match="CUDA"):
        lot.lot_cache4_attention(q, cache, pages, one)
    with pytest.raises(lot.LotError, match="unsupported sizes"):
        lot.lot_cache4_empty(3, 1, 10, 64, "cpu")
