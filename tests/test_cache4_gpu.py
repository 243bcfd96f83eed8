"""The 4-bit cache (lot_cache4_write, lot_cache4_read) against its definition in 64 bits, the attention over it (lot_cache4_attention)
against 64 bits on the values the codes stand for, and a decoder's use of them together."""
import numpy as np
import pytest
import torch

from paper_2509_23436_b200 import binding as lot
from window_testutil import centres, check, quantise, reference

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def make(B, Hkv, tokens, d, page, seed=0, spare=2):
    """An empty cache with its pages in a shuffled order."""
    g = torch.Generator().manual_seed(seed)
    per = (tokens + page - 1) // page
    n = B * per + spare
    pages = torch.randperm(n, generator=g)[:B * per].view(B, per).to(torch.int32).to(DEV)
    return lot.lot_cache4_empty(n, Hkv, page, d, DEV), pages


def rows(seed, B, Hkv, m, d, dtype, kind="normal"):
    g = torch.Generator(device=DEV).manual_seed(seed)
    k, v = (torch.randn(B, Hkv, m, d, generator=g, device=DEV) for _ in range(2))
    if kind == "wide":                                     # all magnitudes
        k, v = (x * torch.exp2(torch.randint(-110, 110, (B, Hkv, m, 1), generator=g, device=DEV).float()) for x in (k, v))
    if kind == "offset":
        k, v = k + 40.0, v * 0.01 - 3.0
    if kind == "grid":                                     # many quotients exactly between two codes
        k, v = (torch.randint(0, 31, (B, Hkv, m, d), generator=g, device=DEV).float() for _ in range(2))
        k[..., 0::32], k[..., 1::32], v[..., 0::32], v[..., 1::32] = 0.0, 30.0, 0.0, 30.0
    return k.to(dtype), v.to(dtype)


def ints(x):
    return torch.tensor(x, device=DEV, dtype=torch.int32)


def bits(x):
    return x.contiguous().view(torch.int16 if x.dtype == BF else torch.int32)


def same(got, want64):
    """Every value is the one the definition gives, rounded to the tensor's type."""
    want = torch.from_numpy(want64).to(torch.float32).to(got.dtype)
    assert torch.equal(torch.isnan(got.cpu()), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got.cpu()), torch.nan_to_num(want))


@pytest.mark.parametrize("kind", ["normal", "wide", "offset", "grid"])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d,page,m,start", [(32, 16, 1, [0, 7, 33]), (64, 16, 50, [0, 1, 15]), (128, 64, 333, [3, 64, 0]), (64, 48, 97, [47, 48, 0]),
                                            (128, 256, 2, [254, 255, 256]), (32, 32, 100, [5, 6, 7])])
def test_write_and_read_back(d, page, m, start, dtype, kind):
    B, Hkv = 3, 2
    cache, pages = make(B, Hkv, max(start) + m, d, page)
    k, v = rows(d + m, B, Hkv, m, d, dtype, kind)
    status = torch.zeros(1, device=DEV, dtype=torch.int32)
    lot.lot_cache4_write(cache, pages, k, v, ints(start), status=status)
    for out in (F32, BF):
        gk, gv = lot.lot_cache4_read(cache, pages, ints(start), m, d=d, dtype=out, status=status)
        same(gk, quantise(k)[0])
        same(gv, quantise(v)[0])
    assert int(status) == 0


@pytest.mark.parametrize("d", [32, 64, 128])
def test_values_of_all_kinds(d):
    """Zeros, constants, the smallest and largest numbers, infinities and NaN, each group by itself."""
    x = torch.zeros(1, 1, 12, d, device=DEV)
    x[0, 0, 1] = 5.0
    x[0, 0, 2] = -1e-40
    x[0, 0, 3, ::2], x[0, 0, 3, 1::2] = 3.3e38, -3.3e38
    x[0, 0, 4, 5] = 1e-45
    x[0, 0, 5, 3] = float("nan")
    x[0, 0, 6, 31] = float("inf")
    x[0, 0, 7] = torch.linspace(-1, 1, d)
    x[0, 0, 8] = torch.linspace(0, 3e-38, d)
    x[0, 0, 9, 0] = -float("inf")
    x[0, 0, 10] = 1e30 * torch.linspace(-1, 1, d)
    x[0, 0, 11] = torch.arange(d) * 1e-32
    for dtype in (F32, BF):
        y = x.to(dtype)
        cache, pages = make(1, 1, 12, d, 16)
        lot.lot_cache4_write(cache, pages, y, y.flip(2).contiguous(), ints([0]))
        k, v = lot.lot_cache4_read(cache, pages, ints([0]), 12, d=d, dtype=F32)
        same(k, quantise(y)[0])
        same(v, quantise(y.flip(2))[0])


def test_token_by_token_is_the_same_as_at_once():
    for d, page in ((64, 16), (128, 32)):
        k, v = rows(5, 2, 3, 70, d, BF)
        a, pages = make(2, 3, 80, d, page)
        b = a.clone()
        lot.lot_cache4_write(a, pages, k, v, ints([0, 9]))
        for i in range(70):
            lot.lot_cache4_write(b, pages, k[:, :, i:i + 1].contiguous(), v[:, :, i:i + 1].contiguous(), ints([i, 9 + i]))
        assert torch.equal(a, b)


def test_only_the_call_s_tokens_are_written():
    """Counts, other pages, rows behind the count on reading; calls with a batch that is all padding."""
    d, page = 64, 16
    cache, pages = make(3, 2, 64, d, page)
    cache.fill_(0xA5)
    before = cache.clone()
    k, v = rows(6, 3, 2, 20, d, BF)
    lot.lot_cache4_write(cache, pages, k, v, ints([3, 0, 30]), count=ints([7, 0, 20]))
    touched = {int(pages[0, 0]), int(pages[2, 1]), int(pages[2, 2]), int(pages[2, 3])}
    for p in range(cache.shape[0]):
        if p not in touched:
            assert torch.equal(cache[p], before[p])
    fk, fv = torch.full((3, 2, 20, d), 9.0, device=DEV, dtype=BF), torch.full((3, 2, 20, d), 9.0, device=DEV, dtype=BF)
    lot.lot_cache4_read(cache, pages, ints([3, 0, 30]), 20, d=d, count=ints([7, 0, 20]), k=fk, v=fv)
    same(fk[0, :, :7], quantise(k[0, :, :7])[0])
    same(fv[2], quantise(v[2])[0])
    assert (fk[0, :, 7:] == 9).all() and (fv[1] == 9).all()
    # neighbours of the tokens in their own pages: what was there still reads the same
    a = lot.lot_cache4_read(before, pages, ints([0, 0, 0]), 3, d=d, dtype=F32)
    b = lot.lot_cache4_read(cache, pages, ints([0, 0, 0]), 3, d=d, dtype=F32)
    assert all(torch.equal(bits(x), bits(y)) for x, y in zip(a, b))
    c, e = (lot.lot_cache4_read(x, pages, ints([10, 0, 0]), 6, d=d, dtype=F32)[1][0] for x in (before, cache))
    assert torch.equal(bits(c), bits(e))


def test_missing_pages_and_places():
    d, page = 64, 16
    cache, pages = make(2, 1, 48, d, page)
    k, v = rows(7, 2, 1, 40, d, BF)
    bad = pages.clone()
    bad[0, 1], bad[1, 0] = -1, cache.shape[0]
    status = torch.zeros(1, device=DEV, dtype=torch.int32)
    lot.lot_cache4_write(cache, bad, k, v, ints([0, 20]), status=status)                 # row 1 runs over the table's end
    assert int(status) == lot.LOT_DEV_PAGE
    status.zero_()
    gk, gv = lot.lot_cache4_read(cache, bad, ints([0, 20]), 40, d=d, status=status)
    assert int(status) == lot.LOT_DEV_PAGE
    want = quantise(k)[0]
    want[0, :, 16:32] = 0
    want[1, :, 28:] = 0
    same(gk, want)
    status.zero_()
    gk, _ = lot.lot_cache4_read(cache, bad, ints([-5, 16]), 8, d=d, status=status)       # places before the first
    assert int(status) == lot.LOT_DEV_PAGE and (gk[0, :, :5] == 0).all() and not (gk[0, :, 5:] == 0).all()
    # attention: tokens of a missing page are not attended to
    q = torch.randn(2, 2, 1, d, device=DEV).to(BF)
    status.zero_()
    out, lse, _ = lot.lot_cache4_attention(q, cache, bad, ints([40, 48]), want_lse=True, status=status)
    assert int(status) == lot.LOT_DEV_PAGE
    kk, vv = lot.lot_cache4_read(cache, pages, ints([0, 0]), 48, d=d, dtype=F32)
    mid = centres(cache, pages, page, d)
    keep = [[j for j in range(40) if not 16 <= j < 32], list(range(16, 48))]
    for b in range(2):
        ref, tol = reference(q[b:b + 1], kk[b:b + 1, :, keep[b]], vv[b:b + 1, :, keep[b]], [len(keep[b]) - 1], [len(keep[b])], -1, 0, 0, d ** -0.5,
                             centre=mid[b:b + 1, :, keep[b]])
        check("out", out[b:b + 1], ref["out"], tol["out"])
        check("lse", lse[b:b + 1], ref["lse"], tol["lse"])


def fill(B, Hkv, tokens, d, page, seed=1):
    cache, pages = make(B, Hkv, tokens, d, page, seed)
    k, v = rows(seed, B, Hkv, tokens, d, BF)
    lot.lot_cache4_write(cache, pages, k, v, ints([0] * B))
    return cache, pages


def attend(q, cache, pages, length, left, sinks, page, scale=None):
    B, H, nq, d = q.shape
    status = torch.zeros(1, device=DEV, dtype=torch.int32)
    out, lse, _ = lot.lot_cache4_attention(q, cache, pages, ints(length), left=left, sinks=sinks, want_lse=True, status=status, scale=scale)
    torch.cuda.synchronize()
    assert int(status) == 0
    cap = pages.shape[1] * page
    k, v = lot.lot_cache4_read(cache, pages, ints([0] * B), cap, d=d, dtype=F32)
    lens = [min(max(n, 0), cap) for n in length]
    ref, tol = reference(q, k, v, [n - nq for n in lens], lens, left, 0, sinks, d ** -0.5 if scale is None else scale, centre=centres(cache, pages, page, d))
    check("out", out, ref["out"], tol["out"])
    check("lse", lse, ref["lse"], tol["lse"])
    return out, lse


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(32, 16), (64, 48), (128, 64), (64, 256)])
@pytest.mark.parametrize("left,sinks", [(-1, 0), (0, 0), (100, 4), (31, 40), (32, 300), (2000, 1)])
def test_attention(d, page, left, sinks, dtype):
    B, H, Hkv = 5, 4, 2
    cache, pages = fill(B, Hkv, 700, d, page)
    q = torch.randn(B, H, 1, d, generator=torch.Generator(device=DEV).manual_seed(d), device=DEV).to(dtype)
    attend(q, cache, pages, [700, 0, 1, 33, 512], left, sinks, page)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv,nq", [(1, 1, 1), (8, 1, 1), (6, 2, 1), (9, 1, 1), (16, 1, 2), (4, 4, 7), (12, 4, 5), (2, 1, 40)])
def test_attention_rows(H, Hkv, nq, dtype):
    cache, pages = fill(3, Hkv, 600, 64, 32)
    q = torch.randn(3, H, nq, 64, generator=torch.Generator(device=DEV).manual_seed(nq), device=DEV).to(dtype)
    attend(q, cache, pages, [600, nq, max(nq - 3, 0)], 90, 3, 32)
    attend(q, cache, pages, [599, 64, 255], -1, 0, 32)


def test_attention_over_a_long_cache_in_splits():
    cache, pages = fill(1, 2, 20000, 128, 64)
    q = torch.randn(1, 8, 1, 128, device=DEV).to(BF)
    assert lot.lib().lot_cache4_attention_workspace_bytes(lot.LOT_BF16, 1, 8, 2, 1, 128, 64, pages.shape[1], -1, 0) > 0
    attend(q, cache, pages, [19999], -1, 0, 64)
    attend(q, cache, pages, [31], -1, 0, 64)               # most splits have nothing
    attend(q * 30, cache, pages, [20000], -1, 0, 64)       # peaked
    attend(q, cache, pages, [1 << 30], -1, 0, 64)          # a length past the table is cut


def test_attention_reads_no_page_it_does_not_need():
    """Window and sinks: entries of pages in between, and behind the length, may be anything; what lies there too."""
    d, page = 64, 16
    cache, pages = fill(2, 2, 400, d, page)
    q = torch.randn(2, 4, 1, d, device=DEV).to(BF)
    want = attend(q, cache, pages, [333, 200], 50, 3, page)
    loose = pages.clone()
    loose[0, 1:17], loose[0, 21:] = -7, 1 << 30
    loose[1, 1:9], loose[1, 13:] = 1 << 30, -1
    status = torch.zeros(1, device=DEV, dtype=torch.int32)
    got = lot.lot_cache4_attention(q, cache, loose, ints([333, 200]), left=50, sinks=3, want_lse=True, status=status)
    assert int(status) == 0 and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # tokens of the needed pages that no query sees: NaN parameters change nothing
    nan = torch.full((2, 2, 400, d), float("nan"), device=DEV, dtype=BF)
    lot.lot_cache4_write(cache, pages, nan[:, :, :67].contiguous(), nan[:, :, :67].contiguous(), ints([333, 200]))
    lot.lot_cache4_write(cache, pages, nan[:, :, :13].contiguous(), nan[:, :, :13].contiguous(), ints([3, 3]))
    got = lot.lot_cache4_attention(q, cache, pages, ints([333, 200]), left=50, sinks=3, want_lse=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_decoder_s_use_together():
    """A prompt through lot_window_fwd, its keys and values into the cache, then tokens one by one: every step's output is window attention
    over what the cache holds; the prompt's last row and the first step differ by the quantisation alone."""
    B, H, Hkv, n, d, page, left, sinks = 2, 8, 2, 150, 64, 32, 63, 4
    g = torch.Generator(device=DEV).manual_seed(3)
    q, k, v = (torch.randn(B, h, n + 20, d, generator=g, device=DEV).to(BF) for h in (H, Hkv, Hkv))
    cut = lambda x, a, b: x[:, :, a:b].contiguous()  # noqa: E731
    cache, pages = make(B, Hkv, n + 20, d, page)
    prompt, _, _ = lot.lot_window_fwd(cut(q, 0, n), cut(k, 0, n), cut(v, 0, n), left=left, sinks=sinks)
    lot.lot_cache4_write(cache, pages, cut(k, 0, n), cut(v, 0, n), ints([0] * B))
    held = lambda m: lot.lot_cache4_read(cache, pages, ints([0] * B), m, d=d, dtype=BF)  # noqa: E731
    for i in range(n, n + 20):
        lot.lot_cache4_write(cache, pages, cut(k, i, i + 1), cut(v, i, i + 1), ints([i] * B))
        out, lse = attend(cut(q, i, i + 1), cache, pages, [i + 1] * B, left, sinks, page)
        # the dense operator on what the cache reads as (rounded to bf16) gives nearly the same
        hk, hv = held(i + 1)
        dense, _, _ = lot.lot_window_fwd(cut(q, i, i + 1), hk, hv, left=left, sinks=sinks)
        assert float((dense.float() - out.float()).abs().max()) < 0.03
    last, _, _ = lot.lot_cache4_attention(cut(q, n - 1, n), cache, pages, ints([n] * B), left=left, sinks=sinks)
    # codes are within half a scale, a fifteenth of a group's range (about 4): 0.14 of a value and, through the scores, of its weight
    assert float((last.float() - prompt[:, :, -1:].float()).abs().max()) < 1.0


def test_streams_and_graphs():
    d, page = 128, 64
    cache, pages = fill(2, 2, 5000, d, page)
    q = torch.randn(2, 8, 1, d, device=DEV).to(BF)
    length = ints([5000, 4000])
    want = lot.lot_cache4_attention(q, cache, pages, length, want_lse=True)[:2]
    outs = []
    for _ in range(3):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            outs.append(lot.lot_cache4_attention(q, cache, pages, length, want_lse=True)[:2])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o in outs for a, b in zip(o, want))
    # a step captured once serves every position: start and length are read on the device
    k, v = rows(8, 2, 2, 1, d, BF)
    start, count = ints([10, 20]), ints([11, 21])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        lot.lot_cache4_write(cache, pages, k, v, start)
        out, lse, _ = lot.lot_cache4_attention(q, cache, pages, count, left=300, sinks=2, want_lse=True)
    for at in (100, 101, 2000):
        start.fill_(at)
        count.fill_(at + 1)
        graph.replay()
        torch.cuda.synchronize()
        a, b = attend(q, cache, pages, [at + 1] * 2, 300, 2, page)
        assert torch.equal(a, out) and torch.equal(b, lse)
