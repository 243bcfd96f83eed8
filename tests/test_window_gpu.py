"""lot_window_fwd and lot_window_bwd against 64 bits: sizes, masks, head layouts where they can go wrong, empty rows, whatever stands in
places no query sees, streams, devices and graphs."""
import itertools

import pytest
import torch

from paper_2509_23436_b200 import binding as lot
from window_testutil import check, reference

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def draw(seed, B, H, Hkv, nq, nk, d, dtype, spread=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    return (r(B, H, nq, d) * spread).to(dtype), r(B, Hkv, nk, d).to(dtype), r(B, Hkv, nk, d).to(dtype), r(B, H, nq, d).to(dtype)


def both(q, k, v, dout, left, right, sinks, key_len=None, q_start=None, scale=None, backward=True):
    """Runs forward and backward and checks them; returns what they gave."""
    B, H, nq, d = q.shape
    nk = k.shape[2]
    i32 = lambda x: None if x is None else torch.tensor(x, device=DEV, dtype=torch.int32)  # noqa: E731
    band = dict(left=left, right=right, sinks=sinks, scale=scale, key_len=i32(key_len), q_start=i32(q_start))
    status = torch.zeros(1, device=DEV, dtype=torch.int32)
    out, lse, _ = lot.lot_window_fwd(q, k, v, want_lse=True, status=status, **band)
    got = {"out": out, "lse": lse}
    if backward:
        got["dq"], got["dk"], got["dv"], _ = lot.lot_window_bwd(q, k, v, out, lse, dout, status=status, **band)
    torch.cuda.synchronize()
    assert int(status) == 0
    starts = [nk - nq] * B if q_start is None else q_start
    lengths = [nk] * B if key_len is None else key_len
    ref, tol = reference(q, k, v, starts, lengths, left, right, sinks, d ** -0.5 if scale is None else scale, dout if backward else None)
    for n, x in got.items():
        check(n, x, ref[n], tol[n])
    return got


# n, left, right, sinks: tile edges (64, 128, 256), windows of nothing but the own key, wider than the sequence, without limits
BANDS = [(1, 0, 0, 0), (1, -1, -1, 3), (2, 0, 0, 1), (63, 7, 0, 2), (64, 63, 0, 0), (65, 64, 64, 1), (127, -1, 0, 0), (128, 127, 0, 4), (129, 128, 3, 0),
         (200, 0, 0, 0), (255, 16, 16, 1), (256, 1000, 0, 0), (257, 31, 0, 130), (300, -1, -1, 0), (385, 100, 5, 7), (513, 129, 0, 257), (640, 255, 0, 4),
         (700, 0, 300, 2), (1025, 300, 0, 1), (900, -1, 17, 3)]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n,left,right,sinks", BANDS)
def test_bands(n, left, right, sinks, dtype):
    both(*draw(n, 2, 2, 1, n, n, 64, dtype), left, right, sinks)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [8, 16, 24, 32, 40, 64, 72, 96, 104, 128])
def test_widths(d, dtype):
    both(*draw(d, 1, 4, 2, 333, 333, d, dtype), 90, 0, 3)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (3, 1), (6, 2), (8, 8), (10, 2), (16, 1)])
def test_heads(H, Hkv, dtype):
    both(*draw(H, 2, H, Hkv, 290, 290, 32, dtype), 70, 33, 1)


# queries and keys differ in number: a chunk behind a prefix, the next token, more queries than keys (the first see nothing)
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("nq,nk,left,sinks", [(1, 1, -1, 0), (1, 700, 200, 4), (1, 5000, -1, 0), (3, 4100, 2000, 5), (9, 600, 64, 0), (17, 1000, 300, 2),
                                              (100, 777, 128, 3), (500, 130, 40, 1), (129, 2000, -1, 0), (2, 1, 0, 0), (40, 0, 5, 0)])
def test_lengths(nq, nk, left, sinks, dtype):
    both(*draw(nq, 2, 4, 2, nq, nk, 64, dtype), left, 0, sinks)


# more query rows of a key head than one tile of any kernel takes, at the last numbers of queries that count as few and the first that do not
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hkv,nq,nk,d,left,right,sinks", [(1, 3, 1, 7, 2100, 32, -1, 0, 0), (2, 8, 2, 17, 1300, 64, 500, 0, 3), (1, 32, 4, 33, 700, 128, 90, 5, 70),
                                                              (1, 4, 4, 32, 5000, 64, 4000, 0, 1), (1, 6, 2, 64, 900, 96, -1, -1, 0), (1, 2, 1, 65, 900, 64, 200, 0, 2),
                                                              (40, 5, 5, 31, 130, 40, 20, 0, 1), (1, 1, 1, 1, 20000, 128, -1, 0, 0)])
def test_few_queries(B, H, Hkv, nq, nk, d, left, right, sinks, dtype):
    lens = [nk - 11 * b % nk for b in range(B)]
    both(*draw(nq, B, H, Hkv, nq, nk, d, dtype), left, right, sinks, key_len=lens, q_start=[max(n - nq, -nq // 2) for n in lens], backward=False)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("nq,nk", [(300, 300), (1, 900), (5, 900)])
def test_padding_and_starts(nq, nk, dtype):
    """Lengths of zero, one, all and more; positions before the first key and behind the last."""
    lens, starts = [0, 1, 130, nk, nk + 9, 257], [0, 0, 4, nk - nq, -3, 600]
    both(*draw(3, 6, 2, 1, nq, nk, 64, dtype), 60, 0, 2, key_len=lens, q_start=starts)
    both(*draw(4, 6, 2, 1, nq, nk, 64, dtype), 60, 20, 2, key_len=lens)
    both(*draw(5, 6, 2, 1, nq, nk, 40, dtype), -1, -1, 0, key_len=lens, q_start=[-1000, 0, 5000, -(1 << 29), 1 << 29, 100])


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("nq,nk", [(200, 200), (64, 500), (1, 500)])
@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -3.0e38])
def test_nothing_comes_from_places_no_query_sees(nq, nk, junk, dtype):
    q, k, v, dout = draw(9, 2, 2, 2, nq, nk, 64, dtype)
    lens, start, left, sinks = [nk - 37, nk - 100], [nk - nq - 60] * 2, 50, 3
    for b, L in enumerate(lens):
        for x in (k, v):
            x[b, :, L:] = junk
            x[b, :, start[b] + nq:] = junk                     # keys behind every query
            if start[b] - left > sinks:
                x[b, :, sinks:start[b] - left] = junk          # keys the window has passed
    both(q, k, v, dout, left, 0, sinks, key_len=lens, q_start=start)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_peaked_and_flat_scores(dtype):
    """Scores of hundreds, growing along the keys so that the running maximum keeps moving, and all alike."""
    q, k, v, dout = draw(11, 1, 2, 2, 400, 400, 64, dtype, spread=8.0)
    k *= torch.linspace(0.1, 4.0, 400, device=DEV).view(1, 1, -1, 1).to(dtype)
    both(q, k, v, dout, -1, 0, 0)
    both(q, k, v, dout, 100, 0, 1, scale=2.0 ** -20)
    both(torch.zeros_like(q), k, v, dout, 100, 10, 1)


def test_long_sequence_past_one_tile_of_everything():
    q, k, v, dout = draw(12, 1, 2, 1, 5000, 5000, 128, BF)
    both(q, k, v, dout, 1023, 0, 4)


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def _run(q, k, v, dout, **kw):
    out, lse, _ = lot.lot_window_fwd(q, k, v, left=100, right=0, sinks=2, want_lse=True, **kw)
    return (out, lse) + lot.lot_window_bwd(q, k, v, out, lse, dout, left=100, right=0, sinks=2, **kw)[:3]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_repeats_bit_for_bit_on_streams_and_in_a_graph(dtype):
    x = draw(13, 2, 8, 2, 600, 600, 64, dtype)
    want = _run(*x)
    assert _same(want, _run(*x))
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [None, None]
    for i, s in enumerate(side):
        with torch.cuda.stream(s):
            got[i] = _run(*x)
    explicit = _run(*x, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert _same(want, got[0]) and _same(want, got[1]) and _same(want, explicit)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = _run(*x)
    for _ in range(2):
        for h in held:
            h.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert _same(want, held)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_gradients_against_differences(dtype):
    """d(loss) along a random direction, from the forward in 64 bits at two points, against the gradients' inner product."""
    q, k, v, dout = draw(14, 1, 4, 2, 150, 150, 32, dtype)
    got = both(q, k, v, dout, 40, 0, 2)
    g = torch.Generator(device=DEV).manual_seed(1)
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        step = torch.randn(x.shape, generator=g, device=DEV, dtype=torch.float64)
        h, loss = 1e-4, []
        for sign in (1, -1):
            moved = {"dq": q.double(), "dk": k.double(), "dv": v.double()}
            moved[name] = x.double() + sign * h * step
            s = torch.einsum("bhid,bhjd->bhij", moved["dq"], moved["dk"].repeat_interleave(2, 1)) * 32 ** -0.5
            i = torch.arange(150, device=DEV)
            ok = (i[None] <= i[:, None]) & ((i[None] >= i[:, None] - 40) | (i[None] < 2))
            o = torch.softmax(s.masked_fill(~ok, float("-inf")), -1) @ moved["dv"].repeat_interleave(2, 1)
            loss.append(float((o * dout.double()).sum()))
        want, have = (loss[0] - loss[1]) / (2 * h), float((got[name].double() * step).sum())
        # roundings of the gradient are independent of the direction: their sum is far below the bound of them all in one sense
        bound = 2 * (2.0 ** -8 if dtype == BF else 2.0 ** -20) * float((got[name].double() * step).norm()) + 1e-4 * abs(want) + 1e-5
        assert abs(want - have) <= 4 * bound, (name, want, have)


def test_outputs_may_be_given_and_only_they_are_written():
    q, k, v, dout = draw(15, 1, 2, 1, 100, 100, 64, BF)
    out, lse = torch.empty_like(q), torch.empty(1, 2, 100, device=DEV)
    a, b, _ = lot.lot_window_fwd(q, k, v, left=20, out=out, lse=lse)
    assert a is out and b is lse
    c, none, _ = lot.lot_window_fwd(q, k, v, left=20)
    assert none is None and torch.equal(c, out)
    pool = torch.full((3, 1, 1, 100, 64), 7.0, device=DEV, dtype=BF)          # gradients between rows that stay as they were
    lot.lot_window_bwd(q, k, v, out, lse, dout, left=20, dk=pool[1], dv=torch.empty_like(v))
    assert (pool[0] == 7).all() and (pool[2] == 7).all() and not (pool[1] == 7).all()


@pytest.mark.parametrize("raw", [False, True])
def test_a_call_on_another_stream_makes_its_tensors_there(raw):
    """The current stream still writes memory that it has given back: a call on another stream must not get it for its results."""
    q, k, v, dout = draw(17, 2, 4, 2, 300, 300, 64, BF)
    lens, table = torch.full((2,), 300, device=DEV, dtype=torch.int32), torch.arange(10, device=DEV, dtype=torch.int32).view(2, 5)
    cache = lot.lot_cache4_empty(10, 2, 64, 64, DEV)
    lot.lot_cache4_write(cache, table, k, v, torch.zeros(2, device=DEV, dtype=torch.int32))
    side = torch.cuda.Stream()
    stream = side.cuda_stream if raw else side

    def calls(s):
        out, lse, ws = lot.lot_window_fwd(q, k, v, left=50, want_lse=True, stream=s)
        few, _, ws2 = lot.lot_window_fwd(one, k, v, left=-1, stream=s)
        return [out, lse, few, *lot.lot_window_bwd(q, k, v, out, lse, dout, left=50, stream=s)[:3], *lot.lot_cache4_read(cache, table, zero, 300, d=64, stream=s),
                lot.lot_cache4_attention(q, cache, table, lens, left=90, stream=s)[0]]

    one, zero = q[:, :, :1].contiguous(), torch.zeros(2, device=DEV, dtype=torch.int32)
    want = calls(None)
    torch.cuda.synchronize()
    junk = [torch.empty_like(x) for _ in range(3) for x in want]
    torch.cuda._sleep(200_000_000)
    for x in junk:
        x.fill_(float("nan"))
    del junk, x
    got = calls(stream)
    side.synchronize()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_no_queries_no_keys_no_batch():
    for B, nq, nk in itertools.product((0, 1), (0, 5), (0, 5)):
        q, k, v, dout = draw(16, B, 2, 1, nq, nk, 32, F32)
        out, lse, _ = lot.lot_window_fwd(q, k, v, left=3, want_lse=True)
        dq, dk, dv, _ = lot.lot_window_bwd(q, k, v, out, lse, dout, left=3)
        torch.cuda.synchronize()
        if nk == 0 and B and nq:
            assert (out == 0).all() and torch.isinf(lse).all() and (dq == 0).all()
        if nq == 0 and B and nk:
            assert (dk == 0).all() and (dv == 0).all()
