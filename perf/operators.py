"""Window attention with sinks, and the 4-bit cache with the attention that reads it: the calls users make, their plain forms and
their 64-bit definitions.

A case names one pass with its sizes; prepare() makes what a user's program holds before it, run() makes it.

  fwd     lot_window_fwd: a prompt or an encoder's layer; with nq = 1 a decoder's next token over tensors of keys and values
  train   lot_window_fwd and lot_window_bwd: one layer's part of a training step; returns the output and all gradients
  write   lot_cache4_write of new tokens, and lot_cache4_read of the same ones
  read    lot_cache4_read of whole sequences
  attend  lot_cache4_attention: the next tokens of a batch over their pages
"""
import math

import torch

own = False

DEV = "cuda"
_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
GROUP = 32


def _case(name, op, dtype, B, H, Hkv, nq, nk, d, left, right, sinks, **options):
    """left, right: keys visible before and after a query's own position (-1: all); sinks: first keys that stay visible.
    ragged: sequence lengths (or key lengths) differ over the batch.  page: tokens of a cache page (cache operators)."""
    c = dict(op=op, dtype=dtype, B=B, H=H, Hkv=Hkv, nq=nq, nk=nk, d=d, left=left, right=right, sinks=sinks, ragged=False, page=64)
    c.update(options)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # local attention of an image encoder's layer in float32: a band of 32 patches to each side, the class token always visible
        _case("image-local-f32", "fwd", "f32", 32, 3, 3, 197, 197, 64, 32, 32, 1),
        # a long prompt through one decoder layer, four query heads to a key head, wide heads
        _case("prompt-n16384-d128-bf16", "fwd", "bf16", 4, 8, 2, 16384, 16384, 128, 4095, 0, 4),
        # the next token of 64 sequences of different lengths over bf16 keys and values
        _case("token-b64-bf16", "fwd", "bf16", 64, 16, 4, 1, 8192, 128, 4095, 0, 4, ragged=True),
        # training: a batch of padded sentences, bidirectional band, class token visible, three query heads to a key head
        _case("train-n512-masked-bf16", "train", "bf16", 16, 12, 4, 512, 512, 64, 64, 64, 1, ragged=True),
        # training: a long document through a causal layer
        _case("train-n16384-bf16", "train", "bf16", 1, 16, 16, 16384, 16384, 64, 1023, 0, 4),
        # training in float32 at an odd length and narrow heads
        _case("train-n1001-d32-f32", "train", "f32", 2, 8, 4, 1001, 1001, 32, 255, 0, 2),
        # one token of eight sequences goes into the cache: the smallest call
        _case("write-token-bf16", "write", "bf16", 8, 8, 8, 1, 2048, 64, -1, 0, 0, ragged=True),
        # a prompt's keys and values go into the cache
        _case("write-prompt-bf16", "write", "bf16", 4, 8, 8, 8192, 8192, 128, -1, 0, 0),
        # a short prefix comes back in float32, pages of 16 tokens ...
        _case("read-prefix-f32", "read", "f32", 2, 4, 4, 777, 1000, 64, -1, 0, 0, page=16),
        # ... and whole long sequences in bf16
        _case("read-long-bf16", "read", "bf16", 8, 8, 8, 8192, 8192, 128, -1, 0, 0),
        # the next token of one sequence, window and sinks: latency
        _case("attend-b1-window-bf16", "attend", "bf16", 1, 16, 4, 1, 4001, 64, 1023, 0, 4, page=16),
        # the next token of a serving batch over all of its caches
        _case("attend-b32-bf16", "attend", "bf16", 32, 32, 8, 1, 16384, 128, -1, 0, 0, ragged=True),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["fwd", "fwd", "train", "train", "write", "read", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    Hkv = rng.choice([1, 2, 3, 4, 8])
    G = rng.choice([1, 1, 2, 3, 4, 6, 8])
    ragged = rng.random() < 0.5
    sinks = rng.choice([0, 1, 4, rng.randint(2, 130)])
    if op in ("fwd", "train"):
        d = rng.choice([8, 32, 40, 64, 64, 96, 128])
        if op == "fwd" and rng.random() < 0.35:                    # the next token, or a few, over keys of earlier ones
            nq, nk = rng.choice([1, 1, rng.randint(2, 9)]), log(16, 16384)
            left, right, B = rng.choice([-1, log(16, 8192)]), 0, log(1, 64)
        else:
            nq = nk = log(16, 8192 if dtype == "bf16" else 2048)
            if op == "fwd" and rng.random() < 0.3:                 # a chunk behind a prefix
                nq = rng.randint(1, nk)
            left, right = log(8, 2048), 0
            if rng.random() < 0.4:
                right = log(8, 1024)
            B = log(1, 16)
        span = lambda: B * Hkv * G * nq * min(nk, (nk if left < 0 else left) + right + 1 + sinks)  # noqa: E731
        most = (1 << 28) if dtype == "bf16" else (1 << 26)
        while span() > most and B > 1:
            B = (B + 1) // 2
        while span() > most and G > 1:
            G = (G + 1) // 2
        return _case(None, op, dtype, B, Hkv * G, Hkv, nq, nk, d, left, right, sinks, ragged=ragged)
    d = rng.choice([32, 64, 64, 128, 128])
    page = rng.choice([16, 32, 48, 64, 128, 256])
    B = log(1, 32)
    nk = log(16, 16384)
    while B > 1 and B * Hkv * nk * d > (1 << 27):
        B = (B + 1) // 2
    if op == "attend":
        nq = rng.choice([1, 1, 1, rng.randint(2, 8)])
        return _case(None, op, dtype, B, Hkv * G, Hkv, min(nq, nk), nk, d, rng.choice([-1, log(16, 8192)]), 0, sinks, ragged=ragged, page=page)
    nq = rng.choice([1, nk, rng.randint(1, nk)])
    return _case(None, op, dtype, B, Hkv, Hkv, nq, nk, d, -1, 0, 0, ragged=ragged, page=page)


# ---- what a user's program holds ------------------------------------------------------------------------------------------


def _quantise(x):
    """Codes 0..15, scale and least value of groups of 32 channels: ([.., d] float) -> codes [.., d], s, z [.., d/32] bf16.  In 64 bits: the
    quotient decides a rounding."""
    g = x.double().unflatten(-1, (-1, GROUP))
    lo, hi = g.amin(-1), g.amax(-1)
    s, z = ((hi - lo) / 15.0).to(torch.float32).to(torch.bfloat16), lo.to(torch.float32).to(torch.bfloat16)
    sd = s.double().unsqueeze(-1)
    codes = torch.round((g - z.double().unsqueeze(-1)) / torch.where(sd == 0, torch.ones_like(sd), sd)).clamp(0, 15)
    codes = torch.where(sd == 0, torch.zeros_like(codes), codes)
    return codes.to(torch.uint8).flatten(-2), s, z


def _order(d, side, dev):
    """Channel of every nibble of a stored row, low nibble of byte 0 first; side 0: keys, 1: values."""
    w = d // GROUP
    nib = torch.arange(d, device=dev)
    if side == 0:                                                  # word t w + group: channels 8 t .. 8 t + 7 of the group
        word, i = nib // 8, nib % 8
        return (word % w) * GROUP + (word // w) * 8 + i
    half, i = nib // 4, nib % 4                                    # half g w + group: channels g, 8 + g, 16 + g, 24 + g of the group
    return (half % w) * GROUP + i * 8 + half // w


def _places(at, d, side):
    """Bytes of a page's code area that the row of place `at` [..] of the page takes: [.., d/2]."""
    byte = torch.arange(d // 2, device=at.device)
    if side == 0:                                                  # keys: one row after the other
        return at.unsqueeze(-1) * (d // 2) + byte
    # values: blocks of 16 tokens, [token / 8][g][token / 2 % 4][group][token % 2] halves
    w = d // GROUP
    half, low = byte // 2, byte % 2
    g, group = half // w, half % w
    tok = (at % 16).unsqueeze(-1)
    unit = ((tok // 8 * 32 + g * 4 + tok // 2 % 4) * w + group) * 2 + tok % 2
    return (at // 16).unsqueeze(-1) * (8 * d) + unit * 2 + low


def _areas(state, cache):
    """Code and parameter areas of the pages: [pages, Hkv, 2, page d/2], [pages, Hkv, 2, page, d/8] bytes."""
    c = state["case"]
    cut = c["page"] * (c["d"] // 2)
    blk = cache.view(cache.shape[0], c["Hkv"], 2, -1)
    return blk[..., :cut], blk[..., cut:].unflatten(-1, (c["page"], c["d"] // 8))


def _rows(state, pos):
    """Page and place of the tokens pos [B, m] of every sequence: [B, m] each."""
    page = state["case"]["page"]
    return torch.gather(state["pages"].long(), 1, pos // page), pos % page


def _plain_write(state, cache, k, v, pos):
    """Rows k, v [B, Hkv, m, d] into the pages at positions pos [B, m]."""
    d = state["case"]["d"]
    codes, pars = _areas(state, cache)
    pg, at = _rows(state, pos)
    for side, x in enumerate((k, v)):
        code, s, z = _quantise(x)
        n = code[..., _order(d, side, x.device)]
        codes[:, :, side][pg.unsqueeze(-1), :, _places(at, d, side)] = (n[..., 0::2] | (n[..., 1::2] << 4)).permute(0, 2, 3, 1)
        pars[:, :, side][pg, :, at] = torch.stack([s, z], -1).view(torch.uint8).flatten(-2).transpose(1, 2)


def _plain_read(state, cache, pos):
    """Values of the tokens pos [B, m]: k, v [B, Hkv, m, d] float32."""
    d = state["case"]["d"]
    codes, pars = _areas(state, cache)
    pg, at = _rows(state, pos)
    got = []
    for side in (0, 1):
        b = codes[:, :, side][pg.unsqueeze(-1), :, _places(at, d, side)].permute(0, 3, 1, 2)          # [B, Hkv, m, d/2]
        par = pars[:, :, side][pg, :, at].transpose(1, 2).contiguous().view(torch.bfloat16).unflatten(-1, (-1, 2)).float()
        nib = torch.stack([b & 15, b >> 4], -1).flatten(-2).float()
        val = torch.empty_like(nib)
        val[..., _order(d, side, b.device)] = nib
        got.append((par[..., 1:2] + par[..., 0:1] * val.unflatten(-1, (-1, GROUP))).flatten(-2))
    return got


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt = _DTYPES[c["dtype"]]
    B, H, Hkv, nq, nk, d = (c[x] for x in ("B", "H", "Hkv", "nq", "nk", "d"))

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    def lengths(lo):
        if not c["ragged"]:
            return torch.full((B,), nk, device=DEV, dtype=torch.int32)
        return torch.randint(max(lo, nk // 2), nk + 1, (B,), generator=g, device=DEV, dtype=torch.int32)

    # keys have a few channels of larger spread and an offset, the first ones draw attention, as trained layers' do
    mean, spread = normal(Hkv, 1, d), 1.0 + 2.0 * (torch.rand(Hkv, 1, d, generator=g, device=DEV) < 0.05)
    state = {"case": c}
    if c["op"] in ("fwd", "train", "attend"):
        q = normal(B, H, nq, d) + 0.5 * mean.repeat_interleave(H // Hkv, 0)
        state["q"] = q.to(dt)
        state["scale"] = d ** -0.5

    def key_value(m):
        k = normal(B, Hkv, m, d) * spread + 0.3 * mean
        k[:, :, :c["sinks"]] += 0.7 * mean
        return k, normal(B, Hkv, m, d)

    if c["op"] in ("fwd", "train"):
        k, v = key_value(nk)
        state.update(k=k.to(dt), v=v.to(dt), key_len=None, q_start=None)
        if c["ragged"]:
            state["key_len"] = lengths(min(nq, nk))
            # padded rows of equal numbers of queries and keys stand at their own places; else the last query is the last token
            if nq != nk:
                state["q_start"] = state["key_len"] - nq
        if c["op"] == "train":
            state["dout"] = normal(B, H, nq, d).to(dt)
        return state
    page = c["page"]
    per = (nk + page - 1) // page
    total = B * per + 3
    state["pages"] = torch.randperm(total, generator=g, device=DEV)[:B * per].view(B, per).to(torch.int32)
    state["cache"] = torch.zeros(total, Hkv, 2, page * (d // 2 + d // 8), device=DEV, dtype=torch.uint8)
    state["length"] = lengths(nq)
    state["start"] = state["length"] - nq
    if c["op"] == "write":
        k, v = key_value(nq)
        state.update(k=k.to(dt), v=v.to(dt))
    else:
        pos = torch.arange(nk, device=DEV).expand(B, nk)
        step = max(1, (1 << 25) // (B * Hkv * d))
        for at in range(0, nk, step):
            k, v = key_value(min(step, nk - at))
            _plain_write(state, state["cache"], k, v, pos[:, at:at + step])
    return state


# ---- the plain forms ------------------------------------------------------------------------------------------------------


def _visible(c, q_start, key_len):
    """Blocks of queries and the keys that any of a block may see: (index [B, nb, L] of keys, mask [B, nb, c, L], c)."""
    nq, nk, left, right, sinks = c["nq"], c["nk"], c["left"], c["right"], c["sinks"]
    rows = nq if left < 0 or right < 0 else min(nq, 512)
    nb = (nq + rows - 1) // rows
    pos = q_start.long()[:, None, None] + torch.arange(nb * rows, device=DEV).view(1, nb, rows)              # [B, nb, rows]
    whole = left < 0 or right < 0 or rows + left + right + sinks >= nk
    if whole:
        j = torch.arange(nk, device=DEV).expand(pos.shape[0], nb, nk)
    else:                                                          # the first keys apart, for rows whose band has passed them
        band = pos[:, :, :1] - left + torch.arange(rows + left + right, device=DEV)
        j = torch.cat([torch.arange(sinks, device=DEV).expand(pos.shape[0], nb, sinks), band], -1)
    p, jj = pos.unsqueeze(-1), j.unsqueeze(2)
    seen = jj >= p - left if left >= 0 else torch.ones_like(jj >= p)
    if whole:
        seen = seen | (jj < sinks)
    else:
        seen = seen ^ (torch.arange(j.shape[-1], device=DEV) < sinks)
    if right >= 0:
        seen = seen & (jj <= p + right)
    seen = seen & (jj >= 0) & (jj < key_len.long()[:, None, None, None])
    seen = seen & (torch.arange(nb * rows, device=DEV).view(1, nb, rows, 1) < nq)
    return j.clamp(0, nk - 1), seen, rows


def _blocks(x, rows):
    """[B, H, n, d] -> [B, H, nb, rows, d] float32, zeros behind the end."""
    n = x.shape[2]
    nb = (n + rows - 1) // rows
    return torch.nn.functional.pad(x.float(), (0, 0, 0, nb * rows - n)).unflatten(2, (nb, rows))


def _take(x, j):
    """Rows j [B, nb, L] of x [B, Hkv, n, d]: [B, Hkv, 1, nb, L, d] float32."""
    b = torch.arange(j.shape[0], device=x.device)[:, None, None]
    return x[b, :, j].permute(0, 3, 1, 2, 4).float().unsqueeze(2)


def _weights(q, kj, seen, scale):
    s = torch.matmul(q, kj.transpose(-1, -2)).mul_(scale)
    s = s.masked_fill_(~seen[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = (s - m).exp_()
    total = p.sum(-1, keepdim=True)
    lse = torch.log(total) + m
    return p.div_(torch.where(total == 0, torch.ones_like(total), total)), lse


def _starts(state):
    c = state["case"]
    key_len, q_start = state.get("key_len"), state.get("q_start")
    if key_len is None:
        key_len = torch.full((c["B"],), c["nk"], device=DEV)
    if q_start is None:
        q_start = torch.full((c["B"],), c["nk"] - c["nq"], device=DEV)
    return q_start, key_len


def _join(x, n):
    """[B, Hkv, G, nb, rows, ..] -> [B, H, n, ..]"""
    return x.flatten(1, 2).flatten(2, 3)[:, :, :n]


def _plain_fwd(state):
    c = state["case"]
    j, seen, rows = _visible(c, *_starts(state))
    q = _blocks(state["q"], rows).unflatten(1, (c["Hkv"], -1))
    p, lse = _weights(q, _take(state["k"], j), seen, state["scale"])
    o = _join(torch.matmul(p, _take(state["v"], j)), c["nq"])
    return [o.to(state["q"].dtype), _join(lse, c["nq"]).squeeze(-1)]


def _plain_train(state):
    c = state["case"]
    dt = state["q"].dtype
    j, seen, rows = _visible(c, *_starts(state))
    heads = (c["Hkv"], -1)
    q, do = _blocks(state["q"], rows).unflatten(1, heads), _blocks(state["dout"], rows).unflatten(1, heads)
    kj, vj = _take(state["k"], j), _take(state["v"], j)
    p, lse = _weights(q, kj, seen, state["scale"])
    o = torch.matmul(p, vj)
    dp = torch.matmul(do, vj.transpose(-1, -2))
    ds = p * (dp - (do * o).sum(-1, keepdim=True)) * state["scale"]
    dq = torch.matmul(ds, kj)
    where = (j + torch.arange(c["B"], device=DEV)[:, None, None] * c["nk"]).flatten()
    grads = []
    for w, x in ((ds, q), (p, do)):
        part = torch.matmul(w.transpose(-1, -2), x).sum(2)                              # [B, Hkv, nb, L, d]
        full = torch.zeros(c["B"] * c["nk"], c["Hkv"], c["d"], device=DEV)
        full.index_add_(0, where, part.permute(0, 2, 3, 1, 4).flatten(0, 2))
        grads.append(full.unflatten(0, (c["B"], c["nk"])).transpose(1, 2))
    return [_join(o, c["nq"]).to(dt), _join(dq, c["nq"]).to(dt), grads[0].to(dt), grads[1].to(dt)]


def _plain_attend(state):
    c = state["case"]
    j, seen, rows = _visible(c, state["start"], state["length"])
    q = _blocks(state["q"], rows).unflatten(1, (c["Hkv"], -1))
    k, v = _plain_read(state, state["cache"], j.flatten(1))
    k, v = (x.unflatten(2, tuple(j.shape[1:])).unsqueeze(2) for x in (k, v))
    p, lse = _weights(q, k, seen, state["scale"])
    o = _join(torch.matmul(p, v), c["nq"])
    return [o.to(state["q"].dtype), _join(lse, c["nq"]).squeeze(-1)]


def _plain(state):
    c = state["case"]
    if c["op"] == "fwd":
        return _plain_fwd(state)
    if c["op"] == "train":
        return _plain_train(state)
    if c["op"] == "attend":
        return _plain_attend(state)
    pos = state["start"].long()[:, None] + torch.arange(c["nq"], device=DEV)
    if c["op"] == "write":
        _plain_write(state, state["cache"], state["k"], state["v"], pos)
    return [x.to(_DTYPES[c["dtype"]]) for x in _plain_read(state, state["cache"], pos)]


def _own(state):
    from paper_2509_23436_b200 import binding as lot

    c = state["case"]
    if c["op"] in ("fwd", "train"):
        band = dict(left=c["left"], right=c["right"], sinks=c["sinks"], scale=state["scale"], key_len=state["key_len"], q_start=state["q_start"])
        q, k, v = state["q"], state["k"], state["v"]
        out, lse, _ = lot.lot_window_fwd(q, k, v, want_lse=True, **band)
        if c["op"] == "fwd":
            return [out, lse]
        dq, dk, dv, _ = lot.lot_window_bwd(q, k, v, out, lse, state["dout"], **band)
        return [out, dq, dk, dv]
    if c["op"] == "attend":
        out, lse, _ = lot.lot_cache4_attention(state["q"], state["cache"], state["pages"], state["length"], left=c["left"], sinks=c["sinks"],
                                               scale=state["scale"], want_lse=True)
        return [out, lse]
    if c["op"] == "write":
        lot.lot_cache4_write(state["cache"], state["pages"], state["k"], state["v"], state["start"])
    return list(lot.lot_cache4_read(state["cache"], state["pages"], state["start"], c["nq"], d=c["d"], dtype=_DTYPES[c["dtype"]]))


def run(state):
    if own:
        return _own(state)
    return _plain(state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------


def _pairs(c):
    """Visible (query, key) pairs of one head of one full-length row, and how many keys any query sees."""
    start, total = c["nk"] - c["nq"], 0
    lowest = c["nk"]
    for i in range(c["nq"]):
        p = start + i
        hi = c["nk"] if c["right"] < 0 else min(c["nk"], p + c["right"] + 1)
        lo = 0 if c["left"] < 0 else min(hi, max(0, p - c["left"]))
        total += hi - lo + min(lo, c["sinks"])
        lowest = min(lowest, lo)
    return total, c["nk"] - lowest + min(lowest, c["sinks"])


def work(case):
    c = case
    size = 2 if c["dtype"] == "bf16" else 4
    B, H, Hkv, nq, nk, d = (c[x] for x in ("B", "H", "Hkv", "nq", "nk", "d"))
    part = 0.75 if c["ragged"] else 1.0                            # lengths are drawn from the upper half
    stored = d // 2 + d // 8
    if c["op"] in ("write", "read"):
        rows = 2 * B * Hkv * nq
        return {"bytes": rows * (stored + d * size + (stored + d * size if c["op"] == "write" else 0)), "flops": 0}
    pairs, seen = _pairs(c)
    if c["left"] >= 0 and nq != nk:
        part = 1.0                                                 # a window of the last tokens: the same number whatever the length
    pairs, seen = pairs * part, seen * part
    rows = B * H * nq
    if c["op"] == "attend":
        return {"bytes": rows * (2 * d * size + 4) + 2 * B * Hkv * seen * stored, "flops": 4 * d * B * H * pairs}
    moved = rows * (2 * d * size + 4) + 2 * B * Hkv * seen * d * size
    if c["op"] == "fwd":
        return {"bytes": moved, "flops": 4 * d * B * H * pairs}
    # the backward reads q, k, v, out, dout, lse and writes three gradients
    moved += rows * (4 * d * size + 4) + 4 * B * Hkv * seen * d * size
    return {"bytes": moved, "flops": 14 * d * B * H * pairs}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------


def _values64(x, c):
    """What the cache holds of rows x: the nearest of the sixteen values of its group."""
    g = x.double().unflatten(-1, (-1, GROUP))
    least, most = g.min(-1, keepdim=True).values, g.max(-1, keepdim=True).values
    step = ((most - least) / 15).float().bfloat16().double()
    base = least.float().bfloat16().double()
    best, held = torch.full_like(g, math.inf), torch.zeros_like(g)
    for code in list(range(0, 16, 2)) + list(range(1, 16, 2)):     # of two as near the even code, which comes first
        val = base + step * code
        off = (g - val).abs()
        held = torch.where(off < best, val, held)
        best = torch.minimum(best, off)
    return held.flatten(-2)


def _stored64(state):
    """k, v [B, Hkv, nk, d] in float64 from the bytes of the pages."""
    c = state["case"]
    d, page = c["d"], c["page"]
    raw = state["cache"][state["pages"].long()].permute(0, 2, 3, 1, 4)                    # [B, Hkv, 2, pages, bytes]
    cut = page * (d // 2)
    codes, par = raw[..., :cut], raw[..., cut:].unflatten(-1, (page, -1)).flatten(3, 4)
    par = par.contiguous().view(torch.int16).to(torch.int32).bitwise_left_shift(16).view(torch.float32).double()
    s, z = par[..., 0::2], par[..., 1::2]
    w, chan = d // GROUP, torch.arange(d, device=DEV)
    group, r, t = chan // GROUP, chan % GROUP, torch.arange(page, device=DEV).unsqueeze(1)
    got = []
    for side in (0, 1):
        if side == 0:                                                                     # nibble of channel (group, r) of place t of a page
            nib = t * d + ((r // 8) * w + group) * 8 + r % 8
        else:
            nib = t // 16 * 16 * d + ((t % 16 // 8 * 32 + r % 8 * 4 + t % 8 // 2) * w + group) * 8 + t % 2 * 4 + r // 8
        b = codes[:, :, side][..., (nib // 2).flatten()].unflatten(-1, (page, d)).flatten(2, 3)
        sh = (4 * (nib % 2)).to(torch.uint8).repeat(b.shape[2] // page, 1)
        got.append(z[:, :, side][..., group] + s[:, :, side][..., group] * ((b >> sh) & 15).double())
    return got


def _attention64(q, k, v, pos, length, c, scale, dout=None):
    """One batch row: q [H, nq, d], k, v [Hkv, nk, d]; rows of queries in pieces.  Output, lse, and the gradients if dout is given."""
    H, nq, d = q.shape
    G, nk = H // k.shape[0], k.shape[1]
    out, lse = torch.zeros(H, nq, d, device=DEV, dtype=torch.float64), torch.full((H, nq), -math.inf, device=DEV, dtype=torch.float64)
    dq, dk, dv = torch.zeros_like(out), torch.zeros(k.shape, device=DEV, dtype=torch.float64), torch.zeros(v.shape, device=DEV, dtype=torch.float64)
    step = 1024
    for at in range(0, nq, step):
        p = (pos + torch.arange(at, min(nq, at + step), device=DEV)).unsqueeze(1)
        least = 0 if c["left"] < 0 else max(0, pos + at - c["left"])
        most = length if c["right"] < 0 else min(length, pos + min(nq, at + step) + c["right"])
        cols = torch.arange(nk, device=DEV)
        cols = cols[((cols >= least) | (cols < c["sinks"])) & (cols < most)]
        if cols.numel() == 0:
            continue
        ok = torch.ones(p.shape[0], cols.numel(), device=DEV, dtype=torch.bool)
        if c["right"] >= 0:
            ok &= cols <= p + c["right"]
        if c["left"] >= 0:
            ok &= (cols >= p - c["left"]) | (cols < c["sinks"])
        for h in range(H):
            kk, vv, qq = k[h // G][cols].double(), v[h // G][cols].double(), q[h, at:at + step].double()
            s = (qq @ kk.T * scale).masked_fill(~ok, -math.inf)
            l = torch.logsumexp(s, -1)
            w = torch.exp(s - torch.where(l == -math.inf, torch.zeros_like(l), l).unsqueeze(1))
            o = w @ vv
            out[h, at:at + step], lse[h, at:at + step] = o, l
            if dout is not None:
                do = dout[h, at:at + step].double()
                ds = w * (do @ vv.T - (do * o).sum(1, keepdim=True)) * scale
                dq[h, at:at + step] = ds @ kk
                dk[h // G].index_add_(0, cols, ds.T @ qq)
                dv[h // G].index_add_(0, cols, w.T @ do)
    return out, lse, dq, dk, dv


def exact(case, seed):
    c = case
    state = prepare(case, seed)
    if c["op"] == "write":
        return [_values64(state["k"], c), _values64(state["v"], c)]
    if c["op"] == "read":
        at = state["start"].long()[:, None, None, None] + torch.arange(c["nq"], device=DEV)[:, None]
        return [torch.gather(x, 2, at.expand(c["B"], c["Hkv"], c["nq"], c["d"])) for x in _stored64(state)]
    if c["op"] == "attend":
        k, v = _stored64(state)
        starts, lens = state["start"], state["length"]
    else:
        k, v = state["k"], state["v"]
        lens = [c["nk"]] * c["B"] if state["key_len"] is None else state["key_len"]
        starts = [c["nk"] - c["nq"]] * c["B"] if state["q_start"] is None else state["q_start"]
    rows = [_attention64(state["q"][b], k[b], v[b], int(starts[b]), int(lens[b]), c, state["scale"],
                         state["dout"][b] if c["op"] == "train" else None) for b in range(c["B"])]
    out, lse, dq, dk, dv = (torch.stack(x) for x in zip(*rows))
    return [out, dq, dk, dv] if c["op"] == "train" else [out, lse]
