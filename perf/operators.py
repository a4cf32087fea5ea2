"""Operators around a decode state held in 4 bits: storing into it, generating from it, forking and moving it.

A case is one pass of one of these kinds ("path"):

  compact  a prompt's kept K and V rows go into the 4-bit state (vatp_compact_q4); its rows are then read back as 16- or
           32-bit rows (vatp_cache_unpack_q4)
  pack     a 16- or 32-bit decode state is put away in 4 bits and brought back (vatp_cache_pack_q4, vatp_cache_unpack_q4)
  decode   `steps` generation steps over one layer's 4-bit state (vatp_decode_step_q4); its rows are then read back, the
           state that belongs to them being the same arrays
  copy     entries of a batch are forked, reordered or joined into another batch (vatp_cache_copy; with 4-bit rows
           vatp_cache_copy_q4, whose result is then read back)

A 4-bit row of d channels consists of groups of 32.  Of a group's values x: lo is the largest bf16 that is not above min x,
sc the smallest bf16 that is not below (max x - lo) / 15 (0 where that is under 2^-100), a code is rint((x - lo) * (1 / sc)) and
stands for lo + code * sc; differences, quotients and products are rounded to 32 bits one by one.  Channel
c = 32 g + 4 j + e (j < 8, e < 4) is a nibble of byte j * (d / 16) + 2 g + e / 2, the low one for an even e.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import torch

own = False          # set by the program that measures: the plain forms, or this library's calls

FREE, KEEP = -1, -2  # entries of a copy's map that name no source


def listed():
    return [
        # the benchmark's layer: LLaMA2-7B shape, 4K prompt, half of it kept
        _case("compact_2k", "compact", "bf16", 1, 32, 128, 4096, 2048, n_recent=128),
        # a wide batch of 8K prompts, a fifth kept
        _case("compact_1638_b8", "compact", "bf16", 8, 32, 128, 8192, 1638, n_recent=256),
        # the smallest state there is, 32-bit rows, put away and brought back (latency)
        _case("pack_tiny_f32", "pack", "f32", 1, 2, 64, 512, 256, n_recent=32),
        # idle sequences of the windowed workload: the history goes along
        _case("pack_window_b4", "pack", "bf16", 4, 32, 128, 2048, 1024, n_recent=10, window=256),
        # the smallest step: two heads of 64 channels in 32 bits
        _decode("decode_tiny_f32", "f32", 1, 2, 64, 256, 32, n_recent=32),
        # generation at the benchmark's shape, one token after the other, replayed from a graph
        _decode("decode_2k", "bf16", 1, 32, 128, 2048, 32, n_recent=128),
        # a wide batch
        _decode("decode_1638_b8", "bf16", 8, 32, 128, 1638, 32, n_recent=256),
        # the windowed workload's steps: probabilities leave the window as they enter it
        _decode("decode_window_b4", "bf16", 4, 32, 128, 1024, 32, n_recent=10, window=256),
        # grouped queries, an odd budget, calls issued one by one from the program without a graph
        _decode("decode_gqa_eager", "bf16", 2, 32, 128, 4001, 16, kv_heads=8, n_recent=128, graph=False),
        # one long sequence with grouped queries: a fifth of a 64K prompt
        _decode("decode_gqa_13k", "bf16", 1, 32, 128, 13107, 16, kv_heads=8, n_recent=512),
        # one prompt forked into eight samples
        _copy("fork_2k", "bf16", False, 1, 8, 32, 128, 2048, 2048, "fork"),
        # sequences of a smaller budget join a running 4-bit batch
        _copy("join_q4_b16", "bf16", True, 12, 16, 32, 128, 1638, 2048, "join", kv_heads=8),
    ]


def draw(rng):
    """Another case of the same ranges.  The caps keep every one cheaper than the widest listed decode run."""
    path = rng.choice(("compact", "pack", "decode", "decode", "decode", "copy"))
    dtype, d = rng.choice((("bf16", 128),) * 5 + (("bf16", 64),) * 2 + (("f32", 64), ("f32", 128)))
    kv = rng.choice((0, 0, 8, 4)) if path in ("decode", "copy") else 0
    heads = 32 if kv else rng.choice((2, 8, 12, 16, 32))
    window = rng.choice((0, 0, 0, 100, 256))
    units = kv or heads
    budget = _log(rng, 64, 8192 if path == "decode" else 4096)
    most = (1 << 15 if window else 1 << 18) if path != "decode" else 1 << 17      # slots over all caches
    budget = min(budget, most // units)
    batch = max(1, min(_log(rng, 1, 16), most // (units * budget)))
    sinks = min(rng.choice((0, 0, 2, 20)), budget // 4)
    recent = min(rng.choice((10, 32, 128, budget // 2)), budget - sinks)
    more = dict(window=window, n_sink=sinks, n_recent=recent)
    if path == "decode":
        return _decode("", dtype, batch, heads, d, budget, rng.choice((8, 16, 24)), kv_heads=kv, graph=rng.random() < 0.7, **more)
    if path == "copy":
        other = max(64, int(budget * rng.uniform(0.5, 1.0)))
        return _copy("", dtype, rng.random() < 0.5, _log(rng, 1, max(batch, 2)), batch, heads, d, min(other, budget), budget,
                     rng.choice(("fork", "reorder", "join")), kv_heads=kv, window=window)
    return _case("", path, dtype, batch, heads, d, int(budget * rng.uniform(1.1, 5.0)) + 1, budget, **more)


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _case(name, path, dtype, batch, heads, head_dim, seq_len, budget, *, kv_heads=0, window=0, n_sink=0, n_recent=0, **more):
    c = {"path": path, "dtype": dtype, "batch": batch, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "seq_len": seq_len,
         "budget": budget, "n_sink": n_sink, "n_recent": n_recent, "window": window, **more}
    return {"name": name, **c} if name else c


def _decode(name, dtype, batch, heads, head_dim, budget, steps, *, graph=True, **kw):
    # the states stand for prompts twice as long as the budget
    return _case(name, "decode", dtype, batch, heads, head_dim, 2 * budget, budget, steps=steps, graph=graph, **kw)


def _copy(name, dtype, q4, from_batch, batch, heads, head_dim, from_budget, budget, kind, **kw):
    return _case(name, "copy", dtype, batch, heads, head_dim, 2 * budget, budget, q4=q4, from_batch=from_batch, from_budget=from_budget,
                 kind=kind, **kw)


# ------------------------------------------------------------------------------------------------ the 4-bit format
def _bits(x):
    return x.view(torch.int32)


def _bf16_below(x):
    """The largest bf16 values that are not above the fp32 values x, as fp32."""
    b = _bits(x)
    cut = b & -65536
    return torch.where((x < 0) & (cut != b), cut + 65536, cut).view(torch.float32)


def _bf16_above(x):
    """The smallest bf16 values that are not below the fp32 values x >= 0, as fp32."""
    return ((_bits(x) + 65535) & -65536).view(torch.float32)


def _quantise(x):
    """Rows [..., d] to (codes uint8 [..., d], scales and lows fp32 [..., d / 32], all of them bf16 values)."""
    g = x.float().unflatten(-1, (-1, 32))
    lo = _bf16_below(g.amin(-1))
    sc = _bf16_above((g.amax(-1) - lo) / torch.full_like(lo, 15.0))        # (by a number it would be a product with 1 / 15)
    sc = torch.where(sc < 2.0 ** -100, torch.zeros_like(sc), sc)
    inv = torch.where(sc > 0, 1.0 / sc, torch.zeros_like(sc))
    codes = torch.round((g - lo[..., None]) * inv[..., None]).clamp(max=15.0).to(torch.uint8)
    return codes.flatten(-2), sc, lo


def _to_bytes(codes):
    """codes [..., d] to the bytes of a row [..., d / 2]."""
    c = codes.unflatten(-1, (-1, 8, 2, 2))                     # group, j, e / 2, e mod 2
    return (c[..., 0] | c[..., 1] << 4).transpose(-3, -2).flatten(-3).contiguous()


def _from_bytes(b):
    n = b.shape[-1] // 16                                       # groups
    c = b.unflatten(-1, (8, n, 2)).transpose(-3, -2)
    return torch.stack((c & 15, c >> 4), dim=-1).flatten(-4)


def _store(rows, where, codes, params):
    """Quantises `rows` [..., n, d] into the stored bytes and parameters, where `where` [..., n] says so."""
    c, sc, lo = _quantise(rows)
    codes.copy_(torch.where(where[..., None], _to_bytes(c), codes))
    params.copy_(torch.where(where[..., None, None], torch.stack((sc, lo), dim=-1).to(torch.bfloat16), params))


def _values(codes, params):
    p = params.float()
    return ((_from_bytes(codes).float().unflatten(-1, (-1, 32)) * p[..., :1]) + p[..., 1:]).flatten(-2)


# ------------------------------------------------------------------------------------------------ states
_ROWS16, _ROWS4 = ("k_cache", "v_cache"), ("k_codes", "v_codes", "k_params", "v_params")
_SLOTS, _UNITS, _WINDOW = ("acc", "vnorm", "pos"), ("len", "free_slot", "next_pos", "last_slot"), ("ring", "acc_fixed")


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _params(case, batch=None, budget=None):
    from paper_2406_12335_b200 import vatp as V
    return V.make_params(batch=batch or case["batch"], heads=case["heads"], kv_heads=case["kv_heads"], seq_len=case["seq_len"],
                         head_dim=case["head_dim"], dtype=case["dtype"], budget=budget or case["budget"], n_sink=case["n_sink"],
                         n_recent=case["n_recent"], indicator="window" if case["window"] else "h2o", window=case["window"])


def _empty_state(case, *, q4, batch=None, budget=None, like=None):
    """A state without tokens; like: one whose indicators, norms, positions and history this one shares."""
    if own:
        from paper_2406_12335_b200 import vatp as V
        p = _params(case, batch, budget)
        return V.CacheQ4(p) if q4 else V.Cache(p, share=like) if like is not None else V.Cache(p)
    b, h, d, w = batch or case["batch"], case["kv_heads"] or case["heads"], case["head_dim"], case["window"]
    cap = ((budget or case["budget"]) + 8) & ~7
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    s = SimpleNamespace()
    if q4:
        for x in ("k", "v"):
            setattr(s, x + "_codes", z(b, h, cap, d // 2, dtype=torch.uint8))
            setattr(s, x + "_params", z(b, h, cap, d // 32, 2, dtype=torch.bfloat16))
    else:
        s.k_cache, s.v_cache = z(b, h, cap, d, dtype=_dtype(case)), z(b, h, cap, d, dtype=_dtype(case))
    if like is not None:
        for name in _SLOTS + _UNITS + _WINDOW:
            setattr(s, name, getattr(like, name))
        return s
    s.acc, s.vnorm, s.pos = z(b, h, cap), z(b, h, cap), z(b, h, cap, dtype=torch.int32) - 1
    for name in _UNITS:
        setattr(s, name, z(b, h, dtype=torch.int32))
    s.last_slot -= 1
    s.ring = z(b, h, w, cap) if w else None
    s.acc_fixed = z(b, h, cap, dtype=torch.int64) if w else None
    return s


def _gen(case, seed, stream):
    return torch.Generator(device="cuda").manual_seed(240612335 + 7919 * seed + 104729 * stream)


def _rows(case, seed, n, batch):
    """Keys and values of n tokens as a model's: N(0, 1) keys that lean to a direction of their head at the first two tokens, values
    whose norms differ from token to token."""
    h, d = case["kv_heads"] or case["heads"], case["head_dim"]
    g = _gen(case, seed, 1)
    u = _direction(case, seed, batch)
    k = torch.randn(batch, h, n, d, generator=g, device="cuda")
    k[:, :, :2] += _lean(case) * u
    v = torch.randn(batch, h, n, d, generator=g, device="cuda") * torch.exp(torch.randn(batch, h, n, 1, generator=g, device="cuda"))
    v[:, :, :2] *= 1e-3
    return k.to(_dtype(case)), v.to(_dtype(case))


def _direction(case, seed, batch):
    u = torch.randn(batch, case["kv_heads"] or case["heads"], 1, case["head_dim"], generator=_gen(case, seed, 2), device="cuda")
    return u / u.norm(dim=-1, keepdim=True)


def _lean(case):
    return math.sqrt(math.log(case["seq_len"]) * math.sqrt(case["head_dim"]))


def _kept(case, seed, batch, budget):
    """Ascending positions that a selection keeps: the first, the last and others of the prompt."""
    T, F, R, h = case["seq_len"], case["n_sink"], case["n_recent"], case["kv_heads"] or case["heads"]
    g = _gen(case, seed, 3)
    x = torch.rand(batch, h, T, generator=g, device="cuda")
    x[..., :F] += 2.0
    x[..., T - R:] += 2.0
    return x.topk(budget, dim=-1).indices.sort(dim=-1).values.to(torch.int32)


def _indicator(case, seed, batch, n):
    """Indicators of n tokens as a prompt leaves them: two sinks, the rest falling with the position, log-normal around that."""
    h, T = case["kv_heads"] or case["heads"], case["seq_len"]
    seen = torch.log(T / torch.linspace(1.0, T, n, device="cuda")) + 1.0 / T
    acc = seen * torch.exp(0.3 * torch.randn(batch, h, n, generator=_gen(case, seed, 4), device="cuda"))
    acc[..., :2] += T / 8
    return acc


def _history(case, seed, batch, n):
    """The last w probability rows of n tokens, [batch, heads, w, n]."""
    h, w = case["kv_heads"] or case["heads"], case["window"]
    return torch.exp(torch.randn(batch, h, w, n, generator=_gen(case, seed, 5), device="cuda")) / (2.0 * n)


def _fill(case, seed, s, *, batch=None, budget=None):
    """A pruned prompt's state, full up to its budget."""
    b, B = batch or case["batch"], budget or case["budget"]
    k, v = _rows(case, seed, B, b)
    if hasattr(s, "k_codes"):
        everywhere = torch.ones(k.shape[:3], dtype=torch.bool, device="cuda")
        _store(k, everywhere, s.k_codes[:, :, :B], s.k_params[:, :, :B])
        _store(v, everywhere, s.v_codes[:, :, :B], s.v_params[:, :, :B])
    else:
        s.k_cache[:, :, :B], s.v_cache[:, :, :B] = k, v
    s.pos[:, :, :B] = _kept(case, seed, b, B)
    s.vnorm[:, :, :B] = v.float().abs().sum(-1)
    s.len.fill_(B), s.free_slot.fill_(B), s.next_pos.fill_(case["seq_len"])
    if case["window"]:
        s.ring[..., :B] = _history(case, seed, b, B)
        s.acc_fixed.copy_((s.ring.double() * 2.0 ** 52).long().sum(2))
        s.acc.copy_((s.acc_fixed.double() / 2.0 ** 52).float())
    else:
        s.acc[:, :, :B] = _indicator(case, seed, b, B)
    return s


def _map(case, seed):
    """Which entry of the source each entry of the target takes."""
    n, m, g = case["from_batch"], case["batch"], torch.Generator().manual_seed(seed)
    if case["kind"] == "fork":                       # samples of the same few prompts
        got = (torch.arange(m) * n) // m
    elif case["kind"] == "reorder":                  # a beam search's choice
        got = torch.randint(0, n, (m,), generator=g)
    else:                                            # some go on, some end, the others are new
        got = torch.full((m,), KEEP)
        at = torch.randperm(m, generator=g)
        got[at[:min(n, m)]] = torch.randperm(n, generator=g)[:min(n, m)]
        got[at[min(n, m):][:1]] = FREE
    return got.to(torch.int32)


def prepare(case, seed):
    path = case["path"]
    st = {"case": case, "seed": seed, "path": path, "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    if own:
        st["p"] = _params(case)
    if path == "compact":
        b, T, B = case["batch"], case["seq_len"], case["budget"]
        st["k"], st["v"] = _rows(case, seed, T, b)
        st["kept"] = _kept(case, seed, b, B)
        st["vnorm"] = st["v"].float().abs().sum(-1)
        st["win_rows"] = _history(case, seed, b, T) if case["window"] else None
        if case["window"] > T:                           # (queries before the prompt's first: rows of zeros)
            st["win_rows"][:, :, :case["window"] - T] = 0
        st["attn_acc"] = st["win_rows"].sum(2) if case["window"] else _indicator(case, seed, b, T)
        st["to"] = _empty_state(case, q4=True)
        st["rows"] = _empty_state(case, q4=False, like=st["to"])
    elif path == "pack":
        st["from"] = _fill(case, seed, _empty_state(case, q4=False))
        st["to"], st["rows"] = _empty_state(case, q4=True), _empty_state(case, q4=False)
    elif path == "copy":
        n, Bn = case["from_batch"], case["from_budget"]
        st["from"] = _fill(case, seed, _empty_state(case, q4=case["q4"], batch=n, budget=Bn), batch=n, budget=Bn)
        st["to"] = _fill(case, seed + 1000, _empty_state(case, q4=case["q4"]))
        st["src_of"] = _map(case, seed).cuda()
        if case["q4"]:
            st["rows"] = _empty_state(case, q4=False, like=st["to"])
    else:
        b, hq, h, d, steps = case["batch"], case["heads"], case["kv_heads"] or case["heads"], case["head_dim"], case["steps"]
        st["to"] = _fill(case, seed, _empty_state(case, q4=True))
        st["rows"] = _empty_state(case, q4=False, like=st["to"])
        g, dt = _gen(case, seed, 6), _dtype(case)
        u = _direction(case, seed, b)[None, :, :, 0].repeat_interleave(hq // h, dim=2)
        q = torch.randn(steps, b, hq, d, generator=g, device="cuda") + _lean(case) * u
        k = torch.randn(steps, b, h, d, generator=g, device="cuda")
        v = torch.randn(steps, b, h, d, generator=g, device="cuda") * torch.exp(torch.randn(steps, b, h, 1, generator=g, device="cuda"))
        st["out"] = torch.empty(steps, b, hq, d, dtype=dt, device="cuda")
        st["evicted"] = torch.empty(steps, b, h, dtype=torch.int32, device="cuda")
        # one token's buffers are views that the program makes once
        st["tokens"] = list(zip(q.to(dt), k.to(dt), v.to(dt), st["out"], st["evicted"]))
        if case["graph"]:
            torch.matmul(q[0, 0], k[0, 0].t())           # (the matrix library is set up outside the capture)
            torch.cuda.synchronize()
            st["graph"] = torch.cuda.CUDAGraph()
            with torch.cuda.graph(st["graph"]):
                _steps(st)
    return st


# ------------------------------------------------------------------------------------------------ one pass, plain
def _read_back(s, rows):
    live = (s.pos >= 0)[..., None]
    rows.k_cache.copy_(torch.where(live, _values(s.k_codes, s.k_params).to(rows.k_cache.dtype), rows.k_cache))
    rows.v_cache.copy_(torch.where(live, _values(s.v_codes, s.v_params).to(rows.v_cache.dtype), rows.v_cache))


def _copy_state(a, b):
    for name in _SLOTS + _UNITS + _WINDOW:
        if getattr(a, name) is not None:
            getattr(b, name).copy_(getattr(a, name))


def _compact_plain(st):
    case, s, kept = st["case"], st["to"], st["kept"].long()
    B, T, w = case["budget"], case["seq_len"], case["window"]
    live = torch.ones_like(kept, dtype=torch.bool)
    at = kept[..., None].expand(-1, -1, -1, case["head_dim"])
    _store(st["k"].gather(2, at), live, s.k_codes[:, :, :B], s.k_params[:, :, :B])
    _store(st["v"].gather(2, at), live, s.v_codes[:, :, :B], s.v_params[:, :, :B])
    for to, x in ((s.acc, st["attn_acc"]), (s.vnorm, st["vnorm"])):
        to.zero_()
        to[:, :, :B] = x.gather(2, kept)
    s.pos.fill_(-1)
    s.pos[:, :, :B] = st["kept"]
    s.len.fill_(B), s.free_slot.fill_(B), s.next_pos.fill_(T), s.last_slot.fill_(-1)
    if w:
        s.ring.zero_()
        r = (torch.arange(w, device="cuda") + T - w) % w
        s.ring[:, :, r, :B] = st["win_rows"].gather(3, kept[:, :, None].expand(-1, -1, w, -1))
        s.acc_fixed.copy_((s.ring.double() * 2.0 ** 52).long().sum(2))
        s.acc.copy_((s.acc_fixed.double() / 2.0 ** 52).float())


def _copy_plain(st):
    a, s, src = st["from"], st["to"], st["src_of"].long()
    n = min(a.pos.shape[2], s.pos.shape[2])
    take, free = src >= 0, src == FREE
    src = src.clamp(min=0)

    def put(to, new, where):
        to.copy_(torch.where(where.view(-1, *[1] * (to.dim() - 1)), new, to))

    for name in (_ROWS4 if hasattr(s, "k_codes") else _ROWS16) + _SLOTS + (_WINDOW if s.ring is not None else ()):
        x, to = getattr(a, name), getattr(s, name)
        ring = name == "ring"
        put(to[..., :n] if ring else to[:, :, :n], (x[..., :n] if ring else x[:, :, :n])[src], take)
    s.pos[:, :, n:].masked_fill_(take[:, None, None], -1)
    s.pos.masked_fill_(free[:, None, None], -1)
    for name in _UNITS:
        put(getattr(s, name), getattr(a, name)[src], take)
        getattr(s, name).masked_fill_(free[:, None], -1 if name == "last_slot" else 0)


def _step_plain(st, q, k, v, out, evicted):
    case, s = st["case"], st["to"]
    b, hq, d = q.shape
    h, cap, w, B, F, R = k.shape[1], s.pos.shape[2], case["window"], case["budget"], case["n_sink"], case["n_recent"]
    t, fs = s.next_pos[..., None], s.free_slot[..., None].long()
    slots = torch.arange(cap, device="cuda")
    new = slots == fs
    _store(k[:, :, None].expand(-1, -1, cap, -1), new, s.k_codes, s.k_params)
    _store(v[:, :, None].expand(-1, -1, cap, -1), new, s.v_codes, s.v_params)
    s.pos.copy_(torch.where(new, t, s.pos))
    s.vnorm.copy_(torch.where(new, v.float().abs().sum(-1, keepdim=True), s.vnorm))
    hi = s.len + 1
    live = s.pos >= 0
    logits = torch.matmul(q.float().view(b, h, hq // h, d), _values(s.k_codes, s.k_params).transpose(2, 3)) * d ** -0.5
    logits = logits.masked_fill(~live[:, :, None], -math.inf)
    e = torch.exp(logits - logits.amax(-1, keepdim=True))
    p = e / e.sum(-1, keepdim=True)
    out.copy_(torch.matmul(p, _values(s.v_codes, s.v_params)).reshape(b, hq, d))
    p = p.sum(2) / (hq // h)
    if w:
        now = torch.arange(w, device="cuda")[:, None] == (t % w)[:, :, None]               # the row of this step
        fixed = lambda x: (x.double() * 2.0 ** 52).long()  # noqa: E731
        old = torch.where(now, s.ring, torch.zeros_like(s.ring)).sum(2)
        s.acc_fixed.copy_(torch.where(live, torch.where(new, fixed(p), s.acc_fixed + fixed(p) - fixed(old)), s.acc_fixed))
        s.ring.copy_(torch.where(now & live[:, :, None], p[:, :, None], torch.where(new[:, :, None] & ~now, torch.zeros_like(s.ring), s.ring)))
        s.acc.copy_(torch.where(live, (s.acc_fixed.double() / 2.0 ** 52).float(), s.acc))
    else:
        s.acc.copy_(torch.where(live, torch.where(new, p, s.acc + p), s.acc))
    I = torch.where((s.pos >= F) & (s.pos <= t - R) & live, s.acc * s.vnorm, torch.full_like(s.acc, math.inf))
    least = I == I.amin(-1, keepdim=True)
    out_slot = torch.where(least, s.pos, torch.full_like(s.pos, -1)).argmax(-1)            # among equals the highest position
    full = hi > B
    evicted.copy_(torch.where(full, s.pos.gather(2, out_slot[..., None])[..., 0], torch.full_like(hi, -1)))
    s.pos.masked_fill_(full[..., None] & (slots == out_slot[..., None]), -1)
    s.last_slot.copy_(s.free_slot)
    s.free_slot.copy_(torch.where(full, out_slot.to(torch.int32), hi))
    s.len.copy_(torch.where(full, hi - 1, hi))
    s.next_pos += 1


# ------------------------------------------------------------------------------------------------ one pass
def _steps(st):
    if own:
        from paper_2406_12335_b200 import vatp as V
        for q, k, v, out, evicted in st["tokens"]:
            V.vatp_decode_step_q4(st["p"], st["to"], q, k, v, out, evicted_pos=evicted, dev_status=st["status"])
    else:
        for token in st["tokens"]:
            _step_plain(st, *token)


def _out(s, rows, *, fixed=True):
    # (acc is the float image of the windowed state's integer sums)
    got = {name: getattr(rows, name) for name in _ROWS16}
    got.update({name: getattr(s, name) for name in _SLOTS + _UNITS})
    if s.ring is not None:
        got["ring"] = s.ring
        if fixed:
            got["acc_fixed"] = s.acc_fixed
    return got


def run(st):
    path = st["path"]
    if own:
        from paper_2406_12335_b200 import vatp as V
        p, to = st["p"], st["to"]
    if path == "decode":
        if "graph" in st:
            st["graph"].replay()
        else:
            _steps(st)
    elif path == "compact":
        if own:
            V.vatp_compact_q4(p, st["k"], st["v"], st["attn_acc"], st["vnorm"], st["kept"], to, win_rows=st["win_rows"], dev_status=st["status"])
        else:
            _compact_plain(st)
    elif path == "pack":
        a, s, r = st["from"], st["to"], st["rows"]
        if own:
            V.vatp_cache_pack_q4(p, a, to, dev_status=st["status"])
            V.vatp_cache_unpack_q4(p, to, r, dev_status=st["status"])
        else:
            live = a.pos >= 0
            _store(a.k_cache, live, s.k_codes, s.k_params)
            _store(a.v_cache, live, s.v_codes, s.v_params)
            _copy_state(a, s)
            _read_back(s, r)
            _copy_state(s, r)
        return _out(r, r)
    else:
        if own:
            V.vatp_cache_copy(p, st["from"], to, st["src_of"], dev_status=st["status"])
        else:
            _copy_plain(st)
        if not st["case"]["q4"]:
            return _out(st["to"], st["to"])
    if own:
        V.vatp_cache_unpack_q4(p, to, st["rows"], dev_status=st["status"])
    else:
        _read_back(st["to"], st["rows"])
    got = _out(st["to"], st["rows"], fixed=path != "decode")
    if path == "decode":
        got.update(out=st["out"], evicted=st["evicted"])
    return got


# ------------------------------------------------------------------------------------------------ what a pass needs
def work(case):
    """Inputs read and outputs written once; rows that are read back are read in 4 bits and written once more."""
    d, eb, w = case["head_dim"], 4 if case["dtype"] == "f32" else 2, case["window"]
    units, q_units, B = case["batch"] * (case["kv_heads"] or case["heads"]), case["batch"] * case["heads"], case["budget"]
    row, row4, state = 2 * d * eb, 2 * (d // 2 + d // 8), 12 + (4 * w + 8 if w else 0)
    read_back = units * B * (row4 + row)
    if case["path"] == "decode":
        # K, V; indicator in and out, norm, position; with a window the 64-bit sums in and out and the ring row that leaves and enters
        per_slot = row4 + 16 + (20 if w else 0)
        tokens = 2 * q_units * d * eb + units * row
        return {"bytes": case["steps"] * (units * (B + 1) * per_slot + tokens) + read_back,
                "flops": case["steps"] * q_units * (B + 1) * 4.0 * d}
    if case["path"] == "compact":
        return {"bytes": units * B * (row + row4 + 2 * state + 4) + read_back, "flops": 0}
    if case["path"] == "pack":
        return {"bytes": units * B * (row + row4 + 4 * state) + read_back, "flops": 0}
    m = _map(case, 1)
    h, got, sources = case["kv_heads"] or case["heads"], int((m >= 0).sum()), len({int(x) for x in m if x >= 0})
    entry = h * case["from_budget"] * ((row4 if case["q4"] else row) + state)
    return {"bytes": (got + sources) * entry + (read_back if case["q4"] else 0), "flops": 0}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _stored64(x):
    """What the 4-bit rows of x stand for.  The format's own roundings (to bf16, to 32 bits) are steps of its definition."""
    x = x.double().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    f32 = lambda y: y.float().double()  # noqa: E731
    least, most = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
    lo = least.float().bfloat16()
    lo = torch.where(lo.double() > least, _neighbour(lo, -1), lo).double()
    step = f32(f32(most - lo) / torch.full_like(lo, 15.0))
    sc = step.float().bfloat16()
    sc = torch.where(sc.double() < step, _neighbour(sc, 1), sc).double()
    sc = torch.where(sc < 2.0 ** -100, 0.0 * sc, sc)
    inv = torch.where(sc > 0, f32(1.0 / sc.clamp(min=1e-300)), 0.0 * sc)
    code = f32(f32(x - lo) * inv).round().clamp(max=15.0)
    return (lo + code * sc).flatten(-2)


def _neighbour(x, way):
    """The bf16 value next to x, downwards (-1) or upwards (1); zeros do not occur downwards of a positive number."""
    i = x.view(torch.int16)
    away = torch.where(x < 0, -torch.ones_like(i), torch.ones_like(i)) * way
    at_zero = torch.full_like(i, 1 if way > 0 else -32767)
    return torch.where(x == 0, at_zero, i + away).view(torch.bfloat16)


def exact(case, seed):
    path = case["path"]
    if own:
        return None
    st = prepare({**case, "graph": False}, seed)
    s = st["to"]
    if path == "copy":
        return _exact_copy(case, st)
    if path == "pack":
        a = st["from"]
        live = (a.pos >= 0)[..., None]
        got = {n: torch.where(live, _stored64(getattr(a, n)), torch.zeros((), dtype=torch.float64, device="cuda")) for n in _ROWS16}
        got.update(acc=a.acc.double(), vnorm=a.vnorm.double())
        if case["window"]:
            got["ring"] = a.ring.double()
        return got
    if path == "compact":
        B, cap, kept = case["budget"], s.pos.shape[2], st["kept"].long()
        pad = lambda x, dim: torch.cat((x, torch.zeros(*x.shape[:dim], cap - B, *x.shape[dim + 1:], dtype=x.dtype, device="cuda")), dim)  # noqa: E731
        b, h = torch.arange(kept.shape[0], device="cuda")[:, None, None], torch.arange(kept.shape[1], device="cuda")[None, :, None]
        got = {"k_cache": pad(_stored64(st["k"][b, h, kept]), 2), "v_cache": pad(_stored64(st["v"][b, h, kept]), 2),
               "acc": pad(st["attn_acc"][b, h, kept].double(), 2), "vnorm": pad(st["vnorm"][b, h, kept].double(), 2)}
        if case["window"]:
            w, T = case["window"], case["seq_len"]
            rows = torch.roll(st["win_rows"].double(), (T - w) % w, dims=2)       # row (T - w + r) mod w holds window row r
            got["ring"] = pad(torch.stack([rows[:, :, j][b, h, kept] for j in range(w)], dim=2), 3)
            got["acc"] = got["ring"].sum(2)
        return got
    return _exact_decode(case, st)


def _exact_copy(case, st):
    a, s, m = st["from"], st["to"], st["src_of"].tolist()
    if case["q4"]:
        rows = {n: torch.zeros(*s.pos.shape, case["head_dim"], dtype=torch.float64, device="cuda") for n in _ROWS16}
    else:
        rows = {n: getattr(s, n).double() for n in _ROWS16}
    got = {"acc": s.acc.double(), "vnorm": s.vnorm.double()}
    n = min(a.pos.shape[2], s.pos.shape[2])
    if case["window"]:
        got["ring"] = s.ring.double()
    for i, j in enumerate(m):
        if j == FREE:
            continue
        x, at, cut = (s, i, s.pos.shape[2]) if j == KEEP else (a, j, n)
        for name in rows:
            if not case["q4"]:
                rows[name][i, :, :cut] = getattr(x, name)[at, :, :cut].double()
                continue
            c, p = getattr(x, name[0] + "_codes")[at, :, :cut].int(), getattr(x, name[0] + "_params")[at, :, :cut].double()
            live = (x.pos[at, :, :cut] >= 0).double()
            for g in range(case["head_dim"] // 32):
                for e in range(4):
                    byte = c[..., torch.arange(8, device="cuda") * (case["head_dim"] // 16) + 2 * g + e // 2]
                    code = (byte >> 4 if e % 2 else byte & 15).double()
                    rows[name][i, :, :cut, 32 * g + e:32 * g + 32:4] = (p[..., g, 1:] + code * p[..., g, :1]) * live[..., None]
        if j >= 0:
            got["acc"][i, :, :n], got["vnorm"][i, :, :n] = a.acc[j, :, :n].double(), a.vnorm[j, :, :n].double()
            if case["window"]:
                got["ring"][i, ..., :n] = a.ring[j, ..., :n].double()
    return {**rows, **got}


def _exact_decode(case, st):
    s, B, F, R, w, d = st["to"], case["budget"], case["n_sink"], case["n_recent"], case["window"], case["head_dim"]
    b, h, cap = s.pos.shape
    G, n = case["heads"] // h, b * h
    live_rows = slice(0, B)
    K, Vr = torch.zeros(n, cap, d, dtype=torch.float64, device="cuda"), torch.zeros(n, cap, d, dtype=torch.float64, device="cuda")
    k, v = _rows(case, st["seed"], B, b)
    K[:, live_rows], Vr[:, live_rows] = _stored64(k).view(n, B, d), _stored64(v).view(n, B, d)
    pos, S = s.pos.view(n, cap).long().clone(), s.acc.double().view(n, cap).clone()
    norm = torch.zeros(n, cap, dtype=torch.float64, device="cuda")
    norm[:, live_rows] = v.double().abs().sum(-1).view(n, B)
    hist = s.ring.double().view(n, w, cap).clone() if w else None
    if w:
        S = hist.sum(1)
    unit, outs, place, t = torch.arange(n, device="cuda"), [], torch.full((n,), B, device="cuda"), case["seq_len"]
    ever = pos >= 0
    for q, k, v, _, _ in st["tokens"]:
        K[unit, place], Vr[unit, place] = _stored64(k).view(n, d), _stored64(v).view(n, d)
        pos[unit, place], norm[unit, place] = t, v.double().abs().sum(-1).view(n)
        ever[unit, place] = True
        x = torch.einsum("ngd,ncd->ngc", q.double().view(n, G, d), K) / math.sqrt(d)
        x = torch.softmax(x.masked_fill((pos < 0)[:, None], -math.inf), dim=-1)
        outs.append(torch.einsum("ngc,ncd->ngd", x, Vr).view(b, case["heads"], d))
        x = x.mean(1)
        if w:
            hist[unit, :, place] = 0.0
            hist[:, t % w] = torch.where(pos >= 0, x, hist[:, t % w])
            S = torch.where(pos >= 0, hist.sum(1), S)
        else:
            S[unit, place] = 0.0
            S = S + x
        I = (S * norm).masked_fill((pos < F) | (pos > t - R), math.inf)
        place = I.argmin(-1)
        pos[unit, place] = -1
        t += 1
    last = pos >= 0
    rows = {"k_cache": torch.where(last[..., None], K, 0.0 * K).view(b, h, cap, d), "v_cache": torch.where(last[..., None], Vr, 0.0 * Vr).view(b, h, cap, d)}
    got = {**rows, "acc": S.view(b, h, cap), "vnorm": norm.view(b, h, cap), "out": torch.stack(outs)}
    if w:
        got["ring"] = hist.view(b, h, w, cap)
    return got

