"""The decode state held in 4 bits on the GPU: compaction into it, conversion, generation steps, copies of entries.

Codes, parameters and copies are exact.  Steps are held to bounds that count roundings (tests/q4_reference.py): the logits' 32-bit
sums give a probability a relative error `rel`; the output adds the roundings of its terms and its own to 16 bits.
"""
import os
import subprocess
import sys

import pytest
import torch

from tests import parity as P
from tests import q4_reference as Q

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
STATE = ("acc", "vnorm", "pos", "len", "free_slot", "next_pos", "last_slot")


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(g, *shape, dtype):
    x = torch.randn(*shape, generator=g, device="cuda") * torch.exp(torch.randn(*shape[:-1], 1, generator=g, device="cuda"))
    return x.to(DT[dtype])


def _params(dtype="bf16", b=1, h=3, kv=0, d=128, T=None, B=100, F=0, R=0, window=0, norm="l1", **kw):
    V = P.vatp()
    return V.make_params(batch=b, heads=h, kv_heads=kv, seq_len=T or 2 * B, head_dim=d, dtype=dtype, budget=B, n_sink=F, n_recent=R,
                         indicator="window" if window else "h2o", window=window, norm=norm, **kw)


def _status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def _same_row(rows, codes, params):
    """Stored bytes and parameters are those of the format, for rows [.., d]."""
    c, sc, lo = Q.quantise(rows)
    assert torch.equal(codes, Q.to_bytes(c)), "codes"
    assert torch.equal(params, Q.params(sc, lo)), "parameters"


def _filled(p, n, seed=1, form="q4"):
    """A state of n tokens with rows of the format, indicators, norms and ascending positions."""
    V = P.vatp()
    dtype, d, w, T = "f32" if p.dtype == V.F32 else "bf16", p.head_dim, p.window_w, p.seq_len
    c = V.CacheQ4(p)
    b, h, cap = c.pos.shape
    g = _gen(seed)
    wide = V.Cache(p, share=c)
    wide.k_cache[:, :, :n], wide.v_cache[:, :, :n] = _rows(g, b, h, n, d, dtype=dtype), _rows(g, b, h, n, d, dtype=dtype)
    for x, codes, par in ((wide.k_cache, c.k_codes, c.k_params), (wide.v_cache, c.v_codes, c.v_params)):
        k, sc, lo = Q.quantise(x[:, :, :n])
        codes[:, :, :n], par[:, :, :n] = Q.to_bytes(k), Q.params(sc, lo)
    c.pos[:, :, :n] = (torch.arange(n, device="cuda") * max((T - 1) // max(n, 1), 1)).to(torch.int32)
    c.vnorm[:, :, :n] = wide.v_cache[:, :, :n].float().abs().sum(-1)
    c.len.fill_(n), c.free_slot.fill_(n), c.next_pos.fill_(T)
    if p.indicator == V.IND_WINDOW:
        c.ring[..., :n] = torch.rand(b, h, w, n, generator=g, device="cuda") / max(n, 1)
        c.acc_fixed.copy_((c.ring.double() * 2.0 ** 52).long().sum(2))
        c.acc.copy_((c.acc_fixed.double() / 2.0 ** 52).float())
    else:
        c.acc[:, :, :n] = torch.rand(b, h, n, generator=g, device="cuda") + 0.1
    return c if form == "q4" else wide


def _arrays(c):
    names = (("k_codes", "v_codes", "k_params", "v_params") if hasattr(c, "k_codes") else ("k_cache", "v_cache")) + STATE
    return {n: getattr(c, n) for n in names + (() if c.ring is None else ("ring", "acc_fixed"))}


def _clone(c, p):
    V = P.vatp()
    x = (V.CacheQ4 if hasattr(c, "k_codes") else V.Cache)(p)
    for n, t in _arrays(c).items():
        getattr(x, n).copy_(t)
    return x


def _equal(a, b):
    for n, t in _arrays(a).items():
        assert torch.equal(t, getattr(b, n)), n


# ------------------------------------------------------------------------------------------------ compaction
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("b,h,T,B", [(1, 1, 1, 1), (2, 3, 37, 9), (1, 2, 50, 77), (3, 2, 300, 131), (1, 5, 1000, 256)])
@pytest.mark.parametrize("transposed", [False, True])
def test_compaction(dtype, d, b, h, T, B, transposed):
    """Rows as the format says, everything else as vatp_compact leaves it; rows of slots without a token are left alone."""
    V, g = P.vatp(), _gen(T + B)
    k, v = ((_rows(g, b, T, h, d, dtype=dtype).transpose(1, 2) if transposed else _rows(g, b, h, T, d, dtype=dtype)) for _ in range(2))
    p = V.params_for(k, budget=B)
    acc, vnorm = torch.rand(b, h, T, generator=g, device="cuda"), v.float().abs().sum(-1).contiguous()
    n = min(T, B)
    kept = torch.full((b, h, B), -1, dtype=torch.int32, device="cuda")
    kept[..., :n] = torch.rand(b, h, T, generator=g, device="cuda").topk(n, -1).indices.sort(-1).values
    status, c, ref = _status(), V.CacheQ4(p), V.Cache(p)
    for t in (c.k_codes, c.v_codes):
        t.fill_(0x5a)
    V.vatp_compact_q4(p, k, v, acc, vnorm, kept, c, dev_status=status)
    V.vatp_compact(p, k, v, acc, vnorm, kept, ref, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    for name in STATE:
        assert torch.equal(getattr(c, name), getattr(ref, name)), name
    _same_row(ref.k_cache[:, :, :n], c.k_codes[:, :, :n], c.k_params[:, :, :n])
    _same_row(ref.v_cache[:, :, :n], c.v_codes[:, :, :n], c.v_params[:, :, :n])
    assert torch.all(c.k_codes[:, :, n:] == 0x5a) and torch.all(c.v_codes[:, :, n:] == 0x5a) and torch.all(c.k_params[:, :, n:] == 0)


@pytest.mark.parametrize("T,B,w", [(200, 90, 33), (40, 60, 16), (20, 8, 50)])
def test_compaction_with_a_history_window(T, B, w):
    V, g, b, h, d = P.vatp(), _gen(T), 2, 2, 128
    k, v = _rows(g, b, h, T, d, dtype="bf16"), _rows(g, b, h, T, d, dtype="bf16")
    p = _params(b=b, h=h, T=T, B=B, window=w)
    rows = torch.rand(b, h, w, T, generator=g, device="cuda") / T
    rows[:, :, :max(w - T, 0)] = 0
    acc, vnorm, n = rows.sum(2), v.float().abs().sum(-1), min(T, B)
    kept = torch.full((b, h, B), -1, dtype=torch.int32, device="cuda")
    kept[..., :n] = torch.rand(b, h, T, generator=g, device="cuda").topk(n, -1).indices.sort(-1).values
    c, ref, status = V.CacheQ4(p), V.Cache(p), _status()
    V.vatp_compact_q4(p, k, v, acc, vnorm, kept, c, win_rows=rows, dev_status=status)
    V.vatp_compact(p, k, v, acc, vnorm, kept, ref, win_rows=rows, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    for name in STATE + ("ring", "acc_fixed"):
        assert torch.equal(getattr(c, name), getattr(ref, name)), name
    _same_row(ref.k_cache[:, :, :n], c.k_codes[:, :, :n], c.k_params[:, :, :n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_groups_at_the_edges_of_the_format(dtype):
    """Zeros of both signs, constants, one outlier, halfway codes, ranges without a scale, the largest and smallest magnitudes."""
    V, d = P.vatp(), 64
    x = torch.zeros(12, d, device="cuda")
    x[1] = -0.0
    x[2], x[3] = 3.140625, -3.15                              # constants: a bf16 value, and (in fp32) one between two
    x[4, 5], x[4, 40] = 1e4, -1e4
    x[5] = torch.arange(64, device="cuda") % 16 + 0.5         # lo 0.5, sc 1: whole codes
    x[6] = (torch.arange(64, device="cuda") % 31) / 2         # lo 0, sc 1: every other value lies halfway
    x[7] = 1e-36 * torch.arange(64, device="cuda")
    x[8] = 1e-41 * torch.arange(64, device="cuda")            # subnormal in fp32
    x[9] = torch.linspace(-4e37, 4e37, 64, device="cuda")
    x[10] = 1000.0 + 0.01 * torch.arange(64, device="cuda")   # far from zero
    x[11] = -1000.0 - 0.01 * torch.arange(64, device="cuda")
    x = x.to(DT[dtype])[None, None].contiguous()
    p = _params(dtype, h=1, d=d, T=12, B=12)
    kept = torch.arange(12, dtype=torch.int32, device="cuda")[None, None].contiguous()
    one = torch.ones(1, 1, 12, device="cuda")
    c, back = V.CacheQ4(p), V.Cache(p)
    V.vatp_compact_q4(p, x, x, one, one, kept, c)
    V.vatp_cache_unpack_q4(p, c, back)
    torch.cuda.synchronize()
    _same_row(x, c.k_codes[:, :, :12], c.k_params[:, :, :12])
    _same_row(x, c.v_codes[:, :, :12], c.v_params[:, :, :12])
    assert torch.equal(back.k_cache[:, :, :12], Q.stored(x).float().to(DT[dtype]))


# ------------------------------------------------------------------------------------------------ conversion
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("b,h,kv,B,n,window", [(1, 1, 0, 1, 1, 0), (2, 3, 0, 100, 100, 0), (1, 8, 2, 61, 40, 0), (2, 2, 0, 45, 45, 7), (1, 4, 2, 30, 0, 5)])
def test_conversion_there_and_back(dtype, d, b, h, kv, B, n, window):
    V = P.vatp()
    p = _params(dtype, b, h, kv, d, B=B, window=window)
    a = _filled(p, n, form="wide")
    if n > 3:
        a.pos[:, :, 2] = -1                                   # a slot that was released
    c, back, status = V.CacheQ4(p), V.Cache(p), _status()
    for t in (c.k_codes, c.v_codes):
        t.fill_(0x33)
    for t in (back.k_cache, back.v_cache):
        t.fill_(7.0)
    V.vatp_cache_pack_q4(p, a, c, dev_status=status)
    V.vatp_cache_unpack_q4(p, c, back, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    live = a.pos >= 0
    for name in STATE + (("ring", "acc_fixed") if window else ()):
        assert torch.equal(getattr(c, name), getattr(a, name)) and torch.equal(getattr(back, name), getattr(a, name)), name
    for rows, codes, par, got in ((a.k_cache, c.k_codes, c.k_params, back.k_cache), (a.v_cache, c.v_codes, c.v_params, back.v_cache)):
        _same_row(rows[live], codes[live], par[live])
        assert torch.all(codes[~live] == 0x33) and torch.all(got[~live] == 7.0)
        assert torch.equal(got[live], Q.stored(rows[live]).float().to(DT[dtype]))


def test_conversion_over_shared_state():
    V, p = P.vatp(), _params(B=50, window=6)
    a = _filled(p, 50, form="wide")
    before = {n: t.clone() for n, t in _arrays(a).items()}
    c = V.CacheQ4(p, share=a)
    V.vatp_cache_pack_q4(p, a, c)
    rows = V.Cache(p, share=c)
    V.vatp_cache_unpack_q4(p, c, rows)
    torch.cuda.synchronize()
    for n, t in before.items():
        assert torch.equal(t, getattr(a, n)), n
    assert torch.equal(rows.k_cache[:, :, :50], Q.stored(a.k_cache[:, :, :50]).float().bfloat16())


def test_conversion_with_only_the_units_words_apart():
    """Every per-slot array shared, the words that count tokens not: those are copied."""
    V, p = P.vatp(), _params(B=30, h=4)
    a = _filled(p, 30, form="wide")
    c = V.CacheQ4(p, share=a)
    for name in ("len", "free_slot", "next_pos", "last_slot"):
        setattr(c, name, torch.full_like(getattr(a, name), 77))
    c.struct = V.CacheQ4Struct(c._struct(c.k_codes, c.v_codes), c.k_params.data_ptr(), c.v_params.data_ptr())
    V.vatp_cache_pack_q4(p, a, c)
    torch.cuda.synchronize()
    for name in ("len", "free_slot", "next_pos", "last_slot"):
        assert torch.equal(getattr(c, name), getattr(a, name)), name
    for name in ("len", "free_slot", "next_pos", "last_slot"):
        getattr(a, name).zero_()
    V.vatp_cache_unpack_q4(p, c, a)
    torch.cuda.synchronize()
    for name in ("len", "free_slot", "next_pos", "last_slot"):
        assert torch.equal(getattr(c, name), getattr(a, name)), name


# ------------------------------------------------------------------------------------------------ generation
def _run_steps(p, c, n_steps, dtype, *, seed=9):
    """n_steps steps of the call against 64 bits: outputs, the whole state, the released tokens, the stored rows."""
    V = P.vatp()
    b, h, cap = c.pos.shape
    G, d, w = p.heads // h, p.head_dim, p.window_w if p.indicator == V.IND_WINDOW else 0
    norm = {v: k for k, v in V.NORM_KINDS.items()}[p.norm_kind]
    ref = Q.State(c, d, p.budget, p.n_sink, p.n_recent, p.scale, w, norm)
    g, status, eps = _gen(seed), _status(), torch.finfo(DT[dtype]).eps / 2
    # a term p sc code of the output: with grouped bf16 queries p sc is rounded to fp16 (half a step is 2^-12 of it), else
    # 2^-20 covers what is left of it in two halves or in 32 bits
    term = 2.0 ** -12 + 2.0 ** -20 if G > 1 and dtype == "bf16" else 2.0 ** -20
    p_off = torch.zeros(b * h, 1, dtype=torch.float64, device="cuda")
    for i in range(n_steps):
        q, k, v = torch.randn(b, p.heads, d, generator=g, device="cuda").to(DT[dtype]), _rows(g, b, h, d, dtype=dtype), _rows(g, b, h, d, dtype=dtype)
        out, evicted = torch.full_like(q, 9.0), torch.full((b, h), -7, dtype=torch.int32, device="cuda")
        V.vatp_decode_step_q4(p, c, q, k, v, out, evicted_pos=evicted, dev_status=status)
        torch.cuda.synchronize()
        assert int(status) == 0
        want, pm, I, may_go, rel, v_mag = ref.step(q.view(b * h, G, d), k.view(b * h, d), v.view(b * h, d))
        off = (out.double().view(b * h, G, d) - want).abs()
        bound = (rel[..., None] + term) * v_mag + eps * want.abs() + 1e-30
        assert torch.all(off <= bound), f"step {i}: out, worst {float((off / bound).max())} of the bound"
        # an indicator is what it was plus the steps' probabilities p_j, each off by rel_j p_j at most: together by
        # sum_j rel_j p_j <= (max_j rel_j) S; a step adds a rounding of the sum, and a probability below 2^-126, the smallest normal
        # number of 32 bits, may come out as 0
        p_off = torch.maximum(p_off, rel.amax(-1, keepdim=True))
        acc = c.acc.view(b * h, cap).double()
        live = ref.pos >= 0
        tol = (p_off + (i + 2) * 2.0 ** -23) * ref.S + (i + 1) * 2.0 ** -126 + (w * 2.0 ** -52 if w else 0)
        assert torch.all(((acc - ref.S).abs() <= tol)[live]), f"step {i}: indicators"
        assert torch.all(((c.vnorm.view(b * h, cap).double() - ref.vnorm).abs() <= 2.0 ** -20 * ref.vnorm)[live])
        went = evicted.view(-1).long()
        full = ref.len + 1 > p.budget
        assert torch.all(went[~full] == -1)
        at = (ref.pos == went[:, None])
        assert torch.all((at & may_go).sum(-1)[full] == 1), f"step {i}: released a token that stays"
        least = I.masked_fill(~may_go, float("inf")).amin(-1)
        mine = torch.where(at, I, torch.zeros_like(I)).sum(-1)
        assert torch.all((mine <= least * (1 + 2 * p_off[:, 0] + (i + 4) * 2.0 ** -21))[full]), f"step {i}: not the least important token"
        new_slot = ref.free.clone()
        ref.finish(went)
        u = torch.arange(b * h, device="cuda")
        for rows, codes, par in ((k, c.k_codes, c.k_params), (v, c.v_codes, c.v_params)):
            _same_row(rows.view(b * h, d), codes.view(b * h, cap, -1)[u, new_slot], par.view(b * h, cap, d // 32, 2)[u, new_slot])
        assert torch.equal(c.pos.view(b * h, cap).long(), ref.pos)
        for name, x in (("len", ref.len), ("free_slot", ref.free), ("next_pos", ref.t), ("last_slot", ref.last)):
            assert torch.equal(getattr(c, name).view(-1).long(), x), name
        if w:
            ring = c.ring.view(b * h, w, cap).double()
            assert torch.all(((ring - ref.hist).abs() <= p_off[..., None] * ref.hist + 2.0 ** -126) | ~(ref.pos >= 0)[:, None]), "history"
            assert torch.equal(c.acc_fixed.view(b * h, cap)[ref.pos >= 0],
                               (c.ring.double() * 2.0 ** 52).long().sum(2).view(b * h, cap)[ref.pos >= 0]), "window sums"


SHAPES = [
    # b, h, kv, d, B, window
    (1, 1, 0, 128, 1, 0),        # one slot besides the incoming token's
    (1, 2, 0, 64, 7, 0),
    (2, 3, 0, 128, 16, 0),       # one tile and a row
    (1, 3, 0, 128, 127, 0),
    (1, 3, 0, 64, 128, 0),       # eight tiles and a row
    (2, 60, 0, 128, 200, 0),     # 120 units
    (3, 100, 0, 64, 130, 0),     # more units than SMs
    (1, 3, 0, 128, 1030, 0),
    (1, 2, 0, 64, 2049, 0),
    (1, 4, 0, 128, 777, 40),
    (2, 3, 0, 64, 100, 1),       # a history of one query
    (1, 200, 0, 128, 150, 9),
    (1, 2, 1, 128, 300, 0),
    (2, 9, 3, 64, 210, 0),       # groups of three
    (1, 16, 4, 128, 600, 0),
    (1, 5, 1, 128, 333, 0),      # five heads: beyond the columns' two halves
    (2, 14, 2, 64, 90, 0),
    (1, 16, 2, 128, 500, 33),    # eight heads, a history
    (1, 8, 1, 128, 2500, 0),
    (1, 2, 0, 128, 9000, 0),
]


@pytest.mark.parametrize("b,h,kv,d,B,window", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("grow", [0, 3, 1000000])         # tokens short of the budget; as many as there are: an empty cache
def test_steps_against_64_bits(b, h, kv, d, B, window, dtype, grow):
    n = max(B - grow, 0)
    p = _params(dtype, b, h, kv, d, B=B, F=min(2, B // 4), R=min(3, B // 4), window=window)
    _run_steps(p, _filled(p, n, seed=B + h), 5, dtype)


@pytest.mark.parametrize("b,h,kv,d,B,window,dtype", [
    (1, 32, 0, 128, 2048, 0, "bf16"),       # whole rounds of the warps and the incoming token's slot
    (1, 32, 0, 64, 2055, 0, "f32"),         # ... and eight slots more
    (1, 32, 0, 128, 2056, 0, "bf16"),       # ... one too many for that
    (1, 32, 8, 128, 2050, 20, "bf16"),
    (2, 70, 0, 64, 260, 0, "bf16"),
    (1, 40, 0, 128, 3001, 0, "bf16"),       # CTAs of sixteen warps
    (1, 40, 0, 64, 3001, 0, "f32"),
    (1, 100, 0, 128, 1023, 30, "bf16"),     # ... each a unit of its own, with a history
    (1, 160, 40, 128, 2500, 0, "bf16"),     # ... four heads
    (1, 160, 40, 64, 2500, 5, "f32"),
    (1, 240, 40, 128, 2500, 0, "bf16"),     # ... six heads
    (1, 1600, 200, 128, 3000, 0, "bf16"),   # more units than SMs, eight heads: one CTA of sixteen warps on an SM
    (2, 200, 0, 128, 700, 0, "f32"),
])
@pytest.mark.parametrize("grow", [0, 1500])
def test_steps_of_every_division_of_a_unit(b, h, kv, d, B, window, dtype, grow):
    p = _params(dtype, b, h, kv, d, B=B, F=2, R=3, window=window)
    _run_steps(p, _filled(p, max(B - grow, 0), seed=B + h), 3, dtype)


@pytest.mark.parametrize("units,B,window", [(13, 4500, 0), (16, 4001, 0), (16, 3001, 9), (23, 4600, 0), (8, 13107, 0), (40, 1100, 0), (8, 5000, 40)])
@pytest.mark.parametrize("G,d,dtype", [(1, 128, "bf16"), (1, 64, "f32"), (2, 64, "bf16"), (4, 128, "f32"), (4, 128, "bf16"), (8, 128, "bf16")])
def test_units_over_odd_numbers_of_CTAs(units, B, window, G, d, dtype):
    """Where fewer clusters of the next power of two run at once than there are units: three, five, six, nine or ten CTAs a unit."""
    p = _params(dtype, 1, units * G, units if G > 1 else 0, d, B=B, F=2, R=3, window=window)
    _run_steps(p, _filled(p, B, seed=B + G), 3, dtype)


def test_the_longest_caches_of_eight_heads():
    """Nine CTAs a unit, whose logits do not fit: sixteen, the most there are; beyond that the call is refused."""
    V, p = P.vatp(), _params("bf16", 1, 64, 8, 128, B=45000, F=2, R=3)
    _run_steps(p, _filled(p, 45000), 2, "bf16")
    p = _params("bf16", 1, 64, 8, 128, B=200000, F=2, R=3)
    c = V.CacheQ4(p)
    q = torch.zeros(1, 64, 128, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(1, 8, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(V.VatpError, match="unsupported"):
        V.vatp_decode_step_q4(p, c, q, k, k, torch.empty_like(q))


def test_integer_sums_of_more_slots_than_they_hold():
    """More than 2048 slots of a warp: the integer sums are taken over in between."""
    p = _params("bf16", 1, 150, 0, 64, B=17000)
    c = _filled(p, 17000)
    c.k_params[..., 0] *= 1e-3                                 # (logits near one another: all slots count)
    c.v_codes.fill_(0xff)
    _run_steps(p, c, 2, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv", [0, 2, 1])
@pytest.mark.parametrize("up", [True, False])
def test_scales_that_grow_along_the_cache(dtype, kv, up):
    """The power of two that p sc is scaled by moves again and again, or never after the first rows."""
    p = _params(dtype, 1, 8, kv, 128, B=1100)
    c = _filled(p, 1100)
    grow = torch.exp2(torch.linspace(-30, 30, 1100, device="cuda")).bfloat16()
    c.v_params[:, :, :1100] *= (grow if up else grow.flip(0))[:, None, None]
    _run_steps(p, c, 3, dtype)


@pytest.mark.parametrize("h,kv", [(8, 0), (8, 2)])
def test_precision_of_32_bit_steps(h, kv):
    """Typical errors, against the bounds of the other tests: logits up to 32 (in log2) have an ulp of 2^-19, half of which is
    2^-20 ln 2 = 7e-7 of a probability at most; rounded sums and the exponential add less."""
    V = P.vatp()
    b, d, B = 1, 128, 2000
    p = _params("f32", b, h, kv, d, B=B)
    c = _filled(p, B)
    hk = kv or h
    c.k_params *= 0.5
    ref = Q.State(c, d, B, 0, 0, p.scale)
    g = _gen(3)
    q, k, v = torch.randn(b, h, d, generator=g, device="cuda"), _rows(g, b, hk, d, dtype="f32"), _rows(g, b, hk, d, dtype="f32")
    out, before = torch.empty_like(q), c.acc.double()
    V.vatp_decode_step_q4(p, c, q, k, v, out)
    torch.cuda.synchronize()
    want, pm, _, _, _, v_mag = ref.step(q.view(hk, h // hk, d), k.view(hk, d), v.view(hk, d))
    # grouped queries: sums of fp16 products.  The sixteen of a tile and what they are added to are cut off 2^-24 below the largest
    # one's nominal magnitude, p sc 2^-14, while a code counts p sc 2^-18: 17 * 16 * 2^-24 of the tile's largest p sc, and the
    # sum of those is at most sum p sc <= v_mag / 15
    cut = 17 * 16 / 15 * 2.0 ** -24 * v_mag.norm() if kv else 0.0
    assert (out.double().view(want.shape) - want).norm() <= 1e-6 * want.norm() + cut
    got = (c.acc.double() - before).view(hk, -1)
    got[torch.arange(hk), ref.free] = c.acc.double().view(hk, -1)[torch.arange(hk), ref.free]
    # (the difference of two stored sums: a rounding of the sum, 2^-24 of it, comes on top)
    assert (got - pm).norm() <= 1e-6 * pm.norm() + 2.0 ** -24 * before.norm()


@pytest.mark.parametrize("norm", ["l1", "l2", "linf"])
def test_norms_and_protected_tokens(norm):
    """Sinks and recent tokens stay although they are the least important; the incoming row's norm is that of the row as given."""
    p = _params("bf16", 2, 4, 0, 128, B=40, F=5, R=30, norm=norm)
    c = _filled(p, 40)
    c.acc[:, :, :5] = 1e-6
    _run_steps(p, c, 12, "bf16")


def test_equal_importances_release_the_highest_position():
    V = P.vatp()
    p = _params("f32", 1, 1, 0, 64, B=64)
    c = _filled(p, 64)
    c.vnorm.zero_()                                            # all importances 0
    z = torch.zeros(1, 1, 64, device="cuda")
    ev, out = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.empty_like(z)
    V.vatp_decode_step_q4(p, c, z, z, z, out, evicted_pos=ev)
    torch.cuda.synchronize()
    assert int(ev) == 128                                      # the incoming token itself: the highest position
    assert int(c.free_slot) == int(c.last_slot) == 64 and int(c.len) == 64


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("big", [1e3, 1e-12])
def test_scales_far_from_one(dtype, big):
    """Values of very different magnitudes beside one another: the second product's operands are scaled to fit 16 bits."""
    V = P.vatp()
    p = _params(dtype, 1, 2, 0, 128, B=300)
    c = _filled(p, 300)
    c.v_params[:, :, ::3] *= big
    c.k_params[:, :, 5] = 0                                    # a row of zeros
    c.v_params[:, :, 7] = 0
    c.vnorm.fill_(1.0)
    _run_steps(p, c, 4, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_token_takes_all(dtype):
    """Logits hundreds apart: the others' probabilities vanish; the values come out to the last bit that 16 and 32 bits leave."""
    V = P.vatp()
    p = _params(dtype, 1, 3, 0, 64, B=200)
    c = _filled(p, 200)
    c.k_params[:, :, 150] *= 200
    _run_steps(p, c, 3, dtype)


def test_memory_behind_the_tokens_is_not_read_into_results():
    """Slots without a token hold what looks like NaN; they change nothing, and stay."""
    V, p = P.vatp(), _params("bf16", 1, 4, 0, 128, B=90)
    a = _filled(p, 37)
    b = _clone(a, p)
    b.k_codes[:, :, 38:], b.v_codes[:, :, 38:] = 0xff, 0xff
    b.k_params[:, :, 38:], b.v_params[:, :, 38:] = float("nan"), float("nan")
    b.acc[:, :, 38:], b.vnorm[:, :, 38:] = float("nan"), float("nan")
    g = _gen(4)
    q, k, v = (_rows(g, 1, 4, 128, dtype="bf16") for _ in range(3))
    outs = []
    for c in (a, b):
        out = torch.empty_like(q)
        V.vatp_decode_step_q4(p, c, q, k, v, out)
        torch.cuda.synchronize()
        outs.append(out)
        assert torch.equal(c.pos[:, :, 38:], torch.full_like(c.pos[:, :, 38:], -1))
    assert torch.equal(*outs) and torch.equal(a.acc[:, :, :38], b.acc[:, :, :38])
    assert torch.all(b.k_codes[:, :, 38:] == 0xff) and torch.all(torch.isnan(b.acc[:, :, 38:]))


def test_optional_outputs_and_determinism():
    V, p = P.vatp(), _params("bf16", 2, 16, 4, 128, B=700, window=12)
    a = _filled(p, 700)
    g = _gen(5)
    tokens = [tuple(_rows(g, 2, h, 128, dtype="bf16") for h in (16, 4, 4)) for _ in range(6)]
    runs = []
    for _ in range(2):
        c, outs = _clone(a, p), []
        for q, k, v in tokens:
            outs.append(torch.empty_like(q))
            V.vatp_decode_step_q4(p, c, q, k, v, outs[-1])
        torch.cuda.synchronize()
        runs.append((c, outs))
    _equal(runs[0][0], runs[1][0])
    assert all(torch.equal(x, y) for x, y in zip(runs[0][1], runs[1][1]))


def test_the_overlap_flag_changes_nothing():
    """Steps of several caches one after the other, some in 16 bits, with the flag: as without it."""
    V = P.vatp()
    g = _gen(6)
    p0, p1 = (_params("bf16", 1, 32, 0, 128, B=400, decode_overlap=o) for o in (False, True))
    tokens = [tuple(_rows(g, 1, 32, 128, dtype="bf16") for _ in range(3)) for _ in range(12)]
    got = []
    for p in (p0, p1):
        caches = [_filled(p, 400, seed=s) for s in (1, 2)] + [_filled(p, 400, seed=3, form="wide")]
        outs = []
        for i, (q, k, v) in enumerate(tokens):
            for c in caches:
                outs.append(torch.empty_like(q))
                (V.vatp_decode_step_q4 if hasattr(c, "k_codes") else V.vatp_decode_step)(p, c, q if not i else outs[-2], k, v, outs[-1])
        torch.cuda.synchronize()
        got.append((caches, outs))
    for x, y in zip(got[0][0], got[1][0]):
        _equal(x, y)
    assert all(torch.equal(x, y) for x, y in zip(got[0][1], got[1][1]))


@pytest.mark.parametrize("h,kv,B,window", [(4, 0, 300, 0), (32, 8, 900, 0), (4, 0, 300, 20)])
def test_steps_in_a_graph(h, kv, B, window):
    """Captured and replayed twice, behind work of another kind: as stepping one by one."""
    V = P.vatp()
    p = _params("bf16", 1, h, kv, 128, B=B, window=window)
    a, g = _filled(p, B - 2), _gen(7)
    tokens = [tuple(_rows(g, 1, n, 128, dtype="bf16") for n in (h, kv or h, kv or h)) for _ in range(4)]
    one, two = _clone(a, p), _clone(a, p)
    out = torch.empty(4, 1, h, 128, dtype=torch.bfloat16, device="cuda")
    want = []
    for _ in range(2):
        for q, k, v in tokens:
            o = torch.empty_like(q)
            V.vatp_decode_step_q4(p, one, q, k, v, o)
            want.append(o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for i, (q, k, v) in enumerate(tokens):
            V.vatp_decode_step_q4(p, two, q, k, v, out[i])
    got = []
    for _ in range(2):
        out.fill_(3.0)
        graph.replay()
        got += list(out.clone())
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    _equal(one, two)


def test_two_streams_at_once():
    V = P.vatp()
    p = _params("bf16", 1, 16, 0, 128, B=500)
    g = _gen(8)
    caches = [_filled(p, 500, seed=s) for s in (1, 2)]
    alone = [_clone(c, p) for c in caches]
    tokens = [tuple(_rows(g, 1, 16, 128, dtype="bf16") for _ in range(3)) for _ in range(20)]
    want, got = [[], []], [[], []]
    for c, to in zip(alone, want):
        for q, k, v in tokens:
            to.append(torch.empty_like(q))
            V.vatp_decode_step_q4(p, c, q, k, v, to[-1])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in caches]
    bufs = [[torch.empty_like(t[0]) for t in tokens] for _ in caches]
    for i, (q, k, v) in enumerate(tokens):
        for c, s, b in zip(caches, streams, bufs):
            V.vatp_decode_step_q4(p, c, q, k, v, b[i], stream=s)
    torch.cuda.synchronize()
    for w, b, x, y in zip(want, bufs, caches, alone):
        assert all(torch.equal(m, n) for m, n in zip(w, b))
        _equal(x, y)


def test_offsets_beyond_32_bits():
    """More than 2^31 bytes of codes: the last unit's rows."""
    V, d, B = P.vatp(), 128, 33000
    units = 1100                                               # 1100 * 33008 slots * 64 bytes = 2.3e9
    p = _params("bf16", 1, units, 0, d, B=B)
    c = V.CacheQ4(p)
    one = _params("bf16", 1, 1, 0, d, B=B)
    small = _filled(one, B)
    last = units - 1
    for n, t in _arrays(small).items():
        getattr(c, n)[:, last] = t[:, 0]
    c.next_pos.fill_(int(small.next_pos))
    g = _gen(10)
    q = torch.zeros(1, units, d, dtype=torch.bfloat16, device="cuda")
    k, v, out = q.clone(), q.clone(), torch.empty_like(q)
    q[:, last], k[:, last], v[:, last] = (_rows(g, 1, d, dtype="bf16") for _ in range(3))
    o1 = torch.empty(1, 1, d, dtype=torch.bfloat16, device="cuda")
    status = _status()
    V.vatp_decode_step_q4(p, c, q, k, v, out, dev_status=status)
    V.vatp_decode_step_q4(one, small, q[:, last:].contiguous(), k[:, last:].contiguous(), v[:, last:].contiguous(), o1)
    torch.cuda.synchronize()
    assert int(status) == 0
    assert torch.allclose(out[:, last].float(), o1[:, 0].float(), rtol=2.0 ** -7, atol=1e-3)      # (the unit may be split otherwise)
    slot = int(small.last_slot)
    assert torch.equal(c.k_codes[:, last, slot], small.k_codes[:, 0, slot]) and int(c.free_slot[0, last]) == int(small.free_slot)


# ------------------------------------------------------------------------------------------------ copies
@pytest.mark.parametrize("form", ["q4", "wide"])
@pytest.mark.parametrize("dtype,d,h,kv,window", [("bf16", 128, 4, 0, 0), ("f32", 64, 6, 2, 0), ("bf16", 64, 2, 0, 9)])
@pytest.mark.parametrize("B_from,B_to", [(50, 50), (33, 70), (70, 33), (1, 300)])
def test_copies_between_states(form, dtype, d, h, kv, window, B_from, B_to):
    V = P.vatp()
    pf, pt = (_params(dtype, b, h, kv, d, B=B, window=window) for b, B in ((3, B_from), (7, B_to)))
    n = min(B_from, B_to)
    src, dst = _filled(pf, n, seed=1, form=form), _filled(pt, B_to, seed=2, form=form)
    before, status = _clone(dst, pt), _status()
    m = [2, V.SEQ_KEEP, 0, 0, V.SEQ_FREE, 1, 2]
    V.vatp_cache_copy(pt, src, dst, torch.tensor(m, dtype=torch.int32, device="cuda"), dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    cut = min(src.cap, dst.cap)
    for b, j in enumerate(m):
        for name, t in _arrays(dst).items():
            a, old = getattr(src, name), getattr(before, name)
            if j == V.SEQ_KEEP or (j == V.SEQ_FREE and name not in ("pos", "len", "free_slot", "next_pos", "last_slot")):
                assert torch.equal(t[b], old[b]), (b, name)
            elif j == V.SEQ_FREE:
                assert torch.all(t[b] == (-1 if name in ("pos", "last_slot") else 0)), (b, name)
            elif name in ("len", "free_slot", "next_pos", "last_slot"):
                assert torch.equal(t[b], a[j]), (b, name)
            elif name == "ring":
                assert torch.equal(t[b, ..., :cut], a[j, ..., :cut]) and torch.equal(t[b, ..., cut:], old[b, ..., cut:])
            else:
                assert torch.equal(t[b, :, :cut], a[j, :, :cut]), (b, name)
                assert torch.all(t[b, :, cut:] == -1) if name == "pos" else torch.equal(t[b, :, cut:], old[b, :, cut:]), (b, name)


@pytest.mark.parametrize("form", ["q4", "wide"])
def test_copies_within_a_state(form):
    """An entry may be read where nobody writes it; else the reader is left as it is and the status word says so."""
    V, p = P.vatp(), _params("bf16", 5, 3, 0, 128, B=60, window=4)
    a = _filled(p, 60, form=form)
    a.next_pos.copy_(torch.arange(100, 115, device="cuda").view(5, 3))
    for m, refused in (([0, 1, 1, 3, 3], []), ([4, V.SEQ_KEEP, V.SEQ_KEEP, V.SEQ_FREE, V.SEQ_KEEP], []),
                       ([1, 0, 2, 2, V.SEQ_KEEP], [0, 1]),             # exchanged: each is overwritten while the other reads it
                       ([0, 0, 1, 3, 4], [2]), ([0, 2, V.SEQ_FREE, 3, 4], [1]),
                       ([5, 1, -3, 3, 1], [0, 2])):
        c, status = _clone(a, p), _status()
        V.vatp_cache_copy(p, c, c, torch.tensor(m, dtype=torch.int32, device="cuda"), dev_status=status)
        torch.cuda.synchronize()
        assert int(status) == (1 if refused else 0), m
        for b, j in enumerate(m):
            stays = b in refused or j == V.SEQ_KEEP
            for name, t in _arrays(c).items():
                if j != V.SEQ_FREE or stays:
                    assert torch.equal(t[b], getattr(a, name)[b if stays else j]), (m, b, name)
            if j == V.SEQ_FREE:
                assert torch.all(c.pos[b] == -1) and torch.all(c.len[b] == 0) and torch.equal(c.acc[b], a.acc[b])


def test_entries_that_do_not_fit_are_left_alone():
    V = P.vatp()
    pf, pt = _params(b=2, B=40), _params(b=2, B=24)
    src, dst = _filled(pf, 40), _filled(pt, 24, seed=2)
    src.len[1], src.free_slot[1], src.pos[1, :, 24:] = 24, 24, -1
    before, status = _clone(dst, pt), _status()
    V.vatp_cache_copy(pt, src, dst, torch.tensor([0, 1], dtype=torch.int32, device="cuda"), dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 1
    for name, t in _arrays(dst).items():
        assert torch.equal(t[0], getattr(before, name)[0]), name
    assert torch.equal(dst.k_codes[1, :, :24], src.k_codes[1, :, :24]) and torch.all(dst.len[1] == 24)


def test_budgets_of_equal_capacity_that_differ():
    """Budgets of 70 and 66 have 72 slots each: a full entry of the larger one is too long for the smaller all the same."""
    V = P.vatp()
    pf, pt = _params(b=2, B=70), _params(b=2, B=66)
    src, dst = _filled(pf, 70), _filled(pt, 66, seed=2)
    assert src.cap == dst.cap
    src.len[1], src.free_slot[1], src.pos[1, :, 66:] = 66, 66, -1
    before, status = _clone(dst, pt), _status()
    V.vatp_cache_copy(pt, src, dst, torch.tensor([0, 1], dtype=torch.int32, device="cuda"), dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 1
    for name, t in _arrays(dst).items():
        assert torch.equal(t[0], getattr(before, name)[0]) and torch.equal(t[1], getattr(src, name)[1]), name


def test_a_freed_entry_and_a_joined_one_go_on_generating():
    """Freed: the cache starts anew.  Joined from a smaller budget: it grows to the larger one."""
    V = P.vatp()
    pf, pt = _params(b=1, h=4, B=20), _params(b=3, h=4, B=23)
    src, dst = _filled(pf, 20), _filled(pt, 23, seed=2)
    V.vatp_cache_copy(pt, src, dst, torch.tensor([V.SEQ_FREE, 0, V.SEQ_KEEP], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    dst.acc[0], dst.vnorm[0] = 0, 0                            # (the reference keeps them for slots without a token)
    _run_steps(pt, dst, 8, "bf16")


@pytest.mark.parametrize("bf16_first", [True, False])
def test_a_prompt_from_scores_to_forked_generation(bf16_first):
    """The calls as a program makes them: score, select, store in 4 bits (directly or by way of a 16-bit state), fork into samples,
    generate beside a 16-bit step that reads the same values."""
    V = P.vatp()
    b, hq, h, d, T, B, n = 1, 16, 4, 128, 700, 250, 3
    g = _gen(11)
    q, k, v = (_rows(g, b, x, T, d, dtype="bf16") for x in (hq, h, h))
    p = _params("bf16", b, hq, h, d, T=T, B=B, F=4, R=20)
    status = _status()
    out = {x: torch.empty(b, h, T, device="cuda") for x in ("attn_acc", "vnorm", "score")}
    ws = torch.empty(V.vatp_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    kept = torch.empty(b, h, B, dtype=torch.int32, device="cuda")
    V.vatp_prefill_scores(p, q, k, v, **out, workspace=ws, dev_status=status)
    V.vatp_select(p, out["score"], kept, dev_status=status)
    c = V.CacheQ4(p)
    if bf16_first:
        wide = V.Cache(p)
        V.vatp_compact(p, k, v, out["attn_acc"], out["vnorm"], kept, wide, dev_status=status)
        V.vatp_cache_pack_q4(p, wide, c, dev_status=status)
    else:
        V.vatp_compact_q4(p, k, v, out["attn_acc"], out["vnorm"], kept, c, dev_status=status)
    ps = _params("bf16", n, hq, h, d, T=T, B=B, F=4, R=20)
    samples = V.CacheQ4(ps)
    V.vatp_cache_copy(ps, c, samples, torch.zeros(n, dtype=torch.int32, device="cuda"), dev_status=status)
    # a 32-bit state of the same values: its steps differ from the 4-bit ones by the new rows' quantisation alone, so the
    # incoming rows are given as their stored values
    pw = _params("f32", n, hq, h, d, T=T, B=B, F=4, R=20)
    wide = V.Cache(pw)
    V.vatp_cache_unpack_q4(pw, samples, wide, dev_status=status)
    for _ in range(6):
        qn, kn, vn = (torch.randn(n, x, d, generator=g, device="cuda").bfloat16() for x in (hq, h, h))
        kn, vn = (Q.stored(x).float() for x in (kn, vn))
        o4, e4 = torch.empty(n, hq, d, device="cuda"), torch.empty(n, h, dtype=torch.int32, device="cuda")
        o32, e32 = torch.empty_like(o4), torch.empty_like(e4)
        V.vatp_decode_step_q4(pw, samples, qn.float(), kn, vn, o4, evicted_pos=e4, dev_status=status)
        V.vatp_decode_step(pw, wide, qn.float(), Q.stored(kn).float(), Q.stored(vn).float(), o32, evicted_pos=e32, dev_status=status)
        torch.cuda.synchronize()
        assert int(status) == 0
        # sums of 32 bits on both sides: logits of about 128 * 2^-23 * 4, i.e. 6e-5 of the largest value
        assert (o4 - o32).abs().max() <= 6e-5 * o32.abs().max()
        assert torch.equal(e4, e32)
    assert not torch.equal(samples.k_codes[0], samples.k_codes[1])


def test_bounds_checking_build_reports_no_violation():
    """The small cases again on the library that range-checks every index (libvatp_dbg.so)."""
    if os.environ.get("VATP_LIBRARY"):
        pytest.skip("already the bounds-checking build")
    from paper_2406_12335_b200 import build
    lib = build.build(debug_bounds=True)
    here = os.path.abspath(__file__)
    r = subprocess.run([sys.executable, "-m", "pytest", here, "-x", "-q", "-m", "gpu", "-k",
                        "test_compaction or there_and_back or norms_and_protected or 3-777 or between_states or scores_to_forked"],
                       env={**os.environ, "VATP_LIBRARY": lib}, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "passed" in r.stdout, r.stdout[-2000:]
