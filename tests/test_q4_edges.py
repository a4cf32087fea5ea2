"""The 4-bit decode state at its edges on the GPU: precision where a sum's terms differ much, magnitudes at the ends of the range, values
that are not finite, wide batches of copies.  Tolerances count roundings; the reference is tests/q4_reference.py, in 64 bits."""
import pytest
import torch

from tests import parity as P
from tests import q4_reference as Q
from tests.test_q4 import DT, _arrays, _clone, _filled, _gen, _params, _rows, _status

pytestmark = pytest.mark.gpu


def _packed(p, k, v):
    """A full 4-bit state of the rows k, v [units, B, d]."""
    V = P.vatp()
    wide, c = _filled(p, p.budget, form="wide"), V.CacheQ4(p)
    wide.k_cache[0, :, :p.budget], wide.v_cache[0, :, :p.budget] = k.to(wide.k_cache.dtype), v.to(wide.k_cache.dtype)
    V.vatp_cache_pack_q4(p, wide, c)
    torch.cuda.synchronize()
    return c


def _reference(c, p):
    return Q.State(c, p.head_dim, p.budget, p.n_sink, p.n_recent, p.scale)


# ------------------------------------------------------------------------------------------------ precision
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_products_of_probabilities_and_scales_keep_32_bits(dtype, G):
    """All rows of V the same, all probabilities but one in 32 the same: what rounding p sc does to a term does not average out, and the
    outputs are differences of large terms."""
    V, units, B, d = P.vatp(), 16, 255, 64
    p = _params(dtype, 1, units * G, units if G > 1 else 0, d, B=B)
    k = torch.zeros(units, B, d, device="cuda")
    k[..., 0] = 0.3
    k[:, ::32, 0] = torch.linspace(1.0, 2.0, units, device="cuda")[:, None]        # a warp's 32 rows: one with a larger logit
    v = (torch.arange(d, device="cuda") % 16 - 8.0).expand(units, B, d)            # lo -8, sc 1: code 8 stands for 0
    c = _packed(p, k, v)
    q = torch.zeros(1, units * G, d, device="cuda", dtype=DT[dtype])
    q[0, :, 0] = torch.linspace(2.0, 5.0, units * G, device="cuda").to(q.dtype)    # (logits 0.2 to 1.1 apart, none of them 0)
    k1, v1, out = torch.zeros(1, units, d, device="cuda", dtype=q.dtype), v[:, 0][None].to(q.dtype).contiguous(), torch.empty_like(q)
    want, _, _, _, rel, v_mag = _reference(c, p).step(q.view(units, G, d), k1.view(units, d), v1.view(units, d))
    V.vatp_decode_step_q4(p, c, q, k1, v1, out)
    torch.cuda.synchronize()
    off = (out.double().view(want.shape) - want).abs()
    # rel: what a probability may be off by; 2^-20: p sc in two halves and the sums of 256 terms in 32 bits; half a step of the output.
    # (With one fp16 for p sc: 11 to 15 times the bound.)
    bound = (rel[..., None] + 2.0 ** -20) * v_mag + torch.finfo(q.dtype).eps / 2 * want.abs()
    assert torch.all(off <= bound), float((off / bound).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_logits_beside_a_channel_of_large_queries(dtype, G):
    """A channel of q is 125 times the others, and the keys are nearly constant in it: the other channels decide."""
    V, units, B, d = P.vatp(), 4, 1500, 128
    p = _params(dtype, 1, units * G, units if G > 1 else 0, d, B=B)
    g = _gen(31)
    k, v = (torch.randn(units, B, d, generator=g, device="cuda").clamp(-2.9, 2.9) for _ in range(2))
    k[..., 0] = 3.0                                                                # the largest of its group
    c = _packed(p, k, v)
    c.acc.zero_()
    q = torch.randn(1, units * G, d, generator=g, device="cuda").to(DT[dtype])
    q[..., 0] = 125.0
    k1, v1 = (torch.randn(1, units, d, generator=g, device="cuda").clamp(-2.9, 2.9).to(q.dtype) for _ in range(2))
    k1[..., 0] = 3.0
    _, pm, _, _, _, _ = _reference(c, p).step(q.view(units, G, d), k1.view(units, d), v1.view(units, d))
    V.vatp_decode_step_q4(p, c, q, k1, v1, torch.empty_like(q))
    torch.cuda.synchronize()
    got = c.acc.double().view(units, -1)
    # A sum of products on the tensor cores cuts its terms off 2^-24 below the largest one's nominal magnitude, 2^-14 q where a code counts
    # 2^-18: 2^-20 * 125 * sc * scale = 4.2e-6 of a logit (sc 0.4, scale 128^-1/2) a term.  34 such errors in the group of that channel, even
    # between 0 and that: 7e-6 rms.  Logits of 33 in natural units, 48 in powers of two, have an ulp of 3.8e-6; eight roundings: 4e-6 rms.
    # Together 8e-6, over 6000 slots to a few percent.  (Codes that count 2^-24 were seen to lose 1.1e-5 to 1.5e-5.)
    assert (got - pm).norm() <= 9.7e-6 * pm.norm(), float((got - pm).norm() / pm.norm())


# ------------------------------------------------------------------------------------------------ magnitudes
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G", [1, 4, 8])
@pytest.mark.parametrize("size", [1e3, 1e6, -1e6, 1e12, -1e12])
def test_logits_of_any_size(dtype, G, size):
    """Equal logits of size * 1e6 / sqrt(d), the incoming token's below them: the mean of the rows."""
    V, units, B, d = P.vatp(), 3, 700, 64
    p, g = _params(dtype, 1, units * G, units if G > 1 else 0, d, B=B), _gen(14)
    k, v = torch.zeros(units, B, d, device="cuda"), torch.randn(units, B, d, generator=g, device="cuda")
    k[..., 0] = 1e6
    c = _packed(p, k, v)
    c.acc.zero_()
    ref = _reference(c, p)
    q = torch.zeros(1, units * G, d, device="cuda", dtype=DT[dtype])
    q[..., 0] = size
    k1, v1 = torch.zeros(1, units, d, device="cuda", dtype=q.dtype), torch.randn(1, units, d, generator=g, device="cuda").to(q.dtype)
    k1[..., 0] = 0.0 if size > 0 else 2e6
    out = torch.empty_like(q)
    V.vatp_decode_step_q4(p, c, q, k1, v1, out)
    torch.cuda.synchronize()
    want, v_mag = ref.v[:, :B].mean(1, keepdim=True), ref.mag[1][:, :B].mean(1).repeat_interleave(32, -1)[:, None]
    off = (out.double().view(units, G, d) - want).abs()
    # sums of 700 terms in 32 bits, p sc in two halves, the exponential's 2^-22; half a step of the output
    assert torch.all(off <= 2.0 ** -19 * v_mag + torch.finfo(q.dtype).eps / 2 * want.abs())
    assert torch.all((c.acc.view(units, -1)[:, :B] * B - 1).abs() <= 2.0 ** -19) and torch.all(c.acc[:, :, B] == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G", [1, 4])
def test_values_as_small_as_the_format_holds(dtype, G):
    """Scales of 2^-99, the largest probabilities in a warp's later items."""
    V, units, B, d = P.vatp(), 160, 600, 64
    p, g = _params(dtype, 1, units * G, units if G > 1 else 0, d, B=B), _gen(15)
    k = torch.zeros(units, B, d, device="cuda")
    k[:, :, 0] = torch.linspace(0.0, 1.0, B, device="cuda")
    v = torch.randint(0, 16, (units, B, d), generator=g, device="cuda") * 2.0 ** -99
    v[..., ::32], v[..., 1::32] = 0.0, 15 * 2.0 ** -99                             # lo 0, sc 2^-99
    c = _packed(p, k, v)
    q = torch.zeros(1, units * G, d, device="cuda", dtype=DT[dtype])
    q[..., 0] = 24.0                                                               # (logits 0 to 4.3, in powers of two)
    k1, v1, out = torch.zeros(1, units, d, device="cuda", dtype=q.dtype), v[:, 3][None].to(q.dtype).contiguous(), torch.empty_like(q)
    want, _, _, _, rel, v_mag = _reference(c, p).step(q.view(units, G, d), k1.view(units, d), v1.view(units, d))
    V.vatp_decode_step_q4(p, c, q, k1, v1, out)
    torch.cuda.synchronize()
    off = (out.double().view(want.shape) - want).abs()
    # (p sc of a warp's largest is held to 2^-24 at least where it is this small)
    assert torch.all(off <= (rel[..., None] + 2.0 ** -20) * v_mag + torch.finfo(q.dtype).eps / 2 * want.abs())


# ------------------------------------------------------------------------------------------------ values that are not finite
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_groups_that_are_not_finite_are_stored_as_nan(dtype, d, bad):
    """By compaction, conversion and the step: the group is NaN, its neighbours are what they were."""
    V, B, h = P.vatp(), 40, 3
    p, g = _params(dtype, 1, h, 0, d, T=B, B=B), _gen(12)
    k, v = (_rows(g, 1, h, B, d, dtype=dtype) for _ in range(2))
    group = torch.zeros(1, h, B, d // 32, dtype=torch.bool, device="cuda")
    for row, at in ((0, 0), (7, 33), (20, 31), (39, d - 1)):                       # row 20: every head's whole group
        k[:, 1, row, at], group[:, 1, row, at // 32] = bad, True
    k[:, :, 20, :32], group[:, :, 20, 0] = bad, True
    want = Q.stored(torch.where(group.repeat_interleave(32, -1), torch.zeros_like(k), k)).float().to(k.dtype)
    want.masked_fill_(group.repeat_interleave(32, -1), float("nan"))
    kept = torch.arange(B, dtype=torch.int32, device="cuda").expand(1, h, B).contiguous()
    one = torch.ones(1, h, B, device="cuda")
    wide, back = V.Cache(p), V.Cache(p)
    V.vatp_compact(p, k, v, one, one, kept, wide)
    for call in ("compact", "pack", "step"):
        c = V.CacheQ4(p)
        if call == "compact":
            V.vatp_compact_q4(p, k, v, one, one, kept, c)
        elif call == "pack":
            V.vatp_cache_pack_q4(p, wide, c)
        else:
            for i in range(B):                                                     # into an empty cache, token by token
                q = torch.zeros(1, h, d, dtype=k.dtype, device="cuda")
                V.vatp_decode_step_q4(p, c, q, k[:, :, i].contiguous(), v[:, :, i].contiguous(), torch.empty_like(q))
        V.vatp_cache_unpack_q4(p, c, back)
        torch.cuda.synchronize()
        assert torch.equal(torch.isnan(c.k_params[:, :, :B]), group[..., None].expand(-1, -1, -1, -1, 2)), call
        torch.testing.assert_close(back.k_cache[:, :, :B], want, rtol=0, atol=0, equal_nan=True, msg=call)
        assert torch.equal(back.v_cache[:, :, :B], Q.stored(v).float().to(v.dtype)), call


@pytest.mark.parametrize("where", ["k row", "v row", "k row of a warp's last slots", "q", "q inf", "k_new", "v_new"])
@pytest.mark.parametrize("dtype,G,d,B", [("bf16", 1, 128, 700), ("f32", 1, 64, 150), ("bf16", 4, 128, 700), ("f32", 3, 64, 90), ("bf16", 8, 64, 400)])
def test_a_nan_reaches_the_outputs(dtype, G, d, B, where):
    """Where the formulas give NaN the step gives it; other units and heads are what they would be, and the state's words stay sound."""
    V, units, bad = P.vatp(), 3, float("nan")
    p, g = _params(dtype, 1, units * G, units if G > 1 else 0, d, B=B, F=2, R=3), _gen(13)
    q, k, v = (_rows(g, 1, n, d, dtype=dtype) for n in (units * G, units, units))
    clean, c = _filled(p, B), _filled(p, B)
    q1, k1, v1 = q.clone(), k.clone(), v.clone()
    head = 2 * G - 1                                                               # the last of unit 1
    if "row" in where:
        row = B - 1 if "last" in where else 40
        (c.k_params if where[0] == "k" else c.v_params)[:, 1, row, 1] = bad
    elif where[0] == "q":
        q1[:, head, 5] = float("inf") if "inf" in where else bad
    else:
        (k1 if where[0] == "k" else v1)[:, 1, d - 1] = bad
    want, pm, _, may_go, _, _ = Q.State(c, d, B, 2, 3, p.scale).step(q1.view(units, G, d), k1.view(units, d), v1.view(units, d))
    got = []
    for cache, a, b, e in ((clean, q, k, v), (c, q1, k1, v1)):
        out, evicted, status = torch.empty_like(q), torch.empty(1, units, dtype=torch.int32, device="cuda"), _status()
        V.vatp_decode_step_q4(p, cache, a, b, e, out, evicted_pos=evicted, dev_status=status)
        torch.cuda.synchronize()
        assert int(status) == 0
        got.append(out.view(units, G, d))
    assert torch.any(torch.isnan(want)) and torch.equal(torch.isnan(got[1]), torch.isnan(want))
    same = ~torch.isnan(want).flatten(1).any(-1)
    assert torch.equal(got[0][same], got[1][same]) and same.tolist() == [True, False, True]
    if where[0] == "q":                                                            # the unit's other heads
        assert torch.equal(got[0][1, :G - 1], got[1][1, :G - 1])
    live, acc = c.pos.view(units, -1) >= 0, c.acc.view(units, -1)
    assert torch.equal(torch.isnan(acc)[live], torch.isnan(pm)[live])
    assert torch.equal(acc[[0, 2]], clean.acc.view(units, -1)[[0, 2]])
    assert torch.all(c.len == B) and torch.all(live[:, :B + 1].sum(-1) == B)
    slot = c.free_slot.view(-1).long()
    u = torch.arange(units, device="cuda")
    assert torch.all(may_go[u, slot]) and not torch.any(live[u, slot])


# ------------------------------------------------------------------------------------------------ copies
@pytest.mark.parametrize("form", ["q4", "wide"])
@pytest.mark.parametrize("in_place", [False, True])
def test_copies_of_more_entries_than_a_warp_has_lanes(form, in_place):
    """Entries that take the same source lie more than 32 apart, the first of them beyond the first 32 or not."""
    V, n = P.vatp(), 101
    p = _params("bf16", n, 2, 0, 64, B=23)
    src = _filled(p, 23, seed=1, form=form)
    src.next_pos.copy_(torch.arange(2 * n, device="cuda").view(n, 2) + 1000)
    dst = src if in_place else _filled(p, 23, seed=2, form=form)
    before_src, before = _clone(src, p), _clone(dst, p)
    m = [V.SEQ_KEEP] * n
    for b in (1, 2, 31, 32, 33, 64, 100):
        m[b] = 40                                                                  # entries before and behind their source
    for b in (35, 70, 99):
        m[b] = 5                                                                   # the first taker in the second 32
    m[98], m[97], m[96] = 66, V.SEQ_FREE, 96
    status = _status()
    V.vatp_cache_copy(p, src, dst, torch.tensor(m, dtype=torch.int32, device="cuda"), dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    for name, t in _arrays(dst).items():
        for b, j in enumerate(m):
            if j == V.SEQ_FREE:
                if name in ("pos", "last_slot"):
                    assert torch.all(t[b] == -1)
                elif name in ("len", "free_slot", "next_pos"):
                    assert torch.all(t[b] == 0)
            else:
                want = getattr(before, name)[b] if j == V.SEQ_KEEP else getattr(before_src, name)[j]
                assert torch.equal(t[b], want), (name, b)


def _whole(g, *shape, dtype):
    """Rows that both forms hold exactly: whole numbers, -8 and 7 in every group (lo -8, sc 1)."""
    x = torch.randint(-8, 8, shape, generator=g, device="cuda").to(DT[dtype])
    x[..., ::32], x[..., 5::32] = -8, 7
    return x


@pytest.mark.parametrize("dtype,h,kv,d,window", [("bf16", 4, 0, 128, 0), ("bf16", 8, 2, 64, 0), ("f32", 3, 0, 64, 0), ("bf16", 4, 0, 64, 6), ("f32", 4, 2, 128, 6)])
def test_freed_and_joined_entries_go_on_generating_in_either_form(dtype, h, kv, d, window):
    """One entry freed, one joined from a smaller budget, one kept: 16- or 32-bit steps and 4-bit steps on the same values."""
    V, hk, g = P.vatp(), kv or h, _gen(16)
    pf, pt = (_params(dtype, n, h, kv, d, B=B, F=1, R=2, window=window) for n, B in ((1, 20), (3, 23)))
    states = []
    for p, n in ((pf, 20), (pt, 23)):
        wide, c = _filled(p, n, form="wide"), V.CacheQ4(p)
        for x in (wide.k_cache, wide.v_cache):
            x[:, :, :n] = _whole(g, *x[:, :, :n].shape, dtype=dtype)
        V.vatp_cache_pack_q4(p, wide, c)
        states.append((wide, c))
    m = torch.tensor([V.SEQ_FREE, 0, V.SEQ_KEEP], dtype=torch.int32, device="cuda")
    (src, src4), (dst, dst4) = states
    V.vatp_cache_copy(pt, src, dst, m)
    V.vatp_cache_copy(pt, src4, dst4, m)
    status, eps = _status(), torch.finfo(DT[dtype]).eps / 2
    for i in range(12):
        q = torch.randn(3, h, d, generator=g, device="cuda").to(DT[dtype])
        k, v = (_whole(g, 3, hk, d, dtype=dtype) for _ in range(2))
        got = []
        for step, c in ((V.vatp_decode_step, dst), (V.vatp_decode_step_q4, dst4)):
            out, evicted = torch.empty_like(q), torch.empty(3, hk, dtype=torch.int32, device="cuda")
            step(pt, c, q, k, v, out, evicted_pos=evicted, dev_status=status)
            got.append((out.double(), evicted))
        torch.cuda.synchronize()
        (o, e), (o4, e4) = got
        assert int(status) == 0
        if i == 0:                                                                 # the freed entry's only token
            assert torch.equal(o[0].view(hk, -1, d), v[0].double()[:, None].expand(hk, h // hk, d))
        # each side: its own rounding; p in 16 bits or more (2^-16 of values up to 8); logits, sums of d products up to 8 * 4.5, to
        # 2^-23 d 36 / sqrt(d) of a probability
        assert torch.all((o - o4).abs() <= eps * (o.abs() + o4.abs()) + 2 * 8 * (2.0 ** -16 + 2.0 ** -23 * 36 * d ** 0.5))
        assert torch.equal(e, e4)
        for name in ("pos", "len", "free_slot", "next_pos", "last_slot"):
            assert torch.equal(getattr(dst, name), getattr(dst4, name)), name
    assert dst.next_pos[0].tolist() == [12] * hk and dst.len.flatten().tolist() == [12] * hk + [23] * hk * 2
