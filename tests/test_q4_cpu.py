"""The 4-bit decode state and the copies between states without a GPU: the format's properties and what the host refuses."""
import ctypes as C

import pytest
import torch

from tests import q4_reference as Q


@pytest.fixture(scope="module")
def V():
    from paper_2406_12335_b200 import build
    build.build()
    from paper_2406_12335_b200 import vatp
    return vatp


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_format_clamps_nothing_and_is_off_by_half_a_step(dtype):
    g = torch.Generator().manual_seed(3)
    x = torch.randn(500, 128, generator=g) * torch.exp(4 * torch.randn(500, 4, generator=g)).repeat_interleave(32, -1)
    x += 20 * torch.randn(500, 1, generator=g)
    x = x.to(dtype)
    codes, sc, lo = Q.quantise(x)
    assert codes.min() == 0 and codes.max() == 15
    # (two roundings to 32 bits of the difference and one each of reciprocal and product: 15 steps times 2^-22)
    off = (x.double() - Q.values(codes, sc, lo)).abs().unflatten(-1, (-1, 32))
    assert torch.all(off <= sc[..., None] * (0.5 + 15 * 2.0 ** -22) + x.double().abs().unflatten(-1, (-1, 32)) * 2.0 ** -23)
    assert torch.all(lo <= x.double().unflatten(-1, (-1, 32)).amin(-1))


def test_format_of_single_groups():
    row = torch.zeros(4, 64)
    row[1] = 2.5                                      # constant, a bf16 value
    row[2, :32] = torch.linspace(-1.0, 14.0, 32)      # lo -1, sc 1
    row[3] = 1e-35 * torch.arange(64)                 # a range too small for a scale
    codes, sc, lo = Q.quantise(row)
    assert torch.all(codes[:2] == 0) and torch.all(sc[:2] == 0) and torch.all(lo[1] == 2.5)
    assert lo[2, 0] == -1.0 and sc[2, 0] == 1.0 and codes[2, 0] == 0 and codes[2, 31] == 15
    assert torch.all(sc[3] == 0) and torch.all(codes[3] == 0)
    b = Q.to_bytes(torch.arange(64)[None] % 16)[0]    # codes of channel c: c mod 16
    # channels 0, 1 | 2, 3 (group 0), 32, 33 | 34, 35 (group 1), then channels 4 .. 7 of both
    assert [int(x) for x in b[:8]] == [0x10, 0x32, 0x10, 0x32, 0x54, 0x76, 0x54, 0x76]


def _params(V, **kw):
    return V.make_params(**{**dict(batch=2, heads=4, seq_len=64, head_dim=64, dtype="f32", budget=16, n_sink=2, n_recent=4), **kw})


def _q4(V, base=1 << 20, **kw):
    """A struct of distinct, aligned, imaginary arrays."""
    names = ["k_cache", "v_cache", "acc", "vnorm", "pos", "len", "free_slot", "next_pos", "ring", "acc_fixed", "last_slot"]
    at = {n: base + (i << 20) for i, n in enumerate(names + ["k_params", "v_params"])}
    at.update(kw)
    return V.CacheQ4Struct(V.CacheStruct(*[at[n] for n in names]), at["k_params"], at["v_params"])


def test_struct_layout(V):
    assert C.sizeof(V.CacheQ4Struct) == 104 and V.CacheQ4Struct.k_params.offset == 88


def test_refusals_of_the_four_bit_calls(V):
    p, null = _params(V), None
    c, bad = _q4(V), [_q4(V, k_params=None), _q4(V, v_params=8), _q4(V, k_cache=None), _q4(V, len=None), _q4(V, acc=4)]
    compact = lambda p, c, k=16, v=16, win=null, kept=16: V.lib.vatp_compact_q4(C.byref(p), k, v, 16, 16, win, kept, C.byref(c), null, null)  # noqa: E731
    step = lambda p, c, q=16, out=16: V.lib.vatp_decode_step_q4(C.byref(p), C.byref(c), q, 16, 16, out, null, null, null)  # noqa: E731
    for b in bad:
        assert compact(p, b) == 1 and step(p, b) == 1
        assert V.lib.vatp_cache_unpack_q4(C.byref(p), C.byref(b), C.byref(_q4(V, 1 << 30).state), null, null) == 1
    assert compact(p, c, k=8) == 1 and compact(p, c, v=null) == 1 and compact(p, c, kept=null) == 1
    assert step(p, c, q=null) == 1 and step(p, c, out=8) == 1
    assert V.lib.vatp_decode_step_q4(C.byref(p), null, 16, 16, 16, 16, null, null, null) == 1
    assert compact(_params(V, head_dim=96), c) == 2 and step(_params(V, head_dim=96), c) == 2
    assert compact(_params(V, n_recent=15), c) == 1 and step(_params(V, n_sink=20), c) == 1
    w = _params(V, indicator="window", window=8)
    assert compact(w, c) == 1                                                      # no probability rows
    assert compact(_params(V, indicator="window", window=8, kv_heads=2), c, win=16) == 2
    assert step(w, _q4(V, ring=None)) == 1
    # more query heads than a step takes, more logits than the shared memory of a unit's CTAs holds
    assert step(_params(V, batch=1, heads=9, kv_heads=1), c) == 2
    assert step(_params(V, batch=1, heads=8, kv_heads=1, budget=1 << 20), c) == 2


def test_refusals_of_the_conversions(V):
    p, null = _params(V), None
    pack = lambda p, a, b: V.lib.vatp_cache_pack_q4(C.byref(p), C.byref(a), C.byref(b), null, null)  # noqa: E731
    unpack = lambda p, a, b: V.lib.vatp_cache_unpack_q4(C.byref(p), C.byref(a), C.byref(b), null, null)  # noqa: E731
    wide, narrow = _q4(V, 1 << 30).state, _q4(V)
    cap, units = 24, 8
    # rows of one form over rows of the other; arrays that overlap their counterparts by a part
    over = _q4(V, k_cache=(1 << 30) + units * cap * 64 * 4 - 16)
    assert pack(p, wide, over) == 1 and unpack(p, over, wide) == 1
    over = _q4(V, v_params=(1 << 30) + (1 << 20))                          # on the wide rows of v
    assert pack(p, wide, over) == 1
    over = _q4(V, acc=(1 << 30) + (2 << 20) + 16)
    assert pack(p, wide, over) == 1 and unpack(p, over, wide) == 1
    over = _q4(V, len=(1 << 30) + (5 << 20) + 4)
    assert pack(p, wide, over) == 1
    w = _params(V, indicator="window", window=8)
    assert pack(w, wide, _q4(V, ring=(1 << 24) + 8)) == 1                   # not 16-byte aligned
    assert pack(w, wide, _q4(V, acc_fixed=None)) == 1
    assert pack(_params(V, head_dim=32), wide, narrow) == 2


def test_refusals_of_the_copies(V):
    p, null = _params(V), None
    a, b = _q4(V, 1 << 30), _q4(V)
    copy = lambda p, a, b, n=2, B=16, m=16: V.lib.vatp_cache_copy(C.byref(p), C.byref(a.state), n, B, C.byref(b.state), m, null, null)  # noqa: E731
    copy4 = lambda p, a, b, n=2, B=16, m=16: V.lib.vatp_cache_copy_q4(C.byref(p), C.byref(a), n, B, C.byref(b), m, null, null)  # noqa: E731
    for f in (copy, copy4):
        assert f(p, a, b, m=null) == 1 and f(p, a, b, n=0) == 1 and f(p, a, b, B=0) == 1 and f(p, a, b, n=-3) == 1
        assert f(_params(V, head_dim=96), a, b) == 2
        assert f(p, _q4(V, 1 << 30, pos=None), b) == 1
        assert f(p, a, _q4(V, vnorm=(1 << 30) + (3 << 20) + 32)) == 1        # overlaps its counterpart by a part
        assert f(p, a, _q4(V, acc=(1 << 30) + (2 << 20))) == 1               # one array shared, the others not
        assert f(p, b, b, n=1) == 1 and f(p, b, b, B=8) == 1                 # one state under two descriptions
    assert copy4(p, a, _q4(V, k_params=8)) == 1
    assert V.lib.vatp_cache_copy(C.byref(p), null, 2, 16, C.byref(b.state), 16, null, null) == 1
    assert V.lib.vatp_cache_copy_q4(C.byref(p), null, 2, 16, C.byref(b), 16, null, null) == 1


def test_states_share_arrays_only_where_parameters_agree(V):
    p = _params(V)
    a = V.CacheQ4(p, device="cpu")
    b = V.Cache(p, device="cpu", share=a)
    assert b.acc is a.acc and b.struct.acc == a.struct.state.acc and b.k_cache.shape == (2, 4, 24, 64)
    assert a.k_codes.shape == (2, 4, 24, 32) and a.k_params.shape == (2, 4, 24, 2, 2)
    for other in (_params(V, budget=24), _params(V, batch=3), _params(V, indicator="window", window=8), _params(V, kv_heads=2)):
        with pytest.raises(ValueError):
            V.Cache(other, device="cpu", share=a)
    with pytest.raises(TypeError):
        V.vatp_cache_copy(p, a, b, None)


@pytest.mark.parametrize("name,kernels", [("pack_q4.cu", {"pack_q4_kernel", "unpack_q4_kernel"}), ("decode_q4.cu", {"decode_q4_kernel"}),
                                          ("cache_copy.cu", {"cache_copy_kernel"})])
def test_dependent_kernels_read_by_ordinary_loads(name, kernels):
    """As tests/test_dependent_launches_cpu.py for the other kernels; and none of those that write cache rows lets a successor start
    before it has finished, since a step requests rows before it waits."""
    import re

    from tests.test_dependent_launches_cpu import _code, _dependent_kernels
    text = _code(name)
    found = _dependent_kernels(text)
    assert {k for k, _, _ in found} == kernels
    for kernel, params, _ in found:
        assert not re.findall(r"const\s+[\w:]+\s*\*\s*__restrict__", params), kernel
    assert "__ldg" not in text and "ld.global.nc" not in text
    if name != "decode_q4.cu":
        assert "launch_dependents" not in text
