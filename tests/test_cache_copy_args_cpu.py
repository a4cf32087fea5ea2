"""What the binding refuses before a copy of entries is launched: maps and states that the C call would take at their word."""
import pytest
import torch


@pytest.fixture(scope="module")
def V():
    from paper_2406_12335_b200 import build
    build.build()
    from paper_2406_12335_b200 import vatp
    return vatp


def _params(V, **kw):
    return V.make_params(**{**dict(batch=3, heads=4, seq_len=64, head_dim=64, dtype="f32", budget=16), **kw})


@pytest.fixture
def launched(V, monkeypatch):
    """The C calls' stand-ins: the arguments of those that the binding made."""
    made = []
    for name in ("vatp_cache_copy", "vatp_cache_copy_q4"):
        monkeypatch.setattr(V.lib, name, lambda *a: made.append(a) or 0)
    monkeypatch.setattr(V, "_stream", lambda stream=None: 0)
    return made


@pytest.mark.parametrize("form", ["Cache", "CacheQ4"])
def test_maps(V, launched, form):
    p = _params(V)
    a, b = getattr(V, form)(p, device="cpu"), getattr(V, form)(p, device="cpu")
    good = torch.tensor([0, V.SEQ_KEEP, 2], dtype=torch.int32)
    V.vatp_cache_copy(p, a, b, good)
    assert len(launched) == 1
    for bad in (good.long(), good.float(), good[:2], torch.cat((good, good)), good[None], torch.stack((good, good), 1)[:, 0], good.to("meta")):
        with pytest.raises(ValueError, match="src_of"):
            V.vatp_cache_copy(p, a, b, bad)
    assert len(launched) == 1


@pytest.mark.parametrize("form", ["Cache", "CacheQ4"])
def test_states(V, launched, form):
    p, m = _params(V), torch.zeros(3, dtype=torch.int32)
    state = lambda **kw: getattr(V, form)(_params(V, **kw), device="cpu")  # noqa: E731
    b = state()
    for a in (state(batch=7), state(budget=40)):                    # the source's own
        V.vatp_cache_copy(p, a, b, m)
    assert len(launched) == 2 and [x[2:4] for x in launched] == [(7, 16), (3, 40)]
    others = [dict(kv_heads=2), dict(head_dim=128), dict(indicator="window", window=5)]
    for kw in others + [dict(budget=17), dict(batch=4)] + ([dict(dtype="bf16")] if form == "Cache" else []):
        with pytest.raises(ValueError, match="other parameters"):
            V.vatp_cache_copy(p, b, state(**kw), m)
    for kw in others:
        with pytest.raises(ValueError, match="other parameters"):
            V.vatp_cache_copy(p, state(**kw), b, m)
    assert len(launched) == 2
    if form == "CacheQ4":                                           # rows in 4 bits have no type of their own
        V.vatp_cache_copy(p, state(dtype="bf16"), state(dtype="bf16"), m)
        assert len(launched) == 3
