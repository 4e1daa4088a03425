"""Rotary positions on the host: struct layouts, the frequencies of every scaling,
their turns, and the refusals, each of which comes back before the library touches
a GPU."""
import ctypes
import math
from fractions import Fraction

import pytest
import torch

import paper_2510_15545_gb300 as tt
from paper_2510_15545_gb300 import _build, binding

P = ctypes.byref
INVALID, UNSUPPORTED = 1, 2
MEMORY = 1 << 20  # stands for device memory; never read or written


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return tt.load()


def test_struct_layouts():
    assert ctypes.sizeof(binding._RopeConfig) == 48 and binding._RopeConfig.base.offset == 8
    assert ctypes.sizeof(binding._RopePlan) == 24 and binding._RopePlan.mscale.offset == 16
    R = binding._Rotate
    assert R.positions.offset == 24 and R.q.offset == 32 and R.k_out.offset == 104
    assert R.plan.offset == 128 and ctypes.sizeof(R) == 152
    assert binding._ROTATE.size == ctypes.sizeof(R)


@pytest.mark.parametrize("rot", [2, 4, 10, 64, 128, 256])
@pytest.mark.parametrize("base", [10000.0, 500000.0, 1.0])
def test_frequencies(lib, rot, base):
    plain = tt.rope_freqs(rot, base=base)
    assert plain.dtype is torch.float64 and plain.shape == (rot // 2,)
    for i, f in enumerate(plain.tolist()):
        assert f == pytest.approx(base ** (-2.0 * i / rot), rel=1e-14)
    assert torch.allclose(tt.rope_freqs(rot, base=base, scaling="linear", factor=8.0), plain / 8,
                          rtol=1e-15, atol=0)


def test_scaled_by_base():
    """The fastest pair stays, the slowest is slowed by the whole factor."""
    plain, scaled = tt.rope_freqs(64), tt.rope_freqs(64, scaling="base", factor=4.0)
    assert scaled[0] == plain[0] == 1.0
    assert scaled[-1].item() == pytest.approx(plain[-1].item() / 4, rel=1e-12)


def test_scaled_by_parts():
    plain = tt.rope_freqs(128, base=500000.0)
    f = tt.rope_freqs(128, base=500000.0, scaling="parts", factor=8.0, original=8192, low=1, high=4)
    turns = 8192 * plain / (2 * math.pi)
    fast, slow = turns >= 4, turns <= 1
    assert fast.any() and slow.any() and (~fast & ~slow).any()
    assert torch.equal(f[fast], plain[fast])
    assert torch.allclose(f[slow], plain[slow] / 8, rtol=1e-15, atol=0)
    g = (turns - 1) / 3
    want = plain * ((1 - g) / 8 + g)
    assert torch.allclose(f[~fast & ~slow], want[~fast & ~slow], rtol=1e-13, atol=0)


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=-2),
                                dict(rot_dim=258), dict(base=0.0), dict(base=-1.0),
                                dict(base=math.nan), dict(base=math.inf),
                                dict(scaling="linear", factor=0.0),
                                dict(scaling="linear", factor=math.inf),
                                dict(scaling="base", factor=-2.0),
                                dict(scaling="base", rot_dim=2),
                                dict(scaling="parts", original=0.0),
                                dict(scaling="parts", original=100.0, low=4.0, high=4.0),
                                dict(scaling="parts", original=100.0, low=math.nan)])
def test_frequencies_refused(lib, kw):
    kw.setdefault("rot_dim", 64)
    with pytest.raises(tt.TTError) as e:
        tt.rope_freqs(**kw)
    assert e.value.code == INVALID


def test_unknown_scaling_is_refused(lib):
    with pytest.raises(ValueError):
        tt.rope_freqs(64, scaling="longer")
    c = binding._RopeConfig(64, 4, 10000.0, 1.0, 1.0, 1.0, 2.0)
    out = (ctypes.c_double * 32)()
    assert lib.tt_rope_freqs(P(c), out) == INVALID
    assert lib.tt_rope_freqs(None, out) == INVALID
    assert lib.tt_rope_freqs(P(binding._RopeConfig(64, 0, 10000.0)), None) == INVALID


def test_turns(lib):
    """Within 2^-52 of a turn per position, relative (the division and the constant of
    2 pi are rounded)."""
    freqs = [1.0, 0.3, 1e-3, 1e-9, 0.0, 6.25, 100.0, -0.5, -1e-30, 3.0 * math.pi]
    turns = tt.rope_turns(freqs, "cpu")
    assert turns.dtype is torch.int64
    two_pi = Fraction(62831853071795864769252867665590, 10 ** 31)
    for f, t in zip(freqs, turns.tolist()):
        want = Fraction(f) / two_pi
        got = Fraction(t % 2 ** 64, 2 ** 64)
        off = abs((got - want + Fraction(1, 2)) % 1 - Fraction(1, 2))
        assert off <= abs(want) * Fraction(1, 2 ** 51) + Fraction(1, 2 ** 53), f
    assert tt.rope_turns([], "cpu").numel() == 0
    for bad in (math.nan, math.inf):
        with pytest.raises(tt.TTError):
            tt.rope_turns([1.0, bad], "cpu")


def heads(data=MEMORY, token=1024, head=128):
    return binding._Heads(data, token, head)


def rotate(lib, **kw):
    f = dict(n_tokens=4, dtype=1, head_dim=128, n_q_heads=8, n_k_heads=2, transpose=0,
             positions=MEMORY, q=heads(), k=heads(), q_out=heads(2 * MEMORY), k_out=heads(3 * MEMORY),
             plan=binding._RopePlan(MEMORY, 128, 0, 1.0))
    f.update(kw)
    return lib.tt_rope(P(binding._Rotate(**f)), None)


@pytest.mark.parametrize("kw", [
    dict(n_tokens=-1), dict(dtype=-1), dict(dtype=3), dict(head_dim=4), dict(head_dim=264),
    dict(head_dim=100), dict(n_q_heads=0), dict(n_k_heads=-1), dict(transpose=2),
    dict(positions=None),
    dict(plan=binding._RopePlan(None, 128, 0, 1.0)), dict(plan=binding._RopePlan(MEMORY + 4, 128, 0, 1.0)),
    dict(plan=binding._RopePlan(MEMORY, 0, 0, 1.0)), dict(plan=binding._RopePlan(MEMORY, 63, 0, 1.0)),
    dict(plan=binding._RopePlan(MEMORY, 130, 0, 1.0)), dict(plan=binding._RopePlan(MEMORY, 128, 2, 1.0)),
    dict(plan=binding._RopePlan(MEMORY, 128, 0, math.nan)),
    dict(plan=binding._RopePlan(MEMORY, 128, 0, math.inf))])
def test_refusals(lib, kw):
    assert rotate(lib, **kw) == INVALID


@pytest.mark.parametrize("bad", [heads(None), heads(MEMORY + 8), heads(token=1020), heads(token=-1024),
                                 heads(head=4)])
def test_heads_refused(lib, bad):
    for name in ("q", "k", "q_out", "k_out"):
        assert rotate(lib, **{name: bad}) == INVALID


@pytest.mark.parametrize("out", [heads(2 * MEMORY, 0, 128), heads(2 * MEMORY, 1024, 0),
                                 heads(2 * MEMORY, 1024, 64), heads(2 * MEMORY, 512, 128),
                                 heads(2 * MEMORY, 128, 128), heads(2 * MEMORY, 128, 256)])
def test_outputs_whose_heads_overlap_are_refused(lib, out):
    assert rotate(lib, q_out=out) == INVALID


def test_outputs_over_other_strides_of_their_input_are_refused(lib):
    assert rotate(lib, q=heads(), q_out=heads(MEMORY, 2048, 128)) == INVALID
    assert rotate(lib, k=heads(), k_out=heads(MEMORY, 1024, 256)) == INVALID


def test_no_tokens_need_nothing(lib):
    none = heads(None)
    assert rotate(lib, n_tokens=0, positions=None, q=none, k=none, q_out=none, k_out=none) == 0


def test_too_many_heads(lib):
    assert rotate(lib, n_q_heads=65536, q=heads(token=65536 * 128),
                  q_out=heads(2 * MEMORY, 65536 * 128)) == UNSUPPORTED


def test_tensors_on_the_host_are_refused():
    x, at = torch.zeros((3, 2, 64)), torch.zeros(3, dtype=torch.int32)
    turns = tt.rope_turns(tt.rope_freqs(64), "cpu")
    with pytest.raises(ValueError, match="GPU"):
        tt.tt_rope(x, None, at, turns)


@pytest.fixture
def anywhere(monkeypatch):
    """The binding's checks on host tensors; a call that passes them fails."""
    class Library:
        def __getattr__(self, name):
            raise AssertionError(name)
    monkeypatch.setattr(binding, "_gpu_of", lambda *t: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(binding, "load", Library)


def test_shapes_and_types_refused(anywhere):
    x, at = torch.zeros((3, 2, 64)), torch.zeros(3, dtype=torch.int32)
    turns = torch.zeros(32, dtype=torch.int64)
    for bad in (dict(q=x[0]), dict(k=x[:2]), dict(k=x[:, :, :32]), dict(k=x.bfloat16()),
                dict(positions=at[:2]), dict(positions=at.long()), dict(turns=turns.int()),
                dict(turns=turns[::2]), dict(q=x.transpose(1, 2)), dict(out=dict(q=x[:2])),
                dict(out=dict(k=x)), dict(out=dict(q=x.bfloat16()))):
        a = dict(q=x, k=None, positions=at, turns=turns)
        a.update(bad)
        with pytest.raises(ValueError):
            tt.tt_rope(**a)
    with pytest.raises(TypeError):
        tt.tt_rope(x.double(), None, at, turns)
