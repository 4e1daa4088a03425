"""Rotary positions against the definition in 64 bits: types, layouts, parts of a
head, head sizes, strides, far and negative positions, in place, the gradient, and
graphs and streams.

Tolerances. The angle is exact to 2^-32 turns; its fp32 rest r, at most pi / 4, is
rounded twice (2^-23 r), and the series of sine and cosine to 2^-24 each at the last
step and as much before it: each is within 2^-22 of its value. A result sums two
products: (|a| + |b|) m times that, the rounding of m, of the products and of the sum
(3 of 2^-24): (|a| + |b|) m 2^-21 in all, and the output's own rounding: half a step,
and half of the type's least number."""
import math

import pytest
import torch

import paper_2510_15545_gb300 as tt

pytestmark = pytest.mark.gpu

F, H, E = torch.float32, torch.bfloat16, torch.float16
HALF = {t: torch.finfo(t).eps / 2 for t in (F, H, E)}
LEAST = {F: 2.0 ** -150, H: 2.0 ** -134, E: 2.0 ** -25}      # half of the least number


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    tt.load(build_if_missing=True)


def angles(positions, turns):
    """x F mod 2^64, exactly (int64 products wrap), as radians within a half turn."""
    return (positions.long()[:, None] * turns).double() * (2 * math.pi / 2.0 ** 64)


def expected(x, positions, turns, interleaved, mscale=1.0, transpose=False):
    """The result and its error bound."""
    n = turns.numel()
    c, s = (f(angles(positions, turns))[:, None] * mscale for f in (torch.cos, torch.sin))
    if transpose:
        s = -s
    y = x.double()
    a, b = (y[..., 0:2 * n:2], y[..., 1:2 * n:2]) if interleaved else (y[..., :n], y[..., n:2 * n])
    u, v, size = a * c - b * s, a * s + b * c, (a.abs() + b.abs()) * abs(mscale)
    out, bound = y.clone(), torch.zeros_like(y)
    at = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    for where, z in zip(at, (u, v)):
        out[..., where] = z
        bound[..., where] = size * 2.0 ** -21 * (1 + HALF[x.dtype]) + z.abs() * HALF[x.dtype] + LEAST[x.dtype]
    return out, bound


def make(N, Hq, Hk, D, dtype, seed=0, far=1 << 17):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((N, Hq + 2 * Hk, D), generator=gen, device="cuda").to(dtype)
    at = torch.randint(0, far, (N,), generator=gen, device="cuda", dtype=torch.int32)
    return x[:, :Hq], x[:, Hq:Hq + Hk], at


def check(q, k, at, turns, interleaved=False, mscale=1.0, transpose=False, **kw):
    want = [None if x is None else expected(x, at, turns, interleaved, mscale, transpose) for x in (q, k)]
    o = tt.tt_rope(q, k, at, turns, interleaved=interleaved, mscale=mscale, transpose=transpose, **kw)
    torch.cuda.synchronize()
    for name, x, w in (("q", q, want[0]), ("k", k, want[1])):
        if x is None:
            assert name not in o
            continue
        off = (o[name].double() - w[0]).abs()
        assert (off <= w[1]).all(), (name, (off - w[1]).max())
    return o


def turns_of(rot, **kw):
    return tt.rope_turns(tt.rope_freqs(rot, **kw))


@pytest.mark.parametrize("dtype", [F, H, E])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(8, 8), (8, 2), (64, 64), (64, 32), (64, 16), (64, 50), (80, 80),
                                   (80, 20), (96, 48), (128, 128), (128, 126), (128, 2), (256, 256),
                                   (256, 64), (256, 2), (248, 36)])
def test_layouts(dtype, interleaved, D, rot):
    q, k, at = make(7, 5, 3, D, dtype, seed=D + rot)
    check(q, k, at, turns_of(rot), interleaved)
    check(q, None, at, turns_of(rot), interleaved, mscale=1.3)
    check(q, k, at, turns_of(rot), interleaved, mscale=0.7, transpose=True)


@pytest.mark.parametrize("N", [0, 1, 2, 31, 32, 33, 257, 1000, 5000])
@pytest.mark.parametrize("Hq,Hk", [(1, 1), (32, 8), (7, 1), (9, 0), (100, 3)])
def test_sizes(N, Hq, Hk):
    q, k, at = make(N, Hq, max(Hk, 1), 64, H, seed=N)
    check(q, k if Hk else None, at, turns_of(64))


def test_far_and_negative_positions():
    """Positions to either end of 32 bits, whose angles no fp32 number holds."""
    at = torch.tensor([0, 1, -1, 2 ** 24, 2 ** 24 + 1, -2 ** 30, 2 ** 31 - 1, -2 ** 31],
                      dtype=torch.int32, device="cuda")
    q, k, _ = make(8, 4, 2, 128, F, seed=5)
    check(q, k, at, turns_of(128, base=500000.0))
    check(q, k, at, tt.rope_turns([1.0, -2.5, 0.0, math.pi, 1e-7, 100.25]), True)
    # a million: the angle in radians itself, formed in 64 bits
    at = torch.full((8,), 10 ** 6, dtype=torch.int32, device="cuda")
    f = tt.rope_freqs(128)
    o = tt.tt_rope(q, k, at, tt.rope_turns(f))
    c, s = torch.cos(1e6 * f).cuda(), torch.sin(1e6 * f).cuda()
    a, b = q[..., :64].double(), q[..., 64:].double()
    assert (o["q"][..., :64].double() - (a * c - b * s)).abs().max() < 5e-6


@pytest.mark.parametrize("scaling", [dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0),
                                     dict(scaling="parts", factor=8.0, original=8192, low=1, high=4)])
def test_scaled_contexts(scaling):
    q, k, at = make(100, 4, 2, 128, H, far=65536)
    check(q, k, at, turns_of(128, **scaling), mscale=0.1 * math.log(8.0) + 1)


@pytest.mark.parametrize("dtype", [F, H, E])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [128, 64, 30])
def test_in_place(dtype, interleaved, rot):
    """Of q and k both, of one of them, and what lies between the heads stays."""
    q, k, at = make(50, 6, 2, 128, dtype, seed=3)
    turns = turns_of(rot)
    want = tt.tt_rope(q, k, at, turns, interleaved=interleaved)
    whole = q._base.clone()
    q2, k2 = whole[:, :6], whole[:, 6:8]
    o = tt.tt_rope(q2, k2, at, turns, interleaved=interleaved, out=dict(q=q2, k=k2))
    assert o["q"] is q2 and torch.equal(q2, want["q"]) and torch.equal(k2, want["k"])
    assert torch.equal(whole[:, 8:], q._base[:, 8:])
    whole = q._base.clone()
    q2, k2 = whole[:, :6], whole[:, 6:8]
    o = tt.tt_rope(q2, k2, at, turns, interleaved=interleaved, out=dict(q=q2))
    assert torch.equal(q2, want["q"]) and torch.equal(o["k"], want["k"])
    assert torch.equal(k2, k)


def test_strides():
    """Heads outside tokens, gaps between heads, one head for all, one token for all."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((4, 60, 128), generator=gen, device="cuda").bfloat16()
    at = torch.arange(60, dtype=torch.int32, device="cuda") * 37
    turns = turns_of(128)
    q, k = x.transpose(0, 1), x[:2].transpose(0, 1)
    check(q, k, at, turns)
    check(x.view(4, 60, 128)[:, ::2].transpose(0, 1), None, at[:30], turns)
    out = torch.full((60, 4, 144), 7.0, dtype=H, device="cuda")
    check(q, k, at, turns, out=dict(q=out[:, :, 8:136]))
    assert (out[:, :, :8] == 7).all() and (out[:, :, 136:] == 7).all()
    check(x[0][:, None].expand(60, 9, 128), x[0, :1][None].expand(60, 1, 128), at, turns)
    one = x[:1, :1].as_strided((1, 1, 128), (1, 3, 1))
    check(one, None, at[:1], turns)


def test_numbers_that_are_not_finite_stay_in_their_pair():
    q, _, at = make(3, 2, 1, 64, H, seed=6)
    q = q.contiguous()
    q[1, 0, 5], q[2, 1, 40] = math.inf, math.nan
    o = tt.tt_rope(q, None, at, turns_of(64))["q"]
    bad = ~torch.isfinite(o)
    want = torch.zeros_like(bad)
    want[1, 0, [5, 37]] = True
    want[2, 1, [8, 40]] = True
    assert torch.equal(bad, want)


def test_more_than_2_to_the_31_elements():
    N, Hq, D = 70000, 256, 128
    q = torch.empty((N, Hq, D), dtype=H, device="cuda")
    q[-5:] = 1.0
    at = torch.arange(N, dtype=torch.int32, device="cuda")
    turns = turns_of(D)
    o = tt.tt_rope(q, None, at, turns, out=dict(q=q))["q"]
    want, bound = expected(torch.ones((5, Hq, D), dtype=H, device="cuda"), at[-5:], turns, False)
    assert ((o[-5:].double() - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype", [F, H, E])
@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient(dtype, interleaved):
    """The formula's: the transposed map of what comes from above."""
    q, k, at = make(33, 4, 2, 64, dtype, seed=7)
    turns, m = turns_of(48), 1.25
    q, k = (x.detach().clone().requires_grad_() for x in (q, k))
    ups = [torch.randn_like(q), torch.randn_like(k)]
    out = tt.rope(q, k, at, turns, interleaved=interleaved, mscale=m)
    grads = torch.autograd.grad(out, (q, k), ups)
    for g, up in zip(grads, ups):
        want, bound = expected(up, at, turns, interleaved, m, True)
        assert ((g.double() - want).abs() <= bound).all()


def test_gradient_against_differences():
    """Of a linear map and of a square, whose central differences are exact but for
    rounding: of the moved inputs (half a step), of the results, and of the gradient."""
    q, k, at = make(20, 3, 2, 64, F, seed=8)
    turns, m, h = turns_of(64), 0.9, 2.0 ** -7
    q, k = (x.detach().clone().requires_grad_() for x in (q, k))
    up, dq, dk = torch.randn_like(q), torch.randn_like(q), torch.randn_like(k)

    def loss(a, b):
        x, y = tt.rope(a, b, at, turns, interleaved=True, mscale=m)
        return (x.double() * up.double()).sum() + (y.double() * y.double()).sum()

    gq, gk = torch.autograd.grad(loss(q, k), (q, k))
    with torch.no_grad():
        diff = (loss(q + h * dq, k + h * dk) - loss(q - h * dq, k - h * dk)) / (2 * h)
        got = (gq.double() * dq.double()).sum() + (gk.double() * dk.double()).sum()
        off = 0.0
        for s in (h, -h):  # of each side's loss, then over 2 h
            for x, d, w in ((q, dq, up.abs().double()), (k, dk, None)):
                y, bound = expected(x + s * d, at, turns, True, m)
                w = 2 * y.abs() + bound if w is None else w
                moved = (x.abs() + h * d.abs()).double() * 2.0 ** -23
                pair = moved.view(*moved.shape[:2], -1, 2).sum(3, keepdim=True).expand(-1, -1, -1, 2)
                off += (w * (bound + pair.reshape(moved.shape) * m)).sum() / (2 * h)
        y, bound = expected(k, at, turns, True, m)
        for g, up_g, more, d in ((gq, up, 0.0, dq), (gk, 2 * y, 2 * bound + y.abs() * 2.0 ** -22, dk)):
            want, bound_g = expected(up_g.float(), at, turns, True, m, True)
            off += ((bound_g + 2 * m * more) * d.abs().double()).sum()
    assert abs((diff - got).item()) <= off.item()


def test_gradients_of_one_and_of_broadcast_inputs():
    q, k, at = make(10, 4, 2, 64, H, seed=9)
    turns = turns_of(64)
    q, k = (x.detach().clone().requires_grad_() for x in (q, k))
    a, b = tt.rope(q, k, at, turns)
    b.sum().backward()  # (from above: one number, strides of 0)
    assert q.grad is None
    want, bound = expected(torch.ones_like(k), at, turns, False, transpose=True)
    assert ((k.grad.double() - want).abs() <= bound).all()
    k.grad = None
    a, b = tt.rope(q, k, at, turns)
    a.sum().backward()
    assert k.grad is None and q.grad is not None
    # one head for all: its gradient sums those of the copies
    one = torch.randn((10, 1, 64), device="cuda", requires_grad=True)
    out = tt.rope(one.expand(10, 6, 64), None, at, turns)
    up = torch.randn_like(out)
    (g,) = torch.autograd.grad(out, one, up)
    want, bound = expected(up, at, turns, False, transpose=True)
    assert ((g.double() - want.sum(1, keepdim=True)).abs()
            <= bound.sum(1, keepdim=True) + 2.0 ** -21 * want.abs().sum(1, keepdim=True)).all()


def test_second_derivative():
    """The map is linear: the gradient's gradient is the map again."""
    q, _, at = make(5, 2, 1, 64, F, seed=10)
    turns = turns_of(64)
    q = q.detach().clone().requires_grad_()
    up = torch.randn_like(q, requires_grad=True)
    (g,) = torch.autograd.grad(tt.rope(q, None, at, turns), q, up, create_graph=True)
    d = torch.randn_like(q)
    (gg,) = torch.autograd.grad(g, up, d)
    want, bound = expected(d, at, turns, False)
    assert ((gg.double() - want).abs() <= bound).all()


def test_leaves_that_need_no_gradient():
    q, k, at = make(5, 2, 1, 64, F, seed=11)
    turns = turns_of(64)
    k = k.detach().clone().requires_grad_()
    a, b = tt.rope(q, k, at, turns)
    (a.sum() + b.sum()).backward()
    assert k.grad.shape == k.shape


class _Nothing(torch.autograd.Function):
    """A function that gives no gradient."""

    @staticmethod
    def forward(ctx, x):
        return x.clone()

    @staticmethod
    def backward(ctx, up):
        return None


def test_results_whose_gradients_do_not_come():
    q, k, at = make(5, 4, 2, 64, F, seed=21)
    turns = turns_of(64)
    q, k = (x.detach().clone().requires_grad_() for x in (q, k))
    a, b = tt.rope(q, k, at, turns)
    (_Nothing.apply(a).sum() + _Nothing.apply(b).sum()).backward()
    assert q.grad is None and k.grad is None
    a, b = tt.rope(q, k, at, turns)
    (_Nothing.apply(a).sum() + b.sum()).backward()
    assert q.grad is None
    want, bound = expected(torch.ones_like(k), at, turns, False, transpose=True)
    assert ((k.grad.double() - want).abs() <= bound).all()


def test_captured_in_a_graph():
    q, k, at = make(9, 4, 2, 128, H, seed=12)
    turns = turns_of(128)
    out = dict(q=torch.empty_like(q), k=torch.empty_like(k))
    tt.tt_rope(q, k, at, turns, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tt.tt_rope(q, k, at, turns, out=out)
    q.mul_(2.0)
    at.add_(100)
    graph.replay()
    torch.cuda.synchronize()
    for name, x in (("q", q), ("k", k)):
        want, bound = expected(x, at, turns, False)
        assert ((out[name].double() - want).abs() <= bound).all()


def test_a_step_captured_in_a_graph():
    """Forward and backward in one graph, as a training loop captures them."""
    q, k, at = make(9, 4, 2, 64, F, seed=13)
    turns = turns_of(64)
    q, k = (x.detach().clone().requires_grad_() for x in (q, k))
    up = torch.randn_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            a, b = tt.rope(q, k, at, turns)
            torch.autograd.grad(((a * up).sum() + b.sum(),), (q, k))
        del a, b
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, b = tt.rope(q, k, at, turns)
        grads = torch.autograd.grad(((a * up).sum() + b.sum(),), (q, k))
    at.add_(1000)
    graph.replay()
    torch.cuda.synchronize()
    want, bound = expected(up, at, turns, False, transpose=True)
    assert ((grads[0].double() - want).abs() <= bound).all()


def test_on_a_stream():
    q, k, at = make(4000, 32, 8, 128, H, seed=14)
    turns = turns_of(128)
    stream = torch.cuda.Stream()
    ready = torch.cuda.Event()
    ready.record()
    stream.wait_event(ready)
    o = tt.tt_rope(q, k, at, turns, stream=stream)
    with torch.cuda.stream(stream):
        copy = o["q"].clone()
    stream.synchronize()
    assert torch.equal(copy, tt.tt_rope(q, k, at, turns)["q"])
