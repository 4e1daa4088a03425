"""tt_tree_attn over caches in 8 bits at the ends of its numbers: NaN under scores that
jump, values far smaller than what scales them, and the largest ones.

Tolerances. A score's error is that of the tests beside this one (fp32 products, pieces of
queries). Weights of cached keys are fp16 numbers of a row's sum in units in which its
largest is 2^7 or more: beyond 2^-11 of each they are off by 2^-25, so by 2^-32 of the
largest, times the sizes of all values. Cached values are fp16 numbers in units of 2^-7 of the
largest scale so far: off by 2^-32 of it; those of scales from 2^-32 of it on, which are at most
448 times theirs, are none: off by 2^-23. Their mean is off by no more. Weights of drafted keys
have the inputs' type (in fp16 off by 2^-32 of the largest, too), the output is rounded to it
once (in fp16 to 2^-25 at least)."""
import math

import pytest
import torch

import paper_2510_15545_gb300 as tt
from test_gpu_tree import ancestors
from test_gpu_tree8 import E, H, call, hold, make8, power

pytestmark = pytest.mark.gpu

NAN = float("nan")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    tt.load(build_if_missing=True)


def where(c, b):
    """Pages and slots of request b's cached keys, in order."""
    page = c.k_cache.shape[1]
    x = torch.arange(c.lens[b], device="cuda")
    return c.table[b].long()[x // page], x % page


def expected(c, b, scale, unit):
    """Output, its error bound and lse of request b's nodes; cached values are off by 2^-25
    of `unit` at most."""
    Hkv, D = c.k.shape[1:]
    G = c.q.shape[1] // Hkv
    lo, n = sum(c.nodes[:b]), c.nodes[b]
    at, slot = where(c, b)
    number = lambda y, s: (y.view(torch.uint8)[at, slot].view(torch.float8_e4m3fn).double()  # noqa: E731
                           * power(s[at, slot // 16].int())[..., None])
    k = torch.cat([number(c.k_cache, c.ks), c.k[lo:lo + n].double()])
    v = torch.cat([number(c.v_cache, c.vs), c.v[lo:lo + n].double()])
    seen = torch.cat([torch.ones((n, len(at)), dtype=torch.bool),
                      ancestors(n, None if c.parents is None else c.parents[b])], 1).cuda()
    q = c.q[lo:lo + n].double().view(n, Hkv, G, D)
    s = torch.einsum("nhgd,lhd->hgnl", q, k) * scale
    es = torch.einsum("nhgd,lhd->hgnl", q.abs(), k.abs()) * 2.0 ** -20
    es += torch.einsum("nhg,lh->hgnl", q.abs().amax(-1), k.abs().sum(-1)) * 2.0 ** -17
    es = (es * scale).masked_fill(~seen, 0).amax(-1)
    s = s.masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - lse[..., None])
    u = 2.0 ** -8 if c.q.dtype == H else 2.0 ** -11
    order = lambda y: y.permute(2, 0, 1, 3).reshape(n, Hkv * G, -1)  # noqa: E731
    out = order(torch.einsum("hgnl,lhd->hgnd", p, v))
    mean = order(torch.einsum("hgnl,lhd->hgnd", p, v.abs()))
    every = torch.einsum("nl,lhd->hnd", seen.double(), v.abs()).permute(1, 0, 2).repeat_interleave(G, 1)
    bound = (1.02 * u * (mean + out.abs()) + (2 * order(es[..., None]) + 2e-5) * mean
             + 2.0 ** -32 * every + 2.0 ** -25 * unit)
    if c.q.dtype == E:
        bound = bound + 2.0 ** -25
    flat = lambda y: y.permute(2, 0, 1).reshape(n, Hkv * G)  # noqa: E731
    return out, bound, flat(lse), flat(es) + 1e-5


def check(c, requests, unit, scale=None, **kw):
    kw.setdefault("max_len", max(c.lens))
    kw.setdefault("max_nodes", max(c.nodes))
    g = call(c, scale=scale, **kw)
    scale = c.q.shape[2] ** -0.5 if scale is None else scale
    assert g["status"].tolist() == [0] * len(c.lens)
    for b in requests:
        lo, n = sum(c.nodes[:b]), c.nodes[b]
        out, bound, lse, el = expected(c, b, scale, unit)
        off = (g["out"][lo:lo + n].double() - out).abs() / bound
        assert off.max() <= 1, (b, off.max())  # (NaN fails, too)
        off = (g["lse"][lo:lo + n].double() - lse).abs() / el
        assert off.max() <= 1, (b, "lse", off.max())
    return g


@pytest.mark.parametrize("n", [1, 9, 40])  # of few rows, and of many
@pytest.mark.parametrize("D,dtype", [(64, H), (128, E)])
@pytest.mark.parametrize("what", ["key", "scale", "drafted"])
def test_rows_stay_nan_when_scores_jump(n, D, dtype, what):
    """A NaN key comes early, scores that make what came before it nothing later: the row's
    sum is NaN, not that of what came later."""
    B, L = 150, 128 * 7
    c = make8([L] * B, [n] * B, 2, 1, D, 64, dtype, seed=1, parents=None)
    c.q.fill_(8.0)
    keys = torch.zeros(c.k_cache.shape, device="cuda")
    for b in range(B):
        at, slot = where(c, b)
        keys[at[128 * 5:], slot[128 * 5:]] = 8.0  # (scores of 8 * 8 * sqrt(D), base e)
    c.k_cache, c.ks = hold(keys)
    clean = call(c, max_len=L, max_nodes=n)
    assert torch.isfinite(clean["out"]).all() and torch.isfinite(clean["lse"]).all()
    if what == "drafted":
        c.k[0::n] = NAN  # (every token's first ancestor)
    for b in range(B if what != "drafted" else 0):
        at, slot = where(c, b)
        for x in (5, 128 + 7):  # (of tiles one after the other)
            if what == "key":
                c.k_cache.view(torch.uint8)[at[x], slot[x], 0, 3] = 0x7f
            else:
                c.ks[at[x], slot[x] // 16] = 255
    g = call(c, max_len=L, max_nodes=n)
    assert torch.isnan(g["out"]).all() and torch.isnan(g["lse"]).all()


@pytest.mark.parametrize("n", [1, 9, 40])
def test_rows_of_nan_and_scores_far_below_zero(n):
    """A NaN key beside keys whose scores are all negative."""
    B, L = 150, 128 * 5
    c = make8([L] * B, [n] * B, 2, 1, 64, 64, H, seed=2, parents=None)
    c.q.fill_(8.0)
    c.k.fill_(-8.0)
    c.k_cache, c.ks = hold(torch.full(c.k_cache.shape, -8.0, device="cuda"))
    check(c, range(0, B, 37), 1.0)
    for b in range(0, B, 2):
        at, slot = where(c, b)
        c.k_cache.view(torch.uint8)[at[200], slot[200], 0, 3] = 0x7f
    g = call(c, max_len=L, max_nodes=n)
    bad = (torch.arange(B, device="cuda") % 2 == 0).repeat_interleave(n)
    assert torch.isnan(g["out"][bad]).all() and torch.isnan(g["lse"][bad]).all()
    assert torch.isfinite(g["out"][~bad]).all() and torch.isfinite(g["lse"][~bad]).all()


def strong_and_weak(c, D, lift):
    """Keys: one in each of the first four tiles whose weight is e^lift of all others'."""
    c.q.fill_(1.0)
    c.k.fill_(0.0)
    keys = torch.zeros(c.k_cache.shape, device="cuda")
    for b in range(len(c.lens)):
        at, slot = where(c, b)
        for x in range(3, 512, 128):
            keys[at[x], slot[x]] = lift / math.sqrt(D)
    c.k_cache, c.ks = hold(keys)


@pytest.mark.parametrize("n", [1, 8, 40])
@pytest.mark.parametrize("D,dtype", [(64, E), (128, E), (64, H)])
def test_small_values_of_many_weak_keys(n, D, dtype):
    """Thousands of keys whose weights are e^-10 of the largest, with values far below
    what the drafted ones' may be: together they count."""
    B, L = 304, 4096 + 77
    c = make8([L] * B, [n] * B, 2, 1, D, 64, dtype, seed=3, parents=None)
    strong_and_weak(c, D, 10.0)
    gen = torch.Generator(device="cuda").manual_seed(3)
    values = torch.randn(c.v_cache.shape, generator=gen, device="cuda").abs_().mul_(2.0 ** -11)
    c.v_cache, c.vs = hold(values)
    c.v.mul_(2.0 ** -11)
    check(c, (0, 1, 150, 303), 1.0 if dtype == E else 2.0 ** -17)


@pytest.mark.parametrize("n", [1, 8, 40])
@pytest.mark.parametrize("dtype", [H, E])
def test_scales_far_apart(n, dtype):
    """Values of 1 in keys that do not count beside values of 2^-14 in those that do."""
    B, L, D = 304, 4096 + 77, 64
    c = make8([L] * B, [n] * B, 2, 1, D, 64, dtype, seed=4, parents=None)
    strong_and_weak(c, D, 10.0)
    keys, values = c.numbers()
    gen = torch.Generator(device="cuda").manual_seed(4)
    values = torch.randn(c.v_cache.shape, generator=gen, device="cuda").abs_().mul_(2.0 ** -14)
    for b in range(B):
        at, slot = where(c, b)
        keys[at[16:32], slot[16:32]] = -8.0  # (64 below the weak ones)
        values[at[16:32], slot[16:32]] = 1.0
    c.k_cache, c.ks = hold(keys)
    c.v_cache, c.vs = hold(values)
    c.v.mul_(2.0 ** -14)
    check(c, (0, 1, 150, 303), 1.0 if dtype == E else 2.0 ** -8)


@pytest.mark.parametrize("n", [1, 3, 60])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,L", [(1, 20001), (3, 3000), (2, 130), (200, 700)])
def test_the_largest_values_of_bf16(n, D, B, L):
    """Cached values up to the type's largest, in items that are cut and in whole ones."""
    c = make8([L] * B, [n] * B, 4, 2, D, 16, H, seed=5)
    gen = torch.Generator(device="cuda").manual_seed(5)
    values = torch.rand(c.v_cache.shape, generator=gen, device="cuda").double() * 2 - 1
    values.sign_().mul_(1.875 * 2.0 ** 127)
    values[..., ::2] = values[..., ::2].abs()  # (means near the largest as well)
    c.v_cache, c.vs = hold(values)
    check(c, range(0, B, 67), 2.0 ** 120)


@pytest.mark.parametrize("n", [1, 3, 60, 200])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("power_of_2", [41, 53, 60, 100, 127])
def test_large_drafted_values_of_bf16(n, D, power_of_2):
    """Drafted values far above any usual ones, alone and beside cached ones of their
    size."""
    for B, L in ((1, 0), (4, 300), (160, 130)):
        c = make8([L] * B, [n] * B, 4, 2, D, 16, H, seed=6, parents="forest")
        gen = torch.Generator(device="cuda").manual_seed(6)
        c.v[:] = ((torch.rand(c.v.shape, generator=gen, device="cuda").double() * 2 - 1)
                  * 1.875 * 2.0 ** power_of_2).to(H)
        c.v[..., ::2] = c.v[..., ::2].abs()
        # (numbers of up to 2^E make the unit 2^(E - 102) at the most)
        check(c, range(0, B, 53), max(1.0, 2.0 ** (power_of_2 - 102)))
        values = torch.randn(c.v_cache.shape, generator=gen, device="cuda").clamp_(-3, 3).double()
        c.v_cache, c.vs = hold(values * 2.0 ** (power_of_2 - 2))
        check(c, range(0, B, 53), 2.0 ** (power_of_2 - 8))


def test_large_drafted_values_stay_in_their_branch_and_item():
    """Rows that do not see them keep their digits, those of other requests every bit."""
    up = [-1, 0, 0, 1, 2]
    lens, nodes = [300, 150, 700], [4, 5, 6]
    c = make8(lens, nodes, 4, 2, 64, 32, H, seed=7)
    c.parents[1] = up
    clean = call(c, max_len=700, max_nodes=6)
    c.v[4 + 2] *= 2.0 ** 90
    g = check(c, (1,), 1.0, max_len=700, max_nodes=6)
    rest = torch.ones(15, dtype=torch.bool, device="cuda")
    rest[4:9] = False
    assert torch.equal(g["out"][rest], clean["out"][rest]) and torch.equal(g["lse"], clean["lse"])


@pytest.mark.parametrize("n", [3, 60])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("power_of_2", [60, 100, 126])
def test_rows_beside_large_drafted_values(n, D, power_of_2):
    """The first token of a request is large, the others do not see it: what their cached
    keys give counts to 2^-118 of it for each key (weights of 2^-25 in units of 2^-102 of it,
    of elements of up to 448 2^7 < 2^16, over sums of 2^7), and no more is lost."""
    B, L = 40, 300
    c = make8([L] * B, [n] * B, 4, 2, D, 16, H, seed=8)
    c.parents = [[-1] * n for _ in range(B)]
    c.v[0::n] = 2.0 ** power_of_2
    g = call(c, max_len=L, max_nodes=n)
    for b in (0, 39):
        out, bound, lse, el = expected(c, b, D ** -0.5, 1.0)
        bound = bound + L * 2.0 ** (power_of_2 - 118)
        off = (g["out"][b * n:b * n + n].double() - out).abs() / bound
        assert off.max() <= 1, (b, off.max())
        assert ((g["lse"][b * n:b * n + n].double() - lse).abs() <= el).all()


@pytest.mark.parametrize("n", [1, 9, 40])
@pytest.mark.parametrize("D,dtype", [(64, E), (128, E), (64, H), (128, H)])
@pytest.mark.parametrize("L", [100, 128 * 9])
def test_scales_at_the_end_of_their_units(n, D, dtype, L):
    """Scales of 2^-20 to 2^-36, and of that times the largest one of the head."""
    B = 34
    c = make8([L] * B, [n] * B, 2, 1, D, 16, dtype, seed=9)
    gen = torch.Generator(device="cuda").manual_seed(9)
    values = torch.randn(c.v_cache.shape, generator=gen, device="cuda").double().clamp(-3, 3)
    values[..., 1] = 3.0  # (between 224 and 448 times 2^-7)
    for b in range(B):
        at, slot = where(c, b)
        if dtype == E:
            values[at, slot] *= 2.0 ** (7 - 20 - b % 17)
        else:  # (16 keys have a scale of 2^-7, for one of their elements)
            values[at[16:], slot[16:]] *= 2.0 ** (-20 - b % 17)
            values[at[:16], slot[:16]] = 0.0
            values[at[:16], slot[:16], 0, 0] = 3.0
    c.v_cache, c.vs = hold(values)
    c.v.zero_()
    for b in range(B):
        check(c, (b,), 2.0 ** (-20 - b % 17) if dtype == E else 2.0 ** (2 - 7))
