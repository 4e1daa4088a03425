"""tt_tree_attn over caches in 8 bits against the definition in 64 bits: what the
elements and scales stand for, as numbers of 64 bits, goes through the same reference
as for caches of 16 bits.

Tolerances. As there (scores, weights, output), with three additions.
Queries meet the e4m3 keys as sums of e4m3 pieces of q 2^-e, e the least with which the
row's largest element is 448 or less, so that it is over 224. Each piece takes four binary
digits off what is left, until that is below 2^-9, the distance of the smallest e4m3
numbers: then it is off by half of that, 2^-10, which is less than 2^-17 of the largest
element. That times the keys' sizes joins a score's error.
Weights of cached keys are fp16 numbers, of a row's sum in units in which its largest is
2^7 or more; with few rows they take the values' scales, relative to the largest scale 2^k so
far. Beyond 2^-11 of each they are off by half of fp16's least number, 2^-25, so by 2^-32 of
the largest; times 448 2^k, at most twice the largest value, for every key: 2^-31.
With many rows the values take the scales: they are off by 2^-25 2^k, k of the largest scale
so far, so by 2^-32 of the largest value, and their mean by no more.
"""
import ctypes
import dataclasses
import math

import pytest
import torch

import paper_2510_15545_gb300 as tt
from paper_2510_15545_gb300 import binding
from test_gpu_tree import Case, ancestors, make

pytestmark = pytest.mark.gpu

H, E = torch.bfloat16, torch.float16
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
NAN = float("nan")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    tt.load(build_if_missing=True)


def power(codes):
    return torch.where(codes == 255, NAN, torch.exp2(codes.double() - 127))


@dataclasses.dataclass
class Case8(Case):
    """k_cache and v_cache: e4m3; their scales' bytes beside them."""
    ks: torch.Tensor = None
    vs: torch.Tensor = None

    def numbers(self):
        """The caches as 64-bit numbers."""
        return (x.view(torch.uint8).view(E4M3).double()
                * power(s.repeat_interleave(16, 1).int())[..., None]
                for x, s in ((self.k_cache, self.ks), (self.v_cache, self.vs)))


def hold(x):
    """e4m3 elements and scale bytes of numbers [pages, page, heads, D]; where a number is
    not finite, NaN; groups with nothing finite have NaN for a scale."""
    P, page, Hkv, D = x.shape
    g = x.double().view(P, page // 16, 16, Hkv, D)
    fine = torch.isfinite(g)
    top = torch.where(fine, g.abs(), 0.0).amax((2, 4))
    m, e = torch.frexp(top)
    code = torch.where(top > 0, e - 9 + (m > 0.875).int() + 127, 1).clamp(min=1)
    y = g * torch.exp2(127 - code.double())[:, :, None, :, None]
    y = torch.where(fine, y, NAN).float().to(E4M3).view(torch.uint8)
    y = torch.where(fine, y, 0x7f).byte()
    code = torch.where(fine.any(4).any(2), code, 255)
    return y.view(P, page, Hkv, D).view(E4M3), code.byte()


def make8(*args, loud=1.0, **kw):
    c = make(*args, **kw)
    gen = torch.Generator(device="cuda").manual_seed(kw.get("seed", 0) + 1000)
    # (groups of many sizes; whatever slots that are not in use hold, NaN here)
    for x in (c.k_cache, c.v_cache):
        P, page, Hkv, _ = x.shape
        f = torch.exp2(torch.randint(-3, 3, (P, page // 16, Hkv), generator=gen, device="cuda").float() * loud)
        x.mul_(f.to(x.dtype).repeat_interleave(16, 1)[..., None])
    kq, ks = hold(c.k_cache)
    vq, vs = hold(c.v_cache)
    return Case8(c.q, c.k, c.v, kq, vq, c.table, c.lens, c.nodes, c.parents, ks, vs)


def expected(c, b, scale, skip_pages=()):
    """Output, its error bound, lse and its bound of request b's nodes."""
    page, (Hkv, D) = c.k_cache.shape[1], c.k.shape[1:]
    G = c.q.shape[1] // Hkv
    lo = sum(c.nodes[:b])
    n, L = c.nodes[b], c.lens[b]
    x = torch.arange(L, device="cuda")
    if skip_pages:
        x = x[~torch.isin(x // page, torch.tensor(skip_pages, device="cuda"))]
    at = c.table[b].long()[x // page]
    number = lambda y, s: (y.view(torch.uint8)[at, x % page].view(E4M3).double()  # noqa: E731
                           * power(s[at, x % page // 16].int())[..., None])
    k = torch.cat([number(c.k_cache, c.ks), c.k[lo:lo + n].double()])
    v = torch.cat([number(c.v_cache, c.vs), c.v[lo:lo + n].double()])
    seen = torch.cat([torch.ones((n, len(x)), dtype=torch.bool),
                      ancestors(n, None if c.parents is None else c.parents[b])], 1).cuda()
    q = c.q[lo:lo + n].double().view(n, Hkv, G, D)
    s = torch.einsum("nhgd,lhd->hgnl", q, k) * scale
    sizes = torch.einsum("nhgd,lhd->hgnl", q.abs(), k.abs()) * 2.0 ** -20
    sizes += torch.einsum("nhg,lh->hgnl", q.abs().amax(-1), k.abs().sum(-1)) * 2.0 ** -17
    es = (sizes * scale).masked_fill(~seen, 0).amax(-1)
    s = s.masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - lse[..., None])
    u = 2.0 ** -8 if c.q.dtype == H else 2.0 ** -11
    order = lambda y: y.permute(2, 0, 1, 3).reshape(n, Hkv * G, -1)  # noqa: E731
    out = order(torch.einsum("hgnl,lhd->hgnd", p, v))
    mean = order(torch.einsum("hgnl,lhd->hgnd", p, v.abs()))
    every = torch.einsum("nl,lhd->hnd", seen.double(), v.abs()).permute(1, 0, 2)
    every = every.repeat_interleave(G, 1)
    bound = (1.02 * u * (mean + out.abs()) + (2 * order(es[..., None]) + 2e-5) * mean
             + 2.0 ** -30 * every + 2.0 ** -25)
    if len(x):
        bound = bound + 2.0 ** -31 * len(x) * torch.nan_to_num(v[:len(x)].abs()).amax()
    flat = lambda y: y.permute(2, 0, 1).reshape(n, Hkv * G)  # noqa: E731
    return out, bound, flat(lse), flat(es) + 1e-5


def call(c, args=None, **kw):
    return tt.tt_tree_attn(*(c.args() if args is None else args), k_scale=c.ks, v_scale=c.vs, **kw)


def check(c, scale=None, requests=None, **kw):
    kw.setdefault("max_len", max(c.lens))
    kw.setdefault("max_nodes", max(1, max(c.nodes)))
    g = call(c, scale=scale, **kw)
    torch.cuda.synchronize()
    scale = c.q.shape[2] ** -0.5 if scale is None else scale
    assert g["status"][:len(c.lens)].tolist() == [0] * len(c.lens)
    lo = 0
    for b, n in enumerate(c.nodes):
        if n and (requests is None or b in requests):
            out, bound, lse, el = expected(c, b, scale)
            off = (g["out"][lo:lo + n].double() - out).abs() / bound
            assert off.max() <= 1, (b, off.max())
            off = (g["lse"][lo:lo + n].double() - lse).abs() / el
            assert off.max() <= 1, (b, "lse", off.max())
        lo += n
    return g


LENGTHS = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 130, 255, 256, 257, 500, 1000]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [H, E])
@pytest.mark.parametrize("page", [16, 48, 64, 128, 256])
def test_lengths(D, dtype, page):
    nodes = [1 + (7 * b) % 11 for b in range(len(LENGTHS))]
    check(make8(LENGTHS, nodes, 8, 2, D, page, dtype, seed=page))


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 1), (3, 3), (6, 2), (7, 1), (20, 4), (32, 8),
                                    (16, 1), (48, 1), (128, 1), (100, 1)])
@pytest.mark.parametrize("dtype", [H, E])
def test_heads(Hq, Hkv, dtype):
    check(make8([300, 0, 77], [5, 9, 33], Hq, Hkv, 128, 32, dtype, seed=Hq))
    check(make8([300, 0, 77], [1, 2, 3], Hq, Hkv, 64, 16, dtype, parents=None, seed=Hq + 1))


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 511, 512])
@pytest.mark.parametrize("parents", ["tree", "forest", None])
def test_nodes(n, parents):
    check(make8([200, 0, 33], [n, 1, max(1, n // 2)], 4, 2, 64, 16, H, parents=parents, seed=n))
    check(make8([129], [n], 5, 1, 128, 64, E, parents=parents, seed=n + 1))


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 1, 128), (9, 3, 64), (5, 1, 128), (32, 2, 64)])
@pytest.mark.parametrize("dtype", [H, E])
def test_several_row_tiles_over_long_caches(Hq, Hkv, D, dtype):
    check(make8([20001, 9000, 131, 0, 4097], [100, 33, 130, 65, 1], Hq, Hkv, D, 48, dtype, seed=9))


@pytest.mark.parametrize("L", [3000, 8191, 20001, 70000])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 1, 128), (4, 2, 64), (32, 8, 128)])
def test_long_caches(L, Hq, Hkv, D):
    check(make8([L, 5, L // 2 + 1], [9, 3, 17], Hq, Hkv, D, 64, H, seed=L))


def test_one_request_of_one_token():
    for L in (0, 1, 100, 1000, 5000):
        for dtype in (H, E):
            check(make8([L], [1], 32, 8, 128, 16, dtype, seed=L, parents=None))


def test_ragged_batches_with_empty_requests():
    gen = torch.Generator().manual_seed(3)
    lens = torch.randint(0, 1500, (70,), generator=gen).tolist()
    nodes = torch.randint(0, 12, (70,), generator=gen).tolist()
    check(make8(lens, nodes, 16, 4, 64, 32, H, seed=4))
    check(make8(lens, nodes, 8, 4, 128, 32, E, seed=5))


def test_single_tokens_of_many_requests():
    gen = torch.Generator().manual_seed(6)
    lens = torch.randint(0, 700, (300,), generator=gen).tolist()
    check(make8(lens, [1] * 300, 8, 2, 128, 16, H, seed=7, parents=None))


@pytest.mark.parametrize("Hq,Hkv,D,n", [(8, 2, 128, 4), (16, 4, 64, 3), (32, 1, 64, 4), (32, 8, 128, 9)])
@pytest.mark.parametrize("dtype", [H, E])
def test_items_that_follow_each_other_within_caches(Hq, Hkv, D, n, dtype):
    """The same bits each time."""
    gen = torch.Generator().manual_seed(31)
    lens = torch.randint(500, 3500, (150,), generator=gen).tolist()
    c = make8(lens, [n] * 150, Hq, Hkv, D, 64, dtype, seed=32)
    first = check(c, requests=range(0, 150, 7))
    for _ in range(20):
        g = call(c, max_len=max(lens), max_nodes=n)
        assert torch.equal(g["out"], first["out"]) and torch.equal(g["lse"], first["lse"])


@pytest.mark.parametrize("size", [0.05, 6.0])
def test_flat_and_sharp_softmax(size):
    for dtype in (H, E):
        check(make8([2000, 100], [8, 3], 8, 2, 128, 32, dtype, seed=11, size=size))


def test_scales_of_all_sizes():
    """Groups whose numbers differ by 2^24 beside each other."""
    for dtype, loud in ((H, 4.0), (E, 2.0)):
        check(make8([1000, 70], [5, 3], 4, 2, 64, 64, dtype, seed=12, loud=loud, size=2.0 ** -3))


@pytest.mark.parametrize("dtype", [H, E])
def test_queries_of_all_sizes(dtype):
    """Rows far apart in size, and elements within a row: pieces keep a row's own
    digits."""
    c = make8([700, 64], [5, 9], 8, 2, 128, 32, dtype, seed=13)
    gen = torch.Generator(device="cuda").manual_seed(13)
    c.q.mul_(torch.exp2(torch.randint(-6, 3, c.q.shape, generator=gen, device="cuda").float()).to(dtype))
    c.q.mul_(torch.exp2(torch.randint(-7, 1, (*c.q.shape[:2], 1), generator=gen, device="cuda").float()).to(dtype))
    c.q[0, 3] = 0.0
    check(c)


def test_running_maximum_that_keeps_rising():
    """Scores that rise from tile to tile, fall, and jump at the end."""
    for dtype in (H, E):
        for order in (1, -1):
            c = make8([3000, 2000], [4, 2], 4, 1, 64, 64, dtype, seed=12)
            c.q[:] = c.q.abs() * 0.5
            ramp = torch.linspace(-3, 3, 3000, device="cuda")[::1]
            ramp = ramp if order == 1 else ramp.flip(0)
            x = torch.empty(c.k_cache.shape, device="cuda")
            for b, L in enumerate(c.lens):
                s = torch.arange(L, device="cuda")
                x[c.table[b].long()[s // 64], s % 64] = ramp[:L, None, None]
            c.k_cache, c.ks = hold(x)
            check(c)


def test_drafted_keys_that_are_masked():
    """Own keys whose score is -inf have no weight; a row without any has none at
    all: output 0, lse -inf."""
    c = make8([0, 33], [2, 3], 2, 1, 64, 16, H, seed=13, parents=None)
    c.q[:, :, 0], c.k[:, :, 0] = 1.0, 0.0
    c.k[:2, :, 0] = -math.inf
    c.k[3, :, 0] = -math.inf
    g = call(c, max_len=40, max_nodes=3)
    assert (g["out"][:2] == 0).all() and (g["lse"][:2] == -math.inf).all()
    without = dataclasses.replace(c, k=c.k.clone(), v=c.v.clone(), parents=[[-1, 0], [-1, -1, 0]])
    without.k[3] = 0.0
    out, bound, lse, el = expected(without, 1, 0.125)
    for i in (0, 2):
        assert ((g["out"][2 + i].double() - out[i]).abs() <= bound[i]).all()
        assert ((g["lse"][2 + i].double() - lse[i]).abs() <= el[i]).all()


def test_other_requests_do_not_matter():
    """NaN in one request's tokens, cache, scales and query stays there."""
    for part in range(4):
        c = make8([100, 130, 90], [5, 6, 7], 4, 2, 64, 32, H, seed=14)
        mine = c.table[1].long()[:5]
        if part == 0:
            c.q[5:11] = NAN
        elif part == 1:
            c.k_cache.view(torch.uint8)[mine] = 0xff
        elif part == 2:
            c.ks[mine] = 255
        else:
            c.vs[mine] = 255
        g = check(c, requests=(0, 2))
        assert torch.isnan(g["out"][5:11]).all()


@pytest.mark.parametrize("dtype", [H, E])
def test_elements_that_are_nan(dtype):
    """A NaN value reaches its own element of every row, a NaN key whole rows of its
    head."""
    c = make8([300], [3], 4, 2, 64, 32, dtype, seed=15)
    clean = call(c, max_len=300, max_nodes=3)
    page, slot = int(c.table[0, 7]), 5
    c.v_cache.view(torch.uint8)[page, slot, 1, 9] = 0x7f
    g = call(c, max_len=300, max_nodes=3)
    bad = torch.isnan(g["out"])
    assert bad[:, 2:, 9].all() and bad.sum() == 6
    assert torch.equal(g["out"][~bad], clean["out"][~bad]) and torch.equal(g["lse"], clean["lse"])
    c.k_cache.view(torch.uint8)[page, slot, 0, 3] = 0xff
    g = call(c, max_len=300, max_nodes=3)
    assert torch.isnan(g["out"][:, :2]).all() and torch.isnan(g["lse"][:, :2]).all()
    assert torch.equal(g["lse"][:, 2:], clean["lse"][:, 2:])


@pytest.mark.parametrize("value", [math.inf, -math.inf, NAN])
def test_queries_that_are_not_finite(value):
    """Their rows are NaN, and no others."""
    c = make8([200, 30], [3, 2], 4, 2, 128, 32, H, seed=16)
    clean = call(c, max_len=200, max_nodes=3)
    c.q[1, 2, 77] = value
    g = call(c, max_len=200, max_nodes=3)
    assert torch.isnan(g["out"][1, 2]).all() and torch.isnan(g["lse"][1, 2])
    rest = torch.ones((5, 4), dtype=torch.bool, device="cuda")
    rest[1, 2] = False
    assert torch.equal(g["out"][rest], clean["out"][rest]) and torch.equal(g["lse"][rest], clean["lse"][rest])


@pytest.mark.parametrize("dtype", [H, E])
def test_values_that_are_not_finite_stay_in_their_branch(dtype):
    """A drafted token with infinite and NaN keys and values reaches its own
    descendants and no other branch."""
    up = [-1, 0, 0, 1, 2, 4, 3, -1]
    c = make8([150], [8], 4, 2, 64, 32, dtype, seed=30)
    c.parents = [up]
    clean = dataclasses.replace(c, k=c.k.clone(), v=c.v.clone())
    c.v[2, 0, 5], c.v[2, 1, 7], c.v[2, 1, 63] = math.inf, NAN, -math.inf
    c.k[6] = NAN  # (a leaf: itself only)
    g = call(c, max_len=150, max_nodes=8)
    out, bound, _, _ = expected(clean, 0, 0.125)
    off = (g["out"].double() - out).abs() <= bound
    for i in (0, 1, 3, 7):
        assert off[i].all(), i
    for i in (2, 4, 5):  # element by element
        x = g["out"][i]
        assert (x[:2, 5] == math.inf).all() and torch.isnan(x[2:, 7]).all()
        assert (x[2:, 63] == -math.inf).all()
        off[i, :2, 5], off[i, 2:, 7], off[i, 2:, 63] = True, True, True
        assert off[i].all(), i
    assert torch.isnan(g["out"][6]).all()


@pytest.mark.parametrize("dtype", [H, E])
def test_the_largest_values(dtype):
    """Elements of 448 and the largest scale that the type's numbers need."""
    c = make8([200], [3], 4, 2, 64, 16, dtype, seed=17)
    big = 61440.0 if dtype == E else 1.875 * 2.0 ** 100
    x = torch.randn(c.v_cache.shape, generator=torch.Generator(device="cuda").manual_seed(1),
                    device="cuda").double().clamp(-1, 1) * big
    c.v_cache, c.vs = hold(x)
    g = call(c, max_len=200, max_nodes=3)
    out, bound, _, _ = expected(c, 0, 0.125)
    assert ((g["out"].double() - out).abs() <= bound).all()


def test_strides():
    """Heads cut out of a fused projection, caches with the heads outermost, both
    caches in one tensor, scales within a larger one, a longer table."""
    c = make8([300, 70], [6, 9], 8, 2, 64, 32, H, seed=15)
    N, P = 15, c.k_cache.shape[0]
    g = check(c)
    fused = torch.full((N, 8 + 2 + 2 + 3, 64), NAN, dtype=H, device="cuda")
    fused[:, :8], fused[:, 8:10], fused[:, 10:12] = c.q, c.k, c.v
    both = torch.full((P, 2, 2, 32, 64), 0x7f, dtype=torch.uint8, device="cuda")
    both[:, 0] = c.k_cache.view(torch.uint8).transpose(1, 2)
    both[:, 1] = c.v_cache.view(torch.uint8).transpose(1, 2)
    both = both.view(E4M3)
    scales = torch.full((P, 2, 3, 7), 255, dtype=torch.uint8, device="cuda")
    scales[:, 0, :2, 3:5], scales[:, 1, :2, :2] = c.ks.transpose(1, 2), c.vs
    table = torch.full((2, 40), -7, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    d = dataclasses.replace(c, q=fused[:, :8], k=fused[:, 8:10], v=fused[:, 10:12],
                            k_cache=both[:, 0].transpose(1, 2), v_cache=both[:, 1].transpose(1, 2),
                            ks=scales[:, 0, :2, 3:5].transpose(1, 2), vs=scales[:, 1, :2, :2], table=table)
    h = check(d)
    assert torch.equal(g["out"], h["out"]) and torch.equal(g["lse"], h["lse"])
    h = call(dataclasses.replace(c, ks=c.ks.view(E8M0), vs=c.vs.view(E8M0)), max_len=300, max_nodes=9)
    assert torch.equal(g["out"], h["out"])


@pytest.mark.parametrize("D", [64, 128])
def test_keys_and_values_laid_out_differently(D):
    """Slots outermost in one cache, heads in the other."""
    c = make8([300, 70], [6, 9], 8, 2, D, 32, E, seed=18)
    g = check(c)
    for name in ("k_cache", "v_cache"):
        turned = getattr(c, name).view(torch.uint8).transpose(1, 2).contiguous().transpose(1, 2).view(E4M3)
        h = check(dataclasses.replace(c, **{name: turned}))
        assert torch.equal(g["out"], h["out"]) and torch.equal(g["lse"], h["lse"])


def test_offsets_beyond_32_bits():
    """Pages that start billions of bytes apart, their scales too."""
    c = make8([60, 40], [3, 2], 4, 2, 128, 32, H, seed=19, extra=0)
    g = check(c)
    far = {}
    for name in ("k_cache", "v_cache"):
        x = getattr(c, name).view(torch.uint8)
        step = 2 ** 31 + 64
        buf = torch.empty(x.shape[0] * step, dtype=torch.uint8, device="cuda")
        far[name] = buf.as_strided(x.shape, (step, 256, 128, 1))
        far[name].copy_(x)
        far[name] = far[name].view(E4M3)
    for name in ("ks", "vs"):
        x = getattr(c, name)
        buf = torch.empty(x.shape[0] * (2 ** 31 + 3), dtype=torch.uint8, device="cuda")
        far[name] = buf.as_strided(x.shape, (2 ** 31 + 3, 2, 1))
        far[name].copy_(x)
    h = check(dataclasses.replace(c, **far))
    assert torch.equal(g["out"], h["out"]) and torch.equal(g["lse"], h["lse"])


def test_bounds_above_what_is_there():
    """max_len and max_nodes may be larger than any request's."""
    c = make8([300, 0, 70], [6, 1, 9], 8, 2, 128, 32, H, seed=16)
    table = torch.zeros((3, 500), dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    c.table = table
    check(c, max_len=16000, max_nodes=512)
    check(c, max_len=300, max_nodes=9, scale=0.3)
    assert call(c)["status"].tolist() == [0, 0, 0]


def test_statuses():
    c = make8([100, 200, 50, 60, 30], [3, 4, 5, 6, 2], 4, 2, 64, 16, H, seed=18)
    args = list(c.args())
    full = check(c)
    # too long a cache, a negative length; their outputs stay as they were
    args[6] = torch.tensor([100, 201, 50, -1, 30], dtype=torch.int32, device="cuda")
    out = dict(out=torch.full((20, 4, 64), 7.0, dtype=H, device="cuda"))
    g = call(c, args, max_len=200, max_nodes=6, out=dict(out))
    assert g["status"].tolist() == [0, 2, 0, 2, 0]
    near = lambda lo, hi: (g["out"][lo:hi].float() - full["out"][lo:hi].float()).abs().max() < 0.05  # noqa: E731
    for lo, hi in ((0, 3), (7, 12), (18, 20)):
        assert near(lo, hi)
    assert (g["out"][3:7] == 7).all() and (g["out"][12:18] == 7).all()
    # more nodes than max_nodes
    args = list(c.args())
    g = call(c, args, max_len=200, max_nodes=5, out=dict(out))
    assert g["status"].tolist() == [0, 0, 0, 2, 0]
    # offsets that fall or leave the nodes (no two requests share nodes)
    args[7] = torch.tensor([0, 3, 7, 2, 2, 21], dtype=torch.int32, device="cuda")
    g = call(c, args, max_len=200, max_nodes=20)
    assert g["status"].tolist() == [0, 0, 8, 0, 8]
    assert near(0, 7)
    # pages out of range are left out, parents out of range make roots
    args = list(c.args())
    table = c.table.clone()
    table[1, 2], table[1, 5] = -1, c.k_cache.shape[0]
    up = args[8].clone()
    up[7 + 3], up[12 + 1] = 3, -2
    args[5], args[8] = table, up
    g = call(c, args, max_len=200, max_nodes=6)
    assert g["status"].tolist() == [0, 1, 1, 1, 0]
    outp, bound, _, _ = expected(c, 1, 0.125, skip_pages=(2, 5))
    assert ((g["out"][3:7].double() - outp).abs() <= bound).all()
    c.parents[2][3] = -1
    outp, bound, _, _ = expected(c, 2, 0.125)
    assert ((g["out"][7:12].double() - outp).abs() <= bound).all()


def test_every_page_out_of_range():
    """Nothing but the drafted tokens is left; and nothing at all for none."""
    c = make8([100, 40], [3, 1], 4, 2, 64, 16, H, seed=22)
    c.table[:] = -5
    g = call(c, max_len=100, max_nodes=3)
    assert g["status"].tolist() == [1, 1]
    alone = dataclasses.replace(c, lens=[0, 0])
    for b, lo, n in ((0, 0, 3), (1, 3, 1)):
        out, bound, _, _ = expected(alone, b, 0.125)
        assert ((g["out"][lo:lo + n].double() - out).abs() <= bound).all()


def test_outputs_streams_and_repeats():
    c = make8([3000, 10], [8, 2], 8, 2, 128, 16, H, seed=19)
    out = dict(out=torch.zeros_like(c.q), lse=torch.zeros(c.q.shape[:2], device="cuda"),
               status=torch.ones(2, dtype=torch.int32, device="cuda"))
    ws = tt.tt_tree_workspace(*c.args(), max_len=3000, max_nodes=8)
    ws.fill_(255)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = check(c, out=out, ws=ws, stream=side)
    assert all(g[k] is out[k] for k in out)
    h = check(c)
    assert torch.equal(g["out"], h["out"]) and torch.equal(g["lse"], h["lse"])
    # two calls of other sizes on one workspace, one after the other
    d = make8([10, 2500], [3, 7], 8, 2, 128, 16, H, seed=20)
    d.table = torch.cat([d.table, torch.zeros_like(d.table[:, :40])], 1)  # (room for 3000)
    a = call(c, max_len=3000, max_nodes=8, ws=ws)
    b = call(d, max_len=3000, max_nodes=8, ws=ws)
    assert torch.equal(a["out"], h["out"])
    assert torch.equal(b["out"], check(d, max_len=3000)["out"])


def test_two_calls_at_once():
    """On two streams, each with a workspace of its own."""
    cases = [make8([9000, 700], [8, 20], 8, 2, 128, 16, H, seed=40),
             make8([100] * 40, [3] * 40, 16, 4, 64, 32, E, seed=41)]
    want = [check(c) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    args = [c.args() for c in cases]  # (held until the streams are done with them)
    torch.cuda.synchronize()
    for _ in range(10):
        got = [call(c, a, stream=s, max_len=max(c.lens), max_nodes=max(c.nodes))
               for c, a, s in zip(cases, args, streams)]
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g["out"], w["out"]) and torch.equal(g["lse"], w["lse"])


def test_captured_in_a_graph():
    c = make8([3000, 700], [8, 2], 8, 2, 128, 16, H, seed=21)
    args = c.args()
    kw = dict(max_len=3000, max_nodes=8)
    call(c, args, **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g = call(c, args, **kw)
    c.q.neg_()
    args[6].copy_(torch.tensor([100, 690]))
    graph.replay()
    torch.cuda.synchronize()
    c.lens = [100, 690]
    h = check(c, max_len=3000)
    assert torch.equal(g["out"], h["out"])


def test_no_requests_and_no_nodes():
    c = make8([5], [1], 4, 2, 64, 16, H)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    g = call(c, (c.q[:0], c.k[:0], c.v[:0], c.k_cache, c.v_cache, c.table, i32([5]), i32([0, 0])))
    assert g["out"].shape == (0, 4, 64) and g["status"].tolist() == [0]
    g = call(c, (c.q[:0], c.k[:0], c.v[:0], c.k_cache, c.v_cache, c.table[:0], i32([]), i32([0])))
    assert g["out"].shape == (0, 4, 64)


def test_refusals():
    c = make8([50], [3], 4, 2, 64, 16, H)
    a = list(c.args())

    def refuse(error, at=None, to=None, **kw):
        b = list(a)
        if at is not None:
            b[at] = to
        kw.setdefault("k_scale", c.ks)
        kw.setdefault("v_scale", c.vs)
        with pytest.raises(error) as e:
            tt.tt_tree_attn(*b, **kw)
        return e.value

    for kw in (dict(scale=0.0), dict(scale=math.inf), dict(max_nodes=0), dict(max_nodes=513), dict(max_len=-1)):
        assert refuse(tt.TTError, **kw).code == binding.TT_ERR_INVALID_ARG
    for kw in (dict(k_scale=None), dict(v_scale=None), dict(k_scale=c.ks[:1]), dict(v_scale=c.vs.float()),
               dict(k_scale=c.ks.cpu()), dict(max_len=65)):
        refuse(ValueError, **kw)
    refuse(ValueError, 3, torch.zeros(c.k_cache.shape, dtype=H, device="cuda"))
    refuse(ValueError, 4, torch.zeros(c.k_cache.shape, dtype=H, device="cuda"))
    sixteen = torch.zeros(c.k_cache.shape, dtype=H, device="cuda")
    with pytest.raises(ValueError):  # scales beside a cache of 16 bits
        tt.tt_tree_attn(*a[:3], sixteen, sixteen, *a[5:], k_scale=c.ks, v_scale=c.vs)
    T = binding._tree(*a, None, None, None)
    S = binding._Scales(c.ks.data_ptr(), *c.ks.stride())
    P = ctypes.byref
    lib, p = tt.load(), ctypes.c_void_p(256)
    assert lib.tt_tree_attn8(P(T), P(S), None, p, 1 << 40, p, None, p, None) == binding.TT_ERR_INVALID_ARG
    assert lib.tt_tree_attn8(P(T), P(S), P(binding._Scales()), p, 1 << 40, p, None, p, None) == \
        binding.TT_ERR_INVALID_ARG


@pytest.mark.parametrize("dtype", [H, E])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 128), (4, 1, 64)])
def test_a_serving_loop(dtype, Hq, Hkv, D):
    """The operators as they are used: a prompt appended in 8 bits, then rounds of
    drafted trees that are rotated and scored, and whose accepted paths are appended;
    each round against the definition over what the cache stands for."""
    gen = torch.Generator(device="cuda").manual_seed(50)
    g2 = torch.Generator().manual_seed(50)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    B, page, per = 3, 32, 12
    turns = tt.rope_turns(tt.rope_freqs(D, base=500000.0))
    caches = [torch.zeros((B * per, page, Hkv, D), dtype=torch.uint8, device="cuda").view(E4M3) for _ in "kv"]
    scales = [torch.zeros((B * per, page // 16, Hkv), dtype=torch.uint8, device="cuda") for _ in "kv"]
    table = torch.randperm(B * per, generator=g2)[:B * per].view(B, per).int().cuda()
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dtype)  # noqa: E731
    prompt = [100, 1, 37]
    off = i32([0, 100, 101, 138])
    o = tt.tt_cache_append(randn(138, Hkv, D), randn(138, Hkv, D), *caches, table, i32([0, 0, 0]), off,
                           k_scale=scales[0], v_scale=scales[1], turns=turns)
    lens = o["new_len"]
    assert lens.tolist() == prompt
    for _ in range(6):
        nodes = [6, 9, 3]
        up = [[-1] + [int(torch.randint(max(0, i - 3), i, (1,), generator=g2)) for i in range(1, n)] for n in nodes]
        depth = [[0] * n for n in nodes]
        for d, p in zip(depth, up):
            for i in range(1, len(p)):
                d[i] = d[p[i]] + 1
        off, N = i32([0, 6, 15, 18]), 18
        at = torch.cat([lens[b] + i32(d) for b, d in enumerate(depth)])
        q, k, v = randn(N, Hq, D), randn(N, Hkv, D), randn(N, Hkv, D)
        r = tt.tt_rope(q, k, at, turns)
        c = Case8(r["q"], r["k"], v, *caches, table, lens.tolist(), nodes, up, *scales)
        check(c, max_len=per * page, max_nodes=9)
        paths, keep = [], []
        for p in up:  # the branch of a request's last token
            branch, i = [], len(p) - 1
            while i >= 0:
                branch.insert(0, i)
                i = p[i]
            keep.append(len(branch))
            paths += branch + [0] * (len(p) - len(branch))
        o = tt.tt_cache_append(r["k"], v, *caches, table, lens, off, k_scale=scales[0], v_scale=scales[1],
                               keep=i32(keep), path=i32(paths))
        assert o["status"].tolist() == [0, 0, 0]
        lens = o["new_len"]
