"""tt_tree_attn against the definition in 64 bits: head layouts, both types, cache
lengths around every page and tile boundary (none and one among them), chains,
trees and forests of one node to the most, strides, stale slots, bad tables, a
cache of more than 2^31 elements, and the refusals.

Tolerances. A score has the error of a fp32 sum of the head's products, under
2^-20 of the sum of their sizes; it moves the log-normaliser by as much (and
1e-5 for its own sums) and a weight by that relative amount. The weights are
rounded to the inputs' type (u = 2^-8 or 2^-11 of each at most; fp16 weights keep
2^-30 of the largest as well), so the output is off by u sum p |v| and its own
rounding."""
import ctypes
import dataclasses
import math

import pytest
import torch

import paper_2510_15545_gb300 as tt
from paper_2510_15545_gb300 import binding

pytestmark = pytest.mark.gpu

H, E = torch.bfloat16, torch.float16
NAN = float("nan")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    tt.load(build_if_missing=True)


@dataclasses.dataclass
class Case:
    q: torch.Tensor
    k: torch.Tensor
    v: torch.Tensor
    k_cache: torch.Tensor
    v_cache: torch.Tensor
    table: torch.Tensor
    lens: list
    nodes: list
    parents: list  # per request; None: chains

    def args(self):
        off = [0]
        for n in self.nodes:
            off.append(off[-1] + n)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        up = None if self.parents is None else i32([p for ps in self.parents for p in ps])
        return (self.q, self.k, self.v, self.k_cache, self.v_cache, self.table, i32(self.lens),
                i32(off), up)


def make(lens, nodes, Hq, Hkv, D, page, dtype, parents="tree", seed=0, size=1.0, extra=2):
    """Random tokens and caches; slots past a request's length and pages that no
    request has hold NaN and infinities."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    g2 = torch.Generator().manual_seed(seed)
    B, N = len(lens), sum(nodes)
    randn = lambda *s: (torch.randn(s, generator=gen, device="cuda") * size).to(dtype)  # noqa: E731
    per = max(1, max((n + page - 1) // page for n in lens))
    pages = B * per + extra
    table = torch.randperm(pages, generator=g2)[:B * per].view(B, per).int()
    kc, vc = randn(pages, page, Hkv, D), randn(pages, page, Hkv, D)
    used = torch.zeros((pages, page), dtype=torch.bool)
    for b, n in enumerate(lens):
        x = torch.arange(n)
        used[table[b].long()[x // page], x % page] = True
    kc[~used.cuda()] = NAN
    vc[~used.cuda()] = math.inf
    if parents == "tree":
        parents = [[-1 if i == 0 else int(torch.randint(max(0, i - 5), i, (1,), generator=g2))
                    for i in range(n)] for n in nodes]
    elif parents == "forest":
        parents = [[int(torch.randint(-1, i, (1,), generator=g2)) if i else -1
                    for i in range(n)] for n in nodes]
    return Case(randn(N, Hq, D), randn(N, Hkv, D), randn(N, Hkv, D), kc, vc, table.cuda(),
                list(lens), list(nodes), parents)


def ancestors(n, up):
    sees = torch.zeros((n, n), dtype=torch.bool)
    for i in range(n):
        sees[i, i] = True
        p = i - 1 if up is None else up[i]
        if p >= 0:
            sees[i] |= sees[p]
    return sees


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
    k, v = (torch.cat([cache[at, x % page], new[lo:lo + n]]).double()
            for cache, new in ((c.k_cache, c.k), (c.v_cache, c.v)))
    seen = torch.cat([torch.ones((n, len(x)), dtype=torch.bool),
                      ancestors(n, None if c.parents is None else c.parents[b])], 1).cuda()
    q = c.q[lo:lo + n].double().view(n, Hkv, G, D)
    s = torch.einsum("nhgd,lhd->hgnl", q, k) * scale
    sizes = (torch.einsum("nhgd,lhd->hgnl", q.abs(), k.abs()) * scale).masked_fill(~seen, 0)
    es = sizes.amax(-1) * 2.0 ** -20
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
    flat = lambda y: y.permute(2, 0, 1).reshape(n, Hkv * G)  # noqa: E731
    return out, bound, flat(lse), flat(es) + 1e-5


def check(c, scale=None, requests=None, **kw):
    kw.setdefault("max_len", max(c.lens))
    kw.setdefault("max_nodes", max(1, max(c.nodes)))
    g = tt.tt_tree_attn(*c.args(), scale=scale, **kw)
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
    check(make(LENGTHS, nodes, 8, 2, D, page, dtype, seed=page))


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 1), (3, 3), (6, 2), (7, 1), (20, 4), (32, 8),
                                    (16, 1), (48, 1), (128, 1), (100, 1)])
@pytest.mark.parametrize("dtype", [H, E])
def test_heads(Hq, Hkv, dtype):
    check(make([300, 0, 77], [5, 9, 33], Hq, Hkv, 128, 32, dtype, seed=Hq))
    check(make([300, 0, 77], [1, 2, 3], Hq, Hkv, 64, 16, dtype, parents=None, seed=Hq + 1))


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 511, 512])
@pytest.mark.parametrize("parents", ["tree", "forest", None])
def test_nodes(n, parents):
    check(make([200, 0, 33], [n, 1, max(1, n // 2)], 4, 2, 64, 16, H, parents=parents, seed=n))
    check(make([129], [n], 5, 1, 128, 64, E, parents=parents, seed=n + 1))


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 1, 128), (9, 3, 64), (5, 1, 128), (32, 2, 64)])
@pytest.mark.parametrize("dtype", [H, E])
def test_several_row_tiles_over_long_caches(Hq, Hkv, D, dtype):
    """Rows of a key head beyond one tile: each tile of rows goes round its keys
    from a place of its own, and is cut at others."""
    check(make([20001, 9000, 131, 0, 4097], [100, 33, 130, 65, 1], Hq, Hkv, D, 48, dtype, seed=9))


@pytest.mark.parametrize("L", [3000, 8191, 20001, 70000])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 1, 128), (4, 2, 64), (32, 8, 128)])
def test_long_caches(L, Hq, Hkv, D):
    check(make([L, 5, L // 2 + 1], [9, 3, 17], Hq, Hkv, D, 64, H, seed=L))


def test_one_request_of_one_token():
    for L in (0, 1, 100, 1000, 5000):
        check(make([L], [1], 32, 8, 128, 16, H, seed=L, parents=None))


def test_ragged_batches_with_empty_requests():
    gen = torch.Generator().manual_seed(3)
    lens = torch.randint(0, 1500, (70,), generator=gen).tolist()
    nodes = torch.randint(0, 12, (70,), generator=gen).tolist()
    check(make(lens, nodes, 16, 4, 64, 32, H, seed=4))


@pytest.mark.parametrize("Hq,Hkv,D,n", [(8, 2, 128, 4), (16, 4, 64, 3), (32, 1, 64, 4)])
@pytest.mark.parametrize("dtype", [H, E])
def test_items_that_follow_each_other_within_caches(Hq, Hkv, D, n, dtype):
    """CTAs that end one item and begin another, which they leave before its drafted
    tokens: the two threads of a row add up the one's sum while the other's first
    scores come. The same bits each time."""
    gen = torch.Generator().manual_seed(31)
    lens = torch.randint(500, 3500, (150,), generator=gen).tolist()
    c = make(lens, [n] * 150, Hq, Hkv, D, 64, dtype, seed=32)
    first = check(c)
    for _ in range(30):
        g = tt.tt_tree_attn(*c.args(), max_len=max(lens), max_nodes=n)
        assert torch.equal(g["out"], first["out"]) and torch.equal(g["lse"], first["lse"])


@pytest.mark.parametrize("size", [0.05, 6.0])
def test_flat_and_sharp_softmax(size):
    for dtype in (H, E):
        check(make([2000, 100], [8, 3], 8, 2, 128, 32, dtype, seed=11, size=size))


def test_running_maximum_that_keeps_rising():
    """Scores that rise from tile to tile, fall, and jump at the end: what was
    summed before is scaled each time, or hardly counts."""
    for dtype in (H, E):
        for order in (1, -1):
            c = make([3000, 2000], [4, 2], 4, 1, 64, 64, dtype, seed=12)
            c.q[:] = c.q.abs() * 0.5
            ramp = torch.linspace(-3, 3, 3000, device="cuda").to(dtype)[::order] \
                if order == 1 else torch.linspace(3, -3, 3000, device="cuda").to(dtype)
            for b, L in enumerate(c.lens):
                x = torch.arange(L, device="cuda")
                c.k_cache[c.table[b].long()[x // 64], x % 64] = ramp[:L, None, None]
            check(c)


def test_masked_scores():
    """Keys whose score is -inf have no weight; a row whose every score is -inf
    has none at all: output 0, lse -inf."""
    c = make([40, 200], [2, 3], 2, 1, 64, 16, H, seed=13, parents=None)
    c.q[:, :, 0], c.k[:, :, 0] = 1.0, 0.0
    x = torch.arange(200, device="cuda")
    at = (c.table[1].long()[x // 16], x % 16)
    c.k_cache[at[0][::2], at[1][::2], :, 0] = -math.inf
    g = tt.tt_tree_attn(*c.args(), max_len=200, max_nodes=3)
    want = make([40, 100], [2, 3], 2, 1, 64, 16, H, seed=13, parents=None)
    want.q, want.k, want.v = c.q, c.k, c.v
    y = torch.arange(100, device="cuda")
    where = (want.table[1].long()[y // 16], y % 16)
    for a, o in ((c.k_cache, want.k_cache), (c.v_cache, want.v_cache)):
        o[where] = a[at[0][1::2], at[1][1::2]]
    out, bound, lse, el = expected(want, 1, 0.125)
    assert ((g["out"][2:].double() - out).abs() <= bound).all()
    assert ((g["lse"][2:].double() - lse).abs() <= el).all()
    c.k[:2, :, 0] = -math.inf
    x = torch.arange(40, device="cuda")
    c.k_cache[c.table[0].long()[x // 16], x % 16, :, 0] = -math.inf
    g = tt.tt_tree_attn(*c.args(), max_len=200, max_nodes=3)
    assert (g["out"][:2] == 0).all() and (g["lse"][:2] == -math.inf).all()
    assert ((g["out"][2:].double() - out).abs() <= bound).all()


def test_other_requests_do_not_matter():
    """NaN in one request's tokens, cache and query stays there."""
    c = make([100, 130, 90], [5, 6, 7], 4, 2, 64, 32, H, seed=14)
    c.q[5:11], c.k[5:11], c.v[5:11] = NAN, NAN, NAN
    c.k_cache[c.table[1].long()[:4]] = NAN
    c.v_cache[c.table[1].long()[:4]] = NAN
    g = check(c, requests=(0, 2))
    assert torch.isnan(g["out"][5:11]).all()


@pytest.mark.parametrize("dtype", [H, E])
def test_values_that_are_not_finite_stay_in_their_branch(dtype):
    """A drafted token with infinite and NaN keys and values reaches its own
    descendants and no other branch."""
    up = [-1, 0, 0, 1, 2, 4, 3, -1]
    c = make([150], [8], 4, 2, 64, 32, dtype, seed=30)
    c.parents = [up]
    clean = dataclasses.replace(c, k=c.k.clone(), v=c.v.clone())
    c.v[2, 0, 5], c.v[2, 1, 7], c.v[2, 1, 63] = math.inf, NAN, -math.inf
    c.k[6] = NAN  # (a leaf: itself only)
    g = tt.tt_tree_attn(*c.args(), max_len=150, max_nodes=8)
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


def test_strides():
    """Heads cut out of a fused projection, caches with the heads outermost,
    queries with gaps, a table with more pages than are used."""
    c = make([300, 70], [6, 9], 8, 2, 64, 32, H, seed=15)
    N = 15
    fused = torch.full((N, 8 + 2 + 2 + 3, 64), NAN, dtype=H, device="cuda")
    fused[:, :8], fused[:, 8:10], fused[:, 10:12] = c.q, c.k, c.v
    both = torch.full((c.k_cache.shape[0], 2, 2, 32, 64), NAN, dtype=H, device="cuda")
    both[:, 0] = c.k_cache.transpose(1, 2)
    both[:, 1] = c.v_cache.transpose(1, 2)
    table = torch.full((2, 40), -7, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    g = check(c)
    d = dataclasses.replace(c, q=fused[:, :8], k=fused[:, 8:10], v=fused[:, 10:12],
                            k_cache=both[:, 0].transpose(1, 2), v_cache=both[:, 1].transpose(1, 2),
                            table=table)
    h = check(d)
    assert torch.equal(g["out"], h["out"]) and torch.equal(g["lse"], h["lse"])
    wide = torch.full((N, 8, 192), NAN, dtype=H, device="cuda")[:, :, 64:128]
    wide.copy_(c.q)
    assert torch.equal(check(dataclasses.replace(d, q=wide))["out"], g["out"])


def test_keys_and_values_laid_out_differently():
    """Slots outermost in one cache, heads in the other."""
    c = make([300, 70], [6, 9], 8, 2, 64, 32, E, seed=18)
    g = check(c)
    for name in ("k_cache", "v_cache"):
        turned = getattr(c, name).transpose(1, 2).contiguous().transpose(1, 2)
        h = check(dataclasses.replace(c, **{name: turned}))
        assert torch.equal(g["out"], h["out"]) and torch.equal(g["lse"], h["lse"])


def test_offsets_beyond_32_bits():
    """Pages that start billions of bytes apart."""
    c = make([60, 40], [3, 2], 4, 2, 128, 32, H, seed=19, extra=0)
    g = check(c)
    pages, far = c.k_cache.shape[0], {}
    for name in ("k_cache", "v_cache"):
        step = 2 ** 30 + 64
        buf = torch.empty(pages * step, dtype=H, device="cuda")
        far[name] = buf.as_strided(c.k_cache.shape, (step, 256, 128, 1))
        far[name].copy_(getattr(c, name))
    h = check(dataclasses.replace(c, **far))
    assert torch.equal(g["out"], h["out"]) and torch.equal(g["lse"], h["lse"])


def test_bounds_above_what_is_there():
    """max_len and max_nodes may be larger than any request's."""
    c = make([300, 0, 70], [6, 1, 9], 8, 2, 128, 32, H, seed=16)
    table = torch.zeros((3, 500), dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    c.table = table
    check(c, max_len=16000, max_nodes=512)
    check(c, max_len=300, max_nodes=9, scale=0.3)
    g = tt.tt_tree_attn(*c.args())
    assert g["status"].tolist() == [0, 0, 0]


def test_a_cache_of_more_than_2_31_elements():
    """The used pages lie at both ends of caches of 2.2e9 elements each."""
    D, Hkv, page = 128, 8, 128
    pages = 2_200_000_000 // (D * Hkv * page)
    lens, nodes = [1000, 300], [4, 9]
    small = make(lens, nodes, 16, Hkv, D, page, H, seed=17, extra=0)
    kc = torch.empty((pages, page, Hkv, D), dtype=H, device="cuda")
    vc = torch.empty((pages, page, Hkv, D), dtype=H, device="cuda")
    n = small.k_cache.shape[0]
    at = torch.tensor([p if p % 2 else pages - 1 - p for p in range(n)], device="cuda")
    kc[at], vc[at] = small.k_cache, small.v_cache
    big = dataclasses.replace(small, k_cache=kc, v_cache=vc, table=at[small.table.long()].int())
    assert torch.equal(check(big)["out"], check(small)["out"])


def test_statuses():
    c = make([100, 200, 50, 60, 30], [3, 4, 5, 6, 2], 4, 2, 64, 16, H, seed=18)
    args = list(c.args())
    full = check(c)
    # too long a cache, a negative length; their outputs stay as they were
    args[6] = torch.tensor([100, 201, 50, -1, 30], dtype=torch.int32, device="cuda")
    out = dict(out=torch.full((20, 4, 64), 7.0, dtype=H, device="cuda"))
    g = tt.tt_tree_attn(*args, max_len=200, max_nodes=6, out=dict(out))
    assert g["status"].tolist() == [0, 2, 0, 2, 0]
    for lo, hi in ((0, 3), (7, 12), (18, 20)):
        assert torch.equal(g["out"][lo:hi], full["out"][lo:hi])
    assert (g["out"][3:7] == 7).all() and (g["out"][12:18] == 7).all()
    # more nodes than max_nodes
    args = list(c.args())
    g = tt.tt_tree_attn(*args, max_len=200, max_nodes=5, out=dict(out))
    assert g["status"].tolist() == [0, 0, 0, 2, 0]
    # offsets that fall or leave the nodes (no two requests share nodes)
    args[7] = torch.tensor([0, 3, 7, 2, 2, 21], dtype=torch.int32, device="cuda")
    g = tt.tt_tree_attn(*args, max_len=200, max_nodes=20)
    assert g["status"].tolist() == [0, 0, 8, 0, 8]
    assert torch.equal(g["out"][:7], full["out"][:7])
    # pages out of range are left out, parents out of range make roots
    args = list(c.args())
    table = c.table.clone()
    table[1, 2], table[1, 5] = -1, c.k_cache.shape[0]
    up = args[8].clone()
    up[7 + 3], up[12 + 1] = 3, -2
    args[5], args[8] = table, up
    g = tt.tt_tree_attn(*args, max_len=200, max_nodes=6)
    assert g["status"].tolist() == [0, 1, 1, 1, 0]
    outp, bound, _, _ = expected(c, 1, 0.125, skip_pages=(2, 5))
    assert ((g["out"][3:7].double() - outp).abs() <= bound).all()
    c.parents[2][3] = -1
    outp, bound, _, _ = expected(c, 2, 0.125)
    assert ((g["out"][7:12].double() - outp).abs() <= bound).all()


def test_outputs_streams_and_repeats():
    c = make([3000, 10], [8, 2], 8, 2, 128, 16, H, seed=19)
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
    d = make([10, 2500], [3, 7], 8, 2, 128, 16, H, seed=20)
    d.table = torch.cat([d.table, torch.zeros_like(d.table[:, :40])], 1)  # (room for 3000)
    a = tt.tt_tree_attn(*c.args(), max_len=3000, max_nodes=8, ws=ws)
    b = tt.tt_tree_attn(*d.args(), max_len=3000, max_nodes=8, ws=ws)
    assert torch.equal(a["out"], h["out"])
    assert torch.equal(b["out"], check(d, max_len=3000)["out"])


def test_captured_in_a_graph():
    c = make([3000, 700], [8, 2], 8, 2, 128, 16, H, seed=21)
    args = c.args()
    kw = dict(max_len=3000, max_nodes=8)
    tt.tt_tree_attn(*args, **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g = tt.tt_tree_attn(*args, **kw)
    c.q.neg_()
    args[6].copy_(torch.tensor([100, 690]))
    graph.replay()
    torch.cuda.synchronize()
    c.lens = [100, 690]
    h = check(c, max_len=3000)
    assert torch.equal(g["out"], h["out"])


def test_no_requests_and_no_nodes():
    c = make([5], [1], 4, 2, 64, 16, H)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    g = tt.tt_tree_attn(c.q[:0], c.k[:0], c.v[:0], c.k_cache, c.v_cache, c.table, i32([5]),
                        i32([0, 0]))
    assert g["out"].shape == (0, 4, 64) and g["status"].tolist() == [0]
    g = tt.tt_tree_attn(c.q[:0], c.k[:0], c.v[:0], c.k_cache, c.v_cache, c.table[:0], i32([]),
                        i32([0]))
    assert g["out"].shape == (0, 4, 64)


def test_refusals():
    c = make([50], [3], 4, 2, 64, 16, H)
    a = list(c.args())

    def refuse(error, at=None, to=None, **kw):
        b = list(a)
        if at is not None:
            b[at] = to
        with pytest.raises(error) as e:
            tt.tt_tree_attn(*b, **kw)
        return e.value

    for kw in (dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(max_nodes=0),
               dict(max_nodes=513), dict(max_len=-1)):
        assert refuse(tt.TTError, **kw).code == binding.TT_ERR_INVALID_ARG
    refuse(ValueError, max_len=65)
    refuse(TypeError, 0, c.q.float())
    refuse(ValueError, 1, c.k.to(E))
    refuse(ValueError, 1, c.k[:2])
    refuse(ValueError, 3, c.k_cache[:, :, :1])
    refuse(ValueError, 5, c.table.long())
    refuse(ValueError, 6, a[6].long())
    refuse(ValueError, 7, a[7][:1])
    refuse(ValueError, 8, a[8][:2])
    refuse(ValueError, ws=None, out=dict(out=torch.zeros((3, 4, 63), dtype=H, device="cuda")))
    refuse(tt.TTError, 0, c.q[:, :3])  # 3 query heads on 2
    for D in (32, 96, 256):
        d = make([50], [3], 4, 2, D, 16, H)
        with pytest.raises(tt.TTError):
            tt.tt_tree_attn(*d.args())
    d = make([50], [3], 4, 2, 64, 24, H)  # pages of 24 slots
    with pytest.raises(tt.TTError):
        tt.tt_tree_attn(*d.args())
    odd = torch.zeros((3, 4, 65), dtype=H, device="cuda")[:, :, 1:]  # not on 16 bytes
    refuse(tt.TTError, 0, odd)
    big = make([50], [3], 129, 1, 64, 16, H)
    with pytest.raises(tt.TTError):
        tt.tt_tree_attn(*big.args())
    T = binding._tree(*a, None, None, None)
    P = ctypes.byref
    lib, p = tt.load(), ctypes.c_void_p(256)
    assert lib.tt_tree_attn(P(T), p, 1 << 40, p, None, None, None) == binding.TT_ERR_INVALID_ARG
    T.dtype = binding.TT_F32
    assert lib.tt_tree_attn(P(T), p, 1 << 40, p, None, p, None) == binding.TT_ERR_INVALID_ARG
