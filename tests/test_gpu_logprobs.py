"""tt_logprobs against the definition in 64 bits: widths around every vector,
batch and split boundary, both types, ties, masks that leave few columns or
none, rows that are not finite, and the refusals.

Tolerances. A term of the normaliser has the relative error of its exponent
(|d| 2^-24 with |d| <= 40 where it counts), of the exponential (2^-22) and of
the sum (under 2^-20 for the sums' lengths here), together under 5e-6; log S
has that as absolute error, the entropy that of its two sums. A log probability
adds two roundings of its own size (2^-23)."""
import ctypes
import math

import pytest
import torch

import paper_2510_15545_gb300 as tt
from paper_2510_15545_gb300 import binding

pytestmark = pytest.mark.gpu

ABS, REL = 1e-5, 2.0 ** -22


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    tt.load(build_if_missing=True)


def rows_of(z, dtype, pad=0):
    """z on the GPU, its rows apart by a multiple of 16 bytes, NaN between them."""
    R, V = z.shape
    buf = torch.full((R, (V + 7) // 8 * 8 + pad), float("nan"), dtype=dtype, device="cuda")
    buf[:, :V] = z.cuda().to(dtype)
    return buf[:, :V]


def expected(rows, ids, temp, n):
    z = rows.cpu().double()
    R, V = z.shape
    top = z.amax(1)
    bad = ~torch.isfinite(top)
    s = (z - top[:, None]) / temp
    e = torch.exp(s)
    S = e.sum(1)
    t = ids.long().cpu().clamp(0, V - 1)
    zt = z.gather(1, t[:, None])
    col = torch.arange(V)
    rank = ((z > zt) | ((z == zt) & (col < t[:, None]))).sum(1)
    v, i = torch.sort(z, dim=1, descending=True, stable=True)
    pad = max(0, n - V)
    v = torch.nn.functional.pad(v, (0, pad), value=-math.inf)[:, :n]
    i = torch.nn.functional.pad(i, (0, pad), value=-1)[:, :n]
    gone = bad[:, None] | (v == -math.inf)
    none, off = ids.cpu() == -1, (ids.cpu() < -1) | (ids.cpu() >= V)
    logprob = (zt[:, 0] - top) / temp - torch.log(S)
    logprob[none] = 0.0
    logprob[off | bad] = math.nan
    rank[none | off | bad] = -1
    return dict(
        lse=torch.where(bad, math.nan, top / temp + torch.log(S)),
        entropy=torch.where(bad, math.nan,
                            torch.log(S) - torch.where(e > 0, e * s, 0.0).sum(1) / S),
        logprob=logprob, rank=rank, top_ids=torch.where(gone, -1, i),
        top_logprobs=torch.where(bad[:, None], math.nan,
                                 (v - top[:, None]) / temp - torch.log(S)[:, None]),
        status=bad * binding.TT_REQ_NOT_FINITE + off * binding.TT_REQ_ID_OUT_OF_RANGE)


def check(rows, ids, temp=1.0, n=20, **kw):
    g = tt.tt_logprobs(rows, ids, temp=temp, top_n=n, **kw)
    torch.cuda.synchronize()
    o = expected(rows, ids, temp, n)
    for key, want in o.items():
        got = g[key].cpu()
        if key in ("rank", "top_ids", "status"):
            assert torch.equal(got.long(), want.long()), key
        else:
            torch.testing.assert_close(got.double(), want, rtol=REL, atol=ABS, equal_nan=True,
                                       msg=lambda m: "%s: %s" % (key, m))
    return g


F, H = torch.float32, torch.bfloat16
WIDTHS = [1, 2, 7, 8, 9, 31, 255, 1023, 1025, 2048, 2049, 4096, 4100, 8191, 16385, 50257, 65537]


def random_ids(R, V, gen):
    ids = torch.randint(V, (R,), generator=gen)
    ids[::5] = -1
    return ids.int().cuda()


@pytest.mark.parametrize("V", WIDTHS)
@pytest.mark.parametrize("dtype", [F, H])
def test_widths(V, dtype):
    gen = torch.Generator().manual_seed(V)
    z = torch.randn((5, V), generator=gen) * 4
    for n, temp, pad in ((20, 1.0, 0), (32, 0.6, 8), (1, 2.0, 64), (0, 1.0, 0)):
        check(rows_of(z, dtype, pad), random_ids(5, V, gen), temp, n)


@pytest.mark.parametrize("R", [1, 2, 3, 10, 37, 75, 150, 151, 310, 700, 2000])
@pytest.mark.parametrize("dtype", [F, H])
def test_row_counts(R, dtype):
    gen = torch.Generator().manual_seed(R)
    V = 40001 if R < 100 else 9001
    check(rows_of(torch.randn((R, V), generator=gen) * 3, dtype), random_ids(R, V, gen), n=12)


@pytest.mark.parametrize("V", [201088, 1000003])
def test_wide_rows(V):
    gen = torch.Generator().manual_seed(3)
    z = torch.randn((2, V), generator=gen) * 3
    for dtype in (F, H):
        check(rows_of(z, dtype), random_ids(2, V, gen), 0.7, 20)


@pytest.mark.parametrize("V", [300, 4096, 30011, 70001])
@pytest.mark.parametrize("dtype", [F, H])
def test_ties(V, dtype):
    """Coarse logits, constant rows, and -0 beside 0: smaller columns first."""
    gen = torch.Generator().manual_seed(V)
    z = torch.randint(-3, 4, (6, V), generator=gen).float()
    z[1] = 2.5
    z[2] = 0.0
    z[2, ::3] = -0.0
    z[3] = -1.0
    z[3, V // 2:] = 0.0
    z[4] = torch.arange(V).float() // 64  # rising: every batch beats the ones before
    z[5] = -torch.arange(V).float() // 7
    check(rows_of(z, dtype), random_ids(6, V, gen), n=32)
    check(rows_of(z, dtype), random_ids(6, V, gen), n=7)


@pytest.mark.parametrize("V", [9, 5000, 66000])
@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("low", [-math.inf, "lowest"])
def test_masks(V, dtype, low):
    """Masks that leave every column, some, one and (with -inf) none; all columns
    at the type's lowest value are a uniform row."""
    low = torch.finfo(dtype).min if low == "lowest" else low
    gen = torch.Generator().manual_seed(V)
    z = torch.randn((7, V), generator=gen) * 3
    z[1, torch.rand(V, generator=gen) < 0.9] = low
    z[2, 5:] = low
    z[3, :-3] = low
    z[4] = low
    z[4, V // 2] = 1.0
    z[5] = low
    z[6, ::2] = low
    ids = torch.tensor([V - 1, 0, 1, V - 1, V // 2, 3, 2]).int().cuda()
    check(rows_of(z, dtype), ids, 1.0, 20)
    # (below 1 the lowest value over the temperature leaves the type's range)
    g = tt.tt_logprobs(rows_of(z, dtype), ids, temp=0.6, top_n=20)
    o = expected(rows_of(z, dtype), ids, 0.6, 20)
    assert torch.equal(g["top_ids"].cpu().long(), o["top_ids"])
    torch.testing.assert_close(g["lse"].cpu().double()[:5], o["lse"][:5], rtol=REL, atol=ABS)


@pytest.mark.parametrize("V", [1, 9, 1025, 8200, 20011])
@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("n", [1, 32])
def test_rows_beyond_the_machine(V, dtype, n):
    """More rows than are computed at once, every kind among them: ordinary ones,
    masked ones, empty ones, ties beyond every list, single columns, NaN."""
    gen = torch.Generator().manual_seed(V + n)
    R = 1300
    z = torch.randn((R, V), generator=gen) * 3
    kind = torch.arange(R) % 7
    z[kind == 1] = torch.where(torch.rand((R, V), generator=gen) < 0.9, -math.inf, z)[kind == 1]
    z[kind == 2] = -math.inf
    z[kind == 3] = 0.5
    z[kind == 4] = (torch.arange(V) // 64).float()
    z[kind == 5] = -math.inf
    z[kind == 5, V // 2] = -2.0
    z[5::70, V // 3] = math.nan  # (beside a single column)
    check(rows_of(z, dtype), random_ids(R, V, gen), n=n)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("V", [3000, 70001])
@pytest.mark.parametrize("lead", [8.0, 14.0, 20.0, 40.0])
def test_rows_that_one_column_dominates(dtype, V, lead):
    """The log probability of a column that holds nearly all of the mass is the
    rest's, relative to its size: the terms' 2^-22 and |d| 2^-23, and the sums'
    (1e-6); its entropy alike."""
    gen = torch.Generator().manual_seed(V)
    z = torch.randn((6, V), generator=gen)
    at = torch.randint(V, (6,), generator=gen)
    at[0], at[1] = 0, V - 1
    z[torch.arange(6), at] = lead + math.log(V)
    z[5, 10:20] = z[5, at[5]]  # (and one with equals)
    rows, ids = rows_of(z, dtype), at.int().cuda()
    g, o = tt.tt_logprobs(rows, ids, top_n=2), expected(rows, ids, 1.0, 2)
    zd = rows.cpu().double()
    for r in range(5):
        rest = torch.exp(zd[r] - zd[r, at[r]])
        rest[at[r]] = 0.0
        want = -torch.log1p(rest.sum())
        assert abs(g["logprob"][r].item() - want) <= 1e-5 * abs(want), r
        assert g["top_logprobs"][r, 0].item() == g["logprob"][r].item()
        h = -want + (rest * (zd[r, at[r]] - zd[r])).sum() / (1 + rest.sum())
        assert abs(g["entropy"][r].item() - h) <= 1e-5 * h, r
    torch.testing.assert_close(g["logprob"].cpu().double(), o["logprob"], rtol=REL, atol=ABS)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("temp", [1e-30, 1e-4, 0.01, 100.0, 1e30])
@pytest.mark.parametrize("size", [1e-3, 1.0, 1e4, 1e30])
def test_temperatures_and_sizes(dtype, temp, size):
    """Far temperatures and logits, with and without masked columns. (The
    entropy's terms have the rounding of d, 2^-23 |d|, where |d| < 100.)"""
    gen = torch.Generator().manual_seed(21)
    V = 9000
    z = torch.randn((4, V), generator=gen) * size
    z[1, torch.rand(V, generator=gen) < 0.5] = -math.inf
    z[2] -= 50 * size
    z[3, ::2] = torch.finfo(dtype).min
    rows = rows_of(z, dtype)
    ids = rows.float().argmax(1).int()
    g = tt.tt_logprobs(rows, ids, temp=temp, top_n=4)
    o = expected(rows, ids, temp, 4)
    assert g["status"].tolist() == [0] * 4
    assert torch.equal(g["top_ids"].cpu().long(), o["top_ids"])
    torch.testing.assert_close(g["logprob"].cpu().double(), o["logprob"], rtol=REL, atol=ABS)
    torch.testing.assert_close(g["entropy"].cpu().double(), o["entropy"], rtol=1e-5, atol=2e-5)


@pytest.mark.parametrize("V", [40, 5000, 70001])
@pytest.mark.parametrize("dtype", [F, H])
def test_rows_that_are_not_finite(V, dtype):
    gen = torch.Generator().manual_seed(V)
    z = torch.randn((6, V), generator=gen)
    z[0, V // 3] = math.nan
    z[1, V - 1] = math.inf
    z[2] = -math.inf
    z[4] = math.nan
    rows = rows_of(z, dtype)
    ids = torch.tensor([V // 3, 0, 1, 2, 3, 4]).int().cuda()
    g = tt.tt_logprobs(rows, ids, top_n=4)
    bad = [0, 1, 2, 4]
    assert g["status"].tolist() == [16, 16, 16, 0, 16, 0]
    for key in ("lse", "entropy", "logprob", "top_logprobs"):
        assert torch.isnan(g[key][bad]).all(), key
    assert (g["rank"][bad] == -1).all() and (g["top_ids"][bad] == -1).all()
    check(rows_of(z[[3, 5]], dtype), ids[[3, 5]], n=4)


def test_rows_billions_of_bytes_apart():
    gen = torch.Generator().manual_seed(8)
    step = 2 ** 29 + 8
    rows = torch.empty(9 * step, device="cuda").as_strided((9, 3001), (step, 1))
    rows.copy_(torch.randn((9, 3001), generator=gen))
    check(rows, random_ids(9, 3001, gen), n=9)


def test_ids_out_of_range():
    gen = torch.Generator().manual_seed(1)
    rows = rows_of(torch.randn((5, 1000), generator=gen), F)
    ids = torch.tensor([1000, -2, -1, 999, 2 ** 31 - 1]).int().cuda()
    check(rows, ids, n=3)


def test_outputs_in_place_and_streams():
    gen = torch.Generator().manual_seed(2)
    rows = rows_of(torch.randn((9, 4000), generator=gen), H)
    ids = random_ids(9, 4000, gen)
    out = {k: torch.zeros(9, dtype=torch.int32 if k in ("rank", "status") else F, device="cuda")
           for k in ("logprob", "rank", "entropy", "lse", "status")}
    out["top_ids"] = torch.zeros((9, 5), dtype=torch.int32, device="cuda")
    out["top_logprobs"] = torch.zeros((9, 5), device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = check(rows, ids, 1.0, 5, out=out, stream=side)
    assert all(g[k] is out[k] for k in out)
    # the same call twice gives the same bits
    h = tt.tt_logprobs(rows, ids, top_n=5)
    for k in out:
        assert torch.equal(h[k].reshape(-1), g[k].reshape(-1)), k


def test_captured_in_a_graph():
    gen = torch.Generator().manual_seed(4)
    rows = rows_of(torch.randn((3, 20000), generator=gen), F)
    ids = random_ids(3, 20000, gen)
    tt.tt_logprobs(rows, ids, top_n=5)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g = tt.tt_logprobs(rows, ids, top_n=5)
    rows.copy_(torch.randn((3, 20000), generator=gen))
    graph.replay()
    torch.cuda.synchronize()
    o = expected(rows, ids, 1.0, 5)
    assert torch.equal(g["top_ids"].cpu().long(), o["top_ids"])
    torch.testing.assert_close(g["lse"].cpu().double(), o["lse"], rtol=REL, atol=ABS)


def test_no_rows():
    g = tt.tt_logprobs(torch.zeros((0, 64), device="cuda"), top_n=3)
    assert g["top_ids"].shape == (0, 3)


def test_refusals():
    rows = rows_of(torch.zeros((2, 64)), F)
    ids = torch.zeros(2, dtype=torch.int32, device="cuda")
    for kw in (dict(temp=0.0), dict(temp=-1.0), dict(temp=math.nan), dict(temp=math.inf),
               dict(top_n=33)):
        with pytest.raises(tt.TTError) as e:
            tt.tt_logprobs(rows, ids, **kw)
        assert e.value.code == binding.TT_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        tt.tt_logprobs(rows, ids.long())
    with pytest.raises(ValueError):
        tt.tt_logprobs(rows, ids[:1])
    with pytest.raises(TypeError):
        tt.tt_logprobs(rows.half(), ids)
    with pytest.raises(tt.TTError):  # rows that do not start on 16 bytes
        tt.tt_logprobs(torch.zeros((2, 65), device="cuda")[:, 1:], ids)
    lib, out = tt.load(), binding._LogprobsOut(status=256, logprob=256)
    L = binding._logits(rows)
    assert lib.tt_logprobs(ctypes.byref(L), None, 1.0, 0, ctypes.byref(out), None) \
        == binding.TT_ERR_INVALID_ARG  # a log probability of no column
    out = binding._LogprobsOut(lse=256)
    assert lib.tt_logprobs(ctypes.byref(L), None, 1.0, 0, ctypes.byref(out), None) \
        == binding.TT_ERR_INVALID_ARG  # no status
