"""tt_distill and tt_distill_grad against the definition in 64 bits, whose own
gradient is checked against differences: widths around every vector, share and
part, both types, lists with unused, repeated and unusable entries, masked and
empty rows, weights, and the refusals.

Tolerances. A log probability of the student has the error of the normaliser
(1e-5, as for tt_logprobs) and 2^-22 of its size; the loss is a mean of such
terms over a mass of 1. The mass outside the list, 1 - P, has the rounding of
P's exponentials (1e-6). A gradient is w / T times q (W - r / t) or W q - p: the
exponentials' and sums' relative 1e-5 of each term, and the error of r; bf16
gradients are rounded once (2^-8 of the value at most)."""
import ctypes
import math

import pytest
import torch

import paper_2510_15545_gb300 as tt
from paper_2510_15545_gb300 import binding

pytestmark = pytest.mark.gpu

F, H = torch.float32, torch.bfloat16


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


def teacher(R, V, K, gen, unused=0.2, mass=0.9):
    """Lists of distinct columns whose probabilities sum to about `mass`."""
    ids = torch.stack([torch.randperm(V, generator=gen)[:K] for _ in range(R)])
    logp = torch.log_softmax(torch.randn((R, K), generator=gen) * 2, 1) + math.log(mass)
    ids[torch.rand((R, K), generator=gen) < unused] = -1
    return ids.int(), logp


def loss_of(z, ids, logp, temp, tail):
    """The loss of one row in 64 bits; ids distinct and usable."""
    logq = torch.log_softmax(z / temp, 0)
    lp = logp if tail else torch.log_softmax(logp, 0)
    p = torch.exp(lp)
    loss = (p * (lp - logq[ids])).sum()
    if tail:
        r = (1 - p.sum()).clamp(min=0)
        out = torch.ones_like(z, dtype=torch.bool)
        out[ids] = False
        if r > 0:
            loss = loss + r * (torch.log(r) - torch.logsumexp(logq[out], 0))
    return loss


def expected(rows, ids, logp, temp, tail, weight):
    """Loss [R], gradient [R, V], the gradient's error bound [R, V] in 64 bits."""
    z, logp, ids = rows.cpu().double(), logp.cpu().double(), ids.cpu().long()
    R, V = z.shape
    loss, grad, bound = torch.zeros(R).double(), torch.zeros_like(z), torch.zeros_like(z)
    for r in range(R):
        use = (ids[r] >= 0) & (logp[r] > -math.inf)
        if not use.any():
            continue
        # entries of one column add up
        lp = logp[r][use] if tail else torch.log_softmax(logp[r][use], 0)
        col, at = torch.unique(ids[r][use], return_inverse=True)
        p = torch.zeros(len(col)).double().scatter_add_(0, at, torch.exp(lp))
        loss[r] = loss_of(z[r], col, torch.log(p), temp, tail)
        q = torch.softmax(z[r] / temp, 0)
        rest = (1 - p.sum()).clamp(min=0) if tail else torch.zeros(()).double()
        out = torch.ones(V, dtype=torch.bool)
        out[col] = False
        t = q[out].sum()
        W = p.sum() + rest
        ratio = rest / t if t > 0 else torch.zeros(()).double()
        g = q * (W - ratio) if t > 0 else torch.zeros_like(q)
        b = q * (1e-5 * (W + ratio) + (1e-6 / t if tail and t > 0 else 0))
        g[col] = W * q[col] - p
        b[col] = 1e-5 * (W * q[col] + p)
        w = (1.0 if weight is None else weight[r].item()) / temp
        grad[r], bound[r] = w * g, abs(w) * b
    return loss, grad, bound


def check_grad(got, want, bound, dtype):
    got = got.cpu().double()
    assert torch.isfinite(got).all()
    bound = bound + want.abs() * (2.0 ** -8 if dtype == H else 0) + 1e-37
    worst = ((got - want).abs() / bound).max()
    assert worst <= 1, worst


def check(z, ids, logp, dtype, temp=1.0, tail=False, weight=None, pad=0):
    rows = rows_of(z, dtype, pad)
    ids_d, logp_d = ids.cuda(), logp.float().cuda()
    w = None if weight is None else weight.cuda()
    loss, grad, bound = expected(rows, ids_d, logp_d, temp, tail, weight)
    g = tt.tt_distill(rows, ids_d, logp_d, temp=temp, tail=tail, weight=w)
    torch.testing.assert_close(g["loss"].cpu().double(), loss, rtol=1e-5, atol=2e-5)
    check_grad(g["grad"], grad, bound, dtype)
    # as two calls, after either form of the first
    h = tt.tt_distill(rows, ids_d, logp_d, temp=temp, tail=tail, grad=False)
    assert "grad" not in h
    torch.testing.assert_close(h["loss"].cpu().double(), loss, rtol=1e-5, atol=2e-5)
    for first in (g, h):
        back = tt.tt_distill_grad(rows, ids_d, logp_d, first["stats"], temp=temp, tail=tail, weight=w)
        check_grad(back, grad, bound, dtype)
    return g


@pytest.mark.parametrize("V", [2, 7, 8, 9, 255, 2047, 2049, 4100, 16385, 65543])
@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("tail", [False, True])
def test_widths(V, dtype, tail):
    gen = torch.Generator().manual_seed(V)
    K = min(20, max(1, V // 2))
    ids, logp = teacher(4, V, K, gen)
    z = torch.randn((4, V), generator=gen) * 3
    check(z, ids, logp, dtype, 1.0, tail)
    w = torch.tensor([1.0, 0.0, -0.5, 3.0])
    check(z, ids, logp, dtype, 2.0, tail, w, pad=16)


@pytest.mark.parametrize("R,V", [(1, 1000), (2, 50257), (5, 128256), (33, 20000), (400, 5003)])
@pytest.mark.parametrize("dtype", [F, H])
def test_row_counts(R, V, dtype):
    gen = torch.Generator().manual_seed(R)
    ids, logp = teacher(R, V, 12, gen)
    check(torch.randn((R, V), generator=gen) * 3, ids, logp, dtype, 0.7, True,
          torch.rand(R, generator=gen))


@pytest.mark.parametrize("V", [201088, 700001])
@pytest.mark.parametrize("dtype", [F, H])
def test_wide_rows(V, dtype):
    gen = torch.Generator().manual_seed(V)
    ids, logp = teacher(2, V, 64, gen)
    ids[0, :2] = torch.tensor([0, V - 1]).int()
    check(torch.randn((2, V), generator=gen) * 3, ids, logp, dtype, 1.0, True)


@pytest.mark.parametrize("K", [1, 2, 31, 33, 127, 128])
@pytest.mark.parametrize("tail", [False, True])
def test_list_lengths(K, tail):
    gen = torch.Generator().manual_seed(K)
    ids, logp = teacher(3, 3000, K, gen, unused=0.0)
    check(torch.randn((3, 3000), generator=gen), ids, logp, F, 1.0, tail)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", [F, H])
def test_lists_as_they_come(tail, dtype):
    """Repeated columns, unused entries in between, entries of probability 0,
    lists that hold the whole row, all of the mass, or more than it by rounding."""
    gen = torch.Generator().manual_seed(5)
    V = 24
    ids, logp = teacher(6, V, V, gen, unused=0.0)
    ids[0, 3] = ids[0, 9]
    ids[0, 11] = ids[0, 9]
    ids[1, ::2] = -1
    logp[2, 4:] = -math.inf
    logp[3] = torch.log_softmax(logp[3], 0) + 3e-8  # the whole mass on the whole row
    ids[4, 1:] = -1
    ids[5, 5:] = -1
    logp[5, :5] = torch.log_softmax(logp[5, :5], 0)
    z = torch.randn((6, V), generator=gen)
    if tail:  # (a teacher with mass outside a list that holds the whole row has loss inf)
        for r in (0, 2):
            logp[r] = torch.log_softmax(logp[r], 0) + 1e-6
    check(z, ids, logp, dtype, 1.0, tail)


@pytest.mark.parametrize("dtype", [F, H])
def test_a_student_that_knows_its_teacher(dtype):
    """All but 1e-6 of the student's mass is on the list: the mass outside it is
    what 1 - Q could not give."""
    gen = torch.Generator().manual_seed(6)
    V = 5000
    z = torch.randn((3, V), generator=gen)
    ids, logp = teacher(3, V, 8, gen, unused=0.0, mass=1 - 1e-4)
    z.scatter_(1, ids.long(), z.gather(1, ids.long()) + 22.0)
    check(z, ids, logp, dtype, 1.0, True)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("lead", [60.0, 150.0, 1000.0])
def test_a_student_sure_beyond_fp32(dtype, lead):
    """The mass outside the list is below what fp32 holds; its logarithm and its
    shares of the teacher's rest are not."""
    gen = torch.Generator().manual_seed(16)
    V = 5000
    z = torch.randn((3, V), generator=gen)
    ids, logp = teacher(3, V, 8, gen, unused=0.0, mass=0.9)
    z.scatter_(1, ids.long(), z.gather(1, ids.long()) + lead)
    rows = rows_of(z, dtype)
    loss, grad, bound = expected(rows, ids, logp, 1.0, True, None)
    out = torch.ones((3, V), dtype=torch.bool).scatter_(1, ids.long(), False)
    # (t in 64 bits is 0 from a lead of 745 on: the shares of r outside the list, directly)
    zo = rows.cpu().double().masked_fill(~out, -math.inf)
    rest = 1 - torch.exp(logp.double()).sum(1, keepdim=True)
    q = torch.softmax(rows.cpu().double(), 1)
    want = torch.where(out, q - rest * torch.softmax(zo, 1), grad)
    bound = torch.where(out, 1e-5 * (q + want.abs()), bound)
    for g in (True, False):
        o = tt.tt_distill(rows, ids.cuda(), logp.cuda(), tail=True, grad=g)
        torch.testing.assert_close(o["loss"].cpu().double(), loss, rtol=1e-5, atol=2e-5)
        back = tt.tt_distill_grad(rows, ids.cuda(), logp.cuda(), o["stats"], tail=True)
        check_grad(back, want, bound, dtype)
    check_grad(tt.tt_distill(rows, ids.cuda(), logp.cuda(), tail=True)["grad"], want, bound, dtype)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("level", [-500.0, 500.0])
def test_columns_masked_in_a_run(dtype, level):
    """Every column but the first few hundred masked, at a level far from 0: what
    shares of a row hold nothing say nothing about its maximum."""
    gen = torch.Generator().manual_seed(17)
    V = 90000
    z = torch.full((2, V), -math.inf)
    z[:, :700] = torch.randn((2, 700), generator=gen) + level
    ids, logp = teacher(2, 700, 6, gen, unused=0.0)
    for tail in (False, True):
        check(z, ids, logp, dtype, 1.0, tail)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("low", [-math.inf, "lowest"])
@pytest.mark.parametrize("tail", [False, True])
def test_masked_students(dtype, low, tail):
    low = torch.finfo(dtype).min if low == "lowest" else low
    gen = torch.Generator().manual_seed(7)
    V = 6000
    ids, logp = teacher(3, V, 9, gen, unused=0.0)
    z = torch.randn((3, V), generator=gen)
    keep = torch.rand((3, V), generator=gen) < 0.1
    keep.scatter_(1, ids.long(), True)
    z[~keep] = low
    check(z, ids, logp, dtype, 1.0, tail)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("low", [-math.inf, "lowest"])
@pytest.mark.parametrize("V,R,left", [(3000, 300, 1), (3000, 300, 3), (3000, 300, 20), (70001, 40, 9)])
def test_lists_that_hold_the_whole_mass(dtype, low, V, R, left):
    """A mask leaves fewer columns than the teacher lists, and the student is masked
    alike: nothing is outside the list on either side, and what 1 - P says is
    rounding. (A list's log probabilities are off by 1e-5 at most, so p by that
    relative amount and the loss by that much of sum p (1 + |ln p - ln q|).)"""
    gen = torch.Generator().manual_seed(V + left)
    keep = torch.zeros((R, V), dtype=torch.bool)
    keep.scatter_(1, torch.stack([torch.randperm(V, generator=gen)[:left] for _ in range(R)]), True)
    low = torch.finfo(dtype).min if low == "lowest" else low
    target, student = (rows_of((torch.randn((R, V), generator=gen) * 3).masked_fill(~keep, low), dtype)
                       for _ in range(2))
    for temp in (0.6, 1.0):
        o = tt.tt_logprobs(target, temp=temp, top_n=32)
        logp = torch.log_softmax((target.cpu().double() / temp).masked_fill(~keep, -math.inf), 1)
        logq = torch.log_softmax(student.cpu().double().masked_fill(~keep, -math.inf), 1)
        p, q = torch.exp(logp), torch.exp(logq)
        apart = torch.where(keep, logp - logq, 0.0)
        loss = (p * apart).sum(1)
        room = 1e-5 * ((p * (1 + apart.abs())).sum(1) + loss.abs()) + 2e-5
        for grad in (True, False):
            g = tt.tt_distill(student, o["top_ids"], o["top_logprobs"], tail=True, grad=grad)
            assert (g["status"] == 0).all() and torch.isfinite(g["loss"]).all()
            assert ((g["loss"].cpu().double() - loss).abs() <= room).all()
            back = tt.tt_distill_grad(student, o["top_ids"], o["top_logprobs"], g["stats"], tail=True)
            for x in (back, g.get("grad", back)):
                check_grad(x, q - p, 2e-5 * (q + p), dtype)


@pytest.mark.parametrize("missing", [0.0, 1e-7, 1e-5])
def test_what_counts_as_a_rest(missing):
    """A whole row's list: mass that is missing beyond rounding has no place in the
    student, whose loss is inf; up to rounding there is none."""
    gen = torch.Generator().manual_seed(18)
    logp = torch.log_softmax(torch.randn((50, 16), generator=gen).double(), 1) + math.log1p(-missing)
    ids = torch.arange(16).expand(50, 16).int().contiguous().cuda()
    z = rows_of(torch.randn((50, 16), generator=gen), F)
    loss = tt.tt_distill(z, ids, logp.float().cuda(), tail=True)["loss"]
    assert (loss == math.inf).all() if missing > 1e-6 else torch.isfinite(loss).all()


@pytest.mark.parametrize("dtype", [F, H])
def test_rows_without_a_loss(dtype):
    """No usable entry: 0 and EMPTY. No normaliser or an entry that is no log
    probability: NaN, gradient 0, NOT_FINITE. An impossible column: loss inf, the
    gradient as ever. A column outside the row: the entry is left out."""
    gen = torch.Generator().manual_seed(8)
    V = 3001
    ids, logp = teacher(9, V, 4, gen, unused=0.0)
    z = torch.randn((9, V), generator=gen)
    ids[0] = -1
    logp[1] = -math.inf
    z[2] = -math.inf
    z[3, 17] = math.nan
    z[4, 2999] = math.inf
    logp[5, 2] = math.nan
    logp[6, 0] = math.inf
    z[7, ids[7, 1].item()] = -math.inf
    ids[8, 3] = V
    rows = rows_of(z, dtype)
    for tail in (False, True):
        g = tt.tt_distill(rows, ids.cuda(), logp.cuda(), tail=tail)
        h = tt.tt_distill(rows, ids.cuda(), logp.cuda(), tail=tail, grad=False)
        back = tt.tt_distill_grad(rows, ids.cuda(), logp.cuda(), h["stats"], tail=tail)
        for x in (g, h):
            assert x["status"].tolist() == [4, 4, 16, 16, 16, 16, 16, 0, 1]
            assert x["loss"][:2].tolist() == [0.0, 0.0]
            assert torch.isnan(x["loss"][2:7]).all() and x["loss"][7] == math.inf
        for grad in (g["grad"], back):
            assert (grad[:7] == 0).all()
            assert torch.isfinite(grad).all() and (grad[7:].abs().sum(1) > 0).all()
    some = ids.clone()
    some[8, 3] = -1
    check(z[8:], some[8:], logp[8:], dtype, 1.0, True)


@pytest.mark.parametrize("tail", [False, True])
def test_the_formula_against_differences(tail):
    """The 64-bit gradient that the kernels are held to is the loss's slope."""
    gen = torch.Generator().manual_seed(9)
    V, T, eps = 30, 1.7, 1e-5
    z = (torch.randn((1, V), generator=gen) * 2).double()
    ids, logp = teacher(1, V, 6, gen, unused=0.0)
    logp = logp.double()
    grad = expected(z, ids, logp, T, tail, None)[1][0]
    for j in range(V):
        d = torch.zeros(V).double()
        d[j] = eps
        slope = (loss_of(z[0] + d, ids[0].long(), logp[0], T, tail)
                 - loss_of(z[0] - d, ids[0].long(), logp[0], T, tail)) / (2 * eps)
        assert abs(slope - grad[j]) < 1e-8, j  # (eps^2 and 2^-52 / eps)


@pytest.mark.parametrize("dtype", [F, H])
def test_gradient_in_the_logits_place(dtype):
    gen = torch.Generator().manual_seed(10)
    V = 40007
    ids, logp = (x.cuda() for x in teacher(6, V, 16, gen))
    rows = rows_of(torch.randn((6, V), generator=gen), dtype)
    want = tt.tt_distill(rows, ids, logp, tail=True)
    one, two = rows_of(rows, dtype), rows_of(rows, dtype)
    g = tt.tt_distill(one, ids, logp, tail=True, grad=one)
    assert g["grad"] is one and torch.equal(one, want["grad"])
    assert torch.equal(g["loss"], want["loss"])
    back = tt.tt_distill_grad(two, ids, logp, want["stats"], tail=True, grad=two)
    assert back is two
    assert torch.equal(two, tt.tt_distill_grad(rows, ids, logp, want["stats"], tail=True))


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("R,V", [(3000, 2051), (700, 33001), (60, 151939)])
def test_many_gradients_in_the_logits_place(dtype, R, V):
    """More rows than run at once, ragged ends, lists at both ends of a row."""
    gen = torch.Generator().manual_seed(R)
    ids = torch.randint(V, (R, 8), generator=gen).int().cuda()
    ids[:, 0], ids[:, 1] = 0, V - 1
    logp = (torch.log_softmax(torch.randn((R, 8), generator=gen), 1) - 0.2).cuda()
    rows = rows_of(torch.randn((R, V), generator=gen), dtype)
    want = tt.tt_distill(rows, ids, logp, tail=True)
    later = tt.tt_distill_grad(rows, ids, logp, want["stats"], tail=True)
    one, two = rows_of(rows, dtype), rows_of(rows, dtype)
    tt.tt_distill(one, ids, logp, tail=True, grad=one)
    tt.tt_distill_grad(two, ids, logp, want["stats"], tail=True, grad=two)
    assert torch.equal(one, want["grad"]) and torch.equal(two, later)


def test_autograd():
    gen = torch.Generator().manual_seed(11)
    R, V = 7, 4096
    ids, logp = (x.cuda() for x in teacher(R, V, 10, gen))
    x = torch.randn((R, 64), generator=gen).cuda()
    head = (torch.randn((64, V), generator=gen) / 8).cuda().requires_grad_()
    up = torch.rand(R, generator=gen).cuda()
    loss = tt.distill_loss(x @ head, ids, logp, temp=1.5, tail=True)
    (loss * up).sum().backward()
    z = (x @ head).detach()
    want = x.t() @ tt.tt_distill(z, ids, logp, temp=1.5, tail=True, weight=up)["grad"]
    torch.testing.assert_close(head.grad, want, rtol=1e-4, atol=1e-6)


@pytest.mark.parametrize("dtype", [F, H])
def test_rows_billions_of_bytes_apart(dtype):
    """The same bits as rows that are close, in one call and in two."""
    gen = torch.Generator().manual_seed(13)
    R, V, step = 5, 3001, 2 ** 30 + 8
    ids, logp = (x.cuda() for x in teacher(R, V, 6, gen))
    near = rows_of(torch.randn((R, V), generator=gen), dtype)
    far = torch.empty(R * step, dtype=dtype, device="cuda").as_strided((R, V), (step, 1))
    far.copy_(near)
    g, h = (tt.tt_distill(z, ids, logp, tail=True) for z in (near, far))
    two = tt.tt_distill_grad(far, ids, logp, h["stats"], tail=True)
    tt.tt_distill(far, ids, logp, tail=True, grad=far)
    assert torch.equal(g["loss"], h["loss"])
    for got in (h["grad"], two, far):
        assert torch.equal(g["grad"], got)


def test_a_gradient_has_none_of_its_own():
    """Second derivatives are refused, not taken for zero."""
    gen = torch.Generator().manual_seed(12)
    ids, logp = (x.cuda() for x in teacher(3, 512, 4, gen))
    z = torch.randn((3, 512), generator=gen).cuda().requires_grad_()
    g, = torch.autograd.grad(tt.distill_loss(z * z, ids, logp).sum(), z, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


def test_logprobs_lists_and_streams():
    """What tt_logprobs answers about the target's rows is the teacher's list; the
    calls take the stream they are given, and repeat to the bit."""
    gen = torch.Generator().manual_seed(12)
    target = rows_of(torch.randn((5, 9000), generator=gen) * 3, F)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    o = tt.tt_logprobs(target, top_n=20, temp=0.8, stream=side)
    z = torch.randn((5, 9000), generator=gen)
    rows = rows_of(z, F)
    torch.cuda.synchronize()
    g = tt.tt_distill(rows, o["top_ids"], o["top_logprobs"], tail=True, stream=side)
    torch.cuda.synchronize()
    check(z, o["top_ids"].cpu(), o["top_logprobs"].cpu(), F, 1.0, True)
    h = tt.tt_distill(rows, o["top_ids"], o["top_logprobs"], tail=True)
    assert torch.equal(g["grad"], h["grad"]) and torch.equal(g["loss"], h["loss"])


def test_no_rows():
    g = tt.tt_distill(torch.zeros((0, 64), device="cuda"), torch.zeros((0, 3), dtype=torch.int32),
                      torch.zeros((0, 3)))
    assert g["grad"].shape == (0, 64)


def test_refusals():
    rows = rows_of(torch.zeros((2, 64)), F)
    ids, logp = torch.zeros((2, 3), dtype=torch.int32, device="cuda"), torch.zeros((2, 3), device="cuda")
    for kw in (dict(temp=0.0), dict(temp=math.nan), dict(grad=rows.bfloat16()),
               dict(grad=rows[:1]), dict(grad=rows[:, :60])):
        with pytest.raises(tt.TTError) as e:
            tt.tt_distill(rows, ids, logp, **kw)
        assert e.value.code == binding.TT_ERR_INVALID_ARG
    many = torch.zeros((2, 129), dtype=torch.int32, device="cuda")
    with pytest.raises(tt.TTError):
        tt.tt_distill(rows, many, many.float())
    for a, b in ((ids.long(), logp), (ids, logp.double()), (ids[:1], logp[:1]), (ids, logp[:, :2])):
        with pytest.raises(ValueError):
            tt.tt_distill(rows, a, b)
    with pytest.raises(ValueError):
        tt.tt_distill(rows, ids, logp, weight=torch.zeros(1, device="cuda"))
    with pytest.raises(ValueError):
        tt.tt_distill_grad(rows, ids, logp, torch.zeros(4, device="cuda"))
    lib = tt.load()
    T = binding._Teacher(256, 256, 3)
    wide = binding._Logits(256, binding.TT_F32, 819201, 819204, 2)
    assert lib.tt_distill(ctypes.byref(wide), ctypes.byref(T), 1.0, 0, None, None, None, None,
                          ctypes.c_void_p(256), None) == binding.TT_ERR_UNSUPPORTED
    L = binding._logits(rows)
    assert lib.tt_distill(ctypes.byref(L), ctypes.byref(T), 1.0, 2, None, None, None, None,
                          ctypes.c_void_p(256), None) == binding.TT_ERR_INVALID_ARG
    assert lib.tt_distill(ctypes.byref(L), ctypes.byref(T), 1.0, 0, None, None, None, None, None,
                          None) == binding.TT_ERR_INVALID_ARG
