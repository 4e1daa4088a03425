"""The operators' bounded waits run out without a GPU fault: the library's test hook
(TT_TEST_STALL_STAGE, TT_TEST_WAIT_MS, read once per process) has one CTA of the
process's first launch wait for copies that nobody issues, with a limit of 50 ms.
The call must end on its own and report TT_REQ_TIMEOUT where that CTA's work was
needed and nowhere else, and the next call must be as any. Each case runs in a
child process of its own."""
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

DISTILL = r"""
import math, sys, time
sys.path.insert(0, %(root)r)
import torch
import paper_2510_15545_gb300 as tt
from paper_2510_15545_gb300 import binding
tt.load(build_if_missing=True)
gen = torch.Generator(device="cuda").manual_seed(1)
R, V, row, tail = %(R)d, %(V)d, %(row)d, %(tail)r
z = torch.randn((R, V), generator=gen, device="cuda").to(torch.%(dtype)s)
ids = torch.randint(V, (R, 8), generator=gen, device="cuda").int()
logp = torch.log_softmax(torch.randn((R, 8), generator=gen, device="cuda"), 1) - 0.1
torch.cuda.synchronize()
t0 = time.perf_counter()
g = tt.tt_distill(z, ids, logp, tail=tail, grad=%(grad)r)
torch.cuda.synchronize()
assert time.perf_counter() - t0 < 20.0
assert binding.load().tt_last_cuda_error() == 0
want = [0] * R
want[row] = 32
assert g["status"].tolist() == want, g["status"]
h = tt.tt_distill(z, ids, logp, tail=tail, grad=%(grad)r)
assert h["status"].tolist() == [0] * R and torch.isfinite(h["loss"]).all()
other = torch.arange(R, device="cuda") != row
assert math.isnan(g["loss"][row].item())
for x, y in ((g, h),) if %(grad)r else ():
    assert (x["grad"][row] == 0).all() and (y["grad"][row] != 0).any()
    assert torch.equal(x["grad"][other], y["grad"][other])
for key in ("loss", "stats"):
    assert torch.equal(g[key][other], h[key][other])
# statistics of a row that was given up say so to a later gradient
back = tt.tt_distill_grad(z, ids, logp, g["stats"], tail=tail)
assert (back[row] == 0).all() and (back[other].abs().sum(1) > 0).all()
print("child ok")
"""


def _run_child(code, cta):
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    env = dict(os.environ, TT_TEST_STALL_STAGE=str(cta), TT_TEST_WAIT_MS="50")
    p = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True,
                       timeout=300)
    assert p.returncode == 0 and "child ok" in p.stdout, (p.stdout[-2000:], p.stderr[-4000:])


# rows of one CTA (with and without a gradient), of six and of twelve (its first, others)
@pytest.mark.parametrize("R,V,dtype,tail,grad,cta,row", [
    (9, 3000, "float32", True, True, 5, 5), (9, 3000, "bfloat16", False, False, 0, 0),
    (30, 128256, "bfloat16", True, True, 0, 0), (30, 128256, "bfloat16", True, True, 21, 3),
    (40, 151936, "float32", False, True, 47, 3)])
def test_a_row_whose_logits_do_not_come(R, V, dtype, tail, grad, cta, row):
    _run_child(DISTILL % dict(root=ROOT, R=R, V=V, dtype=dtype, tail=tail, grad=grad, row=row), cta)


TREE = r"""
import sys, time
sys.path.insert(0, %(root)r)
import torch
import paper_2510_15545_gb300 as tt
from paper_2510_15545_gb300 import binding
tt.load(build_if_missing=True)
gen = torch.Generator(device="cuda").manual_seed(2)
lens, n, Hq, Hkv, D, hit, may = %(lens)r, %(n)d, %(Hq)d, %(Hkv)d, %(D)d, %(hit)r, %(may)r
B, page = len(lens), 64
P = (max(lens) + page - 1) // page
randn = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.%(dtype)s)
i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
args = (randn(B * n, Hq, D), randn(B * n, Hkv, D), randn(B * n, Hkv, D),
        randn(B * P, page, Hkv, D), randn(B * P, page, Hkv, D),
        torch.arange(B * P, device="cuda").int().view(B, P), i32(lens),
        torch.arange(B + 1, device="cuda").int() * n)
torch.cuda.synchronize()
t0 = time.perf_counter()
g = tt.tt_tree_attn(*args, max_len=max(lens), max_nodes=n)
torch.cuda.synchronize()
assert time.perf_counter() - t0 < 20.0
assert binding.load().tt_last_cuda_error() == 0
status = g["status"].tolist()
late = [b for b in range(B) if status[b]]
assert all(status[b] == 32 for b in late) and set(hit) <= set(late) <= set(may), (late, hit, may)
h = tt.tt_tree_attn(*args, max_len=max(lens), max_nodes=n)
assert h["status"].tolist() == [0] * B and torch.isfinite(h["out"]).all()
for b in range(B):
    if b not in late:
        for key in ("out", "lse"):
            assert torch.equal(g[key][b * n:(b + 1) * n], h[key][b * n:(b + 1) * n]), (b, key)
print("child ok")
"""


def _list(lens, n, Hq, Hkv):
    """The requests of the places of the list that the CTAs share, and a CTA's share."""
    per_tile = 128 // (Hq // Hkv)
    tiles = lambda x: (x + 127) // 128  # noqa: E731
    places = []
    for b, L in enumerate(lens):
        for _ in range(Hkv):
            for first in range(0, n, per_tile):
                places += [b] * (3 + tiles(L) + tiles(min(n, first + per_tile)))
    ctas = 2 * torch.cuda.get_device_properties(0).multi_processor_count
    return places, max(2, -(-len(places) // ctas))


# one row tile a head, and two; wide heads, and narrow ones, whose products run ahead
@pytest.mark.parametrize("n,Hq,Hkv,D,dtype", [
    (4, 8, 2, 128, "bfloat16"), (5, 4, 2, 64, "float16"), (32, 16, 2, 128, "bfloat16"),
    (64, 8, 2, 64, "float16")])
@pytest.mark.parametrize("two", [False, True])
def test_requests_whose_keys_do_not_come(n, Hq, Hkv, D, dtype, two):
    """A CTA that gives up within one request, or before it comes to the next one:
    both are told, and no others."""
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    lens = [40000, 39000, 38500, 41000, 37777, 40001, 36000, 42000]
    places, share = _list(lens, n, Hq, Hkv)
    assert share >= 8
    for cta in range(3, len(places) // share):
        mine = places[cta * share:(cta + 1) * share]
        # (two tiles at least before the next request begins)
        if (mine[0] != mine[-1] and mine.count(mine[0]) >= 5) if two else mine[0] == mine[-1]:
            break
    else:
        pytest.skip("no such CTA among these places")
    _run_child(TREE % dict(root=ROOT, lens=lens, n=n, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype,
                           hit=sorted({mine[0], mine[-1]}), may=sorted(set(mine))), cta)
