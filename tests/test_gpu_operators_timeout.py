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
