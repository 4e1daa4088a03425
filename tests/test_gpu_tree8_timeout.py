"""The bounded waits of tt_tree_attn over caches in 8 bits run out without a GPU fault, as
those of the other operators do: one CTA of the process's first launch waits for copies that
nobody issues, with a limit of 50 ms. The call must end on its own and report TT_REQ_TIMEOUT
where that CTA's work was needed and nowhere else, and the next call must be as any."""
import pytest
import torch

from test_gpu_operators_timeout import ROOT, _run_child

pytestmark = pytest.mark.gpu

TREE8 = r"""
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
cache = lambda: randn(B * P, page, Hkv, D).to(torch.float8_e4m3fn)
scale = lambda: torch.randint(120, 130, (B * P, page // 16, Hkv), generator=gen, device="cuda").byte()
args = (randn(B * n, Hq, D), randn(B * n, Hkv, D), randn(B * n, Hkv, D), cache(), cache(),
        torch.arange(B * P, device="cuda").int().view(B, P), i32(lens),
        torch.arange(B + 1, device="cuda").int() * n)
kw = dict(k_scale=scale(), v_scale=scale(), max_len=max(lens), max_nodes=n)
torch.cuda.synchronize()
t0 = time.perf_counter()
g = tt.tt_tree_attn(*args, **kw)
torch.cuda.synchronize()
assert time.perf_counter() - t0 < 20.0
assert binding.load().tt_last_cuda_error() == 0
status = g["status"].tolist()
late = [b for b in range(B) if status[b]]
assert all(status[b] == 32 for b in late) and set(hit) <= set(late) <= set(may), (late, hit, may)
h = tt.tt_tree_attn(*args, **kw)
assert h["status"].tolist() == [0] * B and torch.isfinite(h["out"]).all()
for b in range(B):
    if b not in late:
        for key in ("out", "lse"):
            assert torch.equal(g[key][b * n:(b + 1) * n], h[key][b * n:(b + 1) * n]), (b, key)
print("child ok")
"""


def _list(lens, n, Hq, Hkv, rows):
    """The requests of the places of the list that the CTAs share, and a CTA's share."""
    group = Hq // Hkv
    tiles = lambda x: (x + 127) // 128  # noqa: E731
    places = []
    for _ in range(Hkv):
        for b, L in enumerate(lens):
            for row in range(0, n * group, rows):
                end = (min(n * group, row + rows) - 1) // group + 1
                places += [b] * (5 + tiles(L) + tiles(end))
    ctas = torch.cuda.get_device_properties(0).multi_processor_count
    return places, max(2, -(-len(places) // ctas))


# few rows (16 and 32 columns) and many, of one item a head and of two
@pytest.mark.parametrize("n,Hq,Hkv,D,dtype,rows", [
    (4, 8, 2, 128, "bfloat16", 16), (10, 4, 2, 64, "float16", 32), (12, 8, 2, 128, "bfloat16", 128),
    (16, 8, 2, 64, "bfloat16", 128), (40, 8, 2, 128, "float16", 128)])
@pytest.mark.parametrize("two", [False, True])
def test_requests_whose_keys_do_not_come(n, Hq, Hkv, D, dtype, rows, two):
    """A CTA that gives up within one request, or before it comes to the next one:
    both are told, and no others."""
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    lens = [40000, 39000, 38500, 41000, 37777, 40001, 36000, 42000]
    places, share = _list(lens, n, Hq, Hkv, rows)
    assert share >= 16
    for cta in range(3, len(places) // share):
        mine = places[cta * share:(cta + 1) * share]
        # (two tiles at least before the next request begins, and two of that, each behind what
        # an item costs)
        if (mine[0] != mine[-1] and mine.count(mine[0]) >= 8 and mine.count(mine[-1]) >= 8
                if two else mine[0] == mine[-1]):
            break
    else:
        pytest.skip("no such CTA among these places")
    _run_child(TREE8 % dict(root=ROOT, lens=lens, n=n, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype,
                            hit=sorted({mine[0], mine[-1]}), may=sorted(set(mine))), cta)
