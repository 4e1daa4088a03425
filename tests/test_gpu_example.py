"""The example's loop: its calls work together, and the draft learns."""
import importlib.util
import os

import pytest
import torch

import paper_2510_15545_gb300 as tt

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    tt.load(build_if_missing=True)
    spec = importlib.util.spec_from_file_location(
        "online_draft", os.path.join(ROOT, "examples", "online_draft.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_the_draft_learns_from_the_target(example):
    history = torch.tensor(example.run(rounds=120, seed=3))
    assert torch.isfinite(history).all()
    first, last = history[:20].mean(0), history[-20:].mean(0)
    # a draft that knows nothing is accepted by chance; one that has learned, often
    assert last[0] > first[0] + 0.5
    assert last[1] < 0.7 * first[1]


def test_the_target_pass_matches_plain_attention(example):
    """One round's target rows, from the paged cache and the drafted chain, are
    those of plain causal attention over the whole text in 32 bits (bf16 heads:
    the weights' rounding, 2^-8, on an update of the residual stream's size / 2,
    through a head of 16 times its root)."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    B, k, L = 3, 4, 37
    target, cache = example.Target(gen), example.Cache(B, 64, gen)
    text = torch.randint(example.V, (B, L + k + 1), generator=gen, device="cuda")
    _, _, key, value = target.project(text[:, :L].flatten())
    shape = (B, L, example.KV_HEADS, example.HEAD)
    cache.append(key.reshape(shape), value.reshape(shape),
                 torch.full((B,), L, dtype=torch.int32, device="cuda"))
    x, q, key, value = target.project(text[:, L:].flatten())
    off = torch.arange(B + 1, dtype=torch.int32, device="cuda") * (k + 1)
    a = tt.tt_tree_attn(q, key, value, cache.k, cache.v, cache.table, cache.len, off)["out"]
    for b in range(B):
        _, qs, ks, vs = (y.float() for y in target.project(text[b]))
        group = example.HEADS // example.KV_HEADS
        s = torch.einsum("ihd,jhd->hij", qs, ks.repeat_interleave(group, 1)) * example.HEAD ** -0.5
        n = L + k + 1
        s = s.masked_fill(torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1), -torch.inf)
        want = torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), vs.repeat_interleave(group, 1))
        got = a.view(B, k + 1, example.HEADS, example.HEAD)[b].float()
        torch.testing.assert_close(got, want[L:], rtol=2.0 ** -7, atol=2.0 ** -7)
