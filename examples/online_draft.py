"""A serving loop whose draft model learns from the target as it goes: the
library's calls around one verification step, on a toy pair of models.

Each round, for a batch of requests:

1. the draft (a bigram model: the next token from the last one) proposes k tokens;
2. the target (one attention layer) scores them in one pass: ``tt_tree_attn`` over
   the requests' paged caches (here the drafts are chains; a tree of alternatives
   gives its parents);
3. ``tt_step`` verifies them: accepted tokens and the next one, distributed as if
   the target had drawn each;
4. ``tt_logprobs`` answers with the emitted tokens' log probabilities and gives the
   target's top alternatives at every position that was reached;
5. ``tt_distill`` is the draft's loss against those, and its gradient to the draft
   logits; plain products carry it into the draft's weights;
6. ``tt_cache_append`` puts keys and values of the accepted tokens into the cache.

    python examples/online_draft.py [--rounds N]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2510_15545_gb300 as tt  # noqa: E402

V, WIDTH, HEADS, KV_HEADS, HEAD, PAGE = 256, 256, 8, 2, 64, 16
TOP = 20  # alternatives that the draft learns from


class Target:
    """Embedding, one attention layer, output head (fixed random weights)."""

    def __init__(self, gen):
        def randn(*size, scale):
            return torch.randn(size, generator=gen, device="cuda") * scale
        self.embed = randn(V, WIDTH, scale=1.0)
        self.wq = randn(WIDTH, HEADS * HEAD, scale=WIDTH ** -0.5)
        self.wkv = randn(WIDTH, 2 * KV_HEADS * HEAD, scale=WIDTH ** -0.5)
        self.wo = randn(HEADS * HEAD, WIDTH, scale=0.25 * (HEADS * HEAD) ** -0.5)
        self.head = randn(WIDTH, V, scale=3.0 * WIDTH ** -0.5)

    def project(self, tokens):
        x = self.embed[tokens]
        q = (x @ self.wq).bfloat16().view(-1, HEADS, HEAD)
        kv = (x @ self.wkv).bfloat16().view(-1, 2 * KV_HEADS, HEAD)
        return x, q, kv[:, :KV_HEADS], kv[:, KV_HEADS:]


class Cache:
    """Paged keys and values of B requests of up to `length` tokens."""

    def __init__(self, B, length, gen):
        per = (length + PAGE - 1) // PAGE
        self.k = torch.zeros((B * per, PAGE, KV_HEADS, HEAD), dtype=torch.bfloat16, device="cuda")
        self.v = torch.zeros_like(self.k)
        self.table = torch.randperm(B * per, generator=gen, device="cuda").int().view(B, per)
        self.len = torch.zeros(B, dtype=torch.int32, device="cuda")

    def append(self, k, v, counts):
        """The first counts[b] of request b's n tokens, k and v [B, n, heads, head]."""
        B, n = k.shape[:2]
        off = torch.arange(B + 1, dtype=torch.int32, device="cuda") * n
        self.len = tt.tt_cache_append(k.flatten(0, 1), v.flatten(0, 1), self.k, self.v, self.table,
                                      self.len, off, keep=counts, max_new=n)["new_len"]


def run(rounds=60, B=32, k=4, rate=3.0, seed=0, report=None):
    """Returns the mean accepted tokens and the mean loss of each round."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    target, cache = Target(gen), Cache(B, rounds * (k + 1) + 1, gen)
    draft = torch.zeros((V, V), device="cuda")  # logits of the next token, by the last one
    strings = torch.arange(V, dtype=torch.int32)
    table = tt.VocabTable.from_host(torch.stack([strings // 256, strings % 256], 1).flatten(),
                                    torch.arange(V + 1) * 2)
    params = tt.Params(full_q=True, seed=seed)
    last = torch.randint(V, (B,), generator=gen, device="cuda")
    tree_off = torch.arange(B + 1, dtype=torch.int32, device="cuda") * (k + 1)
    history = []
    for step in range(rounds):
        # 1. draft
        rows, drafted = [], [last]
        for _ in range(k):
            rows.append(draft[drafted[-1]])
            drafted.append(torch.multinomial(torch.softmax(rows[-1], 1), 1, generator=gen)[:, 0])
        draft_rows = torch.stack(rows, 1).view(B * k, V)
        nodes = torch.stack(drafted, 1)  # [B, k + 1], the last known token first
        # 2. the target's rows: one more than drafted tokens, in tt_step's order
        x, q, key, value = target.project(nodes.flatten())
        a = tt.tt_tree_attn(q, key, value, cache.k, cache.v, cache.table, cache.len, tree_off,
                            max_nodes=k + 1)
        target_rows = (x + a["out"].float().flatten(1) @ target.wo) @ target.head
        # 3. verify
        ids = nodes[:, 1:].int().flatten()
        off = torch.arange(B + 1, dtype=torch.int32) * k
        batch = tt.Batch.from_host(off, ids.cpu(), off, ids.cpu(), max_k=k, max_m=k)
        params.request_base = step * B
        out = tt.tt_step(batch, table, table, draft_rows, target_rows, params)
        accepted, following = out["accepted"].long(), out["next_token"].long()
        # 4. what is answered: every position up to the one that decided
        i = torch.arange(k + 1, device="cuda")
        emitted = torch.cat([nodes[:, 1:], following[:, None]], 1)
        emitted = torch.where(i == accepted[:, None], following[:, None], emitted)
        reached = i <= accepted[:, None]
        answer = tt.tt_logprobs(target_rows, torch.where(reached, emitted, -1).int().flatten(),
                                top_n=TOP)
        # 5. learn from the positions that were reached (draft row i is the target's row i)
        keep = (i < k).expand(B, -1).flatten()
        weight = reached[:, :k].float().flatten()
        loss = tt.tt_distill(draft_rows, answer["top_ids"][keep], answer["top_logprobs"][keep],
                             tail=True, weight=weight)
        draft.index_add_(0, nodes[:, :k].flatten(), loss["grad"], alpha=-rate)
        # 6. the last known token and the accepted ones enter the cache
        cache.append(key.reshape(B, k + 1, KV_HEADS, HEAD), value.reshape(B, k + 1, KV_HEADS, HEAD),
                     (accepted + 1).int())
        last = following
        mean = (loss["loss"] * weight).sum() / weight.sum()
        logprob = answer["logprob"].sum() / reached.sum()
        history.append((accepted.float().mean().item(), mean.item(), logprob.item()))
        if report and (step % report == 0 or step + 1 == rounds):
            print("round %3d  accepted %.2f of %d  draft loss %.3f  log p of emitted tokens %.3f"
                  % (step, history[-1][0], k, history[-1][1], history[-1][2]), flush=True)
    return history


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--rounds", type=int, default=200)
    run(ap.parse_args().rounds, report=20)
