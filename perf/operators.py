"""The operators that stand around a verification step in a serving loop whose
draft model keeps learning, over the range of the framework's own workloads:

* ``tree``: attention of a target model's layer for the drafted tokens of every
  request (a chain, or a tree of alternatives) over the request's paged cache --
  the scoring pass whose logits the verification step reads;
* ``logprobs``: what a server answers about those logits rows: log probability
  and rank of a given token, entropy, and the top alternatives;
* ``distill``: the draft model's loss against the target's top log
  probabilities and its gradient to the draft logits, in one call (``both``) or
  as a forward and a backward call (``split``).

Logits are Zipf-distributed over permuted columns with Gaussian noise, as in
the package's synthetic workloads; the widths are those of its configurations,
or odd ones.
"""
from __future__ import annotations

import math

import torch

own = False

LOG2E = 1.4426950408889634


def _lp(name, R, V, dtype, top_n, temp=1.0, masked="none", pad=0):
    """masked: share of columns that a grammar or a ban list takes out, with
    -inf ("inf", which also leaves row 0 empty when there are more rows than
    one) or the type's lowest value ("low"); pad: columns between rows beyond
    the alignment's."""
    return dict(name=name, op="logprobs", R=R, V=V, dtype=dtype, top_n=top_n, temp=temp,
                masked=masked, pad=pad)


def _ds(name, form, R, V, dtype, K, tail, temp=1.0):
    return dict(name=name, op="distill", form=form, R=R, V=V, dtype=dtype, K=K, tail=tail,
                temp=temp)


def _ta(name, B, nodes, Hq, Hkv, D, length, page, dtype="bf16", ragged=True, chain=False):
    """nodes: most drafted tokens of a request; length: longest cache."""
    return dict(name=name, op="tree", B=B, nodes=nodes, Hq=Hq, Hkv=Hkv, D=D, length=length,
                page=page, dtype=dtype, ragged=ragged, chain=chain)


def listed():
    return [
        # One interactive request, one logits row: latency.
        _lp("logprobs_one_row", 1, 32768, "f32", 5),
        # A few rows of an odd width under a grammar mask, one of them empty.
        _lp("logprobs_masked_odd", 37, 50257, "bf16", 32, masked="inf", pad=8),
        # The rows of a 64-request step (9.5 target rows each), fp32.
        _lp("logprobs_b64_f32", 608, 151936, "f32", 20, temp=0.6),
        # Rows of a full serving batch, bf16: bandwidth.
        _lp("logprobs_serving_bf16", 4096, 201088, "bf16", 20),
        # The rows of one interactive request's draft, learned from at once.
        _ds("distill_one_draft", "both", 4, 32000, "f32", 8, False),
        # A training batch over a bf16 vocabulary, with the mass outside the list.
        _ds("distill_batch_bf16", "both", 2048, 128256, "bf16", 20, True),
        # fp32 draft logits, an odd number of rows, a softened student.
        _ds("distill_batch_f32", "both", 1001, 151936, "f32", 32, False, temp=2.0),
        # Forward and backward as two calls, longer teacher lists.
        _ds("distill_split_bf16", "split", 1024, 151936, "bf16", 64, True),
        # One interactive request with a chain of four drafted tokens and the last one.
        _ta("tree_one_chain", 1, 5, 32, 8, 128, 1000, 16, ragged=False, chain=True),
        # A serving batch: eight drafted tokens and the last one, ragged caches.
        _ta("tree_serving", 64, 9, 32, 8, 128, 8192, 64),
        # Two long documents with wide trees; few heads, so the cache is split.
        _ta("tree_long", 2, 32, 16, 2, 128, 131072, 128),
        # Wide trees over medium caches, narrow heads, fp16.
        _ta("tree_wide_f16", 16, 64, 32, 8, 64, 4096, 32, dtype="f16"),
    ]


# Bounds of drawn cases: the largest listed ones.
MOST_LOGITS = {"logprobs": 4096 * 201088 * 2, "distill": 1001 * 151936 * 4}
MOST_CACHE = 2 * 131072 * 2 * 128 * 4  # bytes of keys and values that are read
MOST_SCORES = 64 * 32 * 9 * 8192       # scores of the plain form


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "distill", "tree"])
    if op == "tree":
        G = rng.choice([1, 2, 3, 4, 5, 7, 8, 16])
        Hkv = rng.choice([1, 2, 4, 8])
        D = rng.choice([64, 128])
        nodes = _log(rng, 1, 64)
        B = _log(rng, 1, 64)
        page = rng.choice([16, 32, 48, 64, 128])
        room = min(MOST_CACHE // (B * Hkv * D * 4), MOST_SCORES // (B * G * Hkv * nodes), 131072)
        length = _log(rng, 16, max(17, room))
        c = _ta("", B, nodes, G * Hkv, Hkv, D, length, page, rng.choice(["bf16", "f16"]),
                ragged=rng.random() < 0.75, chain=rng.random() < 0.3)
    else:
        dtype = rng.choice(["f32", "bf16"])
        V = rng.choice([32000, 32768, 50257, 128256, 151936, 201088, _log(rng, 2048, 201088),
                        _log(rng, 2048, 201088) | 1])
        R = _log(rng, 1, min(4096, MOST_LOGITS[op] // (V * (4 if dtype == "f32" else 2))))
        temp = rng.choice([0.6, 0.7, 1.0, 1.0, 2.0])
        if op == "logprobs":
            c = _lp("", R, V, dtype, rng.choice([0, 1, 5, 8, 20, 32]), temp,
                    rng.choice(["none", "none", "inf", "low"]), rng.choice([0, 0, 8, 64]))
        else:
            c = _ds("", rng.choice(["both", "both", "split"]), R, V, dtype,
                    rng.choice([1, 8, 20, 32, 64, 128]), rng.random() < 0.5, temp)
    del c["name"]
    return c


# ------------------------------------------------------------------- inputs

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _rows(R, V, dtype, pad=0):
    """R logits rows of V columns whose stride is a multiple of 16 bytes."""
    stride = (V + 7) // 8 * 8 + pad
    return torch.zeros((R, stride), dtype=dtype, device="cuda")[:, :V]


def _zipf(R, V, gen):
    """fp32 rows: -1.1 log(rank) of columns permuted by a rotation of one random
    permutation per row, and Gaussian noise."""
    rank = torch.randperm(V, generator=gen, device="cuda")
    at = torch.randint(V, (R, 1), generator=gen, device="cuda")
    z = torch.log1p(rank.float()).mul_(-1.1)
    z = torch.cat([z, z])
    out = torch.randn((R, V), generator=gen, device="cuda")
    for r0 in range(0, R, 256):  # (the index of a block at a time)
        out[r0:r0 + 256] += z[at[r0:r0 + 256] + torch.arange(V, device="cuda")]
    return out


def _prepare_logprobs(c, gen):
    R, V = c["R"], c["V"]
    z = _zipf(R, V, gen)
    ids = torch.where(torch.rand(R, generator=gen, device="cuda") < 0.7, z.argmax(1),
                      torch.randint(V, (R,), generator=gen, device="cuda"))
    rows = _rows(R, V, DTYPES[c["dtype"]], c["pad"])
    if c["masked"] != "none":
        out = torch.rand(V, generator=gen, device="cuda") < 0.9
        out[:3] = torch.tensor([False, False, True], device="cuda")
        z.masked_fill_(out, -math.inf if c["masked"] == "inf" else torch.finfo(rows.dtype).min)
        if c["masked"] == "inf" and R > 1:
            z[0] = -math.inf
    rows.copy_(z)
    return dict(logits=rows, ids=ids.int())


def _prepare_distill(c, gen):
    R, V = c["R"], c["V"]
    z = _zipf(R, V, gen)
    v, i = z.topk(c["K"], 1)  # the teacher's list, at its own temperature 1
    lse = torch.logsumexp(z, 1, keepdim=True)
    rows = _rows(R, V, DTYPES[c["dtype"]])
    rows.copy_(z.mul_(0.9).add_(torch.randn((R, V), generator=gen, device="cuda"), alpha=0.4))
    kept = torch.rand(R, generator=gen, device="cuda") < 0.9  # positions that are learned from
    kept[0] = True
    return dict(logits=rows, ids=i.int(), logp=v - lse,
                weight=kept.float() / kept.sum())


def _prepare_tree(c, gen):
    B, n, Hq, Hkv, D, page = c["B"], c["nodes"], c["Hq"], c["Hkv"], c["D"], c["page"]
    dt = DTYPES[c["dtype"]]

    def ints(lo, hi, size):
        return torch.randint(lo, hi, size, generator=gen, device="cuda")

    # (ragged trees of n / 2 to n nodes; how many a request has goes by the case alone)
    counts = n - torch.arange(B, device="cuda") * 7 % (n - max(1, n // 2) + 1 if c["ragged"] else 1)
    length = ints(0, c["length"] + 1, (B,)) if c["ragged"] else torch.full((B,), c["length"], device="cuda")
    length[0] = c["length"]
    off = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), counts.cumsum(0)])
    N = int(off[-1])
    req = torch.repeat_interleave(torch.arange(B, device="cuda"), counts)
    node = torch.arange(N, device="cuda") - off[req]
    up = node - 1
    if not c["chain"]:  # a node's parent: any of the few before it
        up = torch.minimum(torch.clamp(node - 1 - ints(0, 4, (N,)), min=0), up)
    P = (c["length"] + page - 1) // page
    pages = B * P + 3
    table = torch.randperm(pages, generator=gen, device="cuda")[:B * P].view(B, P)
    randn = lambda *size: torch.randn(size, generator=gen, device="cuda").to(dt)  # noqa: E731
    return dict(q=randn(N, Hq, D), k=randn(N, Hkv, D), v=randn(N, Hkv, D),
                k_cache=randn(pages, page, Hkv, D), v_cache=randn(pages, page, Hkv, D),
                page_table=table.int(), cache_len=length.int(), tree_off=off.int(),
                parents=up.int())


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"logprobs": _prepare_logprobs, "distill": _prepare_distill,
         "tree": _prepare_tree}[case["op"]](case, gen)
    return dict(s, case=dict(case))


# -------------------------------------------------------------- plain forms

def _plain_logprobs(s):
    c = s["case"]
    z = s["logits"].float() + 0.0  # (-0 as 0)
    R, V = z.shape
    top = z.amax(1)
    bad = ~(top.abs() < math.inf)  # an empty row, +inf or NaN
    d = (z - top[:, None]) / c["temp"]
    e = torch.exp(d)
    S = e.sum(1)
    lse = top / c["temp"] + torch.log(S)
    entropy = torch.log(S) - torch.where(e > 0, e * d, 0.0).sum(1) / S
    del d, e
    t = s["ids"].long()[:, None]
    zt = z.gather(1, t)
    col = torch.arange(V, device=z.device)
    rank = ((z > zt) | ((z == zt) & (col < t))).sum(1)
    bits = z.view(torch.int32)
    key = (bits ^ ((bits >> 31) & 0x7fffffff)).long() * 2**32 + (V - 1 - col)
    best = V - 1 - (key.topk(c["top_n"], 1).values & 0xffffffff)
    zb = z.gather(1, best)
    gone = bad[:, None] | (zb == -math.inf)

    def nan(x):
        return torch.where(bad, math.nan, x)

    return dict(logprob=nan(zt[:, 0] / c["temp"] - lse), rank=torch.where(bad, -1, rank).int(),
                entropy=nan(entropy), lse=nan(lse),
                top_ids=torch.where(gone, -1, best).int(),
                top_logprobs=torch.where(bad[:, None], math.nan, zb / c["temp"] - lse[:, None]))


def _plain_distill(s):
    c = s["case"]
    z = s["logits"].float() / c["temp"]
    top = z.amax(1, keepdim=True)
    lse = top + torch.log(torch.exp(z - top).sum(1, keepdim=True))
    at = s["ids"].long()
    logp = s["logp"]
    if not c["tail"]:
        lead = logp.amax(1, keepdim=True)
        logp = logp - lead - torch.log(torch.exp(logp - lead).sum(1, keepdim=True))
    p = torch.exp(logp)
    mass = p.sum(1)
    loss = (p * (logp - (z.gather(1, at) - lse))).sum(1)
    q = torch.exp(z - lse)
    listed_q = q.gather(1, at)
    if c["tail"]:
        rest = torch.clamp(1.0 - mass, min=0.0)
        q.scatter_(1, at, 0.0)
        out = q.sum(1)
        loss = loss + torch.where(rest > 0, rest * (torch.log(rest) - torch.log(out)), 0.0)
        mass = mass + rest
        q *= (mass - rest / out)[:, None]
    else:
        q *= mass[:, None]
    q.scatter_(1, at, listed_q * mass[:, None] - p)
    q *= (s["weight"] / c["temp"])[:, None]
    return dict(loss=loss, grad=q.to(s["logits"].dtype))


def _padded(s):
    """Node indices [B, nodes] of every request and which of them exist."""
    off = s["tree_off"].long()
    at = off[:-1, None] + torch.arange(s["case"]["nodes"], device=off.device)
    there = at < off[1:, None]
    return torch.where(there, at, off[:-1, None]), there


def _ancestors(s, at, there):
    """[B, nodes, nodes]: whether node j is node i or above it in the tree: the
    paths of any length along the parents' edges."""
    n = s["case"]["nodes"]
    up = s["parents"].long()[at]
    edge = (up[:, :, None] == torch.arange(n, device=at.device)) & there[:, :, None]
    step = edge.double() + torch.eye(n, dtype=torch.float64, device=at.device)
    return torch.linalg.matrix_power(step, n) > 0


def _plain_tree(s):
    c = s["case"]
    B, n, Hq, Hkv, D = c["B"], c["nodes"], c["Hq"], c["Hkv"], c["D"]
    at, there = _padded(s)
    L = c["length"]
    table = s["page_table"].long()
    seen = torch.cat([(torch.arange(L, device=at.device) < s["cache_len"][:, None])[:, None]
                      .expand(B, n, L), _ancestors(s, at, there)], 2)  # [B, n, L + n]

    def heads(cache, new):  # [B, Hkv, L + n, D]
        old = cache[table].view(B, -1, Hkv, D)[:, :L]
        x = torch.cat([old, new[at]], 1).float().transpose(1, 2)
        return torch.where(seen.any(1)[:, None, :, None], x, 0.0)

    q = s["q"][at].float().view(B, n, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4)
    k = heads(s["k_cache"], s["k"])
    score = (q.reshape(B, Hkv, -1, D) @ k.transpose(2, 3)).view(B, Hkv, Hq // Hkv, n, L + n)
    del k
    score = torch.where(seen[:, None, None], score / math.sqrt(D), -math.inf)
    top = score.amax(-1, keepdim=True)
    e = torch.exp(score.sub_(top))
    S = e.sum(-1, keepdim=True)
    x = e.view(B, Hkv, -1, L + n) @ heads(s["v_cache"], s["v"])
    x = x.view(B, Hkv, Hq // Hkv, n, D) / S
    lse = (top + torch.log(S))[..., 0]
    return dict(out=x.permute(0, 3, 1, 2, 4)[there].reshape(-1, Hq, D).to(s["q"].dtype),
                lse=lse.permute(0, 3, 1, 2)[there].reshape(-1, Hq))


# -------------------------------------------------------- the framework's own

def _own(s):
    from paper_2510_15545_gb300 import binding as tt
    c = s["case"]
    if c["op"] == "logprobs":
        o = tt.tt_logprobs(s["logits"], s["ids"], temp=c["temp"], top_n=c["top_n"])
        return {x: o[x] for x in ("logprob", "rank", "entropy", "lse", "top_ids", "top_logprobs")}
    if c["op"] == "tree":
        o = tt.tt_tree_attn(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["page_table"],
                            s["cache_len"], s["tree_off"], s["parents"], max_len=c["length"],
                            max_nodes=c["nodes"])
        return dict(out=o["out"], lse=o["lse"])
    o = tt.tt_distill(s["logits"], s["ids"], s["logp"], temp=c["temp"], tail=c["tail"],
                      weight=s["weight"], grad=c["form"] == "both")
    if c["form"] == "both":
        return dict(loss=o["loss"], grad=o["grad"])
    return dict(loss=o["loss"],
                grad=tt.tt_distill_grad(s["logits"], s["ids"], s["logp"], o["stats"],
                                        temp=c["temp"], tail=c["tail"], weight=s["weight"]))


def run(state):
    if own:
        return _own(state)
    return {"logprobs": _plain_logprobs, "distill": _plain_distill,
            "tree": _plain_tree}[state["case"]["op"]](state)


# --------------------------------------------------------------------- work

def _lengths(c):
    """Mean cache length and nodes of a case's requests."""
    if not c["ragged"]:
        return c["length"], c["nodes"]
    B, n = c["B"], c["nodes"]
    low = max(1, n // 2)
    return ((c["length"] + (B - 1) * c["length"] / 2) / B, (n + (B - 1) * (low + n) / 2) / B)


def work(case):
    """Logits or cache read once, outputs written once."""
    c = case
    if c["op"] == "tree":
        L, n = _lengths(c)
        cache = c["B"] * L * c["Hkv"] * c["D"] * 4
        new = c["B"] * n * c["D"] * 2 * (2 * c["Hq"] + 2 * c["Hkv"])
        return {"bytes": cache + new + 4 * c["B"] * n * c["Hq"],
                "flops": 4 * c["B"] * n * c["Hq"] * c["D"] * (L + (n + 1) / 2)}
    esz = 4 if c["dtype"] == "f32" else 2
    cells = c["R"] * c["V"]
    if c["op"] == "logprobs":  # difference, scale, exponential, two sums
        return {"bytes": esz * cells + c["R"] * (20 + 8 * c["top_n"]), "flops": 6 * cells}
    # the logits once and the gradient; as two calls, the logits twice
    passes = 2 if c["form"] == "both" else 3
    return {"bytes": passes * esz * cells + c["R"] * (8 + 8 * c["K"]), "flops": 8 * cells}


# ------------------------------------------------------ the same in 64 bits

def _exact_logprobs(s):
    c, T = s["case"], s["case"]["temp"]
    parts = []
    for rows, ids in zip(s["logits"].split(256), s["ids"].split(256)):
        x = rows.double()
        lse = torch.logsumexp(x / T, 1)
        logp = x / T - lse[:, None]
        p = torch.exp(logp)
        entropy = -torch.nansum(torch.where(p == 0, 0.0, p * logp), 1)
        best = torch.topk(x, c["top_n"], 1).values / T - lse[:, None]
        bad = ~torch.isfinite(lse)
        out = [logp.gather(1, ids.long()[:, None])[:, 0], entropy, lse]
        parts.append([torch.where(bad, math.nan, o) for o in out]
                     + [torch.where(bad[:, None], math.nan, best)])
    one = [torch.cat(x) for x in zip(*parts)]
    return dict(logprob=one[0], rank=None, entropy=one[1], lse=one[2], top_ids=None,
                top_logprobs=one[3])


def _exact_distill(s):
    """The loss as a divergence of two distributions, its gradient by the
    softmax's derivative: with d the loss's derivative to the student's log
    probabilities, (d - q sum(d)) / T."""
    c = s["case"]
    losses, grads = [], []
    for rows, ids, logp, w in zip(*(s[x].split(128) for x in ("logits", "ids", "logp", "weight"))):
        logq = torch.log_softmax(rows.double() / c["temp"], 1)
        logp, ids = logp.double(), ids.long()
        if not c["tail"]:
            logp = torch.log_softmax(logp, 1)
        p = torch.exp(logp)
        loss = (p * (logp - logq.gather(1, ids))).sum(1)
        d = torch.zeros_like(logq)
        if c["tail"]:
            rest = (1.0 - p.sum(1)).clamp(min=0.0)
            inside = torch.zeros_like(logq, dtype=torch.bool).scatter_(1, ids, True)
            lout = torch.logsumexp(logq.masked_fill(inside, -math.inf), 1)
            loss = loss + torch.special.xlogy(rest, rest) - rest * lout
            d = torch.exp(logq - lout[:, None]).masked_fill(inside, 0.0) * -rest[:, None]
        d.scatter_(1, ids, -p)
        q = torch.exp(logq)
        losses.append(loss)
        grads.append((d - q * d.sum(1, keepdim=True)) * (w.double() / c["temp"])[:, None])
    return dict(loss=torch.cat(losses), grad=torch.cat(grads))


def _exact_tree(s):
    c = s["case"]
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    G = Hq // Hkv
    off, length = s["tree_off"].tolist(), s["cache_len"].tolist()
    up = s["parents"].tolist()
    outs, lses = [], []
    for b in range(c["B"]):
        lo, hi, L = off[b], off[b + 1], length[b]
        n = hi - lo
        at = torch.arange(L, device="cuda")
        page = s["page_table"][b].long()[at // c["page"]]
        keys, vals = (torch.cat([cache[page, at % c["page"]], new[lo:hi]]).double()
                      for cache, new in ((s["k_cache"], s["k"]), (s["v_cache"], s["v"])))
        sees = [[False] * n for _ in range(n)]
        for i in range(n):
            j = i
            while j >= 0:
                sees[i][j] = True
                j = up[lo + j]
        hidden = ~torch.cat([torch.ones((n, L), dtype=torch.bool), torch.tensor(sees)], 1).cuda()
        q = s["q"][lo:hi].double().view(n, Hkv, G, D)
        x = torch.einsum("nhgd,lhd->hgnl", q, keys) * D ** -0.5
        x = x.masked_fill(hidden, -math.inf)
        lse = torch.logsumexp(x, -1)
        x = torch.einsum("hgnl,lhd->nhgd", torch.exp(x - lse[..., None]), vals)
        outs.append(x.reshape(n, Hq, D))
        lses.append(lse.permute(2, 0, 1).reshape(n, Hq))
    return dict(out=torch.cat(outs), lse=torch.cat(lses))


def exact(case, seed):
    s = prepare(case, seed)
    return {"logprobs": _exact_logprobs, "distill": _exact_distill,
            "tree": _exact_tree}[case["op"]](s)
