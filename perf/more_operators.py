"""What a layer of the target model does around the attention of drafted tokens
when its paged cache is held in 8 bits, over the range of the framework's own
workloads:

* ``rope``: rotary positions of a layer's query and key heads -- for tokens that
  are scored, for prompts, and with the gradient for a draft that learns;
* ``append``: the keys and values that a verification step accepted, or a
  prompt's, into the requests' paged caches, keys rotated on the way or before;
* ``attn8``: attention of drafted tokens, or of single ones, over a cache of
  e4m3 elements with a power of two for each 16 slots and head.

An 8-bit element stands for its e4m3 value times 2^e, e that of the 16 slots of
its page and of its head. What a call writes is rounded to the nearest e4m3 value,
e being the least with which the largest element fits; slots in use whose e a
later call raises are rounded again.
"""
from __future__ import annotations

import math

import torch

own = False

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
GROUP = 16  # slots that share an exponent


def _ro(name, N, Hq, Hk, D, rot, dtype, layout, scaled, far, grad=False):
    """far: positions lie below it; scaled: frequencies by parts of the head for a
    context ``scaled`` times as long, 0 for none; grad: the gradient too."""
    return dict(name=name, op="rope", N=N, Hq=Hq, Hk=Hk, D=D, rot=rot, dtype=dtype, layout=layout,
                scaled=scaled, far=far, grad=grad)


def _ap(name, B, new, length, Hkv, D, page, dtype, held, form="all", rot=0, layout="half"):
    """new: most tokens that a request brings; length: longest cache before; held:
    "16" (the tokens' type) or "8"; form: every token ("all"), a request's first
    ones ("keep") or a path through its tree ("path"); rot: leading elements of a
    key that are rotated on the way."""
    return dict(name=name, op="append", B=B, new=new, length=length, Hkv=Hkv, D=D, page=page,
                dtype=dtype, held=held, form=form, rot=rot, layout=layout)


def _at(name, B, nodes, Hq, Hkv, D, length, page, dtype="bf16", ragged=True, chain=False):
    """nodes: most drafted tokens of a request; length: longest cache."""
    return dict(name=name, op="attn8", B=B, nodes=nodes, Hq=Hq, Hkv=Hkv, D=D, length=length,
                page=page, dtype=dtype, ragged=ragged, chain=chain)


def listed():
    return [
        # One interactive request's next token: latency.
        _ro("rope_one_token", 1, 32, 8, 128, 128, "bf16", "half", 0, 4096),
        # A batch of prompts at far positions of an extended context: bandwidth.
        _ro("rope_prompts", 16384, 32, 8, 128, 128, "bf16", "half", 8, 131072),
        # A draft's training batch: part of the head, pairs side by side, fp32, odd.
        _ro("rope_train_f32", 4095, 12, 12, 64, 32, "f32", "pairs", 0, 4095, grad=True),
        # One decoded token of every request into an 8-bit cache.
        _ap("append_decode8", 256, 1, 1024, 8, 128, 64, "bf16", "8", rot=128),
        # What a step accepted of the drafted tokens (rotated when they were scored).
        _ap("append_accepted", 64, 9, 1024, 8, 128, 64, "bf16", "16", form="keep"),
        # The accepted path of wide trees, 8 bits, fp16 and narrow heads.
        _ap("append_path8_f16", 16, 64, 515, 8, 64, 32, "f16", "8", form="path"),
        # Prompts of up to 8192 tokens into an empty 8-bit cache: bandwidth.
        _ap("append_prompts8", 8, 8192, 0, 8, 128, 64, "bf16", "8", rot=128),
        # One interactive request with a chain of four drafted tokens and the last one.
        _at("attn8_one_chain", 1, 5, 32, 8, 128, 1000, 16, ragged=False, chain=True),
        # Single tokens of many requests: plain decoding.
        _at("attn8_single_tokens", 256, 1, 32, 8, 128, 4096, 64, chain=True),
        # A serving batch: eight drafted tokens and the last one, ragged caches.
        _at("attn8_serving", 64, 9, 32, 8, 128, 8192, 64),
        # Two long documents with wide trees; few heads, so the cache is split.
        _at("attn8_long", 2, 32, 16, 2, 128, 131072, 128),
        # Wide trees over medium caches, narrow heads, fp16.
        _at("attn8_wide_f16", 16, 64, 32, 8, 64, 4096, 32, dtype="f16"),
    ]


# Bounds of drawn cases: the largest listed ones.
MOST_ROPE = 16384 * 40 * 128          # elements that are rotated
MOST_NEW = 8 * 8192 * 8 * 128         # elements of keys that are appended
MOST_OLD = 256 * 1024 * 8 * 128       # elements of a cache that is appended to
MOST_CACHE = 256 * 4096 * 8 * 128     # elements of a cache that is attended to
MOST_SCORES = 64 * 32 * 9 * 8192      # scores of the plain form


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "attn8"])
    dtype = rng.choice(["bf16", "f16"])
    G = rng.choice([1, 2, 3, 4, 5, 7, 8, 16])
    Hkv = rng.choice([1, 2, 4, 8])
    D = rng.choice([64, 128])
    page = rng.choice([16, 32, 48, 64, 128])
    layout = rng.choice(["half", "pairs"])
    if op == "rope":
        grad = rng.random() < 0.4
        D = rng.choice([64, 80, 96, 128, 256])
        N = _log(rng, 1, MOST_ROPE // ((G + 1) * Hkv * D * (4 if grad else 2)))
        c = _ro("", N, G * Hkv, Hkv, D, rng.choice([D, D, D // 2, D // 4, 2 * rng.randint(1, D // 2)]),
                rng.choice([dtype, "f32"]), layout, rng.choice([0, 0, 4, 8.5, 32]),
                _log(rng, 16, 1 << 20), grad)
    elif op == "append":
        B = _log(rng, 1, 256)
        form = rng.choice(["all", "all", "keep", "path"])
        new = _log(rng, 1, min(8192 if form == "all" else 512, MOST_NEW // (B * Hkv * D)))
        length = _log(rng, 1, min(8192, MOST_OLD // (B * Hkv * D))) - 1
        c = _ap("", B, new, length, Hkv, D, page, dtype, rng.choice(["8", "8", "16"]), form,
                rng.choice([0, D, D, D // 2, 2 * rng.randint(1, D // 2)]), layout)
    else:
        nodes = _log(rng, 1, 64)
        B = _log(rng, 1, 256)
        room = min(MOST_CACHE // (B * Hkv * D), MOST_SCORES // (B * G * Hkv * nodes), 131072)
        c = _at("", B, nodes, G * Hkv, Hkv, D, _log(rng, 16, max(17, room)), page, dtype,
                ragged=rng.random() < 0.75, chain=rng.random() < 0.3)
    del c["name"]
    return c


# ------------------------------------------------------------------- inputs

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BASE = 500000.0
ORIGINAL, LOW, HIGH = 8192.0, 1.0, 4.0  # the context before scaling, and the parts' ends in turns


def _freqs(rot, scaled):
    """Angles per position of the rotated pairs, fp64: base^(-2 i / rot); scaled by
    parts: pairs that turn fewer than LOW times within the original context are
    slowed by the factor, those with more than HIGH turns are left, a ramp between."""
    f = [BASE ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaled:
        for i, x in enumerate(f):
            ramp = min(1.0, max(0.0, (ORIGINAL * x / (2 * math.pi) - LOW) / (HIGH - LOW)))
            f[i] = x * ((1.0 - ramp) / scaled + ramp)
    return f


def _plan(rot, scaled):
    """The frequencies, and as turns per position in 64-bit fractions of a turn."""
    f = _freqs(rot, scaled)
    turns = [int(round(x / (2 * math.pi) * 2.0 ** 64)) % 2 ** 64 for x in f]
    signed = [t - 2 ** 64 if t >= 2 ** 63 else t for t in turns]
    return dict(freqs=torch.tensor(f, dtype=torch.float64, device="cuda"),
                turns=torch.tensor(signed, dtype=torch.int64, device="cuda"))


def _ints(gen, lo, hi, size):
    return torch.randint(lo, hi, size, generator=gen, device="cuda")


def _heads(gen, size, dtype):
    """Heads as a projection leaves them: some elements of a head are much larger
    than others in every token."""
    loud = torch.exp(0.7 * torch.randn(size[-2:], generator=gen, device="cuda"))
    return (torch.randn(size, generator=gen, device="cuda") * loud).to(dtype)


def _prepare_rope(c, gen):
    N, Hq, Hk, D = c["N"], c["Hq"], c["Hk"], c["D"]
    # (one projection's output: keys lie behind the queries, values behind them)
    x = _heads(gen, (N, Hq + 2 * Hk, D), DTYPES[c["dtype"]])
    s = dict(_plan(c["rot"], c["scaled"]), q=x[:, :Hq], k=x[:, Hq:Hq + Hk],
             positions=_ints(gen, 0, c["far"], (N,)).int())
    if c["grad"]:
        s["up_q"], s["up_k"] = _heads(gen, (N, Hq, D), x.dtype), _heads(gen, (N, Hk, D), x.dtype)
    return s


def _counts(B, most, ragged):
    """From half of the most to the most; how many a request has goes by the case alone."""
    low = max(1, most // 2)
    return most - torch.arange(B, device="cuda") * 7 % (most - low + 1 if ragged else 1)


def _offsets(counts):
    return torch.cat([counts.new_zeros(1), counts.cumsum(0)])


def _tables(gen, B, slots, page):
    P = max(1, (slots + page - 1) // page)
    pages = B * P + 3
    return torch.randperm(pages, generator=gen, device="cuda")[:B * P].view(B, P).int(), pages


def _exponents(x):
    """The least e with x <= 448 2^e (448 = 0.875 2^9), within what 8 bits hold."""
    m, e = torch.frexp(x)
    return torch.where(x > 0, e - 9 + (m > 0.875).int(), -126).clamp(-126, 127)


def _power(e, dtype=torch.float32):
    return torch.ldexp(torch.ones(e.shape, dtype=dtype, device=e.device), e)


def _cache8(gen, pages, page, Hkv, D, dtype):
    """A cache that holds random heads: elements and exponents."""
    held = torch.empty((pages, page, Hkv, D), dtype=E4M3, device="cuda")
    codes = torch.empty((pages, page // GROUP, Hkv), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 27) // (page * Hkv * D))
    for p in range(0, pages, step):
        n = min(step, pages - p)
        x = _heads(gen, (n, page // GROUP, GROUP, Hkv, D), dtype).float()
        e = _exponents(x.abs().amax((2, 4)))
        held[p:p + n] = (x * _power(-e)[:, :, None, :, None]).view(n, page, Hkv, D).to(E4M3)
        codes[p:p + n] = (e + 127).to(torch.uint8)
    return held, codes.view(E8M0)


def _prepare_append(c, gen):
    B, n, Hkv, D, page = c["B"], c["new"], c["Hkv"], c["D"], c["page"]
    dt = DTYPES[c["dtype"]]
    counts = _counts(B, n, n > 1)
    off = _offsets(counts)
    N = int(off[-1])
    length = _ints(gen, 0, c["length"] + 1, (B,))
    length[0] = c["length"]
    table, pages = _tables(gen, B, c["length"] + n, page)
    x = _heads(gen, (N, 2 * Hkv, D), dt)
    s = dict(k=x[:, :Hkv], v=x[:, Hkv:], page_table=table, cache_len=length.int(),
             token_off=off.int(), keep=None, path=None)
    if c["rot"]:
        s.update(_plan(c["rot"], 0))
    for name in ("k", "v"):
        if c["held"] == "8":
            s[name + "_cache"], s[name + "_scale"] = _cache8(gen, pages, page, Hkv, D, dt)
        else:
            s[name + "_cache"] = _heads(gen, (pages * page, Hkv, D), dt).view(pages, page, Hkv, D)
            s[name + "_scale"] = None
    if c["form"] != "all":  # (the last token is always kept, as by a step)
        s["keep"] = (1 + (torch.rand(B, generator=gen, device="cuda") * counts).long()).int()
    if c["form"] == "path":  # tokens of the tree in order, the first among them
        req = torch.repeat_interleave(torch.arange(B, device="cuda"), counts)
        key = torch.rand(N, generator=gen, device="cuda")
        at = torch.arange(N, device="cuda") - off[req]
        key[off[:-1]] = -1.0
        rank = torch.argsort(torch.argsort(key + 2 * req)) - off[req]
        taken = rank < s["keep"][req]
        s["path"] = (torch.argsort(at + 2 * N * req + N * ~taken) - off[req]).int()
    return s


def _prepare_attn8(c, gen):
    B, n, Hq, Hkv, D, page = c["B"], c["nodes"], c["Hq"], c["Hkv"], c["D"], c["page"]
    dt = DTYPES[c["dtype"]]
    counts = _counts(B, n, c["ragged"])
    length = _ints(gen, 0, c["length"] + 1, (B,)) if c["ragged"] else torch.full((B,), c["length"], device="cuda")
    length[0] = c["length"]
    off = _offsets(counts)
    N = int(off[-1])
    req = torch.repeat_interleave(torch.arange(B, device="cuda"), counts)
    node = torch.arange(N, device="cuda") - off[req]
    up = node - 1
    if not c["chain"]:  # a node's parent: any of the few before it
        up = torch.minimum(torch.clamp(node - 1 - _ints(gen, 0, 4, (N,)), min=0), up)
    table, pages = _tables(gen, B, c["length"], page)
    kc, ks = _cache8(gen, pages, page, Hkv, D, dt)
    vc, vs = _cache8(gen, pages, page, Hkv, D, dt)
    randn = lambda h: torch.randn((N, h, D), generator=gen, device="cuda").to(dt)  # noqa: E731
    return dict(q=randn(Hq), k=randn(Hkv), v=randn(Hkv), k_cache=kc, v_cache=vc, k_scale=ks,
                v_scale=vs, page_table=table, cache_len=length.int(), tree_off=off.int(),
                parents=up.int())


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"rope": _prepare_rope, "append": _prepare_append,
         "attn8": _prepare_attn8}[case["op"]](case, gen)
    return dict(s, case=dict(case))


# -------------------------------------------------------------- plain forms

def _turned(x, angle, layout, back=False):
    """x [N, H, D] with its leading pairs turned by angle [N, pairs] (or back by
    it); the angles are 64-bit: far positions."""
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if back:
        sin = -sin
    n = angle.shape[1]
    x = x.float()
    head, rest = x[..., :2 * n], x[..., 2 * n:]
    if layout == "half":
        a, b = head[..., :n], head[..., n:]
        head = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = head[..., ::2], head[..., 1::2]
        head = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([head, rest], -1)


def _plain_rope(s):
    c = s["case"]
    angle = s["positions"].double()[:, None] * s["freqs"]
    out = {x: _turned(s[x], angle, c["layout"]).to(s[x].dtype) for x in ("q", "k")}
    if c["grad"]:
        out.update({"grad_" + x: _turned(s["up_" + x], angle, c["layout"], True).to(s[x].dtype)
                    for x in ("q", "k")})
    return out


def _kept(s):
    """Of the tokens that are appended: request, number among its kept ones, row."""
    off = s["token_off"].long()
    N = s["k"].shape[0]
    row = torch.arange(N, device=off.device)
    req = torch.searchsorted(off, row, right=True) - 1
    at = row - off[req]
    if s["keep"] is not None:
        there = at < s["keep"][req]
        req, at, row = req[there], at[there], row[there]
    return req, at, row if s["path"] is None else off[req] + s["path"][row]


def _plain_append(s):
    c = s["case"]
    req, at, row = _kept(s)
    slot = s["cache_len"].long()[req] + at
    page = s["page_table"].long()[req, slot // c["page"]]
    k, v = s["k"][row].float(), s["v"][row].float()
    if c["rot"]:
        k = _turned(k, slot.double()[:, None] * s["freqs"], c["layout"])
    out = {}
    for name, x in (("k", k), ("v", v)):
        cache, scale = s[name + "_cache"], s[name + "_scale"]
        if scale is None:
            cache[page, slot % c["page"]] = x.to(cache.dtype)
        else:
            _append8(s, cache, scale.view(torch.uint8), x, req, at, slot, page)
            out[name + "_scale"] = scale
        out[name + "_cache"] = cache
    return out


def _append8(s, cache, codes, x, req, at, slot, page):
    """Appends x, at slots of pages, to the e4m3 elements `cache` and the exponents
    `codes` (those and 127)."""
    Hkv, D, per = cache.shape[2], cache.shape[3], s["case"]["page"]
    length = s["cache_len"].long()
    # the groups of slots that are written to, in order of their requests
    first = (at == 0) | (slot % GROUP == 0)
    group = first.cumsum(0) - 1
    of, where = page[first], slot[first] % per // GROUP
    n = of.shape[0]
    limit = 61440.0 if s["k"].dtype == torch.float16 else 1.875 * 2.0 ** 127
    x = x.clamp(-limit, limit)
    top = torch.zeros((n, Hkv), device=x.device).scatter_reduce_(
        0, group[:, None].expand(-1, Hkv), x.abs().amax(2), "amax")
    old = codes[of, where].int() - 127
    used = torch.where(at[first] == 0, length[req[first]] % GROUP, 0)  # slots in use before
    e = _exponents(top)
    e = torch.where(used[:, None] > 0, torch.maximum(e, old), e)
    slots = where[:, None] * GROUP + torch.arange(GROUP, device=x.device)
    held = cache[of[:, None], slots].float() * _power(old - e)[:, None, :, None]
    before = torch.arange(GROUP, device=x.device) < used[:, None]
    there = before.nonzero(as_tuple=True)
    cache[of[there[0]], slots[there]] = held[there].to(E4M3)
    cache[page, slot % per] = (x * _power(-e)[group][:, :, None]).to(E4M3)
    codes[of, where] = (e + 127).to(torch.uint8)


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


def _plain_attn8(s):
    c = s["case"]
    B, n, Hq, Hkv, D = c["B"], c["nodes"], c["Hq"], c["Hkv"], c["D"]
    at, there = _padded(s)
    L = c["length"]
    table = s["page_table"].long()
    seen = torch.cat([(torch.arange(L, device=at.device) < s["cache_len"][:, None])[:, None]
                      .expand(B, n, L), _ancestors(s, at, there)], 2)  # [B, n, L + n]
    used = seen.any(1)[:, None, :, None]

    def heads(cache, scale, new):  # [B, Hkv, L + n, D]
        old = cache.view(torch.uint8)[table].view(E4M3).float()
        power = _power(scale.view(torch.uint8)[table].int() - 127)
        old = old.view(B, -1, GROUP, Hkv, D).mul_(power.view(B, -1, 1, Hkv, 1))
        old = old.view(B, -1, Hkv, D)[:, :L]
        x = torch.cat([old, new[at].float()], 1).transpose(1, 2)
        return torch.where(used, x, 0.0)

    q = s["q"][at].float().view(B, n, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4)
    k = heads(s["k_cache"], s["k_scale"], s["k"])
    score = (q.reshape(B, Hkv, -1, D) @ k.transpose(2, 3)).view(B, Hkv, Hq // Hkv, n, L + n)
    del k
    score = torch.where(seen[:, None, None], score / math.sqrt(D), -math.inf)
    top = score.amax(-1, keepdim=True)
    e = torch.exp(score.sub_(top))
    S = e.sum(-1, keepdim=True)
    x = e.view(B, Hkv, -1, L + n) @ heads(s["v_cache"], s["v_scale"], s["v"])
    x = x.view(B, Hkv, Hq // Hkv, n, D) / S
    lse = (top + torch.log(S))[..., 0]
    return dict(out=x.permute(0, 3, 1, 2, 4)[there].reshape(-1, Hq, D).to(s["q"].dtype),
                lse=lse.permute(0, 3, 1, 2)[there].reshape(-1, Hq))


# -------------------------------------------------------- the framework's own

def _own(s):
    from paper_2510_15545_gb300 import binding as tt
    c = s["case"]
    if c["op"] == "rope":
        pairs = c["layout"] == "pairs"
        if not c["grad"]:
            o = tt.tt_rope(s["q"], s["k"], s["positions"], s["turns"], interleaved=pairs)
            return dict(q=o["q"], k=o["k"])
        leaves = [s[x].detach().requires_grad_() for x in ("q", "k")]
        q, k = tt.rope(*leaves, s["positions"], s["turns"], interleaved=pairs)
        grads = torch.autograd.grad((q, k), leaves, (s["up_q"], s["up_k"]))
        return dict(q=q.detach(), k=k.detach(), grad_q=grads[0], grad_k=grads[1])
    if c["op"] == "append":
        tt.tt_cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["page_table"],
                           s["cache_len"], s["token_off"], k_scale=s["k_scale"],
                           v_scale=s["v_scale"], keep=s["keep"], path=s["path"],
                           turns=s["turns"] if c["rot"] else None,
                           interleaved=c["layout"] == "pairs", max_new=c["new"])
        return {x: s[x] for x in ("k_cache", "v_cache", "k_scale", "v_scale") if s[x] is not None}
    o = tt.tt_tree_attn(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["page_table"],
                        s["cache_len"], s["tree_off"], s["parents"], k_scale=s["k_scale"],
                        v_scale=s["v_scale"], max_len=c["length"], max_nodes=c["nodes"])
    return dict(out=o["out"], lse=o["lse"])


def run(state):
    if own:
        return _own(state)
    return {"rope": _plain_rope, "append": _plain_append,
            "attn8": _plain_attn8}[state["case"]["op"]](state)


# --------------------------------------------------------------------- work

def _mean_count(most, B):
    low = max(1, most // 2)
    return (most + (B - 1) * (low + most) / 2) / B if most > 1 else 1.0


def work(case):
    """Each input that is used read once, each output written once."""
    c = case
    if c["op"] == "rope":
        esz = 4 if c["dtype"] == "f32" else 2
        cells = c["N"] * (c["Hq"] + c["Hk"]) * c["D"]
        passes = 2 if c["grad"] else 1
        turned = cells * c["rot"] // c["D"]
        return {"bytes": passes * (2 * esz * cells + 4 * c["N"]), "flops": passes * 3 * turned}
    if c["op"] == "append":
        n = _mean_count(c["new"], c["B"])
        if c["form"] != "all":
            n = (1 + n) / 2
        cells = 2 * c["B"] * n * c["Hkv"] * c["D"]
        held = 1 if c["held"] == "8" else 2
        return {"bytes": (2 + held) * cells, "flops": cells * (2 if c["held"] == "8" else 1)}
    B, n, L = c["B"], c["nodes"], c["length"]
    if c["ragged"]:
        n, L = _mean_count(n, B), (L + (B - 1) * L / 2) / B
    cache = B * L * c["Hkv"] * (2 * c["D"] + 2 / GROUP)
    new = B * n * c["D"] * 2 * (2 * c["Hq"] + 2 * c["Hkv"])
    return {"bytes": cache + new + 4 * B * n * c["Hq"],
            "flops": 4 * B * n * c["Hq"] * c["D"] * (L + (n + 1) / 2)}


# ------------------------------------------------------ the same in 64 bits

def _exact_turn(x, at, freqs, layout, sign=1.0):
    """The pairs as complex numbers, times e^(i angle)."""
    x = x.double()
    n = freqs.shape[0]
    z = torch.polar(torch.ones((), dtype=torch.float64, device=x.device).expand(at.shape[0], n),
                    sign * at.double()[:, None] * freqs)[:, None]
    out = x.clone()
    a, b = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    y = torch.complex(x[..., a], x[..., b]) * z
    out[..., a], out[..., b] = y.real, y.imag
    return out


def _exact_rope(s):
    c = s["case"]
    out = {x: _exact_turn(s[x], s["positions"], s["freqs"], c["layout"]) for x in ("q", "k")}
    if c["grad"]:
        out.update({"grad_" + x: _exact_turn(s["up_" + x], s["positions"], s["freqs"], c["layout"], -1.0)
                    for x in ("q", "k")})
    return out


def _exact_append(s):
    """The caches with what is appended as it is before it is rounded; in 8 bits, in
    units of the group's power of two."""
    c = s["case"]
    off, length = s["token_off"].tolist(), s["cache_len"].tolist()
    keep = None if s["keep"] is None else s["keep"].tolist()
    out = {}
    for name in ("k", "v"):
        cache, scale = s[name + "_cache"].double(), s[name + "_scale"]
        code = None if scale is None else scale.view(torch.uint8).int() - 127
        for b in range(c["B"]):
            n = off[b + 1] - off[b] if keep is None else keep[b]
            rows = torch.arange(off[b], off[b] + n, device="cuda")
            if s["path"] is not None:
                rows = off[b] + s["path"][rows].long()
            slots = length[b] + torch.arange(n, device="cuda")
            x = s[name][rows].double()
            if name == "k" and c["rot"]:
                x = _exact_turn(x, slots, s["freqs"], c["layout"])
            page, at = s["page_table"][b].long()[slots // c["page"]], slots % c["page"]
            if scale is None:
                cache[page, at] = x
                continue
            # the groups from the first slot's on, as [groups, 16 slots, heads, D] in units of 1
            g0 = length[b] // GROUP
            groups = (length[b] + n + GROUP - 1) // GROUP - g0
            g = g0 + torch.arange(groups, device="cuda")
            of, where = s["page_table"][b].long()[g * GROUP // c["page"]], g % (c["page"] // GROUP)
            lead = length[b] - g0 * GROUP
            new = torch.zeros((groups * GROUP, c["Hkv"], c["D"]), dtype=torch.float64, device="cuda")
            new[lead:lead + n] = x
            top = new.view(groups, GROUP, c["Hkv"], c["D"]).abs().amax((1, 3))
            e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -150) / 448))
            # (the logarithm may be rounded past a whole number)
            e = torch.where(top <= 448 * torch.exp2(e - 1), e - 1, e)
            e = torch.where(top > 448 * torch.exp2(e), e + 1, e).clamp(-126, 127).int()
            if lead:
                e[0] = torch.maximum(e[0], code[of[0], where[0]])
                old = slice(int(where[0]) * GROUP, int(where[0]) * GROUP + lead)
                cache[of[0], old] *= _power(code[of[0], where[0]] - e[0], torch.float64)[:, None]
            cache[page, at] = x * _power(-e, torch.float64)[(slots // GROUP) - g0][:, :, None]
            code[of, where] = e
        out[name + "_cache"] = cache
        if scale is not None:
            out[name + "_scale"] = _power(code, torch.float64)
    return out


def _exact_attn8(s):
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
        page, slot = s["page_table"][b].long()[at // c["page"]], at % c["page"]
        keys, vals = (
            torch.cat([cache.view(torch.uint8)[page, slot].view(E4M3).double()
                       * torch.exp2(scale.view(torch.uint8)[page, slot // GROUP].double() - 127)[..., None],
                       new[lo:hi].double()])
            for cache, scale, new in ((s["k_cache"], s["k_scale"], s["k"]),
                                      (s["v_cache"], s["v_scale"], s["v"])))
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
    return {"rope": _exact_rope, "append": _exact_append,
            "attn8": _exact_attn8}[case["op"]](s)
