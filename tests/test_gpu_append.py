"""tt_cache_append against its definition: whole caches and scales, every slot that is
not written among them, bit by bit. Values that are not rotated are numbers of 16
bits, which a power of two scales exactly, so the e4m3 value nearest to each is one;
keys that are rotated are held against tt_rope's, in fp32 where the cache has 8 bits
(whose own tests hold those against 64 bits), and against the 64-bit rotation within
half a step: 2^-4 of the value, 2^-10 of the scale below its normal range, and what
the rotation may be off, 2^-21 of the pair's sizes."""
import math

import pytest
import torch

import paper_2510_15545_gb300 as tt
from paper_2510_15545_gb300 import binding

pytestmark = pytest.mark.gpu

H, E = torch.bfloat16, torch.float16
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
LIMIT = {E: 61440.0, H: 1.875 * 2.0 ** 127}
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    tt.load(build_if_missing=True)


def i32(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


def power(code):
    """2^(code - 127) in 64 bits, NaN for 255."""
    return torch.where(code == 255, NAN, torch.exp2(code.double() - 127))


def codes_for(top):
    """The least code from 1 on with top <= 448 2^(code - 127)."""
    m, e = torch.frexp(top)
    return torch.where(top > 0, e - 9 + (m > 0.875).int() + 127, 1).clamp(min=1)


def rounded(x):
    """The nearest e4m3 values (of at most 448), as bytes; NaN has one code here."""
    y = x.float().to(E4M3).view(torch.uint8)
    return torch.where(torch.isnan(x), 0x7f, y)


class Case:
    """Requests that bring `news` tokens behind `lens` slots. Caches hold random
    elements everywhere, in use or not."""

    def __init__(self, lens, news, Hkv=2, D=64, page=16, dtype=H, held="8", seed=0, room=0, size=1.0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.gen, self.lens, self.news, self.page, self.dtype, self.held = gen, lens, news, page, dtype, held
        B, N = len(lens), sum(news)
        randn = lambda *s: torch.randn(s, generator=gen, device="cuda") * size  # noqa: E731
        x = randn(N, 2 * Hkv, D).to(dtype)
        self.k, self.v = x[:, :Hkv], x[:, Hkv:]
        per = max(1, max(((a + b + room + page - 1) // page for a, b in zip(lens, news)), default=1))
        pages = B * per + 2
        self.table = torch.randperm(pages, generator=gen, device="cuda")[:B * per].view(B, per).int()
        self.off = [sum(news[:b]) for b in range(B + 1)]
        self.scale = {}
        self.cache = {}
        for name in "kv":
            if held == "8":
                # (bytes of every finite value)
                y = torch.randint(0, 256, (pages, page, Hkv, D), generator=gen, device="cuda").byte()
                self.cache[name] = torch.where((y & 0x7f) == 0x7f, 0, y).byte().view(E4M3)
                self.scale[name] = torch.randint(110, 128, (pages, page // 16, Hkv), generator=gen,
                                                 device="cuda").byte().view(E8M0)
            else:
                self.cache[name] = randn(pages, page, Hkv, D).to(dtype)
        self.keep = self.path = self.positions = self.turns = None
        self.interleaved, self.mscale = False, 1.0

    def rotate(self, rot, interleaved=False, mscale=1.0, positions=None):
        self.turns = tt.rope_turns(tt.rope_freqs(rot))
        self.interleaved, self.mscale, self.positions = interleaved, mscale, positions
        return self

    def choose(self, keep=None, path=None):
        self.keep, self.path = keep, path
        return self

    def call(self, **kw):
        more = {} if self.held != "8" else dict(k_scale=self.scale["k"], v_scale=self.scale["v"])
        more.update(kw)
        o = tt.tt_cache_append(self.k, self.v, self.cache["k"], self.cache["v"], self.table, i32(self.lens),
                               i32(self.off), keep=i32(self.keep), path=i32(self.path), turns=self.turns,
                               positions=i32(self.positions), interleaved=self.interleaved,
                               mscale=self.mscale, **more)
        torch.cuda.synchronize()
        return o

    def rows(self, b):
        """The batch's rows that request b appends, and the slots they go to."""
        n = self.news[b] if self.keep is None else self.keep[b]
        lo = self.off[b]
        rows = [lo + (i if self.path is None else self.path[lo + i]) for i in range(n)]
        return (torch.tensor(rows, dtype=torch.long, device="cuda"),
                torch.arange(self.lens[b], self.lens[b] + n, device="cuda"))

    def expected(self, only=None):
        """Caches and scales after the call, and of 8 bits the exact values too."""
        want = {x: c.clone() for x, c in self.cache.items()}
        codes = {x: c.view(torch.uint8).clone() for x, c in self.scale.items()}
        for b in range(len(self.lens)) if only is None else only:
            rows, slots = self.rows(b)
            if not len(rows):
                continue
            page, at = self.table[b].long()[slots // self.page], slots % self.page
            for name, x in (("k", self.k[rows]), ("v", self.v[rows])):
                if name == "k" and self.turns is not None:
                    pos = slots.int() if self.positions is None else i32(self.positions)[rows]
                    x = x.float() if self.held == "8" else x.contiguous()
                    x = tt.tt_rope(x, None, pos, self.turns, interleaved=self.interleaved,
                                   mscale=self.mscale)["q"]
                if self.held != "8":
                    want[name][page, at] = x
                    continue
                bytes_ = want[name].view(torch.uint8)
                x = torch.where(torch.isfinite(x), x.double().clamp(-LIMIT[self.dtype], LIMIT[self.dtype]), NAN)
                size = torch.where(torch.isnan(x), 0.0, x.abs())
                for g in range(self.lens[b] // 16, (int(slots[-1])) // 16 + 1):
                    p, y = int(self.table[b, g * 16 // self.page]), g % (self.page // 16)
                    mine = slots // 16 == g
                    code = codes_for(size[mine].amax((0, 2)))
                    lead = max(0, self.lens[b] - g * 16)
                    old = codes[name][p, y].int()
                    if lead:
                        code = torch.where(old == 255, code, torch.maximum(code, old))
                        s = slice(y * 16, y * 16 + lead)
                        before = bytes_[p, s].view(E4M3).double() * (power(old) / power(code))[:, None]
                        bytes_[p, s] = torch.where((code != old)[:, None], rounded(before), bytes_[p, s])
                    bytes_[p, at[mine]] = rounded(x[mine] / power(code)[:, None])
                    codes[name][p, y] = code.byte()
        return want, codes

    def check(self, **kw):
        want, codes = self.expected()
        o = self.call(**kw)
        kept = self.news if self.keep is None else self.keep
        assert o["status"][:len(self.lens)].tolist() == [0] * len(self.lens)
        assert o["new_len"][:len(self.lens)].tolist() == [a + b for a, b in zip(self.lens, kept)]
        self.same(want, codes)
        return o

    def same(self, want, codes):
        for name in "kv":
            if self.held == "8":
                assert torch.equal(self.scale[name].view(torch.uint8), codes[name]), name
                got, y = (c.view(torch.uint8) for c in (self.cache[name], want[name]))
                both = ((got & 0x7f) == 0x7f) & ((y & 0x7f) == 0x7f)  # NaN of either sign
                bad = (got != y) & ~both
            else:
                bad = self.cache[name].view(torch.int16) != want[name].view(torch.int16)
            assert not bad.any(), (name, bad.nonzero()[:4].tolist())


LENS = [0, 1, 2, 7, 15, 16, 17, 31, 32, 33, 47, 48, 63, 64, 65, 100, 127, 128]
NEWS = [0, 1, 2, 3, 14, 15, 16, 17, 18, 31, 32, 33, 48, 50, 64, 65, 100, 130]


@pytest.mark.parametrize("held", ["8", "16"])
@pytest.mark.parametrize("dtype", [H, E])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 48, 64])
def test_lengths(held, dtype, D, page):
    """Every length with several numbers of new tokens."""
    for shift in (0, 5, 11):
        news = NEWS[shift:] + NEWS[:shift]
        Case(LENS, news, 2, D, page, dtype, held, seed=shift).check()


@pytest.mark.parametrize("held", ["8", "16"])
@pytest.mark.parametrize("Hkv", [1, 2, 3, 4, 5, 7, 8, 9, 16, 20])
def test_heads(held, Hkv):
    for D in (64, 128):
        Case([0, 20, 37, 64], [40, 1, 29, 0], Hkv, D, 32, H, held, seed=Hkv).rotate(D).check()


@pytest.mark.parametrize("held", ["8", "16"])
@pytest.mark.parametrize("dtype", [H, E])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(64, 64), (64, 2), (64, 16), (64, 50), (128, 128), (128, 64),
                                   (128, 96), (128, 126), (128, 10)])
def test_rotations(held, dtype, interleaved, D, rot):
    c = Case([0, 5, 30, 100], [33, 1, 20, 16], 3, D, 32, dtype, held, seed=rot)
    c.rotate(rot, interleaved, mscale=1.2).check()
    c = Case([3, 16], [9, 40], 1, D, 16, dtype, held, seed=rot + 1)
    c.rotate(rot, interleaved, positions=[(7919 * i) % 200000 - 1000 for i in range(49)]).check()


def test_rotated_keys_against_64_bits():
    for dtype in (H, E):
        c = Case([0, 5], [100, 60], 4, 128, 64, dtype, seed=3).rotate(128)
        c.call()
        for b in range(2):
            rows, slots = c.rows(b)
            angle = (slots[:, None] * c.turns).double() * (2 * math.pi / 2.0 ** 64)
            cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
            a, d = c.k[rows, :, :64].double(), c.k[rows, :, 64:].double()
            want = torch.cat([a * cos - d * sin, a * sin + d * cos], 2)
            sizes = (a.abs() + d.abs()).repeat(1, 1, 2)
            page, at = c.table[b].long()[slots // 64], slots % 64
            scale = power(c.scale["k"].view(torch.uint8)[page, at // 16].int())[..., None]
            got = c.cache["k"].view(torch.uint8)[page, at].view(E4M3).double() * scale
            bound = want.abs() * 2.0 ** -4 + scale * 2.0 ** -10 + sizes * 2.0 ** -20
            assert ((got - want).abs() <= bound).all()


@pytest.mark.parametrize("held", ["8", "16"])
def test_accepted_tokens(held):
    """What a step keeps: first tokens of each request, none and all among them."""
    news = [5, 9, 1, 9, 4, 20]
    c = Case([0, 100, 16, 31, 7, 250], news, 8, 128, 64, H, held, seed=4)
    c.choose(keep=[3, 0, 1, 9, 2, 17]).check()


@pytest.mark.parametrize("held", ["8", "16"])
def test_accepted_branches(held):
    """Paths through trees; what the path says behind the kept ones does not matter."""
    c = Case([0, 40, 15], [6, 64, 3], 4, 64, 32, E, held, seed=5)
    path = [0, 2, 5, 99, -1, 7] + [0, 3, 4, 10, 20, 33, 60, 63] + [1 << 30] * 56 + [2, 2, 0]
    c.choose(keep=[3, 8, 3], path=path).rotate(64, True).check()
    c = Case([0, 40], [6, 4], 4, 64, 32, E, held, seed=5)
    c.choose(path=[5, 4, 3, 2, 1, 0, 3, 3, 3, 3]).check()  # (all kept, in another order)


def test_scales_that_rise_and_stay():
    """Slots in use are rounded again where new ones are larger, and only there."""
    for sizes in ([1e-3, 1.0, 100.0], [100.0, 1.0, 1e-3], [1.0, 0.0, 3e4]):
        c = Case([0, 0, 0], [5, 5, 5], 3, 64, 16, H, seed=6, room=32)
        for size in sizes:
            c.k = (torch.randn((15, 3, 64), generator=c.gen, device="cuda") * size).to(H)
            c.v = (torch.randn((15, 3, 64), generator=c.gen, device="cuda") * size).to(H)
            o = c.check()
            c.lens = o["new_len"].tolist()


@pytest.mark.parametrize("old", [0, 1, 2, 100, 127, 150, 253, 254, 255])
def test_every_old_scale(old):
    c = Case([7, 8, 20], [3, 12, 1], 2, 64, 16, H, seed=7)
    for name in "kv":
        c.scale[name].view(torch.uint8).fill_(old)
    c.check()


@pytest.mark.parametrize("dtype", [H, E])
def test_extreme_elements(dtype):
    """Zeros, the least and the largest numbers of the type, infinities and NaN: a
    group's scale comes from what is finite, what is not is NaN."""
    top = torch.finfo(dtype).max
    least = {H: 2.0 ** -133, E: 2.0 ** -24}[dtype]
    for special in ([0.0], [-0.0, 0.0], [least], [least, -3 * least], [top], [-top, 1.0], [INF, 1.0],
                    [-INF, NAN, 2.0], [NAN], [INF], [448.0], [449.0, 464.0, 465.0, 480.0], [1.75, 1.76]):
        c = Case([0, 3], [16, 20], 2, 64, 16, dtype, seed=8)
        for x in (c.k, c.v):
            x.zero_()
            for i, y in enumerate(special):
                x[i::7, :, i::5] = y
        c.check()


def test_requests_that_fail_leave_the_others_alone():
    c = Case([0, 10, 20, 30, 40], [4, 4, 4, 4, 4], 2, 64, 16, H, seed=9)
    good = [0, 4]
    want, codes = c.expected(good)
    c.keep = [4, 5, -1, 4, 4]      # beyond its tokens, negative
    c.lens = [0, 10, 20, -3, 40]
    o = c.call()
    assert o["status"].tolist() == [0, 8, 8, 2, 0]
    assert o["new_len"].tolist() == [4, 10, 20, -3, 44]
    c.same(want, codes)
    # offsets that fall, or end behind the tokens
    c = Case([0, 10, 20], [4, 4, 4], 2, 64, 16, H, seed=10)
    for off, status in (([0, 8, 4, 12], [0, 8, 0]), ([0, 4, 8, 13], [0, 0, 8]), ([-1, 4, 8, 12], [8, 0, 0])):
        c = Case([0, 10, 20], [4, 4, 4], 2, 64, 16, H, seed=10)
        c.off, c.news = off, [max(0, b - a) for a, b in zip(off, off[1:])]
        c.table = torch.arange(9, dtype=torch.int32, device="cuda").view(3, 3) % c.cache["k"].shape[0]
        c.table[:, 2] = 5
        c.lens = [0, 10, 12]
        want, codes = c.expected([b for b in range(3) if not status[b]])
        assert c.call(max_new=12)["status"].tolist() == status
        c.same(want, codes)


def test_lengths_and_tokens_beyond_their_bounds():
    c = Case([0, 10, 20], [4, 4, 7], 2, 64, 16, H, seed=11)
    want, codes = c.expected([0])
    o = c.call(max_len=13)
    assert o["status"].tolist() == [0, 2, 2] and o["new_len"].tolist() == [4, 10, 20]
    c.same(want, codes)
    want, codes = c.expected([0, 1])
    o = c.call(max_new=4)
    assert o["status"].tolist() == [0, 0, 2]
    c.same(want, codes)


def test_entries_out_of_range_are_left_out():
    c = Case([0, 10, 20], [4, 4, 4], 2, 64, 16, H, seed=12)
    c.path = [0, 1, 2, 3, 0, 4, -1, 3, 0, 1, 2, 3]
    whole, news = c.path, c.news
    # (request 1 without its two bad tokens: what the others get is the same)
    want, codes = c.expected([0, 2])
    before = {x: y.clone() for x, y in c.cache.items()}
    o = c.call()
    assert o["status"].tolist() == [0, 1, 0] and o["new_len"].tolist() == [4, 10, 24]
    p = int(c.table[1, 0])
    for name in "kv":
        got = c.cache[name].view(torch.uint8)
        assert torch.equal(got[p, 11:13], before[name].view(torch.uint8)[p, 11:13])
        others = torch.arange(got.shape[0], device="cuda") != p
        assert torch.equal(got[others], want[name].view(torch.uint8)[others])
    # pages
    c = Case([0, 10, 20], [4, 4, 4], 2, 64, 16, H, seed=12)
    want, codes = c.expected([0, 2])
    for page in (-1, c.cache["k"].shape[0], 1 << 30):
        c.table[1, 0] = page
        o = c.call()
        assert o["status"].tolist() == [0, 1, 0] and o["new_len"].tolist() == [4, 10, 24]
        c.same(want, codes)


@pytest.mark.parametrize("held", ["8", "16"])
def test_other_strides(held):
    """Heads outside slots, gaps between heads, tokens and pages, one key for all
    heads, scales within a larger table."""
    for D in (64, 128):
        c = Case([0, 17, 33], [20, 16, 1], 4, D, 32, H, held, seed=13)
        for name in "kv":
            c.cache[name] = c.cache[name].permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
        if held == "8":
            for name in "kv":
                big = torch.zeros((*c.scale[name].shape[:2], 9), dtype=torch.uint8, device="cuda")
                big[..., 2:6] = c.scale[name].view(torch.uint8)
                c.scale[name] = big[..., 2:6]
            c.scale["v"] = c.scale["v"].view(E8M0)
        c.k = c.k.transpose(0, 1).contiguous().transpose(0, 1)
        c.v = c.v[:, :1].expand(-1, 4, -1)
        c.rotate(D).check()
        c = Case([5, 8], [20, 16], 2, D, 16, H, held, seed=14)
        for name in "kv":
            x = c.cache[name].view(torch.uint8 if held == "8" else H)
            y = torch.zeros((x.shape[0], 16, 3, D + 16), dtype=x.dtype, device="cuda")
            y[:, :, :2, :D] = x
            c.cache[name] = y.view(c.cache[name].dtype)[:, :, :2, :D]
        c.check()


def test_no_requests_and_no_tokens():
    for held in ("8", "16"):
        c = Case([], [], held=held)
        assert c.call()["status"].numel() == 0
        Case([0, 33], [0, 0], held=held).check()
        Case([0, 33], [5, 3], held=held).choose(keep=[0, 0]).check()


@pytest.mark.parametrize("B", [70, 300, 2000])
def test_many_requests(B):
    gen = torch.Generator().manual_seed(B)
    draw = lambda hi: torch.randint(0, hi, (B,), generator=gen).tolist()  # noqa: E731
    Case(draw(60), draw(4 if B > 500 else 40), 2, 64, 16, H, "16", seed=15).rotate(64).check()
    Case(draw(60), draw(3 if B > 500 else 20), 1, 64, 16, H, "8", seed=16).check() if B < 500 else None


def test_one_long_prompt_among_single_tokens():
    lens, news = [40] * 20, [1] * 20
    lens[7], news[7] = 3, 3000
    Case(lens, news, 8, 128, 64, H, "8", seed=17).rotate(128).check()


def test_caches_of_more_than_2_to_the_31_elements():
    pages, page = 70000, 64
    for held in ("8", "16"):
        dt = torch.uint8 if held == "8" else H
        c = Case([30], [40], 4, 128, page, H, held, seed=18)
        small = dict(c.cache)
        c.table = i32([[pages - 1, pages - 2]])
        for name in "kv":
            big = torch.zeros((pages, page, 4, 128), dtype=dt, device="cuda")
            big[-3:] = small[name].view(dt)[:3]
            small[name] = big[-3:].clone().view(small[name].dtype)
            c.cache[name] = big.view(small[name].dtype)
            if held == "8":
                scale = torch.full((pages, 4, 4), 120, dtype=torch.uint8, device="cuda")
                c.scale[name] = scale.view(E8M0)
        want = Case([30], [40], 4, 128, page, H, held, seed=18)
        want.table = i32([[2, 1]])
        want.cache = small
        if held == "8":
            want.scale = {x: y.view(torch.uint8)[-3:].clone().view(E8M0) for x, y in c.scale.items()}
        want_cache, codes = want.expected()
        c.call()
        for name in "kv":
            assert torch.equal(c.cache[name].view(dt)[-3:], want_cache[name].view(dt))
            if held == "8":
                assert torch.equal(c.scale[name].view(torch.uint8)[-3:], codes[name])
        del c, big


def test_again_and_again():
    """The same call changes nothing more (a group's scale is at least its own)."""
    c = Case([10, 100, 0], [30, 1, 17], 8, 128, 64, H, seed=19).rotate(128)
    c.call()
    held = [y.view(torch.uint8) for y in (*c.cache.values(), *c.scale.values())]
    first = [y.clone() for y in held]
    for _ in range(5):
        c.call()
    assert all(torch.equal(x, y) for x, y in zip(held, first))


def test_captured_in_a_graph():
    c = Case([10, 100, 0], [3, 1, 17], 8, 128, 64, H, seed=20, room=200).rotate(128)
    lens, off = i32(c.lens), i32(c.off)
    out = dict(new_len=torch.empty_like(lens), status=torch.empty_like(lens))
    call = lambda: tt.tt_cache_append(  # noqa: E731
        c.k, c.v, c.cache["k"], c.cache["v"], c.table, lens, off, k_scale=c.scale["k"],
        v_scale=c.scale["v"], turns=c.turns, out=out)
    call()
    torch.cuda.synchronize()
    c.lens = out["new_len"].tolist()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):  # (each replay appends behind the last one)
        c.k.mul_(1.5)
        lens.copy_(out["new_len"])
        c.lens = lens.tolist()
        want, codes = c.expected()
        graph.replay()
        torch.cuda.synchronize()
        assert out["status"].tolist() == [0, 0, 0]
        c.same(want, codes)


def test_on_a_stream():
    c = Case([10, 0], [300, 1700], 8, 128, 64, H, seed=21).rotate(128)
    want, codes = c.expected()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    o = tt.tt_cache_append(c.k, c.v, c.cache["k"], c.cache["v"], c.table, i32(c.lens), i32(c.off),
                           k_scale=c.scale["k"], v_scale=c.scale["v"], turns=c.turns,
                           stream=stream)
    stream.synchronize()
    assert o["new_len"].tolist() == [310, 1700]
    c.same(want, codes)


def test_refused_by_the_library():
    c = Case([0], [4], 2, 64, 16, H)
    with pytest.raises(tt.TTError):  # new_len in cache_len's place
        lens = i32([0])
        tt.tt_cache_append(c.k, c.v, c.cache["k"], c.cache["v"], c.table, lens, i32(c.off),
                           k_scale=c.scale["k"], v_scale=c.scale["v"], out=dict(new_len=lens))
    with pytest.raises(ValueError):
        c.call(out=dict(status=torch.empty(1, dtype=torch.int32)))
