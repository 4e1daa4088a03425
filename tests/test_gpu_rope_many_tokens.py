"""tt_rope over as many tokens as its type counts: a CTA's share does not divide them, and
the last one's numbers pass 2^31."""
import pytest
import torch

import paper_2510_15545_gb300 as tt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rot", [6, 8])
def test_the_most_tokens(rot):
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    tt.load(build_if_missing=True)
    N, D = 2 ** 31 - 1, 8
    if torch.cuda.mem_get_info()[0] < 64 << 30:
        pytest.skip("needs 64 GB of memory")
    gen = torch.Generator(device="cuda").manual_seed(rot)
    one = torch.randn((1, 1, D), generator=gen, device="cuda").bfloat16()
    positions = torch.arange(N, dtype=torch.int32, device="cuda")
    turns = tt.rope_turns(tt.rope_freqs(rot))
    # (what lies behind the output is looked at, too)
    room = torch.full(((N + 64) * D,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = room[:N * D].view(N, 1, D)
    tt.tt_rope(one.expand(N, 1, D), None, positions, turns, out={"q": out})
    assert (room[N * D:] == 7).all()
    for lo, hi in ((0, 100), (2 ** 30 - 50, 2 ** 30 + 50), (N - 100, N)):
        few = tt.tt_rope(one.expand(hi - lo, 1, D), None, positions[lo:hi].clone(), turns)["q"]
        assert torch.equal(out[lo:hi], few)
    # (the angle of the last one in 64 bits; a rounding of 2^-8 and the sines' 2^-20)
    x = one[0, 0].double()
    f = tt.rope_freqs(rot).cuda()
    turn = (N - 1) * f / (2 * torch.pi)  # (2^31 turns at most: 2^-22 of a turn left in 64 bits)
    c, s = torch.cos(2 * torch.pi * (turn % 1)), torch.sin(2 * torch.pi * (turn % 1))
    h = rot // 2
    want = torch.cat([x[:h] * c - x[h:rot] * s, x[h:rot] * c + x[:h] * s, x[rot:]])
    size = torch.cat([(x[:h].abs() + x[h:rot].abs()).repeat(2), x[rot:].abs()])
    assert ((out[N - 1, 0].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -16) * size).all()
