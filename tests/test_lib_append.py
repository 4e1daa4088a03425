"""tt_cache_append on the host: struct layouts and the refusals, each of which comes
back before the library touches a GPU."""
import ctypes
import math

import pytest
import torch

import paper_2510_15545_gb300 as tt
from paper_2510_15545_gb300 import _build, binding

P = ctypes.byref
INVALID = 1
MEMORY = 1 << 20  # stands for device memory; never read or written


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return tt.load()


def test_struct_layouts():
    assert ctypes.sizeof(binding._Scales) == 32
    A = binding._Append
    assert A.token_off.offset == 32 and A.k.offset == 64 and A.k_cache.offset == 112
    assert A.k_scale.offset == 176 and A.n_pages.offset == 240 and A.table_stride.offset == 256
    assert A.max_len.offset == 272 and ctypes.sizeof(A) == 280
    assert binding._APPEND.size == ctypes.sizeof(A)
    assert binding.TT_E4M3 == 3 and binding.TT_SCALE_SLOTS == 16


def append(lib, plan=None, new_len=3 * MEMORY, status=4 * MEMORY, **kw):
    heads = binding._Heads(MEMORY, 1024, 128)
    pages = binding._Pages(MEMORY, 16 * 1024, 1024, 128)
    more = binding._Pages(8 * MEMORY, 16 * 1024, 1024, 128)
    scales, scales_too = binding._Scales(MEMORY, 8, 8, 1), binding._Scales(2 * MEMORY, 8, 8, 1)
    f = dict(B=2, n_tokens=8, max_new=4, dtype=1, cache_dtype=3, n_heads=8, head_dim=128,
             page_size=16, token_off=MEMORY, k=heads, v=heads, k_cache=pages, v_cache=more,
             k_scale=scales, v_scale=scales_too, n_pages=100, page_table=MEMORY, table_stride=8,
             cache_len=2 * MEMORY, max_len=100)
    f.update(kw)
    return lib.tt_cache_append(P(binding._Append(**f)), P(plan) if plan else None, new_len, status,
                               None)


@pytest.mark.parametrize("kw", [dict(B=-1), dict(n_tokens=-1), dict(max_new=0), dict(dtype=0),
                                dict(dtype=3), dict(cache_dtype=0), dict(cache_dtype=2),
                                dict(n_heads=0), dict(head_dim=96), dict(page_size=8),
                                dict(page_size=24), dict(max_len=-1), dict(max_len=(1 << 30) + 1),
                                dict(token_off=None), dict(cache_len=None), dict(n_pages=0),
                                dict(page_table=None), dict(table_stride=6), dict(status=None),
                                dict(new_len=2 * MEMORY),
                                dict(plan=binding._RopePlan(None, 128, 0, 1.0)),
                                dict(plan=binding._RopePlan(MEMORY, 130, 0, 1.0)),
                                dict(plan=binding._RopePlan(MEMORY, 63, 0, 1.0)),
                                dict(plan=binding._RopePlan(MEMORY, 128, 2, 1.0)),
                                dict(plan=binding._RopePlan(MEMORY, 128, 0, math.inf))])
def test_refusals(lib, kw):
    assert append(lib, **kw) == INVALID


def test_tensors_refused(lib):
    for bad in (binding._Heads(None, 1024, 128), binding._Heads(MEMORY + 8, 1024, 128),
                binding._Heads(MEMORY, 1028, 128), binding._Heads(MEMORY, 1024, -128)):
        assert append(lib, k=bad) == INVALID and append(lib, v=bad) == INVALID
    for cache in (1, 3):
        for bad in (binding._Pages(None, 16384, 1024, 128), binding._Pages(MEMORY + 2, 16384, 1024, 128),
                    binding._Pages(MEMORY, 16388, 1024, 128), binding._Pages(MEMORY, 16384, 1020, 128),
                    binding._Pages(MEMORY, 16384, 1024, -128)):
            assert append(lib, cache_dtype=cache, k_cache=bad) == INVALID
            assert append(lib, cache_dtype=cache, v_cache=bad) == INVALID
    # elements of one byte: the strides' 16 bytes are 16 elements
    odd = binding._Pages(MEMORY, 16384, 1032, 128)
    assert append(lib, k_cache=odd) == INVALID
    for bad in (binding._Scales(None, 8, 8, 1), binding._Scales(MEMORY, -8, 8, 1),
                binding._Scales(MEMORY, 8, -8, 1), binding._Scales(MEMORY, 8, 8, -1)):
        assert append(lib, k_scale=bad) == INVALID and append(lib, v_scale=bad) == INVALID


def test_memory_that_is_read_and_written_refused(lib):
    for at in (MEMORY, MEMORY + 8, MEMORY - 4, 2 * MEMORY, 2 * MEMORY + 4):
        assert append(lib, new_len=at) == INVALID and append(lib, status=at) == INVALID
    for name in ("keep", "path"):
        for at in (16 * MEMORY, 16 * MEMORY - 4, 16 * MEMORY + 4):
            for out in ("new_len", "status"):
                assert append(lib, **{name: 16 * MEMORY, out: at}) == INVALID
    assert append(lib, new_len=4 * MEMORY) == INVALID
    one = binding._Pages(MEMORY, 16384, 1024, 128)
    for cache in (1, 3):
        assert append(lib, cache_dtype=cache, k_cache=one, v_cache=one) == INVALID
    assert append(lib, v_scale=binding._Scales(MEMORY, 8, 8, 1)) == INVALID


def test_no_requests_need_nothing(lib):
    assert append(lib, B=0, status=None, token_off=None, k=binding._Heads()) == 0


@pytest.fixture
def anywhere(monkeypatch):
    """The binding's checks on host tensors; a call that passes them fails."""
    class Library:
        def __getattr__(self, name):
            raise AssertionError(name)
    monkeypatch.setattr(binding, "_gpu_of", lambda *t: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(binding, "load", Library)


def arguments(**kw):
    i32 = torch.int32
    a = dict(k=torch.zeros((4, 2, 64), dtype=torch.bfloat16), v=torch.zeros((4, 2, 64), dtype=torch.bfloat16),
             k_cache=torch.zeros((6, 32, 2, 64)).to(torch.float8_e4m3fn),
             v_cache=torch.zeros((6, 32, 2, 64)).to(torch.float8_e4m3fn),
             page_table=torch.zeros((2, 3), dtype=i32), cache_len=torch.zeros(2, dtype=i32),
             token_off=torch.zeros(3, dtype=i32), k_scale=torch.zeros((6, 2, 2), dtype=torch.uint8),
             v_scale=torch.zeros((6, 2, 2), dtype=torch.uint8).view(torch.float8_e8m0fnu))
    a.update(kw)
    return a


def test_arguments_refused(anywhere):
    x, i32 = arguments(), torch.int32
    half = torch.zeros((6, 32, 2, 64), dtype=torch.bfloat16)
    for bad in (dict(k=x["k"][:3]), dict(k=x["k"][0]), dict(k=x["k"].half()), dict(v=x["v"][:, :1]),
                dict(k_cache=x["k_cache"][:5]), dict(k_cache=half), dict(v_cache=half),
                dict(k_cache=half, v_cache=half), dict(k_cache=half.half(), v_cache=half.half(),
                                                      k_scale=None, v_scale=None),
                dict(k_scale=None), dict(v_scale=None), dict(k_scale=x["k_scale"][:, :1]),
                dict(k_scale=x["k_scale"].float()), dict(v_scale=x["k_scale"].transpose(1, 2)[:, :, :1]),
                dict(page_table=x["page_table"].long()), dict(page_table=x["page_table"][:1]),
                dict(page_table=torch.zeros(3, dtype=i32).expand(2, 3)),
                dict(cache_len=x["cache_len"].long()), dict(token_off=x["token_off"][:2]),
                dict(keep=torch.zeros(1, dtype=i32)), dict(path=torch.zeros(3, dtype=i32)),
                dict(positions=torch.zeros(4, dtype=i32)), dict(max_len=97),
                dict(turns=torch.zeros(32, dtype=torch.int32)),
                dict(turns=torch.zeros(32, dtype=torch.int64), positions=torch.zeros(3, dtype=i32)),
                dict(max_new=1 << 40)):
        with pytest.raises(ValueError):
            tt.tt_cache_append(**arguments(**bad))
    with pytest.raises(TypeError):
        tt.tt_cache_append(**arguments(k=x["k"].float(), v=x["v"].float()))


def test_tensors_on_the_host_are_refused():
    with pytest.raises(ValueError, match="GPU"):
        tt.tt_cache_append(**arguments())
