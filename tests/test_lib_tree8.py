"""tt_tree_attn over caches in 8 bits, on the host: the refusals, each of which comes back
before the library touches a GPU, and the workspace's size."""
import ctypes

import pytest
import torch

import paper_2510_15545_gb300 as tt
from paper_2510_15545_gb300 import _build, binding
from test_lib_append import anywhere  # noqa: F401
from test_lib_operators import BAD_HEADS, BAD_PAGES, INVALID, MEMORY, SIZES, UNSUPPORTED, tree

P = ctypes.byref
SCALES = binding._Scales(MEMORY, 8, 8, 1)


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return tt.load()


def attend(lib, t, ks=SCALES, vs=SCALES, ws=MEMORY, ws_bytes=1 << 40, out=MEMORY, status=MEMORY):
    return lib.tt_tree_attn8(P(t), P(ks) if ks else None, P(vs) if vs else None, ws, ws_bytes, out,
                             MEMORY, status, None)


@pytest.mark.parametrize("kw", SIZES)
def test_sizes_refused(lib, kw):
    assert attend(lib, tree(**kw)) == INVALID
    assert lib.tt_tree8_workspace_bytes(P(tree(**kw))) == 0


@pytest.mark.parametrize("kw", [dict(dtype=0), dict(dtype=3), dict(scale=0.0), dict(scale=-1.0),
                                dict(tree_off=None), dict(cache_len=None), dict(n_pages=0),
                                dict(page_table=None), dict(table_stride=6)])
def test_refusals(lib, kw):
    assert attend(lib, tree(**kw)) == INVALID


@pytest.mark.parametrize("i", range(5))
def test_tensors_refused(lib, i):
    for name in ("q", "k", "v"):
        assert attend(lib, tree(**{name: BAD_HEADS[i]})) == INVALID
    for name in ("k_cache", "v_cache"):
        assert attend(lib, tree(**{name: BAD_PAGES[i]})) == INVALID


def test_strides_of_bytes(lib):
    """Elements of one byte: 16 bytes are 16 elements."""
    for odd in (binding._Pages(MEMORY, 16384 + 8, 1024, 128), binding._Pages(MEMORY, 16384, 1032, 128),
                binding._Pages(MEMORY, 16384, 1024, 136)):
        assert attend(lib, tree(k_cache=odd)) == INVALID
        assert attend(lib, tree(v_cache=odd)) == INVALID


def test_scales_refused(lib):
    for bad in (None, binding._Scales(None, 8, 8, 1), binding._Scales(MEMORY, -8, 8, 1),
                binding._Scales(MEMORY, 8, -8, 1), binding._Scales(MEMORY, 8, 8, -1)):
        assert attend(lib, tree(), ks=bad) == INVALID
        assert attend(lib, tree(), vs=bad) == INVALID


def test_outputs_and_workspace_refused(lib):
    assert attend(lib, tree(), out=None) == INVALID
    assert attend(lib, tree(), out=MEMORY + 8) == INVALID
    assert attend(lib, tree(), status=None) == INVALID
    # (few rows and many, whose items are of different sizes)
    for nodes in (1, 4, 512):
        t = tree(max_nodes=nodes, max_len=100000, table_stride=6250, n_pages=20000)
        need = lib.tt_tree8_workspace_bytes(P(t))
        assert need > 0
        assert attend(lib, t, ws=None) == INVALID
        assert attend(lib, t, ws=MEMORY + 16, ws_bytes=need) == INVALID
        assert attend(lib, t, ws_bytes=need - 1) == INVALID


def test_no_requests_need_nothing(lib):
    assert attend(lib, tree(B=0), status=None) == 0


def test_places_beyond_32_bits(lib):
    big = tree(B=65535, max_nodes=512, max_len=1 << 20, table_stride=65536, n_pages=65536)
    assert attend(lib, big) == UNSUPPORTED
    assert attend(lib, tree(B=1 << 20, max_nodes=512)) == UNSUPPORTED
    assert attend(lib, tree(B=2**31 - 1)) == UNSUPPORTED


def arguments(**kw):
    i32, bf16 = torch.int32, torch.bfloat16
    a = dict(q=torch.zeros((4, 4, 64), dtype=bf16), k=torch.zeros((4, 2, 64), dtype=bf16),
             v=torch.zeros((4, 2, 64), dtype=bf16),
             k_cache=torch.zeros((6, 32, 2, 64)).to(torch.float8_e4m3fn),
             v_cache=torch.zeros((6, 32, 2, 64)).to(torch.float8_e4m3fn),
             page_table=torch.zeros((2, 3), dtype=i32), cache_len=torch.zeros(2, dtype=i32),
             tree_off=torch.zeros(3, dtype=i32), k_scale=torch.zeros((6, 2, 2), dtype=torch.uint8),
             v_scale=torch.zeros((6, 2, 2), dtype=torch.uint8).view(torch.float8_e8m0fnu))
    a.update(kw)
    return a


def test_arguments_refused(anywhere):  # noqa: F811
    x = arguments()
    half = torch.zeros((6, 32, 2, 64), dtype=torch.bfloat16)
    for bad in (dict(q=x["q"][:3]), dict(k=x["k"].half()), dict(v=x["v"][:, :1]),
                dict(k_cache=x["k_cache"][:5]), dict(k_cache=half), dict(v_cache=half),
                dict(k_cache=half, v_cache=half), dict(k_scale=None), dict(v_scale=None),
                dict(k_scale=x["k_scale"][:, :1]), dict(k_scale=x["k_scale"].float()),
                dict(v_scale=x["k_scale"].transpose(1, 2)[:, :, :1]),
                dict(page_table=x["page_table"].long()), dict(page_table=x["page_table"][:1]),
                dict(cache_len=x["cache_len"].long()), dict(tree_off=x["tree_off"][:2]),
                dict(parents=torch.zeros(3, dtype=torch.int32)), dict(max_len=97),
                dict(max_nodes=1 << 40)):
        with pytest.raises(ValueError):
            tt.tt_tree_attn(**arguments(**bad))
    with pytest.raises(TypeError):
        tt.tt_tree_attn(**arguments(q=x["q"].float()))


def test_tensors_on_the_host_are_refused():
    with pytest.raises(ValueError, match="GPU"):
        tt.tt_tree_attn(**arguments())
