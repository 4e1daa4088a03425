"""tt_cache_append writes its caches and their scales: entries that share memory would be
written by several warps in no order, and are refused before the library touches a GPU."""
import ctypes

import pytest
import torch

import paper_2510_15545_gb300 as tt
from paper_2510_15545_gb300 import binding
from test_lib_append import INVALID, MEMORY, append, lib  # noqa: F401

P = ctypes.byref
H, D, PAGE, PAGES = 8, 128, 32, 100  # heads, elements, slots of a page, pages


def appended(lib, **kw):  # noqa: F811
    """The status of a call whose caches are [pages, slots, heads, elements]; without
    requests' tokens it goes no further than its checks on a host without a GPU."""
    f = dict(page_size=PAGE, k_cache=pages(), v_cache=pages(at=8 * MEMORY), k_scale=scales(),
             v_scale=scales(at=2 * MEMORY), cache_dtype=3)
    f.update(kw)
    return append(lib, **f)


def pages(page=PAGE * H * D, slot=H * D, head=D, at=MEMORY):
    return binding._Pages(at, page, slot, head)


def scales(page=2 * H, group=H, head=1, at=MEMORY):
    return binding._Scales(at, page, group, head)


@pytest.mark.parametrize("cache", [1, 3])
@pytest.mark.parametrize("name", ["k_cache", "v_cache"])
@pytest.mark.parametrize("bad", [dict(head=0), dict(slot=0), dict(page=0), dict(head=D - 16),
                                 dict(slot=H * D - 16), dict(slot=D, head=D), dict(page=H * D),
                                 dict(page=PAGE * H * D - 16), dict(slot=D, head=PAGE * D - 16),
                                 dict(page=D, slot=PAGES * D, head=(PAGE - 1) * PAGES * D)])
def test_pages_that_overlap_are_refused(lib, cache, name, bad):  # noqa: F811
    at = MEMORY if name == "k_cache" else 8 * MEMORY
    assert appended(lib, cache_dtype=cache, **{name: pages(**bad, at=at)}) == INVALID


@pytest.mark.parametrize("name", ["k_scale", "v_scale"])
@pytest.mark.parametrize("bad", [dict(head=0), dict(group=0), dict(page=0), dict(group=H - 1),
                                 dict(page=2 * H - 1), dict(group=1), dict(group=1, head=1),
                                 dict(page=1, group=PAGES, head=PAGES)])
def test_scales_that_overlap_are_refused(lib, name, bad):  # noqa: F811
    at = MEMORY if name == "k_scale" else 2 * MEMORY
    assert appended(lib, **{name: scales(**bad, at=at)}) == INVALID


@pytest.fixture
def reaches_the_gpu(lib):  # noqa: F811
    if torch.cuda.is_available():
        pytest.skip("would launch on addresses that stand for memory")
    return lambda **kw: appended(lib, **kw) not in (0, INVALID)


def test_other_orders_of_pages_are_taken(reaches_the_gpu):
    """Heads or slots outermost within a page, pages innermost, room between, and any stride
    where there is one entry."""
    assert reaches_the_gpu()
    for good in (pages(slot=D, head=PAGE * D), pages(page=D, slot=PAGES * D, head=PAGE * PAGES * D),
                 pages(page=H * D, slot=PAGES * H * D), pages(page=2 * PAGE * H * D, slot=2 * H * D, head=2 * D),
                 pages(page=1 << 40)):
        for cache in (1, 3):
            assert reaches_the_gpu(cache_dtype=cache, k_cache=good)
    for good in (scales(group=1, head=2), scales(page=1, group=PAGES, head=2 * PAGES), scales(page=1 << 40),
                 scales(page=56, group=1, head=7)):
        assert reaches_the_gpu(k_scale=good)
    assert reaches_the_gpu(n_heads=1, k_cache=pages(head=0), k_scale=scales(head=0))
    assert reaches_the_gpu(n_pages=1, k_cache=pages(page=0), k_scale=scales(page=0))
    assert reaches_the_gpu(page_size=16, max_len=100, k_scale=scales(group=0))
    assert reaches_the_gpu(page_size=16, n_heads=1, n_pages=1, max_len=16, table_stride=1,
                           k_scale=scales(0, 0, 0), v_scale=scales(0, 0, 0, at=2 * MEMORY))
    assert reaches_the_gpu(max_len=0, k_cache=pages(0, 0, 0), k_scale=scales(0, 0, 0))


@pytest.mark.gpu
@pytest.mark.parametrize("name,dims", [("k_scale", 1), ("k_scale", 2), ("v_scale", 2), ("v_cache", 2), ("k_cache", 1)])
def test_expanded_tensors_are_refused(name, dims):
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    tt.load(build_if_missing=True)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    k = torch.ones((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    a = dict(k=k, v=k.clone(), page_table=i32([[0, 1]]), cache_len=i32([0]), token_off=i32([0, 4]),
             **{c: torch.zeros((6, 32, 2, 64), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
                for c in ("k_cache", "v_cache")},
             **{c: torch.zeros((6, 2, 2), dtype=torch.uint8, device="cuda") for c in ("k_scale", "v_scale")})
    assert tt.tt_cache_append(**a)["status"].tolist() == [0]
    a[name] = a[name].narrow(dims, 0, 1).expand(a[name].shape)
    with pytest.raises(tt.TTError) as e:
        tt.tt_cache_append(**a)
    assert e.value.code == binding.TT_ERR_INVALID_ARG
