"""The operators' part of the C ABI, on the host: struct layouts, workspace
sizes, and the refusals, each of which comes back before the library touches a
GPU (no call here passes its checks)."""
import ctypes
import math

import pytest
import torch

import paper_2510_15545_gb300 as tt
from paper_2510_15545_gb300 import _build, binding

P = ctypes.byref
INVALID, UNSUPPORTED = 1, 2
MEMORY = 1 << 20  # stands for device memory; never read or written


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return tt.load()


def test_struct_layouts():
    assert ctypes.sizeof(binding._LogprobsOut) == 56 and binding._LogprobsOut.status.offset == 48
    assert ctypes.sizeof(binding._Teacher) == 24 and binding._Teacher.k.offset == 16
    assert ctypes.sizeof(binding._Heads) == 24 and ctypes.sizeof(binding._Pages) == 32
    T = binding._Tree
    assert T.page_size.offset == 28 and T.tree_off.offset == 32 and T.q.offset == 48
    assert T.v.offset == 96 and T.k_cache.offset == 120 and T.v_cache.offset == 152
    assert T.n_pages.offset == 184 and T.table_stride.offset == 200
    assert T.max_len.offset == 216 and T.scale.offset == 220 and ctypes.sizeof(T) == 224
    assert binding._TREE.size == ctypes.sizeof(T)


def logits(**kw):
    f = dict(data=MEMORY, dtype=0, n_cols=1000, row_stride=1000, n_rows=4)
    f.update(kw)
    return binding._Logits(**f)


def logprobs(lib, rows=None, ids=MEMORY, temp=1.0, n=4, **out):
    f = {name: MEMORY for name, _ in binding._LogprobsOut._fields_}
    f.update(out)
    return lib.tt_logprobs(P(rows or logits()), ids, ctypes.c_float(temp), n,
                           P(binding._LogprobsOut(**f)), None)


BAD_ROWS = [dict(n_rows=-1), dict(data=None), dict(data=MEMORY + 8), dict(dtype=2), dict(dtype=-1),
            dict(n_cols=0), dict(row_stride=996), dict(row_stride=1001)]


@pytest.mark.parametrize("kw", BAD_ROWS)
def test_logprobs_refuses_rows(lib, kw):
    assert logprobs(lib, logits(**kw)) == INVALID


@pytest.mark.parametrize("kw", [dict(temp=0.0), dict(temp=-1.0), dict(temp=math.nan),
                                dict(temp=math.inf), dict(temp=1e-37), dict(n=-1), dict(n=33),
                                dict(status=None), dict(ids=None)])
def test_logprobs_refuses(lib, kw):
    assert logprobs(lib, **kw) == INVALID


def test_no_rows_need_nothing(lib):
    assert logprobs(lib, logits(n_rows=0, data=None), ids=None, status=None) == 0
    assert distill(lib, logits(n_rows=0, data=None), status=None) == 0


def distill(lib, student=None, ids=MEMORY, logp=MEMORY, k=8, temp=1.0, tail=0, stats=MEMORY,
            grad=None, status=MEMORY):
    return lib.tt_distill(P(student or logits()), P(binding._Teacher(ids, logp, k)),
                          ctypes.c_float(temp), tail, None, MEMORY, stats,
                          P(grad) if grad else None, status, None)


@pytest.mark.parametrize("kw", BAD_ROWS)
def test_distill_refuses_rows(lib, kw):
    assert distill(lib, logits(**kw)) == INVALID


@pytest.mark.parametrize("kw", [dict(ids=None), dict(logp=None), dict(k=-1), dict(k=129),
                                dict(temp=0.0), dict(temp=math.nan), dict(tail=2), dict(tail=-1),
                                dict(stats=MEMORY + 4), dict(status=None)])
def test_distill_refuses(lib, kw):
    assert distill(lib, **kw) == INVALID


@pytest.mark.parametrize("kw", [dict(dtype=1), dict(n_cols=999), dict(n_rows=3), dict(data=None),
                                dict(row_stride=998)])
def test_distill_refuses_gradients(lib, kw):
    assert distill(lib, grad=logits(**kw)) == INVALID
    assert lib.tt_distill_grad(P(logits()), P(binding._Teacher(MEMORY, MEMORY, 8)),
                               ctypes.c_float(1.0), 0, None, MEMORY, P(logits(**kw)),
                               None) == INVALID


def test_distill_grad_needs_its_stats(lib):
    for stats in (None, MEMORY + 4):
        assert lib.tt_distill_grad(P(logits()), P(binding._Teacher(MEMORY, MEMORY, 8)),
                                   ctypes.c_float(1.0), 0, None, stats, P(logits()),
                                   None) == INVALID


def test_distill_row_width(lib):
    wide = 819208
    assert distill(lib, logits(n_cols=wide, row_stride=wide)) == UNSUPPORTED


def tree(**kw):
    heads = binding._Heads(MEMORY, 1024, 128)
    pages = binding._Pages(MEMORY, 16 * 1024, 1024, 128)
    f = dict(B=2, n_nodes=8, max_nodes=4, dtype=1, n_q_heads=8, n_kv_heads=2, head_dim=128,
             page_size=16, tree_off=MEMORY, parents=MEMORY, q=heads, k=heads, v=heads,
             k_cache=pages, v_cache=pages, n_pages=100, page_table=MEMORY, table_stride=8,
             cache_len=MEMORY, max_len=100, scale=0.1)
    f.update(kw)
    return binding._Tree(**f)


def attend(lib, t, ws=MEMORY, ws_bytes=1 << 40, out=MEMORY, status=MEMORY):
    return lib.tt_tree_attn(P(t), ws, ws_bytes, out, MEMORY, status, None)


SIZES = [dict(B=-1), dict(n_nodes=-1), dict(max_nodes=0), dict(max_nodes=513), dict(n_q_heads=9),
         dict(n_q_heads=0), dict(n_kv_heads=0), dict(n_q_heads=258), dict(head_dim=96),
         dict(page_size=8), dict(page_size=24), dict(max_len=-1)]
BAD_HEADS = [binding._Heads(None, 1024, 128), binding._Heads(MEMORY + 8, 1024, 128),
             binding._Heads(MEMORY, 1028, 128), binding._Heads(MEMORY, -1024, 128),
             binding._Heads(MEMORY, 1024, 4)]
BAD_PAGES = [binding._Pages(None, 16384, 1024, 128), binding._Pages(MEMORY + 2, 16384, 1024, 128),
             binding._Pages(MEMORY, 16388, 1024, 128), binding._Pages(MEMORY, 16384, 1020, 128),
             binding._Pages(MEMORY, 16384, 1024, -128)]


@pytest.mark.parametrize("kw", SIZES)
def test_tree_refuses_sizes(lib, kw):
    assert attend(lib, tree(**kw)) == INVALID
    assert lib.tt_tree_workspace_bytes(P(tree(**kw))) == 0


@pytest.mark.parametrize("kw", [dict(dtype=0), dict(dtype=3), dict(scale=0.0), dict(scale=-1.0),
                                dict(scale=math.nan), dict(scale=math.inf), dict(tree_off=None),
                                dict(cache_len=None), dict(n_pages=0), dict(page_table=None),
                                dict(table_stride=6)])
def test_tree_refuses(lib, kw):
    assert attend(lib, tree(**kw)) == INVALID


@pytest.mark.parametrize("i", range(5))
def test_tree_refuses_tensors(lib, i):
    for name in ("q", "k", "v"):
        assert attend(lib, tree(**{name: BAD_HEADS[i]})) == INVALID
    for name in ("k_cache", "v_cache"):
        assert attend(lib, tree(**{name: BAD_PAGES[i]})) == INVALID


def test_tree_refuses_outputs_and_workspace(lib):
    assert attend(lib, tree(), out=None) == INVALID
    assert attend(lib, tree(), out=MEMORY + 8) == INVALID
    assert attend(lib, tree(), status=None) == INVALID
    t = tree(max_len=100000, table_stride=6250, n_pages=20000)
    need = lib.tt_tree_workspace_bytes(P(t))
    assert need > 0
    assert attend(lib, t, ws=None) == INVALID
    assert attend(lib, t, ws=MEMORY + 16, ws_bytes=need) == INVALID
    assert attend(lib, t, ws_bytes=need - 1) == INVALID


def test_tree_of_no_requests(lib):
    assert attend(lib, tree(B=0), status=None) == 0


def test_tree_refuses_what_its_numbers_do_not_hold(lib):
    """The list's places (one per tile of every request, key head and row tile, at
    the longest) and the rows of the join are counted in 32 bits."""
    big = tree(B=65535, max_nodes=512, max_len=1 << 20, table_stride=65536, n_pages=65536)
    assert attend(lib, big) == UNSUPPORTED
    assert attend(lib, tree(B=1 << 20, max_nodes=512)) == UNSUPPORTED
    assert attend(lib, tree(B=2**31 - 1)) == UNSUPPORTED


def described(table, B, **kw):
    """The descriptor of a call with a page table, of pages of 16 slots."""
    heads = torch.zeros((B, 2, 64), dtype=torch.bfloat16)
    cache = torch.zeros((9, 16, 2, 64), dtype=torch.bfloat16)
    lens, off = torch.zeros(B, dtype=torch.int32), torch.arange(B + 1, dtype=torch.int32)
    a = dict(scale=None, max_len=None, max_nodes=None)
    a.update(kw)
    return binding._tree(heads, heads, heads, cache, cache, table, lens, off, None, **a)


def test_page_tables_whose_rows_share_memory_are_refused():
    """A stride of theirs, or one made up, would have the kernel read other entries
    than the table's, or past its end."""
    row = torch.arange(5, dtype=torch.int32)
    for table in (row.expand(4, 5), row.repeat(2).unfold(0, 5, 1)[:4]):
        with pytest.raises(ValueError):
            described(table, 4)
        with pytest.raises(ValueError):
            described(table, 4, max_len=33)
    # rows that share only what no request reaches keep their own stride
    T = described(torch.arange(20, dtype=torch.int32).unfold(0, 5, 3)[:4], 4, max_len=48)
    assert T.table_stride == 3 and T.max_len == 48
    for B in (1, 4):
        assert described(row.repeat(B, 1), B).table_stride == 5
        assert described(torch.zeros((B, 12), dtype=torch.int32)[:, :5], B).table_stride == 12
    # one row has any stride; no length needs no row
    assert described(row.expand(1, 5).as_strided((1, 5), (0, 1)), 1).table_stride == 5
    assert described(torch.zeros((4, 0), dtype=torch.int32), 4).max_len == 0


class Calls:
    """Stands for the library on the host: keeps the arguments of its calls, whose
    sizes the real one gives, and answers that all went well."""

    def __init__(self, monkeypatch, lib):
        self.lib, self.args = lib, {}
        monkeypatch.setattr(binding, "load", lambda: self)
        monkeypatch.setattr(binding, "_stream", lambda stream: None)

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return getattr(self.lib, name)

        def call(*args):
            self.args[name] = args
            return 0
        return call


def test_results_of_tree_attention_hold_no_scratch(lib, monkeypatch):
    calls = Calls(monkeypatch, lib)
    heads = torch.zeros((8, 8, 128), dtype=torch.bfloat16)
    cache = torch.zeros((4, 16, 8, 128), dtype=torch.bfloat16)
    table = torch.zeros((2, 2), dtype=torch.int32)
    lens, off = torch.zeros(2, dtype=torch.int32), torch.tensor([0, 4, 8], dtype=torch.int32)
    status = torch.zeros(2, dtype=torch.int32)
    for out in (None, dict(status=status), dict(out=torch.zeros_like(heads))):
        o = tt.tt_tree_attn(heads, heads, heads, cache, cache, table, lens, off, out=out)
        need = calls.args["tt_tree_attn"][2]
        assert need >= lib.tt_tree_workspace_bytes(calls.args["tt_tree_attn"][0]) > 100000
        for name, x in o.items():
            assert x.untyped_storage().nbytes() < 20000, name


@pytest.mark.parametrize("change", [lambda x: x.mul_(2.0), lambda x: x.div_(4.0),
                                    lambda x: x[0].zero_()])
def test_losses_may_be_changed_in_place(lib, monkeypatch, change):
    """As any loss may: what the backward pass keeps is no part of them."""
    Calls(monkeypatch, lib)
    z = torch.zeros((3, 8), requires_grad=True)
    loss = tt.distill_loss(z, torch.zeros((3, 2), dtype=torch.int32), torch.zeros((3, 2)))
    assert loss.shape == (3,) and loss.dtype is torch.float32
    change(loss)
    loss.sum().backward()
    assert z.grad.shape == z.shape


def test_status_bits_and_types():
    assert (binding.TT_F32, binding.TT_BF16, binding.TT_F16) == (0, 1, 2)
