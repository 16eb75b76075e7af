"""CPU-only checks of what the Python binding lets through to the tree, prompt and page calls: the library is replaced by a
recorder, so a call that should have been refused is seen and never runs."""
import gc
import weakref

import pytest
import torch

import paper_2601_21686_b200 as S

BF = torch.bfloat16


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return S.STIEF_OK
        return call


@pytest.fixture
def calls(monkeypatch):
    """Host tensors pass for the current device's; the list of calls that reached the library."""
    rec = Recorder()
    monkeypatch.setattr(S, "lib", lambda: rec)
    monkeypatch.setattr(S, "_here", lambda t, name, device=None: 0)
    monkeypatch.setattr(S, "_raw_stream", lambda device: 0)
    return rec.calls


def i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def layer(Hq=8, Hkv=2, r_k=64, r_v=64, pages=4, k=None, v=None):
    pool = lambda r: torch.zeros(pages, Hkv, 64, r, dtype=BF)
    basis = lambda r: torch.zeros(Hkv, 128, r, dtype=BF)
    return S.Layer(Hq, Hkv, r_k, r_v, basis(r_k), basis(r_v), pool(r_k) if k is None else k, pool(r_v) if v is None else v)


def accept(layers):
    S.stief_tree_accept(layers, S.Batch(i32(2, 2), i32(2)), i32(2, 3), i32(2))


def test_accept_refuses_pools_that_are_not_what_the_layer_says(calls):
    good = layer()
    accept([good])
    assert len(calls) == 1
    pool = lambda *shape, dtype=BF: torch.zeros(*shape, dtype=dtype)
    for bad in (layer(r_k=128, k=pool(4, 2, 64, 64)), layer(r_v=32, v=pool(4, 2, 64, 64)),          # other ranks than the pools'
                layer(r_k=32, r_v=64, k=pool(4, 2, 64, 64), v=pool(4, 2, 64, 32)),                    # swapped
                layer(Hkv=8, k=pool(4, 2, 64, 64), v=pool(4, 2, 64, 64)),                             # other heads
                layer(k=pool(4, 2, 32, 64)), layer(k=pool(4, 128, 64)), layer(v=pool(3, 2, 64, 64)),
                layer(k=pool(4, 2, 64, 64, dtype=torch.float16)), layer(v=pool(4, 2, 64, 64, dtype=torch.float32)),
                layer(k=pool(4, 2, 64, 128)[..., :64])):
        for layers in ([bad], [good, bad]):
            with pytest.raises(ValueError):
                accept(layers)
    codes = lambda *shape: torch.zeros(*shape, dtype=torch.uint8)
    quantised = S.QLayer(8, 2, 64, 64, None, None, None, codes(4, 2, 64, 64), codes(4, 2, 64, 64), torch.zeros(4, 2, 64, 1, 2))
    with pytest.raises(ValueError):
        accept([good, quantised])
    assert len(calls) == 1


def tree(l, n_q=4):
    q, out = torch.zeros(2, n_q, l.Hq, 128, dtype=BF), torch.zeros(2, n_q, l.Hq, 128, dtype=BF)
    S.stief_tree_attention(l, S.Batch(i32(2, 2), i32(2)), q, i32(2, n_q, 1), torch.zeros(1 << 10, dtype=torch.uint8), out)


def _set(name, value):
    return lambda l: setattr(l, name, value)


CHANGES = {
    "smaller key rank": _set("r_k", 32), "larger key rank": _set("r_k", 128), "smaller value rank": _set("r_v", 48), "larger value rank": _set("r_v", 96),
    "more heads": _set("Hkv", 4), "fewer heads": _set("Hkv", 1),
    "pool resized in place": lambda l: l.k_pool.resize_(4, 2, 32, 64),
    "pool re-laid in place": lambda l: l.v_pool.transpose_(2, 3),
    "pool pointed elsewhere in place": lambda l: l.v_pool.set_(torch.zeros(4, 2, 64, 32, dtype=BF)),
    "pool of another type in place": lambda l: setattr(l.k_pool, "data", torch.zeros(4, 2, 64, 64)),
    "basis resized in place": lambda l: l.U_k.resize_(2, 64, 64),
    "basis pointed elsewhere in place": lambda l: l.U_v.set_(torch.zeros(2, 128, 32, dtype=BF)),
}


@pytest.mark.parametrize("change", CHANGES)
def test_tree_attention_looks_at_the_layer_in_every_call(calls, change):
    l = layer()
    tree(l)
    tree(l)
    assert [name for name, _ in calls].count("stief_tree_attention") == 2
    CHANGES[change](l)
    with pytest.raises(ValueError):
        tree(l)
    assert [name for name, _ in calls].count("stief_tree_attention") == 2


TABLE_CHANGES = {
    "fewer lengths at the same address": lambda t: setattr(t, "seq_lens", t.seq_lens[:2]),
    "fewer counts at the same address": lambda t: setattr(t, "page_counts", t.page_counts[:2]),
    "lengths of another type": lambda t: setattr(t, "seq_lens", t.seq_lens.view(torch.float32)),
    "a transposed table": lambda t: t.block_table.t_(), "counts in two dimensions": lambda t: t.page_counts.resize_(3, 1),
    "fewer lengths in place": lambda t: t.seq_lens.resize_(2), "references in two dimensions": lambda t: t.ref_counts.resize_(4, 2),
}


@pytest.mark.parametrize("change", TABLE_CHANGES)
def test_page_calls_look_at_the_table_in_every_call(calls, change):
    table = S.PageTable(i32(3, 3), i32(3), i32(3), i32(8))
    reserve = lambda: S.stief_pages_reserve(table, 5)
    reserve()
    reserve()
    assert len(calls) == 2
    TABLE_CHANGES[change](table)
    with pytest.raises(ValueError):
        reserve()
    assert len(calls) == 2


def fork(layers, table):
    S.stief_pages_fork(table, layers, i32(3), torch.zeros(1024, dtype=torch.uint8))


@pytest.mark.parametrize("call", ["accept", "fork"])
def test_kept_descriptors_own_no_cache_memory(calls, call):
    """What is kept of a call must not hold the pools: a cache that is replaced is freed at once, without the collector."""
    table = S.PageTable(i32(3, 3), i32(3), i32(3), i32(4))
    run = (lambda ls: accept(ls)) if call == "accept" else (lambda ls: fork(ls, table))
    gc.collect()
    gc.disable()
    try:
        layers = [layer() for _ in range(3)]
        run(layers)
        tree(layers[1])
        old = [weakref.ref(layers[1].k_pool), weakref.ref(layers[0].v_pool)]
        layers[1].k_pool, layers[0].v_pool = torch.zeros(4, 2, 64, 64, dtype=BF), torch.zeros(4, 2, 64, 64, dtype=BF)
        assert [r() for r in old] == [None, None]
        run(layers)
        every = [weakref.ref(x) for l in layers for x in (l, l.k_pool, l.v_pool, l.U_k)]
        del layers
        assert all(r() is None for r in every)
    finally:
        gc.enable()


def pools_of(call, calls):
    """Addresses that the last call was given."""
    name, args = calls[-1]
    if call == "accept":
        return [p for l in args[0] for p in (l.k_pool, l.v_pool)]
    return [p.base for p in args[1]]


@pytest.mark.parametrize("call", ["accept", "fork"])
def test_kept_descriptors_follow_every_change(calls, call):
    table = S.PageTable(i32(3, 3), i32(3), i32(3), i32(4))
    run = (lambda ls: accept(ls)) if call == "accept" else (lambda ls: fork(ls, table))
    layers = [layer() for _ in range(3)]
    now = lambda: [t.data_ptr() for l in layers for t in (l.k_pool, l.v_pool)]
    for change in (lambda: None, lambda: setattr(layers[2], "k_pool", layers[2].k_pool.clone()), lambda: layers[1].v_pool.set_(layers[1].v_pool.clone()),
                   lambda: layers.pop(), lambda: layers.reverse(), lambda: layers.append(layer()), lambda: layers.__setitem__(1, layer())):
        change()
        for _ in range(2):
            run(layers)
            assert pools_of(call, calls) == now()
    seen = len(calls)
    layers[1].k_pool.resize_(3, 2, 64, 64)                     # fewer pages at the same address
    with pytest.raises(ValueError):
        run(layers)
    assert len(calls) == seen


def test_pools_of_a_derived_layer_are_counted_once_each(calls):
    class Named(S.Layer):
        pass

    l = layer()
    layers = [l, Named(l.Hq, l.Hkv, l.r_k, l.r_v, l.U_k, l.U_v, l.k_pool.clone(), l.v_pool.clone())]
    fork(layers, S.PageTable(i32(3, 3), i32(3), i32(3), i32(4)))
    assert calls[-1][1][2] == 4 and len(calls[-1][1][1]) == 4


@pytest.mark.parametrize("stride", [1, 1029, 1 << 40])
def test_an_extent_of_one_may_carry_any_stride(calls, stride):
    l, row = layer(), 8 * 128
    storage = torch.zeros(2 * 4 * row + 64, dtype=BF)
    ws, batch = torch.zeros(16, dtype=torch.uint8), S.Batch(i32(2, 2), i32(2))
    q = storage.as_strided((2, 1, 8, 128), (row, stride, 128, 1))
    S.stief_tree_attention(l, batch, q, i32(2, 1, 1), ws, q)
    args = calls[-1][1]
    assert args[3:5] == (row, row) and args[12:14] == (row, row)
    q = storage.as_strided((1, 3, 8, 128), (stride, row, 128, 1))
    S.stief_tree_attention(l, S.Batch(i32(1, 2), i32(1)), q, i32(1, 3, 1), ws, q)
    args = calls[-1][1]
    assert args[3:5] == (row, row) and args[12:14] == (row, row)
    q = storage.as_strided((1, 8, 128), (stride, 128, 1))
    S.stief_prompt_attention(q, q, q, i32(2), q)
    args = calls[-1][1]
    assert [args[i] for i in (6, 8, 10, 12)] == [row] * 4


def test_pages_are_counted_as_the_descriptors_were_built(calls):
    """A pool reshaped in place to more, smaller pages: ids go by the pages that the kept descriptors know."""
    layers, table = [layer(), layer()], S.PageTable(i32(3, 3), i32(3), i32(3), i32(4))
    fork(layers, table)
    layers[0].k_pool.resize_(8, 2, 32, 64)
    table.ref_counts = i32(8)
    with pytest.raises(ValueError):
        fork(layers, table)
    S.stief_pages_copy(layers, i32(2), i32(2))
    assert calls[-1][1][2] == 4 and len(calls) == 2
