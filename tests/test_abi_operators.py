"""CPU-only checks of the tree, prompt and page entry points: what the host refuses comes back before CUDA is touched."""
import ctypes

import pytest
import torch

import paper_2601_21686_b200 as S
from paper_2601_21686_b200 import build as B

BAD, UNSUP, SMALL = S.STIEF_ERR_INVALID_ARG, S.STIEF_ERR_UNSUPPORTED, S.STIEF_ERR_WORKSPACE
P = 4096                                                       # an aligned address that nobody reads


@pytest.fixture(scope="module")
def lib():
    B.build()
    return S.lib()


def _layer(Hq=8, Hkv=2, d=128, r_k=64, r_v=64, pages=10, k=P, v=P):
    return S._CLayer(Hq, Hkv, d, r_k, r_v, pages, P, 128 * r_k, P, 128 * r_v, k, v)


def test_tree_attention_refuses(lib):
    ws = S.stief_tree_workspace_bytes(2, 8, 8, 2, 64)
    assert ws > 0 and S.stief_tree_workspace_bytes(2, 8, 8, 3, 64) == 0 and S.stief_tree_workspace_bytes(0, 8, 8, 2, 64) == 0
    batch = S._CBatch(2, 4, P, P)

    def call(layer=_layer(), q=P, sb=8 * 1024, st=1024, n=8, mask=P, words=1, w=P, wb=ws, out=P, flags=0, bt=batch):
        return lib.stief_tree_attention(ctypes.byref(layer), ctypes.byref(bt), q, sb, st, n, None, mask, words, w, wb, out, sb, st, None, flags, None, None)

    assert call(q=None) == call(mask=None) == call(out=None) == call(w=None) == call(flags=1) == call(words=0) == call(n=0) == BAD
    assert call(q=P + 2) == call(st=1020) == call(st=512) == call(sb=8) == call(w=P + 64) == BAD
    assert call(layer=_layer(Hq=9)) == call(layer=_layer(k=None)) == call(layer=_layer(k=P + 16)) == call(layer=_layer(pages=1 << 25)) == BAD
    assert call(layer=_layer(d=64)) == call(layer=_layer(r_k=40)) == call(layer=_layer(r_v=160)) == UNSUP
    assert call(n=1025, words=40) == UNSUP and call(wb=ws - 128) == SMALL
    assert call(bt=S._CBatch(1025, 4, P, P)) == call(bt=S._CBatch(2, 0, P, P)) == BAD
    assert lib.stief_tree_attention(None, None, None, 0, 0, 0, None, None, 0, None, 0, None, 0, 0, None, 0, None, None) == BAD


def test_tree_accept_refuses(lib):
    batch = S._CBatch(2, 4, P, P)
    two = (S._CLayer * 2)(_layer(v=2 * P), _layer(pages=11))

    def call(layers=two, n=1, acc=P, most=4, cnt=P):
        return lib.stief_tree_accept(layers, n, ctypes.byref(batch), acc, most, cnt, None, None)

    assert call(layers=None) == call(n=0) == call(acc=None) == call(most=0) == call(cnt=None) == call(n=2) == BAD
    assert call(layers=(S._CLayer * 1)(_layer(r_k=33))) == UNSUP
    assert call(layers=(S._CLayer * 1)(_layer())) == BAD                                     # one pool for keys and values
    for n in (3, 300):                                                                       # the last layer's pool is the first's
        ls = (S._CLayer * n)(*[_layer(k=P * (2 * i + 1), v=P * (2 * i + 2)) for i in range(n - 1)], _layer(k=P * (2 * n + 1), v=P))
        assert call(layers=ls, n=n) == BAD
    assert lib.stief_advance_seq_lens_by(None, P, 4, None) == lib.stief_advance_seq_lens_by(P, P, 0, None) == BAD


def test_prompt_attention_refuses(lib):
    def call(Hq=8, Hkv=2, n=2, total=64, cu=P, q=P, qs=1024, k=P, ks=256, v=P, vs=256, out=P, os=1024, flags=0):
        return lib.stief_prompt_attention(Hq, Hkv, n, total, cu, q, qs, k, ks, v, vs, out, os, None, flags, None, None)

    assert call(Hq=9) == call(Hkv=0) == call(n=0) == call(n=1025) == call(total=-1) == call(cu=None) == call(flags=2) == BAD
    assert call(q=None) == call(k=None) == call(v=None) == call(out=None) == call(q=P + 8) == call(k=P + 4) == call(out=P + 2) == BAD
    assert call(qs=1023) == call(qs=1028) == call(ks=255) == call(vs=248) == call(os=512) == BAD
    assert call(total=0, q=None) == S.STIEF_OK


def test_page_calls_refuse(lib):
    good = S._CPageTable(4, 8, 100, P, P, P, P)
    pool = (S._CPagePool * 1)(S._CPagePool(P, 8192))
    need = S.stief_pages_workspace_bytes(4, 8)
    assert need > 0 and S.stief_pages_workspace_bytes(0, 8) == 0 and S.stief_pages_workspace_bytes(1025, 8) == 0

    def fork(t=good, pools=pool, n=1, parent=P, ws=P, wb=need):
        return lib.stief_pages_fork(ctypes.byref(t), pools, n, parent, ws, wb, None, None)

    for t in (S._CPageTable(0, 8, 100, P, P, P, P), S._CPageTable(1025, 8, 100, P, P, P, P), S._CPageTable(4, 0, 100, P, P, P, P),
              S._CPageTable(4, 8, 0, P, P, P, P), S._CPageTable(4, 8, (1 << 30) + 1, P, P, P, P), S._CPageTable(1024, (1 << 20) + 1, 100, P, P, P, P), S._CPageTable(4, 8, 100, None, P, P, P), S._CPageTable(4, 8, 100, P, P, P, None)):
        assert fork(t=t) == lib.stief_pages_reserve(ctypes.byref(t), P, 0, None, None) == BAD
    assert fork(pools=None) == fork(n=-1) == fork(parent=None) == fork(ws=None) == fork(ws=P + 4) == BAD
    assert fork(wb=need - 4) == SMALL
    for bad in (S._CPagePool(None, 8192), S._CPagePool(P + 8, 8192), S._CPagePool(P, 0), S._CPagePool(P, 8200)):
        arr = (S._CPagePool * 1)(bad)
        assert fork(pools=arr) == lib.stief_pages_copy(arr, 1, 100, P, P, 3, None, None) == BAD
    assert lib.stief_pages_copy(pool, 1, 100, None, P, 3, None, None) == lib.stief_pages_copy(pool, 0, 100, P, P, 3, None, None) == BAD
    assert lib.stief_pages_copy(pool, 1, 100, P, P, -1, None, None) == BAD and lib.stief_pages_copy(pool, 1, 100, None, None, 0, None, None) == S.STIEF_OK
    assert lib.stief_pages_reserve(ctypes.byref(good), None, -1, None, None) == BAD
    assert "pages" in S.status_string(S.STIEF_ERR_NO_PAGES)


def test_tensors_of_the_host_are_refused():
    t = torch.zeros(4, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        S.stief_prompt_attention(t, t, t, torch.zeros(2, dtype=torch.int32), t)
    with pytest.raises(ValueError):
        S.stief_advance_seq_lens_by(torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))


def test_descriptors_follow_the_tensors():
    """A view at the same address with another size or stride is another descriptor."""
    U, pool = torch.zeros(2, 128, 64, dtype=torch.bfloat16), torch.zeros(10, 2, 64, 64, dtype=torch.bfloat16)
    layer = S.Layer(8, 2, 64, 64, U, U, pool, pool.clone())
    assert layer.c().num_pages == 10 and layer.c().uk_head_stride == 128 * 64
    layer.k_pool, layer.U_k = pool[:5], U[:1]
    assert layer.c().num_pages == 5 and layer.c().uk_head_stride == 0 and layer.c().uv_head_stride == 128 * 64
