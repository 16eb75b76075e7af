"""CPU-only checks of the rotated appends and of the 8-bit cache's calls: what the C entry points refuse before CUDA is touched, and
what the Python binding lets through to them (the library is replaced by a recorder)."""
import ctypes

import pytest
import torch

import paper_2601_21686_b200 as S
from paper_2601_21686_b200 import build as B

BAD, UNSUP, SMALL = S.STIEF_ERR_INVALID_ARG, S.STIEF_ERR_UNSUPPORTED, S.STIEF_ERR_WORKSPACE
P = 4096                                                       # an aligned address that nobody reads
BF = torch.bfloat16


@pytest.fixture(scope="module")
def lib():
    B.build()
    return S.lib()


def _layer(Hq=8, Hkv=2, d=128, r_k=64, r_v=64, pages=10, U_k=P, U_v=P, k=P, v=P, uk=None, scales=P):
    return S._CLayer(Hq, Hkv, d, r_k, r_v, pages, U_k, 128 * r_k if uk is None else uk, U_v, 128 * r_v, k, v)


def _f8layer(Hq=8, Hkv=2, d=128, r_k=64, r_v=64, pages=10, U_k=P, U_v=P, k=P, v=P, uk=None, scales=P):
    return S._CF8Layer(Hq, Hkv, d, r_k, r_v, pages, U_k, 128 * r_k if uk is None else uk, U_v, 128 * r_v, k, v, scales)


@pytest.mark.parametrize("name,make", [("stief_rope_append", _layer), ("stief_f8_append", _f8layer)])
def test_append_refuses(lib, name, make):
    batch = S._CBatch(2, 4, P, P)

    def call(layer=None, bt=batch, rot=(P, 100, 128, 0), q=P, qs=1024, k=P, ks=256, v=P, vs=256, n=0, cu=P, pos=None, ends=0, out=2 * P, os=1024, **kw):
        l = make(**kw) if layer is None else layer
        r = None if rot is None else ctypes.byref(S._CRotation(*rot))
        return getattr(lib, name)(ctypes.byref(l), ctypes.byref(bt), r, q, qs, k, ks, v, vs, n, cu, pos, ends, out, os, None, None)

    assert call() == call(q=None, out=None, rot=None) == call(q=None, out=None) == call(out=P) == call(rot=(P, 1, 16, 1)) == S.STIEF_OK   # no tokens: nothing to do
    assert call(k=None) == call(v=None) == call(cu=None) == call(n=-1) == call(ends=2) == call(ends=-1) == BAD
    assert call(q=None) == call(out=None) == call(rot=None) == call(out=P, os=2048) == BAD
    assert call(q=P + 2) == call(out=P + 8) == call(k=P + 4) == call(v=P + 8) == call(cu=P + 1) == call(pos=P + 2) == BAD
    assert call(qs=1020) == call(qs=1016) == call(os=512) == call(ks=248) == call(ks=260) == call(vs=128) == BAD
    for rot in ((None, 100, 128, 0), (P + 8, 100, 128, 0), (P, 0, 128, 0), (P, 100, 0, 0), (P, 100, 136, 0), (P, 100, 144, 0), (P, 100, 24, 0), (P, 100, 64, 2)):
        assert call(rot=rot) == BAD
    assert call(Hq=9) == call(pages=0) == call(k=None) == call(U_k=P + 64) == call(uk=-8) == call(uk=4) == BAD
    assert call(layer=make(k=None)) == call(layer=make(v=P + 64)) == call(layer=make(k=P + 16)) == BAD
    assert call(d=64) == call(r_k=40) == call(r_v=160) == UNSUP
    assert call(U_k=None, ks=128) == UNSUP and call(U_k=None, r_k=128) == call(U_k=None, ks=128, rot=None, q=None, out=None) == call(U_v=None, vs=128) == S.STIEF_OK
    assert call(U_v=None, vs=120) == BAD
    assert call(bt=S._CBatch(1025, 4, P, P)) == call(bt=S._CBatch(2, 0, P, P)) == call(bt=S._CBatch(2, 4, None, P)) == BAD
    if make is _f8layer:
        assert call(scales=None) == call(scales=P + 8) == BAD
    assert getattr(lib, name)(None, None, None, None, 0, None, 0, None, 0, 0, None, None, 0, None, 0, None, None) == BAD


def test_decode_attention_refuses(lib):
    ws = S.stief_decode_workspace_bytes(2, 8, 2, 64)

    def call(bt=S._CBatch(2, 4, P, P), q=P, add=0, w=P, wb=ws - 1, parts=0, out=P, flags=0, **kw):
        return lib.stief_f8_decode_attention(ctypes.byref(_f8layer(**kw)), ctypes.byref(bt), q, add, w, wb, parts, out, None, flags, None, None)

    assert call() == SMALL
    assert call(q=None) == call(out=None) == call(w=None) == call(w=P + 64) == call(q=P + 8) == call(out=P + 8) == call(add=2) == call(add=-1) == BAD
    assert call(flags=2) == call(parts=-1) == call(parts=1 << 16) == call(bt=S._CBatch(2, 0, P, P)) == call(bt=S._CBatch(1025, 1, P, P)) == BAD
    assert call(Hq=9) == call(k=P + 64) == call(v=None) == call(scales=None) == call(U_k=P + 32) == call(uk=32) == call(pages=1 << 25) == BAD
    assert call(d=64) == call(r_k=16) == call(r_v=80) == UNSUP


def test_run_attention_refuses_and_plans(lib):
    need = S.stief_f8_mq_workspace_bytes(2, 8, 8, 64, 4)
    assert need >= 2 * 8 * 8 * 2 * 4 * 66 * 4 and S.stief_f8_mq_workspace_bytes(2, 8, 8, 64, 1) == 0 == S.stief_f8_mq_workspace_bytes(2, 8, 8, 64, 0)
    assert S.stief_f8_mq_num_splits(1, 4, 10, 2, 1000) >= 1 and S.stief_f8_mq_num_splits(1, 4, 129, 1, 10) == 0 == S.stief_f8_mq_num_splits(1, 0, 8, 2, 10)
    assert S.stief_f8_mq_num_splits(1, 65536, 1, 1, 2 ** 31 - 1) == 1 and 1 <= S.stief_f8_mq_num_splits(1, 65535, 1, 1, 2 ** 31 - 1) <= 32
    assert S.stief_f8_mq_num_splits(8, 4096, 32, 8, 1000) == 1 and S.stief_f8_mq_num_splits(1, 2 ** 31 - 1, 32, 8, 1000) == 1

    def call(bt=S._CBatch(2, 4, P, P), q=P, sb=8 * 1024, st=1024, n=8, w=P, wb=need - 1, splits=4, out=P, ob=8 * 1024, ot=1024, flags=0, **kw):
        return lib.stief_f8_mq_attention(ctypes.byref(_f8layer(**kw)), ctypes.byref(bt), q, sb, st, n, None, w, wb, splits, out, ob, ot, None, flags, None, None)

    assert call() == SMALL
    assert call(q=None) == call(out=None) == call(w=None) == call(w=P + 64) == call(n=0) == call(splits=0) == call(splits=33) == call(flags=1) == BAD
    for kw in ({"q": P + 8}, {"out": P + 8}, {"sb": 8}, {"st": 1020}, {"st": 512}, {"ob": 1016}, {"ot": 8}, {"Hq": 9}, {"pages": 1 << 25}, {"scales": P + 4}, {"v": P + 64}):
        assert call(wb=need, splits=1, **kw) == BAD, kw
    assert call(d=64, splits=1) == call(r_k=16, splits=1) == call(Hq=258, sb=1 << 20, st=258 * 128, ob=1 << 20, ot=258 * 128, splits=1) == UNSUP


# ------------------------------------------------------------------------------------------------- the binding
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
    rec = Recorder()
    monkeypatch.setattr(S, "lib", lambda: rec)
    monkeypatch.setattr(S, "_here", lambda t, name, device=None: 0)
    monkeypatch.setattr(S, "_raw_stream", lambda device: 0)
    return rec.calls


def i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def bf(*shape):
    return torch.zeros(*shape, dtype=BF)


def f8(Hq=8, Hkv=2, r_k=64, r_v=64, pages=4):
    codes = lambda r: torch.zeros(pages, Hkv, 64, r, dtype=torch.uint8)  # noqa: E731
    return S.F8Layer(Hq, Hkv, r_k, r_v, bf(Hkv, 128, r_k), bf(Hkv, 128, r_v), codes(r_k), codes(r_v), torch.zeros(pages, Hkv, 4))


def plain(Hq=8, Hkv=2, r_k=64, r_v=64, pages=4):
    return S.Layer(Hq, Hkv, r_k, r_v, bf(Hkv, 128, r_k), bf(Hkv, 128, r_v), bf(pages, Hkv, 64, r_k), bf(pages, Hkv, 64, r_v))


def append(layer, batch=None, k=None, v=None, cu=None, **kw):
    call = S.stief_f8_append if isinstance(layer, S.F8Layer) else S.stief_rope_append
    kw.setdefault("rotation", S.Rotation(torch.zeros(50, 128)))
    call(layer, S.Batch(i32(2, 3), i32(2)) if batch is None else batch, bf(5, 2, 128) if k is None else k, bf(5, 2, 128) if v is None else v,
         i32(3) if cu is None else cu, **kw)


@pytest.mark.parametrize("make", [f8, plain])
def test_append_binding_of_no_tokens(lib, calls, make):
    """A step without new tokens: empty tensors have no address, which the entry points refuse.  What the binding hands over is taken."""
    for kw in (dict(), dict(q=bf(0, 8, 128), q_out=bf(0, 8, 128)), dict(rotation=None)):
        l = make()
        append(l, k=bf(0, 2, 128), v=bf(0, 2, 128), **kw)
        name, args = calls[-1]
        assert args[9] == 0 and args[5] and args[7] and bool(args[3]) == bool(args[13]) == ("q" in kw)
        c = args[0]._obj
        for field in ("U_k", "U_v", "k_pool", "v_pool", "k_codes", "v_codes", "scales"):
            if hasattr(c, field):
                setattr(c, field, P)                             # (host memory need not be aligned)
        aligned = lambda x: P if x else None  # noqa: E731
        assert getattr(lib, name)(*args[:3], aligned(args[3]), args[4], aligned(args[5]), args[6], aligned(args[7]), *args[8:13], aligned(args[13]), *args[14:]) == S.STIEF_OK


@pytest.mark.parametrize("make", [f8, plain])
def test_append_binding(calls, make):
    wide = bf(5, 12, 128)
    append(make(), k=wide[:, 8:10], v=wide[:, 10:], q=wide[:, :8], q_out=bf(5, 8, 128), positions=i32(5))
    (_, args), = calls
    assert args[4] == 12 * 128 and args[6] == args[8] == 12 * 128 and args[9] == 5 and args[14] == 8 * 128
    refused = [
        dict(k=bf(5, 3, 128)), dict(k=bf(5, 2, 64)), dict(v=bf(4, 2, 128)), dict(k=torch.zeros(5, 2, 128)), dict(k=bf(5, 128, 2).transpose(1, 2)),
        dict(k=bf(5, 2, 256)[..., ::2]), dict(q=bf(5, 8, 128)), dict(q_out=bf(5, 8, 128)), dict(q=bf(5, 8, 128), q_out=bf(5, 4, 128)),
        dict(q=bf(5, 8, 64), q_out=bf(5, 8, 64)), dict(positions=i32(4)), dict(positions=torch.zeros(5, dtype=torch.int64)), dict(cu=i32(2)),
        dict(cu=torch.zeros(3)), dict(batch=S.Batch(i32(2, 3), i32(3))), dict(batch=S.Batch(i32(3, 2).T, i32(2))), dict(status=torch.zeros(1)),
        dict(rotation=S.Rotation(torch.zeros(50, 128, dtype=BF))), dict(rotation=S.Rotation(torch.zeros(50, 256)[:, ::2])), dict(rotation=S.Rotation(torch.zeros(128))),
    ]
    for kw in refused:
        with pytest.raises(ValueError):
            append(make(), **kw)
    with pytest.raises(ValueError):
        (S.stief_rope_append if make is f8 else S.stief_f8_append)(make(), S.Batch(i32(2, 3), i32(2)), bf(5, 2, 128), bf(5, 2, 128), i32(3))
    assert len(calls) == 1


def decode(l):
    S.stief_f8_decode_attention(l, S.Batch(i32(2, 3), i32(2)), bf(2, l.Hq, 128), torch.zeros(1 << 10, dtype=torch.uint8), bf(2, l.Hq, 128))


def attend(l):
    S.stief_f8_mq_attention(l, S.Batch(i32(2, 3), i32(2)), bf(2, 4, l.Hq, 128), bf(2, 4, l.Hq, 128))


CHANGES = {
    "smaller key rank": lambda l: setattr(l, "r_k", 32), "larger value rank": lambda l: setattr(l, "r_v", 96), "more heads": lambda l: setattr(l, "Hkv", 4),
    "codes resized in place": lambda l: l.k_codes.resize_(4, 2, 32, 64), "codes re-laid in place": lambda l: l.v_codes.transpose_(2, 3),
    "codes of another type": lambda l: setattr(l, "k_codes", l.k_codes.view(torch.int8)), "fewer value pages": lambda l: setattr(l, "v_codes", l.v_codes[:3]),
    "fewer scales": lambda l: setattr(l, "scales", l.scales[:3]), "scales of one word": lambda l: setattr(l, "scales", torch.zeros(4, 2, 1)),
    "scales in bf16": lambda l: setattr(l, "scales", l.scales.to(BF)), "basis resized in place": lambda l: l.U_k.resize_(2, 64, 64),
    "basis in fp32": lambda l: setattr(l, "U_v", l.U_v.float()), "strided basis": lambda l: setattr(l, "U_k", bf(2, 128, 128)[..., ::2]),
}


@pytest.mark.parametrize("change", CHANGES)
@pytest.mark.parametrize("call", [append, decode, attend])
def test_the_8_bit_layer_is_looked_at_in_every_call(calls, call, change):
    l = f8()
    call(l)
    call(l)
    assert len(calls) == 2
    CHANGES[change](l)
    with pytest.raises(ValueError):
        call(l)
    assert len(calls) == 2


def test_replaced_tensors_reach_the_library(calls):
    l = f8()
    for name in ("k_codes", "v_codes", "scales", "U_k", "U_v"):
        decode(l)
        setattr(l, name, getattr(l, name).clone())
        decode(l)
        c = calls[-1][1][0]._obj
        assert getattr(c, name) == getattr(l, name).data_ptr()
    l.U_k = l.U_k[:1]
    decode(l)
    assert calls[-1][1][0]._obj.uk_head_stride == 0
    l.k_codes, l.v_codes = l.k_codes.view(torch.float8_e4m3fn), l.v_codes.view(torch.float8_e4m3fn)
    decode(l)


def test_attention_bindings_refuse(calls):
    l, batch, ws = f8(), S.Batch(i32(2, 3), i32(2)), torch.zeros(1 << 10, dtype=torch.uint8)
    ok = dict(q=bf(2, 8, 128), workspace=ws, out=bf(2, 8, 128))
    S.stief_f8_decode_attention(l, batch, **ok)
    for kw in (dict(q=bf(3, 8, 128)), dict(q=bf(2, 8, 64)), dict(q=bf(2, 8, 256)[..., ::2]), dict(out=bf(2, 4, 128)), dict(out=torch.zeros(2, 8, 128)),
               dict(out_lse=torch.zeros(2, 4)), dict(out_lse=bf(2, 8)), dict(workspace=torch.zeros(64, 64)[:, :32]), dict(status=torch.zeros(1))):
        with pytest.raises(ValueError):
            S.stief_f8_decode_attention(l, batch, **{**ok, **kw})
    ok = dict(q=bf(2, 4, 8, 128), out=bf(2, 4, 8, 128))
    S.stief_f8_mq_attention(l, batch, **ok)
    S.stief_f8_mq_attention(l, batch, q=bf(4, 2, 8, 128).transpose(0, 1), out=bf(2, 4, 16, 128)[:, :, :8], q_lens=i32(2))
    for kw in (dict(q=bf(2, 4, 4, 128)), dict(q=bf(3, 4, 8, 128)), dict(q=bf(2, 8, 4, 128).transpose(1, 2)), dict(out=bf(2, 4, 8, 64)), dict(q_lens=i32(3)),
               dict(q_lens=torch.zeros(2)), dict(out_lse=torch.zeros(2, 4)), dict(workspace=torch.zeros(64, 64)[:, :32]), dict(status=torch.zeros(1))):
        with pytest.raises(ValueError):
            S.stief_f8_mq_attention(l, batch, **{**ok, **kw})
    with pytest.raises(ValueError):
        S.stief_f8_mq_attention(plain(), batch, **ok)
    assert len(calls) == 3


def test_page_calls_take_the_8_bit_layer(calls):
    table = S.PageTable(i32(3, 3), i32(3), i32(3), i32(4))
    l = f8()
    S.stief_pages_fork(table, [l], i32(3), torch.zeros(128, dtype=torch.uint8))
    pools = calls[-1][1][1]
    assert [(p.base, p.page_bytes) for p in pools] == [(l.k_codes.data_ptr(), 2 * 64 * 64), (l.v_codes.data_ptr(), 2 * 64 * 64), (l.scales.data_ptr(), 32)]
    l.scales = l.scales[:3]
    with pytest.raises(ValueError):
        S.stief_pages_copy([l], i32(1), i32(1))
    with pytest.raises(ValueError):
        S.stief_tree_accept([f8()], S.Batch(i32(2, 2), i32(2)), i32(2, 3), i32(2))
