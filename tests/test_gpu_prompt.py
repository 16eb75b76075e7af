"""Causal attention over packed prompts against the definition in fp64.  Tolerance: the probabilities are rounded to bf16
(half a step, 2^-8) and so is the output; scores are exact products summed in fp32, exponentials good to 1e-4."""
import math

import pytest
import torch

import paper_2601_21686_b200 as S

pytestmark = pytest.mark.gpu
HALF = torch.finfo(torch.bfloat16).eps / 2
NAN = float("nan")


def _inputs(seed, lens, Hq, Hkv, q_scale=2.0, gap=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    total = sum(lens) + gap
    qkv = torch.randn(total, Hq + 2 * Hkv, 128, generator=g, device="cuda")
    qkv[:, :Hq] *= q_scale
    qkv = qkv.to(torch.bfloat16)
    cu = torch.zeros(len(lens) + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(torch.tensor(lens), 0)
    return qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], cu.cuda()


def _run(q, k, v, cu, lse=True):
    out = torch.full((q.shape[0], q.shape[1], 128), NAN, dtype=torch.bfloat16, device="cuda")
    out_lse = torch.full(q.shape[:2], NAN, dtype=torch.float32, device="cuda") if lse else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    S.stief_prompt_attention(q, k, v, cu, out, out_lse=out_lse, status=status)
    assert int(status) == 0
    return out, out_lse


def _check(q, k, v, cu, out, out_lse=None, heads=None, rows=None):
    G = q.shape[1] // k.shape[1]
    c = cu.tolist()
    for lo, hi in zip(c[:-1], c[1:]):
        if lo == hi:
            continue
        at = torch.arange(lo, hi, device="cuda")
        if rows is not None and hi - lo > rows:
            pick = torch.randperm(hi - lo, generator=torch.Generator().manual_seed(hi))[:rows]
            pick[:4] = torch.tensor([0, 127, 128, hi - lo - 1])
            at = lo + pick.cuda()
        for g in heads if heads is not None else range(q.shape[1]):
            K, V = k[lo:hi, g // G].double(), v[lo:hi, g // G].double()
            Q = q[at, g].double()
            s = (Q @ K.T / math.sqrt(128)).masked_fill(torch.arange(lo, hi, device="cuda")[None] > at[:, None], -math.inf)
            lse = torch.logsumexp(s, -1)
            p = torch.exp(s - lse[:, None])
            o, size = p @ V, p @ V.abs()
            delta = 256 * 2.0 ** -24 * (Q.abs() @ K.abs().T).amax(-1) / math.sqrt(128)
            bound = (HALF + 3e-4 + torch.expm1(2 * delta)[:, None]) * size + HALF * o.abs() + 1e-6
            got = out[at, g].double()
            assert torch.isfinite(got).all()
            worst = ((got - o).abs() / bound).max().item()
            assert worst <= 1.0, f"prompt at {lo}, head {g}: {worst:.2f} of the bound"
            if out_lse is not None:
                err = (out_lse[at, g].double() - lse).abs() / (2e-4 + delta + 1e-6 * lse.abs())
                assert err.max().item() <= 1.0
    assert torch.isnan(out[c[-1]:]).all() and (out_lse is None or torch.isnan(out_lse[c[-1]:]).all())


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 1), (6, 2), (3, 3), (5, 1), (16, 2)])
@pytest.mark.parametrize("lens", [[1], [2], [127], [128], [129], [255, 256, 257], [1, 300, 64, 0, 17, 513], [700]])
def test_lengths_and_head_groups(lens, Hq, Hkv):
    x = _inputs(sum(lens) * 7 + Hq, lens, Hq, Hkv)
    _check(*x, *_run(*x))


def test_many_short_prompts():
    lens = [(i * 29) % 70 for i in range(300)]
    x = _inputs(3, lens, 4, 2)
    _check(*x, *_run(*x), heads=[0, 3])


@pytest.mark.parametrize("n", [1024, 1023])
def test_largest_number_of_prompts(n):
    x = _inputs(9, [1 + (i % 3) for i in range(n)], 2, 1)
    _check(*x, *_run(*x), heads=[1])


def test_long_prompts():
    x = _inputs(11, [5000, 33, 2049], 8, 2)
    _check(*x, *_run(*x), heads=[0, 5], rows=300)


def test_growing_scores_rescale():
    q, k, v, cu = _inputs(13, [1500], 2, 1, q_scale=0.1)
    k[:, 0, 0] = torch.linspace(0, 40, 1500, device="cuda").to(torch.bfloat16)
    q[:, 0, 0], q[:, 1, 0] = 20.0, -20.0
    _check(q, k, v, cu, *_run(q, k, v, cu))


@pytest.mark.parametrize("exponent", [-9, -2, 4, 8, 13, 16, 19, 24, 28, 30, 31, 60, 100, 120])
def test_scores_far_from_zero(exponent):
    """Scores that are exact in fp32 (19 bits), of sizes up to 2^125 and either sign: nothing but the rounding of probabilities and
    output remains.  In large ones the largest score's ties share the row."""
    q, k, v, cu = _inputs(43 + exponent, [700, 1, 90], 4, 2)
    q.zero_(), k.zero_()
    for i in range(2):
        k[..., i] = (1 + torch.randint(0, 64, k.shape[:2], generator=torch.Generator().manual_seed(5 + i)).cuda() / 64).to(torch.bfloat16)
    q[:, ::2, 0], q[:, 1::2, 0] = 2.0 ** exponent * 4, -2.0 ** exponent * 4      # odd heads: all scores far below zero
    q[..., 1] = q[..., 0] * 2.0 ** -12                         # and scores close to one another
    out, lse = _run(q, k, v, cu)
    for lo, hi in zip(cu.tolist()[:-1], cu.tolist()[1:]):
        past = torch.ones(hi - lo, hi - lo, dtype=torch.bool, device="cuda").tril()
        for g in range(4):
            s = (q[lo:hi, g].double() @ k[lo:hi, g // 2].double().T / math.sqrt(128)).masked_fill(~past, -math.inf)
            want_lse = torch.logsumexp(s, -1)
            p, V = torch.softmax(s, -1), v[lo:hi, g // 2].double()          # (the lse of far scores has lost the number of ties)
            o, size = p @ V, p @ V.abs()
            # what the rounding of a reference does to its row's exponents, it does to all alike
            bound = (HALF + 3e-4) * size + HALF * o.abs() + 1e-6
            err = (out[lo:hi, g].double() - o).abs()
            assert torch.isfinite(err).all() and (err <= bound).all(), f"prompt at {lo}, head {g}: {(err / bound).max().item():.2f} of the bound"
            assert ((lse[lo:hi, g].double() - want_lse).abs() <= 2e-4 + 1e-6 * want_lse.abs()).all()


def test_separate_contiguous_tensors_and_strided_output():
    q, k, v, cu = (t.contiguous() for t in _inputs(17, [200, 90], 4, 2))
    buf = torch.full((290, 7, 128), NAN, dtype=torch.bfloat16, device="cuda")
    out = buf[:, 1:5]
    S.stief_prompt_attention(q, k, v, cu, out)
    _check(q, k, v, cu, out)
    assert torch.isnan(buf[:, 0]).all() and torch.isnan(buf[:, 5:]).all()


def test_rows_of_other_prompts_and_of_none_influence_nothing():
    lens = [100, 60, 200]
    q, k, v, cu = _inputs(19, lens, 4, 2, gap=40)
    k[360:], v[360:], q[360:] = NAN, NAN, NAN
    q[100:160], k[100:160], v[100:160] = NAN, math.inf, NAN    # the middle prompt is poisoned
    out, lse = _run(q, k, v, cu)
    keep = torch.tensor([0, 100], dtype=torch.int32, device="cuda")
    _check(q[:100], k[:100], v[:100], keep, out[:100], lse[:100])
    _check(q[160:360], k[160:360], v[160:360], keep * 2, out[160:360], lse[160:360])
    assert torch.isnan(out[360:]).all() and torch.isnan(lse[360:]).all()


def test_only_empty_prompts():
    q, k, v, _ = _inputs(21, [64], 4, 2)
    out, lse = _run(q, k, v, torch.zeros(4, dtype=torch.int32, device="cuda"))
    assert torch.isnan(out).all() and torch.isnan(lse).all()


def test_later_tokens_do_not_change_earlier_rows():
    q, k, v, cu = _inputs(23, [400], 4, 2)
    a, _ = _run(q, k, v, cu)
    k[333:], v[333:] = 100.0, -1e30
    b, _ = _run(q, k, v, cu)
    assert torch.equal(a[:333], b[:333])


def test_bad_boundaries_are_reported():
    q, k, v, cu = _inputs(29, [100, 60, 40], 4, 2)
    want, _ = _run(q, k, v, cu)
    for bad in ([0, 100, 90, 200], [0, 100, 160, 201], [-3, 100, 160, 200], [0, 100, 160, 2 ** 31 - 1]):
        out = torch.full_like(want, NAN)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        S.stief_prompt_attention(q, k, v, torch.tensor(bad, dtype=torch.int32, device="cuda"), out, status=status)
        assert int(status) == S.STIEF_ERR_BOUNDS
        if bad[0] == 0:
            assert torch.equal(out[:90], want[:90])


def test_repeats_streams_and_graphs_give_the_same_bits():
    q, k, v, cu = _inputs(31, [1000, 1, 300], 8, 2)
    want, _ = _run(q, k, v, cu)
    for _ in range(3):
        assert torch.equal(_run(q, k, v, cu)[0], want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = _run(q, k, v, cu)[0]
        b = _run(q, k, v, cu)[0]
    side.synchronize()
    assert torch.equal(a, want) and torch.equal(b, want)
    out = torch.zeros_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.stief_prompt_attention(q, k, v, cu, out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    cu.copy_(torch.tensor([0, 700, 700, 1301], dtype=torch.int32))       # the captured call serves other boundaries
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    _check(q, k, v, cu, out)


def test_two_streams_at_once():
    xs = [_inputs(37 + i, [900, 300], 8, 2) for i in range(2)]
    want = [_run(*x)[0] for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    outs = [torch.zeros_like(w) for w in want]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, x, o in zip(streams, xs, outs):
            with torch.cuda.stream(s):
                S.stief_prompt_attention(*x, o)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_refusals_and_no_tokens():
    q, k, v, cu = _inputs(41, [64], 4, 2)
    out = torch.empty(64, 4, 128, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(q=q.float()), dict(k=k[:, :, :64]), dict(v=v[:32]), dict(out=out[:, :2]), dict(cu_seqlens=cu.long()), dict(cu_seqlens=cu[:1]),
                dict(q=q.cpu()), dict(k=k.transpose(0, 1)), dict(out_lse=torch.empty(64, 2, device="cuda"))):
        with pytest.raises(ValueError):
            S.stief_prompt_attention(**(dict(q=q, k=k, v=v, cu_seqlens=cu, out=out) | bad))
    with pytest.raises(S.StiefError):
        S.stief_prompt_attention(q[:, :3], k, v, cu, out[:, :3])             # 3 query heads over 2
    none = torch.zeros(3, dtype=torch.int32, device="cuda")
    S.stief_prompt_attention(q[:0], k[:0], v[:0], none, out[:0])
    torch.cuda.synchronize()
