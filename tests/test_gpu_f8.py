"""Attention over the 8-bit cache, against the definition in fp64 on the values that its codes stand for.  Tolerances are error
bounds: the decode call's q' is two f16 terms (2^-22 of the row's largest), the run call's one (2^-11 of the value, or 2^-25 of
the row's largest); the probabilities are rounded to f16 once (2^-11), the output to bf16 (2^-8) after a mix that keeps 16 bits;
everything else is fp32 (and exponentials good to 3e-5)."""
import math

import pytest
import torch

import paper_2601_21686_b200 as S

pytestmark = pytest.mark.gpu
BF, F8 = torch.bfloat16, torch.float8_e4m3fn
HALF = torch.finfo(BF).eps / 2
HALF16 = torch.finfo(torch.float16).eps / 2
NAN = float("nan")


class Case:
    """Rows behind a sequence's end, pages of nobody and unused scales are NaN."""

    def __init__(self, seed, lens, n=None, counts=None, Hq=8, Hkv=2, r_k=64, r_v=64, fold_k=False, fold_v=False, shared=False, q_scale=2.0, spare=3,
                 exponents=(-8, -4), extra=0, token_major=False):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        c = torch.Generator()
        c.manual_seed(seed)
        self.lens, self.n = list(lens), n
        B = len(lens)
        self.counts = [1] * B if n is None else [min(n, t) for t in lens] if counts is None else list(counts)
        pages = [(t + extra + 63) // 64 for t in self.lens]
        P = sum(pages) + spare
        order = torch.randperm(P, generator=c)
        table = torch.full((B, max(max(pages), 1)), -3, dtype=torch.int32)
        codes = [torch.full((P, Hkv, 64, r), 0x7F, dtype=torch.uint8, device="cuda") for r in (r_k, r_v)]
        scales = torch.full((P, Hkv, 4), NAN, device="cuda")
        self.K, self.V, at = [], [], 0
        for b, t in enumerate(self.lens):
            ids = order[at:at + pages[b]]
            table[b, :pages[b]] = ids.to(torch.int32)
            at += pages[b]
            both = []
            for i, r in enumerate((r_k, r_v)):
                x = (80 * torch.randn(pages[b], Hkv, 64, r, generator=g, device="cuda")).clamp(-448, 448).to(F8)
                s = torch.exp2(torch.randint(exponents[0], exponents[1] + 1, (pages[b], Hkv), generator=c).float()).cuda()
                both.append((x.double() * s[:, :, None, None]).transpose(1, 2).reshape(-1, Hkv, r)[:t])
                x = x.view(torch.uint8)
                if t % 64 and pages[b]:
                    x[t // 64, :, t % 64:] = 0x7F
                codes[i][ids.cuda()] = x
                scales[ids.cuda(), :, i] = s
            self.K.append(both[0])
            self.V.append(both[1])
        nb = 1 if shared else Hkv
        basis = lambda r: torch.linalg.qr(torch.randn(nb, 128, 128, generator=g, device="cuda", dtype=torch.float64))[0][:, :, :r].to(BF).contiguous()  # noqa: E731
        self.layer = S.F8Layer(Hq, Hkv, r_k, r_v, None if fold_k else basis(r_k), None if fold_v else basis(r_v), *codes, scales)
        self.batch = S.Batch(table.cuda(), torch.tensor(self.lens, dtype=torch.int32, device="cuda"))
        rows = 1 if n is None else n
        d_q, self.d_out = r_k if fold_k else 128, r_v if fold_v else 128
        self.q = (q_scale * torch.randn(B, rows, Hq, d_q, generator=g, device="cuda")).to(BF)
        self.out = torch.full((B, rows, Hq, self.d_out), NAN, dtype=BF, device="cuda")
        if token_major:
            self.q = self.q.transpose(0, 1).contiguous().transpose(0, 1)
            self.out = self.out.transpose(0, 1).contiguous().transpose(0, 1)
        self.lse = torch.full((B, rows, Hq), NAN, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def decode(self, parts=0, len_add=0, flags=0, workspace=None):
        L, B = self.layer, len(self.lens)
        if workspace is None:
            workspace = torch.full((S.stief_decode_workspace_bytes(B, L.Hq, L.Hkv, L.r_v, parts),), 0xFF, dtype=torch.uint8, device="cuda")
            S.stief_decode_workspace_init(workspace)
        self.workspace = workspace
        S.stief_f8_decode_attention(L, self.batch, self.q[:, 0], workspace, self.out[:, 0], num_parts=parts, out_lse=self.lse[:, 0], len_add=len_add,
                                    status=self.status, flags=flags)
        return self

    def attend(self, splits=None, counts=True):
        L, B = self.layer, len(self.lens)
        if splits is None:
            splits = S.stief_f8_mq_num_splits(B, self.n, L.Hq, L.Hkv, self.batch.block_table.shape[1])
        ws = torch.full((max(128, S.stief_f8_mq_workspace_bytes(B, self.n, L.Hq, L.r_v, splits)),), 0xFF, dtype=torch.uint8, device="cuda")
        S.stief_f8_mq_attention(L, self.batch, self.q, self.out, q_lens=torch.tensor(self.counts, dtype=torch.int32, device="cuda") if counts else None,
                                out_lse=self.lse, status=self.status, workspace=ws, num_splits=splits)
        return self

    def check(self, status=0, skip=()):
        torch.cuda.synchronize()
        assert self.status.item() == status
        L, G, decode = self.layer, self.layer.Hq // self.layer.Hkv, self.n is None
        for b, (t, m) in enumerate(zip(self.lens, self.counts)):
            if b in skip:
                assert torch.isnan(self.out[b]).all()
                continue
            assert torch.isnan(self.out[b, m:]).all() and torch.isnan(self.lse[b, m:]).all(), "rows behind the last were written"
            if t == 0:
                assert (self.out[b, :m] == 0).all() and (self.lse[b, :m] == -math.inf).all()
                continue
            if m == 0:
                continue
            future = torch.ones(m, t, dtype=torch.bool, device="cuda").triu(t - m + 1)[:, None]
            for h in range(L.Hkv):
                Uk = None if L.U_k is None else L.U_k[h if L.U_k.shape[0] > 1 else 0].double()
                Uv = None if L.U_v is None else L.U_v[h if L.U_v.shape[0] > 1 else 0].double()
                K, V = self.K[b][:, h], self.V[b][:, h]
                q = self.q[b, :m, h * G:h * G + G].double()
                qp, q_sum = (q, q.abs()) if Uk is None else (q @ Uk, q.abs() @ Uk.abs())
                s = (qp @ K.T / math.sqrt(128)).masked_fill(future, -math.inf)
                lse = torch.logsumexp(s, -1)
                p = torch.exp(s - lse[..., None])
                o, size = p @ V, p @ V.abs()
                top = qp.abs().amax(-1, keepdim=True)
                q_err = (2.0 ** -22 * top).expand_as(qp) if decode else torch.maximum(HALF16 * qp.abs(), 2.0 ** -25 * top)
                q_err = q_err + 256 * 2.0 ** -24 * q_sum
                delta = ((q_err @ K.abs().T + 256 * 2.0 ** -24 * (qp.abs() @ K.abs().T)) / math.sqrt(128)).masked_fill(future, 0.0).amax(-1)
                if Uv is not None:
                    o, size = o @ Uv.T, size @ Uv.abs().T
                bound = (HALF16 + 1e-4 + HALF * HALF + torch.expm1(2 * delta)[..., None]) * size + HALF * o.abs() + 1e-30
                got = self.out[b, :m, h * G:h * G + G].double()
                assert torch.isfinite(got).all(), f"sequence {b}, head {h}"
                worst = ((got - o).abs() / bound).max().item()
                assert worst <= 1.0, f"sequence {b}, head {h}: {worst:.2f} of the bound"
                g_lse = self.lse[b, :m, h * G:h * G + G].double()
                assert ((g_lse - lse).abs() <= delta + 1e-4 + 2.0 ** -22 * lse.abs()).all()
        return self


PAIRS = [(32, 32), (48, 48), (64, 64), (96, 96), (128, 128), (32, 128), (128, 32), (48, 96), (96, 48), (64, 128)]
LENS = [1, 0, 63, 64, 65, 130, 700, 2000]


# ------------------------------------------------------------------------------------------------- one token per sequence
@pytest.mark.parametrize("r_k,r_v", PAIRS)
def test_decode_ragged(r_k, r_v):
    Case(r_k + 3 * r_v, LENS, r_k=r_k, r_v=r_v).decode().check()


@pytest.mark.parametrize("Hq,Hkv", [(32, 8), (8, 8), (10, 2), (6, 6), (16, 1), (1, 1), (40, 2), (9, 3)])
def test_decode_heads(Hq, Hkv):
    Case(Hq, [129, 1, 1000], Hq=Hq, Hkv=Hkv).decode().check()


@pytest.mark.parametrize("parts", [1, 7, 148, 400])
def test_decode_parts(parts):
    Case(parts, [5000, 3, 777], Hq=4, Hkv=1).decode(parts=parts).check()


@pytest.mark.parametrize("fold_k,fold_v,r_k,r_v", [(True, True, 128, 128), (True, False, 48, 64), (False, True, 64, 96), (True, True, 32, 48)])
def test_decode_without_basis_and_shared(fold_k, fold_v, r_k, r_v):
    Case(5, LENS, fold_k=fold_k, fold_v=fold_v, r_k=r_k, r_v=r_v).decode().check()
    Case(6, LENS, shared=True, r_k=r_k, r_v=r_v).decode().check()


@pytest.mark.parametrize("exponents", [(-100, -100), (-90, -60), (-30, 6), (-6, -6)])
def test_decode_scales_far_apart(exponents):
    """The scores stay moderate (keys of one scale), the values' scales lie up to 2^36 apart."""
    c = Case(9, [1500, 70], exponents=exponents)
    c.layer.scales[:, :, 0] = 2.0 ** -7
    c.K = _values(c, 0)
    c.decode().check()
    d = Case(9, [1500, 70], n=5, exponents=exponents)
    d.layer.scales[:, :, 0] = 2.0 ** -7
    d.K = _values(d, 0)
    d.attend().check()


def _values(c, side):
    """The rows that the cache holds for every sequence, [t, Hkv, r] in fp64, read back."""
    codes = (c.layer.k_codes, c.layer.v_codes)[side].view(F8).double() * c.layer.scales[:, :, side].double()[:, :, None, None]
    return [codes[c.batch.block_table[b, :(t + 63) // 64].long()].transpose(1, 2).flatten(0, 1)[:t] for b, t in enumerate(c.lens)]


@pytest.mark.parametrize("q_scale", [0.0, 1e-20, 60.0, 3000.0])
def test_scores_from_nothing_to_far_apart(q_scale):
    Case(10, [900, 33], q_scale=q_scale).decode().check()
    Case(10, [900, 33], n=9, q_scale=q_scale).attend().check()


def test_decode_long_and_many():
    Case(11, [32768, 12345], Hq=8, Hkv=2).decode().check()
    Case(12, [(31 * i) % 400 for i in range(1024)], Hq=2, Hkv=1, r_k=32, r_v=32).decode().check()


def test_decode_len_add_and_bad_pages():
    c = Case(13, [100, 64], extra=1)
    c.batch.seq_lens.sub_(1)
    c.decode(len_add=1).check()
    c = Case(14, [300, 200])
    c.batch.block_table[1, 1] = 10 ** 6
    c.decode()
    torch.cuda.synchronize()
    assert c.status.item() == S.STIEF_ERR_BOUNDS
    good = Case(14, [300, 200]).decode()
    assert torch.equal(c.out[0], good.out[0])
    c = Case(15, [300, 200])
    c.batch.seq_lens[0] = 100000                                            # longer than its table
    c.decode()
    torch.cuda.synchronize()
    assert c.status.item() == S.STIEF_ERR_BOUNDS and torch.equal(c.out[1], Case(15, [300, 200]).decode().out[1])


def test_decode_is_repeatable_overlapped_and_captured():
    """Layers of different ranks in one run of overlapped launches on one workspace, called, captured and replayed."""
    cases = [Case(20 + i, LENS, r_k=a, r_v=b) for i, (a, b) in enumerate([(64, 64), (32, 128), (128, 96), (48, 32), (96, 64)])]
    ws = torch.zeros(max(S.stief_decode_workspace_bytes(len(LENS), 8, 2, 128), 1), dtype=torch.uint8, device="cuda")
    S.stief_decode_workspace_init(ws)
    torch.cuda.synchronize()
    for i, c in enumerate(cases):
        c.decode(workspace=ws, flags=S.STIEF_DECODE_OVERLAP_PREVIOUS if i else 0)
    first = [c.check().out.clone() for c in cases]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        for i, c in enumerate(cases):
            c.decode(workspace=ws, flags=S.STIEF_DECODE_OVERLAP_PREVIOUS if i else 0)
    for c in cases:
        c.out.fill_(NAN)
        c.lse.fill_(NAN)
    torch.cuda.synchronize()
    for _ in range(3):
        graph.replay()
    for c, f in zip(cases, first):
        c.check()
        assert torch.equal(c.out, f)


# ------------------------------------------------------------------------------------------------- runs of query tokens
@pytest.mark.parametrize("r_k,r_v", PAIRS)
def test_runs_ragged(r_k, r_v):
    lens = [1, 5, 64, 200, 700, 300, 129]
    counts = [1, 0, 64, 7, 130, 300, 66]
    Case(r_k + 5 * r_v, lens, n=300, counts=counts, r_k=r_k, r_v=r_v).attend(splits=1).check()


@pytest.mark.parametrize("Hq,Hkv", [(32, 8), (8, 8), (10, 2), (6, 6), (16, 1), (1, 1), (40, 2), (9, 3), (128, 1)])
@pytest.mark.parametrize("n", [1, 3, 40])
def test_runs_heads(Hq, Hkv, n):
    Case(Hq + n, [129, 40, 1000], n=n, Hq=Hq, Hkv=Hkv).attend().check()
    Case(Hq + n, [129, 40, 1000], n=n, Hq=Hq, Hkv=Hkv).attend(splits=3).check()


@pytest.mark.parametrize("fold_k,fold_v,r_k,r_v", [(True, True, 128, 128), (True, False, 48, 64), (False, True, 64, 96), (True, True, 32, 48)])
@pytest.mark.parametrize("splits", [1, 4])
def test_runs_without_basis_and_shared(fold_k, fold_v, r_k, r_v, splits):
    Case(25, [300, 90, 1], n=70, fold_k=fold_k, fold_v=fold_v, r_k=r_k, r_v=r_v).attend(splits=splits).check()
    Case(26, [300, 90, 1], n=70, shared=True, r_k=r_k, r_v=r_v, token_major=True).attend(splits=splits).check()


@pytest.mark.parametrize("splits", [1, 2, 5, 32])
@pytest.mark.parametrize("n,lens", [(8, [4096, 700]), (33, [2000, 2000, 5]), (257, [3000])])
def test_runs_split(splits, n, lens):
    Case(splits, lens, n=n).attend(splits=splits).check()


@pytest.mark.parametrize("r_k,r_v", PAIRS)
def test_parts_joined(r_k, r_v):
    """Sequences of unequal numbers of rows, and more tiles of rows than blocks that join them."""
    Case(r_k + 7 * r_v, [1, 700, 64, 300, 129], n=90, counts=[1, 90, 0, 77, 13], r_k=r_k, r_v=r_v).attend(splits=3).check()
    if r_k == r_v:
        Case(r_v, [900], n=700, Hq=16, Hkv=1, r_k=r_k, r_v=r_v).attend(splits=2).check()


@pytest.mark.parametrize("r_k,r_v", [(64, 64), (64, 128), (48, 48), (96, 96)])
@pytest.mark.parametrize("splits", [1, 2])
def test_runs_whose_largest_score_grows(r_k, r_v, splits):
    """The scale of the keys doubles every second page, so that every step moves the references of most rows."""
    c = Case(27, [1300, 500], n=200, r_k=r_k, r_v=r_v)
    pages = torch.arange(c.batch.block_table.shape[1], device="cuda")
    for b, t in enumerate(c.lens):
        c.layer.scales[c.batch.block_table[b, : (t + 63) // 64].long(), :, 0] = torch.exp2(-14.0 + pages[: (t + 63) // 64] // 2)[:, None]
    c.K = _values(c, 0)
    c.attend(splits=splits).check()


def test_runs_long():
    Case(30, [9000], n=2048, Hq=4, Hkv=1).attend().check()
    c = Case(31, [500, 400], n=6)
    c.counts = [6, 6]
    c.attend(counts=False).check()


def test_runs_refused_on_the_device():
    c = Case(32, [100, 70, 10], n=20, counts=[20, 20, 20])                   # more query tokens than cached ones
    c.attend().check(status=S.STIEF_ERR_BOUNDS, skip=(2,))
    c = Case(33, [300, 200], n=20)
    c.batch = S.Batch(c.batch.block_table[:, :4].contiguous(), c.batch.seq_lens)      # a table too short for the first sequence
    c.attend().check(status=S.STIEF_ERR_BOUNDS, skip=(0,))
    c = Case(34, [300, 200], n=20)
    c.batch.block_table[1, 1] = -1
    c.attend()
    torch.cuda.synchronize()
    assert c.status.item() == S.STIEF_ERR_BOUNDS and torch.equal(c.out[0], Case(34, [300, 200], n=20).attend().out[0])


def test_runs_on_two_streams_and_captured():
    a, b = Case(35, [3000, 100], n=8), Case(36, [500, 1000], n=200, r_k=96, r_v=128)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for c, s in zip((a, b), streams):
        with torch.cuda.stream(s):
            c.attend()
    a.check()
    b.check()
    first = a.out.clone()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    L = a.layer
    ws = torch.zeros(S.stief_f8_mq_workspace_bytes(2, 8, L.Hq, L.r_v, 4), dtype=torch.uint8, device="cuda")
    ql = torch.tensor(a.counts, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        S.stief_f8_mq_attention(L, a.batch, a.q, a.out, q_lens=ql, workspace=ws, num_splits=4, out_lse=a.lse)
    for _ in range(2):
        a.out.fill_(NAN)
        graph.replay()
        a.check()
    assert (a.out.float() - first.float()).abs().max() <= 2 ** -6 * first.float().abs().max()


def test_runs_of_many_sequences():
    """More sequences than the kernel lists the work of, many without a query."""
    lens = [(53 * i) % 400 + 1 for i in range(130)]
    counts = [0 if i % 3 == 0 else min(n, (7 * i) % 90) for i, n in enumerate(lens)]
    Case(37, lens, n=90, counts=counts, Hq=4, Hkv=1, r_k=48, r_v=32).attend(splits=1).check()
    Case(38, lens[:96], n=90, counts=counts[:96], Hq=4, Hkv=1).attend(splits=1).check()
    Case(39, lens, n=4, counts=[min(c, 4) for c in counts], Hq=8, Hkv=2).attend(splits=2).check()
    Case(40, [500, 90], n=3, counts=[0, 0]).attend(splits=1).check()


def test_nan_codes_stay_nan_where_they_are_attended():
    c = Case(41, [200, 200])
    page = int(c.batch.block_table[0, 1])
    c.layer.v_codes[page, :, 5, 7] = 0x7F
    c.decode()
    good = Case(41, [200, 200]).decode()
    torch.cuda.synchronize()
    assert torch.isnan(c.out[0]).all() and torch.equal(c.out[1], good.out[1])      # one NaN channel reaches all through the basis
    d = Case(42, [200, 200], n=4)
    d.layer.k_codes[int(d.batch.block_table[1, 0]), 0, 9, 3] = 0xFF
    d.attend(splits=1)
    torch.cuda.synchronize()
    assert torch.isnan(d.out[1, :, :4]).all() and torch.isfinite(d.out[1, :, 4:]).all() and torch.isfinite(d.out[0]).all()


def test_pages_far_into_large_pools():
    """Byte offsets beyond 2^32, all three kernels."""
    Hkv, r = 8, 128
    P = 2 ** 32 // (Hkv * 64 * r) + 9
    for n, splits in ((None, 1), (6, 4), (40, 1)):
        c = Case(43, [500, 300], n=n, Hq=8, Hkv=Hkv, r_k=r, r_v=r)
        (c.decode() if n is None else c.attend(splits=splits)).check()
        first, L = c.out.clone(), c.layer
        small = L.k_codes.shape[0]
        far = lambda t: torch.empty(P, *t.shape[1:], dtype=t.dtype, device="cuda")  # noqa: E731
        for name in ("k_codes", "v_codes", "scales"):
            t = getattr(L, name)
            big = far(t)
            big[P - small:] = t
            setattr(L, name, big)
        c.batch.block_table.add_(P - small)
        c.out.fill_(NAN)
        (c.decode() if n is None else c.attend(splits=splits)).check()
        assert torch.equal(c.out, first)
        del L, c


def test_two_captured_graphs_share_a_workspace():
    """One after the other on one stream, replayed in turn."""
    cases = [Case(44 + i, [3000, 700], n=8, r_k=64, r_v=rv) for i, rv in enumerate((64, 128))]
    ws = torch.zeros(S.stief_f8_mq_workspace_bytes(2, 8, 8, 128, 4), dtype=torch.uint8, device="cuda")
    graphs, side = [], torch.cuda.Stream()
    for c in cases:
        call = lambda: S.stief_f8_mq_attention(c.layer, c.batch, c.q, c.out, out_lse=c.lse, workspace=ws, num_splits=4)  # noqa: E731
        call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            call()
        graphs.append(g)
    for _ in range(3):
        for c, g in zip(cases, graphs):
            c.out.fill_(NAN)
            g.replay()
    for c in cases:
        c.check()


def _forms(seed, lens, **kw):
    """The three kernels: one token in one part and in many, a few rows (the kernel for them from two parts on), tiles of rows."""
    yield Case(seed, lens, **kw), lambda c: c.decode(parts=1)
    yield Case(seed, lens, **kw), lambda c: c.decode()
    for n, splits in ((3, 1), (3, 2), (3, None), (70, 1), (70, 3)):
        yield Case(seed, lens, n=n, **kw), lambda c, splits=splits: c.attend(splits=splits)


def _fill(c, side, pages, scale, code=None):
    """Pages (a mask over the places of each sequence's table) get one scale, and one code where it is given."""
    codes = (c.layer.k_codes, c.layer.v_codes)[side]
    for b, t in enumerate(c.lens):
        ids = c.batch.block_table[b, :(t + 63) // 64].long()
        ids = ids[pages(torch.arange(ids.numel(), device="cuda"))]
        c.layer.scales[ids, :, side] = scale
        if code is not None:
            codes[ids] = code
    if side:
        c.V = _values(c, 1)
    else:
        c.K = _values(c, 0)


@pytest.mark.parametrize("code", [0x00, 0x01, 0x7E])
def test_long_sequences_of_zeros_and_tiny_values(code):
    """Rows of zeros and of the smallest scale: each page's share of a row's sum is 2^100 times its weights."""
    for c, call in _forms(50, [16384] * 4, Hq=4, Hkv=1, r_k=32, r_v=32, spare=0):
        _fill(c, 0, lambda i: i >= 0, 2.0 ** -100, 0x00)
        _fill(c, 1, lambda i: i >= 0, 2.0 ** -100, code)
        call(c).check()


def test_zeros_over_the_longest_batches():
    """16 x 16384 in a decode step, 4 x 32768 in runs: zeros, and the logarithm of the length."""
    for n, lens, splits in ((None, [16384] * 16, None), (8, [32768] * 4, None), (8, [32768] * 4, 1), (40, [32768] * 4, 1)):
        c = Case(51, lens, n=n, Hq=32, Hkv=8, r_k=32, r_v=32, spare=0)
        for side in (0, 1):
            _fill(c, side, lambda i: i >= 0, 2.0 ** -100, 0x00)
        (c.decode() if n is None else c.attend(splits=splits))
        torch.cuda.synchronize()
        assert c.status.item() == 0 and (c.out == 0).all()
        seen = torch.full_like(c.lse, lens[0])
        if n is not None:
            seen -= torch.arange(n - 1, -1, -1, device="cuda")[:, None]
        assert ((c.lse - seen.log()).abs() <= 1e-4 + 2.0 ** -22 * 11).all()


@pytest.mark.parametrize("low,high", [(-100, 119), (-100, 20), (-100, -6), (-60, 40)])
def test_pages_of_scales_as_far_apart_as_they_can_be(low, high):
    """Every third page of the lower scale, scores of the same range in all: those pages are part of the sum, whatever their weights."""
    for c, call in _forms(52, [1500, 130, 40], r_k=48, r_v=64):
        _fill(c, 0, lambda i: i >= 0, 2.0 ** -7)
        _fill(c, 1, lambda i: i % 3 != 1, 2.0 ** (high - 10))
        _fill(c, 1, lambda i: i % 3 == 1, 2.0 ** low)
        call(c).check()


def test_zero_pages_between_ordinary_ones():
    """... with scores that grow from page to page on top."""
    for c, call in _forms(53, [2500, 700], r_k=64, r_v=48):
        _fill(c, 1, lambda i: i % 2 == 0, 2.0 ** -100, 0x00)
        for k in range(12):
            _fill(c, 0, lambda i, k=k: i // 4 == k, 2.0 ** (k - 12))
        call(c).check()


@pytest.mark.parametrize("q_scale", [3e4, 1e6, 4e6, 1e7, 3e7, 1e8, 1e12, 1e25])
def test_scores_far_from_zero(q_scale):
    """References whose steps are as wide as the headroom of the weights (2^24 to 2^28 in base 2) and wider."""
    for c, call in _forms(54, [900, 33], q_scale=q_scale):
        call(c).check()


@pytest.mark.parametrize("q_scale", [1.0, 3e4, 1e6, 1e7, 1e8, 1e12])
def test_far_scores_of_equal_rows(q_scale):
    """One key for every token: the mean of the values, whose scales differ from page to page.  (Decode in one part: the parts of a
    decode step are joined by their log-sum-exps, which far scores leave no room for.)"""
    for n, splits in ((None, None), (3, 1), (3, 4), (70, 1), (70, 3)):
        c = Case(55, [700, 130], n=n, q_scale=q_scale, exponents=(-9, -4))
        _fill(c, 0, lambda i: i >= 0, 2.0 ** -3, 0x38)
        c.decode(parts=1) if n is None else c.attend(splits=splits)
        torch.cuda.synchronize()
        assert c.status.item() == 0
        Uv, G = c.layer.U_v.double(), c.layer.Hq // c.layer.Hkv
        for b, t in enumerate(c.lens):
            for i in range(c.counts[b]):
                V = c.V[b][:t - c.counts[b] + 1 + i]
                o, size = (torch.einsum("hr,hdr->hd", x.mean(0), y).repeat_interleave(G, 0) for x, y in ((V, Uv), (V.abs(), Uv.abs())))
                assert ((c.out[b, i].double() - o).abs() <= (HALF16 + 1e-4 + HALF * HALF) * size + HALF * o.abs()).all(), f"sequence {b}, token {i}"


def test_scores_beyond_the_range():
    """Queries and keys whose products leave fp32's range downwards, but for the rows of zeros, whose score is zero: their mean."""
    for n, splits in ((None, None), (3, 1), (3, 4), (70, 1), (70, 3)):
        c = Case(56, [700, 130], n=n, fold_k=True, exponents=(-6, -6))
        _fill(c, 0, lambda i: i >= 0, 2.0 ** 60, 0xFE)                      # -448
        for b, t in enumerate(c.lens):
            c.layer.k_codes[c.batch.block_table[b, :(t + 63) // 64].long(), :, ::7] = 0
        c.q.fill_(2.0 ** 80)
        c.decode(parts=1) if n is None else c.attend(splits=splits)
        torch.cuda.synchronize()
        assert c.status.item() == 0
        Uv, G = c.layer.U_v.double(), c.layer.Hq // c.layer.Hkv
        for b, t in enumerate(c.lens):
            for i in range(c.counts[b]):
                seen = t - c.counts[b] + 1 + i
                V = c.V[b][:seen][(torch.arange(seen, device="cuda") % 64) % 7 == 0]
                o, size = (torch.einsum("hr,hdr->hd", x.mean(0), y).repeat_interleave(G, 0) for x, y in ((V, Uv), (V.abs(), Uv.abs())))
                assert ((c.out[b, i].double() - o).abs() <= (HALF16 + 1e-4 + HALF * HALF) * size + HALF * o.abs()).all(), f"sequence {b}, token {i}"


@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (10, 2), (6, 2)])
@pytest.mark.parametrize("other", [1e4, 1e7, 1e30, NAN])
def test_rows_do_not_depend_on_their_neighbours(Hq, Hkv, other):
    """Queries behind a sequence's last, and other rows of the tile, of any size: the same bits."""
    def outputs(scale, first):
        c = Case(57, [700, 90], n=30, counts=[17, 30], Hq=Hq, Hkv=Hkv, r_k=48, r_v=64, exponents=(-9, -4))
        c.q[0, 17:] *= scale
        c.q[1, :first] *= scale
        c.attend(splits=1)
        torch.cuda.synchronize()
        assert c.status.item() == 0
        return c.out[0, :17], c.lse[0, :17], c.out[1, 3:], c.lse[1, 3:]

    for first in (0, 3):
        for x, y in zip(outputs(1.0, 0), outputs(other, first)):
            assert torch.equal(x, y)


def test_nan_queries_and_pages_of_nan_keys_are_not_passed_over():
    """A query of NaN, or a page whose keys are NaN throughout, leaves no score to go by: the rows are NaN, the others what they were."""
    for what in ("query", "page"):
        for (c, call), (good, _) in zip(_forms(58, [700, 90]), _forms(58, [700, 90])):
            call(good).check()
            if what == "query":
                c.q[0, -1, 1] = NAN
            else:
                c.layer.k_codes[int(c.batch.block_table[0, 3]), 0] = 0x7F
            call(c)
            torch.cuda.synchronize()
            assert c.status.item() == 0 and torch.equal(c.out[1], good.out[1])
            if what == "query":
                assert torch.isnan(c.out[0, -1, 1]).all() and torch.equal(c.out[0, -1, 2:], good.out[0, -1, 2:]) and torch.equal(c.out[0, -1, 0], good.out[0, -1, 0])
            else:
                assert torch.isnan(c.out[0, :, :4]).all() and torch.equal(c.out[0, :, 4:], good.out[0, :, 4:])


@pytest.mark.parametrize("splits", [1, 2, 4])
@pytest.mark.parametrize("other", [1e4, 1e30, NAN])
def test_few_rows_do_not_depend_on_their_neighbours(splits, other):
    def outputs(scale):
        c = Case(59, [700, 90], n=8, counts=[5, 8], exponents=(-9, -4))
        c.q[0, 5:] *= scale
        c.q[1, :3] *= scale
        c.attend(splits=splits)
        torch.cuda.synchronize()
        assert c.status.item() == 0
        return c.out[0, :5], c.lse[0, :5], c.out[1, 3:], c.lse[1, 3:]

    for x, y in zip(outputs(1.0), outputs(other)):
        assert torch.equal(x, y)


# ------------------------------------------------------------------------------------------------- together
def test_prompt_chunks_and_decode_in_one_run():
    """What a server does with one layer: prompts appended (rotated) and attended in chunks, pages reserved, a sequence forked, then
    decode steps.  Compared with causal attention in fp64 over the rows that the cache holds."""
    torch.manual_seed(1)
    Hq, Hkv, r_k, r_v, B, P = 8, 2, 96, 64, 3, 40
    basis = lambda r: torch.linalg.qr(torch.randn(Hkv, 128, 128, device="cuda"))[0][:, :, :r].to(BF).contiguous()  # noqa: E731
    L = S.F8Layer(Hq, Hkv, r_k, r_v, basis(r_k), basis(r_v), torch.zeros(P, Hkv, 64, r_k, dtype=torch.uint8, device="cuda"),
                  torch.zeros(P, Hkv, 64, r_v, dtype=torch.uint8, device="cuda"), torch.zeros(P, Hkv, 4, device="cuda"))
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    lens = i32(0, 0, 0)
    pages = S.PageTable(torch.zeros(B, 10, dtype=torch.int32, device="cuda"), lens, i32(0, 0, 0), torch.zeros(P, dtype=torch.int32, device="cuda"))
    batch, status = pages.batch, i32(0)
    angle = torch.arange(700, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, 128, 2, device="cuda").double() / 128)
    turn = S.Rotation(torch.cat([angle.cos(), angle.sin()], 1).float())

    def reference(b, q):                                                     # q [m, Hq, 128]: the last m tokens, rotated already
        t = int(lens[b])
        ids = pages.block_table[b, :(t + 63) // 64].long()
        rows = [(c[ids].view(F8).double() * L.scales[ids, :, i].double()[:, :, None, None]).transpose(1, 2).flatten(0, 1)[:t] for i, c in enumerate((L.k_codes, L.v_codes))]
        K, V = (torch.einsum("thr,hdr->thd", x, U.double()) for x, U in zip(rows, (L.U_k, L.U_v)))
        s = torch.einsum("mhgd,thd->hgmt", q.double().view(-1, Hkv, Hq // Hkv, 128), K) / math.sqrt(128)
        s.masked_fill_(torch.ones(q.shape[0], t, dtype=torch.bool, device="cuda").triu(t - q.shape[0] + 1), -math.inf)
        return torch.einsum("hgmt,thd->mhgd", s.softmax(-1), V).reshape(-1, Hq, 128)

    for counts in ((100, 1, 64), (130, 70, 0), (3, 200, 90)):                 # chunks
        cu, total, most = i32(0, *torch.tensor(counts).cumsum(0).tolist()), sum(counts), max(counts)
        wide = torch.randn(total, Hq + 2 * Hkv, 128, device="cuda").to(BF)
        S.stief_pages_reserve(pages, i32(*counts), status=status)
        q = torch.empty(total, Hq, 128, dtype=BF, device="cuda")
        S.stief_f8_append(L, batch, wide[:, Hq:Hq + Hkv], wide[:, Hq + Hkv:], cu, rotation=turn, q=wide[:, :Hq], q_out=q, status=status)
        S.stief_advance_seq_lens_by(lens, i32(*counts))
        padded, out = torch.zeros(B, most, Hq, 128, dtype=BF, device="cuda"), torch.zeros(B, most, Hq, 128, dtype=BF, device="cuda")
        for b, m in enumerate(counts):
            padded[b, :m] = q[int(cu[b]):int(cu[b]) + m]
        S.stief_f8_mq_attention(L, batch, padded, out, q_lens=i32(*counts), status=status)
        for b, m in enumerate(counts):
            if m:
                want = reference(b, padded[b, :m])
                assert (out[b, :m].double() - want).norm() <= (HALF + 2 * HALF16) * want.norm()
    ws = torch.zeros(S.stief_pages_workspace_bytes(B, 10), dtype=torch.uint8, device="cuda")
    S.stief_pages_fork(pages, [L], i32(1, 1, 2), ws, status=status)            # slot 0 becomes a copy of slot 1
    dws = torch.zeros(S.stief_decode_workspace_bytes(B, Hq, Hkv, r_v), dtype=torch.uint8, device="cuda")
    S.stief_decode_workspace_init(dws)
    cu, out = i32(0, 1, 2, 3), torch.zeros(B, Hq, 128, dtype=BF, device="cuda")
    for step in range(70):
        wide = torch.randn(B, Hq + 2 * Hkv, 128, device="cuda").to(BF) * (1 + step % 3)
        S.stief_pages_reserve(pages, 1, status=status)
        S.stief_f8_append(L, batch, wide[:, Hq:Hq + Hkv], wide[:, Hq + Hkv:], cu, rotation=turn, q=wide[:, :Hq], q_out=wide[:, :Hq], status=status)
        q = wide[:, :Hq].contiguous()
        S.stief_f8_decode_attention(L, batch, q, dws, out, len_add=1, status=status)
        S.stief_advance_seq_lens(lens, 1)
        if step in (0, 30, 69):
            for b in range(B):
                want = reference(b, q[b:b + 1])[0]
                assert (out[b].double() - want).norm() <= (HALF + 2 * HALF16) * want.norm()
    assert status.item() == 0
