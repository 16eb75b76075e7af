"""Attention of a tree of drafted tokens over the compressed cache, against the definition in fp64 on the cache rows the GPU
holds.  Tolerances are error bounds: the probabilities are rounded to bf16 once (half a step = 2^-8 of the value), the
output once more, q' to two bf16 terms (2^-16); everything else is fp32 (and exponentials good to 1e-4)."""
import math

import pytest
import torch

import paper_2601_21686_b200 as S

pytestmark = pytest.mark.gpu
HALF = torch.finfo(torch.bfloat16).eps / 2
NAN = float("nan")


def _bases(g, n, r):
    u = torch.linalg.qr(torch.randn(n, 128, 128, generator=g, device="cuda", dtype=torch.float64))[0]
    return u[:, :, :r].to(torch.bfloat16).contiguous()


def tree_masks(g, B, n, words=None):
    """Ancestor masks of random trees, as bool [B, n, n] and packed int32 [B, n, words]."""
    up = (torch.rand(B, n, generator=g, device="cuda") * torch.arange(n, device="cuda")).long().cpu()
    m = torch.zeros(B, n, n, dtype=torch.bool)
    for b in range(B):
        for i in range(n):
            if i:
                m[b, i] = m[b, up[b, i]]
            m[b, i, i] = True
    return m.cuda(), pack(m, words).cuda()


def pack(m, words=None):
    B, n, _ = m.shape
    words = words or (n + 31) // 32
    full = torch.zeros(B, n, words * 32, dtype=torch.int64)
    full[:, :, :n] = m.cpu().long()
    w = (full.view(B, n, words, 32) << torch.arange(32)).sum(-1)
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32)


class TreeCase:
    def __init__(self, seed, lens, n, counts=None, Hq=8, Hkv=2, r_k=64, r_v=64, fold_k=False, fold_v=False, q_scale=2.0, shared=False, spare=3, words=None):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        c = torch.Generator()
        c.manual_seed(seed)
        self.n, self.lens, self.counts = n, list(lens), [n] * len(lens) if counts is None else list(counts)
        B = len(lens)
        pages = [(a + m + 63) // 64 for a, m in zip(self.lens, self.counts)]
        width = max(max(pages), 1)
        order = torch.randperm(sum(pages) + spare, generator=c)
        table = torch.zeros(B, width, dtype=torch.int32)
        kp = torch.full((sum(pages) + spare, Hkv, 64, r_k), NAN, dtype=torch.bfloat16, device="cuda")
        vp = torch.full((sum(pages) + spare, Hkv, 64, r_v), NAN, dtype=torch.bfloat16, device="cuda")
        self.K, self.V, at = [], [], 0
        for b in range(B):
            t = self.lens[b] + self.counts[b]
            K = torch.randn(t, Hkv, r_k, generator=g, device="cuda").to(torch.bfloat16)
            V = torch.randn(t, Hkv, r_v, generator=g, device="cuda").to(torch.bfloat16)
            for i in range(pages[b]):
                p = int(order[at + i])
                table[b, i] = p
                k = min(64, t - 64 * i)
                kp[p, :, :k] = K[64 * i:64 * i + k].transpose(0, 1)
                vp[p, :, :k] = V[64 * i:64 * i + k].transpose(0, 1)
            at += pages[b]
            self.K.append(K)
            self.V.append(V)
        nb = 1 if shared else Hkv
        self.layer = S.Layer(Hq, Hkv, r_k, r_v, None if fold_k else _bases(g, nb, r_k), None if fold_v else _bases(g, nb, r_v), kp, vp)
        self.batch = S.Batch(table.cuda(), torch.tensor(self.lens, dtype=torch.int32, device="cuda"))
        self.q = (q_scale * torch.randn(B, n, Hq, r_k if fold_k else 128, generator=g, device="cuda")).to(torch.bfloat16)
        self.n_nodes = torch.tensor(self.counts, dtype=torch.int32, device="cuda")
        self.seen, self.mask = tree_masks(g, B, n, words)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.workspace = torch.full((S.stief_tree_workspace_bytes(B, n, Hq, Hkv, r_v),), 0xFF, dtype=torch.uint8, device="cuda")

    def run(self, q=None, out=None, lse=True, mask=None, n_nodes="own"):
        q = self.q if q is None else q
        B, n, Hq = q.shape[:3]
        if out is None:
            out = torch.full((B, n, Hq, 128 if self.layer.U_v is not None else self.layer.r_v), NAN, dtype=torch.bfloat16, device="cuda")
        out_lse = torch.full((B, n, Hq), NAN, dtype=torch.float32, device="cuda") if lse else None
        S.stief_tree_attention(self.layer, self.batch, q, self.mask if mask is None else mask, self.workspace, out,
                               n_nodes=self.n_nodes if isinstance(n_nodes, str) else n_nodes, out_lse=out_lse, status=self.status)
        return out, out_lse

    def check(self, out, out_lse=None, seen=None):
        seen = self.seen if seen is None else seen
        L = self.layer
        G = L.Hq // L.Hkv
        for b, (ctx, m) in enumerate(zip(self.lens, self.counts)):
            assert torch.isnan(out[b, m:]).all(), "rows behind the last node were written"
            for h in range(L.Hkv):
                Uk = None if L.U_k is None else L.U_k[h if L.U_k.shape[0] > 1 else 0].double()
                Uv = None if L.U_v is None else L.U_v[h if L.U_v.shape[0] > 1 else 0].double()
                K, V = self.K[b][:, h].double(), self.V[b][:, h].double()
                q = self.q[b, :m, h * G:h * G + G].double()
                qp = q if Uk is None else q @ Uk
                keep = torch.cat([torch.ones(m, ctx, dtype=torch.bool, device="cuda"), seen[b, :m, :m]], 1)[:, None]
                s = (qp @ K.T / math.sqrt(128)).masked_fill(~keep, -math.inf)
                empty = ~keep.any(-1).expand(m, G)
                lse = torch.logsumexp(s, -1)
                p = torch.exp(s - lse.masked_fill(empty, 0.0)[..., None])
                o, size = p @ V, p @ V.abs()
                # scores are off by at most delta: q' in two terms (exact when it is handed over), and fp32 sums
                rounding = (0.0 if Uk is None else HALF * HALF) + 256 * 2.0 ** -24
                delta = (rounding * (qp.abs() @ K.abs().T) / math.sqrt(128)).masked_fill(~keep, 0.0).amax(-1) if K.shape[0] else torch.zeros_like(lse)
                if Uv is not None:
                    o, size = o @ Uv.T, size @ Uv.abs().T
                bound = (HALF + 3e-4 + torch.expm1(2 * delta)[..., None]) * size + HALF * o.abs() + 1e-6
                got = out[b, :m, h * G:h * G + G].double()
                assert torch.isfinite(got).all()
                worst = ((got - o).abs() / bound).max().item() if m else 0.0
                assert worst <= 1.0, f"sequence {b}, head {h}: {worst:.2f} of the bound"
                assert (got[empty] == 0).all()
                if out_lse is not None:
                    g_lse = out_lse[b, :m, h * G:h * G + G].double()
                    assert (g_lse[empty] == -math.inf).all()
                    err = ((g_lse - lse).abs() / (delta + 2e-4 + 1e-6 * lse.abs()))[~empty]
                    assert err.numel() == 0 or err.max().item() <= 1.0
            if out_lse is not None:
                assert torch.isnan(out_lse[b, m:]).all()


@pytest.mark.parametrize("r_k,r_v", [(64, 64), (32, 32), (48, 96), (96, 48), (128, 128), (32, 128), (128, 32), (64, 128), (96, 64), (48, 48)])
def test_ranks_and_ragged_trees(r_k, r_v):
    c = TreeCase(r_k * 7 + r_v, [300, 0, 1, 63, 64, 1000], 13, [13, 5, 1, 2, 13, 0], r_k=r_k, r_v=r_v)
    c.check(*c.run())
    assert int(c.status) == 0


@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (8, 2), (10, 2), (16, 1), (7, 1), (32, 8), (40, 1)])
@pytest.mark.parametrize("n", [1, 9, 40])
def test_head_groups_and_tree_sizes(Hq, Hkv, n):
    c = TreeCase(Hq * 31 + n, [129, 257], n, [n, max(1, n - 1)], Hq=Hq, Hkv=Hkv)
    c.check(*c.run())
    assert int(c.status) == 0


@pytest.mark.parametrize("n,G", [(32, 4), (33, 4), (64, 4), (65, 4), (128, 1), (129, 1), (200, 2), (300, 1), (1024, 1)])
def test_tile_edges_of_large_trees(n, G):
    c = TreeCase(n + G, [70, 200], n, [n, n - 1], Hq=2 * G, Hkv=2, r_k=48, r_v=64)
    c.check(*c.run())
    assert int(c.status) == 0


@pytest.mark.parametrize("lens", [[5000], [20000], [8000] * 4, [3, 9000, 500, 0], [127, 128, 129, 191, 192, 193, 255, 256, 257, 383, 384, 385]])
@pytest.mark.parametrize("n", [3, 16, 17, 32, 64])
def test_long_contexts_are_cut_and_joined(lens, n):
    c = TreeCase(sum(lens) + n, lens, n, Hq=32, Hkv=8)
    c.check(*c.run())
    assert int(c.status) == 0


@pytest.mark.parametrize("r_k", [32, 48, 64, 96, 128])
@pytest.mark.parametrize("r_v", [32, 48, 64, 96, 128])
@pytest.mark.parametrize("n", [8, 50])
def test_many_blocks_per_segment_at_every_rank_pair(r_k, r_v, n):
    c = TreeCase(r_k + 3 * r_v + n, [150 * 128 * 6 + 77, 40], n, [n, 3], Hq=8, Hkv=1, r_k=r_k, r_v=r_v)
    c.check(*c.run())
    assert int(c.status) == 0


def test_token_major_queries_and_outputs():
    c = TreeCase(71, [400, 90, 1000], 21, [21, 8, 1])
    want, _ = c.run()
    B, n, Hq, d = c.q.shape
    out = torch.full((n, B, Hq, 128), NAN, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    c.run(q=c.q.transpose(0, 1).contiguous().transpose(0, 1), out=out)
    c.check(out)
    assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(want))
    c = TreeCase(72, [400, 90, 1000], 1)                       # one node each: [1, B, ...] seen as [B, 1, ...]
    c.check(*c.run(q=c.q.transpose(0, 1).contiguous().transpose(0, 1)))
    assert int(c.status) == 0


def test_a_call_without_any_node_and_the_next_on_its_stream():
    """Such a call ends in stream order like any other: the counts that the next call reads may be written behind it."""
    c = TreeCase(67, [9000, 300, 40, 0], 16, [16, 3, 0, 1], Hq=32, Hkv=8)
    counts, none = c.n_nodes.clone(), torch.zeros_like(c.n_nodes)
    want, want_lse = c.run()
    c.check(want, want_lse)
    for _ in range(20):
        c.n_nodes.copy_(none)
        out, lse = c.run()
        c.n_nodes.copy_(counts)
        again, again_lse = c.run()
        assert torch.isnan(out).all() and torch.isnan(lse).all()
        assert torch.equal(again.view(torch.int16), want.view(torch.int16)) and torch.equal(again_lse.view(torch.int32), want_lse.view(torch.int32))
    lens = c.batch.seq_lens.clone()
    c.batch.seq_lens.fill_(-1)                                 # nothing to do because everything is refused
    out, _ = c.run()
    c.batch.seq_lens.copy_(lens)
    again, _ = c.run()
    assert torch.isnan(out).all() and torch.equal(again.view(torch.int16), want.view(torch.int16))
    assert int(c.status) == S.STIEF_ERR_BOUNDS


def test_many_sequences():
    lens = [(37 * i) % 450 for i in range(200)]
    c = TreeCase(5, lens, 6, [(i % 7) for i in range(200)], Hq=8, Hkv=2)
    c.check(*c.run())
    assert int(c.status) == 0


def test_largest_batch():
    lens = [(53 * i) % 200 for i in range(1024)]
    c = TreeCase(6, lens, 3, [(i % 4) for i in range(1024)], Hq=2, Hkv=1, r_k=32, r_v=48)
    c.check(*c.run())
    assert int(c.status) == 0


def test_two_captured_calls_share_a_workspace():
    a, b = TreeCase(61, [3000, 500], 20, Hq=8, Hkv=2), TreeCase(62, [70, 9000, 10], 40, Hq=8, Hkv=2, r_k=96, r_v=128)
    ws = torch.full((max(a.workspace.numel(), b.workspace.numel()),), 0xFF, dtype=torch.uint8, device="cuda")
    want = [x.run()[0] for x in (a, b)]
    outs, graphs = [], []
    for x, w in zip((a, b), want):
        out = torch.zeros_like(w)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            S.stief_tree_attention(x.layer, x.batch, x.q, x.mask, ws, out, n_nodes=x.n_nodes)
        outs.append(out)
        graphs.append(graph)
    for i in (0, 1, 1, 0, 0, 1):
        outs[i].zero_()
        graphs[i].replay()
        S.stief_tree_attention(b.layer, b.batch, b.q, b.mask, ws, torch.empty_like(want[1]), n_nodes=b.n_nodes)     # an eager one between
        torch.cuda.synchronize()
        assert torch.equal(torch.nan_to_num(outs[i]), torch.nan_to_num(want[i], nan=0.0))


@pytest.mark.parametrize("fold_k,fold_v", [(True, True), (True, False), (False, True)])
def test_folded_sides(fold_k, fold_v):
    c = TreeCase(17, [400, 90], 21, [21, 8], r_k=96, r_v=48, fold_k=fold_k, fold_v=fold_v)
    c.check(*c.run())


def test_shared_basis_strided_tensors_and_wide_mask_rows():
    c = TreeCase(23, [400, 90], 21, [21, 8], shared=True, words=3)
    c.mask[:, :, 1:] = -1                                      # bits of nodes that do not exist
    c.mask[:, :, 0] |= ~((1 << 21) - 1)
    B, n, Hq, d = c.q.shape
    buf = torch.full((B, n + 2, Hq + 3, d), NAN, dtype=torch.bfloat16, device="cuda")
    q = buf[:, 1:n + 1, 2:Hq + 2]
    q.copy_(c.q)
    obuf = torch.full((B, n + 5, Hq + 1, 128), NAN, dtype=torch.bfloat16, device="cuda")
    out = obuf[:, 2:n + 2, :Hq]
    _, lse = c.run(q=q, out=out)
    c.check(out, lse)
    assert torch.isnan(obuf[:, :2]).all() and torch.isnan(obuf[:, n + 2:]).all() and torch.isnan(obuf[:, :, Hq:]).all()
    assert int(c.status) == 0


@pytest.mark.parametrize("ctx", [0, 1, 64, 700])
def test_rows_that_see_little_or_nothing(ctx):
    n = 40
    c = TreeCase(31 + ctx, [ctx, ctx], n, [n, 33])
    seen = torch.rand(2, n, n, generator=torch.Generator().manual_seed(1)) < 0.3      # no tree: any set, own node not implied
    seen[:, ::3] = False
    seen[:, 1, :] = False
    seen[:, 1, 32] = True
    c.check(*c.run(mask=pack(seen).cuda()), seen=seen.cuda())
    assert int(c.status) == 0


def test_nodes_outside_a_row_s_mask_do_not_reach_it():
    c = TreeCase(37, [100], 10)
    a, _ = c.run()
    # every node but 0 gets other (huge) rows: node 0 sees itself and the context only
    pages = c.batch.block_table[0].tolist()
    for pos in range(101, 110):
        c.layer.k_pool[pages[pos // 64], :, pos % 64] = 300.0
        c.layer.v_pool[pages[pos // 64], :, pos % 64] = 1e30
    b, _ = c.run()
    assert torch.equal(a[0, 0], b[0, 0])


def test_growing_scores_rescale():
    c = TreeCase(41, [3000], 30, Hq=4, Hkv=1, fold_k=True, q_scale=1.0)
    ramp = torch.linspace(0, 40, 3030, device="cuda")[:, None]
    unit = torch.zeros(64, device="cuda")
    unit[0] = 1.0
    K = (ramp * unit + 0.05 * c.K[0][:, 0].float()).to(torch.bfloat16)
    c.K[0] = K[:, None]
    for i, p in enumerate(c.batch.block_table[0].tolist()):
        part = K[64 * i:64 * i + 64]
        c.layer.k_pool[p, 0, :len(part)] = part
    c.q[..., 0] = 20.0
    c.check(*c.run())
    c.q[..., 0] = -20.0                                        # and falling ones: the first page holds the maximum
    c.check(*c.run())
    assert int(c.status) == 0


@pytest.mark.parametrize("exponent", [-9, -2, 4, 8, 13, 16, 19, 24, 28, 30, 31, 60, 100, 120])
@pytest.mark.parametrize("r_v,n,lens", [(64, 3, [9000, 0, 5]), (64, 12, [700, 1]), (128, 8, [3000, 90]), (48, 64, [2000, 0])])
def test_scores_far_from_zero(exponent, r_v, n, lens):
    """Scores that are exact in fp32 (19 bits), of sizes up to 2^125 and either sign: nothing but the rounding of probabilities and
    output remains.  In large ones the largest score's ties share the row."""
    c = TreeCase(83 + exponent, lens, n, r_v=r_v, fold_k=True, fold_v=True)
    keys = [torch.zeros_like(K) for K in c.K]
    for b, K in enumerate(keys):
        for i in range(2):
            K[..., i] = (1 + torch.randint(0, 64, K.shape[:2], generator=torch.Generator().manual_seed(b + n + 7 * i)).cuda() / 64).to(torch.bfloat16)
        for i in range((len(K) + 63) // 64):
            part = K[64 * i:64 * i + 64].transpose(0, 1)
            c.layer.k_pool[c.batch.block_table[b, i], :, :part.shape[1]] = part
    c.q.zero_()
    sign = torch.tensor([1.0, -1.0], device="cuda").repeat(c.layer.Hq // 2)
    c.q[..., 0] = (sign * 2.0 ** exponent * 4).to(torch.bfloat16)          # odd heads: all scores far below zero
    c.q[..., 1] = c.q[..., 0] * 2.0 ** -12                     # and scores close to one another
    out, lse = c.run()
    assert int(c.status) == 0
    G = c.layer.Hq // c.layer.Hkv
    for b, (ctx, m) in enumerate(zip(c.lens, c.counts)):
        for g in range(c.layer.Hq):
            s = c.q[b, :m, g].double() @ keys[b][:, g // G].double().T / math.sqrt(128)
            s[:, ctx:].masked_fill_(~c.seen[b, :m, :m], -math.inf)
            V = c.V[b][:, g // G].double()
            want_lse = torch.logsumexp(s, -1)
            p = torch.softmax(s, -1)                           # (the lse of far scores has lost the number of ties)
            o, size = p @ V, p @ V.abs()
            # what the rounding of a reference does to its row's exponents, it does to all alike
            bound = (HALF + 3e-4) * size + HALF * o.abs() + 1e-6
            err = (out[b, :m, g].double() - o).abs()
            assert torch.isfinite(err).all() and (err <= bound).all(), f"sequence {b}, head {g}: {(err / bound).max().item():.2f} of the bound"
            assert ((lse[b, :m, g].double() - want_lse).abs() <= 2e-4 + 1e-6 * want_lse.abs()).all()


def test_offsets_beyond_32_bits():
    c = TreeCase(43, [150], 8, Hq=8, Hkv=8, r_k=128, r_v=128)
    num_pages = 33000                                          # 2^31 elements are 32768 pages of 8 heads x 64 x 128
    kp = torch.empty(num_pages, 8, 64, 128, dtype=torch.bfloat16, device="cuda")
    vp = torch.empty(num_pages, 8, 64, 128, dtype=torch.bfloat16, device="cuda")
    for i, p in enumerate(c.batch.block_table[0].tolist()):
        kp[num_pages - 1 - i], vp[num_pages - 1 - i] = c.layer.k_pool[p], c.layer.v_pool[p]
        c.batch.block_table[0, i] = num_pages - 1 - i
    c.layer.k_pool, c.layer.v_pool = kp, vp
    c.check(*c.run())
    assert int(c.status) == 0


def test_bad_pages_and_lengths_are_reported():
    c = TreeCase(47, [200, 200], 8)
    want, _ = c.run()
    good = c.batch.block_table[0, 1].clone()
    for bad in (-1, c.layer.num_pages, 2 ** 31 - 1):
        c.batch.block_table[0, 1] = bad
        c.status.zero_()
        out, _ = c.run()
        assert int(c.status) == S.STIEF_ERR_BOUNDS
        assert torch.equal(out[1], want[1])
    c.batch.block_table[0, 1] = good
    for bad in (-5, 64 * c.batch.block_table.shape[1] - 7, 2 ** 31 - 1):
        c.batch.seq_lens[0] = bad
        c.status.zero_()
        out, _ = c.run()
        assert int(c.status) == S.STIEF_ERR_BOUNDS
        assert torch.equal(out[1], want[1]) and torch.isnan(out[0]).all()


def test_repeats_streams_and_graphs_give_the_same_bits():
    c = TreeCase(53, [9000, 100, 2500], 16, Hq=32, Hkv=8)
    want, want_lse = c.run()
    c.check(want, want_lse)
    for _ in range(3):
        out, lse = c.run()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out, lse = c.run()
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    out = torch.zeros_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.stief_tree_attention(c.layer, c.batch, c.q, c.mask, c.workspace, out, n_nodes=c.n_nodes)
        S.stief_tree_attention(c.layer, c.batch, c.q, c.mask, c.workspace, out, n_nodes=c.n_nodes)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    # the captured step serves other lengths and trees
    c.lens, c.counts = [c.lens[0] - 300, 60, 2500], [16, 16, 4]
    c.batch.seq_lens.copy_(torch.tensor(c.lens, dtype=torch.int32))
    c.n_nodes.copy_(torch.tensor(c.counts, dtype=torch.int32))
    out.fill_(NAN)
    graph.replay()
    torch.cuda.synchronize()
    for b in range(3):
        c.K[b], c.V[b] = c.K[b][:c.lens[b] + c.counts[b]], c.V[b][:c.lens[b] + c.counts[b]]
    c.check(out)


def test_two_streams_at_once():
    cases = [TreeCase(91, [6000, 100, 900], 20, Hq=32, Hkv=8), TreeCase(92, [70, 4000], 60, Hq=8, Hkv=2, r_k=96, r_v=128)]
    want = [c.run()[0] for c in cases]
    outs, streams = [torch.full_like(w, NAN) for w in want], [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(10):
        for c, o, s in zip(cases, outs, streams):
            with torch.cuda.stream(s):
                c.run(out=o, lse=False)
    torch.cuda.synchronize()
    assert all(torch.equal(o.view(torch.int16), w.view(torch.int16)) for o, w in zip(outs, want))
    assert all(int(c.status) == 0 for c in cases)


def test_refusals():
    c = TreeCase(3, [100], 8)
    out = torch.empty(1, 8, 8, 128, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(q=c.q.float()), dict(q=c.q[:, :, :4]), dict(out=out[..., :64]), dict(tree_mask=c.mask.long()), dict(tree_mask=c.mask[:, :4]),
                dict(n_nodes=c.n_nodes.long()), dict(batch=S.Batch(c.batch.block_table, c.batch.seq_lens.long())), dict(q=c.q.cpu()), dict(out_lse=torch.empty(1, 8, 4, device="cuda"))):
        args = dict(layer=c.layer, batch=c.batch, q=c.q, tree_mask=c.mask, workspace=c.workspace, out=out) | bad
        with pytest.raises(ValueError):
            S.stief_tree_attention(**args)
    l, bt = c.layer, c.batch.block_table
    wide = torch.cat([l.k_pool, l.k_pool], 3)[..., :l.r_k]                                  # rows that do not lie end to end
    for bad in (S.Layer(l.Hq, l.Hkv, l.r_k, l.r_v, l.U_k, l.U_v, wide, l.v_pool), S.Layer(l.Hq, l.Hkv, l.r_k, l.r_v, l.U_k, l.U_v, l.k_pool, l.v_pool[:-1]),
                S.Layer(l.Hq, l.Hkv, l.r_k, l.r_v, l.U_k[..., :32], l.U_v, l.k_pool, l.v_pool), S.Layer(l.Hq, l.Hkv, l.r_k, l.r_v, l.U_k, l.U_v.cpu(), l.k_pool, l.v_pool)):
        with pytest.raises(ValueError):
            S.stief_tree_attention(bad, c.batch, c.q, c.mask, c.workspace, out)
    with pytest.raises(ValueError):
        S.stief_tree_attention(l, S.Batch(torch.cat([bt, bt], 1)[:, ::2], c.batch.seq_lens), c.q, c.mask, c.workspace, out)
    with pytest.raises(S.StiefError) as e:
        S.stief_tree_attention(c.layer, c.batch, c.q, c.mask, c.workspace[:64], out)
    assert e.value.code == S.STIEF_ERR_WORKSPACE
    with pytest.raises(S.StiefError) as e:
        S.stief_tree_attention(c.layer, c.batch, c.q, c.mask, c.workspace, out, flags=1)
    assert e.value.code == S.STIEF_ERR_INVALID_ARG


# ---- accepting the drafted rows
@pytest.mark.parametrize("r_k,r_v,Hkv", [(64, 64, 8), (32, 128, 2), (48, 96, 1)])
def test_accept_moves_rows_in_every_layer(r_k, r_v, Hkv):
    g = torch.Generator().manual_seed(r_k)
    B, n, L, pages = 5, 200, 3, 40
    lens = torch.tensor([0, 63, 64, 130, 10], dtype=torch.int32)
    table = torch.randperm(pages, generator=g)[:B * 7].view(B, 7).to(torch.int32)
    layers = [S.Layer(Hkv, Hkv, r_k, r_v, None, None, torch.randn(pages, Hkv, 64, r_k, generator=g).bfloat16().cuda(),
                      torch.randn(pages, Hkv, 64, r_v, generator=g).bfloat16().cuda()) for _ in range(L)]
    count = torch.tensor([3, 150, 0, 1, 200], dtype=torch.int32)
    acc = torch.zeros(B, n, dtype=torch.int32)
    for b in range(B):
        acc[b, :count[b]] = torch.sort(torch.randperm(n, generator=g)[:count[b]]).values.to(torch.int32)
    want = []
    for l in layers:
        for pool in (l.k_pool, l.v_pool):
            w, old = pool.clone(), pool.clone()
            for b in range(B):
                for j in range(int(count[b])):
                    a, t = int(lens[b] + acc[b, j]), int(lens[b]) + j
                    w[table[b, t // 64], :, t % 64] = old[table[b, a // 64], :, a % 64]
            want.append(w)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    batch = S.Batch(table.cuda(), lens.cuda())
    S.stief_tree_accept(layers, batch, acc.cuda(), count.cuda(), status=status)
    assert int(status) == 0
    for got, w in zip((p for l in layers for p in (l.k_pool, l.v_pool)), want):
        assert torch.equal(got, w)
    S.stief_advance_seq_lens_by(batch.seq_lens, count.cuda())
    assert torch.equal(batch.seq_lens.cpu(), lens + count)


def test_accept_of_more_layers_than_one_launch_takes():
    L = 70
    pools = torch.randn(2 * L, 2, 1, 64, 32).bfloat16().cuda()
    want = pools.clone()
    want[:, 1, :, 5] = pools[:, 1, :, 7]
    layers = [S.Layer(1, 1, 32, 32, None, None, pools[2 * i], pools[2 * i + 1]) for i in range(L)]
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    S.stief_tree_accept(layers, S.Batch(i32(1).view(1, 1), i32(5)), i32(2).view(1, 1), i32(1))
    assert torch.equal(pools, want)


def test_accept_refuses_lists_that_are_not_increasing_or_leave_the_table():
    pool = torch.randn(4, 2, 64, 64).bfloat16().cuda()
    layer = S.Layer(2, 2, 64, 64, None, None, pool, pool.clone())
    before = pool.clone()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    batch = S.Batch(i32([[0, 1], [2, 3]]), i32([60, 100]))
    for acc, cnt in (([[3, 3], [0, 1]], [2, 0]), ([[5, 2], [0, 1]], [2, 0]), ([[-1, 2], [0, 1]], [2, 0]), ([[0, 68], [0, 1]], [2, 0]),
                     ([[0, 2 ** 31 - 1], [0, 1]], [2, 0]), ([[1, 2], [0, 1]], [3, 0]), ([[1, 2], [0, 1]], [-1, 0])):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        S.stief_tree_accept([layer], batch, i32(acc), i32(cnt), status=status)
        assert int(status) == S.STIEF_ERR_BOUNDS
        assert torch.equal(pool, before)
