"""Page operations of the cache against a plain model on the host, and a run of them with the attention calls that read the
pages.  Everything is integers or moved bits, so every comparison is exact."""
import pytest
import torch

import paper_2601_21686_b200 as S
from paper_2601_21686_b200 import inputs as I
from tests.test_gpu_tree import pack

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Model:
    """The same state as lists."""

    def __init__(self, B, width, num_pages):
        self.B, self.width = B, width
        self.rows, self.lens, self.refs = [[] for _ in range(B)], [0] * B, [0] * num_pages

    def free(self):
        return [p for p, n in enumerate(self.refs) if n == 0]

    def reserve(self, extra):
        free, short = self.free(), False
        for b in range(self.B):
            need = max(0, (self.lens[b] + extra[b] + 63) // 64 - len(self.rows[b]))
            for _ in range(need):
                if not free:
                    short = True
                    break
                p = free.pop(0)
                self.refs[p] = 1
                self.rows[b].append(p)
        return short

    def fork(self, parent):
        rows, lens, copies, wants = [], [], [], []
        for b, p in enumerate(parent):
            if p < 0:
                rows.append([])
                lens.append(0)
                continue
            heir = p if parent[p] == p else min(s for s in range(self.B) if parent[s] == p)
            rows.append(list(self.rows[p]) if heir == b else self.rows[p][:self.lens[p] // 64])
            lens.append(self.lens[p])
            if heir != b and self.lens[p] % 64:
                wants.append((b, self.rows[p][self.lens[p] // 64]))
        self.refs = [0] * len(self.refs)
        for r in rows:
            for p in r:
                self.refs[p] += 1
        free, short = self.free(), False
        for b, src in wants:
            if free:
                p = free.pop(0)
                copies.append((src, p))
                rows[b].append(p)
                self.refs[p] = 1
            else:
                short, lens[b] = True, 64 * len(rows[b])
        self.rows, self.lens = rows, lens
        return copies, short


class State:
    def __init__(self, B, width, num_pages, layers):
        self.model = Model(B, width, num_pages)
        self.table = S.PageTable(torch.full((B, width), -7, dtype=torch.int32, device="cuda"), i32([0] * B), i32([0] * B), i32([0] * num_pages))
        self.layers = layers
        self.work = torch.full((S.stief_pages_workspace_bytes(B, width),), 0xFF, dtype=torch.uint8, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def take_status(self):
        s = int(self.status)
        self.status.zero_()
        return s

    def check(self):
        m, t = self.model, self.table
        assert t.seq_lens.tolist() == m.lens and t.page_counts.tolist() == [len(r) for r in m.rows] and t.ref_counts.tolist() == m.refs
        for b, r in enumerate(m.rows):
            assert t.block_table[b, :len(r)].tolist() == r

    def reserve(self, extra):
        short = self.model.reserve(extra if isinstance(extra, list) else [extra] * self.model.B)
        S.stief_pages_reserve(self.table, i32(extra) if isinstance(extra, list) else extra, status=self.status)
        assert self.take_status() == (S.STIEF_ERR_NO_PAGES if short else 0)
        self.check()

    def grow(self, by):
        self.model.lens = [min(a + d, 64 * len(r)) for a, d, r in zip(self.model.lens, by, self.model.rows)]
        self.table.seq_lens.copy_(i32(self.model.lens))

    def fork(self, parent):
        pools = [t for l in self.layers for t in S._page_tensors(l)]
        want = [p.clone() for p in pools]
        copies, short = self.model.fork(parent)
        for w in want:
            for a, b in copies:
                w[b] = w[a]
        S.stief_pages_fork(self.table, self.layers, i32(parent), self.work, status=self.status)
        assert self.take_status() == (S.STIEF_ERR_NO_PAGES if short else 0)
        self.check()
        assert all(torch.equal(p.view(torch.uint8), w.view(torch.uint8)) for p, w in zip(pools, want))


def bf16_layers(n, num_pages, Hkv=2, ranks=((64, 64), (32, 128), (48, 96))):
    mk = lambda r: torch.randn(num_pages, Hkv, 64, r, device="cuda").to(torch.bfloat16)
    return [S.Layer(Hkv, Hkv, *ranks[i % len(ranks)], None, None, mk(ranks[i % len(ranks)][0]), mk(ranks[i % len(ranks)][1])) for i in range(n)]


def q8_layer(num_pages, Hkv=2, r_k=64, r_v=48):
    codes = lambda *s: torch.randint(0, 256, s, dtype=torch.uint8, device="cuda")
    return S.QLayer(Hkv, Hkv, r_k, r_v, None, None, None, codes(num_pages, Hkv, 64, r_k), codes(num_pages, Hkv, r_v, 64),
                    torch.randn(num_pages, Hkv, 64, 1, 2, device="cuda"))


@pytest.mark.parametrize("seed", range(6))
def test_random_sequences_of_operations(seed):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda lo, hi: int(torch.randint(lo, hi, (1,), generator=g))
    B, width, num_pages = rnd(1, 13), 8, rnd(20, 70)
    s = State(B, width, num_pages, bf16_layers(2, num_pages) + [q8_layer(num_pages)])
    for _ in range(12):
        room = [64 * width - a for a in s.model.lens]
        s.reserve([rnd(0, min(r, 200) + 1) for r in room] if rnd(0, 2) else min(rnd(0, 100), min(room)))
        s.grow([rnd(0, 150) for _ in range(B)])
        s.fork([rnd(-1, B) if rnd(0, 3) else b for b in range(B)])


def test_beams_of_many_layers_share_full_pages():
    B, num_pages, L = 16, 200, 70                            # more pools than one launch takes
    s = State(B, 6, num_pages, bf16_layers(L, num_pages, Hkv=1, ranks=((32, 32),)))
    s.reserve([300] + [0] * (B - 1))
    s.grow([300] + [0] * (B - 1))
    s.fork([0] * B)
    assert sum(x > 0 for x in s.model.refs) == 5 + B - 1 and max(s.model.refs) == B
    s.fork([b // 2 for b in range(B)])
    s.fork([B - 1 - b for b in range(B)])                    # a permutation copies nothing and moves every row
    s.fork([-1] * B)
    assert max(s.model.refs) == 0


def test_lengths_on_page_boundaries_need_no_copies():
    s = State(4, 4, 8, bf16_layers(1, 8))
    s.reserve([128, 64, 0, 0])
    s.grow([128, 64, 0, 0])
    s.fork([0, 0, 1, 1])
    assert s.model.lens == [128, 128, 64, 64] and sorted(s.model.refs)[-3:] == [2, 2, 2]


def test_running_out_of_pages():
    s = State(3, 4, 4, bf16_layers(1, 4))
    s.reserve([100, 0, 0])
    s.grow([100, 0, 0])
    s.fork([0, 0, 0])                                        # one full page shared, two copies for two free pages
    s.reserve([100, 1, 1])                                   # nothing left
    s.fork([0, 0, 0])
    s.fork([0, -1, -1])
    s.reserve([90, 0, 64])
    s.fork([0, 0, 0])


def test_many_slots_and_large_pools():
    B, num_pages = 1024, 9000
    s = State(B, 3, num_pages, bf16_layers(1, num_pages, Hkv=1, ranks=((32, 32),)))
    s.reserve([(b % 3) * 50 for b in range(B)])
    s.grow([(b % 3) * 50 for b in range(B)])
    s.fork([(b * 7 + 3) % B if b % 5 else b // 2 for b in range(B)])
    s.reserve(64)


def test_bad_values_are_reported_and_change_nothing_else():
    s = State(3, 4, 12, bf16_layers(1, 12))
    s.reserve(100)
    s.grow([100, 70, 30])
    S.stief_pages_fork(s.table, s.layers, i32([0, 3, -2]), s.work, status=s.status)      # no such slots: they stay
    assert s.take_status() == S.STIEF_ERR_BOUNDS
    s.check()
    S.stief_pages_reserve(s.table, i32([0, 10_000, -1]), status=s.status)
    assert s.take_status() == S.STIEF_ERR_BOUNDS
    s.check()
    pool = s.layers[0].k_pool.clone()
    S.stief_pages_copy(s.layers, i32([0, 12, 1]), i32([11, 2, -1]), status=s.status)
    assert s.take_status() == S.STIEF_ERR_BOUNDS
    pool[11] = pool[0]
    assert torch.equal(s.layers[0].k_pool, pool)


def test_copy_and_graph_replay():
    layers = bf16_layers(3, 20) + [q8_layer(20)]
    pools = [t for l in layers for t in S._page_tensors(l)]
    want = [p.clone() for p in pools]
    src, dst = i32([3, 9, 3, 0]), i32([4, 10, 11, 19])
    for w in want:
        w[dst.long()] = w[src.long()]
    S.stief_pages_copy(layers, src, dst)
    assert all(torch.equal(p.view(torch.uint8), w.view(torch.uint8)) for p, w in zip(pools, want))
    S.stief_pages_copy(layers, src[:0], dst[:0])
    s = State(4, 6, 40, bf16_layers(2, 40))
    s.reserve([200, 0, 0, 0])
    s.grow([200, 0, 0, 0])
    parent, extra = i32([0, 0, 0, 0]), i32([5, 6, 7, 8])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.stief_pages_fork(s.table, s.layers, parent, s.work)
        S.stief_pages_reserve(s.table, extra)
    for p in ([0, 0, 0, 0], [3, 3, 1, 1], [2, 2, -1, 0], [0, 1, 0, 3]):
        parent.copy_(i32(p))
        graph.replay()
        s.model.fork(p)
        s.model.reserve([5, 6, 7, 8])
        s.check()


def test_refusals():
    s = State(2, 4, 8, bf16_layers(1, 8))
    with pytest.raises(S.StiefError) as e:
        S.stief_pages_fork(s.table, s.layers, i32([0, 1]), s.work[:64])
    assert e.value.code == S.STIEF_ERR_WORKSPACE
    with pytest.raises(S.StiefError):
        S.stief_pages_reserve(s.table, -1)
    with pytest.raises(ValueError):
        S.stief_pages_reserve(s.table, (1 << 32) + 1)
    with pytest.raises(ValueError):
        S.stief_pages_fork(s.table, s.layers, i32([0, 1, 2]), s.work)
    with pytest.raises(ValueError):
        S.stief_pages_fork(s.table, bf16_layers(1, 5), i32([0, 1]), s.work)            # pools smaller than the table
    with pytest.raises(ValueError):
        S.stief_pages_copy(s.layers, i32([0]).long(), i32([1]))
    with pytest.raises(ValueError):
        S.PageTable(s.table.block_table.cpu(), s.table.seq_lens, s.table.page_counts, s.table.ref_counts).c()


def test_prompt_draft_accept_and_beams_in_one_run():
    """A server's life: prompts attended and compressed, a tree drafted, verified and accepted, beams forked and decoded.  The
    cache the run leaves is the one that feeding the kept tokens one by one leaves, and so is what decode reads from it."""
    Hq, Hkv, r, lens, n = 8, 2, 64, [150, 70], 6
    B, width, num_pages, L = 4, 6, 24, 2
    U = [tuple(u.cuda() for u in I.stiefel_bases(3, l, Hkv, r, r)) for l in range(L)]
    mk = lambda l: S.Layer(Hq, Hkv, r, r, U[l][0], U[l][1], torch.zeros(num_pages, Hkv, 64, r, dtype=torch.bfloat16, device="cuda"),
                           torch.zeros(num_pages, Hkv, 64, r, dtype=torch.bfloat16, device="cuda"))
    s = State(B, width, num_pages, [mk(l) for l in range(L)])
    s.table.block_table.zero_()
    g = torch.Generator().manual_seed(9)
    rand = lambda *shape: torch.randn(*shape, generator=g).to(torch.bfloat16).cuda()
    s.reserve(lens + [0, 0])
    qkv = [rand(sum(lens), Hq + 2 * Hkv, 128) for _ in range(L)]
    cu, status = i32([0, lens[0], sum(lens)]), s.status
    s.model.lens = lens + [0, 0]
    s.table.seq_lens.copy_(i32(s.model.lens))
    for l, layer in enumerate(s.layers):
        out = torch.empty(sum(lens), Hq, 128, dtype=torch.bfloat16, device="cuda")
        S.stief_prompt_attention(qkv[l][:, :Hq], qkv[l][:, Hq:Hq + Hkv], qkv[l][:, Hq + Hkv:], cu, out, status=status)
        assert torch.isfinite(out).all()
        for b in range(2):
            lo, hi = cu[b], cu[b + 1]
            kv = qkv[l][lo:hi].contiguous()[None]
            one = S.Batch(s.table.block_table[b:b + 1], s.table.seq_lens[b:b + 1])
            S.stief_prefill_compress(layer, one, kv[:, :, Hq:Hq + Hkv], kv[:, :, Hq + Hkv:], status=status)
    # a chain 0-1-4 and two side branches 0-2, 0-3-5; slots 2 and 3 are idle
    up, counts = [-1, 0, 0, 0, 1, 3], i32([n, n, 0, 0])
    m = torch.zeros(B, n, n, dtype=torch.bool)
    for i in range(n):
        m[:, i, i] = True
        if up[i] >= 0:
            m[:, i] |= m[:, up[i]]
    s.reserve([n, n, 0, 0])
    dk, dv, dq = [rand(B, n, Hkv, 128) for _ in range(L)], [rand(B, n, Hkv, 128) for _ in range(L)], [rand(B, n, Hq, 128) for _ in range(L)]
    ws = torch.zeros(S.stief_tree_workspace_bytes(B, n, Hq, Hkv, r), dtype=torch.uint8, device="cuda")
    touts = []
    for l, layer in enumerate(s.layers):
        S.stief_append_chunk(layer, s.table.batch, dk[l], dv[l], chunk_lens=counts, status=status)
        touts.append(torch.zeros(B, n, Hq, 128, dtype=torch.bfloat16, device="cuda"))
        S.stief_tree_attention(layer, s.table.batch, dq[l], pack(m).cuda(), ws, touts[-1], n_nodes=counts, status=status)
    acc, cnt = i32([[0, 1, 4], [0, 3, 5], [0, 0, 0], [0, 0, 0]]), i32([3, 2, 0, 0])
    S.stief_tree_accept(s.layers, s.table.batch, acc, cnt, status=status)
    S.stief_advance_seq_lens_by(s.table.seq_lens, cnt)
    s.model.lens = [lens[0] + 3, lens[1] + 2, 0, 0]
    s.fork([0, 1, 0, 1])
    assert s.take_status() == 0
    # the same tokens one by one through the decode step, on a cache of its own
    ref = State(B, width, num_pages, [mk(l) for l in range(L)])
    ref.table.block_table.zero_()
    ref.reserve([64 * 5] * B if num_pages >= 20 else lens)
    order, where = [[0, 1, 4], [0, 3, 5]], [0, 1, 0, 1]
    ref.model.lens = [lens[w] for w in where]
    ref.table.seq_lens.copy_(i32(ref.model.lens))
    dws = torch.zeros(S.stief_decode_workspace_bytes(B, Hq, Hkv, r), dtype=torch.uint8, device="cuda")
    for l, layer in enumerate(ref.layers):
        for b in range(B):
            lo, hi = cu[where[b]], cu[where[b] + 1]
            kv = qkv[l][lo:hi].contiguous()[None]
            S.stief_prefill_compress(layer, S.Batch(ref.table.block_table[b:b + 1], ref.table.seq_lens[b:b + 1]), kv[:, :, Hq:Hq + Hkv], kv[:, :, Hq + Hkv:], status=status)
    for j in range(3):
        for l, layer in enumerate(ref.layers):
            pick = lambda t: torch.stack([t[l][where[b], order[where[b]][j]] for b in range(B)])
            out = torch.empty(B, Hq, 128, dtype=torch.bfloat16, device="cuda")
            S.stief_decode_step(layer, ref.table.batch, pick(dq), pick(dk), pick(dv), dws, out, status=status)
            for b in range(2):                               # a chain's node attends exactly what the token would
                if j < int(cnt[b]):
                    assert (out[b].float() - touts[l][b, order[b][j]].float()).abs().max() < 1e-2
        ref.table.seq_lens.add_(1)
    ref.table.seq_lens.copy_(s.table.seq_lens)
    for l in range(L):
        outs = []
        q, k, v = rand(B, Hq, 128), rand(B, Hkv, 128), rand(B, Hkv, 128)
        for st in (s, ref):
            st.layers[l].U_k, st.layers[l].U_v = U[l]
            out = torch.empty(B, Hq, 128, dtype=torch.bfloat16, device="cuda")
            S.stief_decode_step(st.layers[l], st.table.batch, q, k, v, dws, out, status=status)
            outs.append(out)
        assert torch.equal(outs[0], outs[1])
    assert int(status) == 0
