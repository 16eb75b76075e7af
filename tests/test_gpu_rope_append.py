"""New tokens into the bf16 and the 8-bit cache with the rotation on the way, against the definition in fp64.  Tolerances are
error bounds: a rotated channel takes three fp32 roundings (2^-24 each) of |a cos| + |b sin|; a rotated key goes into the product
in two bf16 terms (off by 2^-16 of the value) or three (2^-24); fp32 sums of 128 products are off by at most 128 * 2^-24 of the
sum of magnitudes, doubled for the tensor core's own order and truncation; outputs are rounded once (half a step, eps / 2)."""
import math

import pytest
import torch

import paper_2601_21686_b200 as S

pytestmark = pytest.mark.gpu
BF, F8 = torch.bfloat16, torch.float8_e4m3fn
HALF = torch.finfo(BF).eps / 2
HALF8 = torch.finfo(F8).eps / 2
SUM = 256 * 2.0 ** -24


def to_e4m3(x):
    """Doubles rounded to the nearest e4m3 value, ties to even."""
    step = torch.ldexp(torch.ones_like(x), torch.frexp(x)[1].clamp(min=-5) - 4)
    return torch.round(x / step) * step


def scale_for(top):
    """Least power of two s with top <= 448 s, exponents -100 .. 119 (one value)."""
    e = -100
    while e < 119 and top > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def table(max_pos, rot, device="cuda"):
    a = torch.arange(max_pos, device=device, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, device=device, dtype=torch.float64) / rot)
    return torch.cat([a.cos(), a.sin()], 1).float()


def rotate(x, pos, tab, interleaved):
    """Rows [n, heads, 128] in fp64, and the sums of magnitudes that the rounding of each channel goes by."""
    x, half = x.double(), tab.shape[1] // 2
    c, s = tab[pos].double()[:, None, :half], tab[pos].double()[:, None, half:]
    y, size = x.clone(), x.abs()
    ia = torch.arange(half, device=x.device) * (2 if interleaved else 1)
    ib = ia + (1 if interleaved else half)
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    size[..., ia], size[..., ib] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
    return y, size


class Case:
    """B sequences with `lens` cached tokens and `counts` new ones.  The pools start with random rows; everything that the call has
    to leave alone is compared with them bit by bit."""

    def __init__(self, seed, lens, counts, f8=False, Hq=8, Hkv=2, r_k=64, r_v=64, rot=128, inter=False, fold_k=False, fold_v=False, shared=False,
                 front=0, behind=0, ends=False, positions=False, pages=0, k_scale=4.0, queries=True):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        c = torch.Generator()
        c.manual_seed(seed)
        self.f8, self.rot, self.inter, self.ends, self.lens, self.counts, self.front = f8, rot, inter, ends, list(lens), list(counts), front
        B, total = len(lens), front + sum(counts) + behind
        need = [(a + n + 63) // 64 for a, n in zip(lens, counts)]
        self.P = max(sum(need) + 2, pages)
        order = torch.randperm(self.P, generator=c)
        tab = torch.full((B, max(max(need), 1)), -7, dtype=torch.int32)           # entries that no token needs are never looked at
        at = 0
        for b, n in enumerate(need):
            tab[b, :n] = order[at:at + n].to(torch.int32)
            at += n
        self.table = tab
        basis = lambda r: torch.linalg.qr(torch.randn(1 if shared else Hkv, 128, 128, generator=g, device="cuda", dtype=torch.float64))[0][:, :, :r].to(BF).contiguous()  # noqa: E731
        U = [None if fold_k else basis(r_k), None if fold_v else basis(r_v)]
        if f8:
            codes = [(60 * torch.randn(self.P, Hkv, 64, r, generator=g, device="cuda")).clamp(-448, 448).to(F8) for r in (r_k, r_v)]
            scales = torch.full((self.P, Hkv, 4), 7.0, device="cuda")
            scales[:, :, :2] = torch.exp2(torch.randint(-9, -2, (self.P, Hkv, 2), generator=c).float()).cuda()
            self.layer = S.F8Layer(Hq, Hkv, r_k, r_v, *U, *codes, scales)
            self.before = [codes[0].clone(), codes[1].clone(), scales.clone()]
        else:
            pools = [torch.randn(self.P, Hkv, 64, r, generator=g, device="cuda").to(BF) for r in (r_k, r_v)]
            self.layer = S.Layer(Hq, Hkv, r_k, r_v, *U, *pools)
            self.before = [p.clone() for p in pools]
        wide = torch.randn(total, Hq + 2 * Hkv, 128, generator=g, device="cuda").to(BF)
        self.q = wide[:, :Hq] if queries else None
        spread = torch.exp2(torch.linspace(2, -3, 128, device="cuda"))
        self.k = wide[:, Hq:Hq + Hkv] if not fold_k else torch.randn(total, Hkv, r_k, generator=g, device="cuda").to(BF)
        self.v = wide[:, Hq + Hkv:] if not fold_v else torch.randn(total, Hkv, r_v, generator=g, device="cuda").to(BF)
        if not fold_k:
            self.k.copy_((k_scale * wide[:, Hq:Hq + Hkv].float() * spread).to(BF))
        cu = [front]
        for n in counts:
            cu.append(cu[-1] + n)
        self.cu_list, self.cu = cu, torch.tensor(cu, dtype=torch.int32, device="cuda")
        self.batch = S.Batch(tab.cuda(), torch.tensor([a + (n if ends else 0) for a, n in zip(lens, counts)], dtype=torch.int32, device="cuda"))
        self.max_pos = max(a + n for a, n in zip(lens, counts)) + 5
        self.rotation = S.Rotation(table(self.max_pos, rot), interleaved=inter) if rot else None
        self.positions = torch.randint(0, self.max_pos, (total,), generator=c).to(torch.int32).cuda() if positions else None
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        if not rot:
            self.q = None
        self.q_out = None if self.q is None else torch.full((total, Hq, 128), float("nan"), dtype=BF, device="cuda")

    def call(self, **kw):
        fn = S.stief_f8_append if self.f8 else S.stief_rope_append
        args = dict(rotation=self.rotation, q=self.q, q_out=self.q_out, positions=self.positions, ends_at_len=self.ends, status=self.status)
        args.update(kw)
        fn(self.layer, self.batch, self.k, self.v, self.cu, **args)
        return self

    def pools(self):
        L = self.layer
        return [L.k_codes, L.v_codes] if self.f8 else [L.k_pool, L.v_pool]

    def check(self, status=0, skip_pages=()):
        L, dev = self.layer, "cuda"
        torch.cuda.synchronize()
        assert self.status.item() == status
        total = self.k.shape[0]
        place = torch.full((total,), -1, dtype=torch.long)
        for b, (a, n) in enumerate(zip(self.lens, self.counts)):
            place[self.cu_list[b]:self.cu_list[b + 1]] = torch.arange(a, a + n)
        mine = (place >= 0).to(dev)
        pos = (place.clamp(min=0).to(dev) if self.positions is None else self.positions.long()) if self.rot else torch.zeros(total, dtype=torch.long, device=dev)
        good = mine & (pos >= 0) & (pos < self.max_pos)
        pos = pos.clamp(0, self.max_pos - 1)
        if self.q is not None:
            y, size = rotate(self.q, pos, self.rotation.table, self.inter)
            assert torch.isnan(self.q_out[~good]).all(), "a token of no sequence was written"
            assert ((self.q_out.double() - y).abs() <= HALF * y.abs() + 4 * 2.0 ** -24 * size + 1e-30)[good].all()
        sides = []
        for x, U, turned in ((self.k, L.U_k, self.rot > 0), (self.v, L.U_v, False)):
            y, size = rotate(x, pos, self.rotation.table, self.inter) if turned else (x.double(), x.double().abs())
            off = (3 * 2.0 ** -24 + (2.0 ** -24 if self.f8 else HALF * HALF)) if turned else 0.0
            if U is None:
                sides.append((y, off * size))
                continue
            Ud = U.double().expand(L.Hkv, -1, -1)
            sides.append((torch.einsum("thd,hdr->thr", y, Ud), (off + SUM) * torch.einsum("thd,hdr->thr", size, Ud.abs())))
        want = [p.clone() for p in self.before]
        touched = [torch.zeros(p.shape[:3], dtype=torch.bool, device=dev) for p in self.before[:2]]
        for b, (a, n) in enumerate(zip(self.lens, self.counts)):
            for pi in range(a // 64, (a + n + 63) // 64 if n else 0):
                page = int(self.table[b, pi])
                lo, hi = max(a, pi * 64), min(a + n, pi * 64 + 64)
                tok = torch.arange(self.cu_list[b] + lo - a, self.cu_list[b] + hi - a, device=dev)
                ok = good[tok]
                if page in skip_pages or not ok.any():
                    continue
                for i, (rows, err) in enumerate(sides):
                    got, r, e = self.pools()[i][page, :, lo % 64:lo % 64 + hi - lo], rows[tok].transpose(0, 1), err[tok].transpose(0, 1)
                    touched[i][page, :, lo % 64:lo % 64 + hi - lo] = ok
                    if not self.f8:
                        worst = ((got.double() - r).abs() - HALF * r.abs() - e)[:, ok]
                        assert torch.isfinite(got[:, ok]).all() and (worst <= 1e-30).all(), f"side {i}, sequence {b}, page {pi}"
                        continue
                    for h in range(L.Hkv):
                        s = scale_for(r[h][ok].abs().max().item())
                        if lo % 64:
                            old = self.before[2][page, h, i].item()
                            s = max(s, old)
                            want[i][page, h, :lo % 64] = to_e4m3(self.before[i][page, h, :lo % 64].double() * (old / s)).to(F8)
                        want[2][page, h, i] = s
                        assert L.scales[page, h, i].item() == s, f"scale of side {i}, sequence {b}, page {pi}, head {h}"
                        v = r[h][ok] / s
                        off = (got[h][ok].double() - v).abs() - (HALF8 * v.abs()).clamp(min=2.0 ** -10) - e[h][ok] / s
                        assert (off <= 0).all(), f"side {i}, sequence {b}, page {pi}, head {h}"
                        assert (got[h][ok].double() != to_e4m3(v)).sum() <= 1 + v.numel() // 1000
        for i, p in enumerate(self.pools()):
            same = p.view(torch.uint8 if self.f8 else torch.int16) == want[i].view(torch.uint8 if self.f8 else torch.int16)
            assert (same | touched[i][..., None]).all(), "rows that no token belongs to were written"
        if self.f8:
            assert torch.equal(L.scales, want[2])


RAGGED = ([0, 63, 64, 100, 5, 0, 190, 7], [1, 1, 65, 0, 200, 64, 130, 57])


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("r_k,r_v", [(32, 32), (48, 96), (64, 64), (96, 48), (128, 128), (128, 32), (64, 128)])
def test_ragged_batch(f8, r_k, r_v):
    Case(r_k + r_v, *RAGGED, f8=f8, r_k=r_k, r_v=r_v).call().check()


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("rot,inter", [(128, True), (64, False), (64, True), (16, False), (96, False), (112, True), (0, False)])
def test_rotations(f8, rot, inter):
    Case(rot, *RAGGED, f8=f8, rot=rot, inter=inter, r_k=64, r_v=48).call().check()


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("Hq,Hkv", [(32, 8), (8, 8), (10, 2), (6, 6), (4, 1), (1, 1), (64, 4), (9, 3)])
def test_heads_and_strides(f8, Hq, Hkv):
    Case(Hq, [3, 70], [40, 33], f8=f8, Hq=Hq, Hkv=Hkv).call().check()


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("n", [1, 2, 17, 64, 256, 1024])
def test_one_token_per_sequence(f8, n):
    Case(n, [(37 * i) % 131 for i in range(n)], [1] * n, f8=f8, r_k=96, r_v=64).call().check()


@pytest.mark.parametrize("f8", [False, True])
def test_places_positions_and_gaps(f8):
    Case(1, *RAGGED, f8=f8, front=5, behind=9).call().check()
    Case(2, *RAGGED, f8=f8, ends=True).call().check()
    Case(3, *RAGGED, f8=f8, positions=True, ends=True, front=1).call().check()
    Case(4, [0], [0], f8=f8, behind=3).call().check()
    c = Case(5, [64], [1], f8=f8)                                          # tensors of one token carry any stride
    c.k = c.k.as_strided(c.k.shape, (3, 128, 1))
    c.call().check()


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("fold_k,fold_v,r_k,r_v,rot", [(True, True, 128, 128, 128), (True, False, 48, 64, 0), (False, True, 64, 96, 64), (True, True, 32, 48, 0)])
def test_sides_without_basis(f8, fold_k, fold_v, r_k, r_v, rot):
    c = Case(7, *RAGGED, f8=f8, fold_k=fold_k, fold_v=fold_v, r_k=r_k, r_v=r_v, rot=rot).call()
    c.check()
    if not f8 and fold_v:                                                   # stored as they are
        assert torch.equal(c.layer.v_pool[int(c.table[4, 1]), :, 0], c.v[c.cu_list[4] + 59])


@pytest.mark.parametrize("f8", [False, True])
def test_shared_key_basis_and_queries_in_place(f8):
    c = Case(8, *RAGGED, f8=f8, shared=True)
    first = c.q.clone()
    c.call(q_out=c.q)
    c.q_out, c.q = c.q.clone(), first
    c.check()


@pytest.mark.parametrize("f8", [False, True])
def test_no_queries(f8):
    Case(9, *RAGGED, f8=f8, queries=False).call().check()


@pytest.mark.parametrize("f8", [False, True])
def test_bad_pages_and_positions_are_skipped(f8):
    c = Case(10, *RAGGED, f8=f8)
    gone = int(c.table[4, 1])
    c.batch.block_table[4, 1] = c.P                                         # a page outside the pool: its tokens alone are lost
    c.call().check(status=S.STIEF_ERR_BOUNDS, skip_pages=(gone,))
    c = Case(11, *RAGGED, f8=f8, positions=True)
    c.positions[c.cu_list[4] + 3:c.cu_list[4] + 70] = c.max_pos
    c.positions[c.cu_list[6]] = -1
    c.call().check(status=S.STIEF_ERR_BOUNDS)
    c = Case(12, [64, 0], [1, 200], f8=f8)
    gone = [int(x) for x in c.table[1, 2:]]
    c.batch = S.Batch(c.batch.block_table[:, :2].contiguous(), c.batch.seq_lens)   # places behind the table
    c.call().check(status=S.STIEF_ERR_BOUNDS, skip_pages=gone)
    for bad in ((-1, 9, 20), (0, 9, 21), (9, 3, 20)):                       # ranges that do not fit: nothing of those sequences is written
        c = Case(13, [5, 70], [9, 11], f8=f8)
        c.cu.copy_(torch.tensor(bad, dtype=torch.int32))
        c.call()
        torch.cuda.synchronize()
        assert c.status.item() == S.STIEF_ERR_BOUNDS
        page = int(c.table[1, 1])
        kept = torch.equal(c.pools()[0][page].view(torch.uint8), c.before[0][page].view(torch.uint8))
        assert kept == (bad == (0, 9, 21))                                  # the second ranges (9, 20) and (3, 20) are in order
        page = int(c.table[0, 0])
        assert torch.equal(c.pools()[0][page].view(torch.uint8), c.before[0][page].view(torch.uint8)) == (bad != (0, 9, 21))
    for lens, ends in ((-1, False), (2 ** 31 - 1, False), (2 ** 31 - 1, True), (8, True), (-5, True)):
        c = Case(14, [5], [9], f8=f8)
        c.batch.seq_lens.fill_(lens)                                        # (8 tokens in all cannot end with 9 new ones)
        c.call(ends_at_len=ends)
        torch.cuda.synchronize()
        assert c.status.item() == S.STIEF_ERR_BOUNDS
        assert all(torch.equal(p.view(torch.uint8), w.view(torch.uint8)) for p, w in zip(c.pools(), c.before))


def test_growing_scales_move_older_rows_and_keep_their_values():
    """Tokens one by one with magnitudes that grow and shrink: the scale is the block's least, whatever the order."""
    torch.manual_seed(0)
    Hkv, r = 2, 64
    codes = [torch.full((3, Hkv, 64, r), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(2)]       # NaN where nothing was written
    L = S.F8Layer(4, Hkv, r, r, None, None, *codes, torch.full((3, Hkv, 4), float("nan"), device="cuda"))
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    batch, cu = S.Batch(torch.tensor([[2, 0]], dtype=torch.int32, device="cuda"), lens), torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    rows = torch.randn(70, Hkv, r, device="cuda") * torch.exp2(torch.randint(-3, 6, (70, 1, 1), device="cuda").float())
    rows[5] = 0.0
    rows = rows.to(BF)
    for t in range(70):
        S.stief_f8_append(L, batch, rows[t:t + 1], rows[t:t + 1], cu)
        S.stief_advance_seq_lens(lens, 1)
    for page, lo, hi in ((2, 0, 64), (0, 64, 70)):
        for side, got in enumerate(codes):
            for h in range(Hkv):
                s = scale_for(rows[lo:hi, h].abs().max().item())
                assert L.scales[page, h, side].item() == s
                value = got[page, h, :hi - lo].view(F8).double() * s
                x = rows[lo:hi, h].double()
                # rounded once at its first scale, and once more at each growth where it is below 2^-6 of the new scale: 2^-10 s each, halving backwards
                assert ((value - x).abs() <= HALF8 * x.abs() + 2 * 2.0 ** -10 * s).all()
                assert (got[page, h, hi - lo:] == 0x7F).all()
    assert torch.isnan(L.scales[1]).all() and torch.isnan(L.scales[:, :, 2:]).all()


def test_infinities_nan_and_extreme_rows_in_the_8_bit_cache():
    Hkv, r = 1, 32
    codes = [torch.zeros(1, Hkv, 64, r, dtype=torch.uint8, device="cuda") for _ in range(2)]
    L = S.F8Layer(1, Hkv, r, r, None, None, *codes, torch.zeros(1, Hkv, 4, device="cuda"))
    batch = S.Batch(torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"))
    for x, scale in ((448.0, 1.0), (450.0, 2.0), (224.0, 0.5), (225.0, 1.0), (0.0, 2.0 ** -100), (1e-40, 2.0 ** -100), (3e38, 2.0 ** 119), (-7.0, 2.0 ** -6)):
        rows = torch.zeros(4, Hkv, r, dtype=BF, device="cuda")
        rows[0, 0, 0] = x
        rows[1, 0, 1], rows[1, 0, 2], rows[1, 0, 3] = float("inf"), -float("inf"), float("nan")
        S.stief_f8_append(L, batch, rows, rows, torch.tensor([0, 4], dtype=torch.int32, device="cuda"))
        assert L.scales[0, 0, 0].item() == scale and L.scales[0, 0, 1].item() == scale
        want = to_e4m3(rows[:, 0].double() / scale).clamp(-448, 448)
        got = codes[0][0, 0, :4].view(F8).double()
        assert torch.isnan(got[1, 1:4]).all()
        got[1, 1:4] = want[1, 1:4] = 0.0
        assert torch.equal(got, want)


@pytest.mark.parametrize("f8", [False, True])
def test_places_far_into_a_large_pool(f8):
    """Byte and element offsets beyond 2^32."""
    Hkv, r = 8, 128
    P = (2 ** 32 // (Hkv * 64 * r)) + 9
    c = Case(15, [64 * 3 - 2], [5], f8=f8, Hkv=2)
    pool = lambda t: torch.empty(P, Hkv, 64, r, dtype=t, device="cuda")  # noqa: E731
    kp, vp = (pool(torch.uint8), pool(torch.uint8)) if f8 else (pool(BF), pool(BF))
    U = torch.linalg.qr(torch.randn(Hkv, 128, 128, device="cuda"))[0].to(BF).contiguous()
    L = S.F8Layer(8, Hkv, r, r, U, U, kp, vp, torch.zeros(P, Hkv, 4, device="cuda")) if f8 else S.Layer(8, Hkv, r, r, U, U, kp, vp)
    small = S.F8Layer(8, Hkv, r, r, U, U, kp[:4].clone(), vp[:4].clone(), torch.zeros(4, Hkv, 4, device="cuda")) if f8 else S.Layer(8, Hkv, r, r, U, U, kp[:4].clone(), vp[:4].clone())
    k, v = torch.randn(5, Hkv, 128, device="cuda").to(BF), torch.randn(5, Hkv, 128, device="cuda").to(BF)
    fn = S.stief_f8_append if f8 else S.stief_rope_append
    for layer, ids in ((L, [0, 1, P - 2, P - 1]), (small, [0, 1, 2, 3])):
        if f8:
            layer.k_codes[ids[2]] = 0
            layer.v_codes[ids[2]] = 0
        fn(layer, S.Batch(torch.tensor([ids], dtype=torch.int32, device="cuda"), c.batch.seq_lens), k, v, c.cu, rotation=S.Rotation(table(300, 128)), status=c.status)
    a, b = ((L.k_codes, L.v_codes), (small.k_codes, small.v_codes)) if f8 else ((L.k_pool, L.v_pool), (small.k_pool, small.v_pool))
    for x, y in zip(a, b):
        assert torch.equal(x[P - 2, :, 62:].view(torch.uint8), y[2, :, 62:].view(torch.uint8)) and torch.equal(x[P - 1, :, :3].view(torch.uint8), y[3, :, :3].view(torch.uint8))
    assert c.status.item() == 0


@pytest.mark.parametrize("f8", [False, True])
def test_captured_and_replayed(f8):
    """A captured decode step (append, advance) replayed over page borders equals the same tokens in one chunk."""
    n = 70
    one, many = Case(16, [61], [n], f8=f8, r_k=64, r_v=96), Case(16, [61], [n], f8=f8, r_k=64, r_v=96)
    many.call().check()
    k, v, q, out = (torch.empty_like(x[:1]) for x in (one.k, one.v, one.q, one.q_out))
    cu = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    call = S.stief_f8_append if f8 else S.stief_rope_append
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        call(one.layer, one.batch, k, v, cu, rotation=one.rotation, q=q, q_out=out)
        S.stief_advance_seq_lens(one.batch.seq_lens, 1)
    for t in range(n):
        for dst, src in ((k, one.k), (v, one.v), (q, one.q)):
            dst.copy_(src[t:t + 1])
        graph.replay()
        assert torch.equal(out[0], many.q_out[t])
    for a, b in zip(one.pools(), many.pools()):
        if f8:                                                             # a value below 2^-6 may have been rounded again as its page's scale grew
            x, y = a.double(), b.double()
            assert torch.where(y.abs() <= 2.0 ** -6, (x - y).abs() <= 2.0 ** -9, x == y).all()
        else:
            assert torch.equal(a, b)
    if f8:
        assert torch.equal(one.layer.scales, many.layer.scales)


@pytest.mark.parametrize("f8", [False, True])
def test_many_sequences_of_a_few_tokens(f8):
    """Tiles of several pages each, pages without a valid token among them."""
    counts = [(5 * i) % 4 for i in range(600)]
    c = Case(19, [(11 * i) % 70 for i in range(600)], counts, f8=f8, Hq=4, Hkv=1, r_k=48, r_v=32, positions=True)
    for b in range(0, 600, 7):
        c.positions[c.cu_list[b]:c.cu_list[b + 1]] = -3
    c.call().check(status=S.STIEF_ERR_BOUNDS)
    Case(20, [3] * 300, [20] * 300, f8=f8, Hq=2, Hkv=2, r_k=96, r_v=96, rot=32).call().check()


def test_two_streams_at_once():
    a, b = Case(17, *RAGGED, f8=True), Case(18, *RAGGED, f8=True, r_k=96, r_v=128)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for c, s in zip((a, b), streams):
        with torch.cuda.stream(s):
            c.call()
    torch.cuda.synchronize()
    a.check()
    b.check()


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("where", ["behind the pool", "before the pool", "behind the table"])
@pytest.mark.parametrize("lens,counts", [([100], [9]), ([100, 70], [9, 300]), ([64 * (i % 4) + 5 * (i % 3) for i in range(300)], [1 + i % 4 for i in range(300)])])
def test_memory_around_the_pools_is_left_alone(f8, where, lens, counts):
    """Pages outside the pool, one page to a tile and several, with older rows in front of the new ones and without.  The pools lie in
    the middle of larger buffers."""
    c = Case(21, lens, counts, f8=f8, Hq=4, Hkv=2, r_k=64, r_v=48)
    L, around = c.layer, []
    for name in ("k_codes", "v_codes", "scales") if f8 else ("k_pool", "v_pool"):
        t = getattr(L, name)
        big = torch.randint(0, 256, (t.shape[0] + 4, t[0].numel() * t.element_size()), dtype=torch.uint8, device="cuda")
        big[2:-2] = t.view(torch.uint8).view(t.shape[0], -1)
        setattr(L, name, big[2:-2].view(t.dtype).view(t.shape))
        around.append((big, big[:2].clone(), big[-2:].clone()))
    last = [(a + n - 1) // 64 for a, n in zip(lens, counts)]
    if where == "behind the table":
        width = max(last)
        gone = [int(c.table[b, i]) for b, i in enumerate(last) if i == width]
        c.batch = S.Batch(c.batch.block_table[:, :width].contiguous(), c.batch.seq_lens)
    else:
        gone = [int(c.table[b, i]) for b, i in enumerate(last) if b % 2 == 0]
        for b, i in enumerate(last):
            if b % 2 == 0:
                c.batch.block_table[b, i] = c.P if where == "behind the pool" else -1
    c.call().check(status=S.STIEF_ERR_BOUNDS, skip_pages=gone)
    for big, front, back in around:
        assert torch.equal(big[:2], front) and torch.equal(big[-2:], back)


@pytest.mark.parametrize("f8", [False, True])
def test_no_tokens_at_all(f8):
    Case(22, [5, 0, 70], [0, 0, 0], f8=f8).call().check()
    Case(23, [5], [0], f8=f8, queries=False, rot=0).call().check()
