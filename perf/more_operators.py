"""Workloads of the block-scaled 8-bit cache and of the rotation on the way into the cache, each with a plain torch form of
the same computation: new tokens rotated by their position, projected and stored in the paged cache (bf16, and e4m3 with one
power-of-two scale for each page and KV head), and attention over the 8-bit cache for one query token per sequence and for
runs of query tokens.

``own = False`` computes the operators with elementary torch operations in fp32; ``own = True`` calls this package."""
import math

import torch

own = False

PAGE, D = 64, 128
SCALE = 1.0 / math.sqrt(D)
TOP = 448.0                       # the largest e4m3 value
LOWEST, HIGHEST = -100, 119       # exponents that a block's scale can have
F8 = torch.float8_e4m3fn


# ------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one new token of one sequence into the bf16 cache: the call whose latency every decode step pays
        {"name": "append-step", "op": "append", "f8": False, "Hq": 32, "Hkv": 8, "r_k": 64, "r_v": 64, "B": 1, "n": 1, "ragged": False, "T": 1021, "rot": 128, "inter": False, "draft": False},
        # drafted tokens of 16 sequences, rotated by their depth in the tree; interleaved pairs, half of the channels
        {"name": "append-drafts", "op": "append", "f8": False, "Hq": 32, "Hkv": 8, "r_k": 48, "r_v": 96, "B": 16, "n": 26, "ragged": True, "T": 2000, "rot": 64, "inter": True, "draft": True},
        # a prefill batch of prompts of unequal lengths into the bf16 cache
        {"name": "append-prompts", "op": "append", "f8": False, "Hq": 32, "Hkv": 8, "r_k": 64, "r_v": 64, "B": 8, "n": 4096, "ragged": True, "T": 0, "rot": 128, "inter": False, "draft": False},
        # a decode batch into the 8-bit cache: every token joins a page that has rows already
        {"name": "f8-append-step", "op": "append", "f8": True, "Hq": 32, "Hkv": 8, "r_k": 64, "r_v": 64, "B": 64, "n": 1, "ragged": False, "T": 100, "rot": 128, "inter": False, "draft": False},
        # the same prefill batch into the 8-bit cache, ranks of a layer that is hard to compress
        {"name": "f8-append-prompts", "op": "append", "f8": True, "Hq": 32, "Hkv": 8, "r_k": 96, "r_v": 128, "B": 8, "n": 4096, "ragged": True, "T": 70, "rot": 128, "inter": False, "draft": False},
        # one sequence, a short context: the attention call of an interactive user
        {"name": "f8-decode-short", "op": "decode", "B": 1, "Hq": 32, "Hkv": 8, "r_k": 48, "r_v": 64, "T": 1021, "ragged": False},
        # the long-context decode shape (4 sequences of 32768 tokens)
        {"name": "f8-decode-long", "op": "decode", "B": 4, "Hq": 32, "Hkv": 8, "r_k": 64, "r_v": 64, "T": 32768, "ragged": False},
        # a serving batch of unequal lengths (1024 .. 16384), high ranks
        {"name": "f8-decode-ragged", "op": "decode", "B": 16, "Hq": 32, "Hkv": 8, "r_k": 96, "r_v": 128, "T": 16384, "ragged": True},
        # every query head with its own KV head
        {"name": "f8-decode-heads", "op": "decode", "B": 2, "Hq": 16, "Hkv": 16, "r_k": 128, "r_v": 128, "T": 8191, "ragged": False},
        # eight tokens of every sequence verified against a long cache
        {"name": "f8-verify", "op": "run", "B": 4, "Hq": 32, "Hkv": 8, "r_k": 64, "r_v": 64, "T": 32768, "n": 8, "ragged": False},
        # chunks of unequal lengths of a few prompts
        {"name": "f8-chunk-ragged", "op": "run", "B": 5, "Hq": 32, "Hkv": 8, "r_k": 96, "r_v": 128, "T": 4000, "n": 300, "ragged": True},
        # one chunk of a long prompt
        {"name": "f8-chunk", "op": "run", "B": 1, "Hq": 32, "Hkv": 8, "r_k": 64, "r_v": 64, "T": 16384, "n": 2048, "ragged": False},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "decode", "run"])
    ranks = [32, 48, 64, 96, 128]
    case = {"op": op, "r_k": rng.choice(ranks), "r_v": rng.choice(ranks), "ragged": rng.random() < 0.5}
    case["Hq"], case["Hkv"] = rng.choice([(32, 8), (32, 8), (8, 8), (16, 4), (16, 2), (10, 2), (6, 6)])
    if op == "append":
        B = _log_int(rng, 1, 64)
        return {**case, "f8": rng.random() < 0.6, "B": B, "n": _log_int(rng, 1, max(1, 12000 // B)), "T": rng.choice([0, _log_int(rng, 1, 400)]),
                "rot": rng.choice([128, 128, 64, 32, 96]), "inter": rng.random() < 0.3, "draft": rng.random() < 0.2}
    B = _log_int(rng, 1, 16)
    T = _log_int(rng, 1, 131072 // B if op == "decode" else 32768 // B)
    if op == "decode":
        return {**case, "B": B, "T": min(T, 32768)}
    return {**case, "B": B, "T": T, "n": min(T, _log_int(rng, 1, max(1, 1024 // B)))}


# ------------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    c = torch.Generator()
    c.manual_seed(seed)
    return g, c


def _sizes(case, least, most):
    """A length for each sequence, ``most`` where the case is not ragged: part of the case, the same for every seed."""
    c = torch.Generator()
    c.manual_seed(least + 31 * most + 1009 * case["B"])
    got = torch.full((case["B"],), most)
    if case["ragged"]:
        got[1:] = torch.randint(least, most + 1, (case["B"] - 1,), generator=c)
    return got


def _bf16(g, *shape, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(torch.bfloat16)


def _basis(g, Hkv, r):
    q, rr = torch.linalg.qr(torch.randn(Hkv, D, D, generator=g, device="cuda", dtype=torch.float64))
    q = q * torch.sign(torch.diagonal(rr, dim1=1, dim2=2))[:, None, :]
    return q[:, :, :r].to(torch.bfloat16).contiguous()


def _tables(c, pages, spare):
    """Block table with every sequence's pages taken from a shuffled pool."""
    width, total = max(pages), sum(pages)
    order = torch.randperm(total + spare, generator=c)
    table = torch.zeros(len(pages), width, dtype=torch.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n].to(torch.int32)
        at += n
    return table, total + spare


def _blocks(g, c, num_pages, Hkv, r_k, r_v):
    """Pages of the 8-bit cache as earlier tokens left them: codes whose largest lies in the top binade, scales around 2^-6."""
    codes = [(torch.randn(num_pages, Hkv, PAGE, r, generator=g, device="cuda") * 75.0).clamp_(-TOP, TOP).to(F8).view(torch.uint8) for r in (r_k, r_v)]
    scales = torch.zeros(num_pages, Hkv, 4, device="cuda")
    scales[:, :, :2] = torch.exp2(torch.randint(-7, -4, (num_pages, Hkv, 2), generator=c).float()).cuda()
    return codes[0], codes[1], scales


def _rotation_table(max_pos, rot):
    angle = torch.arange(max_pos, device="cuda", dtype=torch.float64)[:, None] * 500000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _append_case(case, seed):
    g, c = _gen(seed)
    B, n, T, Hq, Hkv, rk, rv = (case[x] for x in ("B", "n", "T", "Hq", "Hkv", "r_k", "r_v"))
    counts, lens = _sizes(case, max(1, n // 16), n), _sizes(case, 0, T)
    table, num_pages = _tables(c, [(int(x) + int(y) + PAGE - 1) // PAGE for x, y in zip(lens, counts)], 2)
    cu = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)])
    total = int(cu[-1])
    # queries, keys and values side by side, as the layer's one projection leaves them; keys with a spread over channels
    qkv = _bf16(g, total, Hq + 2 * Hkv, D)
    qkv[:, Hq:Hq + Hkv] *= torch.exp2(torch.linspace(2, -2, D, device="cuda")).to(torch.bfloat16)
    s = {"op": "append", "f8": case["f8"], "Hq": Hq, "Hkv": Hkv, "r_k": rk, "r_v": rv, "rot": case["rot"], "inter": case["inter"],
         "q": qkv[:, :Hq], "k": qkv[:, Hq:Hq + Hkv], "v": qkv[:, Hq + Hkv:], "cu": cu.to(torch.int32).cuda(), "lens": lens.to(torch.int32).cuda(),
         "table": table.cuda(), "U_k": _basis(g, Hkv, rk), "U_v": _basis(g, Hkv, rv), "positions": None,
         "rotation": _rotation_table(T + n + 1, case["rot"]), "q_out": torch.zeros(total, Hq, D, dtype=torch.bfloat16, device="cuda")}
    if case["draft"]:                                        # a node's position is its depth behind the context, not its place in the cache
        depth = torch.cat([(torch.rand(int(x), generator=c) * torch.arange(int(x)).sqrt()).long() for x in counts])
        s["positions"] = (lens.repeat_interleave(counts) + depth).to(torch.int32).cuda()
    if case["f8"]:
        s["k_codes"], s["v_codes"], s["scales"] = _blocks(g, c, num_pages, Hkv, rk, rv)
    else:
        s["k_pool"], s["v_pool"] = _bf16(g, num_pages, Hkv, PAGE, rk), _bf16(g, num_pages, Hkv, PAGE, rv)
    return s


def _attend_case(case, seed):
    g, c = _gen(seed)
    B, T, Hq, Hkv, rk, rv = (case[x] for x in ("B", "T", "Hq", "Hkv", "r_k", "r_v"))
    n = case["n"] if case["op"] == "run" else 1
    lens = _sizes(case, max(1, T // 16), T)
    counts = torch.minimum(_sizes(case, 1, n), lens)
    table, num_pages = _tables(c, [(int(x) + PAGE - 1) // PAGE for x in lens], 3)
    k, v, scales = _blocks(g, c, num_pages, Hkv, rk, rv)
    return {"op": case["op"], "Hq": Hq, "Hkv": Hkv, "r_k": rk, "r_v": rv, "n": n, "U_k": _basis(g, Hkv, rk), "U_v": _basis(g, Hkv, rv),
            "k_codes": k, "v_codes": v, "scales": scales, "table": table.cuda(), "lens": lens.to(torch.int32).cuda(),
            "counts": counts.to(torch.int32).cuda(), "q": _bf16(g, B, n, Hq, D, scale=2.0)}


def prepare(case, seed):
    s = (_append_case if case["op"] == "append" else _attend_case)(case, seed)
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program that uses this package keeps beside its tensors: descriptors, workspace, output buffers."""
    import paper_2601_21686_b200 as st
    shape = (s["Hq"], s["Hkv"], s["r_k"], s["r_v"], s["U_k"], s["U_v"])
    s["layer"] = st.F8Layer(*shape, s["k_codes"], s["v_codes"], s["scales"]) if "k_codes" in s else st.Layer(*shape, s["k_pool"], s["v_pool"])
    s["batch"] = st.Batch(s["table"], s["lens"])
    if s["op"] == "append":
        s["turn"] = st.Rotation(s["rotation"], interleaved=s["inter"])
        return
    B, n, Hq, _ = s["q"].shape
    s["out"] = torch.zeros_like(s["q"])
    if s["op"] == "decode":
        s["workspace"] = torch.zeros(st.stief_decode_workspace_bytes(B, Hq, s["Hkv"], s["r_v"]), dtype=torch.uint8, device="cuda")
        st.stief_decode_workspace_init(s["workspace"])
        s["q_row"], s["out_row"] = s["q"][:, 0], s["out"][:, 0]
    else:
        s["splits"] = st.stief_f8_mq_num_splits(B, n, Hq, s["Hkv"], s["table"].shape[1])
        s["workspace"] = torch.zeros(max(128, st.stief_f8_mq_workspace_bytes(B, n, Hq, s["r_v"], s["splits"])), dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------------------------------------- one pass
def run(state):
    if own:
        return _run_own(state)
    return _plain_append(state) if state["op"] == "append" else _plain_attend(state)


def _run_own(s):
    import paper_2601_21686_b200 as st
    if s["op"] == "append":
        call = st.stief_f8_append if s["f8"] else st.stief_rope_append
        call(s["layer"], s["batch"], s["k"], s["v"], s["cu"], rotation=s["turn"], q=s["q"], q_out=s["q_out"], positions=s["positions"])
        return _appended(s)
    if s["op"] == "decode":
        st.stief_f8_decode_attention(s["layer"], s["batch"], s["q_row"], s["workspace"], s["out_row"])
    else:
        st.stief_f8_mq_attention(s["layer"], s["batch"], s["q"], s["out"], q_lens=s["counts"], workspace=s["workspace"], num_splits=s["splits"])
    return s["out"]


def _appended(s):
    if s["f8"]:
        return {"q": s["q_out"], "k_codes": s["k_codes"].view(F8), "v_codes": s["v_codes"].view(F8), "scales": s["scales"]}
    return {"q": s["q_out"], "k": s["k_pool"], "v": s["v_pool"]}


def _turned(x, at, s):
    """Rows [tokens, heads, 128] turned by the angles of their positions, in the type of the table."""
    half = s["rot"] // 2
    x, (cos, sin) = x.to(s["rotation"].dtype), s["rotation"][at][:, None, :].split(half, -1)
    y = x.clone()
    if s["inter"]:
        a, b = x[..., 0:s["rot"]:2], x[..., 1:s["rot"]:2]
        y[..., 0:s["rot"]:2], y[..., 1:s["rot"]:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :half], x[..., half:s["rot"]]
        y[..., :half], y[..., half:s["rot"]] = a * cos - b * sin, b * cos + a * sin
    return y


def _plain_append(s):
    cu, lens = s["cu"].long(), s["lens"].long()
    tok = torch.arange(s["q"].shape[0], device="cuda")
    b = torch.searchsorted(cu[1:], tok, right=True)
    place = lens[b] + tok - cu[b]
    at = place if s["positions"] is None else s["positions"].long()
    s["q_out"].copy_(_turned(s["q"], at, s))
    k = torch.einsum("thd,hdr->thr", _turned(s["k"], at, s), s["U_k"].float())
    v = torch.einsum("thd,hdr->thr", s["v"].float(), s["U_v"].float())
    page, slot = s["table"].long()[b, place // PAGE], place % PAGE
    if not s["f8"]:
        s["k_pool"][page, :, slot] = k.to(torch.bfloat16)
        s["v_pool"][page, :, slot] = v.to(torch.bfloat16)
        return _appended(s)
    held = lens % PAGE                                                   # rows that the page of each sequence's first token holds already
    n_new = cu[1:] - cu[:-1]
    first = torch.gather(s["table"].long(), 1, (lens // PAGE).clamp(max=s["table"].shape[1] - 1)[:, None])[:, 0]
    joins = (held > 0) & (n_new > 0)
    _plain_store(s["k_codes"], s["scales"][:, :, 0], k, page, slot, first, held, joins)
    _plain_store(s["v_codes"], s["scales"][:, :, 1], v, page, slot, first, held, joins)
    return _appended(s)


def _plain_store(codes, scale, rows, page, slot, first, held, joins):
    P, Hkv = scale.shape
    top = torch.zeros(P, Hkv, device="cuda").index_reduce_(0, page, rows.abs().amax(-1), "amax", include_self=True)
    mantissa, exponent = torch.frexp(top)                                # top = mantissa 2^exponent, 1/2 <= mantissa < 1
    exponent = (exponent - 9 + (mantissa > 0.875).int()).clamp(LOWEST, HIGHEST)
    need = torch.where(top > 0, torch.ldexp(torch.ones_like(top), exponent), 2.0 ** LOWEST)
    old = torch.zeros(P, Hkv, device="cuda")
    old[first] = torch.where(joins[:, None], scale[first], 0.0)
    new = torch.maximum(old, need)
    touched = torch.zeros(P, dtype=torch.bool, device="cuda").index_fill_(0, page, True)
    # rows that the page holds already, under its new scale
    keep = (torch.arange(PAGE, device="cuda")[None] < held[:, None]) & joins[:, None]
    was = codes[first].view(F8).float()
    again = (was * (old[first] / new[first])[:, :, None, None]).to(F8)
    codes[first] = torch.where(keep[:, None, :, None], again.view(torch.uint8), codes[first])
    codes[page, :, slot] = (rows / new[page][:, :, None]).to(F8).view(torch.uint8)
    scale.copy_(torch.where(touched[:, None], new, scale))


def _plain_attend(s):
    B, n, Hq, _ = s["q"].shape
    Hkv, G = s["Hkv"], Hq // s["Hkv"]
    ids = s["table"].long()
    k = (s["k_codes"].view(F8)[ids].float() * s["scales"][ids][..., 0, None, None]).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, s["r_k"])
    v = (s["v_codes"].view(F8)[ids].float() * s["scales"][ids][..., 1, None, None]).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, s["r_v"])
    q = s["q"].float().view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    w = torch.matmul(torch.matmul(q, s["U_k"].float()), k.transpose(2, 3)).mul_(SCALE)
    i = torch.arange(n, device="cuda").repeat_interleave(G)
    seen = torch.arange(k.shape[2], device="cuda")[None, None] <= (s["lens"] - s["counts"])[:, None, None] + i[None, :, None]
    w.masked_fill_(~(seen & (i[None] < s["counts"][:, None])[:, :, None])[:, None], -math.inf)
    w.sub_(w.amax(-1, keepdim=True).clamp_(min=-3e38)).exp_()
    o = torch.matmul(w, v) / w.sum(-1, keepdim=True).clamp(min=1e-37)
    o = torch.matmul(o, s["U_v"].float().transpose(1, 2))
    return o.view(B, Hkv, n, G, D).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    B, Hq, Hkv, rk, rv = (case[x] for x in ("B", "Hq", "Hkv", "r_k", "r_v"))
    half = lambda x: x + (B - 1) * (x // 16 + x) / 2 if case["ragged"] else B * x  # noqa: E731  (one of full size, the others half of it in the mean)
    if case["op"] == "append":
        tokens = half(case["n"])
        row = (rk + rv) * (1 if case["f8"] else 2)
        return {"bytes": tokens * (2 * D * (2 * Hq + 2 * Hkv) + Hkv * row + 4 * case["rot"]) + 2 * Hkv * D * (rk + rv), "flops": tokens * Hkv * D * 2 * (rk + rv)}
    n = case["n"] if case["op"] == "run" else 1
    cached, rows = half(case["T"]), half(n) if case["op"] == "run" else B
    pairs = cached * rows / B - B * n * (n - 1) / 2 if not case["ragged"] else cached * rows / B
    return {"bytes": Hkv * cached * (rk + rv) + 4 * rows * Hq * D, "flops": 2 * Hq * max(pairs, rows) * (rk + rv) + 2 * Hq * rows * D * (rk + rv)}


# ------------------------------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    if case["op"] == "append":
        return _exact_append(_append_case(case, seed))
    return _exact_attend(_attend_case(case, seed))


def _to_e4m3(x):
    """Doubles rounded to the nearest e4m3 value, ties to even."""
    step = torch.ldexp(torch.ones_like(x), torch.frexp(x)[1].clamp(min=-5) - 4)
    return torch.round(x / step) * step


def _exact_append(s):
    cu, lens, table = s["cu"].tolist(), s["lens"].tolist(), s["table"].tolist()
    half, rot = s["rot"] // 2, s["rot"]
    place = torch.cat([torch.arange(n, n + hi - lo) for n, lo, hi in zip(lens, cu[:-1], cu[1:])])
    angles = s["rotation"].double()[place.cuda() if s["positions"] is None else s["positions"].long()]
    turn = torch.complex(angles[:, :half], angles[:, half:])[:, None]

    def rotated(x):
        x = x.double()
        a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if s["inter"] else (x[..., :half], x[..., half:rot])
        z = torch.complex(a, b) * turn
        y = torch.stack([z.real, z.imag], -1).flatten(-2) if s["inter"] else torch.cat([z.real, z.imag], -1)
        return torch.cat([y, x[..., rot:]], -1)

    sides = [(rotated(s["k"]), s["U_k"]), (s["v"].double(), s["U_v"])]
    sides = [torch.stack([x[:, h] @ U[h].double() for h in range(s["Hkv"])], 1) for x, U in sides]
    if s["f8"]:
        pools, scales = [s["k_codes"].view(F8).double(), s["v_codes"].view(F8).double()], s["scales"].double()
    else:
        pools = [s["k_pool"].double(), s["v_pool"].double()]
    for b, n in enumerate(lens):
        at = n
        while at < n + cu[b + 1] - cu[b]:
            page, slot = table[b][at // PAGE], at % PAGE
            m = min(PAGE - slot, n + cu[b + 1] - cu[b] - at)
            lo = cu[b] + at - n
            for i in range(2):
                rows = sides[i][lo:lo + m].transpose(0, 1)                                # [heads, tokens, rank]
                if not s["f8"]:
                    pools[i][page, :, slot:slot + m] = rows
                    continue
                most = rows.abs().flatten(1).amax(1)
                scale = torch.exp2(torch.ceil(torch.log2(most / TOP)).clamp(LOWEST, HIGHEST))
                if slot:
                    scale = torch.maximum(scale, scales[page, :, i])
                    pools[i][page, :, :slot] = _to_e4m3(pools[i][page, :, :slot] * (scales[page, :, i] / scale)[:, None, None])
                pools[i][page, :, slot:slot + m] = _to_e4m3(rows / scale[:, None, None])
                scales[page, :, i] = scale
            at += m
    q = rotated(s["q"])
    return {"q": q, "k_codes": pools[0], "v_codes": pools[1], "scales": scales} if s["f8"] else {"q": q, "k": pools[0], "v": pools[1]}


def _exact_attend(s):
    B, n, Hq, _ = s["q"].shape
    G = Hq // s["Hkv"]
    out = torch.zeros(B, n, Hq, D, dtype=torch.float64, device="cuda")
    for b in range(B):
        m, t = int(s["counts"][b]), int(s["lens"][b])
        ids = s["table"][b, : (t + PAGE - 1) // PAGE].long()
        future = torch.ones(m, t, dtype=torch.bool, device="cuda").triu(t - m + 1)
        for h in range(s["Hkv"]):
            K = (s["k_codes"][ids, h].view(F8).double() * s["scales"][ids, h, 0].double()[:, None, None]).flatten(0, 1)[:t] @ s["U_k"][h].double().T
            V = (s["v_codes"][ids, h].view(F8).double() * s["scales"][ids, h, 1].double()[:, None, None]).flatten(0, 1)[:t] @ s["U_v"][h].double().T
            for g in range(h * G, h * G + G):
                w = (s["q"][b, :m, g].double() @ K.T / math.sqrt(D)).masked_fill_(future, -math.inf)
                out[b, :m, g] = torch.softmax(w, -1) @ V
    return out
