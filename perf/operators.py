"""Workloads of the attention and cache operators beside the decode path, each with a plain torch form of the same
computation: attention of a tree of drafted tokens over the compressed cache, causal attention over packed prompts, and
the page operations of the cache (forking and reordering sequences, accepting drafted rows).

``own = False`` computes the operators with elementary torch operations in fp32; ``own = True`` calls this package."""
import math

import torch

own = False

PAGE, D = 64, 128
SCALE = 1.0 / math.sqrt(D)


# ------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one sequence, a short context and a small tree: the call whose latency an interactive user sees
        {"name": "tree-short", "op": "tree", "B": 1, "Hq": 32, "Hkv": 8, "r_k": 48, "r_v": 64, "T": 1021, "ragged": False, "nodes": 8, "fold": False},
        # the long-context decode shape (4 sequences of 32768 tokens) with a narrow and a wide tree
        {"name": "tree-long-16", "op": "tree", "B": 4, "Hq": 32, "Hkv": 8, "r_k": 64, "r_v": 64, "T": 32768, "ragged": False, "nodes": 16, "fold": False},
        {"name": "tree-long-64", "op": "tree", "B": 4, "Hq": 32, "Hkv": 8, "r_k": 64, "r_v": 64, "T": 32768, "ragged": False, "nodes": 64, "fold": False},
        # a serving batch of unequal lengths (1024 .. 16384) and unequal trees
        {"name": "tree-ragged", "op": "tree", "B": 16, "Hq": 32, "Hkv": 8, "r_k": 64, "r_v": 64, "T": 16384, "ragged": True, "nodes": 26, "fold": False},
        # a layer of high ranks
        {"name": "tree-wide-rank", "op": "tree", "B": 2, "Hq": 32, "Hkv": 8, "r_k": 96, "r_v": 128, "T": 16384, "ragged": False, "nodes": 31, "fold": False},
        # a handful of very short prompts, one token among them
        {"name": "prompt-short", "op": "prompt", "Hq": 32, "Hkv": 8, "lens": "1,17,130,64,5"},
        # a mixed prefill batch: prompts of very different lengths behind one another
        {"name": "prompt-ragged", "op": "prompt", "Hq": 32, "Hkv": 8, "lens": "2741,3,1280,977,512,1,1901,601"},
        # every query head with its own key head
        {"name": "prompt-heads", "op": "prompt", "Hq": 16, "Hkv": 16, "lens": "2048,2048"},
        # one long prompt
        {"name": "prompt-long", "op": "prompt", "Hq": 32, "Hkv": 8, "lens": "16384"},
        # one beam search of 4 over a few layers
        {"name": "fork-few", "op": "fork", "groups": 1, "beams": 4, "layers": 4, "Hkv": 8, "r": 64, "T": 700},
        # beam searches of 8 for 8 requests over all layers of a model
        {"name": "fork-many", "op": "fork", "groups": 8, "beams": 8, "layers": 32, "Hkv": 8, "r": 64, "T": 1000},
        # the accepted path of every drafted tree, all layers
        {"name": "accept", "op": "accept", "B": 16, "nodes": 26, "path": 8, "layers": 32, "Hkv": 8, "r": 64, "T": 2000},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tree", "tree", "prompt", "prompt", "fork", "accept"])
    ranks = [32, 48, 64, 96, 128]
    if op == "tree":
        Hq, Hkv = rng.choice([(32, 8), (32, 8), (8, 8), (16, 4), (16, 2), (10, 2)])
        nodes = _log_int(rng, 1, 64)
        B = _log_int(rng, 1, 16)
        T = _log_int(rng, 1, min(32768, 131072 // B))
        return {"op": op, "B": B, "Hq": Hq, "Hkv": Hkv, "r_k": rng.choice(ranks), "r_v": rng.choice(ranks), "T": T,
                "ragged": rng.random() < 0.5, "nodes": nodes, "fold": rng.random() < 0.2}
    if op == "prompt":
        Hq, Hkv = rng.choice([(32, 8), (32, 8), (8, 8), (16, 4), (16, 2), (14, 2), (6, 6)])
        B, total = _log_int(rng, 1, 16), _log_int(rng, 16, 8000)
        lens = [max(1, int(total / B * rng.uniform(0.2, 1.6))) for _ in range(B)]
        return {"op": op, "Hq": Hq, "Hkv": Hkv, "lens": ",".join(map(str, lens))}
    if op == "fork":
        return {"op": op, "groups": _log_int(rng, 1, 8), "beams": _log_int(rng, 2, 8), "layers": _log_int(rng, 1, 32), "Hkv": rng.choice([2, 4, 8]),
                "r": rng.choice(ranks[:3]), "T": _log_int(rng, 1, 1000)}
    return {"op": op, "B": _log_int(rng, 1, 16), "nodes": _log_int(rng, 2, 64), "path": _log_int(rng, 1, 12), "layers": _log_int(rng, 1, 32),
            "Hkv": rng.choice([2, 4, 8]), "r": rng.choice(ranks[:3]), "T": _log_int(rng, 1, 2000)}


# ------------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    c = torch.Generator()
    c.manual_seed(seed)
    return g, c


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


def _tree_case(case, seed):
    g, c = _gen(seed)
    B, n = case["B"], case["nodes"]
    T = case["T"]
    if case["ragged"]:
        lens = torch.randint(max(0, T // 16), T + 1, (B,), generator=c)
        counts = torch.randint(1, n + 1, (B,), generator=c)
        lens[0], counts[0] = T, n
    else:
        lens, counts = torch.full((B,), T), torch.full((B,), n)
    words = (n + 31) // 32
    mask = torch.zeros(B, n, words, dtype=torch.int64)
    for b in range(B):                                   # a random tree: every node sees its ancestors and itself
        anc = [0] * n
        up = torch.rand(n, generator=c).tolist()
        for i in range(n):
            anc[i] = (anc[int(up[i] * i)] if i else 0) | (1 << i)
            for w in range(words):
                mask[b, i, w] = (anc[i] >> (32 * w)) & 0xFFFFFFFF
    mask = torch.where(mask >= 2 ** 31, mask - 2 ** 32, mask).to(torch.int32)
    pages = [(int(lens[b]) + int(counts[b]) + PAGE - 1) // PAGE for b in range(B)]
    table, num_pages = _tables(c, pages, 3)
    Hq, Hkv, rk, rv = case["Hq"], case["Hkv"], case["r_k"], case["r_v"]
    fold = case["fold"]
    return {
        "op": "tree", "Hq": Hq, "Hkv": Hkv, "r_k": rk, "r_v": rv, "nodes": n,
        "U_k": None if fold else _basis(g, Hkv, rk), "U_v": None if fold else _basis(g, Hkv, rv),
        "k_pool": _bf16(g, num_pages, Hkv, PAGE, rk), "v_pool": _bf16(g, num_pages, Hkv, PAGE, rv),
        "table": table.cuda(), "lens": lens.to(torch.int32).cuda(), "counts": counts.to(torch.int32).cuda(), "mask": mask.cuda(),
        "q": _bf16(g, B, n, Hq, rk if fold else D, scale=2.0),
    }


def _prompt_case(case, seed):
    g, _ = _gen(seed)
    lens = [int(x) for x in case["lens"].split(",")]
    Hq, Hkv, total = case["Hq"], case["Hkv"], sum(lens)
    cu = [0]
    for x in lens:
        cu.append(cu[-1] + x)
    # queries, keys and values side by side, as the layer's one projection leaves them
    qkv = _bf16(g, total, Hq + 2 * Hkv, D)
    qkv[:, :Hq] *= 2.0
    return {"op": "prompt", "Hq": Hq, "Hkv": Hkv, "q": qkv[:, :Hq], "k": qkv[:, Hq:Hq + Hkv], "v": qkv[:, Hq + Hkv:],
            "cu": torch.tensor(cu, dtype=torch.int32, device="cuda"), "max_len": max(lens), "B": len(lens)}


def _fork_case(case, seed):
    g, c = _gen(seed)
    G, W, T, L = case["groups"], case["beams"], case["T"], case["layers"]
    S = G * W
    full, part = T // PAGE, T % PAGE
    width = full + 2
    num_pages = G * full + 2 * S + 5
    order = torch.randperm(num_pages, generator=c)
    table = torch.zeros(S, width, dtype=torch.int32)
    refs = torch.zeros(num_pages, dtype=torch.int32)
    at = G * full
    for s in range(S):                                   # a group's beams share the full pages; each has its own last page
        mine = order[(s // W) * full:(s // W) * full + full].tolist()
        if part:
            mine.append(int(order[at]))
            at += 1
        table[s, :len(mine)] = torch.tensor(mine, dtype=torch.int32)
        for p in mine:
            refs[p] += 1
    parent = torch.tensor([(s // W) * W + int(torch.randint(0, W, (1,), generator=c)) for s in range(S)], dtype=torch.int32)
    return {"op": "fork", "Hkv": case["Hkv"], "r": case["r"], "layers": L, "pools": _bf16(g, 2 * L, num_pages, case["Hkv"], PAGE, case["r"]), "table": table.cuda(),
            "lens": torch.full((S,), T, dtype=torch.int32).cuda(), "counts": torch.full((S,), full + (part > 0), dtype=torch.int32).cuda(),
            "refs": refs.cuda(), "parent": parent.cuda()}


def _accept_case(case, seed):
    g, c = _gen(seed)
    B, n, T, path = case["B"], case["nodes"], case["T"], min(case["path"], case["nodes"])
    lens = torch.randint(0, T + 1, (B,), generator=c)
    pages = [(int(x) + n + PAGE - 1) // PAGE for x in lens]
    table, num_pages = _tables(c, pages, B * ((T + n + PAGE - 1) // PAGE) + 3 - sum(pages))
    nodes = torch.stack([torch.sort(torch.randperm(n, generator=c)[:path]).values for _ in range(B)]).to(torch.int32)
    count = torch.randint(0, path + 1, (B,), generator=c).to(torch.int32)
    count[0] = path
    L = case["layers"]
    return {"op": "accept", "Hkv": case["Hkv"], "r": case["r"], "layers": L, "pools": _bf16(g, 2 * L, num_pages, case["Hkv"], PAGE, case["r"]), "table": table.cuda(),
            "lens": lens.to(torch.int32).cuda(), "accepted": nodes.cuda(), "count": count.cuda()}


def prepare(case, seed):
    s = {"tree": _tree_case, "prompt": _prompt_case, "fork": _fork_case, "accept": _accept_case}[case["op"]](case, seed)
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program that uses this package keeps beside its tensors: descriptors, workspace, output buffers."""
    import paper_2601_21686_b200 as st
    if s["op"] == "tree":
        s["layer"] = st.Layer(s["Hq"], s["Hkv"], s["r_k"], s["r_v"], s["U_k"], s["U_v"], s["k_pool"], s["v_pool"])
        s["batch"] = st.Batch(s["table"], s["lens"])
        B = s["q"].shape[0]
        s["workspace"] = torch.zeros(st.stief_tree_workspace_bytes(B, s["nodes"], s["Hq"], s["Hkv"], s["r_v"]), dtype=torch.uint8, device="cuda")
        s["out"] = torch.zeros(B, s["nodes"], s["Hq"], D if s["U_v"] is not None else s["r_v"], dtype=torch.bfloat16, device="cuda")
    elif s["op"] == "prompt":
        s["out"] = torch.empty(s["q"].shape[0], s["Hq"], D, dtype=torch.bfloat16, device="cuda")
    else:
        L, r = s["layers"], s["r"]
        s["stack"] = [st.Layer(s["Hkv"], s["Hkv"], r, r, None, None, s["pools"][2 * i], s["pools"][2 * i + 1]) for i in range(L)]
        if s["op"] == "fork":
            s["pages"] = st.PageTable(s["table"], s["lens"], s["counts"], s["refs"])
            s["workspace"] = torch.zeros(st.stief_pages_workspace_bytes(*s["table"].shape), dtype=torch.uint8, device="cuda")
        else:
            s["batch"] = st.Batch(s["table"], s["lens"])


# ------------------------------------------------------------------------------------------------- one pass
def run(state):
    if own:
        return _run_own(state)
    return {"tree": _plain_tree, "prompt": _plain_prompt, "fork": _plain_fork, "accept": _plain_accept}[state["op"]](state)


def _run_own(s):
    import paper_2601_21686_b200 as st
    if s["op"] == "tree":
        st.stief_tree_attention(s["layer"], s["batch"], s["q"], s["mask"], s["workspace"], s["out"], n_nodes=s["counts"])
        return s["out"]
    if s["op"] == "prompt":
        st.stief_prompt_attention(s["q"], s["k"], s["v"], s["cu"], s["out"])
        return s["out"]
    if s["op"] == "fork":
        st.stief_pages_fork(s["pages"], s["stack"], s["parent"], s["workspace"])
        return {"pools": s["pools"], "table": s["table"], "lens": s["lens"], "counts": s["counts"], "refs": s["refs"]}
    st.stief_tree_accept(s["stack"], s["batch"], s["accepted"], s["count"])
    return s["pools"]


def _attend(scores, keep, v):
    """softmax(scores) v over the last axis with masked places left out; rows with nothing kept give zeros."""
    scores.masked_fill_(~keep, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp_(min=-3e38)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / total.clamp(min=1e-37)


def _plain_tree(s):
    B, n, Hq, dq = s["q"].shape
    Hkv, G = s["Hkv"], Hq // s["Hkv"]
    pos = torch.arange(s["table"].shape[1] * PAGE, device="cuda")
    ids = s["table"].long()
    k = s["k_pool"][ids].float().permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, s["r_k"])
    v = s["v_pool"][ids].float().permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, s["r_v"])
    live = pos[None] < (s["lens"] + s["counts"])[:, None]
    v = torch.where(live[:, None, :, None], v, 0.0)
    q = s["q"].float().view(B, n, Hkv, G, dq).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, dq)
    if s["U_k"] is not None:
        q = torch.matmul(q, s["U_k"].float())
    j = pos[None] - s["lens"][:, None]                                  # index among the drafted nodes
    inside = (j >= 0) & (j < s["counts"][:, None])
    jc = j.clamp(0, n - 1)
    word = torch.gather(s["mask"].long(), 2, (jc // 32)[:, None, :].expand(B, n, -1))
    seen = (((word >> (jc % 32)[:, None, :]) & 1) == 1) & inside[:, None, :]
    keep = (seen | (j < 0)[:, None, :])[:, None, :, None, :].expand(B, 1, n, G, -1).reshape(B, 1, n * G, -1)
    o = _attend(torch.matmul(q, k.transpose(2, 3)).mul_(SCALE), keep, v)
    if s["U_v"] is not None:
        o = torch.matmul(o, s["U_v"].float().transpose(1, 2))
    o = o.view(B, Hkv, n, G, -1).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, -1)
    real = torch.arange(n, device="cuda")[None] < s["counts"][:, None]
    return torch.where(real[:, :, None, None], o, 0.0).to(torch.bfloat16)          # rows behind the last node stay as they were


def _plain_prompt(s):
    B, n, Hq, Hkv = s["B"], s["max_len"], s["Hq"], s["Hkv"]
    start, end = s["cu"][:-1].long(), s["cu"][1:].long()
    at = start[:, None] + torch.arange(n, device="cuda")[None]
    live = at < end[:, None]
    at = torch.where(live, at, 0)
    q = s["q"][at].float().permute(0, 2, 1, 3).reshape(B, Hkv, Hq // Hkv, n, D)
    k = s["k"][at].float().permute(0, 2, 1, 3)[:, :, None]
    v = torch.where(live[:, :, None, None], s["v"][at].float(), 0.0).permute(0, 2, 1, 3)[:, :, None]
    i = torch.arange(n, device="cuda")
    keep = (i[None, :] <= i[:, None])[None] & live[:, None, :]
    o = _attend(torch.matmul(q, k.transpose(3, 4)).mul_(SCALE), keep[:, None, None], v)
    o = o.reshape(B, Hq, n, D).permute(0, 2, 1, 3).to(torch.bfloat16)
    rows = torch.arange(s["q"].shape[0], device="cuda")
    b = torch.searchsorted(end, rows, right=True)
    return o[b, rows - start[b]]


def _plain_fork(s):
    table, lens, counts, refs, parent, pools = s["table"], s["lens"], s["counts"], s["refs"], s["parent"].long(), s["pools"]
    S, width = table.shape
    slot = torch.arange(S, device="cuda")
    stays = parent[parent] == parent                                     # a parent that stays in place keeps its own pages,
    first = torch.full((S,), S, device="cuda").scatter_reduce_(0, parent, slot, "amin")
    heir = torch.where(stays, slot == parent, slot == first[parent])     # else its first child takes them over
    col = torch.arange(width, device="cuda")[None]
    new_lens, full = lens[parent], lens[parent] // PAGE
    part = new_lens % PAGE > 0
    own_page = ~heir & part
    new_counts = torch.where(heir, counts[parent], full + part.int())
    rows = table[parent]
    delta = torch.zeros_like(refs)
    delta.scatter_add_(0, table.long().reshape(-1), -(col < counts[:, None]).int().reshape(-1))
    shared = (col < new_counts[:, None]) & ~(own_page[:, None] & (col == full[:, None]))
    delta.scatter_add_(0, rows.long().reshape(-1), shared.int().reshape(-1))
    refs += delta
    free = torch.sort(refs > 0, stable=True).indices                     # the lowest free pages, in slot order
    got = free[torch.cumsum(own_page.int(), 0) - 1]
    src = torch.gather(rows, 1, full.long()[:, None])[:, 0].long()
    dst = torch.where(own_page, got, src)
    pools[:, dst] = pools[:, src]
    refs.scatter_add_(0, got.clamp(min=0), own_page.int())
    rows = torch.where(own_page[:, None] & (col == full[:, None]), got[:, None].int(), rows)
    table.copy_(torch.where(col < new_counts[:, None], rows, table))
    lens.copy_(new_lens)
    counts.copy_(new_counts)
    return {"pools": pools, "table": table, "lens": lens, "counts": counts, "refs": refs}


def _plain_accept(s):
    pools, table, lens = s["pools"], s["table"].long(), s["lens"].long()
    B, path = s["accepted"].shape
    j = torch.arange(path, device="cuda")[None].expand(B, path)
    real = (j < s["count"][:, None]).reshape(-1)
    to = lens[:, None] + j
    at = torch.where(real.view(B, path), lens[:, None] + s["accepted"].long(), to)
    last = table.shape[1] * PAGE - 1
    to, at = to.clamp(max=last), at.clamp(max=last)
    page_at, page_to = torch.gather(table, 1, at // PAGE).reshape(-1), torch.gather(table, 1, to // PAGE).reshape(-1)
    rows = pools[:, page_at, :, (at % PAGE).reshape(-1)]                 # all read before any is written
    old = pools[:, page_to, :, (to % PAGE).reshape(-1)]
    keep = real[:, None, None, None]
    pools[:, page_to, :, (to % PAGE).reshape(-1)] = torch.where(keep, rows, old)
    return pools


# ------------------------------------------------------------------------------------------------- what a pass cannot do without
def _tree_sizes(case):
    B, T, n = case["B"], case["T"], case["nodes"]
    if case["ragged"]:          # one sequence of full size, the others half of it in the mean
        return T + (B - 1) * (T // 16 + T) / 2, n + (B - 1) * (n + 1) / 2
    return B * T, B * n


def work(case):
    if case["op"] == "tree":
        ctx, nodes = _tree_sizes(case)
        Hq, Hkv, rk, rv = case["Hq"], case["Hkv"], case["r_k"], case["r_v"]
        dq, do = (rk, rv) if case["fold"] else (D, D)
        pairs = ctx * nodes / case["B"]
        flops = 2 * Hq * pairs * (rk + rv) + (0 if case["fold"] else 2 * Hq * nodes * D * (rk + rv))
        return {"bytes": 2 * Hkv * (ctx + nodes) * (rk + rv) + 2 * nodes * Hq * (dq + do), "flops": flops}
    if case["op"] == "prompt":
        lens = [int(x) for x in case["lens"].split(",")]
        total = sum(lens)
        return {"bytes": 2 * total * D * 2 * (case["Hq"] + case["Hkv"]), "flops": 4 * D * case["Hq"] * sum(x * (x + 1) // 2 for x in lens)}
    page = 2 * case["layers"] * case["Hkv"] * PAGE * case["r"] * 2
    if case["op"] == "fork":
        S = case["groups"] * case["beams"]
        copies = S - case["groups"] * case["beams"] * (1 - (1 - 1 / case["beams"]) ** case["beams"])    # slots whose parent already has an heir
        part = case["T"] % PAGE > 0
        return {"bytes": 2 * copies * page * part + 3 * 4 * S * (case["T"] // PAGE + 1), "flops": 0}
    row = page // PAGE
    path = min(case["path"], case["nodes"])
    return {"bytes": 2 * row * (path + (case["B"] - 1) * path / 2) + 4 * case["B"] * (path + 2), "flops": 0}


# ------------------------------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = {"tree": _tree_case, "prompt": _prompt_case, "fork": _fork_case, "accept": _accept_case}[case["op"]](case, seed)
    if s["op"] == "tree":
        return _exact_tree(s)
    if s["op"] == "prompt":
        return _exact_prompt(s)
    if s["op"] == "fork":
        return _exact_fork(s)
    return _exact_accept(s)


def _exact_tree(s):
    B, n, Hq, _ = s["q"].shape
    G = Hq // s["Hkv"]
    out = torch.zeros(B, n, Hq, D if s["U_v"] is not None else s["r_v"], dtype=torch.float64, device="cuda")
    for b in range(B):
        ctx, m = int(s["lens"][b]), int(s["counts"][b])
        ids = s["table"][b, : (ctx + m + PAGE - 1) // PAGE].long()
        bits = s["mask"][b].tolist()
        tree = torch.tensor([[(bits[i][j // 32] >> (j % 32)) & 1 for j in range(m)] for i in range(m)], dtype=torch.bool, device="cuda")
        for h in range(s["Hkv"]):
            K = s["k_pool"][ids, h].double().flatten(0, 1)[: ctx + m]
            V = s["v_pool"][ids, h].double().flatten(0, 1)[: ctx + m]
            if s["U_k"] is not None:
                K = K @ s["U_k"][h].double().T
            if s["U_v"] is not None:
                V = V @ s["U_v"][h].double().T
            for g in range(h * G, h * G + G):
                w = s["q"][b, :m, g].double() @ K.T / math.sqrt(D)
                w[:, ctx:] += torch.where(tree, 0.0, -math.inf)
                out[b, :m, g] = torch.softmax(w, -1) @ V
    return out


def _exact_prompt(s):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    cu, G = s["cu"].tolist(), s["Hq"] // s["Hkv"]
    for lo, hi in zip(cu[:-1], cu[1:]):
        past = torch.tril(torch.ones(hi - lo, hi - lo, dtype=torch.bool, device="cuda"))
        for g in range(s["Hq"]):
            w = s["q"][lo:hi, g].double() @ s["k"][lo:hi, g // G].double().T / math.sqrt(D)
            w.masked_fill_(~past, -math.inf)
            out[lo:hi, g] = torch.softmax(w, -1) @ s["v"][lo:hi, g // G].double()
    return out


def _exact_fork(s):
    table, lens, counts, refs, parent = (s[x].tolist() for x in ("table", "lens", "counts", "refs", "parent"))
    S = len(parent)
    heirs = {}
    for p in set(parent):
        heirs[p] = p if parent[p] == p else min(b for b in range(S) if parent[b] == p)
    rows, wants = [], []
    for b, p in enumerate(parent):
        if heirs[p] == b:
            rows.append(table[p][:counts[p]])
        else:
            rows.append(table[p][:lens[p] // PAGE])
            if lens[p] % PAGE:
                wants.append((b, table[p][lens[p] // PAGE]))
    refs = [0] * len(refs)
    for r in rows:
        for page in r:
            refs[page] += 1
    free = [p for p in range(len(refs)) if refs[p] == 0]
    pools = s["pools"].clone()
    for (b, src), dst in zip(wants, free):
        pools[:, dst] = s["pools"][:, src]
        rows[b].append(dst)
        refs[dst] = 1
    new = [r + table[b][len(r):] for b, r in enumerate(rows)]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"pools": pools, "table": ints(new), "lens": ints([lens[p] for p in parent]), "counts": ints([len(r) for r in rows]), "refs": ints(refs)}


def _exact_accept(s):
    pools = s["pools"].clone()
    for b, (lens, nodes, count) in enumerate(zip(s["lens"].tolist(), s["accepted"].tolist(), s["count"].tolist())):
        where = lambda t: (int(s["table"][b, t // PAGE]), t % PAGE)  # noqa: E731
        for j in range(count):
            (p0, t0), (p1, t1) = where(lens + nodes[j]), where(lens + j)
            pools[:, p1, :, t1] = s["pools"][:, p0, :, t0]
    return pools
