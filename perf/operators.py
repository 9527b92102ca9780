"""The step of several tokens over the paged cache, as cases that can be timed and checked.

A case is one pass through one of three operators: appending rotated keys and
values to the cache (with the queries rotated on the way), attention of a tree
of drafted tokens over the cache, and keeping the accepted path of such a tree.
With `own` set a pass makes the calls of paper_2607_06827_amd.speechkv that a
serving program makes; without it the same values are computed from elementary
torch operations.  Frames are 80 ms, so 375 are 30 s of audio, 750 are 60 s and
7500 are 10 minutes; a layer from the first compressed one on keeps one entry
per window of w frames.
"""
import math

import numpy as np
import torch

own = False


def _case(name, kind, **kw):
    c = dict(name=name, kind=kind, dtype="bf16", batch=1, q_heads=16, kv_heads=8, dim=128, page=16,
             # text before the speech, frames, window, text already generated
             prefix=32, frames=375, w=4, generated=40, ragged=False)
    c.update(dict(append=dict(new=1, rot=128, layout="halves", fused=True),
                  tree=dict(nodes=8, chain=False, shared=False),
                  commit=dict(nodes=8, path=4, layers=1))[kind])
    c.update(kw)
    return c


def listed():
    return [
        # one token of one user: the smallest call of a decoding loop
        _case("append_one_user", "append"),
        # the drafted tokens of 64 users with 60 s of audio, unequal trees,
        # out of one fused projection
        _case("append_drafts", "append", batch=64, new=16, frames=750, generated=64, ragged=True),
        # the prompt of 8 users with two minutes of audio, a layer that keeps
        # every frame: the keys are rotated on their way into the cache
        _case("append_prompt", "append", batch=8, new=1596, prefix=0, frames=0, generated=0),
        # fp32, a quarter rotation of neighbouring elements, odd lengths,
        # separate projections
        _case("append_f32_pairs", "append", dtype="f32", batch=6, q_heads=8, kv_heads=4, dim=64,
              new=33, rot=32, layout="pairs", fused=False, frames=201, w=3, ragged=True),
        # one user, 30 s of audio, a small tree of drafted tokens
        _case("tree_one_user", "tree"),
        # a serving step: 64 users with 60 s of audio, one compressed layer
        _case("tree_serving", "tree", batch=64, nodes=16, frames=750, generated=64, ragged=True),
        # 16 users with 10 minutes of audio each, a layer that keeps every frame
        _case("tree_10min", "tree", batch=16, nodes=32, frames=7500, w=1, generated=128),
        # one user with 10 minutes of audio: few rows, a long axis
        _case("tree_one_user_10min", "tree", nodes=64, frames=7500, w=1, generated=128),
        # a typed follow-up of 301 tokens over two minutes of audio, plain
        # causal order, eight query heads per KV head, bigger pages
        _case("tree_follow_up", "tree", batch=8, q_heads=64, nodes=301, chain=True, frames=1500,
              page=64, ragged=True),
        # fp32, odd sizes, one tree shape for every sequence
        _case("tree_f32", "tree", dtype="f32", batch=5, q_heads=16, kv_heads=4, dim=64, nodes=21,
              shared=True, frames=601, w=3, ragged=True),
        # the accepted tokens of one user in one layer
        _case("commit_one_layer", "commit"),
        # the accepted tokens of 64 users through all 28 layers
        _case("commit_stack", "commit", batch=64, nodes=16, path=6, layers=28, frames=750,
              generated=64, ragged=True),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        w, k = work(c), c["kind"]
        most[k] = tuple(max(x, y) for x, y in zip(most.get(k, (0, 0)), (w["bytes"], w["flops"])))
    while True:
        kind = rng.choice(["append", "append", "tree", "tree", "tree", "tree", "commit"])
        kv = rng.choice([1, 2, 4, 8])
        dim = rng.choice([64, 128, 128])
        c = _case("", kind, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), batch=_logint(rng, 1, 64),
                  kv_heads=kv, q_heads=kv * rng.choice([1, 2, 2, 4, 8]), dim=dim,
                  page=rng.choice([8, 16, 16, 32, 64, 128]), prefix=rng.randint(0, 64),
                  frames=rng.choice([0, _logint(rng, 1, 7500), _logint(rng, 30, 7500)]),
                  w=rng.choice([1, 1, 2, 3, 4, 4, 8]), generated=rng.randint(0, 256),
                  ragged=rng.random() < 0.5)
        del c["name"]
        if kind == "append":
            c.update(new=_logint(rng, 1, 2000), rot=16 * rng.randint(0, dim // 16),
                     layout=rng.choice(["halves", "halves", "pairs"]), fused=rng.random() < 0.6)
        elif kind == "tree":
            c.update(nodes=rng.choice([_logint(rng, 1, 64), _logint(rng, 1, 64), _logint(rng, 1, 500)]),
                     chain=rng.random() < 0.3, shared=rng.random() < 0.3)
        else:
            nodes = _logint(rng, 1, 64)
            c.update(nodes=nodes, path=rng.randint(1, min(nodes, 12)), layers=rng.choice([1, 4, 28]))
        w = work(c)
        slow = 16 if c["dtype"] == "f32" else 1  # fp32 products run on the fp32 matrix units
        if w["bytes"] <= most[kind][0] and w["flops"] * slow <= most[kind][1]:
            return c


# ---------------------------------------------------------------- the layout

def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _share(case, b):
    """How much of the full length sequence b of a ragged batch has: 30% to 100%."""
    return 0.3 + 0.7 * ((b * 0.6180339887) % 1.0) if case["ragged"] and b else 1.0


def _lengths(case):
    """Per sequence the entries its cache holds and the full-resolution position that follows them."""
    lens, pos = [], []
    for b in range(case["batch"]):
        f = _share(case, b)
        text, frames = int(case["prefix"] * f) + case["generated"], int(case["frames"] * f)
        lens.append(text + -(-frames // case["w"]))
        pos.append(text + frames)
    return lens, pos


def _counts(case, full):
    """Per sequence how many of `full` new tokens it has."""
    return [max(1, int(full * _share(case, b))) for b in range(case["batch"])]


def work(case):
    elt = 2 if case["dtype"] == "bf16" else 4
    row = case["dim"] * elt
    if case["kind"] == "append":
        n = sum(_counts(case, case["new"]))
        return {"bytes": n * (2 * row * (case["q_heads"] + 2 * case["kv_heads"]) + 4),
                "flops": n * 3 * case["rot"] * (case["q_heads"] + case["kv_heads"])}
    lens, _ = _lengths(case)
    if case["kind"] == "tree":
        nodes = _counts(case, case["nodes"])
        # a node of a tree sees itself and about log2 of the nodes before it
        pairs = sum(n * L + (n * (n + 1) // 2 if case["chain"] else int(n * (1 + math.log2(n))))
                    for n, L in zip(nodes, lens))
        return {"bytes": sum(2 * row * (case["kv_heads"] * (L + n) + case["q_heads"] * n)
                             for n, L in zip(nodes, lens)),
                "flops": 4 * case["dim"] * case["q_heads"] * pairs}
    moved = sum(max(0, p - 1) for p in _counts(case, case["path"]))  # (the root stays where it is)
    return {"bytes": max(1, moved) * case["layers"] * 4 * row * case["kv_heads"], "flops": 0}


# ------------------------------------------------------------------ preparing

def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _parents(rng, n, chain):
    """A drafted tree in breadth order: each node's parent comes before it."""
    if chain:
        return [i - 1 for i in range(n)]
    return [-1] + [rng.randint((i - 1) // 4, (i - 1) // 2) for i in range(1, n)]


def _ancestors(parents):
    """bool [n, n]: node i sees node j (itself and its ancestors)."""
    see = np.eye(len(parents), dtype=bool)
    for i, p in enumerate(parents):
        if p >= 0:
            see[i] |= see[p]
    return see


def _words(see, n):
    """Rows of bits as int32 words, bit j % 32 of word j // 32."""
    W = -(-n // 32)
    bits = np.zeros((n, 32 * W), dtype=np.uint64)
    bits[:see.shape[0], :see.shape[1]] = see
    words = (bits.reshape(n, W, 32) << np.arange(32, dtype=np.uint64)).sum(2)
    return words.astype(np.uint32).view(np.int32)


class _Rng:
    """Small whole numbers of one seed, on the host."""

    def __init__(self, seed):
        self.g = np.random.default_rng(seed)

    def randint(self, lo, hi):
        return int(self.g.integers(lo, hi + 1))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    host = torch.Generator()
    host.manual_seed(seed)
    rng = _Rng(seed)
    kind, B, Hq, Hkv, D, ps, dt = (case["kind"], case["batch"], case["q_heads"], case["kv_heads"],
                                   case["dim"], case["page"], _dt(case))
    layers = case.get("layers", 1)
    more = case["new"] if kind == "append" else case["nodes"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt)

    lens, pos = _lengths(case)
    per = -(-(max(lens) + more) // ps)
    total = layers * B * per
    # one pool of pages for every layer and sequence, in the order of a busy
    # server's allocator
    s = dict(case=case, k_pages=torch.empty((total, Hkv, ps, D), dtype=dt, device="cuda").normal_(generator=g),
             v_pages=torch.empty((total, Hkv, ps, D), dtype=dt, device="cuda").normal_(generator=g),
             table=torch.randperm(total, generator=host).to(torch.int32).view(layers, B, per).cuda(),
             lens=_i32([lens] * layers), longest=max(lens),
             lens_out=torch.zeros((layers, B), dtype=torch.int32, device="cuda"))
    if kind == "append":
        S = case["new"]
        if case["fused"]:  # views of one projection's output
            qkv = normal(B, S, Hq + 2 * Hkv, D)
            s.update(q=qkv[:, :, :Hq], k=qkv[:, :, Hq:Hq + Hkv], v=qkv[:, :, Hq + Hkv:])
        else:
            s.update(q=normal(B, S, Hq, D), k=normal(B, S, Hkv, D), v=normal(B, S, Hkv, D))
        counts = _counts(case, S)
        first = torch.tensor(pos, dtype=torch.int32)[:, None]
        rot = case["rot"]
        s.update(positions=(first + torch.arange(S, dtype=torch.int32)).cuda(),
                 new_len=_i32(counts) if case["ragged"] else None,
                 inv_freq=(1e6 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float().cuda()
                 if rot else None,
                 q_out=torch.zeros((B, S, Hq, D), dtype=dt, device="cuda"))
    elif kind == "tree":
        n = case["nodes"]
        counts = _counts(case, n)
        s.update(q=normal(B, n, Hq, D), out=torch.zeros((B, n, Hq, D), dtype=dt, device="cuda"),
                 num_nodes=_i32(counts) if case["ragged"] else None, mask=None)
        if not case["chain"]:
            trees = [_words(_ancestors(_parents(rng, n, False)), n) for _ in range(1 if case["shared"] else B)]
            words = torch.from_numpy(np.stack(trees)).cuda()
            s["mask"] = words[0] if case["shared"] else words
    else:
        n, m = case["nodes"], case["path"]
        counts = _counts(case, m)
        path = np.zeros((B, m), dtype=np.int32)
        for b in range(B):
            # accepted nodes in order: the first ones of the draft, then a jump
            # past the slots that the path fills, as in a tree whose later
            # levels lie behind its early ones (a second pass then moves the
            # same values again)
            stay = rng.randint(1, counts[b])
            free = list(range(m, n))
            jump = sorted(rng.g.choice(free, size=min(counts[b] - stay, len(free)), replace=False)) if free else []
            stay = counts[b] - len(jump)
            path[b, :counts[b]] = list(range(stay)) + [int(x) for x in jump]
        s.update(path=torch.from_numpy(path).cuda(), path_len=_i32(counts))
    if own:
        from paper_2607_06827_amd import speechkv as skv
        s["caches"] = [skv.PagedKV(s["k_pages"], s["v_pages"], s["table"][i]) for i in range(layers)]
        if kind == "tree":
            need = skv.speechkv_tree_workspace_bytes(B, case["nodes"], Hq, Hkv, D, s["longest"])
            s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        if kind == "commit":
            s["stack"] = skv.CacheStack(s["caches"], list(s["lens"]), list(s["lens_out"]))
    return s


# -------------------------------------------------------------------- running

def run(state):
    return {"append": _append, "tree": _tree, "commit": _commit}[state["case"]["kind"]](state)


def _slots(s, c):
    """Page and row of cache entry c [layers, B, ...] of each sequence."""
    ps = s["case"]["page"]
    flat = c.reshape(c.shape[0], c.shape[1], -1).long()
    return s["table"].gather(2, flat // ps).view(c.shape).long(), (flat % ps).view(c.shape)


def _rotated(x, cos, sin, layout):
    """x [B, S, H, D] in fp32 with its first 2 * (last axis of cos) elements rotated."""
    half = cos.shape[-1]
    r, rest = x[..., :2 * half], x[..., 2 * half:]
    cos, sin = cos[:, :, None], sin[:, :, None]
    if layout == "halves":
        a, b = r[..., :half], r[..., half:]
        r = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([r, rest], -1)


def _append(s):
    case = s["case"]
    if own:
        from paper_2607_06827_amd import speechkv as skv
        skv.speechkv_append_kv(s["k"], s["v"], s["caches"][0], s["lens"][0], positions=s["positions"],
                               inv_freq=s["inv_freq"],
                               rope=skv.ROPE_HALVES if case["layout"] == "halves" else skv.ROPE_PAIRS,
                               q=s["q"], q_out=s["q_out"], new_len=s["new_len"],
                               cache_len_out=s["lens_out"][0])
        return s["q_out"], s["k_pages"], s["v_pages"], s["lens_out"]
    B, S = s["positions"].shape
    dt, i = _dt(case), torch.arange(S, device="cuda")
    q, k = s["q"].float(), s["k"].float()
    if s["inv_freq"] is not None:
        # (in 64 bits: positions of minutes of audio times a frequency of 1)
        angle = s["positions"].double()[..., None] * s["inv_freq"].double()
        cos, sin = angle.cos().float(), angle.sin().float()
        q, k = _rotated(q, cos, sin, case["layout"]), _rotated(k, cos, sin, case["layout"])
    page, row = (x[0] for x in _slots(s, s["lens"][:, :, None] + i))
    count = torch.full((B,), S, device="cuda") if s["new_len"] is None else s["new_len"]
    there = (i < count[:, None])[..., None, None]
    s["k_pages"][page, :, row] = torch.where(there, k.to(dt), s["k_pages"][page, :, row])
    s["v_pages"][page, :, row] = torch.where(there, s["v"], s["v_pages"][page, :, row])
    s["q_out"].copy_(torch.where(there, q.to(dt), s["q_out"]))
    s["lens_out"].copy_(s["lens"] + count)
    return s["q_out"], s["k_pages"], s["v_pages"], s["lens_out"]


def _tree(s):
    case = s["case"]
    if own:
        from paper_2607_06827_amd import speechkv as skv
        skv.speechkv_tree_attn(s["q"], s["caches"][0], s["lens"][0], s["longest"], s["out"],
                               tree_mask=s["mask"], num_nodes=s["num_nodes"], workspace=s["workspace"])
        return s["out"]
    B, n, Hq, D = s["q"].shape
    Hkv, dt = case["kv_heads"], _dt(case)
    k = s["k_pages"][s["table"][0].long()].transpose(1, 2).reshape(B, Hkv, -1, D).float()
    v = s["v_pages"][s["table"][0].long()].transpose(1, 2).reshape(B, Hkv, -1, D).float()
    node, j = torch.arange(n, device="cuda"), torch.arange(k.shape[2], device="cuda")
    count = torch.full((B,), n, device="cuda") if s["num_nodes"] is None else s["num_nodes"]
    j = j - s["lens"][0][:, None]  # [B, keys]: which drafted node a cache entry is
    at = j.clamp(0, n - 1)
    if s["mask"] is None:
        bit = at[:, None] <= node[:, None]
    else:
        words = s["mask"].expand(B, n, -1).gather(2, (at // 32)[:, None].expand(B, n, -1))
        bit = (words >> (at % 32)[:, None]) & 1 != 0
    see = (j < 0)[:, None] | ((j < count[:, None])[:, None] & bit)
    see = see[:, None, :, None]  # [B, 1, n, 1, keys]
    q = s["q"].float().view(B, n, Hkv, Hq // Hkv, D).transpose(1, 2)
    z = torch.matmul(q.reshape(B, Hkv, -1, D), k.transpose(2, 3).contiguous()) * D ** -0.5
    z = torch.where(see, z.view(B, Hkv, n, Hq // Hkv, -1), -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul((p / torch.where(total == 0, 1.0, total)).view(B, Hkv, -1, k.shape[2]), v)
    o = o.view(B, Hkv, n, Hq // Hkv, D).transpose(1, 2).reshape(B, n, Hq, D).to(dt)
    s["out"].copy_(torch.where((node < count[:, None])[..., None, None], o, s["out"]))
    return s["out"]


def _commit(s):
    if own:
        from paper_2607_06827_amd import speechkv as skv
        skv.speechkv_tree_commit(s["stack"], s["path"], s["path_len"], s["case"]["nodes"])
        return s["k_pages"], s["v_pages"], s["lens_out"]
    j = torch.arange(s["path"].shape[1], device="cuda")
    page, row = _slots(s, s["lens"][:, :, None] + s["path"])
    to_page, to_row = _slots(s, s["lens"][:, :, None] + j)
    keep = (j < s["path_len"][:, None])[None, :, :, None, None]
    s["k_pages"][to_page, :, to_row] = torch.where(keep, s["k_pages"][page, :, row], s["k_pages"][to_page, :, to_row])
    s["v_pages"][to_page, :, to_row] = torch.where(keep, s["v_pages"][page, :, row], s["v_pages"][to_page, :, to_row])
    s["lens_out"].copy_(s["lens"] + s["path_len"])
    return s["k_pages"], s["v_pages"], s["lens_out"]


# ---------------------------------------------------------------- in 64 bits

def exact(case, seed):
    """What a pass returns, from the definitions, one sequence after the other
    in 64 bits.  Values that are only moved have no such result."""
    if case["kind"] == "commit":
        return None
    s = prepare(case, seed)
    ps, B = case["page"], case["batch"]
    table, lens = s["table"][0].tolist(), s["lens"][0].tolist()
    if case["kind"] == "append":
        new = case["new"]
        counts = [new] * B if s["new_len"] is None else s["new_len"].tolist()
        q_out, k_pages = s["q_out"].double(), s["k_pages"].double()
        for b in range(B):
            n = counts[b]
            q, k = s["q"][b, :n].double(), s["k"][b, :n].double()
            for j in range(case["rot"] // 2):
                x, y = (j, j + case["rot"] // 2) if case["layout"] == "halves" else (2 * j, 2 * j + 1)
                a = s["positions"][b, :n].double()[:, None] * s["inv_freq"][j].double()
                c, d = torch.cos(a), torch.sin(a)
                for t in (q, k):
                    u, w = t[..., x].clone(), t[..., y].clone()
                    t[..., x], t[..., y] = u * c - w * d, u * d + w * c
            q_out[b, :n] = q
            slot = torch.arange(lens[b], lens[b] + n)
            page = torch.tensor(table[b])[slot // ps]
            k_pages[page.cuda(), :, (slot % ps).cuda()] = k
        return q_out, k_pages, None, None
    nodes = case["nodes"]
    counts = [nodes] * B if s["num_nodes"] is None else s["num_nodes"].tolist()
    out, G = s["out"].double(), case["q_heads"] // case["kv_heads"]
    words = None if s["mask"] is None else s["mask"].cpu().numpy().view(np.uint32)
    for b in range(B):
        n, L = counts[b], lens[b]
        pages = torch.tensor(table[b], device="cuda")[:-(-(L + n) // ps)]
        see = np.ones((n, L + n), dtype=bool)
        if words is None:
            see[:, L:] = np.tri(n, dtype=bool)
        else:
            rows = np.ascontiguousarray((words if words.ndim == 2 else words[b])[:n])
            see[:, L:] = np.unpackbits(rows.view(np.uint8), axis=1, bitorder="little")[:, :n]
        hide = torch.from_numpy(~see).cuda()
        for g in range(case["kv_heads"]):
            k = s["k_pages"][pages, g].double().flatten(0, 1)[:L + n]
            v = s["v_pages"][pages, g].double().flatten(0, 1)[:L + n]
            for h in range(g * G, g * G + G):
                z = s["q"][b, :n, h].double() @ k.T.contiguous() / math.sqrt(case["dim"])
                z[hide] = -math.inf
                out[b, :n, h] = torch.softmax(z, 1) @ v
    return out
