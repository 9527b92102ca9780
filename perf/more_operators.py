"""Many questions about recordings, within a budget of cache entries, as cases that can be timed and checked.

A case is one pass through one of five operators: norms of queries and keys for
each head with the position rotation (dense, or straight into the cache), the
gradient of that, attention of single tokens that share a long prefix, the
attention weight that cache entries gather, and the eviction of the entries
that gathered least.  With `own` set a pass makes the calls of
paper_2607_06827_amd.speechkv that a program makes; without it the same values
are computed from elementary torch operations.  Frames are 80 ms, so 375 are
30 s of audio, 750 are 60 s, 1500 are two minutes and 7500 are 10 minutes; a
layer from the first compressed one on keeps one entry per window of w frames.
"""
import math

import torch

own = False
EPS = 1e-6  # of the norms


def _case(name, kind, **kw):
    c = dict(name=name, kind=kind, dtype="bf16", batch=1, q_heads=16, kv_heads=8, dim=128, page=16)
    c.update(dict(
        # rows of a sequence, rotated elements of a head, axes of the positions
        norm=dict(rows=1, rot=128, layout="halves", axes=1, append=False, ragged=False),
        norm_bwd=dict(rows=1, rot=128, layout="halves", axes=1, ragged=False),
        # recordings, their frames and window, text before the speech, a
        # question's own entries
        shared=dict(recordings=1, frames=375, w=4, prefix=32, mine=40, ragged=False),
        # queries of a sequence: the last token, or a whole prompt
        weights=dict(prompt=False, frames=375, w=4, prefix=32, mine=40, ragged=False),
        evict=dict(layers=1, entries=400, keep=256, first=4, recent=32, ragged=False))[kind])
    c.update(kw)
    return c


def listed():
    return [
        # one token of one user into the cache: the smallest call of a decoding loop
        _case("norm_one_token", "norm", append=True),
        # the prompt of 8 users with two minutes of audio, out of one fused
        # projection, positions with time, height and width axes
        _case("norm_prompt", "norm", batch=8, rows=1596, axes=3),
        # the same prompt in training
        _case("norm_bwd_train", "norm_bwd", batch=8, rows=1596),
        # fp32, a quarter of the elements rotated as neighbours, odd lengths
        _case("norm_bwd_f32", "norm_bwd", dtype="f32", batch=5, rows=301, q_heads=8, kv_heads=4, dim=64, rot=32,
              layout="pairs", axes=2, ragged=True),
        # eight questions about 30 s of audio, a compressed layer
        _case("shared_30s", "shared", batch=8),
        # 64 questions about one recording of 10 minutes, a layer that keeps every frame
        _case("shared_10min", "shared", batch=64, frames=7500, w=1, mine=96, ragged=True),
        # 40 questions about six recordings of two minutes, unequal groups and
        # lengths, eight query heads per KV head, bigger pages
        _case("shared_recordings", "shared", batch=40, recordings=6, q_heads=64, frames=1500, w=1, mine=301, page=64,
              ragged=True),
        # fp32, odd sizes
        _case("shared_f32", "shared", dtype="f32", batch=21, recordings=2, q_heads=16, kv_heads=4, dim=64, frames=601,
              w=3, mine=33, ragged=True),
        # a decoding step of 16 users with 10 minutes of audio, a layer that keeps every frame
        _case("weights_step", "weights", batch=16, frames=7500, w=1, mine=128),
        # what the whole prompt of 8 users with two minutes of audio looks at, a compressed layer
        _case("weights_prompt", "weights", batch=8, prompt=True, frames=1500, mine=64),
        # one layer of one user
        _case("evict_one_layer", "evict"),
        # 28 layers of 8 users with 60 s of audio, every frame kept so far
        _case("evict_stack", "evict", batch=8, layers=28, entries=846, keep=512, ragged=True),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        w, k = work(c), c["kind"]
        most[k] = tuple(max(x, y) for x, y in zip(most.get(k, (0, 0)), (w["bytes"], w["flops"])))
    while True:
        kind = rng.choice(["norm", "norm", "norm_bwd", "norm_bwd", "shared", "shared", "shared", "weights", "weights",
                           "evict", "evict"])
        kv = rng.choice([1, 2, 4, 8])
        dim = rng.choice([64, 128, 128])
        c = _case("", kind, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), kv_heads=kv,
                  q_heads=kv * rng.choice([1, 2, 2, 4, 8]), dim=dim, page=rng.choice([8, 16, 16, 32, 64, 128]),
                  ragged=rng.random() < 0.5)
        del c["name"]
        frames, w = rng.choice([_logint(rng, 1, 7500), _logint(rng, 30, 7500)]), rng.choice([1, 1, 2, 3, 4, 8])
        if kind in ("norm", "norm_bwd"):
            c.update(batch=_logint(rng, 1, 64), rows=_logint(rng, 1, 2000), rot=16 * rng.randint(0, dim // 16),
                     layout=rng.choice(["halves", "halves", "pairs"]), axes=rng.choice([1, 1, 2, 3]))
            if kind == "norm":
                c.update(append=rng.random() < 0.5)
        elif kind == "shared":
            batch = _logint(rng, 1, 64)
            c.update(batch=batch, recordings=rng.randint(1, max(1, batch // 3)), frames=frames, w=w,
                     prefix=rng.randint(0, 64), mine=_logint(rng, 1, 400))
        elif kind == "weights":
            c.update(batch=_logint(rng, 1, 32), prompt=rng.random() < 0.5, frames=frames, w=w,
                     prefix=rng.randint(0, 64), mine=rng.randint(1, 256))
        else:
            entries = _logint(rng, 2, 7800)
            first, recent = rng.randint(0, 8), rng.randint(0, 64)
            c.update(batch=_logint(rng, 1, 32), layers=rng.choice([1, 4, 28]), entries=entries,
                     keep=rng.randint(1, entries), first=first, recent=recent)
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


def _counts(case, full):
    """Per sequence how many of `full` rows it has."""
    return [max(1, int(full * _share(case, b))) for b in range(case["batch"])]


def _speech(case, j):
    """(text before the speech, frames) of sequence or recording j."""
    f = _share(case, j)
    return int(case["prefix"] * f), max(1, int(case["frames"] * f))


def _groups(case):
    """First sequence of each recording's group, and the batch: unequal groups."""
    n, B = case["recordings"], case["batch"]
    size = [1.0 + (0.7 * j if case["ragged"] else 0.0) for j in range(n)]
    at, start = 0.0, [0]
    for s in size:
        at += s
        start.append(max(start[-1], int(round(B * at / sum(size)))))
    return start


def _lengths(case):
    """Entries of each sequence's cache (of each recording's, for shared prefixes)."""
    if case["kind"] == "evict":
        return _counts(case, case["entries"])
    n = case["recordings"] if case["kind"] == "shared" else case["batch"]
    more = 0 if case["kind"] == "shared" else case["mine"]
    return [p + -(-t // case["w"]) + more for p, t in (_speech(case, j) for j in range(n))]


def _visible(case):
    """Of a prompt (text, speech, text): how many cache entries each row sees, per sequence."""
    w, out = case["w"], []
    for b in range(case["batch"]):
        p, t = _speech(case, b)
        # a window is seen from its last frame on
        rows = [i + 1 for i in range(p)] + [p + -(-t // w) if i + 1 == t else p + (i + 1) // w for i in range(t)]
        out.append(rows + [p + -(-t // w) + m + 1 for m in range(case["mine"])])
    return out


def work(case):
    elt = 2 if case["dtype"] == "bf16" else 4
    Hq, Hkv, D = case["q_heads"], case["kv_heads"], case["dim"]
    row, kind = D * elt, case["kind"]
    if kind in ("norm", "norm_bwd"):
        n, H = sum(_counts(case, case["rows"])), Hq + Hkv
        if kind == "norm":
            moved = 2 * row * (H + (Hkv if case["append"] else 0))
            return {"bytes": n * (moved + 4 * case["axes"]), "flops": n * H * (4 * D + 3 * case["rot"])}
        return {"bytes": n * (3 * row * H + 4 * case["axes"]), "flops": n * H * (10 * D + 3 * case["rot"])}
    lens = _lengths(case)
    if kind == "shared":
        mine, start = _counts(case, case["mine"]), _groups(case)
        pairs = sum(mine) + sum(n * (e - s) for n, s, e in zip(lens, start, start[1:]))
        read = sum(mine) + sum(n for n, s, e in zip(lens, start, start[1:]) if e > s)
        return {"bytes": 2 * row * (Hkv * read + Hq * case["batch"]) + 4 * Hq * case["batch"],
                "flops": 4 * D * Hq * pairs}
    if kind == "weights":
        rows = [sum(_speech(case, b)) + case["mine"] if case["prompt"] else 1 for b in range(case["batch"])]
        pairs = sum(map(sum, _visible(case))) if case["prompt"] else sum(lens)
        return {"bytes": sum(Hkv * L * (row + 8) + Hq * n * (row + 4) for L, n in zip(lens, rows)),
                "flops": 2 * D * Hq * pairs}
    kept = [min(L, case["keep"]) for L in lens]
    # (entries before the first one that goes stay where they are)
    moved = sum(max(1, k - min(k, case["first"])) if k < L else 0 for k, L in zip(kept, lens))
    return {"bytes": case["layers"] * Hkv * (4 * row * moved + 8 * sum(lens) + 4 * sum(kept)), "flops": 0}


# ------------------------------------------------------------------ preparing

def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _padded(rows, fill=0):
    n = max(map(len, rows))
    return _i32([r + [fill] * (n - len(r)) for r in rows])


def _pages(case, g, host, tables, slots):
    """K and V pages and `tables` block tables with room for `slots` entries a
    sequence, in the order of a busy server's allocator."""
    ps, B = case["page"], slots[1]
    per = -(-slots[0] // ps)
    shape = (tables * B * per, case["kv_heads"], ps, case["dim"])
    k, v = (torch.empty(shape, dtype=_dt(case), device="cuda").normal_(generator=g) for _ in range(2))
    return k, v, torch.randperm(shape[0], generator=host).to(torch.int32).view(tables, B, per).cuda()


def _lse(case, q, k, seen):
    """Natural log-sum-exp of each row of q [n, Hq, D] over the first seen[i] of the keys k [L, Hkv, D]."""
    z = _logits(case, q, k)
    z = torch.where(torch.arange(k.shape[0], device="cuda") < seen[:, None, None], z, -math.inf)
    return z.logsumexp(-1)


def _logits(case, q, k):
    """[n, Hq, L] in fp32."""
    G = case["q_heads"] // case["kv_heads"]
    k = k.float().permute(1, 2, 0).repeat_interleave(G, 0).contiguous()
    return torch.matmul(q.float().transpose(0, 1).contiguous(), k).transpose(0, 1) * case["dim"] ** -0.5


def _entries(s, table, n):
    """The first n entries of a block-table row: K and V [n, Hkv, D]."""
    ps = s["case"]["page"]
    pages = table[:-(-n // ps)].long()
    return tuple(x[pages].transpose(1, 2).flatten(0, 1)[:n] for x in (s["k_pages"], s["v_pages"]))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    host = torch.Generator()
    host.manual_seed(seed)
    kind, B, Hq, Hkv, D, dt = (case["kind"], case["batch"], case["q_heads"], case["kv_heads"], case["dim"], _dt(case))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt)

    s = dict(case=case)
    if kind in ("norm", "norm_bwd"):
        S, rot, A = case["rows"], case["rot"], case["axes"]
        counts = _counts(case, S)
        qkv = 1.7 * normal(B, S, Hq + 2 * Hkv, D)  # one projection's output
        t = (torch.arange(B)[:, None] * 211 + 1000 + torch.arange(S)).to(torch.int32)
        # the first axis is time, the others a picture's rows and columns
        s.update(q=qkv[:, :, :Hq], k=qkv[:, :, Hq:Hq + Hkv], v=qkv[:, :, Hq + Hkv:], counts=counts,
                 positions=torch.stack([t, t // 16 % 31, t % 16][:A]).cuda(),
                 inv_freq=(1e6 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float().cuda(),
                 axis=(torch.arange(rot // 2) * A // max(rot // 2, 1)).to(torch.int32).cuda(),
                 row_len=_i32(counts) if case["ragged"] else None,
                 gamma_q=1 + 0.2 * torch.randn(D, generator=g, device="cuda"),
                 gamma_k=1 + 0.2 * torch.randn(D, generator=g, device="cuda"))
        zeros = lambda h: torch.zeros((B, S, h, D), dtype=dt, device="cuda")  # noqa: E731
        if kind == "norm_bwd":
            s.update(dq_out=normal(B, S, Hq, D), dk_out=normal(B, S, Hkv, D), dq=zeros(Hq), dk=zeros(Hkv),
                     dgamma_q=torch.zeros(D, device="cuda"), dgamma_k=torch.zeros(D, device="cuda"))
        else:
            s.update(q_out=zeros(Hq))
            if case["append"]:
                lens = [(b * 37) % 211 for b in range(B)]
                k, v, table = _pages(case, g, host, 1, (max(lens) + S, B))
                s.update(k_pages=k, v_pages=v, table=table[0], lens=_i32(lens), lens_out=_i32([0] * B))
            else:
                s.update(k_out=zeros(Hkv))
    elif kind == "shared":
        n, lens, start, mine = case["recordings"], _lengths(case), _groups(case), _counts(case, case["mine"])
        ps = case["page"]
        per, per_mine = -(-max(lens) // ps), -(-max(mine) // ps)
        # one pool for the recordings and the questions
        k, v, order = _pages(case, g, host, 1, ((n * per + B * per_mine) * ps, 1))
        order = order.flatten()
        s.update(k_pages=k, v_pages=v, prefix_table=order[:n * per].view(n, per).contiguous(),
                 table=order[n * per:].view(B, per_mine).contiguous(), prefix_len=_i32(lens), longest=max(lens),
                 lens=_i32(mine), longest_mine=max(mine), start=_i32(start), starts=start, mine=mine, prefix=lens,
                 most=max(e - s for s, e in zip(start, start[1:])), q=normal(B, Hq, D),
                 out=torch.zeros((B, Hq, D), dtype=dt, device="cuda"), lse=torch.zeros((B, Hq), device="cuda"))
    elif kind == "weights":
        lens = _lengths(case)
        k, v, table = _pages(case, g, host, 1, (max(lens), B))
        seen = _visible(case) if case["prompt"] else [[n] for n in lens]
        S = max(map(len, seen))
        s.update(k_pages=k, v_pages=v, table=table[0], lens=_i32(lens), lengths=lens, longest=max(lens), q=normal(B, S, Hq, D),
                 visible=_padded(seen), lse=torch.full((B, Hq, S), -math.inf, device="cuda"),
                 weights=torch.rand((B, Hkv, max(lens)), generator=g, device="cuda"),
                 weights_out=torch.zeros((B, Hkv, max(lens)), device="cuda"))
        for b in range(B):
            m = len(seen[b])
            keys = _entries(s, s["table"][b], lens[b])[0]
            s["lse"][b, :, :m] = _lse(case, s["q"][b, :m], keys, s["visible"][b, :m]).T
    else:
        lens, n = _counts(case, case["entries"]), case["layers"]
        k, v, table = _pages(case, g, host, n, (max(lens), B))
        # weights as attention leaves them: few large ones, many small, some
        # entries that nothing looked at
        shape = (n, B, Hkv, max(lens))
        w = torch.exp(2 * torch.randn(shape, generator=g, device="cuda"))
        w = torch.where(torch.rand(shape, generator=g, device="cuda") < 0.05, 0.0, w)
        s.update(k_pages=k, v_pages=v, table=table, lens=_i32([lens] * n), lengths=lens, weights=w,
                 lens_out=_i32([[0] * B] * n), weights_out=torch.zeros_like(w), keep_len=_i32([case["keep"]] * B),
                 kept=torch.zeros((n, B, Hkv, case["keep"]), dtype=torch.int32, device="cuda"))
    if own:
        _plan(s)
    return s


def _plan(s):
    """What a program keeps beside its tensors: descriptions and workspaces."""
    from paper_2607_06827_amd import speechkv as skv
    case, kind = s["case"], s["case"]["kind"]
    B, Hq, Hkv, D = case["batch"], case["q_heads"], case["kv_heads"], case["dim"]
    space = lambda n: torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")  # noqa: E731
    if kind in ("norm", "norm_bwd"):
        s["rope"] = None
        if case["rot"]:
            s["rope"] = skv.Rope(s["positions"], s["inv_freq"], s["axis"] if case["axes"] > 1 else None,
                                 skv.ROPE_HALVES if case["layout"] == "halves" else skv.ROPE_PAIRS)
        if kind == "norm_bwd":
            s["workspace"] = space(skv.speechkv_norm_rope_bwd_workspace_bytes(B, case["rows"], Hq, Hkv, D))
        elif case["append"]:
            s["cache"] = skv.PagedKV(s["k_pages"], s["v_pages"], s["table"])
    elif kind == "shared":
        s["prefix_cache"] = skv.PagedKV(s["k_pages"], s["v_pages"], s["prefix_table"])
        s["cache"] = skv.PagedKV(s["k_pages"], s["v_pages"], s["table"])
        s["workspace"] = space(skv.speechkv_shared_workspace_bytes(B, case["recordings"], s["most"], Hq, Hkv, D,
                                                                   s["longest"], s["longest_mine"]))
    elif kind == "weights":
        s["cache"] = skv.PagedKV(s["k_pages"], s["v_pages"], s["table"])
    else:
        caches = [skv.PagedKV(s["k_pages"], s["v_pages"], t) for t in s["table"]]
        s["stack"] = skv.EvictStack(caches, list(s["lens"]), list(s["lens_out"]), list(s["weights"]),
                                    list(s["weights_out"]), list(s["kept"]))


# -------------------------------------------------------------------- running

def run(state):
    return {"norm": _norm, "norm_bwd": _norm_bwd, "shared": _shared, "weights": _weights,
            "evict": _evict}[state["case"]["kind"]](state)


def _angles(s):
    """cos and sin [B, S, 1, rot / 2] in fp32 (in 64 bits before: positions of
    minutes of audio times a frequency of 1)."""
    pos = s["positions"][s["axis"].long()].permute(1, 2, 0)
    angle = pos.double() * s["inv_freq"].double()
    return angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]


def _rotated(x, cos, sin, layout):
    """x [B, S, H, D] in fp32 with its first 2 * (last axis of cos) elements rotated."""
    half = cos.shape[-1]
    r, rest = x[..., :2 * half], x[..., 2 * half:]
    if layout == "halves":
        a, b = r[..., :half], r[..., half:]
        r = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([r, rest], -1)


def _there(s):
    """bool [B, S, 1, 1]: the rows that their sequence has."""
    i = torch.arange(s["case"]["rows"], device="cuda")
    count = s["row_len"] if s["row_len"] is not None else torch.full((s["case"]["batch"],), i.numel(), device="cuda")
    return (i < count[:, None])[..., None, None]


def _norm(s):
    case = s["case"]
    if own:
        from paper_2607_06827_amd import speechkv as skv
        if case["append"]:
            skv.speechkv_norm_append_kv(s["q"], s["k"], s["v"], s["cache"], s["lens"], s["q_out"], s["gamma_q"],
                                        s["gamma_k"], eps=EPS, rope=s["rope"], new_len=s["row_len"],
                                        cache_len_out=s["lens_out"])
            return s["q_out"], s["k_pages"], s["v_pages"], s["lens_out"]
        skv.speechkv_norm_rope(s["q"], s["k"], s["q_out"], s["k_out"], s["gamma_q"], s["gamma_k"], eps=EPS,
                               rope=s["rope"], row_len=s["row_len"])
        return s["q_out"], s["k_out"]
    dt, there, (cos, sin) = _dt(case), _there(s), _angles(s)
    done = []
    for x, gamma in ((s["q"], s["gamma_q"]), (s["k"], s["gamma_k"])):
        x = x.float()
        x = x * (x * x).mean(-1, keepdim=True).add(EPS).rsqrt() * gamma
        done.append(_rotated(x, cos, sin, case["layout"]).to(dt))
    q, k = done
    s["q_out"].copy_(torch.where(there, q, s["q_out"]))
    if not case["append"]:
        s["k_out"].copy_(torch.where(there, k, s["k_out"]))
        return s["q_out"], s["k_out"]
    slot = s["lens"][:, None] + torch.arange(case["rows"], device="cuda")
    page, row = s["table"].gather(1, slot // case["page"]).long(), slot % case["page"]
    s["k_pages"][page, :, row] = torch.where(there, k, s["k_pages"][page, :, row])
    s["v_pages"][page, :, row] = torch.where(there, s["v"], s["v_pages"][page, :, row])
    s["lens_out"].copy_(s["lens"] + there.flatten(1).sum(1))
    return s["q_out"], s["k_pages"], s["v_pages"], s["lens_out"]


def _norm_bwd(s):
    case = s["case"]
    if own:
        from paper_2607_06827_amd import speechkv as skv
        skv.speechkv_norm_rope_bwd(s["q"], s["k"], s["dq_out"], s["dk_out"], s["dq"], s["dk"], s["gamma_q"],
                                   s["gamma_k"], eps=EPS, rope=s["rope"], row_len=s["row_len"],
                                   dgamma_q=s["dgamma_q"], dgamma_k=s["dgamma_k"], workspace=s["workspace"])
        return s["dq"], s["dk"], s["dgamma_q"], s["dgamma_k"]
    there, (cos, sin) = _there(s), _angles(s)
    for x, dy, gamma, dx, dgamma in ((s["q"], s["dq_out"], s["gamma_q"], s["dq"], s["dgamma_q"]),
                                     (s["k"], s["dk_out"], s["gamma_k"], s["dk"], s["dgamma_k"])):
        x = x.float()
        r = (x * x).mean(-1, keepdim=True).add(EPS).rsqrt()
        x = x * r
        grad = _rotated(dy.float(), cos, -sin, case["layout"])
        h = grad * gamma
        dx.copy_(torch.where(there, (r * (h - x * (h * x).mean(-1, keepdim=True))).to(dx.dtype), dx))
        dgamma.copy_(torch.where(there, grad * x, 0.0).double().sum((0, 1, 2)))  # (a long sum)
    return s["dq"], s["dk"], s["dgamma_q"], s["dgamma_k"]


def _shared(s):
    case = s["case"]
    if own:
        from paper_2607_06827_amd import speechkv as skv
        skv.speechkv_shared_attn(s["q"], s["prefix_cache"], s["prefix_len"], s["longest"], s["start"], s["most"],
                                 s["cache"], s["lens"], s["longest_mine"], s["out"], lse=s["lse"],
                                 workspace=s["workspace"])
        return s["out"], s["lse"]
    B, Hq, D = s["q"].shape
    Hkv, G = case["kv_heads"], Hq // case["kv_heads"]

    def padded(table):
        return tuple(x[table.long()].transpose(1, 2).reshape(table.shape[0], Hkv, -1, D).float()
                     for x in (s["k_pages"], s["v_pages"]))

    def attend(q, k, v, seen):
        """Unnormalised sums, running maxima and weight sums of q [n, Hkv, rows, D] over k, v [n, Hkv, keys, D]."""
        z = torch.matmul(q, k.transpose(2, 3).contiguous()) * D ** -0.5
        z = torch.where(torch.arange(k.shape[2], device="cuda") < seen[:, None, None, None], z, -math.inf)
        top = z.amax(-1, keepdim=True)
        p = torch.exp(z - top)
        return torch.matmul(p, v), top, p.sum(-1, keepdim=True)

    q = s["q"].float().view(B, Hkv, G, D)
    mine = attend(q, *padded(s["table"]), s["lens"])
    prefix = [torch.zeros_like(x) for x in mine]
    k, v = padded(s["prefix_table"])
    for j, (b, e) in enumerate(zip(s["starts"], s["starts"][1:])):
        if b == e:
            continue
        rows = q[b:e].transpose(0, 1).reshape(1, Hkv, -1, D)
        part = attend(rows, k[j:j + 1], v[j:j + 1], s["prefix_len"][j:j + 1])
        for x, y in zip(prefix, part):
            x[b:e] = y.view(Hkv, e - b, G, -1).transpose(0, 1)
    top = torch.maximum(mine[1], prefix[1])
    f, h = torch.exp(mine[1] - top), torch.exp(prefix[1] - top)
    total = f * mine[2] + h * prefix[2]
    s["out"].copy_(((f * mine[0] + h * prefix[0]) / total).view(B, Hq, D))
    s["lse"].copy_((top + total.log()).view(B, Hq))
    return s["out"], s["lse"]


def _weights(s):
    case = s["case"]
    if own:
        from paper_2607_06827_amd import speechkv as skv
        skv.speechkv_attn_weights(s["q"], s["lse"], s["cache"], s["lens"], s["longest"], s["weights_out"],
                                  weights=s["weights"], visible=s["visible"] if case["prompt"] else None)
        return s["weights_out"]
    B, S, Hq, D = s["q"].shape
    Hkv, G = case["kv_heads"], Hq // case["kv_heads"]
    k = s["k_pages"][s["table"].long()].transpose(1, 2).reshape(B, Hkv, -1, D)[:, :, :s["longest"]].float()
    c = torch.arange(s["longest"], device="cuda")
    for b in range(B):
        q = s["q"][b].float().view(S, Hkv, G, D).permute(1, 2, 0, 3).reshape(Hkv, G * S, D)
        z = torch.matmul(q, k[b].transpose(1, 2).contiguous()).view(Hkv, G, S, -1) * D ** -0.5
        z = z - s["lse"][b].view(Hkv, G, S, 1)
        p = torch.where(c < s["visible"][b][:, None], torch.exp(z), 0.0)
        s["weights_out"][b] = torch.where(c < s["lens"][b], s["weights"][b] + p.sum((1, 2)), s["weights_out"][b])
    return s["weights_out"]


def _evict(s):
    if own:
        from paper_2607_06827_amd import speechkv as skv
        skv.speechkv_evict(s["stack"], s["keep_len"], s["case"]["first"], s["case"]["recent"])
        return s["kept"], s["weights_out"], s["k_pages"], s["v_pages"], s["lens_out"]
    case, w = s["case"], s["weights"]
    n, B, Hkv, M = w.shape
    c, keep = torch.arange(M, device="cuda"), case["keep"]
    L = s["lens"][:, :, None, None]
    count = torch.clamp(L, max=keep)  # entries that stay
    f = torch.clamp(count, max=case["first"])
    r = torch.minimum(count - f, torch.full_like(count, case["recent"]))
    # the protected ones before all others, then by weight, ties by slot
    rank = torch.where((c < f) | (c >= L - r), math.inf, w)
    rank = torch.where(c < L, rank, -math.inf)
    order = rank.sort(dim=-1, descending=True, stable=True).indices
    place = torch.empty_like(order).scatter_(-1, order, c.expand_as(order).contiguous())
    stay = (place < count) & (c < L)
    slots = torch.where(stay, c, M).sort(-1).values[..., :min(keep, M)]  # in order, M where there is none
    there = slots < M
    s["kept"][..., :slots.shape[-1]] = torch.where(there, slots, s["kept"][..., :slots.shape[-1]])
    from_ = torch.where(there, slots, 0)
    out = torch.zeros_like(w)
    out[..., :slots.shape[-1]] = torch.where(there, w.gather(-1, from_), 0.0)
    s["weights_out"].copy_(torch.where(c < L, out, s["weights_out"]))
    ps = case["page"]
    table = s["table"].long()[:, :, None].expand(-1, -1, Hkv, -1)
    to = c[:slots.shape[-1]].expand_as(slots)
    page, row = table.gather(-1, from_ // ps), from_ % ps
    to_page, to_row = table.gather(-1, to // ps), to % ps
    head = torch.arange(Hkv, device="cuda")[:, None].expand_as(slots)
    for x in (s["k_pages"], s["v_pages"]):
        x[to_page, head, to_row] = torch.where(there[..., None], x[page, head, row], x[to_page, head, to_row])
    s["lens_out"].copy_(count[..., 0, 0])
    return s["kept"], s["weights_out"], s["k_pages"], s["v_pages"], s["lens_out"]


# ---------------------------------------------------------------- in 64 bits

def exact(case, seed):
    """What a pass returns, from the definitions, in 64 bits, one sequence or
    head after the other.  Values that are only moved or chosen have no such
    result."""
    if case["kind"] == "evict":
        return None
    s = prepare(case, seed)
    return {"norm": _exact_norm, "norm_bwd": _exact_norm_bwd, "shared": _exact_shared,
            "weights": _exact_weights}[case["kind"]](s)


def _pairs(case):
    half = case["rot"] // 2
    return [(j, j + half) if case["layout"] == "halves" else (2 * j, 2 * j + 1) for j in range(half)]


def _turn(s, b, n, x, sign):
    """x [n, H, D] of the first n rows of sequence b with its pairs turned, in 64 bits."""
    x = x.clone()
    for j, (u, w) in enumerate(_pairs(s["case"])):
        a = s["positions"][s["axis"][j].long(), b, :n].double()[:, None] * s["inv_freq"][j].double()
        c, d = torch.cos(a), sign * torch.sin(a)
        x[..., u], x[..., w] = x[..., u] * c - x[..., w] * d, x[..., u] * d + x[..., w] * c
    return x


def _exact_norm(s):
    case = s["case"]
    q_out = s["q_out"].double()
    k_out = s["k_pages"].double() if case["append"] else s["k_out"].double()
    for b, n in enumerate(s["counts"]):
        done = []
        for x, gamma in ((s["q"], s["gamma_q"]), (s["k"], s["gamma_k"])):
            x = x[b, :n].double()
            size = torch.sqrt(torch.linalg.vecdot(x, x) / case["dim"] + EPS)[..., None]
            done.append(_turn(s, b, n, x / size * gamma.double(), 1.0))
        q_out[b, :n] = done[0]
        if case["append"]:
            slot = s["lens"][b] + torch.arange(n, device="cuda")
            k_out[s["table"][b][slot // case["page"]].long(), :, slot % case["page"]] = done[1]
        else:
            k_out[b, :n] = done[1]
    return (q_out, k_out, None, None) if case["append"] else (q_out, k_out)


def _exact_norm_bwd(s):
    case, D = s["case"], s["case"]["dim"]
    out, gammas = [], []
    for x, dy, gamma, dx in ((s["q"], s["dq_out"], s["gamma_q"], s["dq"]), (s["k"], s["dk_out"], s["gamma_k"], s["dk"])):
        dx, gamma, dgamma = dx.double(), gamma.double(), torch.zeros(D, dtype=torch.float64, device="cuda")
        for b, n in enumerate(s["counts"]):
            t, g = x[b, :n].double(), _turn(s, b, n, dy[b, :n].double(), -1.0)
            size = torch.sqrt(torch.linalg.vecdot(t, t) / D + EPS)[..., None]
            dgamma += (g * t / size).flatten(0, 1).sum(0)
            # the quotient rule of gamma t / size
            dx[b, :n] = g * gamma / size - t * torch.linalg.vecdot(g * gamma, t)[..., None] / (D * size ** 3)
        out.append(dx)
        gammas.append(dgamma)
    return (*out, *gammas)


def _exact_shared(s):
    case, G = s["case"], s["case"]["q_heads"] // s["case"]["kv_heads"]
    out, lse = s["out"].double(), s["lse"].double()
    for j, (first, end) in enumerate(zip(s["starts"], s["starts"][1:])):
        pk, pv = _entries(s, s["prefix_table"][j], s["prefix"][j])
        pk, pv = pk.double(), pv.double()
        for b in range(first, end):
            k, v = _entries(s, s["table"][b], s["mine"][b])
            k, v = torch.cat([pk, k.double()]), torch.cat([pv, v.double()])
            for h in range(case["q_heads"]):
                z = k[:, h // G] @ s["q"][b, h].double() / math.sqrt(case["dim"])
                lse[b, h] = torch.logsumexp(z, 0)
                out[b, h] = torch.softmax(z, 0) @ v[:, h // G]
    return out, lse


def _exact_weights(s):
    case, G = s["case"], s["case"]["q_heads"] // s["case"]["kv_heads"]
    out = s["weights_out"].double()
    for b, L in enumerate(s["lengths"]):
        k = _entries(s, s["table"][b], L)[0].double()
        hide = torch.arange(L, device="cuda") >= s["visible"][b][:, None]
        for g in range(case["kv_heads"]):
            total = s["weights"][b, g, :L].double()
            for h in range(g * G, g * G + G):
                z = s["q"][b, :, h].double() @ k[:, g].T.contiguous() / math.sqrt(case["dim"])
                p = torch.exp(z - s["lse"][b, h].double()[:, None])
                total = total + torch.where(hide, 0.0, p).sum(0)
            out[b, g, :L] = total
    return out
