"""The verifier's side of a decode step, as cases that can be timed.

A step of a serving loop drafts a token tree per request (`speculate`), runs the rows [last token, draft nodes] of the
whole batch through the model, accepts the path that the model agrees with and goes on from there (`step`).  The
operators here are what that needs beside the model's matrix products:

  rotate   norms of queries and keys per head, their rotation to the rows' positions, keys and values into the cache
  attend   attention of the rows over the cache under the tree mask (window, sinks, a prefix that the batch shares)
  accept   the model's choice per row, the accepted path, and the tokens and offsets that `step` takes
  commit   keys and values of accepted rows to the places where the sequence continues, in all layers

Rows of a batch are packed: request i has the rows offsets[i] .. offsets[i+1), the first its last token, the others its
draft nodes in the order of `speculate`; row r lies at place cached[i] + r of the request's cache while it is verified.
"""
import math

import torch

own = False                # the plain forms; True: the calls of paper_2411_04975_b200

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
GQA = dict(q_heads=32, kv_heads=8, head=128, type="bf16")
MHA = dict(q_heads=16, kv_heads=16, head=64, type="fp16")
ROTATE = dict(kind="rotate", rot=128, norm=True, interleaved=False, fused=True, given=False)
ATTEND = dict(kind="attend", max_draft=64, window=0, sinks=0, shared=0)


def listed():
    return [
        # one user of a small deployment, a draft of 16: launch and latency are all of it
        dict(ROTATE | MHA, rot=32, norm=False, interleaved=True, name="rotate_1", n=1, ctx_lo=700, ctx_hi=700, draft_lo=16, draft_hi=16, max_draft=64,
             page=16),
        # the headline batch: 256 requests with 4,096 tokens, drafts of up to 64
        dict(ROTATE, **GQA, name="rotate_256", n=256, ctx_lo=3000, ctx_hi=4200, draft_lo=0, draft_hi=64, max_draft=64, page=16),
        # one token after a context of 8,192: a step without a draft
        dict(ATTEND, **GQA, name="attend_1_token", n=1, ctx_lo=8191, ctx_hi=8191, draft_lo=0, draft_hi=0, page=16),
        # a small service: short contexts, every head with keys of its own
        dict(ATTEND, **MHA, name="attend_16_small", n=16, ctx_lo=32, ctx_hi=400, draft_lo=0, draft_hi=32, page=16),
        # one agent whose context has grown to 131,072 tokens
        dict(ATTEND, **GQA, name="attend_1_long", n=1, ctx_lo=131072, ctx_hi=131072, draft_lo=24, draft_hi=24, page=64),
        # 64 agents: long contexts of every length, large drafts
        dict(ATTEND, **GQA, name="attend_64_agentic", n=64, ctx_lo=1000, ctx_hi=8192, draft_lo=0, draft_hi=64, page=64),
        # layers that see the last 1,024 tokens and the first four
        dict(ATTEND | GQA, q_heads=64, name="attend_128_window", n=128, ctx_lo=512, ctx_hi=8192, draft_lo=0, draft_hi=16, max_draft=16, page=32,
             window=1024, sinks=4),
        # 256 requests behind one system prompt of 4,096 tokens
        dict(ATTEND | GQA, name="attend_256_prefix", n=256, ctx_lo=4150, ctx_hi=5100, draft_lo=0, draft_hi=24, page=64, shared=4096),
        # one request's draft of 16 against the model's choices
        dict(kind="accept", name="accept_1", n=1, draft_lo=16, draft_hi=16, max_draft=64, vocab=128256, type="bf16"),
        # the headline batch's drafts
        dict(kind="accept", name="accept_256", n=256, draft_lo=0, draft_hi=64, max_draft=64, vocab=128256, type="bf16"),
        # one request's accepted rows, a small model
        dict(MHA, kind="commit", name="commit_1", n=1, layers=12, ctx_lo=700, ctx_hi=700, draft_lo=16, draft_hi=16, max_draft=64, page=16),
        # the headline batch's, 32 layers
        dict(GQA, kind="commit", name="commit_256", n=256, layers=32, ctx_lo=3000, ctx_hi=4200, draft_lo=0, draft_hi=64, max_draft=64, page=16),
    ]


def _draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rotate", "attend", "attend", "attend", "accept", "commit"])
    case = {"kind": kind, "n": log(1, 256), "max_draft": rng.choice([16, 24, 32, 64, 64])}
    case["draft_hi"] = rng.randint(0, case["max_draft"])
    case["draft_lo"] = rng.choice([0, 0, case["draft_hi"], case["draft_hi"] // 3])
    if kind == "accept":
        case["vocab"] = log(2000, 151000)
        case["type"] = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        return case
    case["kv_heads"] = rng.choice([1, 2, 4, 8, 8, 10])
    case["q_heads"] = case["kv_heads"] * rng.choice([1, 2, 3, 4, 4, 5, 7, 8])
    case["head"] = rng.choice([64, 128, 128])
    case["type"] = rng.choice(["bf16", "bf16", "fp16"])
    case["page"] = rng.choice([8, 16, 32, 64, 64, 128, 256])
    case["ctx_hi"] = log(1, 131072)
    case["ctx_lo"] = rng.choice([0, case["ctx_hi"] // 7, case["ctx_hi"] // 2, case["ctx_hi"]])
    if kind == "rotate":
        case["rot"] = rng.choice([case["head"], case["head"], case["head"] // 2, 32])
        case["norm"], case["interleaved"], case["fused"], case["given"] = (rng.random() < 0.5 for _ in range(4))
    if kind == "commit":
        case["layers"] = rng.choice([1, 4, 12, 16, 32])
    if kind == "attend":
        case["window"], case["sinks"], case["shared"] = 0, 0, 0
        way = rng.choice(["all", "all", "window", "shared"])
        if way == "window":
            case["window"], case["sinks"] = log(16, 8192), rng.choice([0, 1, 4, 37, 128])
        if way == "shared":
            case["shared"] = log(16, 8192)
            case["ctx_lo"] = case["shared"] + log(1, 200)
            case["ctx_hi"] = case["ctx_lo"] + log(1, 2000)
    return case


def draw(rng):
    """A case of these ranges that costs no more than the largest listed one of its kind."""
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0.0), _cost(c))
    while True:
        case = _draw(rng)
        if _cost(case) <= most[case["kind"]] and _fits(case):
            return case


def _fits(case):
    """Whether the plain form has room: a gibibyte of cache elements each, and of scores."""
    if case["kind"] == "accept":
        return True
    cache = _pool_lines(case) * case["kv_heads"] * case["head"] * case.get("layers", 1)
    scores = case["n"] * (1 + case["draft_hi"]) * (case["ctx_hi"] + case["draft_hi"]) * case["q_heads"] if case["kind"] == "attend" else 0
    return max(cache, scores / 2) <= 1 << 30


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 250)


# ---------------------------------------------------------------------------------------- sizes
def _contexts(case):
    n, lo, hi = case["n"], case["ctx_lo"], case["ctx_hi"]
    return [hi] if n == 1 else [lo + round((hi - lo) * (i + 0.5) / n) for i in range(n)]


def _drafts(case):
    n, lo, hi = case["n"], case["draft_lo"], case["draft_hi"]
    return [hi] if n == 1 else [lo + round((hi - lo) * ((i + 0.5) / n) ** 2) for i in range(n)]


def _pool_lines(case):
    """Cache places that the case's requests need, a shared prefix (or, where only the rows are touched, the context) once."""
    if case["kind"] == "accept":
        return 0
    page, top = case["page"], 1 + case["draft_hi"]
    if case["kind"] in ("rotate", "commit"):
        return case["n"] * (top + 2 * page) + case["ctx_hi"] + page
    shared = case["shared"] // page * page
    return sum((c - shared + top + page) // page * page for c in _contexts(case)) + shared


def work(case):
    n, rows = case["n"], case["n"] + sum(_drafts(case))
    if case["kind"] == "accept":
        size = 4 if case["type"] == "fp32" else 2
        return {"bytes": rows * case["vocab"] * size + n * case["max_draft"] * 8 + rows * 8, "flops": rows * case["vocab"]}
    q, kv = case["q_heads"] * case["head"], case["kv_heads"] * case["head"]
    if case["kind"] == "rotate":
        return {"bytes": 2 * 2 * rows * (q + 2 * kv), "flops": rows * (q + kv) * (6 + 4 * case["norm"])}
    if case["kind"] == "commit":
        moved = sum(min(d, 4) for d in _drafts(case))
        return {"bytes": 2 * moved * 2 * kv * 2 * case["layers"] + n * (case["max_draft"] + 1) * 4, "flops": 0}
    ctx, per = _contexts(case), rows / n
    seen = [min(c, case["window"] + case["sinks"]) if case["window"] else c for c in ctx]
    shared = 0 if case["window"] else case["shared"]
    places = shared + sum(s - shared for s in seen) + rows
    return {"bytes": places * 2 * kv * 2 + 2 * 2 * rows * q, "flops": 4 * q * per * (sum(seen) + rows)}


# --------------------------------------------------------------------------------------- inputs
def _tree(rng, m):
    """Parents of a draft of m nodes, in the order that the best-first growth adds them: mostly chains."""
    return [-1 if j == 0 or u < 0.1 else j - 1 if u < 0.75 else rng.randrange(j) for j, u in ((j, rng.random()) for j in range(m))]


def prepare(case, seed):
    import random

    import numpy as np
    rng = random.Random(seed)
    dev = torch.device("cuda" if torch.cuda.is_available() else "cpu")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def randn(*shape, dtype=None):
        return torch.randn(*shape, device=dev, generator=g, dtype=dtype or TYPES[case["type"]])

    n, M = case["n"], case["max_draft"]
    drafts = _drafts(case)
    rng.shuffle(drafts)
    offsets = np.concatenate([[0], np.cumsum(np.asarray(drafts) + 1)]).astype(np.int64)
    rows = int(offsets[-1])
    parents = np.full((n, M), -1, dtype=np.int32)
    bits = np.zeros((n, M, (M + 31) // 32 * 32), dtype=bool)
    path = np.full((n, M + 1), -1, dtype=np.int32)              # an accepted path: some node's way down, mean length about four
    for i, m in enumerate(drafts):
        parents[i, :m] = _tree(rng, m)
        for j in range(m):
            if parents[i, j] >= 0:
                bits[i, j] = bits[i, parents[i, j]]
            bits[i, j, j] = True
        way = np.nonzero(bits[i, min(m - 1, int(rng.expovariate(1 / 5.0)))])[0] if m else []
        path[i, :len(way) + 1] = np.concatenate([[0], np.asarray(way) + 1])
    mask = np.packbits(bits, axis=-1, bitorder="little").view(np.int32)
    s = {"case": case, "offsets": torch.as_tensor(offsets, device=dev), "parents": torch.as_tensor(parents, device=dev),
         "mask": torch.as_tensor(mask, device=dev), "path": torch.as_tensor(path, device=dev)}
    if case["kind"] == "accept":
        V = case["vocab"]
        tokens = (rng.randrange(V) + torch.arange(n * M, device=dev).view(n, M) * 7919) % V
        nodes = torch.arange(M, device=dev) < torch.as_tensor(drafts, device=dev)[:, None]
        s["tokens"] = torch.where(nodes, tokens, -1).to(torch.int32)
        s["logits"] = randn(rows, V)
        for i in range(n):                                       # the model wants the accepted path's tokens; elsewhere whatever is largest
            way = path[i][path[i] >= 0]
            at = torch.as_tensor(offsets[i] + way[:-1], device=dev)
            s["logits"][at, s["tokens"][i, torch.as_tensor(way[1:] - 1, device=dev).long()].long()] = 12.0
        return s
    contexts = _contexts(case)
    rng.shuffle(contexts)
    H, D, page = case["kv_heads"], case["head"], case["page"]
    shared = case.get("shared", 0)
    need = [-(-(c + d + 1) // page) for c, d in zip(contexts, drafts)]
    table = np.full((n, max(need)), -1, dtype=np.int32)
    if case["kind"] == "attend":
        common = shared // page
        own_pages = [p - common for p in need]
        order = np.random.RandomState(seed % (1 << 31)).permutation(common + sum(own_pages)).astype(np.int32)
        at = common
        for i, p in enumerate(own_pages):
            table[i, :common] = order[:common]
            table[i, common:need[i]] = order[at:at + p]
            at += p
        pages = len(order)
    else:                                                        # only the rows' lines are touched: the contexts share their pages
        first = [c // page for c in contexts]
        common = max(first)
        tails = [p - f for p, f in zip(need, first)]
        pages = common + n * (1 + (case["draft_hi"] + page) // page)                  # whatever draft comes behind whatever context
        order = np.random.RandomState(seed % (1 << 31)).permutation(pages).astype(np.int32)
        at = common
        for i, p in enumerate(tails):
            table[i, :first[i]] = order[:first[i]]
            table[i, first[i]:need[i]] = order[at:at + p]
            at += p
    s["table"] = torch.as_tensor(table, device=dev)
    s["cached"] = torch.as_tensor(np.asarray(contexts, dtype=np.int32), device=dev)
    s["max_rows"] = max(drafts) + 1
    layers = (case["layers"],) if case["kind"] == "commit" else ()
    s["k_cache"], s["v_cache"] = randn(*layers, pages, page, H, D), randn(*layers, pages, page, H, D)
    if case["kind"] == "commit":
        return s
    Q = case["q_heads"]
    if case["kind"] == "attend":
        s["q"] = randn(rows, Q, D) * 1.5
        return s
    if case["fused"]:                                            # views of one matrix product's output
        qkv = randn(rows, Q + 2 * H, D)
        s["q"], s["k"], s["v"] = qkv[:, :Q], qkv[:, Q:Q + H], qkv[:, Q + H:]
    else:
        s["q"], s["k"], s["v"] = randn(rows, Q, D), randn(rows, H, D), randn(rows, H, D)
    half = case["rot"] // 2
    s["freq"] = 500000.0 ** (-torch.arange(half, device=dev, dtype=torch.float64) / half)
    s["weights"] = (1 + 0.2 * randn(D), 1 + 0.2 * randn(D)) if case["norm"] else (None, None)
    s["positions"] = (torch.randint(0, 1 << 20, (rows,), device=dev, generator=g, dtype=torch.int64).to(torch.int32) if case["given"] else None)
    return s


# ------------------------------------------------------------------------------------- the pass
def run(state):
    return {"rotate": _rotate, "attend": _attend, "accept": _accept, "commit": _commit}[state["case"]["kind"]](state)


def _bits(mask, M):
    """[n, M, M]: whether bit j of row i is set."""
    b = torch.arange(32, device=mask.device, dtype=torch.int32)
    return (((mask.unsqueeze(-1) >> b) & 1) != 0).flatten(2)[:, :, :M]


def _rows(s):
    """Request and number within it of every packed row."""
    rows = torch.arange(s["q"].shape[0] if "q" in s else s["logits"].shape[0], device=s["offsets"].device)
    req = torch.searchsorted(s["offsets"], rows, right=True) - 1
    return req, rows - s["offsets"][req]


def _depths(s):
    """[n, M + 1]: how far below its request's last token each row is."""
    d = _bits(s["mask"], s["mask"].shape[1]).sum(-1)
    return torch.cat([torch.zeros_like(d[:, :1]), d], 1)


def _rotate(s):
    c = s["case"]
    if own:
        import paper_2411_04975_b200 as sfx
        q = sfx.sd_rotate(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["offsets"], s["cached"], s["freq"], mask=s["mask"],
                          positions=s["positions"], q_weight=s["weights"][0], k_weight=s["weights"][1], eps=1e-6, interleaved=c["interleaved"])
        return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    req, local = _rows(s)
    positions = s["cached"][req] + _depths(s)[req, local] if s["positions"] is None else s["positions"]
    angle = positions.to(torch.float64)[:, None] * s["freq"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def turned(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()
        r, rest = x[..., :c["rot"]], x[..., c["rot"]:]
        a, b = (r[..., 0::2], r[..., 1::2]) if c["interleaved"] else (r[..., :c["rot"] // 2], r[..., c["rot"] // 2:])
        p, q = a * cos - b * sin, b * cos + a * sin
        r = torch.stack([p, q], -1).flatten(-2) if c["interleaved"] else torch.cat([p, q], -1)
        return torch.cat([r, rest], -1).to(s["q"].dtype)

    q, k = turned(s["q"], s["weights"][0]), turned(s["k"], s["weights"][1])
    place = s["cached"][req] + local
    page, line = s["table"][req, place // c["page"]].long(), (place % c["page"]).long()
    s["k_cache"][page, line] = k
    s["v_cache"][page, line] = s["v"]
    return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _attend(s):
    c = s["case"]
    if own:
        import paper_2411_04975_b200 as sfx
        return {"out": sfx.sd_attend(s["q"], s["k_cache"], s["v_cache"], s["table"], s["offsets"], s["cached"], mask=s["mask"],
                                     window=c["window"], sinks=c["sinks"], shared=c["shared"])}
    n, H, G, D, M, R = c["n"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["head"], c["max_draft"], s["max_rows"]
    dev = s["q"].device
    req, local = _rows(s)
    at = (s["offsets"][:-1, None] + torch.arange(R, device=dev)).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][at].float().view(n, R, H, G, D)
    count = (s["offsets"][1:] - s["offsets"][:-1])[:, None]                          # rows of each request
    table = s["table"].clamp(min=0).long()
    place = torch.arange(table.shape[1] * c["page"], device=dev)[None]
    cached = s["cached"].long()[:, None]
    row = place - cached                                                             # of the tree, where not below 0
    used = row < count
    k = s["k_cache"][table].flatten(1, 2).float()
    v = s["v_cache"][table].flatten(1, 2).float().masked_fill_(~used[..., None, None], 0.0)
    depth = _depths(s)
    sees = torch.zeros(n, M + 1, M + 1, dtype=torch.bool, device=dev)
    sees[:, :, 0] = True
    sees[:, 1:, 1:] = _bits(s["mask"], M)
    inside = row.clamp(0, M)
    position = torch.where(row < 0, place, cached + depth.gather(1, inside))
    visible = used[:, None] & ((row < 0)[:, None] | sees[:, :R].gather(2, inside[:, None].expand(n, R, -1)))
    if c["window"]:
        visible &= ((cached + depth[:, :R])[..., None] - position[:, None] < c["window"]) | (position < c["sinks"])[:, None]
    score = torch.einsum("nrhgd,nphd->nhgrp", q, k) * (1 / math.sqrt(D))
    score.masked_fill_(~visible[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp_(score.sub_(top))
    total = p.sum(-1, keepdim=True)
    out = torch.einsum("nhgrp,nphd->nrhgd", p.div_(total.clamp(min=1e-30)), v)
    return {"out": out.reshape(n, R, H * G, D)[req, local].to(s["q"].dtype)}


def _accept(s):
    if own:
        import paper_2411_04975_b200 as sfx
        out = sfx.sd_accept(s["logits"], s["offsets"], s["tokens"], s["parents"])
        return {k: out[k] for k in ("targets", "path", "offsets", "tokens")}
    n, M = s["tokens"].shape
    V = s["logits"].shape[1]
    dev = s["logits"].device
    x = s["logits"].float()
    lowest = torch.where(x == x.amax(1, keepdim=True), torch.arange(V, device=dev, dtype=torch.int32), V)
    targets = lowest.amin(1)
    wanted = targets[s["offsets"][:-1, None] + s["parents"] + 1]                     # at each node's parent
    node = torch.arange(M, device=dev) < (s["offsets"][1:] - s["offsets"][:-1] - 1)[:, None]
    match = node & (wanted == s["tokens"])
    taken = node & (match[:, None] | ~_bits(s["mask"], M)).all(-1)                    # with all of its ancestors
    count = taken.sum(1) + 1
    order = torch.where(taken, torch.arange(1, M + 1, device=dev), M + 1).sort(1).values
    path = torch.cat([torch.zeros(n, 1, dtype=torch.int64, device=dev), torch.where(order <= M, order, -1)], 1)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=dev), count.cumsum(0)])
    k = torch.arange(targets.shape[0], device=dev)
    req = (torch.searchsorted(offsets, k, right=True) - 1).clamp(max=n - 1)
    chosen = targets[s["offsets"][req] + path[req, (k - offsets[req]).clamp(max=M)].clamp(min=0)]
    tokens = torch.where(k < offsets[-1], chosen, -1)
    return {"targets": targets, "path": path.to(torch.int32), "offsets": offsets, "tokens": tokens}


def _commit(s):
    if own:
        import paper_2411_04975_b200 as sfx
        cached = sfx.sd_commit(s["k_cache"], s["v_cache"], s["table"], s["cached"], s["path"])
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "cached": cached}
    page = s["case"]["page"]
    n = s["path"].shape[0]
    j = torch.arange(s["max_rows"], device=s["path"].device)
    path = s["path"][:, :s["max_rows"]].long()
    last = s["table"].shape[1] * page - 1
    cached = s["cached"].long()[:, None]
    kept = path >= 0
    src, dst = (cached + path.clamp(min=0)).clamp(max=last), (cached + torch.where(kept, j, 0)).clamp(max=last)
    rows = torch.arange(n, device=path.device)[:, None]
    src_page, dst_page = s["table"][rows, src // page].long(), s["table"][rows, dst // page].long()
    for cache in (s["k_cache"], s["v_cache"]):                                       # (what is not kept writes row 0 over itself)
        cache[:, dst_page, dst % page] = cache[:, src_page, src % page]
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "cached": (s["cached"] + kept.sum(1)).to(torch.int32)}


# --------------------------------------------------------------------------- definition, 64 bits
def exact(case, seed):
    """The definition, request by request in 64 bits; None where outputs are moved or whole values only."""
    if case["kind"] not in ("rotate", "attend"):
        return None
    s = prepare(case, seed)
    begin, cached = s["offsets"].tolist(), s["cached"].tolist()
    mask = s["mask"].cpu().numpy().view("uint32")
    page, dev = case["page"], s["q"].device

    def ancestors(i, r):                                                             # rows that row r sees, itself among them
        words = [int(w) for w in mask[i, r - 1]] if r else []
        return [0] + [j + 1 for j in range(case["max_draft"]) if r and words[j // 32] >> (j % 32) & 1]

    def lines(i, first, last):
        p = torch.arange(first, last, device=dev)
        return s["table"][i].long()[p // page], p % page

    if case["kind"] == "attend":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device=dev)
        G = case["q_heads"] // case["kv_heads"]
        for i in range(case["n"]):
            R, t = begin[i + 1] - begin[i], cached[i]
            sets = [ancestors(i, r) for r in range(R)]
            see = torch.zeros(R, t + R, dtype=torch.bool)
            for r, a in enumerate(sets):
                at = t + len(a) - 1
                first = max(0, at - case["window"] + 1) if case["window"] else 0
                see[r, first:t] = True
                see[r, :min(t, case["sinks"])] = True
                for j in a:
                    see[r, t + j] = not case["window"] or at - (t + len(sets[j]) - 1) < case["window"] or t + len(sets[j]) - 1 < case["sinks"]
            pg, ln = lines(i, 0, t + R)
            k, v = s["k_cache"][pg, ln].double(), s["v_cache"][pg, ln].double()
            q = s["q"][begin[i]:begin[i + 1]].double()
            see = see.to(dev)[None]
            for h in range(case["kv_heads"]):
                x = torch.matmul(q[:, h * G:(h + 1) * G].transpose(0, 1), k[:, h].T) / math.sqrt(case["head"])
                w = torch.softmax(torch.where(see, x, -math.inf), -1)
                out[begin[i]:begin[i + 1], h * G:(h + 1) * G] = torch.matmul(w, v[:, h]).transpose(0, 1)
        return {"out": out}

    half = case["rot"] // 2

    def rotated(x, w, turn):
        x = x.double()
        if w is not None:
            x = w.double() * x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + 1e-6)
        r = x[..., :case["rot"]]
        z = torch.complex(r[..., 0::2], r[..., 1::2]) if case["interleaved"] else torch.complex(r[..., :half], r[..., half:])
        z = z * turn
        y = x.clone()
        if case["interleaved"]:
            y[..., 0:case["rot"]:2], y[..., 1:case["rot"]:2] = z.real, z.imag
        else:
            y[..., :half], y[..., half:case["rot"]] = z.real, z.imag
        return y

    q = torch.empty(s["q"].shape, dtype=torch.float64, device=dev)
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    for i in range(case["n"]):
        a, b, t = begin[i], begin[i + 1], cached[i]
        at = torch.tensor([t + len(ancestors(i, r)) - 1 for r in range(b - a)], dtype=torch.float64, device=dev) if s["positions"] is None else s["positions"][a:b].double()
        turn = torch.polar(torch.ones_like(at[:, None] * s["freq"]), at[:, None] * s["freq"])[:, None]
        q[a:b] = rotated(s["q"][a:b], s["weights"][0], turn)
        pg, ln = lines(i, t, t + b - a)
        k_cache[pg, ln] = rotated(s["k"][a:b], s["weights"][1], turn)
        v_cache[pg, ln] = s["v"][a:b].double()
    return {"q": q, "k_cache": k_cache, "v_cache": v_cache}
