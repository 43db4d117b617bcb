"""Plain 64-bit forms of the verifier's operators, request by request on the CPU, and batches to try them on."""
import math

import numpy as np
import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}     # half a step, relative


def random_tree(rng, m, chain=0.7):
    """Parents of m draft nodes: each a child of an earlier one or of the last token."""
    return [-1 if j == 0 else (j - 1 if rng.random() < chain else int(rng.integers(-1, j))) for j in range(m)]


def mask_of(parents, M):
    """Mask words of one request as sd_speculate writes them."""
    words = (M + 31) // 32
    out = np.zeros((M, words), dtype=np.uint32)
    for j, p in enumerate(parents):
        if p >= 0:
            out[j] = out[p]
        out[j, j // 32] |= np.uint32(1 << (j % 32))
    return out


class Batch:
    """Requests with `contexts[i]` places in the cache and a draft of `drafts[i]` nodes (-1: no rows at all)."""

    def __init__(self, contexts, drafts, *, kv_heads=2, group=2, head=64, dtype=torch.bfloat16, page=16, M=64, seed=0, shared=0, layout="nhd",
                 mask="tree", extra_rows=0, extra_pages=3, garbage=float("nan"), layers=0, pieces=False):
        rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        self.n, self.M, self.page, self.head, self.kv_heads, self.group, self.dtype = len(contexts), M, page, head, kv_heads, group, dtype
        counts = [d + 1 for d in drafts]
        self.counts, self.cached = counts, list(contexts)
        self.offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)
        self.rows = int(self.offsets[-1]) + extra_rows
        self.parents = np.full((self.n, M), -1, dtype=np.int32)
        self.mask = np.zeros((self.n, M, (M + 31) // 32), dtype=np.uint32)
        for i, d in enumerate(drafts):
            tree = [j - 1 for j in range(max(d, 0))] if mask is None else random_tree(rng, max(d, 0))
            self.parents[i, :len(tree)] = tree
            self.mask[i] = mask_of(tree, M)
        self.masked = mask is not None
        need = [-(-(c + k) // page) if k else 0 for c, k in zip(contexts, counts)]
        common = shared // page
        self.shared = shared
        if pieces:                                               # one page per request
            self.table = np.arange(self.n, dtype=np.int32)[:, None].copy()
            pages = self.n
        else:
            width = max(need + [1]) + 1
            order = rng.permutation(common + sum(max(p - common, 0) for p in need) + extra_pages).astype(np.int32)
            pages = len(order)
            self.table = np.full((self.n, width), -7, dtype=np.int32)
            at = common
            for i, p in enumerate(need):
                own = max(p - common, 0)
                self.table[i, :min(common, p)] = order[:min(common, p)]
                self.table[i, common:common + own] = order[at:at + own]
                at += own
        self.pages = pages
        shape = ((layers,) if layers else ()) + (pages, page, kv_heads, head)
        self.k_cache, self.v_cache = torch.randn(shape, generator=g).to(dtype), torch.randn(shape, generator=g).to(dtype)
        used = torch.zeros(pages, page, dtype=torch.bool)
        for i in range(self.n):
            if counts[i]:
                p = np.arange(contexts[i] + counts[i])
                used[self.table[i][p // page].astype(np.int64), p % page] = True
        if garbage is not None and not layers:
            self.k_cache[~used], self.v_cache[~used] = garbage, garbage
        self.used = used
        self.layout = layout
        heads = kv_heads * group
        self.q = (torch.randn(self.rows, heads, head, generator=g) * 1.5).to(dtype)
        self.k, self.v = torch.randn(self.rows, kv_heads, head, generator=g).to(dtype), torch.randn(self.rows, kv_heads, head, generator=g).to(dtype)

    # ---- on the device
    def device(self, t, dtype=None):
        t = torch.as_tensor(np.ascontiguousarray(t) if isinstance(t, np.ndarray) else t)
        return t.to("cuda:0") if dtype is None else t.to("cuda:0", dtype)

    def caches(self):
        """Both caches on the device, in the layout that the batch asks for: views of [pages, page_size, kv_heads, head_dim]."""
        k, v = self.k_cache.cuda(), self.v_cache.cuda()
        if self.layout == "hnd":                                 # heads outside of lines
            k, v = k.transpose(-3, -2).contiguous().transpose(-3, -2), v.transpose(-3, -2).contiguous().transpose(-3, -2)
        if self.layout == "both":                                # keys and values of a page in one piece
            kv = torch.stack([k, v], -4)
            k, v = kv.select(-4, 0), kv.select(-4, 1)
        if self.layout == "wide":                                # room between the heads' rows
            wide = torch.zeros(*k.shape[:-2], k.shape[-2] + 1, 2 * k.shape[-1], dtype=k.dtype, device=k.device)
            wide[..., :-1, :k.shape[-1]], wide[..., :-1, k.shape[-1]:] = k, v
            k, v = wide[..., :-1, :k.shape[-1]], wide[..., :-1, k.shape[-1]:]
        return k, v

    def args(self):
        return (self.device(self.table), self.device(self.offsets), self.device(np.asarray(self.cached, dtype=np.int32)))

    def mask_arg(self):
        return self.device(self.mask.view(np.int32)) if self.masked else None

    # ---- what it means
    def sees(self, i):
        """bool [count, count]: which rows of request i see which; and how deep each is."""
        c = self.counts[i]
        see = np.zeros((c, c), dtype=bool)
        see[:, 0] = True
        for r in range(1, c):
            for j in range(c - 1):
                see[r, j + 1] = bool(self.mask[i, r - 1, j // 32] >> np.uint32(j % 32) & 1) if self.masked else j + 1 <= r
        deep = np.array([0] + [bin(int.from_bytes(self.mask[i, r - 1].tobytes(), "little")).count("1") if self.masked else r for r in range(1, c)])
        return see, deep[:c]

    def visible(self, i, window=0, sinks=0):
        c, t = self.counts[i], self.cached[i]
        see, deep = self.sees(i)
        out = np.ones((c, t + c), dtype=bool)
        out[:, t:] = see
        position = np.concatenate([np.arange(t), t + deep])
        if window:
            out &= ((t + deep)[:, None] - position[None] < window) | (position < sinks)[None]
        return torch.from_numpy(out)

    def lines(self, i, cache, count=None):
        p = np.arange(self.cached[i] + self.counts[i] if count is None else count)
        return cache[self.table[i][p // self.page].astype(np.int64), p % self.page]


def attend(b, *, scale=None, window=0, sinks=0):
    """(out, lse, size): size[r, h, d] = sum of weight * |value|, which the roundings of the weights are relative to."""
    H, G, D = b.kv_heads, b.group, b.head
    scale = D ** -0.5 if scale is None else scale
    out = torch.full((b.rows, H * G, D), math.nan, dtype=torch.float64)
    size, lse = out.clone(), torch.full((b.rows, H * G), math.inf, dtype=torch.float64)    # (inf: a row of no request)
    for i in range(b.n):
        c = b.counts[i]
        if not c:
            continue
        lo = int(b.offsets[i])
        k, v, q = b.lines(i, b.k_cache).double(), b.lines(i, b.v_cache).double(), b.q[lo:lo + c].double()
        see = b.visible(i, window, sinks)
        for h in range(H * G):
            s = torch.where(see, q[:, h] @ torch.where(see.any(0)[:, None], k[:, h // G], 0.0).T * scale, -math.inf)
            top = s.amax(1, keepdim=True).clamp(min=-1e300)
            w = torch.where(see, torch.exp(s - top), 0.0)
            total = w.sum(1, keepdim=True)
            w = w / total.clamp(min=1e-300)
            for r in range(c):                                   # (over what the row sees and nothing else: 0 * NaN is NaN)
                at = see[r].nonzero()[:, 0]
                out[lo + r, h] = w[r, at] @ v[at, h // G]
                size[lo + r, h] = w[r, at] @ v[at, h // G].abs()
            lse[lo:lo + c, h] = (top + torch.log(total))[:, 0]
            lse[lo:lo + c][~see.any(1)] = -math.inf
    return out, lse, size


def rotate(b, freq, *, positions=None, q_weight=None, k_weight=None, eps=1e-6, interleaved=False, scale=1.0):
    """(q, k): the rows as they are in 64 bits."""
    rot = 2 * len(freq)
    at = torch.zeros(b.rows, dtype=torch.float64)
    for i in range(b.n):
        if b.counts[i]:
            _, deep = b.sees(i)
            at[int(b.offsets[i]):int(b.offsets[i + 1])] = torch.from_numpy(b.cached[i] + deep).double()
    if positions is not None:
        at = positions.double()
    angle = at[:, None] * freq.double()
    cos, sin = torch.cos(angle)[:, None] * scale, torch.sin(angle)[:, None] * scale

    def turned(x, w):
        x = x.double()
        if w is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
        y = x.clone()
        first, second = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
        y[..., first] = x[..., first] * cos - x[..., second] * sin
        y[..., second] = x[..., second] * cos + x[..., first] * sin
        return y
    return turned(b.q, q_weight), turned(b.k, k_weight)


def accept(logits, offsets, tokens, parents):
    """targets, path, offsets, tokens as sd_accept writes them; logits as float64."""
    rows, (n, M) = logits.shape[0], tokens.shape
    targets = []
    for r in logits:
        nan = torch.isnan(r)
        targets.append(int(nan.nonzero()[0]) if nan.any() else int((r == r.max()).nonzero()[0]))
    path = np.full((n, M + 1), -1, dtype=np.int32)
    begin, new = [0], []
    for i in range(n):
        lo, hi = int(offsets[i]), int(offsets[i + 1])
        row, kept = 0, 0
        while lo < hi:
            path[i, kept] = row
            new.append(targets[lo + row])
            kept += 1
            nxt = [j + 1 for j in range(hi - lo - 1) if parents[i, j] == row - 1 and tokens[i, j] == targets[lo + row] and j + 1 > row]
            if not nxt:
                break
            row = nxt[0]
        begin.append(len(new))
    return np.asarray(targets), path, np.asarray(begin), np.asarray(new + [-1] * (rows - len(new)))
