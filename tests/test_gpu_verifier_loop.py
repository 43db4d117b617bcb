"""Drafts through the whole verifier, step after step: sd_speculate, sd_rotate and sd_attend per layer, sd_accept, sd_commit, and the accepted tokens back into the
trees, against the harness's acceptance and a cache filled from scratch."""
import numpy as np
import pytest
import torch

import paper_2411_04975_b200 as sfx
from workload.closed_loop import accept_longest_path
from workload.generator import get_workload
from workload.verifier import Verifier

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def store_of(w, n, room):
    c = w.cfg
    return sfx.SuffixStore(torch.as_tensor(w.corpus(), device=DEV), torch.as_tensor(w.corpus_offsets(), device=DEV), vocab=c.vocab, depth_cap=c.depth_cap,
                           max_requests=n, max_req_tokens=c.prompt_len + room, max_spec_cap=c.max_spec)


def lines(model, layer, slot, count):
    p = np.arange(count)
    page = model.table[slot].cpu().numpy()[p // model.k_cache.shape[2]].astype(np.int64)
    return [cache[layer].cpu()[page, p % cache.shape[2]] for cache in (model.k_cache, model.v_cache)]


def test_steps_of_a_batch():
    w = get_workload("tiny")
    c, n = w.cfg, 8
    prompts = [w.prompt(i) for i in range(n)]
    truth = [w.continuation(i, prompts[i], length=80) for i in range(n)]
    store = store_of(w, n, 200)
    off = np.concatenate([[0], np.cumsum([len(p) for p in prompts])])
    slots = torch.arange(n, dtype=torch.int32, device=DEV)
    store.build_requests(list(range(n)), off, torch.as_tensor(np.concatenate(prompts).astype(np.int32), device=DEV))
    model = Verifier(n, c.prompt_len + 200, c.max_spec, c.vocab, page=16)
    model.start(range(n), prompts)
    cursor, text = [0] * n, [list(p) for p in prompts]
    accepted = 0
    for _ in range(9):
        out = store.speculate(slots, c.max_pattern, c.alpha, c.max_spec)
        host = {k: out[k].cpu().numpy() for k in ("n_draft", "tokens", "parents")}
        follows = np.full((n, c.max_spec + 1), -1, dtype=np.int64)
        for i in range(n):
            t = truth[i][cursor[i]:][:c.max_spec + 1]
            follows[i, :len(t)] = t
        got = model.step(out, torch.tensor([t[-1] for t in text], device=DEV), torch.as_tensor(follows, device=DEV))
        store.append(slots, got["offsets"], got["tokens"])        # as they are, without the host
        begin, tokens = got["offsets"].tolist(), got["tokens"].tolist()
        for i in range(n):
            want = accept_longest_path(host["tokens"][i], host["parents"][i], int(host["n_draft"][i]), truth[i][cursor[i]:])
            new = tokens[begin[i]:begin[i + 1]]
            assert len(new) == want + 1 and new == truth[i][cursor[i]:cursor[i] + want + 1].tolist()
            accepted += want
            cursor[i] += want + 1
            text[i] += new
        assert model.cached.tolist() == [len(t) - 1 for t in text]
        assert store.slot_info(slots)["len"].tolist() == [len(t) for t in text]
        assert max(cursor) <= 80 - 1
        if max(cursor) > 50:
            break
    assert accepted > n                                           # drafts were taken, so lines have moved
    # the cache as if these texts had been prompts
    fresh = Verifier(n, c.prompt_len + 200, c.max_spec, c.vocab, page=16)
    fresh.start(range(n), [np.asarray(t) for t in text])
    for layer in range(model.layers):
        for i in range(n):
            for a, b in zip(lines(model, layer, i, len(text[i]) - 1), lines(fresh, layer, i, len(text[i]) - 1)):
                # the same sums of 256 bf16 products in another order, and in the second layer of two attentions' results, each rounded: some 2^-7 of a value
                assert (a.double() - b.double()).norm() < 2.0 ** -6 * b.double().norm()
    store.free()


def test_what_is_accepted_goes_to_the_next_step_as_it_is():
    """sd_accept's offsets and tokens as sd_step's arguments, on the device, with a slot that idles in every other step; beside a store that is given the known tokens."""
    w = get_workload("tiny")
    c, n = w.cfg, 6
    prompts = [w.prompt(i) for i in range(n)]
    truth = [w.continuation(i, prompts[i], length=120) for i in range(n)]
    off = np.concatenate([[0], np.cumsum([len(p) for p in prompts])])
    slots = torch.arange(n, dtype=torch.int32, device=DEV)
    stores = [store_of(w, n, 250) for _ in range(2)]
    for store in stores:
        store.build_requests(list(range(n)), off, torch.as_tensor(np.concatenate(prompts).astype(np.int32), device=DEV))
    args = (c.max_pattern, c.alpha, c.max_spec)
    out = stores[0].speculate(slots, *args)
    cursor, accepted = [0] * n, 0
    for turn in range(8):
        idle = turn % n if turn % 2 else -1
        drafts = out["n_draft"].cpu().numpy()
        counts = [0 if i == idle else 1 + int(drafts[i]) for i in range(n)]
        offsets = np.concatenate([[0], np.cumsum(counts)])
        tokens, parents = out["tokens"].cpu().numpy(), out["parents"].cpu().numpy()
        positions = out["positions"].cpu().numpy()
        logits = torch.randn(int(offsets[-1]) + 3, c.vocab, generator=torch.Generator().manual_seed(turn))
        for i in range(n):
            for r in range(counts[i]):                            # the model's choice at a row is the token that follows its position
                depth = 0 if r == 0 else int(positions[i, r - 1]) - (len(prompts[i]) + cursor[i]) + 1
                logits[int(offsets[i]) + r, int(truth[i][cursor[i] + depth])] = 50.0
        got = sfx.sd_accept(logits.cuda(), torch.as_tensor(offsets, device=DEV), out["tokens"], out["parents"])
        out = stores[0].step(slots, got["offsets"], got["tokens"], *args)
        known = []
        for i in range(n):
            many = 0 if i == idle else 1 + accept_longest_path(tokens[i], parents[i], int(drafts[i]), truth[i][cursor[i]:])
            known.append(truth[i][cursor[i]:cursor[i] + many])
            cursor[i] += many
            accepted += max(many - 1, 0)
        begin = np.concatenate([[0], np.cumsum([len(t) for t in known])])
        assert got["offsets"].tolist() == begin.tolist() and got["tokens"].tolist() == np.concatenate(known).tolist() + [-1] * (len(logits) - int(begin[-1]))
        stores[1].append(slots, torch.as_tensor(begin, device=DEV), torch.as_tensor(np.concatenate(known).astype(np.int32), device=DEV))
        want = stores[1].speculate(slots, *args)
        for name in ("n_draft", "tokens", "parents", "positions", "mask", "chosen_tree", "chosen_p", "score", "status"):
            assert torch.equal(out[name], want[name]), name
        if max(cursor) > 60:
            break
    assert accepted > n
    for store in stores:
        store.free()


def test_a_step_in_a_graph_with_idle_slots():
    """One captured step of the verifier's calls, replayed with other drafts; slots without rows and room behind the rows."""
    from verifier_ref import Batch, accept, attend, rotate
    bs = [Batch([100, 40, 7, 300], d, seed=s, group=2, M=16, head=64, extra_rows=e) for s, d, e in ((70, [9, -1, 0, 16], 3), (71, [2, 16, 3, -1], 6))]
    rows = max(b.rows for b in bs)
    rng = np.random.default_rng(70)
    i32 = dict(dtype=torch.int32, device=DEV)
    heads = bs[0].q.shape[1]
    width = max(b.table.shape[1] for b in bs)
    pages = max(b.pages for b in bs)
    held = {"q": torch.zeros(rows, heads, 64, dtype=torch.bfloat16, device=DEV), "k": torch.zeros(rows, 2, 64, dtype=torch.bfloat16, device=DEV), "v": torch.zeros(rows, 2, 64, dtype=torch.bfloat16, device=DEV),
            "table": torch.zeros(4, width, **i32), "offsets": torch.zeros(5, dtype=torch.int64, device=DEV), "cached": torch.zeros(4, **i32), "mask": torch.zeros(4, 16, 1, **i32),
            "tokens": torch.zeros(4, 16, **i32), "parents": torch.zeros(4, 16, **i32), "logits": torch.zeros(rows, 777, device=DEV)}
    k_cache, v_cache = (torch.zeros(pages, 16, 2, 64, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    freq = 100.0 ** (-torch.arange(32, dtype=torch.float64, device=DEV) / 32)
    result = {}

    def step():
        h = held
        q = sfx.sd_rotate(h["q"], h["k"], h["v"], k_cache, v_cache, h["table"], h["offsets"], h["cached"], freq, mask=h["mask"])
        result["q"], result["out"] = q, sfx.sd_attend(q, k_cache, v_cache, h["table"], h["offsets"], h["cached"], mask=h["mask"])
        result["accept"] = sfx.sd_accept(h["logits"], h["offsets"], h["tokens"], h["parents"])
        result["cached"] = sfx.sd_commit(k_cache, v_cache, h["table"], h["cached"], result["accept"]["path"])

    def load(b):
        tokens = rng.integers(0, 777, size=(4, 16)).astype(np.int32)
        logits = torch.randn(rows, 777, generator=torch.Generator().manual_seed(b.rows))
        for i, c in enumerate(b.counts):
            for r in range(c):
                kids = [j for j in range(c - 1) if b.parents[i, j] == r - 1]
                if kids:
                    logits[int(b.offsets[i]) + r, int(tokens[i, kids[0]])] = 50.0
        fill = lambda name, x: held[name][:x.shape[0]].copy_(torch.as_tensor(x))      # noqa: E731
        for name, x in (("q", b.q), ("k", b.k), ("v", b.v), ("offsets", b.offsets), ("cached", np.asarray(b.cached, dtype=np.int32)), ("mask", b.mask.view(np.int32)), ("tokens", tokens),
                        ("parents", b.parents), ("logits", logits)):
            fill(name, x)
        held["table"].zero_()
        held["table"][:, :b.table.shape[1]].copy_(torch.as_tensor(np.maximum(b.table, 0)))
        k_cache[:b.pages].copy_(b.k_cache)
        v_cache[:b.pages].copy_(b.v_cache)
        torch.cuda.synchronize()
        return tokens, logits

    load(bs[0])
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for b in bs + bs[:1]:
        tokens, logits = load(b)
        graph.replay()
        torch.cuda.synchronize()
        last = int(b.offsets[-1])
        q, k = rotate(b, freq.cpu())
        assert (result["q"][:last].cpu().double() - q[:last]).abs().max() < 0.05
        for i in range(4):                                        # the rows as the kernel wrote them, for the attention's own error
            lo, c = int(b.offsets[i]), b.counts[i]
            p = b.cached[i] + np.arange(c)
            b.k_cache[b.table[i][p // 16].astype(np.int64), p % 16] = k[lo:lo + c].to(torch.bfloat16)
            b.v_cache[b.table[i][p // 16].astype(np.int64), p % 16] = b.v[lo:lo + c]
        was, b.q = b.q, torch.cat([result["q"][:last].cpu(), b.q[last:]])
        out, _, size = attend(b)
        b.q = was
        assert ((result["out"][:last].cpu().double() - out[:last]).abs() <= 2.0 ** -6 * (size[:last] + out[:last].abs())).all()
        want = accept(logits.double(), b.offsets, tokens, b.parents)
        for name, x in zip(("targets", "path", "offsets", "tokens"), want):
            assert np.array_equal(result["accept"][name].cpu().numpy()[:len(x)], x), name
        assert result["cached"].tolist() == [c + int((p >= 0).sum()) for c, p in zip(b.cached, want[1])]
