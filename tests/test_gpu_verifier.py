"""sd_rotate, sd_attend, sd_accept and sd_commit against plain 64-bit forms."""
import math

import numpy as np
import pytest
import torch

import paper_2411_04975_b200 as sfx
import verifier_ref as R

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16


# ------------------------------------------------------------------------------------- attention
def check_attend(b, *, scale=None, window=0, sinks=0, shared=0, caches=None, **kw):
    out, lse, size = R.attend(b, scale=scale, window=window, sinks=sinks)
    k, v = b.caches() if caches is None else caches
    got_lse = torch.full((b.rows, b.q.shape[1]), 5.0, device="cuda:0")
    q = b.q.cuda()
    got = torch.full_like(q, 7.0)
    status = torch.full((b.n,), 99, dtype=torch.int32, device="cuda:0")
    sfx.sd_attend(q, k, v, *b.args(), mask=b.mask_arg(), scale=scale, window=window, sinks=sinks, shared=shared, out=got, lse=got_lse, status=status, **kw)
    assert status.tolist() == [0] * b.n
    compare(b, got, got_lse, out, lse, size)
    return got, got_lse


def compare(b, got, got_lse, out, lse, size):
    """Half a step for the result, half a step of each weight (relative to the sum of weight * |value|), and 2^-14 of that for 32-bit
    scores (64 to 128 products of a few units each: 2^-17), exponentials (2^-20 for scores below 8) and sums (2^-17)."""
    half = R.HALF[b.dtype]
    got, got_lse = got.cpu().double(), got_lse.cpu().double()
    none = lse[:, 0] == math.inf                                  # rows of no request
    assert (got[none] == 7.0).all() and (got_lse[none] == 5.0).all()
    got, out, size, got_lse, lse = got[~none], out[~none], size[~none], got_lse[~none], lse[~none]
    fine = torch.isfinite(out)
    assert (torch.isfinite(got) == fine).all()
    err = (got - out).abs()
    tol = half * out.abs() + (half + 2.0 ** -14) * size + (2.0 ** -25 if b.dtype == FP16 else 0)
    bad = fine & ~(err <= tol * 1.01)                             # (1.01: the roundings' second order)
    assert not bad.any(), (bad.nonzero()[:5], got[bad][:5], out[bad][:5], int(bad.sum()))
    empty = torch.isinf(lse)
    assert (got_lse[empty] == -math.inf).all() and (torch.isnan(got_lse) == torch.isnan(lse)).all()
    known = torch.isfinite(lse)
    assert ((got_lse - lse)[known].abs() <= 2.0 ** -14).all()


BATCHES = {
    "one_token": ([0], [0]), "first_places": ([1, 2, 3], [0, 1, 2]), "a_page": ([16, 15, 17], [0, 0, 0]), "tile_edges": ([126, 127, 128, 129, 0], [0, 1, 0, 3, 64]),
    "idle_slots": ([5, 40, 7, 300], [-1, 3, -1, -1]), "full_drafts": ([200, 64, 1], [64, 63, 64]), "ragged": ([0, 700, 31, 1290, 256, 5], [5, 33, 0, 31, 32, 17]),
    "long_and_short": ([5000, 3, 12], [9, 2, 0]),
}


@pytest.mark.parametrize("name", BATCHES)
@pytest.mark.parametrize("head,dtype,kv_heads,group,page", [(64, BF16, 2, 2, 16), (128, BF16, 2, 4, 64), (128, FP16, 1, 1, 8), (64, FP16, 3, 5, 32), (128, BF16, 1, 8, 128)])
def test_attend(name, head, dtype, kv_heads, group, page):
    contexts, drafts = BATCHES[name]
    check_attend(R.Batch(contexts, drafts, head=head, dtype=dtype, kv_heads=kv_heads, group=group, page=page, seed=3, extra_rows=2))


@pytest.mark.parametrize("layout", ["nhd", "hnd", "both", "wide"])
@pytest.mark.parametrize("page", [8, 32, 256, 384])
def test_attend_layouts(layout, page):
    check_attend(R.Batch([300, 77, 512], [12, 0, 20], head=128, page=page, layout=layout, seed=4))


@pytest.mark.parametrize("piece", [1, 50, 200, 1000])
def test_attend_one_piece_per_request(piece):
    """A page is a whole request, of any length."""
    contexts = [min(c, piece - 1) for c in (0, 30, 180, 975)]
    check_attend(R.Batch(contexts, [min(7, piece - 1 - c) for c in contexts], page=piece, pieces=True, seed=5, head=128))


def test_attend_without_mask_and_short_masks():
    check_attend(R.Batch([30, 400], [64, 10], mask=None, seed=6))
    for M in (1, 5, 31, 32, 33, 63):
        check_attend(R.Batch([30, 400], [M, M // 2], M=M, seed=7))


def test_attend_strided_rows():
    """Queries as a view of a projection's output, results into a view too."""
    b = R.Batch([200, 31], [6, 9], kv_heads=2, group=3, head=128, seed=8)
    out, lse, size = R.attend(b)
    wide = torch.zeros(b.rows, 10, 128, dtype=b.dtype, device="cuda:0")
    wide[:, :6] = b.q.cuda()
    to = torch.zeros(b.rows, 2, 6, 128, dtype=b.dtype, device="cuda:0")
    got_lse = torch.empty(b.rows, 6, device="cuda:0")
    k, v = b.caches()
    sfx.sd_attend(wide[:, :6], k, v, *b.args(), mask=b.mask_arg(), out=to[:, 1], lse=got_lse)
    compare(b, to[:, 1], got_lse, out, lse, size)
    assert (to[:, 0] == 0).all() and (wide[:, 6:] == 0).all()
    sfx.sd_attend(wide[:, :6], k, v, *b.args(), mask=b.mask_arg(), out=wide[:, :6], lse=got_lse)      # in place
    compare(b, wide[:, :6], got_lse, out, lse, size)


@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 0), (64, 4), (100, 1), (128, 37), (129, 128), (300, 130), (1000, 4), (100000, 3), (2, 100000)])
@pytest.mark.parametrize("head", [64, 128])
def test_attend_window(window, sinks, head):
    check_attend(R.Batch([0, 3, 127, 640, 900, 2000], [5, 0, 20, 64, 3, 11], head=head, seed=9), window=window, sinks=sinks)


@pytest.mark.parametrize("shared", [1, 16, 100, 128, 256, 500])
@pytest.mark.parametrize("head,group", [(128, 4), (64, 1), (128, 1)])
def test_attend_shared_prefix(shared, head, group):
    contexts, drafts = [shared, shared + 1, shared + 300, shared + 90, shared + 128, 3], [0, 40, 3, 0, 64, -1]
    b = R.Batch(contexts, drafts, head=head, group=group, page=16, shared=shared, seed=10, extra_rows=3)
    check_attend(b, shared=shared)
    check_attend(b, shared=shared, window=70, sinks=5)
    check_attend(b, shared=shared // 2)


def test_attend_many_requests():
    rng = np.random.default_rng(11)
    n = 700
    check_attend(R.Batch(rng.integers(0, 80, n).tolist(), rng.integers(-1, 4, n).tolist(), head=64, group=1, seed=11))


@pytest.mark.parametrize("n", [2048, 2049, 2100, 4200])
@pytest.mark.parametrize("shared,kw", [(0, {}), (128, dict(shared=128)), (0, dict(window=40, sinks=2))], ids=str)
def test_attend_requests_by_more_than_32(n, shared, kw):
    """Beyond 2,048 requests the pieces that the list is added up in have more than 32 requests each."""
    rng = np.random.default_rng(1100 + n)
    check_attend(R.Batch((shared + rng.integers(0, 40, n)).tolist(), rng.integers(-1, 3, n).tolist(), M=3, head=64, kv_heads=1, group=1, shared=shared, seed=n), **kw)


def test_attend_empty_rows():
    """A draft node that does not see itself, whose ancestors and the last token are outside its window: nothing is left."""
    b = R.Batch([40, 300], [6, 6], seed=12)
    b.mask[0, 4] = 0b00111                                        # three nodes at other depths: position 43, none of them is there
    b.mask[0, 0], b.mask[0, 1], b.mask[0, 2] = 1, 2, 4
    out, lse, _ = R.attend(b, window=1)
    assert torch.isinf(lse[5]).all() and (out[5] == 0).all()
    check_attend(b, window=1)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_attend_what_is_not_seen_has_no_part(bad):
    """Values and keys that are no numbers, at places that some rows see and others do not."""
    b = R.Batch([140, 20, 600], [20, 9, 30], head=128, group=2, seed=13)
    for i, j in ((0, 4), (1, 2), (2, 25)):                        # draft node j: its row of the cache
        p = b.cached[i] + j + 1
        for cache in (b.v_cache, b.k_cache):
            cache[b.table[i][p // 16], p % 16, 0, ::3] = bad
    out, _, _ = R.attend(b)
    assert not torch.isfinite(out).all() and torch.isfinite(out).any()
    k, v = b.caches()
    got = sfx.sd_attend(b.q.cuda(), k, v, *b.args(), mask=b.mask_arg()).cpu().double()
    clean = torch.isfinite(out).all(-1)
    assert (torch.isfinite(got).all(-1) == clean).all()
    assert (got - out)[clean].abs().max() < 0.05
    # values alone: rows that see them have them where they are, and numbers elsewhere
    b = R.Batch([140, 20], [20, 9], head=128, group=2, seed=14)
    p = b.cached[0] + 3
    b.v_cache[b.table[0][p // 16], p % 16, 0, 5] = bad
    check_attend(b)
    # at the edge of a window
    b = R.Batch([700, 20], [20, 9], head=64, group=2, seed=15)
    for p in (700 - 100, 700 - 97, 2, 5):
        b.v_cache[b.table[0][p // 16], p % 16, 1, 7] = bad
    check_attend(b, window=100, sinks=3)


def test_attend_scores_of_any_size():
    b = R.Batch([300], [3], head=64, seed=16)
    check_attend(b, scale=0.0)
    check_attend(b, scale=-0.1)
    b.q *= 30
    out, lse, _ = R.attend(b)
    k, v = b.caches()
    got_lse = torch.empty(b.rows, 4, device="cuda:0")
    got = sfx.sd_attend(b.q.cuda(), k, v, *b.args(), mask=b.mask_arg(), lse=got_lse)
    assert torch.isfinite(got).all() and (got_lse.cpu().double() - lse).abs().max() < 2.0 ** -10      # (scores of some hundreds: 2^-23 of each)


def test_attend_bad_numbers_are_told_and_left_out():
    b = R.Batch([100, 50, 20, 30], [4, 3, 2, 5], seed=17)
    out, lse, size = R.attend(b)
    k, v = b.caches()
    table, offsets, cached = b.args()
    def run(table, offsets, cached, **kw):
        status = torch.full((4,), 99, dtype=torch.int32, device="cuda:0")
        got, got_lse = torch.full_like(b.q, 7.0, device="cuda:0"), torch.full((b.rows, 4), 5.0, device="cuda:0")
        sfx.sd_attend(b.q.cuda(), k, v, table, offsets, cached, mask=b.mask_arg(), out=got, lse=got_lse, status=status, **kw)
        torch.cuda.synchronize()
        return status.tolist(), got, got_lse
    for entry, value in ((0, -1), (2, b.pages), (2, 2 ** 31 - 1)):
        t = table.clone()
        t[1, entry] = value
        st, got, got_lse = run(t, offsets, cached)
        assert st == [0, 32, 0, 0]
        keep = [r for r in range(b.rows) if not b.offsets[1] <= r < b.offsets[2]]
        o = out.clone()
        part = R.Batch([1], [0])
        part.dtype = b.dtype
        compare(part, got[keep], got_lse[keep], o[keep], lse[keep], size[keep])
    for value in (-1, 2 ** 31 - 1, b.page * table.shape[1]):
        c = cached.clone()
        c[2] = value
        st, got, _ = run(table, offsets, c)
        assert st == [0, 0, 16, 0] and (got[b.offsets[2]:b.offsets[3]] == 7.0).all()
    o = offsets.clone()
    o[1] = 2 ** 40
    st, got, _ = run(table, o, cached)
    assert st[:2] == [16, 16] and (got[:b.offsets[2]] == 7.0).all()
    st, got, _ = run(table, offsets, cached, shared=31)
    assert st == [0, 0, 16, 16]


def test_attend_in_a_cache_past_32_bits():
    """Lines more than 2^31 elements, and more than 2^32 bytes, away from the first."""
    pages, page, H, D = (1 << 31) // (64 * 128) + 600, 64, 1, 128
    k, v = (torch.empty(pages, page, H, D, dtype=BF16, device="cuda:0") for _ in range(2))
    b = R.Batch([400, 90], [10, 3], kv_heads=H, head=D, page=page, seed=18)
    where = torch.arange(pages - b.pages, pages)
    where[::2] = torch.arange(len(where[::2])) * 3
    k[where.cuda()], v[where.cuda()] = b.k_cache.cuda(), b.v_cache.cuda()
    out, lse, size = R.attend(b)
    table = torch.where(torch.from_numpy(b.table) >= 0, where[torch.from_numpy(b.table).clamp(min=0).long()], -1).to(torch.int32).cuda()
    got_lse = torch.empty(b.rows, 2, device="cuda:0")
    got = sfx.sd_attend(b.q.cuda(), k, v, table, *b.args()[1:], mask=b.mask_arg(), lse=got_lse)
    compare(b, got, got_lse, out, lse, size)


def test_attend_streams_and_graphs():
    """Two calls at once on streams of their own, and two captured graphs replayed together with other inputs."""
    bs = [R.Batch([900, 40, 2000], [20, 3, 9], head=128, group=4, seed=s) for s in (19, 20)]
    want = [R.attend(b) for b in bs]
    streams = [torch.cuda.Stream() for _ in bs]
    held = [(b.q.cuda(), *b.caches(), *b.args(), b.mask_arg()) for b in bs]
    torch.cuda.synchronize()

    def call(a, out, lse):
        sfx.sd_attend(*a[:6], mask=a[6], out=out, lse=lse)

    outs = [(torch.empty_like(a[0]), torch.empty(a[0].shape[:2], device="cuda:0")) for a in held]
    for _ in range(20):
        for st, a, (o, l) in zip(streams, held, outs):
            with torch.cuda.stream(st):
                call(a, o, l)
    torch.cuda.synchronize()
    for b, (o, l), w in zip(bs, outs, want):
        compare(b, o, l, *w)
    graphs = []
    for a, (o, l) in zip(held, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(a, o, l)
        graphs.append(g)
        o.zero_()
    for a in held:                                                # other queries, other lengths
        a[0].copy_(a[0].flip(0))
        a[5].copy_(torch.tensor([800, 41, 1990], dtype=torch.int32))
    for b in bs:
        b.q = b.q.flip(0)
        b.cached = [800, 41, 1990]
    torch.cuda.synchronize()
    for _ in range(10):
        for st, g in zip(streams, graphs):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for b, (o, l) in zip(bs, outs):
        compare(b, o, l, *R.attend(b))


def test_attend_repeats_bit_for_bit():
    b = R.Batch([3000, 40, 800, 0], [20, 3, 64, 9], head=128, group=4, seed=21)
    k, v = b.caches()
    a = (b.q.cuda(), k, v, *b.args())
    first = sfx.sd_attend(*a, mask=b.mask_arg())
    for _ in range(5):
        assert torch.equal(first, sfx.sd_attend(*a, mask=b.mask_arg()))


@pytest.mark.parametrize("head,kv_heads,group", [(128, 8, 4), (64, 8, 2), (128, 2, 32)])
def test_attend_long_lists_under_load(head, kv_heads, group):
    """Units of one and of two tiles of rows, with few and with many tiles, in turns, when every multiprocessor fetches: copies land in any order, and groups overtake one another."""
    for seed in range(3):
        rng = np.random.default_rng(900 + seed)
        n = 64
        b = R.Batch(rng.integers(100, 4000, n).tolist(), rng.integers(0, 65, n).tolist(), head=head, kv_heads=kv_heads, group=group, page=64, seed=900 + seed)
        k, v = b.caches()
        a = (b.q.cuda(), k, v, *b.args())
        status = torch.empty(n, dtype=torch.int32, device="cuda:0")
        first = check_attend(b, caches=(k, v))[0] if seed == 0 else sfx.sd_attend(*a, mask=b.mask_arg())
        for _ in range(200):
            again = sfx.sd_attend(*a, mask=b.mask_arg(), status=status)
            assert torch.equal(first, again) and not status.any()


def test_attend_fuzz():
    rng = np.random.default_rng(22)
    for s in range(60):
        n = int(rng.integers(1, 9))
        M = int(rng.choice([1, 7, 32, 64]))
        shared = int(rng.choice([0, 0, 0, 40, 300]))
        ctx = (shared + rng.integers(0, int(rng.choice([3, 200, 3000])), n)).tolist()
        b = R.Batch(ctx, rng.integers(-1, M + 1, n).tolist(), M=M, kv_heads=int(rng.choice([1, 2, 5])), group=int(rng.choice([1, 2, 3, 7, 8])),
                    head=int(rng.choice([64, 128])), dtype=[BF16, FP16][s % 2], page=int(rng.choice([8, 16, 64, 128, 256])), seed=100 + s, shared=shared,
                    layout=str(rng.choice(["nhd", "hnd", "both", "wide"])), mask=None if s % 7 == 0 else "tree")
        window = int(rng.choice([0, 0, 1, 30, 200]))
        check_attend(b, window=window, sinks=int(rng.choice([0, 4, 150])) if window else 0, shared=shared)


# -------------------------------------------------------------------------------------- rotation
def check_rotate(b, rot, *, base=10000.0, given=None, norm="qk", fused=False, in_place=False, **kw):
    freq = base ** (-torch.arange(rot // 2, dtype=torch.float64) / max(rot // 2, 1))
    g = torch.Generator().manual_seed(1)
    qw, kw_ = ((1 + 0.3 * torch.randn(b.head, generator=g)).to(b.dtype) if x in norm else None for x in "qk")
    q, k = R.rotate(b, freq, positions=given, q_weight=qw, k_weight=kw_, **kw)
    heads = b.q.shape[1]
    if fused:
        qkv = torch.cat([b.q, b.k, b.v], 1).cuda()
        dq, dk, dv = qkv[:, :heads], qkv[:, heads:heads + b.kv_heads], qkv[:, heads + b.kv_heads:]
    else:
        dq, dk, dv = b.q.cuda(), b.k.cuda(), b.v.cuda()
    kc, vc = b.caches()
    before_k, before_v = kc.clone(), vc.clone()
    out = dq if in_place else torch.full((b.rows, heads, b.head), 7.0, dtype=b.dtype, device="cuda:0")
    untouched = out.clone()
    status = torch.full((b.n,), 99, dtype=torch.int32, device="cuda:0")
    sfx.sd_rotate(dq, dk, dv, kc, vc, *b.args(), freq.cuda(), mask=b.mask_arg(), positions=None if given is None else given.cuda(),
                  q_weight=None if qw is None else qw.cuda(), k_weight=None if kw_ is None else kw_.cuda(), out=out, status=status, **kw)
    assert status.tolist() == [0] * b.n
    # half a step, and 32-bit arithmetic: the norm's factor (some 2^-21), cosine and sine of an angle off by 2^-22, two products
    half, scale = R.HALF[b.dtype], kw.get("scale", 1.0)

    def near(got, want, x, w):
        x = x.double()
        if w is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + kw.get("eps", 1e-6)) * w.double()
        tol = half * want.abs() + 2.0 ** -19 * abs(scale) * x.abs().amax(-1, keepdim=True) + 2.0 ** -19 * x.abs() + 2.0 ** -25
        bad = ~((got.cpu().double() - want).abs() <= tol)
        assert not bad.any(), (bad.nonzero()[:4], got.cpu()[bad][:4], want[bad][:4])
    last = int(b.offsets[-1])
    near(out[:last], q[:last], b.q[:last], qw)
    assert torch.equal(out[last:], untouched[last:])
    touched = torch.zeros(b.pages, b.page, dtype=torch.bool)
    for i in range(b.n):
        lo, c = int(b.offsets[i]), b.counts[i]
        p = b.cached[i] + np.arange(c)
        pg = b.table[i][p // b.page].astype(np.int64)
        touched[pg, p % b.page] = True
        near(kc.cpu()[pg, p % b.page], k[lo:lo + c], b.k[lo:lo + c], kw_)
        assert torch.equal(vc.cpu()[pg, p % b.page], b.v[lo:lo + c])
    same = lambda x, y: torch.equal(x.nan_to_num(3.0), y.nan_to_num(3.0))   # noqa: E731
    assert same(kc.cpu()[~touched], before_k.cpu()[~touched]) and same(vc.cpu()[~touched], before_v.cpu()[~touched])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("head,rot,dtype", [(64, 64, BF16), (64, 32, FP16), (64, 16, BF16), (64, 0, FP16), (128, 128, BF16), (128, 64, FP16), (128, 48, BF16), (128, 112, BF16)])
def test_rotate(head, rot, dtype, interleaved):
    b = R.Batch([0, 700, 31, 129], [5, 33, -1, 64], head=head, dtype=dtype, group=3, seed=30, extra_rows=3)
    for norm in ("qk", "", "q", "k"):
        check_rotate(b, rot, norm=norm, interleaved=interleaved, fused=norm == "q", in_place=norm in ("qk", "q"))


@pytest.mark.parametrize("kv_heads,group", [(1, 1), (1, 3), (2, 16), (10, 7), (16, 1), (8, 8)])
@pytest.mark.parametrize("head", [64, 128])
def test_rotate_heads(kv_heads, group, head):
    check_rotate(R.Batch([5, 0], [2, 0], head=head, kv_heads=kv_heads, group=group, seed=31, page=8), head)


@pytest.mark.parametrize("layout", ["nhd", "hnd", "both", "wide"])
def test_rotate_layouts(layout):
    check_rotate(R.Batch([300, 77, 512], [12, 0, 20], head=128, page=32, layout=layout, seed=32), 128, fused=True)


def test_rotate_positions_far_out_and_scaled():
    b = R.Batch([100000, 7], [20, 64], head=128, page=256, seed=33)
    check_rotate(b, 128, base=500000.0)
    far = torch.randint(0, 2 ** 31 - 1, (b.rows,), dtype=torch.int32)
    check_rotate(b, 128, base=500000.0, given=far, scale=1.37)
    check_rotate(b, 64, given=-far, interleaved=True, scale=-0.5, eps=0.1)
    check_rotate(R.Batch([30, 400], [64, 10], mask=None, seed=34), 64)


def test_rotate_many_requests():
    rng = np.random.default_rng(35)
    n = 1500
    check_rotate(R.Batch(rng.integers(0, 40, n).tolist(), rng.integers(-1, 3, n).tolist(), head=64, group=1, seed=35), 64)


def test_rotate_bad_numbers_are_told_and_left_out():
    b = R.Batch([100, 50, 20], [4, 30, 2], seed=36)
    table, offsets, cached = b.args()
    freq = torch.zeros(32, dtype=torch.float64, device="cuda:0")
    def run(table, offsets, cached):
        k, v = b.caches()
        k[:], v[:] = 3.0, 3.0
        status = torch.full((3,), 99, dtype=torch.int32, device="cuda:0")
        out = sfx.sd_rotate(b.q.cuda(), b.k.cuda(), b.v.cuda(), k, v, table, offsets, cached, freq, mask=b.mask_arg(), status=status, out=torch.full_like(b.q, 7.0, device="cuda:0"))
        torch.cuda.synchronize()
        return status.tolist(), out.cpu(), (k != 3.0).flatten(2).any(-1).sum().item()
    assert run(table, offsets, cached)[2] == 39
    t = table.clone()
    t[1, 4] = b.pages                                             # places 64 .. 79 of the second request's 50 .. 80
    st, out, lines = run(t, offsets, cached)
    assert st == [0, 32, 0] and lines == 39 - 16 and torch.equal(out, b.q)
    c = cached.clone()
    c[0] = 16 * table.shape[1] - 4                                # five rows, four places
    st, out, lines = run(table, offsets, c)
    assert st == [16, 0, 0] and lines == 34 and (out[:5] == 7.0).all() and torch.equal(out[5:], b.q[5:])
    o = offsets.clone()
    o[1] = -3
    st, out, _ = run(table, o, cached)
    assert st[:2] == [16, 16] and (out[:36] == 7.0).all()


def test_rotary_frequencies():
    freq, scale = sfx.rotary_frequencies(128, 500000.0)
    want = 500000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)
    assert scale == 1.0 and freq.is_cuda and (freq.cpu() - want).abs().max() < 1e-15
    freq, scale = sfx.rotary_frequencies(128, 500000.0, factor=4.0)
    assert scale == 1.0 and (freq.cpu() * 4 - want).abs().max() < 1e-15
    freq, scale = sfx.rotary_frequencies(128, 500000.0, factor=4.0, original=8192)
    part = freq.cpu() / want
    turns = 8192 * want / (2 * math.pi)
    assert abs(scale - (1 + 0.1 * math.log(4.0))) < 1e-12 and (part[turns > 33 * 1.3] > 0.999).all() and ((part[turns < 0.8] - 0.25).abs() < 1e-9).all()
    assert (part[1:] <= part[:-1] + 1e-12).all()


# ------------------------------------------------------------------------------------ acceptance
def check_accept(logits, offsets, tokens, parents):
    want = R.accept(logits.double().cpu(), offsets, tokens, parents)
    dev = lambda a, dt: torch.as_tensor(np.ascontiguousarray(a), dtype=dt, device="cuda:0")    # noqa: E731
    status = torch.full((len(tokens),), 99, dtype=torch.int32, device="cuda:0")
    got = sfx.sd_accept(logits, dev(offsets, torch.int64), dev(tokens, torch.int32), dev(parents, torch.int32), status=status)
    assert status.tolist() == [0] * len(tokens)
    for name, w in zip(("targets", "path", "offsets", "tokens"), want):
        assert np.array_equal(got[name].cpu().numpy(), w), name
    return want


def drafts(b, vocab, rng):
    """Tokens of a batch's drafts and logits that follow some of them."""
    tokens = np.full((b.n, b.M), -1, dtype=np.int32)
    for i, c in enumerate(b.counts):
        tokens[i, :max(c - 1, 0)] = (rng.integers(0, vocab) + np.arange(max(c - 1, 0))) % vocab
    want = {}
    for i, c in enumerate(b.counts):
        for r in range(c):
            kids = [j for j in range(c - 1) if b.parents[i, j] == r - 1]
            if kids and rng.random() < 0.8:
                want[int(b.offsets[i]) + r] = int(tokens[i, rng.choice(kids)])
    return tokens, want


@pytest.mark.parametrize("dtype", [BF16, FP16, torch.float32])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 1000, 4095, 5003, 32000, 128256])
def test_accept(dtype, vocab):
    rng = np.random.default_rng(vocab)
    b = R.Batch([0] * 7, [0, 64, 5, -1, 33, 32, 17], seed=40, extra_rows=2)
    tokens, want = drafts(b, vocab, rng)
    logits = torch.randn(b.rows, vocab, generator=torch.Generator().manual_seed(vocab)).to(dtype)
    for r, t in want.items():
        logits[r, t] = 30.0
    w = check_accept(logits.cuda(), b.offsets, tokens, b.parents)
    if vocab > 100:
        assert w[2][-1] > len(w[2]) + 2                           # some drafts were accepted
    wide = torch.full((b.rows, vocab + 13), 99.0, dtype=dtype, device="cuda:0")   # rows that start anywhere
    wide[:, 5:5 + vocab] = logits.cuda()
    check_accept(wide[:, 5:5 + vocab], b.offsets, tokens, b.parents)


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
def test_accept_ties_and_no_numbers(dtype):
    vocab = 5003
    x = torch.zeros(12, vocab, dtype=dtype)
    x[0] = -math.inf
    x[1, 4000:] = -0.0
    x[1, :4000] = -1.0
    x[2, ::2] = -0.0                                              # zeros of both signs are equal
    x[3, 777], x[3, 4444], x[3, 10] = math.nan, math.nan, math.inf
    x[4, 5002], x[4, 4097] = 1.0, 1.0
    x[5, 1] = math.inf
    x[6] = -3.0
    x[6, 5001] = -2.0
    x[7, 4999] = -math.nan
    x[8] = math.nan
    x[9] = torch.finfo(dtype).min
    x[10] = -math.inf
    x[10, 33] = torch.finfo(dtype).min
    offsets, tokens = np.array([0, 12]), np.arange(16, dtype=np.int32)[None]
    w = check_accept(x.cuda(), offsets, tokens, np.full((1, 16), -1))
    assert w[0].tolist() == [0, 4000, 0, 777, 4097, 1, 5001, 4999, 0, 0, 33, 0]


def test_accept_batches():
    rng = np.random.default_rng(41)
    for n, M in ((1, 1), (3, 64), (33, 5), (1025, 3), (2100, 2)):
        b = R.Batch([0] * n, rng.integers(-1, M + 1, n).tolist(), M=M, seed=n, extra_rows=int(rng.integers(0, 3)), head=64)
        tokens, want = drafts(b, 50, rng)
        logits = torch.randn(b.rows, 50, generator=torch.Generator().manual_seed(n))
        for r, t in want.items():
            logits[r, t] = 30.0
        check_accept(logits.cuda(), b.offsets, tokens, b.parents)
    empty = torch.zeros(0, 50, device="cuda:0")
    check_accept(empty, np.array([0, 0, 0]), np.zeros((2, 4), dtype=np.int32), np.full((2, 4), -1))
    check_accept(torch.randn(2, 9, device="cuda:0"), np.array([0, 1, 2]), np.zeros((2, 0), dtype=np.int32), np.zeros((2, 0), dtype=np.int32))
    check_accept(empty, np.array([0]), np.zeros((0, 4), dtype=np.int32), np.zeros((0, 4), dtype=np.int32))


@pytest.mark.parametrize("n", [15, 16, 17, 18, 23, 31, 32, 33, 64])
def test_accept_batches_of_a_few_clusters(n):
    """From 17 requests on the paths are walked by a cluster of eight blocks, of which the last may have none; few rows of a large vocabulary are a cluster each, too."""
    rng = np.random.default_rng(4100 + n)
    b = R.Batch([0] * n, rng.integers(-1, 3, n).tolist(), M=3, seed=4100 + n, extra_rows=1, head=64)
    tokens, want = drafts(b, 70000, rng)
    logits = torch.randn(b.rows, 70000, generator=torch.Generator().manual_seed(n)).to(BF16)
    for r, t in want.items():
        logits[r, t] = 30.0
    for _ in range(20):
        check_accept(logits.cuda(), b.offsets, tokens, b.parents)


def test_accept_equal_siblings_and_bad_numbers():
    logits = torch.zeros(6, 20, device="cuda:0")
    logits[:, 3] = 1.0
    check_accept(logits, np.array([0, 6]), np.array([[3, 3, 3, 3, 3]]), np.array([[-1, -1, 1, 0, 3]]))
    i32, i64 = dict(dtype=torch.int32, device="cuda:0"), dict(dtype=torch.int64, device="cuda:0")
    tokens, parents = torch.full((3, 4), 3, **i32), torch.tensor([[-1, 0, 5, 7], [3, 3, 2, 1], [-1, 0, 1, 2]], **i32)   # parents that are none
    for offsets, st in (([0, 2, 4, 6], [0, 0, 0]), ([0, 2, 1, 6], [0, 16, 0]), ([-1, 2, 4, 60], [16, 0, 16]), ([0, 6, 6, 6], [16, 0, 0])):
        status = torch.full((3,), 99, **i32)
        out = sfx.sd_accept(logits, torch.tensor(offsets, **i64), tokens, parents, status=status)
        torch.cuda.synchronize()
        assert status.tolist() == st
        for i in range(3):
            kept = int(out["offsets"][i + 1] - out["offsets"][i])
            assert kept == int((out["path"][i] >= 0).sum()) and (kept == 0) == (st[i] != 0 or offsets[i + 1] == offsets[i])


# ---------------------------------------------------------------------------------------- commit
def check_commit(b, paths, in_place=False):
    k, v = b.caches()
    want_k, want_v = k.cpu().clone(), v.cpu().clone()
    path = np.full((b.n, b.M + 1), -1, dtype=np.int32)
    for i, p in enumerate(paths):
        path[i, :len(p)] = p
        at = lambda x: (b.table[i][np.asarray(x, dtype=np.int64) // b.page].astype(np.int64), np.asarray(x, dtype=np.int64) % b.page)   # noqa: E731
        if len(p):
            (sp, sl), (dp, dl) = at(b.cached[i] + np.asarray(p)), at(b.cached[i] + np.arange(len(p)))
            for cache, src in ((want_k, k.cpu()), (want_v, v.cpu())):
                cache[..., dp, dl, :, :] = src[..., sp, sl, :, :]
    cached = torch.tensor(b.cached, dtype=torch.int32, device="cuda:0")
    status = torch.full((b.n,), 99, dtype=torch.int32, device="cuda:0")
    out = sfx.sd_commit(k, v, torch.as_tensor(b.table, device="cuda:0"), cached, torch.as_tensor(path, device="cuda:0"), status=status, out=cached if in_place else None)
    assert status.tolist() == [0] * b.n
    assert out.tolist() == [c + len(p) for c, p in zip(b.cached, paths)]
    assert torch.equal(k.cpu().nan_to_num(3.0), want_k.nan_to_num(3.0)) and torch.equal(v.cpu().nan_to_num(3.0), want_v.nan_to_num(3.0))


@pytest.mark.parametrize("layout", ["nhd", "hnd", "both", "wide"])
@pytest.mark.parametrize("layers,head,kv_heads,page", [(0, 64, 2, 16), (3, 128, 8, 16), (1, 128, 1, 8), (5, 64, 20, 64)])
def test_commit(layout, layers, head, kv_heads, page):
    rng = np.random.default_rng(50)
    counts = [0, 64, 64, 5, -1, 33, 17, 40]
    b = R.Batch([0, 700, 31, 129, 9, 16, 15, 1], counts, head=head, kv_heads=kv_heads, page=page, layout=layout, layers=layers, seed=50)
    paths = [[0], list(range(65)), [0] + sorted(rng.choice(np.arange(1, 65), 30, replace=False).tolist()), [0, 5], [], [0, 1, 2, 9, 33], [0], [0] + list(range(24, 41))]
    check_commit(b, paths)
    check_commit(b, paths, in_place=True)


def test_commit_short_paths_and_bad_numbers():
    b = R.Batch([3, 700], [0, 0], M=0, seed=51)
    check_commit(b, [[0], [0]])
    b = R.Batch([20, 30, 10], [10, 10, 10], M=10, seed=52)
    i32 = dict(dtype=torch.int32, device="cuda:0")
    def run(paths, cached=None, table=None):
        k, v = b.caches()
        before = k.clone()
        path = torch.full((3, 11), -1, **i32)
        for i, p in enumerate(paths):
            path[i, :len(p)] = torch.tensor(p, **i32)
        status = torch.full((3,), 99, **i32)
        out = sfx.sd_commit(k, v, torch.as_tensor(b.table, device="cuda:0") if table is None else table, torch.tensor(b.cached if cached is None else cached, **i32), path, status=status)
        torch.cuda.synchronize()
        moved = (k.nan_to_num(3.0) != before.nan_to_num(3.0)).flatten(2).any(-1).cpu()
        return status.tolist(), out.tolist(), int(moved.sum())
    assert run([[0, 2], [0, 3], [0, 4]]) == ([0, 0, 0], [22, 32, 12], 3)
    for bad in ([0, 3, 2], [1, 2], [0, 2, 2], [0, 11], [0, 2 ** 30], [0, -2], [0, -1, 3]):
        assert run([[0, 2], bad, [0, 4]]) == ([0, 16, 0], [22, 30, 12], 2), bad
    assert run([[0, 2], [0, 3], [0, 4]], cached=[20, 16 * b.table.shape[1] - 2, -5]) == ([0, 16, 16], [22, 16 * b.table.shape[1] - 2, -5], 1)
    t = torch.as_tensor(b.table, device="cuda:0").clone()
    t[1, 2] = b.pages                                             # places 32 .. 47
    assert run([[0, 2], [0, 1, 9], [0, 4]], table=t) == ([0, 32, 0], [22, 33, 12], 2)


# --------------------------------------------------------------------------------------- refusals
def test_arguments_that_are_refused():
    b = R.Batch([20, 30], [10, 10], seed=60)
    k, v = b.caches()
    q, (table, offsets, cached), mask = b.q.cuda(), b.args(), b.mask_arg()
    def refused(error, **kw):
        a = dict(q=q, k_cache=k, v_cache=v, table=table, offsets=offsets, cached=cached, mask=mask) | kw
        with pytest.raises(error):
            sfx.sd_attend(a.pop("q"), a.pop("k_cache"), a.pop("v_cache"), a.pop("table"), a.pop("offsets"), a.pop("cached"), **a)
    wrong, code = TypeError, sfx.SuffixSpecError
    refused(wrong, q=q.cpu())
    refused(wrong, q=q.half())
    refused(wrong, q=q[:, :, ::2])
    refused(wrong, q=q.flatten(1))
    refused(code, q=q[:, :3])                                     # heads that are no multiple
    refused(wrong, k_cache=k[:1])
    refused(wrong, v_cache=v.half())
    refused(wrong, k_cache=k.float(), v_cache=v.float(), q=q)
    refused(code, k_cache=k.float(), v_cache=v.float(), q=q.float())
    refused(code, k_cache=k[..., :32], v_cache=v[..., :32], q=q[..., :32])
    refused(wrong, offsets=offsets.int())
    refused(wrong, cached=cached[:1])
    refused(wrong, table=table[:1])
    refused(wrong, table=table[:, ::2])
    refused(wrong, mask=mask[:, :, :1])
    refused(wrong, out=q[:3])
    refused(wrong, lse=torch.zeros(1, device="cuda:0"))
    refused(wrong, status=torch.zeros(2, device="cuda:0"))
    for name in ("window", "sinks", "shared"):
        refused(code, **{name: -1})
        refused(code, **{name: 2 ** 31})
    refused(code, scale=math.nan)
    odd = torch.zeros(20, 12, 2, 64, dtype=BF16, device="cuda:0")
    refused(code, k_cache=odd, v_cache=odd)                       # pages of 12
    buf = torch.zeros(b.rows * 4 * 64 + 8, dtype=BF16, device="cuda:0")
    refused(code, q=buf[1:1 + b.rows * 256].view(b.rows, 4, 64))   # not on 16 bytes
    refused(code, q=torch.zeros(b.rows, 4, 67, dtype=BF16, device="cuda:0")[:, :, :64])
    freq = torch.zeros(32, dtype=torch.float64, device="cuda:0")
    for f in (freq.float(), freq.cpu(), torch.zeros(65, dtype=torch.float64, device="cuda:0")):
        with pytest.raises(TypeError):
            sfx.sd_rotate(q, b.k.cuda(), b.v.cuda(), k, v, table, offsets, cached, f)
    for f in (freq[:7], torch.zeros(40, dtype=torch.float64, device="cuda:0")):
        with pytest.raises(code):
            sfx.sd_rotate(q, b.k.cuda(), b.v.cuda(), k, v, table, offsets, cached, f)
    with pytest.raises(code):
        sfx.sd_rotate(q, b.k.cuda(), b.v.cuda(), k, v, table, offsets, cached, freq, eps=-1.0)
    with pytest.raises(TypeError):
        sfx.sd_rotate(q, b.k.cuda()[:, :1], b.v.cuda(), k, v, table, offsets, cached, freq)
    tok = torch.zeros(2, 64, dtype=torch.int32, device="cuda:0")
    for x in (torch.zeros(b.rows, 9, 2, device="cuda:0"), torch.zeros(b.rows, 9, device="cuda:0", dtype=torch.int32), torch.zeros(b.rows, 18, device="cuda:0")[:, ::2], torch.zeros(b.rows, 9)):
        with pytest.raises(TypeError):
            sfx.sd_accept(x, offsets, tok, tok)
    with pytest.raises(TypeError):
        sfx.sd_accept(torch.zeros(b.rows, 9, device="cuda:0"), offsets, tok, tok[:, :3].contiguous())
    with pytest.raises(TypeError):
        sfx.sd_commit(k, v, table, cached, torch.zeros(2, 66, dtype=torch.int32, device="cuda:0"))
    with pytest.raises(TypeError):
        sfx.sd_commit(k, v, table, cached.long(), torch.zeros(2, 4, dtype=torch.int32, device="cuda:0"))


def test_accept_rows_that_two_requests_claim():
    """Offsets that descend: what they give to two requests is not written beyond the arrays."""
    dev = lambda a, dt=torch.int32: torch.tensor(a, dtype=dt, device="cuda:0")    # noqa: E731
    logits = torch.zeros(5, 8, device="cuda:0")
    logits[torch.arange(5), torch.arange(1, 6)] = 1.0
    tokens, parents = dev([[1, 2, 3, 4]] * 40), dev([[-1, 0, 1, 2]] * 40)
    offsets = dev(([0, 5, 0, 0] * 10) + [5], torch.int64)
    buf, status = dev([77] * 300), dev([99] * 40)
    out = dict(targets=dev([0] * 5), path=dev([[0] * 5] * 40), offsets=dev([0] * 41, torch.int64), tokens=buf[:5])
    sfx.sd_accept(logits, offsets, tokens, parents, out=out, status=status)
    assert (buf[5:] == 77).all() and out["tokens"].tolist() == [1, 2, 3, 4, 5]
    assert status.tolist() == [0, 16, 0, 0] * 10
    ends = out["offsets"].tolist()
    assert ends == sorted(ends) and ends[0] == 0 and ends[1:] == [5] * 40


def test_attend_rows_that_two_requests_claim():
    b = R.Batch([300, 0, 200, 0, 250], [9, -1, 9, -1, 9], head=64, seed=71)
    k, v = b.caches()
    table, _, cached = b.args()
    offsets = torch.tensor([0, 10, 0, 0, 0, 10], dtype=torch.int64, device="cuda:0")
    status = torch.full((5,), 99, dtype=torch.int32, device="cuda:0")
    out = sfx.sd_attend(b.q.cuda(), k, v, table, offsets, cached, mask=b.mask_arg(), status=status)
    assert status.tolist() == [0, 16, 0, 0, 0] and out.shape == b.q.shape


def test_attend_without_rows_tells_the_status():
    b = R.Batch([3, 40], [2, 4], seed=72)
    k, v = b.caches()
    table, _, cached = b.args()
    status = torch.full((2,), 99, dtype=torch.int32, device="cuda:0")
    sfx.sd_attend(b.q.cuda()[:0], k, v, table, torch.zeros(3, dtype=torch.int64, device="cuda:0"), cached, status=status)
    assert status.tolist() == [0, 0]
    status.fill_(99)
    sfx.sd_attend(b.q.cuda()[:0], k, v, table, torch.tensor([0, 0, 2], device="cuda:0"), cached, status=status)
    assert status.tolist() == [0, 16]


@pytest.mark.parametrize("group,head", [(128, 64), (100, 128), (65, 64), (43, 128), (127, 64)])
def test_attend_many_heads_of_one(group, head):
    check_attend(R.Batch([200, 3, 129, 1000], [4, 0, 17, 64], kv_heads=1, group=group, head=head, seed=73))


def test_calls_through_ctypes_alone(monkeypatch):
    """The conversions in Python, which stand in where the native module cannot be had."""
    from paper_2411_04975_b200 import binding
    monkeypatch.setattr(binding, "_call", binding._PlainCall(sfx.library()))
    check_attend(R.Batch([200, 31], [6, 9], head=128, seed=61), window=100, sinks=2)
    check_rotate(R.Batch([200, 31], [6, 9], head=128, seed=62, layout="hnd"), 64, fused=True)
    check_accept(torch.randn(5, 77, device="cuda:0"), np.array([0, 3, 5]), np.arange(8, dtype=np.int32).reshape(2, 4), np.array([[-1, 0, -1, -1]] * 2))
    check_commit(R.Batch([20, 30], [10, 10], M=10, seed=63, layers=2), [[0, 4], [0]])


def test_small_arrays_in_pinned_memory():
    """What says where rows and pages are, and what is told of them, in pinned host memory; queries, keys, values and results on the device."""
    b = R.Batch([200, 31, 700], [6, 9, 64], head=128, seed=65, shared=16)
    pin = lambda t: t.cpu().pin_memory()                          # noqa: E731
    table, offsets, cached = (pin(t) for t in b.args())
    k, v = b.caches()
    lse, status = torch.zeros(b.rows, 4).pin_memory(), torch.full((3,), 99, dtype=torch.int32).pin_memory()
    got = sfx.sd_attend(b.q.cuda(), k, v, table, offsets, cached, mask=pin(b.mask_arg()), lse=lse, status=status)
    torch.cuda.synchronize()
    assert got.is_cuda and status.tolist() == [0, 0, 0]
    compare(b, got, lse, *R.attend(b))
    freq = torch.zeros(32, dtype=torch.float64).pin_memory()
    got = sfx.sd_rotate(b.q.cuda(), b.k.cuda(), b.v.cuda(), k, v, table, offsets, cached, freq, mask=pin(b.mask_arg()))
    assert got.is_cuda and torch.equal(got.cpu(), b.q)


def test_no_requests():
    b = R.Batch([3], [2], seed=64)
    k, v = b.caches()
    none = dict(dtype=torch.int32, device="cuda:0")
    q = b.q.cuda()
    out = torch.full_like(q, 7.0)
    sfx.sd_attend(q, k, v, torch.zeros(0, 4, **none), torch.zeros(1, dtype=torch.int64, device="cuda:0"), torch.zeros(0, **none), out=out)
    sfx.sd_attend(q[:0], k, v, *b.args(), out=out[:0])
    sfx.sd_commit(k, v, torch.zeros(0, 4, **none), torch.zeros(0, **none), torch.zeros(0, 9, **none))
    torch.cuda.synchronize()
    assert (out == 7.0).all()
