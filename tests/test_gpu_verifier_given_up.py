"""Waits of sd_attend that run out (a test hook makes their limit short): the call returns, and the device is as good as before."""
import time

import pytest
import torch

import paper_2411_04975_b200 as sfx
import verifier_ref as R

pytestmark = pytest.mark.gpu

BATCHES = {
    "one_token": (dict(contexts=[5000], drafts=[0], head=128, group=4), {}),
    "narrow": (dict(contexts=[700, 31, 1290, 256], drafts=[5, 0, 31, 17], head=128, group=2), {}),
    "one_tile_each": (dict(contexts=[20] * 600, drafts=[1] * 600, head=64, group=2), {}),
    "wide": (dict(contexts=[2000, 3000, 900], drafts=[63, 50, 40], head=128, group=4), {}),
    "wide_64": (dict(contexts=[2000, 300, 90], drafts=[64, 50, 40], head=64, group=8), {}),
    "prefix": (dict(contexts=[512 + 40 * i for i in range(20)], drafts=[9] * 20, head=128, group=4, shared=512), dict(shared=512)),
    "window": (dict(contexts=[2000, 1500, 800], drafts=[20, 3, 64], head=128, group=4), dict(window=300, sinks=4)),
}


@pytest.fixture
def limit():
    yield sfx.library().sd_debug_attend_limit
    sfx.library().sd_debug_attend_limit(0)


@pytest.mark.parametrize("name", BATCHES)
def test_a_call_that_gives_up_returns(name, limit):
    args, kw = BATCHES[name]
    b = R.Batch(args["contexts"], args["drafts"], **{k: v for k, v in args.items() if k not in ("contexts", "drafts")}, seed=90)
    k, v = b.caches()
    a, mask = (b.q.cuda(), k, v, *b.args()), b.mask_arg()
    want = sfx.sd_attend(*a, mask=mask, **kw)
    for cycles in (1, 1000, 5000, 12000, 20000):
        for _ in range(5):
            limit(cycles)
            begin = time.monotonic()
            sfx.sd_attend(*a, mask=mask, **kw)
            torch.cuda.synchronize()
            assert time.monotonic() - begin < 2.0
            limit(0)
            assert torch.equal(sfx.sd_attend(*a, mask=mask, **kw), want)


def test_a_call_that_gives_up_waits_for_what_it_has_asked_for_and_for_no_more(limit):
    """Units of one tile, whose queries the walker waits for first: a tenth of a second goes by for a copy that is waited for but was not asked for."""
    args, kw = BATCHES["one_tile_each"]
    b = R.Batch(args["contexts"], args["drafts"], head=64, group=2, seed=91)
    k, v = b.caches()
    a, mask = (b.q.cuda(), k, v, *b.args()), b.mask_arg()
    sfx.sd_attend(*a, mask=mask)
    torch.cuda.synchronize()
    for cycles in list(range(1, 4000, 250)) + list(range(4000, 20000, 500)):
        limit(cycles)
        begin = time.monotonic()
        sfx.sd_attend(*a, mask=mask)
        torch.cuda.synchronize()
        assert time.monotonic() - begin < 0.08, cycles


@pytest.mark.parametrize("name", BATCHES)
def test_a_call_that_gives_up_says_so(name, limit):
    """In every status, whichever block was the last, and in the rows, as statuses need not be asked for."""
    args, kw = BATCHES[name]
    b = R.Batch(args["contexts"], args["drafts"], **{k: v for k, v in args.items() if k not in ("contexts", "drafts")}, seed=92, extra_rows=2)
    k, v = b.caches()
    (table, offsets, cached), mask = b.args(), b.mask_arg()
    bad = int(b.n > 1)
    if bad:
        cached[0] = -1                                            # (a request that makes no sense has its own status beside it)
    heads, last, first = b.q.shape[1], int(b.offsets[-1]), int(b.offsets[bad])
    wide = torch.empty(b.rows, heads + 1, b.head, dtype=b.dtype, device="cuda:0")
    out, lse, status = wide[:, 1:], torch.empty(b.rows, heads, device="cuda:0"), torch.empty(b.n, dtype=torch.int32, device="cuda:0")

    def run(cycles):
        wide.fill_(7.0), lse.fill_(5.0), status.fill_(99)
        limit(cycles)
        sfx.sd_attend(b.q.cuda(), k, v, table, offsets, cached, mask=mask, out=out, lse=lse, status=status, **kw)
        limit(0)
        return status.tolist(), out.clone(), lse.clone()

    sound = run(0)
    assert sound[0] == [16] * bad + [0] * (b.n - bad)
    seen = 0
    for cycles in [1] * 20 + list(range(500, 20000, 250)):
        got = run(cycles)
        failed = got[0][0] & sfx.STATUS_FAILED
        assert got[0] == [s | failed for s in sound[0]], cycles
        seen += failed != 0
        if failed:
            assert torch.isnan(got[1][first:last]).all() and torch.isnan(got[2][first:last]).all()
            for t, was in ((got[1], 7.0), (got[2], 5.0), (wide[:, :1], 7.0)):
                assert (t[:first] == was).all() and (t[last:] == was).all()
            assert (wide[:, 0] == 7.0).all()
        else:
            assert torch.equal(got[1], sound[1]) and torch.equal(got[2], sound[2])
    assert seen >= 20
