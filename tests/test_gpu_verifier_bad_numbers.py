"""Calls in which some requests' numbers make no sense: the others' rows are what they are without them."""
import numpy as np
import pytest
import torch

import paper_2411_04975_b200 as sfx
import verifier_ref as R
from test_gpu_verifier import compare

pytestmark = pytest.mark.gpu

FIVE = ([300, 140, 129, 128, 400], [4, 3, 5, 0, 9])               # contexts, drafts: rows 0 .. 4, 5 .. 8, 9 .. 14, 15, 16 .. 25


def run(b, offsets=None, table=None, **kw):
    """(status, out, lse) of a call with these in place of the batch's own."""
    k, v = b.caches()
    t, o, cached = b.args()
    o = o if offsets is None else torch.tensor(offsets, dtype=torch.int64, device="cuda:0")
    got, lse = torch.full_like(b.q, 7.0, device="cuda:0"), torch.full((b.rows, b.q.shape[1]), 5.0, device="cuda:0")
    status = torch.full((b.n,), 99, dtype=torch.int32, device="cuda:0")
    sfx.sd_attend(b.q.cuda(), k, v, t if table is None else table, o, cached, mask=b.mask_arg(), out=got, lse=lse, status=status, **kw)
    return status.tolist(), got, lse


def check_rows(b, requests, got, got_lse):
    """The rows of these requests against the 64-bit form, which knows nothing of the call's offsets; all others as they were."""
    out, lse, size = R.attend(b)
    keep = torch.zeros(b.rows, dtype=torch.bool)
    for i in requests:
        keep[int(b.offsets[i]):int(b.offsets[i + 1])] = True
    compare(b, got[keep], got_lse[keep], out[keep], lse[keep], size[keep])
    assert (got.cpu()[~keep] == 7.0).all() and (got_lse.cpu()[~keep] == 5.0).all()


# offsets, which requests they leave as they are: the others get a status
BROKEN = [([0, 2 ** 40, 9, 15, 16, 26], (2, 3, 4)), ([0, 5, -3, 15, 16, 26], (0, 3, 4)), ([0, 5, 9, 2 ** 62, 16, 26], (0, 1, 4)), ([2 ** 40, 5, 9, 15, 16, 26], (1, 2, 3, 4)),
          ([-1, 5, 9, 15, 16, 26], (1, 2, 3, 4))]


@pytest.mark.parametrize("offsets,sound", BROKEN, ids=lambda x: str(x[:3]))
@pytest.mark.parametrize("shared,kw", [(0, {}), (128, {}), (128, dict(shared=128)), (100, dict(shared=100))], ids=str)
def test_attend_finds_rows_behind_offsets_that_make_no_sense(offsets, sound, shared, kw):
    b = R.Batch(*FIVE, head=64, page=16, shared=shared, seed=80, extra_rows=2)
    status, got, lse = run(b, offsets, **kw)
    assert status == [0 if i in sound else 16 for i in range(5)]
    check_rows(b, sound, got, lse)


@pytest.mark.parametrize("last", [0, 15, -1, -2 ** 40, 2 ** 40])
@pytest.mark.parametrize("kw", [{}, dict(shared=128)], ids=str)
def test_attend_prefix_of_all_sound_rows(last, kw):
    """The last offset alone makes no sense: the rows before it have their prefix all the same."""
    b = R.Batch(*FIVE, head=64, page=16, shared=128, seed=81, extra_rows=2)
    status, got, lse = run(b, b.offsets.tolist()[:-1] + [last], **kw)
    assert status == [0, 0, 0, 0, 16]
    check_rows(b, range(4), got, lse)


@pytest.mark.parametrize("value", [-1, 2 ** 31 - 1])
@pytest.mark.parametrize("idle", [False, True])
def test_attend_bad_page_in_a_shared_prefix_is_told_to_all(value, idle):
    """The prefix is read through one request's pages: where one of them is none of the cache's, no request's rows are of use."""
    b = R.Batch(FIVE[0], ([-1] if idle else [4]) + FIVE[1][1:], head=64, page=16, shared=128, seed=82)
    k, v = b.caches()
    table, offsets, cached = b.args()
    first = 1 if idle else 0
    table[first, 3] = value
    status = torch.full((5,), 99, dtype=torch.int32, device="cuda:0")
    sfx.sd_attend(b.q.cuda(), k, v, table, offsets, cached, mask=b.mask_arg(), status=status, shared=128)
    assert status.tolist() == [0 if idle else 32, 32, 32, 32, 32]
    status.fill_(99)
    sfx.sd_attend(b.q.cuda(), k, v, table, offsets, cached, mask=b.mask_arg(), status=status, shared=128, window=500)     # (each reads its own)
    assert status.tolist() == [32 if i == first else 0 for i in range(5)]
