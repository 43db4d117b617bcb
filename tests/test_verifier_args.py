"""What the verifier's entry points refuse before any device is asked, and what the sizes of a call ask for."""
import ctypes as C

import pytest

import paper_2411_04975_b200 as sfx
from paper_2411_04975_b200 import binding


@pytest.fixture(scope="module")
def lib():
    return sfx.library()


def cache(**kw):
    c = dict(d_k=4096, d_v=8192, dtype=1, kv_heads=2, head_dim=64, n_layers=1, n_pages=4, page_size=16) | kw
    line = c["kv_heads"] * c["head_dim"]
    st = kw.get("strides", (0, c["page_size"] * line, line, c["head_dim"]))
    c.pop("strides", None)
    return binding._Cache(*c.values(), (C.c_int64 * 4)(*st), (C.c_int64 * 4)(*st))


def rows(**kw):
    r = dict(n=2, rows=10, max_draft=8, table_stride=2, d_offsets=256, d_cached=512, d_table=1024, d_mask=None, d_status=None) | kw
    return binding._Rows(*r.values())


def attend(lib, c, r, work=4096, size=1 << 40, **kw):
    p = dict(q_heads=4, scale=1.0, window=0, sinks=0, shared=0) | {k: v for k, v in kw.items() if k in ("q_heads", "scale", "window", "sinks", "shared")}
    prm = binding._AttendParams(*p.values(), (C.c_int64 * 2)(*kw.get("q_stride", (256, 64))), (C.c_int64 * 2)(*kw.get("out_stride", (256, 64))))
    return lib.sd_attend(C.byref(c), C.byref(r), C.byref(prm), kw.get("q", 65536), kw.get("out", 131072), None, work, size, None)


BAD_CACHES = [dict(dtype=3), dict(dtype=0), dict(head_dim=96), dict(head_dim=32), dict(kv_heads=0), dict(n_pages=0), dict(page_size=0), dict(page_size=12),
              dict(page_size=4), dict(page_size=136), dict(d_k=None), dict(d_v=4104), dict(strides=(0, 2048, 130, 64)), dict(strides=(0, 2048, -128, 64)),
              dict(strides=(0, 2048, 0, 64)), dict(n_layers=2, strides=(12, 2048, 128, 64)), dict(n_layers=0)]
BAD_ROWS = [dict(n=-1), dict(rows=-1), dict(max_draft=65), dict(max_draft=-1), dict(table_stride=0), dict(table_stride=1 << 30), dict(d_cached=None), dict(d_table=None),
            dict(d_offsets=None)]
BAD_ATTEND = [dict(q_heads=3), dict(q_heads=0), dict(window=-1), dict(sinks=-2), dict(shared=-1), dict(scale=float("nan")), dict(q=65544), dict(q=None), dict(out=None),
              dict(out=131080), dict(q_stride=(260, 64)), dict(out_stride=(256, 4)), dict(work=None), dict(work=4224)]


@pytest.mark.parametrize("bad", BAD_CACHES + BAD_ROWS + BAD_ATTEND, ids=str)
def test_attend_refuses(lib, bad):
    c = cache(**bad) if bad in BAD_CACHES else cache()
    r = rows(**bad) if bad in BAD_ROWS else rows()
    assert attend(lib, c, r, **(bad if bad in BAD_ATTEND else {})) == -1


@pytest.mark.parametrize("bad", [dict(q_heads=130), dict(q_heads=258), dict(scale=float("inf")), dict(q_stride=(0, 64)), dict(q_stride=(256, 0)), dict(q_stride=(256, -64)),
                                 dict(q_stride=(1 << 38, 64)), dict(out_stride=(0, 64)), dict(out_stride=(256, 0))], ids=str)
def test_attend_refuses_heads_and_strides(lib, bad):
    c = cache(kv_heads=1) if bad.get("q_heads") == 130 else cache()
    assert attend(lib, c, rows(), **bad) == -1


def test_attend_refuses_null_structs(lib):
    assert lib.sd_attend(None, None, None, None, None, None, None, 0, None) == -1
    assert lib.sd_attend_workspace(None, None, None) == -1


@pytest.mark.parametrize("bad", BAD_CACHES + BAD_ROWS, ids=str)
def test_rotate_refuses(lib, bad):
    c = cache(**bad) if bad in BAD_CACHES else cache()
    r = rows(**bad) if bad in BAD_ROWS else rows()
    two = [(C.c_int64 * 2)(256, 64) for _ in range(4)]
    prm = binding._RotateParams(4, 64, 0, 1.0, 1e-6, *two)
    assert lib.sd_rotate(C.byref(c), C.byref(r), C.byref(prm), 65536, 65536, 65536, 4096, None, None, None, 65536, None) == -1


@pytest.mark.parametrize("bad", [dict(rot_dim=8), dict(rot_dim=-16), dict(rot_dim=80), dict(q_heads=5), dict(eps=-1.0), dict(eps=float("nan")), dict(freq=None), dict(q=65544),
                                 dict(weight=4100), dict(stride=(256, 60))], ids=str)
def test_rotate_refuses_its_own(lib, bad):
    c, r = cache(), rows()
    two = [(C.c_int64 * 2)(*bad.get("stride", (256, 64))) for _ in range(4)]
    prm = binding._RotateParams(bad.get("q_heads", 4), bad.get("rot_dim", 64), 0, 1.0, bad.get("eps", 1e-6), *two)
    assert lib.sd_rotate(C.byref(c), C.byref(r), C.byref(prm), bad.get("q", 65536), 65536, 65536, bad.get("freq", 4096), None, bad.get("weight"), None, 65536, None) == -1


@pytest.mark.parametrize("bad", [dict(n=-1), dict(rows=-1), dict(M=65), dict(M=-1), dict(V=0), dict(V=(1 << 30) + 1), dict(dtype=0), dict(dtype=4), dict(stride=99), dict(logits=None),
                                 dict(logits=4097), dict(path=None)], ids=str)
def test_accept_refuses(lib, bad):
    a = dict(n=2, rows=4, M=3, V=100, dtype=1, stride=100, logits=4096, offsets=256, tokens=256, parents=256, targets=256, path=256, begins=256, new=256, status=None) | bad
    assert lib.sd_accept(*a.values(), None) == -1


def test_commit_refuses(lib):
    for bad in BAD_CACHES:
        c, r = cache(**bad), rows()
        assert lib.sd_commit(C.byref(c), C.byref(r), 4096, 4096, None) == -1, bad
    c, r = cache(), rows()
    assert lib.sd_commit(C.byref(c), C.byref(r), None, 4096, None) == -1
    assert lib.sd_commit(C.byref(c), C.byref(r), 4096, None, None) == -1


def test_tensors_that_are_no_device_memory_are_refused():
    import torch
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    k = torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError, match="k_cache: expected a tensor on the current CUDA device"):
        binding._PlainCall(sfx.library()).attend(q, k, k, i[None], i, i, None, 1.0, 0, 0, 0, q, None, None)


def test_plain_calls_take_the_same_arguments():
    import inspect
    sfx.library()
    native = binding._load_call(binding._lib)
    for name in ("rotate", "attend", "accept", "commit"):
        n = len(inspect.signature(getattr(binding._PlainCall(binding._lib), name)).parameters)
        with pytest.raises(TypeError, match=f"{n} arguments expected"):
            getattr(native, name)()


class _Library:
    """Takes every call; what it was given as the workspace of sd_attend is kept."""

    def sd_attend_workspace(self, *a):
        return 1 << 20

    def sd_attend(self, *a):
        self.work = a[6]
        return 0

    def sd_rotate(self, *a):
        return 0

    sd_accept = sd_commit = sd_rotate


def test_results_and_workspaces_are_on_the_device_for_arguments_in_host_memory(monkeypatch):
    """Tensors in pinned host memory are taken; what the call makes itself has to be the device's all the same: pageable memory is not for its kernels."""
    import torch
    made, empty = [], torch.empty

    def record(*a, device=None, **kw):
        made.append(torch.device(device))
        return empty(*a, **kw)

    for name, f in (("_here", lambda t, name: None), ("_ptr", lambda t, dtype, name: None if t is None else t.data_ptr()), ("_stream", lambda: 0), ("_current_device", lambda: 0)):
        monkeypatch.setattr(binding, name, f)
    monkeypatch.setattr(binding.torch, "empty", record)
    lib = _Library()
    call = binding._PlainCall(lib)
    q, k = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16)
    rows = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    table, cached = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    offsets = torch.zeros(2, dtype=torch.int64)
    call.rotate(q, rows, rows, k, k, table, offsets, cached, torch.zeros(32, dtype=torch.float64), None, None, None, None, 1e-6, False, 1.0, None, None)
    assert len(made) == 1
    call.attend(q, k, k, table, offsets, cached, None, None, 0, 0, 0, None, None, None)
    assert len(made) == 3 and lib.work
    call.attend(q, k, k, table, offsets, cached, None, None, 0, 0, 0, q, None, None)
    assert len(made) == 4
    draft = torch.zeros(1, 3, dtype=torch.int32)
    call.accept(torch.zeros(3, 9), offsets, draft, draft, None, None)
    assert len(made) == 8
    call.commit(k, k, table, cached, torch.zeros(1, 4, dtype=torch.int32), None, None)
    assert len(made) == 9
    assert all(d == torch.device("cuda", 0) for d in made)


@pytest.mark.parametrize("size", [2 ** 31, 2 ** 32 + 3])
def test_sizes_beyond_31_bits_are_refused(monkeypatch, size):
    """ctypes keeps the low bits of a number that its field has no room for."""
    import torch
    monkeypatch.setattr(binding, "_here", lambda t, name: None)
    monkeypatch.setattr(binding, "_ptr", lambda t, dtype, name: None if t is None else t.data_ptr())
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    monkeypatch.setattr(binding, "_device", lambda: torch.device("cpu"))
    call = binding._PlainCall(_Library())
    table, cached, offsets = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int64)
    q, k = torch.zeros(1, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16)
    rows, freq = torch.zeros(1, 2, 64, dtype=torch.bfloat16).expand(size, 2, 64), torch.zeros(32, dtype=torch.float64)
    many, path = q.expand(size, 4, 64), torch.zeros(1, 4, dtype=torch.int32)
    wide = table[:, :1].expand(1, size)

    def attend(q=q, k=k, table=table):
        return call.attend(q, k, k, table, offsets, cached, None, None, 0, 0, 0, q, None, None)

    assert attend() is q
    for kw in (dict(q=many), dict(table=wide), dict(k=k[:1].expand(size, 16, 2, 64)), dict(k=k[:, :1].expand(2, size, 2, 64))):
        with pytest.raises(TypeError, match="beyond 31 bits"):
            attend(**kw)
    with pytest.raises(TypeError, match="beyond 31 bits"):
        call.rotate(many, rows, rows, k, k, table, offsets, cached, freq, None, None, None, None, 1e-6, False, 1.0, many, None)
    for kw in (dict(table=wide), dict(k=k[None].expand(size, 2, 16, 2, 64))):
        with pytest.raises(TypeError, match="beyond 31 bits"):
            call.commit(kw.get("k", k), kw.get("k", k), kw.get("table", table), cached, path, cached, None)
