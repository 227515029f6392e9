"""Refusals of the token-table operators on the host: bad arguments are
reported before anything is enqueued (no GPU is needed, addresses are never
followed)."""
import copy
import ctypes as C
import threading
import time

import pytest
import torch

from paper_2206_00470_amd import ClipPlan, MX4, _lib, operators
from paper_2206_00470_amd.store import _pad, _rows

P = lambda a=0x10000: C.c_void_p(a)
BAD, BIG, SMALL = _lib.PS_ERR_INVALID, _lib.PS_ERR_UNSUPPORTED, _lib.PS_ERR_WORKSPACE
F32, BF16, F16 = _lib.PS_F32, _lib.PS_BF16, _lib.PS_F16
NOPAD = _lib.PS_NO_PAD


def test_null_store_is_refused():
    L = _lib.lib()
    assert L.ps_embed(None, P(), 1, NOPAD, 1.0, F32, P(), 8, None) == BAD
    assert b"store" in L.ps_last_error_message()
    assert L.ps_embed_grad(None, P(), 1, NOPAD, 1.0, F32, P(), 8, F32, P(), 8, 0, P(), 1 << 20, None) == BAD
    assert L.ps_embed_grad_rows(None, P(), 1, NOPAD, 1.0, F32, P(), 8, F32, P(), P(), 8, P(), P(), 1 << 20, None) == BAD
    assert L.ps_embed_grad_rows(None, P(), 1, NOPAD, 1.0, F32, P(), 8, F32, P(), P(), 8, None, P(), 1 << 20,
                                None) == BAD
    assert L.ps_wait_count(None, None) == BAD
    assert L.ps_wait_count(C.byref(C.c_int32(3)), None) == 0     # there already: no stream is asked


def test_workspace_sizes():
    L = _lib.lib()
    assert L.ps_embed_grad_workspace_bytes(64, 0) == 0
    assert L.ps_embed_grad_workspace_bytes(0, 10) == 0
    assert L.ps_embed_grad_workspace_bytes(64, (1 << 31)) == 0
    assert 0 < L.ps_embed_grad_workspace_bytes(64, 10) < L.ps_embed_grad_workspace_bytes(64, 100_000)
    assert L.ps_embed_grad_workspace_bytes(64, 100_000) < L.ps_embed_grad_workspace_bytes(4096, 100_000)
    assert L.ps_clip_workspace_bytes(-1) == 0
    assert 0 < L.ps_clip_workspace_bytes(1) <= L.ps_clip_workspace_bytes(1000)


def _clip(grads, outs, numel, types, max_norm=1.0, norm=P(0x8000), ws=P(0x4000), wsb=1 << 30, count=None):
    k = len(grads)
    arr = lambda t, v: None if v is None else (t * k)(*v)
    return _lib.lib().ps_clip_grads(k if count is None else count, arr(C.c_void_p, grads), arr(C.c_void_p, outs),
                                    arr(C.c_int64, numel), arr(C.c_int32, types), max_norm, norm, ws, wsb, None)


def test_clip_refuses_bad_arguments():
    A, B = 0x100000, 0x200000
    ok = ([A], [A], [100], [F32])
    assert _clip(*ok, count=-1) == BAD
    assert _clip([A], [A], [-1], [F32]) == BAD
    assert _clip([A], [A], [1 << 40], [F32]) == BIG
    assert _clip([A], [A], [100], [3]) == BAD
    assert _clip([None], [A], [100], [F32]) == BAD
    assert _clip([A], [None], [100], [F32]) == BAD
    assert _clip([A], None, [100], [F32]) == BAD
    assert _clip([A], [A], None, [F32]) == BAD
    assert _clip([A + 2], [A + 2], [100], [F32]) == BAD
    assert _clip([A + 1], [A + 1], [100], [BF16]) == BAD
    for m in (0.0, -1.0, float("nan")):
        assert _clip(*ok, max_norm=m) == BAD
    assert _clip(*ok, norm=None) == BAD
    assert _clip(*ok, ws=None) == BAD
    assert _clip(*ok, wsb=8) == SMALL
    # overlaps: with an input, between outputs, one tensor twice in place, its own input in part
    assert _clip([A, B], [B + 396, B], [100, 100], [F32, F32]) == BAD
    assert b"overlap" in _lib.lib().ps_last_error_message()
    assert _clip([A, B], [B + 0x1000, B + 0x1000 + 396], [100, 100], [F32, F32]) == BAD
    assert _clip([A, A], [A, A], [100, 100], [F32, F32]) == BAD
    assert _clip([A], [A + 200], [100], [F32]) == BAD
    assert _clip([A, B], [B, B + 0x1000], [100, 100], [BF16, BF16]) == BAD


def test_mx4_refuses_bad_arguments():
    L = _lib.lib()
    q = lambda rows=4, dim=64, t=F32, x=P(), ld=64, c=P(), s=P(): L.ps_mx4_quantize(rows, dim, t, x, ld, c, s, None)
    assert q(rows=0) == _lib.PS_OK
    assert q(rows=-1) == BAD and q(t=3) == BAD and q(ld=63) == BAD
    assert q(dim=0) == BIG and q(dim=16385, ld=1 << 20) == BIG
    assert q(x=None) == BAD and q(c=None) == BAD and q(s=None) == BAD
    assert q(x=P(0x10002)) == BAD and q(c=P(0x10008)) == BAD
    e = lambda c=P(), s=P(), rows=9, dim=64, ids=P(), n=5, t=F32, o=P(), ld=64, err=P(): L.ps_mx4_embed(
        c, s, rows, dim, ids, n, NOPAD, 1.0, t, o, ld, err, None)
    assert e(n=0) == _lib.PS_OK
    assert e(n=-1) == BAD and e(rows=-1) == BAD and e(t=9) == BAD and e(ld=63) == BAD and e(dim=0) == BIG
    assert e(c=None) == BAD and e(s=None) == BAD and e(o=None) == BAD and e(err=None) == BAD
    assert e(ids=None, n=10) == BAD
    assert e(c=P(0x10008)) == BAD and e(o=P(0x10002)) == BAD
    p = lambda m=2, n=3, dim=64, ac=P(), asc=P(), bc=P(), bs=P(), t=F32, o=P(), ld=3: L.ps_mx4_product(
        m, n, dim, ac, asc, bc, bs, 1.0, t, o, ld, None)
    assert p(m=0) == _lib.PS_OK and p(n=0) == _lib.PS_OK
    assert p(m=-1) == BAD and p(n=-1) == BAD and p(t=-1) == BAD and p(ld=2) == BAD and p(dim=20000) == BIG
    for k in ("ac", "asc", "bc", "bs", "o"):
        assert p(**{k: None}) == BAD
    assert p(ac=P(0x10004)) == BAD and p(bc=P(0x10004)) == BAD and p(o=P(0x10001), t=BF16) == BAD
    assert p(m=1 << 30, n=1 << 40, ld=1 << 40) == BIG


def test_sizes_beyond_a_grid_are_refused():
    """A launch counts its threads in 32 bits."""
    L = _lib.lib()
    assert L.ps_mx4_quantize(1 << 40, 64, F32, P(), 64, P(), P(), None) == BIG
    assert L.ps_mx4_quantize(1 << 30, 1024, F32, P(), 1024, P(), P(), None) == BIG
    assert L.ps_mx4_embed(P(), P(), 1 << 41, 64, None, 1 << 40, NOPAD, 1.0, F32, P(), 64, None, None) == BIG
    assert L.ps_mx4_embed(P(), P(), 100, 4096, P(), 1 << 26, NOPAD, 1.0, F32, P(), 4096, P(), None) == BIG
    assert L.ps_mx4_product(1 << 22, 1 << 28, 64, P(), P(), P(), P(), 1.0, F32, P(), 1 << 28, None) == BIG


def test_binding_refuses_host_tensors():
    with pytest.raises(TypeError):
        ClipPlan([torch.zeros(4)])
    with pytest.raises(ValueError):
        ClipPlan([])
    with pytest.raises(TypeError):
        MX4(torch.zeros((2, 16), dtype=torch.uint8), torch.zeros((2, 1), dtype=torch.uint8), 32)
    with pytest.raises(TypeError):
        _rows(torch.zeros((2, 4)), 4, torch.device("cuda", 0), "x")


def test_new_constants_match_the_header():
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "adapm.h")).read()
    defs = {m.group(1): int(m.group(2)) for m in re.finditer(r"#define (PS_[A-Z0-9_]+)\s+\(?(-?\d+)\)?", text)}
    for name in ("PS_F32", "PS_BF16", "PS_F16"):
        assert getattr(_lib, name) == defs[name], name
    assert _lib.PS_NO_PAD == -(2 ** 63)


def test_clip_plans_refuse_bad_arguments():
    L, A, B = _lib.lib(), 0x100000, 0x200000
    arr = lambda t, *v: (t * len(v))(*v)
    i64, i32, ptr = C.c_int64, C.c_int32, C.c_void_p
    assert L.ps_clip_plan_bytes(0, None) == 0 and L.ps_clip_plan_bytes(-1, None) == 0
    assert L.ps_clip_plan_bytes(1, None) == 0 and L.ps_clip_plan_bytes(2, arr(i64, 5, -1)) == 0
    assert L.ps_clip_plan_bytes(1, arr(i64, 0)) == 0
    size = L.ps_clip_plan_bytes(2, arr(i64, 16384, 16385))
    assert size == 3 * 24
    host, apart = (C.c_uint8 * 96)(*[0xee] * 96), C.c_int64(-1)

    def plan(grads, outs, numel, types, to=host, nb=size, ap=apart):
        return L.ps_clip_plan(len(numel), arr(ptr, *grads), None if outs is None else arr(ptr, *outs), arr(i64, *numel),
                              arr(i32, *types), to, nb, None if ap is None else C.byref(ap))

    ok = ([A, B], [A, 0x400000], [16384, 16385], [F32, BF16])
    assert plan(*ok) == 0 and apart.value == 2 * 16385
    assert bytes(host)[size:] == b"\xee" * (96 - size)
    words = (C.c_uint64 * 9).from_buffer(host)
    assert list(words) == [A, A, 16384, B, 0x400000, 16384 | BF16 << 32, B + 32768, 0x400000 + 32768, 1 | BF16 << 32]
    assert plan(*ok, nb=size - 24) == BAD and plan(*ok, to=None) == BAD and plan(*ok, ap=None) == BAD
    assert plan([A, B], None, *ok[2:]) == BAD
    assert plan([A, A], [A, A], [10, 10], [F32, F32], nb=48) == BAD        # both write one tensor
    assert plan([A, B], [A, A + 4], [10, 10], [F32, F32], nb=48) == BAD
    assert plan([A, B], [A, B], [10, -1], [F32, F32], nb=0) == BAD
    assert plan([A + 2, B], [A + 2, B], *ok[2:]) == BAD
    run = lambda p=P(), nb=size, scaling=1, m=1.0, norm=P(0x8000), ws=P(0x4000), wsb=1 << 20: L.ps_clip_run(
        p, nb, 0, scaling, m, norm, ws, wsb, None)
    for bad in (dict(p=None), dict(p=P(0x10001)), dict(nb=size - 1), dict(m=0.0), dict(m=float("nan")), dict(norm=None),
                dict(norm=P(0x8004)), dict(ws=None), dict(ws=P(0x4001))):
        assert run(**bad) == BAD, bad
    assert run(wsb=8) == SMALL and run(scaling=0, m=0.0, wsb=8) == SMALL


def test_a_quantised_tables_first_lookups_share_one_cleared_flag(monkeypatch):
    """Two threads look a table up for the first time, the second while the first
    waits for the flag's zeros: both launches get one flag, after that wait."""
    x = MX4.__new__(MX4)._set(torch.zeros((4, 16), dtype=torch.uint8), torch.zeros((4, 1), dtype=torch.uint8), 32)
    ids = torch.zeros(2, dtype=torch.int64)
    waiting, second, flags, waits = threading.Event(), threading.Event(), [], []

    class On:
        def __init__(self, *a):
            pass

        def __enter__(self):
            second.set() if threading.current_thread().name == "second" else None

        def __exit__(self, *a):
            pass

    class Stream:
        def synchronize(self):
            waits.append(1)
            waiting.set()
            second.wait(5)
            time.sleep(0.3)   # the other thread goes as far as it can
            assert not flags, "a lookup was launched before the flag was cleared"

    class Lib:
        def ps_mx4_embed(self, *a):
            flags.append(a[-2])
            return _lib.PS_OK

    monkeypatch.setattr(operators, "_On", On)
    monkeypatch.setattr(operators, "lib", Lib)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream())
    failed = []

    def look():
        try:
            x._lookup(ids, 2, ids.shape, 1.0, torch.float32, None, None, None)
        except BaseException as e:
            failed.append(e)

    a, b = threading.Thread(target=look, name="first"), threading.Thread(target=look, name="second")
    a.start()
    assert waiting.wait(20)
    b.start()
    a.join(20), b.join(20)
    assert not failed, failed
    assert len(waits) == 1 and len(flags) == 2 and flags[0] == flags[1] == x._err.data_ptr()
    assert not x._err.any()
    assert torch.equal(copy.deepcopy(x).codes, x.codes)       # a table can be copied as it is


@pytest.mark.parametrize("pad", [1 << 63, -(1 << 63) - 1, (1 << 64) + 5, -(1 << 63), 1.5, float("nan")])
def test_pads_that_no_id_can_have_are_refused(pad):
    """An argument of 64 bits would take such a pad for another number, the
    lowest one for "no padding"."""
    with pytest.raises(ValueError, match="pad"):
        _pad(pad)


def test_pads_reach_the_kernels_as_they_are():
    assert _pad(None) == NOPAD
    for pad in (0, -1, 7, (1 << 63) - 1, -(1 << 63) + 1, 4.0, torch.tensor(3)):
        assert _pad(pad) == pad and type(_pad(pad)) is int
