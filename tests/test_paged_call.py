"""The CPython functions of the paged cache's calls: what they hand to the entry points, what they refuse, and the calls without them (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2510_13797_amd import bc

VP, I32, I64 = C.c_void_p, C.c_int32, C.c_int64


def _entries(seen):
    append = C.CFUNCTYPE(I32, VP, VP, I64, VP, I32, VP, I64, VP, VP, I32, VP, VP, C.c_float, VP, VP, VP, VP)(lambda *a: seen.append([x or 0 for x in a]) or 5)
    attend = C.CFUNCTYPE(I32, VP, VP, I64, VP, I32, VP, VP, VP, VP, C.c_size_t, VP)(lambda *a: seen.append([x or 0 for x in a]) or 6)
    return append, attend


def test_native_calls_hand_over_addresses_and_numbers():
    bc.load()
    seen = []
    append, attend = _entries(seen)
    shape, pages = bc.bc_shape(2, 4, 1, 64, bc.BC_BF16, 0.125), bc.bc_pages()
    t = [torch.zeros(3 + i) for i in range(9)]
    p = [x.data_ptr() for x in t]
    args = [C.cast(append, VP).value, shape, pages, 1 << 30, t[0], 7, t[1], 1 << 31, t[2], t[3], 64, None, t[4], 0.25, t[5], None, t[6], 9]
    assert bc._paged_calls[0](*args) == 5
    assert seen[0] == [C.addressof(shape), C.addressof(pages), 1 << 30, p[0], 7, p[1], 1 << 31, p[2], p[3], 64, 0, p[4], 0.25, p[5], 0, p[6], 9]
    for i, bad in ((0, None), (0, 0), (1, 3), (2, None), (3, 1.5), (3, 1 << 70), (5, 1 << 31), (5, None), (6, 4), (7, "8"), (10, 1 << 40), (13, "x"), (17, None)):
        with pytest.raises((TypeError, ValueError, AttributeError, OverflowError, BufferError)):
            bc._paged_calls[0](*[bad if j == i else x for j, x in enumerate(args)])
    args = [C.cast(attend, VP).value, shape, pages, 5, None, 7, t[1], t[2], t[3], t[4], 1 << 40, 9]
    assert bc._paged_calls[2](*args) == 6
    assert seen[1] == [C.addressof(shape), C.addressof(pages), 5, 0, 7, p[1], p[2], p[3], p[4], 1 << 40, 9]
    for i, bad in ((0, None), (1, 3), (2, None), (3, None), (5, 1 << 31), (6, 4), (10, -1), (10, "8"), (11, None)):
        with pytest.raises((TypeError, ValueError, AttributeError, OverflowError, BufferError)):
            bc._paged_calls[2](*[bad if j == i else x for j, x in enumerate(args)])
    for call in (bc._paged_calls[0], bc._paged_calls[2]):
        with pytest.raises(TypeError):
            call(*args[:-1])
    assert len(seen) == 2


@pytest.mark.parametrize("native", [True, False])
def test_cache_hands_the_library_its_tensors(monkeypatch, native):
    # (on the host, with the checks of the device taken out: what goes to the entry points by either way)
    bc.load()
    seen = []
    append, attend = _entries(seen)
    cache = bc.PagedCache(2, 4, 1, 64, 9, 32, 4, "cpu")
    monkeypatch.setattr(bc, "_current_device", lambda: None)
    monkeypatch.setattr(bc, "_stream_ptr", lambda: None if not native else 7)
    monkeypatch.setattr(bc, "_used_here", lambda *t: None)
    cache._home = bc._stream_ptr()

    class Library:
        bc_paged_workspace_bytes = staticmethod(lambda *a: 48)

        @staticmethod
        def bc_paged_attend(*a):
            seen.append([C.addressof(x._obj) if type(x).__name__ == "CArgObject" else x or 0 for x in a])
            return 6

        @staticmethod
        def bc_status_str(st):
            return b"status"

    monkeypatch.setattr(bc, "_lib", Library())
    calls = None if not native else (bc._paged_calls[0], C.cast(append, VP).value, bc._paged_calls[2], C.cast(attend, VP).value)
    monkeypatch.setattr(bc, "_paged_calls", calls)
    q, out, active = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 4, 64), torch.ones(2, dtype=torch.uint8)
    with pytest.raises(bc.BcError):                       # (the status of the stand-in is none that is fine)
        cache.attend(q, out=out, active=active, max_len=70)
    assert len(seen) == 1
    got = seen[0]
    assert got[:8] == [C.addressof(cache.shape), C.addressof(cache._c), 2, 0, 1, q.data_ptr(), out.data_ptr(), active.data_ptr()] and got[9] == 48
    assert cache._c.max_len == 70
    assert [getattr(cache._c, n) for n in ("k", "v", "k_scale", "v_scale", "table", "len", "err")] == [t.data_ptr() for t in cache._own()[:7]]


@pytest.mark.parametrize("at_home", [True, False])
def test_a_given_table_is_noted_at_every_call(monkeypatch, at_home):
    # (it may come from another stream than the cache's, whose own tensors are noted where a call is on another one)
    bc.load()
    noted = []
    table = torch.zeros(2, 4, dtype=torch.int32)
    caches = [bc.PagedCache(2, 4, 1, 64, 9, 32, 4, "cpu", table=t) for t in (table, None)]
    monkeypatch.setattr(bc, "_current_device", lambda: None)
    monkeypatch.setattr(bc, "_stream_ptr", lambda: 7)
    monkeypatch.setattr(bc, "_used_here", lambda *t: noted.extend(x for x in t if x is not None))
    monkeypatch.setattr(bc, "_paged_calls", None)

    class Library:
        bc_paged_workspace_bytes = staticmethod(lambda *a: 48)
        bc_paged_attend = staticmethod(lambda *a: bc.BC_OK)

    monkeypatch.setattr(bc, "_lib", Library())
    for cache, given in zip(caches, (True, False)):
        cache._home = 7 if at_home else 8
        del noted[:]
        cache.attend(torch.zeros(2, 4, 64, dtype=torch.bfloat16))
        assert any(x is cache.table for x in noted) == (given or not at_home)
        assert any(x is cache.lengths for x in noted) == (not at_home)


def test_the_home_of_a_cache_is_its_devices_stream(monkeypatch):
    # built while another device is the current one: that device's current stream is a stranger's (torch's side stands in)
    class Torch:
        _cuda_getDevice = staticmethod(lambda: 0)
        _cuda_getCurrentRawStream = staticmethod(lambda device: 100 + device)

    monkeypatch.setattr(bc, "_torch_c", Torch())
    monkeypatch.setattr(bc, "load", lambda: None)
    monkeypatch.setattr(bc, "_is", lambda *a: None)

    class Pool(torch.Tensor):                              # (host memory that says it is on the second device)
        device = torch.device("cuda", 1)

    full = torch.full
    monkeypatch.setattr(torch, "full", lambda *a, **kw: full(*a, **kw).as_subclass(Pool))
    assert bc.PagedCache(2, 4, 1, 64, 9, 32, 4, "cpu", table=torch.zeros(2, 4, dtype=torch.int32))._home == 101
