"""What the calls of the paged cache refuse (host logic only: no GPU needed; addresses are made up and never dereferenced)."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2510_13797_amd import bc

PTR = 0x7F0000100000
ODD = PTR + 4


def shape(Hq=4, Hkv=2, d=64, dtype=bc.BC_BF16, B=3, scale=1.0):
    return bc.bc_shape(B, Hq, Hkv, d, dtype, scale)


def _pages(**kw):
    f = dict(k=PTR, v=PTR, k_scale=PTR, v_scale=PTR, table=PTR, len=PTR, err=PTR, arrivals=PTR, pages=9, page_rows=32, table_pages=4, max_len=0)
    f.update(kw)
    return bc.bc_pages(**f)


def _append(s=None, pg=None, rows=5, off=PTR, max_new=5, qkv=PTR, stride=512, pos=PTR, freq=PTR, rot=64, qw=PTR, kw=PTR, eps=1e-6, keep=None, active=None,
            q=PTR + 4096):
    return bc.bc_paged_append(s or shape(), pg or _pages(), rows, off, max_new, qkv, stride, pos, freq, rot, qw, kw, eps, keep, active, q, None)


def _attend(s=None, pg=None, rows=5, off=PTR, max_new=5, q=PTR, out=PTR, active=None, ws=PTR, nbytes=1 << 40):
    return bc.bc_paged_attend(s or shape(), pg or _pages(), rows, off, max_new, q, out, active, ws, nbytes, None)


@pytest.mark.parametrize("call", [_append, _attend])
def test_refusals_of_both_calls(call):
    bc.load()
    for kw in (dict(Hq=5), dict(Hkv=0), dict(d=96), dict(d=256), dict(dtype=2), dict(Hq=18), dict(B=0), dict(B=(1 << 23) + 1)):
        assert call(s=shape(**kw)) == bc.BC_ERR_SHAPE, kw
    for field in ("k", "v", "k_scale", "v_scale", "table", "len", "err"):
        assert call(pg=_pages(**{field: None})) == bc.BC_ERR_ARG, field
    for kw in (dict(k=ODD), dict(v=ODD)):
        assert call(pg=_pages(**kw)) == bc.BC_ERR_ARG, kw
    for kw in (dict(page_rows=8), dict(page_rows=48), dict(page_rows=2048), dict(page_rows=0), dict(page_rows=-16), dict(pages=0), dict(pages=-1), dict(table_pages=0),
               dict(pages=1 << 30, page_rows=16), dict(table_pages=1 << 27, page_rows=16)):
        assert call(pg=_pages(**kw)) == bc.BC_ERR_SHAPE, kw
    for kw in (dict(rows=-1), dict(rows=1 << 31), dict(max_new=-1)):
        assert call(**kw) == bc.BC_ERR_SHAPE, kw
    # a row for each sequence, or offsets
    assert call(off=None, rows=5, max_new=1) == bc.BC_ERR_ARG
    for most in (0, 2, 5):
        assert call(off=None, rows=3, max_new=most) == bc.BC_ERR_ARG, most
    # nothing to do is no error
    assert call(rows=0) == bc.BC_OK and call(max_new=0) == bc.BC_OK


def test_append_refusals():
    for rot in (-8, 4, 12, 72):
        assert _append(rot=rot) == bc.BC_ERR_SHAPE, rot
    for eps in (-1e-6, float("nan"), float("inf")):
        assert _append(eps=eps) == bc.BC_ERR_ARG
    for kw in (dict(qkv=None), dict(qkv=ODD), dict(pos=None), dict(freq=None), dict(q=ODD), dict(qw=ODD), dict(kw=ODD), dict(stride=511), dict(stride=516), dict(stride=504),
               dict(stride=-512), dict(stride=1 << 40), dict(q=PTR), dict(pg=_pages(arrivals=None))):
        assert _append(**kw) == bc.BC_ERR_ARG, kw
    # (more blocks than a grid holds)
    assert _append(s=shape(B=1 << 21, Hkv=4), rows=1 << 30, max_new=1 << 20) == bc.BC_ERR_SHAPE
    assert _append(s=shape(Hq=65536, Hkv=8192), stride=1 << 30) == bc.BC_ERR_SHAPE


def test_attend_refusals():
    for scale in (-1.0, float("nan"), float("inf")):
        assert _attend(s=shape(scale=scale)) == bc.BC_ERR_ARG
    for kw in (dict(q=None), dict(out=None), dict(q=ODD), dict(out=ODD), dict(pg=_pages(arrivals=None))):
        assert _attend(**kw) == bc.BC_ERR_ARG, kw
    long = _pages(pages=1000, table_pages=1000)
    need = bc.bc_paged_workspace_bytes(shape(), 5, 5, 32000)
    assert need > 1000
    for kw in (dict(ws=None), dict(ws=ODD), dict(nbytes=1000), dict(nbytes=need - 17)):
        assert _attend(pg=long, **kw) == bc.BC_ERR_WORKSPACE, kw
    size = bc.bc_paged_workspace_bytes
    assert size(shape(d=96), 5, 5, 100) == 0 and size(shape(), 5, -1, 100) == 0 and size(shape(), -1, 5, 100) == 0 and size(shape(), 1 << 31, 5, 100) == 0
    assert size(shape(), 5, 5, 0) == 0 and size(shape(B=(1 << 23) + 1), 5, 5, 100) == 0
    # (more columns than 31 bits count)
    assert size(shape(Hq=8, Hkv=1), 1 << 30, 1 << 29, 1 << 30) == 0
    assert _attend(s=shape(Hq=8, Hkv=1), rows=1 << 30, max_new=1 << 29, pg=_pages(pages=1, table_pages=1 << 24, page_rows=64)) == bc.BC_ERR_SHAPE


def test_workspace_goes_by_the_rows_there_are():
    # one long chunk among many sequences with a row or none: what its own call needs and the others' share
    for B, Hq, Hkv, n in ((128, 4, 1, 4096), (64, 12, 2, 512), (64, 32, 8, 40)):
        for d in (64, 128):
            alone = bc.bc_paged_workspace_bytes(shape(Hq, Hkv, d), n, n, 8192)
            got = bc.bc_paged_workspace_bytes(shape(Hq, Hkv, d, B=B), n + B - 1, n, 8192)
            assert 16 <= got <= max(alone, 16) * (n + B - 1) / n + 64, (B, n, d, got, alone)


@pytest.mark.parametrize("d", [64, 128])
def test_workspace_has_an_end(d):
    # parts are worth their memory where a call does not fill the chip; chunks of thousands of rows, also over a table that could hold far more than they need
    for B, n, longest in ((5, 8200, 131072), (2, 4097, 1 << 20), (17, 8200, 1 << 20), (81, 6028, 1 << 20), (1, 1 << 20, 1 << 20), (512, 4096, 1 << 26), (4, 2048, 30000),
                          (1, 512, 7680), (69, 15, 27900), (1 << 20, 1, 1 << 20), (300, 9, 1 << 20)):
        for Hq, Hkv in ((32, 8), (12, 2), (4, 1), (7, 7)):
            got = bc.bc_paged_workspace_bytes(shape(Hq, Hkv, d, B=B), B * n, n, longest)
            assert 16 <= got <= (256 << 20) + 16, (B, n, longest, Hq, Hkv, got)
    # (512 rows over 7680 in four parts, as measured)
    assert bc.bc_paged_workspace_bytes(shape(32, 8, 128, B=1), 512, 512, 7680) == 4 * 512 * 32 * 130 * 4 + 16


def test_struct_layout_matches_the_header(tmp_path):
    import os
    import shutil
    import subprocess
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no host C compiler")
    src = tmp_path / "layout.c"
    names = [f[0] for f in bc.bc_pages._fields_]
    src.write_text('#include <stdio.h>\n#include "bc.h"\nint main(void) {\n  printf("%zu", sizeof(bc_pages));\n' +
                   "".join('  printf(" %%zu", offsetof(bc_pages, %s));\n' % n for n in names) + "  return 0;\n}\n")
    exe = tmp_path / "layout"
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.check_call([cc, "-std=c99", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)])
    got = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    assert got == [C.sizeof(bc.bc_pages)] + [getattr(bc.bc_pages, n).offset for n in names]


def _host_cache(**kw):
    f = dict(B=3, Hq=4, Hkv=2, d=64, pages=9, page_rows=32, table_pages=4, device="cpu")
    f.update(kw)
    return bc.PagedCache(**f)


def test_binding_refuses_what_the_library_cannot_see(monkeypatch):
    for kw in (dict(page_rows=24), dict(page_rows=8), dict(pages=0), dict(table_pages=0), dict(B=0), dict(table=torch.zeros(3, 4)),
               dict(table=torch.zeros(3, 5, dtype=torch.int32))):
        with pytest.raises(bc.BcError):
            _host_cache(**kw)
    cache = _host_cache()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: None)
    qkv, pos, freq = torch.zeros(3, 512, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32), torch.zeros(32)
    # tensors of the wrong type, length, place or order (here: on the host)
    for args in ((qkv[:, :500], pos, freq), (qkv[0], pos, freq), (qkv, pos, freq), (qkv.half(), pos, freq)):
        with pytest.raises(bc.BcError):
            cache.append(*args)
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    for bad in (q.float(), q[:, :3], q.transpose(0, 1)):
        with pytest.raises(bc.BcError):
            cache.attend(bad)
    for kw in (dict(row_offsets=[0, 1, 2]), dict(row_offsets=[0, 2, 1, 3]), dict(row_offsets=[0, 1, 2, 4]), dict(row_offsets=[-1, 1, 2, 3]),
               dict(active=torch.ones(3)), dict(active=torch.ones(2, dtype=torch.uint8)), dict(out=torch.zeros(3, 4, 64).double())):
        with pytest.raises(bc.BcError):
            cache.attend(q, **kw)
    with pytest.raises(bc.BcError):
        cache.attend(q[:2])
