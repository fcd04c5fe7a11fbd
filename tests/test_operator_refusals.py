"""What the calls around the attention refuse (host logic only: no GPU needed; addresses are made up and never dereferenced)."""
import numpy as np
import pytest
import torch

from paper_2510_13797_amd import bc

PTR = 0x7F0000100000
ODD = PTR + 4


def shape(Hq=4, Hkv=2, d=64, dtype=bc.BC_BF16, B=1, scale=1.0):
    return bc.bc_shape(B, Hq, Hkv, d, dtype, scale)


def _rope(s=None, rows=3, qkv=PTR - 4096, stride=512, pos=PTR, freq=PTR, rot=64, qw=PTR, kw=PTR, eps=1e-6, q=PTR, k=PTR, v=PTR):
    return bc.bc_qk_norm_rope(s or shape(), rows, qkv, stride, pos, freq, rot, qw, kw, eps, q, k, v, None)


def _rope_bwd(s=None, rows=3, qkv=PTR, stride=512, pos=PTR, freq=PTR, rot=64, qw=PTR, kw=PTR, eps=1e-6, dq=PTR, dk=PTR, dv=PTR,
              dqkv=PTR, dstride=512, dqw=PTR, dkw=PTR, ws=PTR, nbytes=1 << 30):
    return bc.bc_qk_norm_rope_bwd(s or shape(), rows, qkv, stride, pos, freq, rot, qw, kw, eps, dq, dk, dv, dqkv, dstride, dqw, dkw,
                                  ws, nbytes, None)


@pytest.mark.parametrize("call", [_rope, _rope_bwd])
def test_rope_refusals_of_both_directions(call):
    bc.load()
    for kw in (dict(Hq=5), dict(Hkv=0), dict(d=96), dict(d=256), dict(dtype=2), dict(Hq=18)):
        assert call(s=shape(**kw)) == bc.BC_ERR_SHAPE, kw
    for rot in (-8, 4, 12, 72):
        assert call(rot=rot) == bc.BC_ERR_SHAPE, rot
    assert call(rows=-1) == bc.BC_ERR_SHAPE and call(rows=1 << 31) == bc.BC_ERR_SHAPE
    for eps in (-1e-6, float("nan"), float("inf")):
        assert call(eps=eps) == bc.BC_ERR_ARG
    for kw in (dict(pos=None), dict(freq=None), dict(stride=511), dict(stride=516), dict(stride=504), dict(stride=0), dict(stride=-512),
               dict(qw=ODD), dict(kw=ODD), dict(qkv=None), dict(qkv=ODD), dict(stride=1 << 40)):
        assert call(**kw) == bc.BC_ERR_ARG, kw


def test_rope_refusals_of_one_direction():
    other = PTR + 4096
    for kw in (dict(q=None), dict(k=None), dict(q=ODD), dict(k=ODD), dict(v=ODD), dict(qkv=other, q=other), dict(qkv=other, k=other),
               dict(qkv=other, v=other)):
        assert _rope(**kw) == bc.BC_ERR_ARG, kw
    for kw in (dict(dq=None), dict(dk=None), dict(dqkv=None), dict(dq=ODD), dict(dk=ODD), dict(dv=ODD), dict(dqkv=ODD), dict(dstride=510),
               dict(dstride=516), dict(dstride=520), dict(qw=None), dict(kw=None)):
        assert _rope_bwd(**kw) == bc.BC_ERR_ARG, kw
    need = bc.bc_qk_norm_rope_bwd_workspace_bytes(shape())
    assert need > 0 and bc.bc_qk_norm_rope_bwd_workspace_bytes(shape(d=96)) == 0
    for kw in (dict(ws=None), dict(ws=ODD), dict(nbytes=need - 1)):
        assert _rope_bwd(**kw) == bc.BC_ERR_WORKSPACE, kw


def test_rope_binding_refuses_what_the_library_cannot_see():
    # tensors of the wrong type, length, place or order (here: on the host)
    qkv, pos, freq = torch.zeros(3, 512, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32), torch.zeros(32)
    for args in ((qkv[:, :500], pos, freq), (qkv[0], pos, freq), (qkv, pos, freq), (qkv.half(), pos, freq)):
        with pytest.raises(bc.BcError):
            bc.qk_norm_rope(*args, 4, 2, 64)


def _cache(**kw):
    f = dict(k_slab=PTR, v_slab=PTR, base=PTR, cap=PTR, P=PTR, c=PTR, nb=PTR, w=PTR, err=PTR, max_cap=64, order=None, uniform_P=0,
             uniform_cap=0, rows_per_workgroup=0, plan=0)
    f.update(kw)
    return bc.bc_cache(**f)


def _prompt(s=None, c=None, k=PTR, v=PTR, q=PTR, off=(0, 3, 8), out=PTR, active=None, ws=PTR, nbytes=1 << 40):
    host = None if off is None else np.asarray(off, np.int64)
    return bc.bc_prompt_step(s or shape(B=2), c or _cache(), k, v, q, None if off is None else host.ctypes.data, out, active, ws, nbytes,
                             None)


def test_prompt_refusals():
    bc.load()
    for kw in (dict(Hq=5), dict(Hkv=0), dict(d=96), dict(dtype=bc.BC_F32), dict(Hq=18)):
        assert _prompt(s=shape(B=2, **kw)) == bc.BC_ERR_SHAPE, kw
    for field in ("k_slab", "v_slab", "base", "cap", "P", "c", "nb", "w", "err"):
        assert _prompt(c=_cache(**{field: None})) == bc.BC_ERR_ARG, field
    assert _prompt(c=_cache(max_cap=0)) == bc.BC_ERR_ARG
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert _prompt(s=shape(B=2, scale=scale)) == bc.BC_ERR_ARG
    for kw in (dict(k=None), dict(v=None), dict(q=None), dict(out=None), dict(k=ODD), dict(v=ODD), dict(q=ODD), dict(out=ODD), dict(off=None),
               dict(off=(0, 3, 2)), dict(off=(-1, 3, 8))):
        assert _prompt(**kw) == bc.BC_ERR_ARG, kw
    assert _prompt(off=(0, 1 << 30, 1 << 30)) == bc.BC_ERR_SHAPE
    need = bc.bc_prompt_workspace_bytes(shape(B=2), 5, 8, 64)
    assert need >= 8
    for kw in (dict(ws=None), dict(ws=ODD), dict(nbytes=need - 1)):
        assert _prompt(**kw) == bc.BC_ERR_WORKSPACE, kw
    # nothing to do is no error
    assert _prompt(off=(4, 4, 4), k=None, v=None, q=None, out=None, ws=None) == bc.BC_OK
    assert bc.bc_prompt_workspace_bytes(shape(d=96), 5, 8, 64) == 0 and bc.bc_prompt_workspace_bytes(shape(), -1, 8, 64) == 0
    assert bc.bc_prompt_workspace_bytes(shape(), 5, 8, 0) == 0


def test_prompt_refuses_what_grids_and_32_bit_offsets_do_not_hold():
    # (2^23 + 1 sequences; rows of 131,072 heads, 32 of which pass 32 bits at 2^19)
    off = np.ones((1 << 23) + 2, np.int64)
    off[0] = 0
    assert _prompt(s=shape(B=(1 << 23) + 1, Hq=1, Hkv=1), off=off) == bc.BC_ERR_SHAPE
    for B in (2, 1 << 21):
        assert _prompt(s=shape(B=B, Hq=1 << 17, Hkv=1 << 14), off=np.arange(B + 1)) == bc.BC_ERR_SHAPE


def _sample(B=2, V=100, z=PTR, dtype=bc.BC_BF16, stride=100, t=None, k=None, p=None, m=None, u=PTR, active=None, tokens=PTR, logprob=None):
    return bc.bc_sample_tokens(B, V, z, dtype, stride, t, k, p, m, u, active, tokens, logprob, None)


def test_sample_refusals():
    bc.load()
    for kw in (dict(B=-1), dict(V=0), dict(V=(1 << 20) + 1, stride=1 << 21), dict(dtype=2)):
        assert _sample(**kw) == bc.BC_ERR_SHAPE, kw
    for kw in (dict(z=None), dict(z=PTR + 1), dict(z=PTR + 2, dtype=bc.BC_F32), dict(u=None), dict(tokens=None), dict(stride=99), dict(stride=-100)):
        assert _sample(**kw) == bc.BC_ERR_ARG, kw
    assert _sample(B=0, z=None, u=None, tokens=None) == bc.BC_OK
    z, u = torch.zeros(2, 100), torch.zeros(2)
    for args in ((z, u), (z[0], u), (z.t(), u)):               # (on the host, wrong orders)
        with pytest.raises(bc.BcError):
            bc.sample_tokens(*args)


def test_prompt_workspace_goes_by_the_rows_there_are():
    # one long chunk among short ones or among slots without rows: no more than the long one's own call, the tables and the short rows' share
    for B, Hq, Hkv, n in ((128, 4, 1, 4096), (64, 8, 1, 2048), (50, 12, 2, 4096), (64, 12, 2, 512), (256, 4, 1, 10000), (64, 32, 8, 7)):
        for d in (64, 128):
            for short in (0, 1):
                total = n + short * (B - 1)
                alone = bc.bc_prompt_workspace_bytes(shape(Hq=Hq, Hkv=Hkv, d=d), n, n, 32768)
                got = bc.bc_prompt_workspace_bytes(shape(Hq=Hq, Hkv=Hkv, d=d, B=B), n, total, 32768)
                # (sums, a maximum and a sum for every part of a row and head; several sequences are cut into half as many parts again, and into two
                # where the one alone is not cut; 20 bytes a sequence of tables, ends of 16)
                assert got <= 1.5 * alone * total / n + 2 * 4 * total * Hq * (d + 2) + 20 * B + 64, (B, Hq, Hkv, n, d, short, got, alone)


def test_prompt_limits_are_those_of_its_workspace():
    # chunks on either side of a limit: no size for what the step refuses
    most = 65535 * 128
    for s, n, total, fits in ((shape(Hq=8, Hkv=1), most // 8, most // 8, True), (shape(Hq=8, Hkv=1), most // 8 + 1, most // 8 + 1, False),
                              (shape(Hq=512, Hkv=512), (1 << 22) - 1, 1 << 22, True), (shape(Hq=512, Hkv=512), 1 << 22, 1 << 22, False),
                              (shape(B=400), most // 2, (1 << 31) - 1, True), (shape(B=400), most // 2, 1 << 31, False),
                              (shape(Hq=1 << 16, Hkv=1 << 13), 5, 5, True), (shape(Hq=1 << 17, Hkv=1 << 14), 5, 5, False),
                              (shape(Hq=1, Hkv=1, B=1 << 23), 1, 1 << 23, True), (shape(Hq=1, Hkv=1, B=(1 << 23) + 1), 1, (1 << 23) + 1, False),
                              (shape(dtype=bc.BC_F32), 5, 5, False), (shape(), 1 << 62, 1 << 62, False)):
        got = bc.bc_prompt_workspace_bytes(s, n, total, 64)
        assert (got > 0) == fits, (s.B, s.Hq, s.Hkv, n, total, got)
        if s.B == 1 and s.kv_dtype == bc.BC_BF16 and n < 1 << 60:     # (what fits goes on to the check of the workspace)
            assert _prompt(s=s, off=(0, n), nbytes=0) == (bc.BC_ERR_WORKSPACE if fits else bc.BC_ERR_SHAPE)


def test_sample_refuses_more_rows_than_a_grid_holds():
    assert _sample(B=1 << 22, V=1, stride=1) == bc.BC_ERR_SHAPE
    assert _sample(B=(1 << 22) - 1, V=1, stride=1, u=None) == bc.BC_ERR_ARG            # (goes on to what follows)
