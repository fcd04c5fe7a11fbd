"""GPU parity: bc_qk_norm_rope / bc_qk_norm_rope_bwd against the fp64 oracle.

The kernels work in fp32 and round once.  An output carries half a step of its type, and of fp32 arithmetic some twenty roundings
(a sum of eight squares a lane, four exchanges, root and quotient, the products; the angles' cos and sin are good to 2e-7) relative to
the terms that are added: 20 * 2^-24 = 1.2e-6, 3e-6 where the norm's factor enters three times (the gradient of x).  A weight's
gradient adds terms one after the other in a lane, at most forty here, then over lanes: (40 + 60) * 2^-24 = 6e-6 of the sum of magnitudes."""
import numpy as np
import pytest

from oracle import rope as OR

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch.device("cuda:0")


def _case(dev, R, Hq, Hkv, d, dtype, rot, norm=(True, True), pad=0, far=1 << 20, seed=0, scale=1.0):
    import torch
    r = np.random.default_rng([seed, R, Hq, d])
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    width = (Hq + 2 * Hkv) * d
    wide = torch.from_numpy((scale * r.standard_normal((R, width + pad))).astype(np.float32)).to(dev).to(tdt)
    pos = torch.from_numpy(r.integers(0, far, R).astype(np.int32)).to(dev)
    freq = torch.tensor([1e6 ** (-2.0 * i / max(rot, 1)) for i in range(rot // 2)], dtype=torch.float32, device=dev)
    w = [torch.from_numpy((1 + 0.3 * r.standard_normal(d)).astype(np.float32)).to(dev).to(tdt) if n else None for n in norm]
    g = [torch.from_numpy(r.standard_normal((R, h, d)).astype(np.float32)).to(dev) for h in (Hq, Hkv, Hkv)]
    return wide[:, :width], pos, freq, w, g


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _half(dtype):
    return 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24


def _pair_sum(a, rot):
    a = np.abs(a)
    h = rot // 2
    out = a.copy()
    out[..., :h] = out[..., h:2 * h] = a[..., :h] + a[..., h:2 * h]
    return out


def _check(dev, R, Hq, Hkv, d, dtype, rot, norm=(True, True), eps=1e-6, backward=True, **kw):
    import torch
    from paper_2510_13797_amd import bc
    qkv, pos, freq, w, g = _case(dev, R, Hq, Hkv, d, dtype, rot, norm, **kw)
    before = qkv.clone()
    q, k, v = bc.qk_norm_rope(qkv, pos, freq, Hq, Hkv, d, *w, eps=eps)
    x = _np(qkv).reshape(R, Hq + 2 * Hkv, d)
    parts = (x[:, :Hq], x[:, Hq:Hq + Hkv])
    P, F, half = _np(pos), _np(freq), _half(dtype)
    for got, xi, wi in zip((q, k), parts, w):
        assert got.dtype == qkv.dtype and got.is_contiguous()
        ref = OR.norm_rope(xi, _np(wi), P, F, eps)
        y = OR.norm_rope(xi, _np(wi), P * 0, F, eps)
        bad = np.abs(_np(got) - ref) > half * np.abs(ref) + 1.2e-6 * _pair_sum(y, rot)
        assert not bad.any(), (int(bad.sum()), float(np.abs(_np(got) - ref).max()))
    assert torch.equal(v, qkv.unflatten(1, (Hq + 2 * Hkv, d))[:, Hq + Hkv:])
    if backward:
        dqkv, *dw = bc.qk_norm_rope_bwd(qkv, *g, pos, freq, Hq, Hkv, d, *w, eps=eps)
        dx = _np(dqkv).reshape(x.shape)
        at = 0
        for xi, wi, gi, dwi in zip(parts, w, g, dw):
            ref, refw = OR.norm_rope_grad(xi, _np(wi), P, F, eps, _np(gi))
            mag = _pair_sum(_np(gi), rot)
            if wi is None:
                assert dwi is None
            else:
                r = 1 / np.sqrt((xi * xi).mean(-1, keepdims=True) + eps)
                sums = (mag * np.abs(xi) * r).sum(axis=(0, 1))
                assert (np.abs(_np(dwi) - refw) <= 6e-6 * sums + 2.0 ** -24 * np.abs(refw)).all()
                a = np.abs(_np(wi)) * mag
                mag = r * (a + np.abs(xi) * r * r * (a * np.abs(xi)).mean(-1, keepdims=True))
            got = dx[:, at:at + xi.shape[1]]
            at += xi.shape[1]
            bad = np.abs(got - ref) > half * np.abs(ref) + 3e-6 * mag
            assert not bad.any(), (int(bad.sum()), float(np.abs(got - ref).max()))
        assert torch.equal(dqkv.unflatten(1, (Hq + 2 * Hkv, d))[:, at:], g[2].to(qkv.dtype))
    assert torch.equal(qkv, before)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,Hq,Hkv,d,rot", [(1, 4, 1, 64, 64), (1, 32, 8, 128, 128), (3, 5, 1, 128, 96), (67, 12, 2, 128, 8),
                                            (129, 14, 2, 64, 32), (200, 8, 2, 64, 0), (33, 7, 7, 128, 120)])
def test_shapes_and_rotated_parts(dev, dtype, R, Hq, Hkv, d, rot):
    _check(dev, R, Hq, Hkv, d, dtype, rot)


@pytest.mark.parametrize("norm", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("dtype,pad", [("bf16", 8), ("f32", 20)])
def test_without_weights_and_with_rows_apart(dev, norm, dtype, pad):
    _check(dev, 37, 12, 2, 128, dtype, 96, norm=norm, pad=pad)


@pytest.mark.parametrize("R", [2047, 2049, 5000])
def test_items_of_several_heads(dev, R):
    # 16 heads: an item is one head up to 4095 rows, two from 4096 on
    _check(dev, R, 12, 2, 64, "bf16", 64)


def test_whole_rows_as_items(dev):
    _check(dev, 33000, 4, 1, 64, "bf16", 64)


@pytest.mark.parametrize("dtype,R", [("bf16", 360000), ("f32", 180000)])
def test_rows_beyond_the_caches_are_those_of_smaller_calls(dev, dtype, R):
    # more than 256 MB of packed rows: the same arithmetic, past the caches
    import torch
    from paper_2510_13797_amd import bc
    Hq, Hkv, d = 4, 1, 64
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device=dev).manual_seed(3)
    qkv = torch.randn(R, 384, generator=g, device=dev).to(tdt)
    pos = torch.randint(0, 9000, (R,), generator=g, device=dev, dtype=torch.int32)
    freq = torch.tensor([1e4 ** (-i / 24.0) for i in range(24)], device=dev)
    w = [(1 + 0.2 * torch.randn(d, generator=g, device=dev)).to(tdt) for _ in range(2)]
    grads = [torch.randn(R, h, d, generator=g, device=dev) for h in (Hq, Hkv, Hkv)]
    whole = bc.qk_norm_rope(qkv, pos, freq, Hq, Hkv, d, *w) + bc.qk_norm_rope_bwd(qkv, *grads, pos, freq, Hq, Hkv, d, *w)
    dw = [torch.zeros(d, dtype=torch.float64, device=dev) for _ in range(2)]
    for lo in range(0, R, 90001):
        rows = slice(lo, min(lo + 90001, R))
        part = bc.qk_norm_rope(qkv[rows], pos[rows], freq, Hq, Hkv, d, *w)
        part += bc.qk_norm_rope_bwd(qkv[rows], *(x[rows] for x in grads), pos[rows], freq, Hq, Hkv, d, *w)
        assert all(torch.equal(a[rows], b) for a, b in zip(whole[:4], part))
        dw = [a + b.double() for a, b in zip(dw, part[4:])]
    for a, b in zip(whole[4:], dw):
        # sums of up to 1.4 million terms of a magnitude near one, by lanes of some hundred each: (100 + 60) * 2^-24 of the sum of magnitudes, both
        assert (a.double() - b).abs().max() <= 2 * 160 * 2.0 ** -24 * 1.5 * R * Hq


def test_small_and_large_values(dev):
    _check(dev, 20, 4, 1, 128, "f32", 128, scale=1e-12)          # the mean square far below eps
    _check(dev, 20, 4, 1, 128, "f32", 128, scale=1e-6, eps=0.0)
    _check(dev, 20, 4, 1, 128, "bf16", 128, scale=1e6)


def test_elements_that_do_not_turn_keep_clear_of_others(dev):
    import torch
    from paper_2510_13797_amd import bc
    # without norms an infinity or NaN stays in its pair
    qkv, pos, freq, w, _ = _case(dev, 9, 4, 1, 64, "bf16", 32, norm=(False, False))
    qkv[:, 40] = float("inf")
    qkv[:, 64 + 3] = float("nan")
    q, k, v = bc.qk_norm_rope(qkv, pos, freq, 4, 1, 64)
    bad = ~torch.isfinite(q)
    want = torch.zeros_like(bad)
    want[:, 0, 40] = want[:, 1, 3] = want[:, 1, 19] = True
    assert torch.equal(bad, want) and torch.isfinite(k).all() and torch.isfinite(v).all()


def test_no_rows(dev):
    import torch
    from paper_2510_13797_amd import bc
    qkv, pos, freq, w, g = _case(dev, 0, 4, 1, 64, "f32", 64)
    q, k, v = bc.qk_norm_rope(qkv, pos, freq, 4, 1, 64, *w)
    assert q.shape == (0, 4, 64) and k.shape == v.shape == (0, 1, 64)
    dqkv, dqw, dkw = bc.qk_norm_rope_bwd(qkv, *g, pos, freq, 4, 1, 64, *w)
    assert dqkv.shape == (0, 384) and not dqw.any() and not dkw.any()


def test_c_abi_forms(dev):
    import torch
    from paper_2510_13797_amd import bc
    # v left out; gradients in place of qkv, without those of v and of the weights; rows of the results apart
    qkv, pos, freq, w, g = _case(dev, 50, 4, 2, 64, "bf16", 64)
    p = lambda t: t.data_ptr()
    shape = bc.bc_shape(1, 4, 2, 64, bc.BC_BF16, 1.0)
    q, k, v = bc.qk_norm_rope(qkv, pos, freq, 4, 2, 64, *w)
    q2, k2 = torch.empty_like(q), torch.empty_like(k)
    assert bc.bc_qk_norm_rope(shape, 50, p(qkv), 512, p(pos), p(freq), 64, p(w[0]), p(w[1]), 1e-6, p(q2), p(k2), None, None) == 0
    torch.cuda.synchronize()
    assert torch.equal(q, q2) and torch.equal(k, k2)
    dqkv, dqw, dkw = bc.qk_norm_rope_bwd(qkv, *g, pos, freq, 4, 2, 64, *w)
    same = qkv.clone()
    assert bc.bc_qk_norm_rope_bwd(shape, 50, p(same), 512, p(pos), p(freq), 64, p(w[0]), p(w[1]), 1e-6, p(g[0]), p(g[1]), None,
                                  p(same), 512, None, None, None, 0, None) == 0
    wide = torch.full((50, 520), 7.0, dtype=torch.bfloat16, device=dev)
    ws = torch.empty(bc.bc_qk_norm_rope_bwd_workspace_bytes(shape), dtype=torch.uint8, device=dev)
    dkw2 = torch.empty_like(dkw)
    assert bc.bc_qk_norm_rope_bwd(shape, 50, p(qkv), 512, p(pos), p(freq), 64, p(w[0]), p(w[1]), 1e-6, p(g[0]), p(g[1]), p(g[2]),
                                  p(wide), 520, None, p(dkw2), p(ws), ws.numel(), None) == 0
    torch.cuda.synchronize()
    assert torch.equal(same[:, :384], dqkv[:, :384]) and torch.equal(same[:, 384:], qkv[:, 384:])
    assert torch.equal(wide[:, :512], dqkv) and (wide[:, 512:] == 7).all() and torch.equal(dkw2, dkw)


def test_results_are_the_same_again_and_in_a_graph(dev):
    import torch
    from paper_2510_13797_amd import bc
    qkv, pos, freq, w, g = _case(dev, 3000, 12, 2, 128, "bf16", 128)
    want = bc.qk_norm_rope(qkv, pos, freq, 12, 2, 128, *w) + bc.qk_norm_rope_bwd(qkv, *g, pos, freq, 12, 2, 128, *w)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            got = bc.qk_norm_rope(qkv, pos, freq, 12, 2, 128, *w) + bc.qk_norm_rope_bwd(qkv, *g, pos, freq, 12, 2, 128, *w)
        for _ in range(3):
            for t in got:
                t.fill_(3.0)
            graph.replay()
            st.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            again = bc.qk_norm_rope(qkv, pos, freq, 12, 2, 128, *w)
            assert all(torch.equal(a, b) for a, b in zip(again, want))


@pytest.mark.parametrize("dtype,R", [("bf16", 360000), ("f32", 180000)])
def test_weight_gradients_of_many_rows(dev, dtype, R):
    """Against sums in 64 bits.  A row is an item and there are 32 * 1024 groups of lanes: a lane adds the terms of ceil(R / 32768) rows and of a row's
    heads, a workgroup those of 32 lanes, in 32 bits; a term carries the twenty roundings above.  Magnitudes: a term's are |p| + |q| of two normal
    numbers times |x| of a third, 1.6 * 0.8 at the mean: 10.5 in all for 360,000 rows of four heads.  A workgroup's own sum, of R * heads / 1024 products of
    variance one, would be missed: its deviation is three times the bound and more."""
    import torch
    from paper_2510_13797_amd import bc
    Hq, Hkv, d, rot = 4, 1, 64, 48
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device=dev).manual_seed(4)
    qkv = torch.randn(R, 384, generator=g, device=dev).to(tdt)
    pos = torch.randint(0, 9000, (R,), generator=g, device=dev, dtype=torch.int32)
    freq = torch.tensor([1e4 ** (-i / 24.0) for i in range(24)], device=dev)
    w = [(1 + 0.2 * torch.randn(d, generator=g, device=dev)).to(tdt) for _ in range(2)]
    grads = [torch.randn(R, h, d, generator=g, device=dev) for h in (Hq, Hkv, Hkv)]
    got = bc.qk_norm_rope_bwd(qkv, *grads, pos, freq, Hq, Hkv, d, *w)[1:]
    first = 0
    for heads, dwi, gi in zip((Hq, Hkv), got, grads):
        want, mag = (torch.zeros(d, dtype=torch.float64, device=dev) for _ in range(2))
        for lo in range(0, R, 60000):
            rows = slice(lo, min(lo + 60000, R))
            a = (pos[rows].double()[:, None] * freq.double())[:, None]
            x = qkv[rows].double().unflatten(1, (Hq + 2 * Hkv, d))[:, first:first + heads]
            x = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt()
            do = gi[rows].double()
            p, q, rest = do[..., :rot // 2], do[..., rot // 2:rot], do[..., rot:]
            want += (torch.cat([p * a.cos() + q * a.sin(), q * a.cos() - p * a.sin(), rest], -1) * x).sum((0, 1))
            mag += (torch.cat([p.abs() + q.abs(), p.abs() + q.abs(), rest.abs()], -1) * x.abs()).sum((0, 1))
        first += heads
        bound = (-(-R // 32768) * heads + 32 + 20) * 2.0 ** -24 * mag
        err = (dwi.double() - want).abs()
        assert (err <= bound).all(), (heads, err.max().item(), bound.max().item())
        assert bound.max().item() < (R * heads / 1024) ** 0.5 / 3
