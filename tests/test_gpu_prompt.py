"""GPU parity: bc_prompt_step against the fp64 oracle.

Softmax weights enter the value product in two bf16 parts (relative error 2^-17), scores are fp32 sums of up to 128 products and go through a
2^x of one step: relative error of a weight below 2e-5 in all, so outputs of N(0,1) values (below 5 in magnitude) are off by less
than 1e-4.  Rows in the slab and tables are exact."""
import numpy as np
import pytest

from oracle import attention as OA

pytestmark = pytest.mark.gpu
TOL = 1e-4


@pytest.fixture(scope="module")
def dev():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch.device("cuda:0")


def _runtime(dev, Hq, Hkv, d, lens, cap, c=16, seed=0):
    """Caches that hold lens = [(P, nb, w)] rows; rows beyond are NaN."""
    import torch
    from paper_2510_13797_amd import bc
    P, nb, w = (np.array(x, np.int32) for x in zip(*lens))
    rt = bc.Runtime(len(P), Hq, Hkv, d, "bf16", 1.0 / np.sqrt(d), P, np.full(len(P), c), cap, dev)
    g = torch.Generator(device=dev).manual_seed(seed)
    for s in range(len(P)):
        L, E = int(P[s] + nb[s] + w[s]), Hkv * d
        for slab in (rt.k_slab, rt.v_slab):
            at = int(rt.base_host[s]) * E
            slab[at:at + int(cap[s]) * E].view(Hkv, int(cap[s]), d)[:, :L] = torch.randn(Hkv, L, d, generator=g, device=dev).bfloat16()
    rt.set_tables(nb, w)
    return rt


def _rows(dev, rt, rows, seed=1):
    import torch
    g = torch.Generator(device=dev).manual_seed(seed)
    return tuple(torch.randn(rows, h, rt.d, generator=g, device=dev).bfloat16() for h in (rt.Hkv, rt.Hkv, rt.Hq))


def _np(t):
    return t.double().cpu().numpy()


def _check(dev, Hq, Hkv, d, lens, n, active=None, first=0, spare=3, cap=None, every=1):
    import torch
    B = len(lens)
    n = np.asarray(n)
    off = first + np.concatenate([[0], np.cumsum(n)])
    L = np.array([sum(x) for x in lens])
    cap = L + n + spare if cap is None else cap
    rt = _runtime(dev, Hq, Hkv, d, lens, cap)
    k, v, q = _rows(dev, rt, int(off[-1]))
    before = [rt.resident(s) for s in range(B)]
    out = torch.full((int(off[-1]), Hq, d), 7.0, device=dev)
    assert rt.prompt_step(k, v, q, off, active=active, out=out) is out
    nb, w, err = rt.tables()
    assert err == 0
    kn, vn, qn, got = _np(k), _np(v), _np(q), _np(out)
    assert (got[:first] == 7).all()
    Pn = rt.P.cpu().numpy()
    for s in range(B):
        K, V = before[s]
        rows = slice(int(off[s]), int(off[s + 1]))
        if n[s] == 0 or (active is not None and not active[s]):
            assert (Pn[s], nb[s], w[s]) == tuple(lens[s]) and (got[rows] == 7).all()
            continue
        assert (Pn[s], nb[s], w[s]) == (L[s] + n[s], 0, 0)
        K, V = np.concatenate([K, kn[rows]]), np.concatenate([V, vn[rows]])
        Kd, Vd = rt.resident(s)
        assert np.array_equal(Kd, K) and np.array_equal(Vd, V)
        for i in range(0, int(n[s]), every):
            ref = OA.decode_attention(qn[off[s] + i], K[:L[s] + i + 1], V[:L[s] + i + 1], rt.shape.scale)
            worst = np.abs(got[off[s] + i] - ref).max()
            assert worst <= TOL, (s, i, worst)


HEADS = [(4, 1, 64), (12, 2, 128), (32, 8, 128), (7, 7, 64), (5, 1, 128), (16, 2, 64)]


@pytest.mark.parametrize("Hq,Hkv,d", HEADS)
def test_few_rows(dev, Hq, Hkv, d):
    # up to 32 columns a pair: no cached row, one, around a tile's 32, several
    _check(dev, Hq, Hkv, d, [(0, 0, 0), (1, 0, 0), (20, 6, 5), (32, 0, 0), (33, 0, 0), (100, 40, 7)], [3, 1, 4, 2, 0, 4])
    _check(dev, Hq, Hkv, d, [(0, 0, 0)], [1])
    _check(dev, Hq, Hkv, d, [(1000, 100, 9)], [4])


@pytest.mark.parametrize("Hq,Hkv,d", HEADS)
def test_many_rows(dev, Hq, Hkv, d):
    _check(dev, Hq, Hkv, d, [(0, 0, 0), (31, 0, 0), (64, 0, 0), (50, 30, 16), (7, 1, 0)], [65, 33, 1, 130, 0], every=5)
    _check(dev, Hq, Hkv, d, [(700, 20, 3)], [97], every=7)


@pytest.mark.parametrize("n", [31, 32, 33, 63, 64, 65, 96, 127, 128, 129])
@pytest.mark.parametrize("L", [0, 32, 45])
def test_ends_of_tiles(dev, n, L):
    _check(dev, 4, 1, 128, [(L, 0, 0)], [n], every=3)
    _check(dev, 4, 4, 64, [(L, 0, 0)], [n], every=3)


@pytest.mark.parametrize("B", [40, 128, 129])
def test_more_sequences_than_travel_in_the_arguments(dev, B):
    r = np.random.default_rng(3)
    lens = [tuple(int(x) for x in (r.integers(0, 80), r.integers(0, 20), r.integers(0, 17))) for _ in range(B)]
    n = r.integers(0, 40, B)
    n[[0, B - 1]] = 0, 5
    _check(dev, 12, 2, 64, lens, n, active=(r.random(B) < 0.8).astype(np.uint8), every=3)
    _check(dev, 12, 2, 128, lens, np.minimum(n, 5), every=2)


def test_ragged_chunks_in_parts(dev):
    # parts whose sums are folded by their place in the output, sequences without rows between others
    r = np.random.default_rng(4)
    lens = [(int(x), 0, 0) for x in r.integers(0, 1500, 7)]
    for n in ([40, 0, 3, 130, 0, 17, 64], [0, 0, 33, 0, 0, 90, 0]):
        for cap in (np.full(7, 1700), np.full(7, 9000)):
            _check(dev, 12, 2, 128, lens, n, cap=cap, every=13)
            _check(dev, 4, 4, 64, lens, n, cap=cap, every=13)


def test_rows_behind_the_last_sequence_are_left_as_they_were(dev):
    import torch
    for n in (3, 40):
        rt = _runtime(dev, 4, 1, 64, [(20, 0, 0)], np.array([200]))
        k, v, q = _rows(dev, rt, n + 9)
        k[n:], v[n:], q[n:] = float("nan"), float("nan"), float("nan")
        out = torch.full((n + 9, 4, 64), 7.0, device=dev)
        rt.prompt_step(k, v, q, [0, n], out=out)
        assert (out[n:] == 7).all() and torch.isfinite(out[:n]).all() and rt.P.item() == 20 + n
        assert torch.isnan(rt.k_slab.view(200, 64)[20 + n:]).all() and torch.isfinite(rt.k_slab.view(200, 64)[:20 + n]).all()


def test_rows_in_front_and_idle_sequences(dev):
    _check(dev, 8, 2, 128, [(40, 2, 1), (9, 0, 0), (60, 0, 3)], [20, 11, 30], active=np.array([1, 0, 1], np.uint8), first=5, every=2)


def test_long_cache_in_parts(dev):
    _check(dev, 4, 1, 128, [(9000, 0, 0)], [5])
    _check(dev, 4, 1, 128, [(9000, 0, 0)], [70], every=23)
    # capacity far beyond what is resident: parts without tiles
    _check(dev, 4, 1, 64, [(3, 0, 0), (40, 0, 0)], [5, 6], cap=np.array([20000, 20000]))
    _check(dev, 4, 1, 64, [(3, 0, 0), (40, 0, 0)], [50, 60], cap=np.array([20000, 20000]), every=7)


def test_offsets_beyond_32_bits(dev):
    # the second sequence starts 4.9 GB into its slab, and its heads lie 1.2 GB apart
    cap = np.array([4800000, 4800000])
    _check(dev, 8, 4, 128, [(3, 0, 0), (77, 0, 2)], [4, 70], cap=cap, every=9)
    _check(dev, 8, 4, 128, [(3, 0, 0), (77, 0, 2)], [4, 7], cap=cap)


def test_peaked_rows(dev):
    # one key dominates, first or last: the reference of the running softmax has to move late
    import torch
    from paper_2510_13797_amd import bc
    for n in (4, 60):
        rt = _runtime(dev, 4, 1, 64, [(150, 0, 0)], np.array([300]))
        k, v, q = _rows(dev, rt, n)
        rt.k_slab.view(300, 64)[140] *= 16
        k[n // 2] *= 24
        K, V = rt.resident(0)
        got = _np(rt.prompt_step(k, v, q, [0, n]))
        K, V = np.concatenate([K, _np(k)]), np.concatenate([V, _np(v)])
        for i in range(n):
            ref = OA.decode_attention(_np(q)[i], K[:151 + i], V[:151 + i], rt.shape.scale)
            # (scores of a hundred: fp32 sums of that size are off by 128 * 2^-24 * 100 in the exponent)
            assert np.abs(got[i] - ref).max() <= 1e-3, i


def test_sequences_that_cannot_take_their_rows_are_left_alone(dev):
    import torch
    from paper_2510_13797_amd import bc
    for n in (3, 50):
        lens, cap = [(10, 0, 0), (20, 1, 17), (12, 0, 2)], np.array([10 + n - 1, 200, 14 + n])
        rt = _runtime(dev, 4, 1, 64, lens, cap)
        k, v, q = _rows(dev, rt, 3 * n)
        keep = [x.clone() for x in (rt.k_slab, rt.v_slab)]
        out = torch.full((3 * n, 4, 64), 7.0, device=dev)
        rt.prompt_step(k, v, q, [0, n, 2 * n, 3 * n], out=out)
        nb, w, err = rt.tables()
        assert err == bc.BC_ERRBIT_CAPACITY | bc.BC_ERRBIT_STATE
        assert rt.P.tolist() == [10, 20, 14 + n] and list(nb) == [0, 1, 0] and list(w) == [0, 17, 0]
        assert (out[:2 * n] == 7).all() and torch.isfinite(out[2 * n:]).all() and not (out[2 * n:] == 7).all()
        own = int(rt.base_host[2]) * 64
        for slab, old in zip((rt.k_slab, rt.v_slab), keep):
            assert torch.equal(slab[:own].view(torch.int16), old[:own].view(torch.int16))


def test_pieces_give_what_the_whole_prompt_gives(dev):
    # a prompt in three chunks against the training-time attention without windows, then decode steps over either
    import torch
    from paper_2510_13797_amd import bc
    n, Hq, Hkv, d = 213, 12, 2, 128
    rt = _runtime(dev, Hq, Hkv, d, [(0, 0, 0)], np.array([400]), c=4)
    k, v, q = _rows(dev, rt, n)
    whole, _ = bc.prefill_attn(q, k, v, [0, n], [n], [0], Hq, Hkv, d, rt.shape.scale)
    outs = []
    for lo, hi in ((0, 100), (100, 103), (103, n)):
        outs.append(rt.prompt_step(k[lo:hi], v[lo:hi], q[lo:hi], [0, hi - lo]))
    assert (torch.cat(outs) - whole).abs().max().item() <= 2 * TOL
    other = bc.Runtime(1, Hq, Hkv, d, "bf16", rt.shape.scale, [n], [4], [400], dev)
    other.cache_init([k.float().cpu().numpy()], [v.float().cpu().numpy()])
    for t in range(10):
        x = [y[:1].contiguous() for y in _rows(dev, rt, 1, seed=50 + t)]
        bk, bv, _ = _rows(dev, rt, 1, seed=80 + t)
        assert torch.equal(rt.decode_step(*x, bk, bv).clone(), other.decode_step(*x, bk, bv).clone())
    assert [list(y) for y in rt.tables()[:2]] == [list(y) for y in other.tables()[:2]] == [[2], [2]]


def test_decode_steps_behind_a_chunk_in_a_uniform_layout(dev):
    # equal prompts and capacities are told the library, which asks for prompt rows before the tables: chunks move the tables away from that
    import torch
    from paper_2510_13797_amd import bc
    Hq, Hkv, d, n = 12, 2, 128, [30, 7]
    rt = _runtime(dev, Hq, Hkv, d, [(40, 0, 0), (40, 0, 0)], np.array([200, 200]), c=4)
    assert rt.cache.uniform_P == 40
    k, v, q = _rows(dev, rt, sum(n))
    rt.prompt_step(k, v, q, [0, n[0], sum(n)])
    K, V = zip(*(rt.resident(s) for s in range(2)))
    other = bc.Runtime(2, Hq, Hkv, d, "bf16", rt.shape.scale, [70, 47], [4, 4], [200, 200], dev)
    other.cache_init(list(K), list(V))
    for t in range(9):
        x, b = _rows(dev, rt, 2, seed=50 + t), _rows(dev, rt, 2, seed=80 + t)
        assert torch.equal(rt.decode_step(*x, *b[:2]).clone(), other.decode_step(*x, *b[:2]).clone()), t
    assert rt.tables()[2] == other.tables()[2] == 0


def test_two_calls_at_once(dev):
    # two batches of caches on two streams, each with a workspace of its own
    import torch
    for n in (3, 60):
        lens = [(700, 0, 0), (30, 2, 1)]
        rts = [_runtime(dev, 12, 2, 128, lens, np.array([1500, 1500]), seed=i) for i in range(2)]
        k, v, q = _rows(dev, rts[0], 2 * n)
        want = []
        for rt in rts:
            start = [t.clone() for t in (rt.P, rt.nb, rt.w)]
            want.append(rt.prompt_step(k, v, q, [0, n, 2 * n]).clone())
            for t, s in zip((rt.P, rt.nb, rt.w), start):
                t.copy_(s)
        torch.cuda.synchronize()
        got = []
        for rt in rts:
            with torch.cuda.stream(torch.cuda.Stream()):
                got.append(rt.prompt_step(k, v, q, [0, n, 2 * n]))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_captured_and_replayed(dev):
    import torch
    lens = [(100, 3, 2), (5, 0, 0)]
    for n in ((3, 2), (90, 40)):
        rt = _runtime(dev, 12, 2, 128, lens, np.array([2000, 2000]))
        start = torch.stack([rt.P, rt.nb, rt.w]).clone()
        tables = start.clone()
        rt.P, rt.nb, rt.w = tables[0], tables[1], tables[2]
        rt.cache.P, rt.cache.nb, rt.cache.w = rt.P.data_ptr(), rt.nb.data_ptr(), rt.w.data_ptr()
        k, v, q = _rows(dev, rt, sum(n))
        off = [0, n[0], sum(n)]
        want = rt.prompt_step(k, v, q, off).clone()
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=st):
                torch.add(start, 0, out=tables)
                out = rt.prompt_step(k, v, q, off)
            for _ in range(3):
                out.fill_(3.0)
                graph.replay()
                st.synchronize()
                assert torch.equal(out, want) and tables[0].tolist() == [105 + n[0], 5 + n[1]]
                rt.decode_attn(q[:2])                          # eager work between replays
                st.synchronize()
            assert rt.tables()[2] == 0


def test_resident_rows_behind_replays(dev):
    # every replay of a captured call appends its rows; `out` on another stream than its own
    import torch
    rt = _runtime(dev, 12, 2, 128, [(100, 0, 0)], np.array([400]))
    k, v, q = _rows(dev, rt, 5)
    out = torch.zeros(5, 12, 128, dtype=torch.float32, device=dev)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            rt.prompt_step(k, v, q, [0, 5], out=out)
        for n in (1, 2, 3):
            graph.replay()
            st.synchronize()
            K, V = rt.resident(0)
            assert K.shape[0] == 100 + 5 * n
            assert np.array_equal(K[-5:], k.float().cpu().numpy()) and np.array_equal(V[-5:], v.float().cpu().numpy())
    assert rt.tables()[2] == 0


@pytest.mark.parametrize("n", [[0] * 9 + [200] + [0] * 30, [1] * 9 + [300] + [2] * 30, [0] * 20 + [5] + [0] * 19, [3] * 10 + [0, 4, 1] + [0] * 27])
def test_few_of_many_sequences_within_the_workspace(dev, n):
    # one long chunk among short ones or none, few rows for few sequences; the workspace as large as asked for, and what lies behind it
    import torch
    from paper_2510_13797_amd import bc
    r = np.random.default_rng(6)
    B, Hq, Hkv, d = len(n), 12, 2, 64
    lens = [(int(x), 0, 0) for x in r.integers(0, 300, B)]
    for cap in (700, 9000):
        rt = _runtime(dev, Hq, Hkv, d, lens, np.full(B, cap))
        off = np.concatenate([[0], np.cumsum(n)]).astype(np.int64) + 3
        total = int(off[-1] - off[0])
        k, v, q = _rows(dev, rt, int(off[-1]))
        before = [rt.resident(s) for s in range(B)]
        nbytes = bc.bc_prompt_workspace_bytes(rt.shape, max(n), total, cap)
        ws = torch.full((nbytes + 4096,), 0x5a, dtype=torch.uint8, device=dev)
        out = torch.full((int(off[-1]), Hq, d), 7.0, device=dev)
        st = bc.bc_prompt_step(rt.shape, rt.cache, k.data_ptr(), v.data_ptr(), q.data_ptr(), off.ctypes.data, out.data_ptr(), None,
                               ws.data_ptr(), nbytes, torch.cuda.current_stream().cuda_stream)
        assert st == bc.BC_OK
        torch.cuda.synchronize()
        assert (ws[nbytes:] == 0x5a).all() and (out[:3] == 7).all() and rt.tables()[2] == 0
        kn, vn, qn, got = _np(k), _np(v), _np(q), _np(out)
        for s in range(B):
            K, V = before[s]
            rows = slice(int(off[s]), int(off[s + 1]))
            K, V = np.concatenate([K, kn[rows]]), np.concatenate([V, vn[rows]])
            for i in range(0, n[s], 1 if n[s] < 9 else 17):
                ref = OA.decode_attention(qn[off[s] + i], K[:lens[s][0] + i + 1], V[:lens[s][0] + i + 1], rt.shape.scale)
                assert np.abs(got[off[s] + i] - ref).max() <= TOL, (s, i)


@pytest.mark.parametrize("s", [11.1875, 11.3125, 12.375, 12.5, 14.125])
def test_parts_of_the_weights(dev, s):
    """Values of one everywhere, one key of weight 1 and three of a weight that two bf16 parts leave most of (an output is one but for that).  Up to 32 columns: three parts
    and fp32 sums of four keys, a step of 2^-23 for each addition of the parts' products, half a step for seven others: 31 * 2^-24; more columns: 2^-17 too."""
    import torch
    from paper_2510_13797_amd import bc
    few, many = 31 * 2.0 ** -24, 31 * 2.0 ** -24 + 2.0 ** -17
    bf = lambda x: torch.tensor(x, dtype=torch.float64).bfloat16().double().item()
    w = float(np.float32(2.0 ** ((s - 16.0) * 0.125 * np.log2(np.e))))
    left = w - bf(w) - bf(w - bf(w))
    assert few < 3 * abs(left) / (1 + 3 * w) < 2.0 ** -17              # two parts alone do not pass as three
    for n, bound in ((1, few), (8, few), (9, many), (70, many)):
        rt = bc.Runtime(1, 4, 1, 64, "bf16", 0.125, [3], [0], [100], dev)
        assert bc.bc_prompt_workspace_bytes(rt.shape, n, n, 100) <= 64          # (one part: nothing is folded)
        rt.k_slab.view(100, 64)[:3] = 0
        rt.k_slab.view(100, 64)[:3, 0] = s
        rt.v_slab.view(100, 64)[:3] = 1
        q = torch.zeros(n, 4, 64, dtype=torch.bfloat16, device=dev)
        q[..., 0] = 1
        k = torch.zeros(n, 1, 64, dtype=torch.bfloat16, device=dev)
        k[..., 0] = -4096                                              # (a weight of nothing,
        k[0, 0, 0] = 16                                                # the first one's is 1)
        got = rt.prompt_step(k, torch.ones_like(k), q, [0, n])
        assert (got.double() - 1).abs().max().item() <= bound, n
