"""GPU parity of the paged 8-bit cache: bc_paged_append and bc_paged_attend against the fp64 oracle.

What is appended without norm and rotation is exact: a scale is a power of two, a byte one rounding to nearest.  With them fp32 arithmetic comes first, off by less
than 2e-6 of the row's largest magnitude (a dozen operations of 2^-24 and a series good to 1e-7), so a value is off by half a step of e4m3 (2^-4 of it, 2^-10 of its scale
below 2^-6 of that) and 2e-6 of the largest; queries by half a step of bf16 (2^-8 of a value, as torch.finfo counts) and the same.
Attention reads exact values; a softmax weight enters its product in two half-precision parts (2^-22), scores are fp32 sums of up to 128 products behind a 2^x of one step:
a weight is off by less than 2e-5, outputs of N(0, 1) values (below 5 in magnitude) by less than 1e-4."""
import numpy as np
import pytest

from oracle import attention as OA
from oracle import paged as OP
from oracle import rope as OR

pytestmark = pytest.mark.gpu
TOL = 1e-4
HEADS = [(4, 1, 64), (12, 2, 128), (32, 8, 128), (7, 7, 64), (5, 1, 128), (16, 2, 64)]


@pytest.fixture(scope="module")
def dev():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch.device("cuda:0")


def _np(t):
    return t.double().cpu().numpy()


class Both:
    """A paged cache and its oracle, pages dealt out in no order, everything else left NaN."""

    def __init__(self, dev, B, Hq, Hkv, d, page, most, dtype="bf16", seed=0, spare=3):
        import torch
        from paper_2510_13797_amd import bc
        self.torch, self.dev, self.B, self.Hq, self.Hkv, self.d, self.page = torch, dev, B, Hq, Hkv, d, page
        per = -(-most // page)
        r = np.random.default_rng(seed)
        self.c = bc.PagedCache(B, Hq, Hkv, d, B * per + spare, page, per, dev, dtype=dtype)
        self.table = r.permutation(B * per + spare)[:B * per].reshape(B, per).astype(np.int32)
        self.c.table.copy_(torch.from_numpy(self.table))
        self.k, self.v = [OP.Sequence(Hkv, d) for _ in range(B)], [OP.Sequence(Hkv, d) for _ in range(B)]
        self.gen = torch.Generator(device=dev).manual_seed(seed)
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.empty = torch.zeros(0, device=dev)

    def packed(self, rows, size=1.0):
        return (size * self.torch.randn(rows, (self.Hq + 2 * self.Hkv) * self.d, generator=self.gen, device=self.dev)).to(self.dtype)

    def append(self, n, size=1.0, active=None, keep=None, first=0, packed=None, device_offsets=False):
        """Rows without norm and rotation, in the cache and in the oracle; -> (packed, q)."""
        torch = self.torch
        n = np.asarray(n)
        off = first + np.concatenate([[0], np.cumsum(n)])
        x = self.packed(int(off[-1]) + 2, size) if packed is None else packed
        pos = torch.zeros(len(x), dtype=torch.int32, device=self.dev)
        q = torch.full((len(x), self.Hq, self.d), 7.0, dtype=torch.bfloat16, device=self.dev)
        how = dict(row_offsets=torch.from_numpy(off).to(self.dev), max_new=int(n.max())) if device_offsets else dict(row_offsets=off)
        t = lambda a, dt: None if a is None else torch.from_numpy(np.asarray(a).astype(dt)).to(self.dev)
        assert self.c.append(x, pos, self.empty, active=t(active, np.uint8), keep=t(keep, np.int32), q=q, **how) is q
        h = _np(x).reshape(len(x), -1, self.d)
        for s in range(self.B):
            if n[s] and (active is None or active[s]):
                for seq, lo in ((self.k[s], self.Hq), (self.v[s], self.Hq + self.Hkv)):
                    seq.append(h[off[s]:off[s + 1], lo:lo + self.Hkv], None if keep is None else keep[s])
                expect = h[off[s]:off[s + 1], :self.Hq]
                assert np.array_equal(_np(q[off[s]:off[s + 1]]), _np(torch.from_numpy(expect).to(torch.bfloat16)))
            else:
                assert (q[off[s]:off[s + 1]] == 7).all()
        assert (q[:first] == 7).all() and (q[off[-1]:] == 7).all()
        return x, q

    def pool(self):
        return (self.c.k_pages.view(self.torch.uint8).cpu().numpy().copy(), self.c.v_pages.view(self.torch.uint8).cpu().numpy().copy(),
                self.c.k_scale.cpu().numpy().copy(), self.c.v_scale.cpu().numpy().copy())

    def check_pool(self, before):
        """Every byte and scale of the pool: the oracle's where a sequence has entries, as before elsewhere."""
        kb, vb, ks, vs = (x.copy() for x in before)
        d, page = self.d, self.page
        for s in range(self.B):
            for seq, pool, scales, place in ((self.k[s], kb, ks, OP.key_place), (self.v[s], vb, vs, OP.value_place)):
                for j in range(len(seq)):
                    p = self.table[s, j // page]
                    for h in range(self.Hkv):
                        pool[p, h].reshape(-1)[place(j % page, np.arange(d), d)] = OP.e4m3_byte(seq.values[h, j])
                for b in range(seq.scales.shape[1]):
                    scales[self.table[s, 16 * b // page], :, 16 * b % page // 16] = seq.scales[:, b]
        got = self.pool()
        for name, x, y in zip(("k", "v"), got[:2], (kb, vb)):
            wrong = np.argwhere((x != y) & ~((x & 0x7f == 0x7f) & (y & 0x7f == 0x7f)))
            assert not len(wrong), (name, len(wrong), wrong[:5])
        for name, x, y in zip(("k", "v"), got[2:], (ks, vs)):
            wrong = np.argwhere((x != y) & ~(np.isnan(x) & np.isnan(y)))
            assert not len(wrong), (name + " scales", len(wrong), wrong[:5])
        assert list(self.c.lengths.cpu().numpy()) == [len(x) for x in self.k]

    def check_attend(self, q, n, active=None, first=0, every=1, max_len=None, tol=TOL, device_offsets=False, scale=None):
        torch = self.torch
        n = np.asarray(n)
        off = first + np.concatenate([[0], np.cumsum(n)])
        out = torch.full((len(q), self.Hq, self.d), 7.0, device=self.dev)
        how = dict(row_offsets=torch.from_numpy(off).to(self.dev), max_new=int(n.max())) if device_offsets else dict(row_offsets=off)
        a = None if active is None else torch.from_numpy(np.asarray(active).astype(np.uint8)).to(self.dev)
        assert self.c.attend(q, active=a, out=out, max_len=max_len, **how) is out
        got, qn = _np(out), _np(q)
        assert (got[:first] == 7).all() and (got[off[-1]:] == 7).all()
        worst = 0.0
        for s in range(self.B):
            rows = slice(int(off[s]), int(off[s + 1]))
            if active is not None and not active[s]:
                assert (got[rows] == 7).all()
                continue
            K, V = self.k[s].numbers(), self.v[s].numbers()
            L = len(K)
            assert np.isfinite(got[rows]).all()
            for i in sorted(set(range(0, int(n[s]), every)) | ({int(n[s]) - 1} if n[s] else set())):
                e = L - int(n[s]) + i + 1
                ref = OA.decode_attention(qn[off[s] + i], K[:e], V[:e], self.c.shape.scale if scale is None else scale)
                worst = max(worst, np.abs(got[off[s] + i] - ref).max())
                assert worst <= tol, (s, i, worst)
        assert self.c.err.item() == 0
        return out


# ------------------------------------------------------------------ append
@pytest.mark.parametrize("Hq,Hkv,d", HEADS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_is_exact_without_norm_and_rotation(dev, Hq, Hkv, d, dtype):
    both = Both(dev, 5, Hq, Hkv, d, 32, 150, dtype)
    before = both.pool()
    both.append([0, 1, 16, 37, 70])                                     # chunks, a block's end, pages
    both.check_pool(before)
    both.append([5, 0, 3, 1, 2], size=30.0, active=[1, 1, 1, 0, 1], first=2)        # scales grow
    both.check_pool(before)
    for i in range(18):                                                 # a row a sequence, across blocks, scales that grow and do not
        both.append([1] * 5, size=(0.1, 4.0, 300.0)[i % 3], active=[1, 1, i % 2, 1, 1], device_offsets=i % 4 == 0)
    both.check_pool(before)
    both.append([17, 33, 1, 0, 2], size=0.01, device_offsets=True)
    both.check_pool(before)
    assert both.c.err.item() == 0


@pytest.mark.parametrize("Hq,Hkv,d", [(32, 8, 128), (7, 7, 64), (4, 1, 64)])
def test_append_without_queries(dev, Hq, Hkv, d):
    # the entry point itself, q NULL: however workgroups share the heads, the same entries
    import torch
    from paper_2510_13797_amd import bc
    for n in ([5, 30, 0], [300, 1, 17], [1, 1, 1]):
        both, other = (Both(dev, 3, Hq, Hkv, d, 32, 400, seed=9) for _ in range(2))
        x, _ = both.append(n)
        pos = torch.zeros(len(x), dtype=torch.int32, device=dev)
        off = torch.from_numpy(np.concatenate([[0], np.cumsum(n)])).to(dev)
        c = other.c
        assert bc.bc_paged_append(c.shape, c._c, len(x), off.data_ptr(), max(n), x.data_ptr(), x.stride(0), pos.data_ptr(), None, 0, None, None, 1e-6,
                                  None, None, None, torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(both.c.lengths, c.lengths)
        for a, b in zip(both.pool(), other.pool()):
            assert np.array_equal(a, b, equal_nan=a.dtype.kind == "f")


@pytest.mark.parametrize("page", [16, 64, 1024])
def test_append_a_row_each_without_offsets(dev, page):
    import torch
    both = Both(dev, 3, 12, 2, 128, page, 60)
    before = both.pool()
    for i in range(35):
        x = both.packed(3, 2.0 ** (i % 7))
        q = both.c.append(x, torch.zeros(3, dtype=torch.int32, device=dev), both.empty)
        h = _np(x).reshape(3, -1, 128)
        assert np.array_equal(_np(q), h[:, :12])
        for s in range(3):
            both.k[s].append(h[s:s + 1, 12:14])
            both.v[s].append(h[s:s + 1, 14:])
    both.check_pool(before)


def test_entries_behind_the_kept_ones_are_dropped(dev):
    both = Both(dev, 6, 4, 2, 64, 16, 120)
    both.append([40, 33, 20, 16, 90, 7])
    lengths = [40, 33, 20, 16, 90, 7]
    # a beacon in the place of its window: one row, from the middle of a block, its first entry, its last, the sequence's first, behind the last
    before = both.pool()
    both.append([1] * 6, size=9.0, keep=[24, 32, 3, 15, 77, 0], active=[1, 1, 1, 1, 0, 1])
    assert [len(x) for x in both.k] == [25, 33, 4, 16, 90, 1]
    both.check_pool(before)
    before = both.pool()                                                # (what is dropped now stays as it is by now)
    both.append([3, 20, 0, 17, 2, 1], keep=[25, 1, 4, 0, 80, 1], size=0.2)
    both.check_pool(before)
    assert both.c.err.item() == 0 and lengths[0] == 40


@pytest.mark.parametrize("Hq,Hkv,d,dtype,rot,norm", [(12, 2, 128, "bf16", 128, True), (4, 1, 64, "f32", 32, True), (14, 2, 64, "bf16", 8, False), (5, 1, 128, "f32", 96, False),
                                                     (32, 8, 128, "bf16", 128, True), (3, 3, 64, "bf16", 64, True)])
@pytest.mark.parametrize("rows", [(1, 1, 1), (30, 0, 47), (3, 1, 16)])
def test_append_with_norm_and_rotation(dev, Hq, Hkv, d, dtype, rot, norm, rows):
    import torch
    both = Both(dev, 3, Hq, Hkv, d, 16, 80, dtype)
    off = np.concatenate([[0], np.cumsum(rows)])
    wide = both.packed(int(off[-1]) * 2).view(int(off[-1]), -1)         # rows that lie apart
    x = wide[:, :(Hq + 2 * Hkv) * d]
    pos = torch.randint(0, 900000, (len(x),), generator=both.gen, device=dev, dtype=torch.int32)
    freq = torch.tensor([1e6 ** (-2.0 * i / rot) for i in range(rot // 2)], device=dev)
    w = [(1 + 0.2 * torch.randn(d, generator=both.gen, device=dev)).to(both.dtype) if norm else None for _ in range(2)]
    q = both.c.append(x, pos, freq, row_offsets=off, q_weight=w[0], k_weight=w[1])
    h = _np(x).reshape(len(x), -1, d)
    ref = [OR.norm_rope(h[:, lo:lo + n], None if u is None else _np(u), pos.cpu().numpy(), _np(freq), 1e-6) for lo, n, u in ((0, Hq, w[0]), (Hq, Hkv, w[1]))]
    most = np.abs(ref[0]).max(axis=-1, keepdims=True)
    assert (np.abs(_np(q) - ref[0]) <= 2.0 ** -8 * np.abs(ref[0]) + 3e-6 * most).all()
    for s in range(3):
        part = slice(int(off[s]), int(off[s + 1]))
        K, V = both.c.entries(s)
        exact = OP.Sequence(Hkv, d)
        exact.append(h[part, Hq + Hkv:])
        assert np.array_equal(V, exact.numbers()) and len(K) == rows[s]
        if not rows[s]:
            continue
        exact = OP.Sequence(Hkv, d)
        exact.append(ref[1][part])
        scale = both.c.k_scale[both.c.table[s].long()].cpu().numpy().transpose(1, 0, 2).reshape(Hkv, -1)[:, :exact.scales.shape[1]]
        for hh, b in np.argwhere(scale != exact.scales):                # only where the largest magnitude is at the border
            most = np.abs(ref[1][part][16 * b:16 * b + 16, hh]).max() / 448
            assert abs(np.log2(most) - np.rint(np.log2(most))) < 1e-5
        scale = np.repeat(scale, 16, axis=1)[:, :rows[s]].T[..., None]
        exact = ref[1][part]
        assert (np.abs(K - exact) <= 2.0 ** -4 * np.abs(exact) + 2.0 ** -10 * scale + 3e-6 * np.abs(exact).max(axis=-1, keepdims=True)).all()


def test_what_is_not_finite(dev):
    import torch
    both = Both(dev, 2, 2, 1, 64, 16, 40)
    x = both.packed(22)
    x[3, 2 * 64 + 5], x[4, 3 * 64 + 6], x[20, 3 * 64 + 1], x[5, 2 * 64] = float("inf"), float("nan"), float("-inf"), float("nan")
    before = both.pool()
    both.append([19, 1], packed=x)
    both.check_pool(before)
    # zeros, and the largest and smallest magnitudes
    x = both.packed(42)
    x[:] = 0
    x[:, -64:] = torch.finfo(torch.bfloat16).tiny * 3
    x[1::2, 128:192] = torch.finfo(torch.bfloat16).max
    both.append([20, 20], packed=x)
    both.check_pool(before)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_the_largest_entries_stay(dev, dtype, d):
    # the largest magnitudes there are become 256 * 2^120, which is no number of 32 bits by itself: chunks and rows that join their block leave them what they are
    import torch
    both = Both(dev, 3, 4, 2, d, 16, 80, dtype)
    x = both.packed(30)
    top = torch.finfo(both.dtype).max
    h = x.view(30, 8, d)
    h[::3, 4:, 1], h[1::4, 4:, d - 2] = top, -top
    before = both.pool()
    both.append([9, 13, 3], packed=x)
    both.check_pool(before)
    for n in ([2, 5, 30], [1, 1, 1], [3, 0, 2]):
        both.append(n)
        both.check_pool(before)
    assert both.c.err.item() == 0


def test_sequences_that_cannot_take_part_are_left_alone(dev):
    import torch
    from paper_2510_13797_amd import bc
    both = Both(dev, 4, 4, 1, 64, 16, 64)
    both.append([20, 30, 60, 5])
    before, ok = both.pool(), torch.ones(4, dtype=torch.uint8, device=dev)
    x, zero = both.packed(40), torch.zeros(40, dtype=torch.int32, device=dev)

    def call(n, bit, lengths, max_new=None, keep=None, off=None, rows=40):
        both.c.err.zero_()
        q = torch.full((rows, 4, 64), 7.0, dtype=torch.bfloat16, device=dev)
        off = np.concatenate([[0], np.cumsum(n)]) if off is None else np.asarray(off)
        both.c.append(x[:rows], zero[:rows], both.empty, row_offsets=torch.from_numpy(off.astype(np.int64)).to(dev), max_new=max_new or int(max(n)), active=ok, q=q,
                      keep=None if keep is None else torch.tensor(keep, dtype=torch.int32, device=dev))
        assert both.c.err.item() == bit and list(both.c.lengths.cpu().numpy()) == lengths
        return q, off

    for big in (False, True):
        n = [0, 0, 5, 0] if big else [0, 0, 1, 0]
        both.c.lengths[2] = 60 if big else 64                             # does not fit
        q, _ = call(n, bc.BC_ERRBIT_CAPACITY, [20, 30, 60 if big else 64, 5])
        assert (q == 7).all()
        both.c.lengths[2] = 60
        n = [0, 5, 0, 0] if big else [0, 1, 0, 0]
        for page in (-1, 1 << 20, both.c.pages):                          # a page that is none, for an entry that is new
            both.c.table[1, 1 + big] = page
            both.c.lengths[1] = 30
            q, _ = call(n, bc.BC_ERRBIT_STATE if big else 0, [20, 30, 60, 5]) if big else (q, 0)
            both.c.table[1, 1 + big] = int(both.table[1, 1 + big])
        for keep in ([20, 31, 60, 5], [20, -1, 60, 5]):                   # keeps more than there is
            q, _ = call(n, bc.BC_ERRBIT_STATE, [20, 30, 60, 5], keep=keep)
            assert (q == 7).all()
        both.c.lengths[1] = -3
        call(n, bc.BC_ERRBIT_STATE, [20, -3, 60, 5])
        both.c.lengths[1] = 30
    # spans beyond the rows, longer than max_new, that decrease
    call(None, bc.BC_ERRBIT_STATE, [20, 30, 60, 5], max_new=8, off=[0, 0, 0, 0, 41])
    call(None, bc.BC_ERRBIT_STATE, [20, 30, 60, 5], max_new=8, off=[0, 9, 9, 9, 9])
    call(None, bc.BC_ERRBIT_STATE, [20, 30, 60, 5], max_new=8, off=[5, 3, 3, 3, 3])
    call(None, bc.BC_ERRBIT_STATE, [20, 30, 60, 5], max_new=8, off=[-2, 0, 0, 0, 0])
    for a, b in zip(before, both.pool()):
        assert np.array_equal(a, b, equal_nan=a.dtype.kind == "f")
    # and the others take part beside them
    both.c.err.zero_()
    off = torch.tensor([0, 9, 11, 11, 14], device=dev)
    both.c.append(x, zero, both.empty, row_offsets=off, max_new=3)
    assert both.c.err.item() == bc.BC_ERRBIT_STATE and list(both.c.lengths.cpu().numpy()) == [20, 32, 60, 8]


def test_a_bad_page_of_one_new_row(dev):
    import torch
    from paper_2510_13797_amd import bc
    both = Both(dev, 2, 4, 1, 64, 16, 64)
    both.append([32, 5])
    before = both.pool()
    for page in (-1, both.c.pages, 0x7fffffff):
        both.c.table[0, 2] = page
        both.c.err.zero_()
        both.c.append(both.packed(2), torch.zeros(2, dtype=torch.int32, device=dev), both.empty, active=torch.tensor([1, 0], dtype=torch.uint8, device=dev))
        assert both.c.err.item() == bc.BC_ERRBIT_STATE and list(both.c.lengths.cpu().numpy()) == [32, 5]
    for a, b in zip(before, both.pool()):
        assert np.array_equal(a, b, equal_nan=a.dtype.kind == "f")


# ------------------------------------------------------------------ attend
@pytest.mark.parametrize("Hq,Hkv,d", HEADS)
def test_a_step_over_every_length(dev, Hq, Hkv, d):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 129, 500]
    both = Both(dev, len(lens), Hq, Hkv, d, 16, 520)
    both.append(lens)
    _, q = both.append([1] * len(lens))
    both.check_attend(q[:len(lens)], [1] * len(lens))
    out = both.c.attend(q[:len(lens)])
    again = both.c.attend(q[:len(lens)], max_len=501)
    assert both.torch.allclose(out, again, atol=2e-6)


@pytest.mark.parametrize("page", [16, 32, 128, 1024])
@pytest.mark.parametrize("d", [64, 128])
def test_pages_of_every_size(dev, page, d):
    both = Both(dev, 3, 8, 2, d, page, 2100)
    both.append([2000, 31, 700])
    _, q = both.append([1, 1, 1])
    both.check_attend(q[:3], [1, 1, 1])
    _, q = both.append([5, 0, 3], first=1)
    both.check_attend(q, [5, 0, 3], first=1)


@pytest.mark.parametrize("Hq,Hkv,d", HEADS)
def test_some_rows(dev, Hq, Hkv, d):
    # up to 16 columns a KV head, up to 32, more; rows that see nothing but themselves
    for n in ([2, 1, 3, 0, 2, 4], [5, 9, 0, 6, 1, 8], [17, 33, 1, 64, 2, 40]):
        both = Both(dev, 6, Hq, Hkv, d, 32, 500, seed=n[0])
        both.append([0, 1, 30, 31, 100, 300])
        _, q = both.append(n)
        both.check_attend(q, n)
        both.check_attend(q, n, active=[1, 0, 1, 1, 0, 1], device_offsets=True)


@pytest.mark.parametrize("n", [9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 96, 127, 128, 129, 300])
@pytest.mark.parametrize("L", [0, 32, 45])
def test_ends_of_tiles(dev, n, L):
    for Hq, Hkv, d in ((4, 1, 128), (4, 4, 64)):
        both = Both(dev, 1, Hq, Hkv, d, 16, L + n)
        both.append([L])
        _, q = both.append([n])
        both.check_attend(q, [n], every=3)


def test_long_sequences_in_parts(dev):
    both = Both(dev, 2, 4, 1, 128, 64, 9100)
    both.append([9000, 20])
    for n in ([1, 1], [4, 2], [70, 3]):
        _, q = both.append(n)
        both.check_attend(q, n, every=23)
        # the same bits again
        off = np.concatenate([[0], np.cumsum(n)])
        a, b = (both.c.attend(q, row_offsets=off)[:off[-1]] for _ in range(2))
        assert both.torch.equal(a, b)


def test_parts_of_more_workgroups_than_run_at_once(dev):
    # 138 and 576 blocks of columns, by the longest there may be in seven and three parts; short sequences among long ones have fewer
    both = Both(dev, 69, 14, 2, 64, 64, 28000)
    n = np.random.default_rng(8).integers(5, 16, 69)
    both.append(np.where(np.arange(69) % 3 == 0, 9000, np.where(np.arange(69) % 3 == 1, 1, 500)))
    _, q = both.append(n)
    both.check_attend(q, n, every=7)
    n = np.random.default_rng(9).integers(0, 10, 69)             # (two waves a column)
    _, q = both.append(n)
    both.check_attend(q, n, every=7)
    both = Both(dev, 9, 16, 8, 128, 32, 5000)
    n = np.array([510, 3, 450, 0, 512, 1, 350, 64, 65])
    both.append(np.full(9, 900))
    _, q = both.append(n)
    both.check_attend(q, n, every=251)


def test_many_sequences(dev):
    r = np.random.default_rng(3)
    for B, Hq, Hkv, d in ((300, 4, 1, 64), (70, 12, 2, 128), (33, 32, 8, 128)):
        both = Both(dev, B, Hq, Hkv, d, 16, 130)
        both.append(r.integers(0, 100, B))
        _, q = both.append([1] * B)
        both.check_attend(q, [1] * B)
        n = r.integers(0, 12, B)
        _, q = both.append(n, active=None)
        both.check_attend(q, n, every=3)


def test_the_sum_where_the_scale_is_zero_and_where_scores_are_large(dev):
    both = Both(dev, 2, 8, 2, 128, 16, 300)
    both.append([200, 90], size=1.0)
    _, q = both.append([1, 1])
    both.c.shape.scale = 0.0
    both.check_attend(q, [1, 1], scale=0.0)
    for n in ([40, 3], [2, 8], [200, 31]):
        both = Both(dev, 2, 8, 2, 128, 16, 900)
        both.append([300, 0])
        _, q = both.append(n)
        for scale in (0.0, 1e-30, 1e-6):
            both.c.shape.scale = scale
            both.check_attend(q, n, scale=scale, every=3)
    # scores of some hundreds: weights of 0 and 1; a score is off by 128 roundings of up to 2^-24 of some 1e4
    both = Both(dev, 2, 8, 2, 128, 16, 300)
    both.append([200, 90], size=20.0)
    _, q = both.append([1, 1], size=20.0)
    both.check_attend(q, [1, 1], tol=0.05)


@pytest.mark.parametrize("n", [[1, 3], [9, 14], [40, 66]])
@pytest.mark.parametrize("d", [64, 128])
def test_scales_of_any_kind(dev, n, d):
    # a cache filled by the caller: scales that are no powers of two, negative ones and zeros among them
    import torch
    both = Both(dev, 2, 4, 1, d, 16, 250)
    both.append([150, 77])
    _, q = both.append(n)
    r = np.random.default_rng(5)
    for s in range(2):
        for seq, scales in ((both.k[s], both.c.k_scale), (both.v[s], both.c.v_scale)):
            f = r.uniform(0.5, 1.5, seq.scales.shape) * r.choice([-1.0, 1.0, 0.0], seq.scales.shape)
            f[:, 3] = 1.0
            seq.scales = np.float64(np.float32(seq.scales * f))
            for b in range(seq.scales.shape[1]):
                scales[int(both.table[s, b]), :, 0] = torch.from_numpy(np.float32(seq.scales[:, b])).to(dev)
    both.check_attend(q, n)


def _two_bf16_parts(w):
    """What two bf16 parts hold of w (rounded to nearest): 17 bits."""
    def bf16(x):
        u = np.float32(x).view(np.uint32).astype(np.uint64)
        return ((u + 0x7fff + (u >> 16 & 1)) >> 16 << 16).astype(np.uint32).view(np.float32).astype(np.float64)
    hi = bf16(w)
    return hi + bf16(w - hi)


@pytest.mark.parametrize("n", [[1], [7], [20], [66], [300]])
@pytest.mark.parametrize("d", [64, 128])
def test_weights_have_22_bits(dev, n, d):
    # entries that are all alike, with values of one: the result is what a weight's parts hold of it, sum over sum.  Two half-precision parts are off by 2^-23, the reciprocal by 2^-23, the sum of
    # weights by 2^-24 at each of 11 steps (eight of a lane 3, lanes 2, blocks and tiles 6), the matrix product's by 2^-24 of what is summed so far at each of up to 44 entries, 22 * 2^-24.  Two
    # bf16 parts would be off by up to 2^-18.
    import torch
    tol = 37 * 2.0 ** -24
    Hq, Hkv = 4, 2
    both = Both(dev, 1, Hq, Hkv, d, 16, 8 + n[0])
    both.c.shape.scale = np.log(2.0)
    x = torch.zeros(8 + n[0], Hq + 2 * Hkv, d, device=dev, dtype=torch.bfloat16)
    x[:, Hq:Hq + Hkv, 0] = 1.0
    x[:, Hq + Hkv:] = 1.0
    both.append([8], packed=x[:8].reshape(8, -1))
    both.append(n, packed=x[8:].reshape(n[0], -1))
    q = torch.zeros(n[0], Hq, d, device=dev, dtype=torch.bfloat16)
    q[:, :, 0] = 3.0 * torch.rand(n[0], Hq, generator=both.gen, device=dev)
    w = np.exp2(_np(q[:36, :, 0]))
    off = (np.abs(_two_bf16_parts(w) - w) / w).max()
    assert n[0] < 20 or off > 1.5 * tol
    got = _np(both.c.attend(q, row_offsets=[0, n[0]])[:36])
    assert np.abs(got - 1.0).max() <= tol, np.abs(got - 1.0).max()


@pytest.mark.parametrize("n", [[1, 2], [6, 8], [20, 31], [40, 66]])
@pytest.mark.parametrize("d", [64, 128])
def test_values_of_very_different_sizes(dev, n, d):
    # blocks of values from 1e-25 to 1e25, empty ones among them, under scores that let now these, now those weigh something.  A product of a weight and a value is in two
    # half-precision parts whose least step is 2^-32 of the largest product so far: an output is off by less than 1e-5 of the largest product of its row
    import torch
    both = Both(dev, 2, 4, 2, d, 16, 700)
    r = np.random.default_rng(7)
    lens = [600, 333]
    for s in range(2):                                                  # sixteen rows at a time, so that a block has a size of its own
        for at in range(0, lens[s], 16):
            m = [0, 0]
            m[s] = min(16, lens[s] - at)
            x = both.packed(m[s])
            size = 10.0 ** r.uniform(-25, 25) if at % 48 else 0.0
            x[:, (4 + 2) * d:] *= size
            x[:, 4 * d:6 * d] *= 10.0 ** r.uniform(-1, 0.7)
            both.append(m, packed=x)
    x = both.packed(sum(n))
    x[:, 6 * d:] *= 1e-3
    both.append(n, packed=x)
    q = (3.0 * torch.randn(sum(n), 4, d, generator=both.gen, device=dev)).bfloat16()
    off = np.concatenate([[0], np.cumsum(n)])
    got, qn = _np(both.c.attend(q, row_offsets=off)), _np(q)
    for s in range(2):
        K, V = both.k[s].numbers(), both.v[s].numbers()
        for i in range(0, n[s], 5):
            e = len(K) - n[s] + i + 1
            for h in range(4):
                z = K[:e, h // 2] @ qn[off[s] + i, h] * both.c.shape.scale
                p = np.exp(z - z.max())
                p /= p.sum()
                products = p[:, None] * V[:e, h // 2]
                assert np.isfinite(got[off[s] + i, h]).all()
                assert np.abs(got[off[s] + i, h] - products.sum(axis=0)).max() <= 1e-5 * np.abs(products).max() + 1e-37, (s, i, h)


@pytest.mark.parametrize("n", [[1, 2], [6, 8], [20, 31], [40, 66]])
@pytest.mark.parametrize("size", [1e-33, 1e-30, 1e30])
def test_values_at_the_ends_of_the_range(dev, n, size):
    # scores that rise with the entries, so that the reference moves all along, over values whose level is as high, or as low, as it goes
    import torch
    d = 128
    both = Both(dev, 2, 4, 2, d, 16, 500)
    lens = [400, 260]
    x = both.packed(sum(lens))
    x[:, 4 * d:6 * d] = 0.1 * x[:, 4 * d:6 * d]
    x[:, 4 * d] = torch.cat([torch.arange(k, device=dev) / 8.0 for k in lens]).to(x.dtype)
    x[:, 5 * d] = x[:, 4 * d]
    x[:, 6 * d:] *= size
    both.append(lens, packed=x)
    x = both.packed(sum(n))
    x[:, 6 * d:] *= size
    both.append(n, packed=x)
    q = torch.randn(sum(n), 4, d, generator=both.gen, device=dev)
    q[:, :, 0] = 4.0
    q = q.bfloat16()
    off = np.concatenate([[0], np.cumsum(n)])
    got, qn = _np(both.c.attend(q, row_offsets=off)), _np(q)
    for s in range(2):
        K, V = both.k[s].numbers(), both.v[s].numbers()
        for i in range(0, n[s], 5):
            e = len(K) - n[s] + i + 1
            ref = OA.decode_attention(qn[off[s] + i], K[:e], V[:e], both.c.shape.scale)
            # (outputs of N(0, 1) values, off by 1e-4 at most)
            assert np.abs(got[off[s] + i] - ref).max() <= TOL * size, (s, i)


@pytest.mark.parametrize("n", [[2, 5], [9, 16], [18, 31], [40, 66], [140, 200]])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("before", [[0, 3], [75, 41], [900, 1500]])
def test_what_a_row_does_not_see_does_not_reach_it(dev, n, d, before):
    # new rows whose values, keys or query are no numbers: rows in front of them, other heads and other sequences have their results
    import torch
    Hq, Hkv = 4, 2
    both = Both(dev, 2, Hq, Hkv, d, 64, max(b + m for b, m in zip(before, n)))
    both.append(before)
    x = both.packed(sum(n))
    h = x.view(-1, Hq + 2 * Hkv, d)
    h[n[0] // 2, Hq + Hkv, 5] = float("inf")                 # a value of sequence 0, head 0,
    h[n[0] - 1, Hq + Hkv + 1, d - 1] = float("nan")          # the last one of head 1,
    h[n[0] + n[1] - 2, Hq + Hkv + 1, 0] = float("-inf")      # of sequence 1
    h[n[0] + n[1] - 1, Hq, 3] = float("nan")                 # and a key
    _, q = both.append(n, packed=x)
    q[n[0], 3] = float("nan")                                # a query of sequence 1
    off = np.concatenate([[0], np.cumsum(n)])
    got, qn, seen = _np(both.c.attend(q, row_offsets=off)), _np(q), 0
    for s in range(2):
        K, V = both.k[s].numbers(), both.v[s].numbers()
        for i in range(n[s]):
            e = before[s] + i + 1
            for head in range(Hq):
                row, kvh = got[off[s] + i, head], head // (Hq // Hkv)
                k, v, query = K[:e, kvh], V[:e, kvh], qn[off[s] + i, head]
                if np.isfinite(k).all() and np.isfinite(query).all():
                    bad = ~np.isfinite(v).all(axis=0)
                    ref = OA.decode_attention(query[None], k[:, None], np.where(np.isfinite(v), v, 0.0)[:, None], both.c.shape.scale)[0]
                    assert np.isnan(row[bad]).all()
                    right = ~bad if not bad.any() else ~bad & ~np.isnan(row)
                    assert np.abs(row - ref)[right].max(initial=0.0) <= TOL, (s, i, head)
                    seen += bad.any()
                else:
                    assert np.isnan(row).all(), (s, i, head)
    assert seen >= 4 and both.c.err.item() == 0


def test_positions_that_are_the_lengths(dev):
    # a step's positions are the lengths themselves, the tensor that the call moves
    import torch
    both, other = (Both(dev, 5, 12, 2, 128, 16, 80, seed=3) for _ in range(2))
    freq = 10000.0 ** (-torch.arange(0, 128, 2, device=dev) / 128)
    for b in (both, other):
        b.append([30, 0, 16, 15, 1])
    for _ in range(20):
        x = both.packed(5)
        got = both.c.append(x, both.c.lengths, freq)
        assert torch.equal(got, other.c.append(x, other.c.lengths.clone(), freq))
    for a, b in zip(both.pool(), other.pool()):
        assert np.array_equal(a, b, equal_nan=a.dtype.kind == "f")


def test_layers_that_share_a_table_and_run_at_once(dev):
    # two layers' caches over one table, each on a stream of its own
    import torch
    from paper_2510_13797_amd import bc
    B, Hq, Hkv, d, page = 6, 12, 2, 128, 32
    table = torch.randperm(64, device=dev)[:B * 10].view(B, 10).int()
    x = torch.randn(2, B * 100, (Hq + 2 * Hkv) * d, device=dev).bfloat16()
    step = torch.randn(2, 20, B, (Hq + 2 * Hkv) * d, device=dev).bfloat16()
    pos, none = torch.arange(B * 100, device=dev).int(), torch.zeros(0, device=dev)

    def layer(i, cache):
        outs = []
        cache.append(x[i], pos, none, row_offsets=range(0, B * 100 + 1, 100))
        for t in range(20):
            outs.append(cache.attend(cache.append(step[i, t], pos[:B], none), max_len=200))
        return outs

    alone = [layer(i, bc.PagedCache(B, Hq, Hkv, d, 64, page, 10, dev, table=table)) for i in range(2)]
    caches = [bc.PagedCache(B, Hq, Hkv, d, 64, page, 10, dev, table=table) for _ in range(2)]
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for i in range(2):
        with torch.cuda.stream(streams[i]):
            got.append(layer(i, caches[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert caches[i].err.item() == 0 and caches[i].table is table
        assert all(torch.equal(a, b) for a, b in zip(got[i], alone[i]))


def test_a_given_table_stays_while_a_call_is_in_work(dev):
    # table and cache are dropped with calls still waiting on a stream of their own: the table's memory is not given out again before them
    import torch
    from paper_2510_13797_amd import bc
    B, Hq, Hkv, d = 2, 4, 1, 64
    x, pos, none = torch.randn(B, (Hq + 2 * Hkv) * d, device=dev).bfloat16(), torch.zeros(B, dtype=torch.int32, device=dev), torch.zeros(0, device=dev)
    q, stream = torch.randn(B, Hq, d, device=dev).bfloat16(), torch.cuda.Stream()

    def call(cache, kind):
        return cache.append(x, pos, none) if kind == "append" else cache.attend(q)

    for kind in ("append", "attend"):
        table = torch.zeros(B, 1 << 16, dtype=torch.int32, device=dev)
        table[:, 0] = torch.arange(B, device=dev)
        at, size = table.data_ptr(), table.shape
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            cache = bc.PagedCache(B, Hq, Hkv, d, B, 16, 1 << 16, dev, table=table)
            cache.append(x, pos, none)
            stream.synchronize()
            torch.cuda._sleep(500_000_000)         # 0.2 s
            call(cache, kind)
        del cache, table
        other = torch.empty(size, dtype=torch.int32, device=dev)
        assert not stream.query() and other.data_ptr() != at, kind
        stream.synchronize()


def test_an_empty_cache_of_zeros(dev):
    both = Both(dev, 2, 8, 2, 128, 16, 400)
    both.append([300, 5], packed=both.packed(305) * 0)
    for n in ([1, 1], [8, 3], [70, 40]):
        x = both.packed(sum(n))
        x[:, 10 * 128:] = 0
        _, q = both.append(n, packed=x)
        out = both.check_attend(q, n, every=7)
        assert (out[:sum(n)] == 0).all()


def test_pages_in_common(dev):
    # samples of one prompt: its whole pages are shared, the rest is each one's own
    import torch
    both = Both(dev, 4, 12, 2, 128, 16, 100)
    both.append([48, 0, 0, 0])
    for s in (1, 2, 3):
        both.table[s, :3] = both.table[0, :3]
        for a in (both.k, both.v):
            a[s].values, a[s].scales = a[0].values.copy(), a[0].scales.copy()
    both.c.table.copy_(torch.from_numpy(both.table))
    both.c.lengths.fill_(48)
    before = both.pool()
    for i in range(5):
        _, q = both.append([1] * 4)
        both.check_attend(q, [1] * 4)
    both.check_pool(before)


def test_attend_leaves_alone_what_cannot_take_part(dev):
    import torch
    from paper_2510_13797_amd import bc
    both = Both(dev, 3, 4, 1, 64, 16, 64)
    both.append([20, 30, 10])
    q = torch.randn(40, 4, 64, device=dev).bfloat16()
    for off, most, lens, max_len in (([0, 1, 32, 33], 40, [20, 30, 10], None), ([0, 1, 9, 10], 7, [20, 30, 10], None), ([0, 1, 41, 41], 50, [20, 30, 10], None),
                                     ([0, 1, 2, 3], 1, [20, 65, 10], None), ([0, 1, 2, 3], 1, [20, -1, 10], None), ([0, 1, 2, 3], 1, [20, 30, 10], 29),
                                     ([0, 1, 2, 3], 1, [20, 0, 10], None)):
        both.c.err.zero_()
        both.c.lengths.copy_(torch.tensor(lens))
        out = torch.full((40, 4, 64), 7.0, device=dev)
        both.c.attend(q, row_offsets=torch.tensor(off, device=dev), max_new=most, out=out, max_len=max_len)
        assert both.c.err.item() == bc.BC_ERRBIT_STATE, off
        assert (out[1:off[2]] == 7).all() and (out[0] != 7).any() and (off[2] >= 40 or (out[off[2]] != 7).any())
    # a page that is none: nothing is read out of range, the others are right
    both.c.lengths.copy_(torch.tensor([20, 30, 10]))
    for page in (-5, 1 << 30, both.c.pages):
        both.c.err.zero_()
        both.c.table[1, 1] = page
        out = both.c.attend(q[:3])
        assert both.c.err.item() == bc.BC_ERRBIT_STATE
        both.c.table[1, 1] = int(both.table[1, 1])
        both.c.err.zero_()
        both.check_attend(q[:3], [1, 1, 1], active=[1, 0, 1])
        assert torch.equal(out[[0, 2]], both.c.attend(q[:3])[[0, 2]])


def test_places_beyond_32_bits(dev):
    # a pool of 5 GB each of keys and values, whose last pages are in use
    import torch
    from paper_2510_13797_amd import bc
    pages, page, Hkv, d = 1250, 1024, 32, 128
    c = bc.PagedCache(2, 32, Hkv, d, pages, page, 2, dev)
    c.table.copy_(torch.tensor([[1248, 3], [1249, 1247]]))
    gen = torch.Generator(device=dev).manual_seed(0)
    n = [1030, 40]
    x = torch.randn(sum(n), 3 * 32 * d, generator=gen, device=dev).bfloat16()
    pos = torch.zeros(len(x), dtype=torch.int32, device=dev)
    q = c.append(x, pos, torch.zeros(0, device=dev), row_offsets=[0, 1030, 1070])
    h = _np(x).reshape(len(x), -1, d)
    out = c.attend(q, row_offsets=[0, 1030, 1070])
    for s, rows in ((0, slice(0, 1030)), (1, slice(1030, 1070))):
        K, V = c.entries(s)
        for got, lo in ((K, 32), (V, 64)):
            for head in (0, 31):
                seq = OP.Sequence(1, d)
                seq.append(h[rows, lo + head:lo + head + 1])
                assert np.array_equal(got[:, head], seq.numbers()[:, 0])
        for i in (0, n[s] // 2, n[s] - 1):
            ref = OA.decode_attention(_np(q[rows][i]), K[:i + 1], V[:i + 1], d ** -0.5)
            assert np.abs(_np(out[rows][i]) - ref).max() <= TOL
    assert c.err.item() == 0


# ------------------------------------------------------------------ ends of the range
def _weighed(dev, n, d, before, z, values, new_z, new_values, page=16, Hq=4, Hkv=2, scale=np.log(2.0)):
    """A cache whose entries have the scores z (log2, exact in e4m3; under a query of ones at element 0) and the values `values` [entries, d], and n new rows a
    sequence with new_z and new_values [row]; -> (what attend gives, as float64, the weights' products [sequence][row] -> [entry, Hkv, d] in 64 bits, and the largest product of a
    weight and its block's value scale [sequence][row] -> [Hkv])."""
    import torch
    both = Both(dev, len(n), Hq, Hkv, d, page, max(b + m for b, m in zip(before, n)))
    both.c.shape.scale = scale

    def rows(count, score, value):
        x = torch.zeros(count, Hq + 2 * Hkv, d, device=dev, dtype=torch.float64)
        x[:, Hq:Hq + Hkv, 0] = torch.as_tensor(np.asarray(score), device=dev)[:, None]
        x[:, Hq + Hkv:] = torch.as_tensor(np.array(value), device=dev)[:, None]
        return x.view(count, -1).to(both.dtype)

    both.append(before, packed=torch.cat([rows(b, z(np.arange(b)), values(np.arange(b))) for b in before]))
    both.append(n, packed=torch.cat([rows(m, new_z(np.arange(m)), new_values(np.arange(m))) for m in n]))
    q = torch.zeros(sum(n), Hq, d, device=dev, dtype=torch.bfloat16)
    q[:, :, 0] = 1.0
    off = np.concatenate([[0], np.cumsum(n)])
    got = _np(both.c.attend(q, row_offsets=off))
    qs, products = float(np.float32(np.float32(scale) * np.float32(1.4426950408889634))), []
    heaviest = []
    for s in range(len(n)):
        K, V = both.k[s].numbers(), both.v[s].numbers()
        products.append([]), heaviest.append([])
        for i in range(n[s]):
            e = before[s] + i + 1
            t = qs * K[:e, :, 0]
            w = np.exp2(t - t.max(axis=0))
            w /= w.sum(axis=0)
            products[-1].append(w[:, :, None] * V[:e])
            heaviest[-1].append((w * np.repeat(both.v[s].scales, 16, axis=1)[:, :e].T).max(axis=0))
    assert both.c.err.item() == 0
    return got, off, products, heaviest


def _close(got, off, products, heaviest, least=2e-38):
    """Outputs within 1e-4 of the sum of their products' magnitudes: scores of up to 128 that are off by 2^-24 make weights that are off by 1e-5, halves in two parts 2^-22; and
    `least`, what 32 bits hold at their end; and what halves hold at theirs: a weight's product with its block's scale is in steps of 2^-24 where the largest sum of up to eight weights
    times their block's scale came to 2^8 or more, so it is off by half of a step, 2^-25 / 2^5 of the largest product of one weight and a scale, and its entry by 448 times that."""
    for s, rows in enumerate(products):
        for i, p in enumerate(rows):
            for h in range(got.shape[1]):
                kvh = h // (got.shape[1] // p.shape[1])
                x = p[:, kvh]
                steps = np.count_nonzero(x, axis=0) * 448 * 2.0 ** -30 * heaviest[s][i][kvh]
                assert (np.abs(got[off[s] + i, h] - x.sum(axis=0)) <= 1e-4 * np.abs(x).sum(axis=0) + steps + least).all(), (s, i, h)


MANY_ROWS = [[1, 2], [6, 8], [20, 31], [40, 66]]


@pytest.mark.parametrize("n", MANY_ROWS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("gap,size", [(104, 2.0 ** -14), (120, 1.0), (28, 1e-28)])
@pytest.mark.parametrize("last", [0.0, 1.0])
def test_sums_stay_where_the_reference_moves_far(dev, n, d, gap, size, last):
    # scores 28 to 120 higher over values of zero: what was summed before is the result, small as its weights are by then.  (New rows with values make their block's scale theirs, and
    # heavy weights of that block hide what is as small.)
    r = np.random.default_rng(2)
    v = size * r.standard_normal((700, d))
    given = _weighed(dev, n, d, [600, 333], lambda j: np.where(j < 256, 0.0, float(gap)), lambda j: np.where(j[:, None] < 256, v[j], 0.0), lambda j: 0.0 * j, lambda j: last * v[j])
    _close(*given)


@pytest.mark.parametrize("n", MANY_ROWS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("gap,stretch", [(56, 1.0), (112, 1.0), (120, 1.0), (120, 1.03), (240, 1.0)])
def test_large_values_of_little_weight_behind_zeros(dev, n, d, gap, stretch):
    # values of thousands whose weights are 2^-56 and less, behind values of zero, whose level is as high as it goes
    r = np.random.default_rng(3)
    v = 3000.0 * r.standard_normal((700, d))
    given = _weighed(dev, n, d, [600, 333], lambda j: np.where(j < 256, 0.0, -float(gap)), lambda j: np.where(j[:, None] < 256, 0.0, v[j]),
                                  lambda j: 0.0 * j - gap, lambda j: v[j], scale=stretch * np.log(2.0))
    _close(*given)


@pytest.mark.parametrize("n", [[2, 3], [8, 5], [20, 31], [40, 66], [200, 130]])
@pytest.mark.parametrize("d", [64, 128])
def test_large_values_that_a_row_does_not_see(dev, n, d):
    # the first new row ends a block of zeros, those behind it have values of thousands: zeros for the one, numbers for the others
    r = np.random.default_rng(4)
    v = 3000.0 * r.standard_normal((700, d))
    given = _weighed(dev, n, d, [15, 47], lambda j: 0.0 * j, lambda j: np.zeros((len(j), d)), lambda j: 0.0 * j, lambda j: np.where(j[:, None] < 1, 0.0, v[j]))
    _close(*given)
    got, off = given[:2]
    assert (got[0] == 0).all() and (got[off[1]] == 0).all()


@pytest.mark.parametrize("n", MANY_ROWS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("before", [[600, 333], [9000, 17]])
@pytest.mark.parametrize("size", [1e36, 3e37])
def test_sums_beyond_the_range_of_results_within(dev, n, d, before, size):
    # hundreds and thousands of equal entries: the sum of the products is no number of 32 bits, their mean is one
    v = np.where(np.arange(d) % 3 == 1, -size, size)
    given = _weighed(dev, n, d, before, lambda j: (j % 8) / 4.0, lambda j: np.broadcast_to(v, (len(j), d)), lambda j: 0.0 * j,
                     lambda j: np.broadcast_to(v, (len(j), d)), page=64)
    _close(*given)


@pytest.mark.parametrize("n", MANY_ROWS)
def test_the_largest_values(dev, n):
    # one entry in hundreds is as large as bf16 gets (in e4m3 240 * 2^120)
    v = np.where(np.arange(700) % 97 == 5, 240 * 2.0 ** 120, 0.0)
    given = _weighed(dev, n, 64, [600, 333], lambda j: 0.0 * j, lambda j: np.repeat(v[j][:, None], 64, axis=1), lambda j: 0.0 * j, lambda j: np.zeros((len(j), 64)))
    _close(*given)


@pytest.mark.parametrize("n", MANY_ROWS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("gap,size", [(28, 1e-28), (104, 2.0 ** -14), (120, 1.0), (120, 1e30)])
@pytest.mark.parametrize("first", [True, False])
def test_parts_whose_references_lie_far_apart(dev, n, d, gap, size, first):
    # parts of long sequences that hold the values, in front of or behind parts of zeros whose scores are up to 120 higher
    r = np.random.default_rng(6)
    v = size * r.standard_normal((9200, d))
    low = (lambda j: j < 4096) if first else (lambda j: j >= 4096)
    given = _weighed(dev, n, d, [9000, 5000], lambda j: np.where(low(j), 0.0, float(gap)), lambda j: np.where(low(j)[:, None], v[j], 0.0), lambda j: 0.0 * j,
                     lambda j: 0.0 * v[j] if first else v[j], page=64)
    _close(*given)


@pytest.mark.parametrize("n", MANY_ROWS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", [1e-33, 1.0, 3e37])
@pytest.mark.parametrize("at", [100, 4000, 8990])
def test_one_heavy_entry_among_thousands(dev, n, d, size, at):
    # the largest weight is alone in its wave and part, thousands of entries 2^-20 of it each lie in others: neither side's share of the other's sums leaves the range
    r = np.random.default_rng(10)
    v = size * r.uniform(0.5, 1.5, (9200, d)) * np.where(np.arange(d) % 2, 1.0, -1.0)
    given = _weighed(dev, n, d, [9000, 5000], lambda j: np.where(j == at, 20.0, 0.0), lambda j: v[j], lambda j: 0.0 * j, lambda j: v[j], page=64)
    _close(*given)


# ------------------------------------------------------------------ together
def test_the_last_places_of_the_longest_table(dev):
    # a row of the table that holds 2^31 - 1024 entries, nearly all of them in one page; new rows at its end, in a call for more of them
    import torch
    from paper_2510_13797_amd import bc
    per, page, Hq, Hkv, d = (1 << 21) - 1, 1024, 2, 1, 64
    c = bc.PagedCache(1, Hq, Hkv, d, 2, page, per, dev)
    for x in (c.k_pages, c.v_pages):
        x.view(torch.uint8).zero_()
    c.k_scale.fill_(OP.LEAST), c.v_scale.fill_(OP.LEAST)
    c.table[0, -1] = 1
    start, n = per * page - 130, 90
    c.lengths.fill_(start)
    x = torch.randn(2000, (Hq + 2 * Hkv) * d, device=dev).bfloat16()
    pos, off = torch.zeros(2000, dtype=torch.int32, device=dev), torch.tensor([0, n], device=dev)
    c.append(x, pos, torch.zeros(0, device=dev), row_offsets=off, max_new=2000)
    assert c.lengths.item() == start + n and c.err.item() == 0
    V = c.v_pages.view(torch.uint8)
    assert (V[0] == 0).all() and (c.v_scale[0] == OP.LEAST).all()
    seq = OP.Sequence(Hkv, d)
    seq.append(np.zeros((page - 130, Hkv, d)))
    seq.append(_np(x[:n]).reshape(n, -1, d)[:, Hq + Hkv:])
    for j in range(page - 130, page - 130 + n):
        assert (V[1, 0].reshape(-1).cpu().numpy()[OP.value_place(j, np.arange(d), d)] == OP.e4m3_byte(seq.values[0, j])).all(), j
    assert (V[1, 0].reshape(page // 4, d, 4)[(page - 130 + n + 3) // 4:] == 0).all()
    # one more than there is room for
    c.append(x, pos, torch.zeros(0, device=dev), row_offsets=torch.tensor([0, 41], device=dev), max_new=2000)
    assert c.err.item() == bc.BC_ERRBIT_CAPACITY and c.lengths.item() == start + n


def test_appended_by_more_workgroups_than_a_launch_takes(dev):
    # chunks whose longest is not given: each of 512 sequences may have all 524,288 rows as far as the host knows.  One sequence's workgroups are in both launches
    import torch
    from paper_2510_13797_amd import bc
    B, n, d = 512, 1024, 128
    gen = torch.Generator(device=dev).manual_seed(1)
    x = torch.randn(B * n, 3 * d, generator=gen, device=dev).bfloat16()
    pos, none, off = torch.zeros(B * n, dtype=torch.int32, device=dev), torch.zeros(0, device=dev), torch.arange(0, B * n + 1, n, device=dev)
    caches, qs = [], []
    for how in (dict(row_offsets=off), dict(row_offsets=off, max_new=n)):
        c = bc.PagedCache(B, 1, 1, d, B, 1024, 1, dev)
        c.table.copy_(torch.randperm(B, generator=torch.Generator().manual_seed(2)).view(B, 1))
        qs.append(c.append(x, pos, none, **how))
        assert (c.lengths == n).all() and c.err.item() == 0 and (c._arrivals == 0).all()
        caches.append(c)
    assert torch.equal(qs[0], x.view(B * n, 3, d)[:, :1]) and torch.equal(qs[0], qs[1])
    for a, b in zip(caches[0]._own()[:4], caches[1]._own()[:4]):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    for s in (0, 255, 256, 511):
        K, V = caches[0].entries(s)
        for got, lo in ((K, 1), (V, 2)):
            exact = OP.Sequence(1, d)
            exact.append(_np(x[s * n:s * n + n]).reshape(n, 3, d)[:, lo:lo + 1])
            assert np.array_equal(got, exact.numbers())


def test_attended_by_more_workgroups_than_a_launch_takes(dev):
    # 4096 sequences, each of which may have all 65,536 rows and a table of 65,536 entries: 2^24 workgroups
    import torch
    from paper_2510_13797_amd import bc
    B, n, Hq, d = 4096, 16, 8, 64
    c = bc.PagedCache(B, Hq, 1, d, B, 16, 4096, dev)
    c.table[:, 0] = torch.randperm(B, device=dev)
    gen = torch.Generator(device=dev).manual_seed(1)
    x = torch.randn(B * n, (Hq + 2) * d, generator=gen, device=dev).bfloat16()
    off = torch.arange(0, B * n + 1, n, device=dev)
    q = c.append(x, torch.zeros(B * n, dtype=torch.int32, device=dev), torch.zeros(0, device=dev), row_offsets=off, max_new=n)
    out = c.attend(q, row_offsets=off)
    assert c.err.item() == 0 and torch.equal(out, c.attend(q, row_offsets=off, max_new=n, max_len=64))
    for s in (0, 1, 2047, 2048, 4095):
        K, V = c.entries(s)
        for i in (0, 7, 15):
            assert np.abs(_np(out[s * n + i]) - OA.decode_attention(_np(q[s * n + i]), K[:i + 1], V[:i + 1], d ** -0.5)).max() <= TOL


def test_a_generation_with_beacons(dev):
    # Alg. 1 over pages: prompts, tokens, and a beacon in the place of every full window (its own attention over the window first), ratios 4 and 7
    both = Both(dev, 3, 12, 2, 128, 16, 80)
    ratio, P = [4, 7, 4], [20, 3, 16]
    _, q = both.append(P)
    both.check_attend(q, P, every=4)
    window, beacons = [0, 0, 0], [0, 0, 0]
    for t in range(25):
        _, q = both.append([1, 1, 1])
        both.check_attend(q, [1, 1, 1])
        window = [w + 1 for w in window]
        due = [w == c for w, c in zip(window, ratio)]
        if any(due):
            x, q = both.append([1, 1, 1], active=due)
            both.check_attend(q, [1, 1, 1], active=due)
            both.append([1, 1, 1], active=due, keep=[p + b for p, b in zip(P, beacons)], packed=x)
            beacons = [b + w for b, w in zip(beacons, due)]
            window = [0 if w else x for w, x in zip(due, window)]
        assert list(both.c.lengths.cpu().numpy()) == [p + b + w for p, b, w in zip(P, beacons, window)]
    before = both.pool()
    both.check_pool(before)
    assert both.c.err.item() == 0


def test_drafted_tokens_are_checked_and_dropped(dev):
    both = Both(dev, 2, 32, 8, 128, 32, 120)
    both.append([50, 9])
    for accepted in ([1, 4], [4, 2], [3, 3]):
        kept = [len(x) for x in both.k]
        _, q = both.append([4, 4])
        both.check_attend(q, [4, 4])
        # the next rows take the place of those that were not accepted
        _, q = both.append([1, 1], keep=[k + a for k, a in zip(kept, accepted)])
        both.check_attend(q, [1, 1])


def test_captured_steps(dev):
    """Two steps captured on a stream of their own, replayed several times with eager work in between; each replay against the eager result."""
    import torch
    both = Both(dev, 4, 12, 2, 128, 16, 400)
    both.append([300, 17, 0, 130])
    start = both.c.lengths.clone()
    x = [both.packed(4) for _ in range(2)]
    pos = torch.zeros(4, dtype=torch.int32, device=dev)
    pool = [both.c.k_pages.view(torch.uint8), both.c.v_pages.view(torch.uint8), both.c.k_scale, both.c.v_scale]
    saved = [p.clone() for p in pool]

    def steps():
        outs = []
        for i in range(2):
            q = both.c.append(x[i], pos, both.empty)
            outs.append(both.c.attend(q, max_len=400))
            outs.append(both.c.attend(q, row_offsets=[0, 1, 2, 3, 4], max_len=400))
        return outs

    def reset():
        both.c.lengths.copy_(start)
        for p, s in zip(pool, saved):
            p.copy_(s)

    eager = [o.clone() for o in steps()]
    end = [p.clone() for p in pool]
    reset()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        steps()
        stream.synchronize()
        reset()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            outs = steps()
    torch.cuda.synchronize()
    for _ in range(4):
        reset()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a, b)
        for a, b in zip(pool, end):
            assert torch.equal(a.nan_to_num() if a.is_floating_point() else a, b.nan_to_num() if b.is_floating_point() else b)
        for a in outs:
            a.zero_()
        reset()
        assert all(torch.equal(a, b) for a, b in zip(steps(), eager))       # eager work between
    assert both.c.err.item() == 0


def test_two_graphs_of_one_cache(dev):
    # a decode step and a check of drafted tokens (a chunk of 40 in the second sequence), captured into one memory pool and replayed by turns
    import torch
    both = Both(dev, 3, 12, 2, 128, 32, 1600)
    both.append([900, 17, 1300])
    pos = torch.zeros(48, dtype=torch.int32, device=dev)
    one, many = both.packed(3), both.packed(46)
    off, accepted = [0, 4, 44, 46], torch.zeros(3, dtype=torch.int32, device=dev)

    def step():
        return both.c.attend(both.c.append(one, pos[:3], both.empty))

    def check():
        accepted.copy_(both.c.lengths)
        accepted.add_(1)
        out = both.c.attend(both.c.append(many, pos[:46], both.empty, row_offsets=off), row_offsets=off)
        both.c.lengths.copy_(accepted)                       # one of the drafted tokens is kept
        return out

    start, pool = both.c.lengths.clone(), [both.c.k_pages.view(torch.uint8), both.c.v_pages.view(torch.uint8), both.c.k_scale, both.c.v_scale]
    saved = [p.clone() for p in pool]

    def reset():
        both.c.lengths.copy_(start)
        for p, x in zip(pool, saved):
            p.copy_(x)

    eager = [f().clone() for _ in range(3) for f in (step, check)]
    end = both.c.lengths.clone()
    reset()
    stream, graphs, outs, memory = torch.cuda.Stream(), [], [], None
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for f in (step, check):
            f()
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream, pool=memory):
                outs.append(f())
            memory = graph.pool()
            graphs.append(graph)
    torch.cuda.synchronize()
    for _ in range(2):
        reset()
        for i in range(6):
            graphs[i % 2].replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[i % 2], eager[i]), i
        assert torch.equal(both.c.lengths, end) and both.c.err.item() == 0
        reset()
        assert all(torch.equal(f(), e) for e, f in zip(eager, 3 * (step, check)))


def test_without_the_native_module(dev, monkeypatch):
    import torch
    from paper_2510_13797_amd import bc
    got = []
    for native in (True, False):
        if not native:
            monkeypatch.setattr(bc, "_paged_calls", None)
        both = Both(dev, 3, 12, 2, 128, 32, 200, seed=5)
        both.append([70, 3, 0], keep=[0, 0, 0])
        _, q = both.append([1, 4, 2], active=[1, 1, 0])
        got += [both.check_attend(q, [1, 4, 2], active=[1, 1, 0]), both.c.attend(both.c.append(both.packed(3), both.c.lengths, both.empty))]
    assert torch.equal(got[0], got[2]) and torch.equal(got[1], got[3])


def test_another_stream(dev):
    import torch
    both = Both(dev, 2, 12, 2, 128, 16, 200)
    both.append([150, 40])
    _, q = both.append([1, 1])
    expect = both.c.attend(q[:2])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = both.c.attend(q[:2].clone())
    stream.synchronize()
    assert torch.equal(got, expect)
