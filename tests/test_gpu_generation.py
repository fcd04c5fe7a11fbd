"""The calls around the attention, run together as a model uses them: a prompt in chunks, decode steps with beacons, sampled tokens, another
turn; and a training step's forward and gradients from the packed projections back to them.

Every stage is checked against the fp64 oracle on what the stage before left on the device, with the tolerances of the stages' own
tests; the training chain against autograd in fp64 as a whole."""
import numpy as np
import pytest

from oracle import attention as OA
from oracle import rope as OR
from oracle import sample as OS

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch.device("cuda:0")


class Model:
    """One attention layer between an embedding and a vocabulary: weights for tests alone."""
    V, E, Hq, Hkv, d = 700, 96, 4, 2, 64

    def __init__(self, dev):
        import torch
        g = torch.Generator(device=dev).manual_seed(11)
        r = lambda *shape: torch.randn(*shape, generator=g, device=dev)
        self.embedding = r(self.V + 1, self.E)                       # (the last one: the beacon)
        self.qkv = r(self.E, (self.Hq + 2 * self.Hkv) * self.d) / self.E ** 0.5
        self.out = r(self.Hq * self.d, self.E) / (self.Hq * self.d) ** 0.5
        self.head = 1.5 * r(self.E, self.V) / self.E ** 0.5
        self.weights = [(1 + 0.2 * r(self.d)).bfloat16() for _ in range(2)]
        self.inv_freq = (1e4 ** (-torch.arange(24, device=dev) / 24.0)).float()      # 48 of 64 elements turn

    def project(self, tokens, positions):
        import torch
        from paper_2510_13797_amd import bc
        x = self.embedding[tokens]
        packed = (x @ self.qkv).bfloat16()
        pos = torch.as_tensor(positions, dtype=torch.int32, device=x.device)
        q, k, v = bc.qk_norm_rope(packed, pos, self.inv_freq, self.Hq, self.Hkv, self.d, *self.weights)
        heads = packed.double().cpu().numpy().reshape(len(x), -1, self.d)
        p, f = pos.cpu().numpy(), self.inv_freq.double().cpu().numpy()
        for got, w, first in ((q, self.weights[0], 0), (k, self.weights[1], self.Hq)):
            ref = OR.norm_rope(heads[:, first:first + got.shape[1]], w.double().cpu().numpy(), p, f, 1e-6)
            # (half a step of bf16, and 1.2e-6 of what is added: values below 8)
            assert (np.abs(got.double().cpu().numpy() - ref) <= 2.0 ** -8 * np.abs(ref) + 2e-5).all()
        return x, q, k, v

    def logits(self, x, attention):
        return (x + attention.flatten(1) @ self.out) @ self.head


def _np(t):
    return t.double().cpu().numpy()


def test_prompt_in_chunks_decode_with_beacons_and_another_turn(dev):
    import torch
    from paper_2510_13797_amd import bc
    m, B, c = Model(dev), 3, 3
    r = np.random.default_rng(0)
    rt = bc.Runtime(B, m.Hq, m.Hkv, m.d, "bf16", 1 / np.sqrt(m.d), np.zeros(B, np.int32), np.full(B, c), np.full(B, 260), dev)
    K = [np.zeros((0, m.Hkv, m.d)) for _ in range(B)]
    V = [np.zeros((0, m.Hkv, m.d)) for _ in range(B)]
    seen = np.zeros(B, int)                                           # position of the next token
    last = None

    def turn(lengths):
        nonlocal last
        off = np.concatenate([[0], np.cumsum(lengths)])
        tokens = torch.from_numpy(r.integers(0, m.V, off[-1])).to(dev)
        pos = np.concatenate([seen[b] + np.arange(n) for b, n in enumerate(lengths)])
        x, q, k, v = m.project(tokens, pos)
        out = rt.prompt_step(k, v, q, off)
        qn, kn, vn, got = _np(q), _np(k), _np(v), _np(out)
        for b, n in enumerate(lengths):
            rows = slice(off[b], off[b + 1])
            L = len(K[b])
            K[b], V[b] = np.concatenate([K[b], kn[rows]]), np.concatenate([V[b], vn[rows]])
            for i in range(n):
                ref = OA.decode_attention(qn[off[b] + i], K[b][:L + i + 1], V[b][:L + i + 1], rt.shape.scale)
                assert np.abs(got[off[b] + i] - ref).max() <= 1e-4
            seen[b] += n
        ends = torch.from_numpy(off[1:] - 1).to(dev)
        return sample(m.logits(x[ends], out[ends]))

    def sample(z):
        u = torch.from_numpy(r.random(B).astype(np.float32)).to(dev)
        kw = dict(temperature=[0.8, 0.0, 1.2], top_k=[40, 0, 0], top_p=[0.95, 1.0, 0.9])
        args = {n: torch.tensor(x, dtype=torch.int32 if n == "top_k" else torch.float32, device=dev) for n, x in kw.items()}
        token, logprob = bc.sample_tokens(z, u, want_logprob=True, **args)
        for b in range(B):
            want, wlp, margin = OS.sample(_np(z[b]), float(u[b]), *(float(args[n][b]) for n in ("temperature", "top_k", "top_p")))
            assert margin > 1e-9 and token[b].item() == want and abs(logprob[b].item() - wlp) <= 2.0 ** -24 * abs(wlp) + 1e-7
        return token.long()

    def decode(steps):
        nonlocal last
        P = [len(x) for x in K]
        nb = w = 0
        for _ in range(steps):
            x, q, k, v = m.project(last, seen)
            _, _, bk, bv = m.project(torch.full((B,), m.V, device=dev), seen + 1)
            out = rt.decode_step(k, v, q, bk, bv)
            w += 1
            for b in range(B):
                K[b], V[b] = np.concatenate([K[b], _np(k[b:b + 1])]), np.concatenate([V[b], _np(v[b:b + 1])])
                ref = OA.decode_attention(_np(q[b]), K[b], V[b], rt.shape.scale)
                assert np.abs(_np(out[b]) - ref).max() <= 1e-4
                if w == c:
                    K[b] = np.concatenate([K[b][:P[b] + nb], _np(bk[b:b + 1])])
                    V[b] = np.concatenate([V[b][:P[b] + nb], _np(bv[b:b + 1])])
            if w == c:
                nb, w = nb + 1, 0
                seen[:] += 1
            seen[:] += 1
            last = sample(m.logits(x, out))

    turn([5, 40, 17])
    last = turn([33, 2, 0])                                           # the same prompts' second pieces
    decode(8)
    last = turn([4, 50, 9])                                           # the next turn: beacons and a part of a window stay
    decode(4)
    for b in range(B):
        Kd, Vd = rt.resident(b)
        assert np.array_equal(Kd, K[b]) and np.array_equal(Vd, V[b])
    assert rt.tables()[2] == 0


def test_training_chain_against_autograd(dev):
    import torch
    from paper_2510_13797_amd import bc
    Hq, Hkv, d, rot = 4, 2, 64, 48
    off, P, c = [0, 37, 90], np.array([10, 21], np.int32), np.array([3, 0], np.int32)
    g = torch.Generator(device=dev).manual_seed(2)
    r = lambda *shape: torch.randn(*shape, generator=g, device=dev)
    qkv, dout = r(90, (Hq + 2 * Hkv) * d).bfloat16(), r(90, Hq, d).bfloat16()
    w = [(1 + 0.2 * r(d)).bfloat16() for _ in range(2)]
    f = (1e4 ** (-torch.arange(rot // 2, device=dev) / (rot // 2))).float()
    pos = torch.cat([torch.arange(37), torch.arange(53)]).int().to(dev)
    scale = d ** -0.5
    q, k, v = bc.qk_norm_rope(qkv, pos, f, Hq, Hkv, d, *w)
    args = (off, P, c, Hq, Hkv, d, scale)
    out, lse = bc.prefill_attn(q, k, v, *args)
    dq, dk, dv = bc.prefill_attn_bwd(q, k, v, out, lse, dout, *args)
    dqkv, dqw, dkw = bc.qk_norm_rope_bwd(qkv, dq, dk, dv, pos, f, Hq, Hkv, d, *w)

    x = qkv.double().cpu().requires_grad_(True)
    wd = [y.double().cpu().requires_grad_(True) for y in w]
    a = pos.double().cpu()[:, None] * f.double().cpu()
    cos, sin = a.cos()[:, None], a.sin()[:, None]
    heads = x.view(90, -1, d)

    def turned(y, weight):
        y = weight * y / (y.square().mean(-1, keepdim=True) + 1e-6).sqrt()
        lo, hi = y[..., :rot // 2], y[..., rot // 2:rot]
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin, y[..., rot:]], -1)

    class Rounded(torch.autograd.Function):               # what the attention is given: bf16, its gradient that of the unrounded
        @staticmethod
        def forward(ctx, y):
            return y.bfloat16().double()

        @staticmethod
        def backward(ctx, dy):
            return dy

    qd, kd, vd = Rounded.apply(turned(heads[:, :Hq], wd[0])), Rounded.apply(turned(heads[:, Hq:Hq + Hkv], wd[1])), heads[:, Hq + Hkv:]
    parts = []
    for b in range(2):
        rows = slice(off[b], off[b + 1])
        S = off[b + 1] - off[b]
        see = torch.from_numpy(OA.visible_mask(S, int(P[b]), int(c[b])))
        s = torch.einsum("ihd,jhd->hij", qd[rows], kd[rows].repeat_interleave(Hq // Hkv, 1)) * scale
        s = s.masked_fill(~see, -torch.inf).softmax(-1)
        parts.append(torch.einsum("hij,jhd->ihd", s, vd[rows].repeat_interleave(Hq // Hkv, 1)))
    ref = torch.cat(parts)
    ref.backward(dout.double().cpu())
    # q and k may lie a step of bf16 apart where the oracle's value falls next to a border (2^-8 of values below 6: scores off by up to 1e-2 for
    # single rows); the gradients' own rounding is half a step of bf16
    assert (out.double().cpu() - ref.detach()).abs().max() <= 2e-2
    for got, want in ((dqkv, x.grad), (dqw, wd[0].grad), (dkw, wd[1].grad)):
        err = (got.double().cpu() - want).norm() / want.norm()
        assert err <= 5e-3, err
