"""What a generation does around the attention over its cache, as cases that can be timed.

Three kinds:

  rope     the heads' norms and the rotation by position, from the packed output of a layer's projections to the
           q, k and v that the attention takes, and for training the gradients back to the packed form
  prompt   a chunk of new prompt rows for every sequence: appended to the cache, and their attention over what is
           resident and over each other (a long prompt in pieces, the next turn of a conversation)
  sample   the next token of every sequence from its logits, with temperature, top-k, top-p and min-p

`own` chooses between the plain form, elementary torch operations, and the calls of `paper_2510_13797_amd.bc`.
"""
import math

import numpy as np
import torch

own = False

# (query heads, KV heads, head dimension)
HEADS = ((12, 2, 128), (32, 8, 128), (14, 2, 64), (4, 1, 64), (4, 1, 128), (16, 2, 128), (5, 1, 128), (12, 2, 64))
MOST_ROPE_ELEMENTS = 16 * 8688 * 16 * 128
MOST_PROMPT_FLOPS = 4.3e12
MOST_LOGITS = 256 * 151936


def _rope(name, **kw):
    case = dict(kind="rope", R=64, Hq=12, Hkv=2, d=128, dtype="bf16", rot=128, norm=True, backward=False,
                far=32768, pad=0, shape=1)
    case.update(kw)
    return dict(name=name, **case) if name else case


def _prompt(name, **kw):
    case = dict(kind="prompt", B=1, Hq=32, Hkv=8, d=128, n_lo=512, n_hi=512, L_lo=7680, L_hi=7680, idle=0, shape=1)
    case.update(kw)
    return dict(name=name, **case) if name else case


def _sample(name, **kw):
    case = dict(kind="sample", B=64, V=151936, dtype="bf16", peaked=True, t_lo=0.6, t_hi=1.0, top_k=0, top_p=1.0,
                min_p=0.0, greedy=0.0, mixed=False, pad=0, shape=1)
    case.update(kw)
    return dict(name=name, **case) if name else case


def listed():
    return [
        # one user's next token in one layer: the latency of the call
        _rope("rope_one_token", R=1, Hq=32, Hkv=8),
        # a server's batch of 64 tokens; rotation alone, of three quarters of the head, as models without head norms have it
        _rope("rope_batch64", norm=False, rot=96),
        # the training step's rows at full size, 16 trajectories of 8688 rows: forward and gradients
        _rope("rope_train_full", R=16 * 8688, far=8192, backward=True),
        # a small fp32 model's micro-batch: odd rows, half of the head rotated, rows that lie apart in memory
        _rope("rope_train_f32_odd", R=1201, Hq=14, Hkv=2, d=64, dtype="f32", rot=32, backward=True, pad=24),
        # a short message to a long conversation: latency, and the bytes of the cache
        _prompt("prompt_short_turn", n_lo=7, n_hi=7, L_lo=16000, L_hi=16000),
        # one chunk of a long prompt, server's ordinary size
        _prompt("prompt_chunk512"),
        # turns of a ragged batch: from no row to some hundreds over caches of all ages, some sequences idle
        _prompt("prompt_ragged", B=24, Hq=12, Hkv=2, n_lo=0, n_hi=300, L_lo=0, L_hi=3500, idle=3),
        # chunks of 2048 rows far into four long documents
        _prompt("prompt_long", B=4, n_lo=2048, n_hi=2048, L_lo=30000, L_hi=30000),
        # one user's next token
        _sample("sample_one", B=1, t_lo=0.6, t_hi=0.6, top_k=20, top_p=0.95),
        # a server's batch, every request with settings of its own, some of them greedy
        _sample("sample_batch64_mixed", mixed=True, top_k=100, top_p=0.9, min_p=0.05, greedy=0.15),
        # rollouts of reinforcement learning: nearly flat rows of a large batch, top-p alone
        _sample("sample_flat256", B=256, peaked=False, t_lo=1.0, t_hi=1.0, top_p=0.95),
        # an odd vocabulary in fp32, min-p alone, rows of a wider buffer
        _sample("sample_f32_odd", B=37, V=50257, dtype="f32", min_p=0.02, t_lo=0.7, t_hi=1.3, pad=3),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("rope", "prompt", "sample"))
    while True:
        shape = rng.randrange(1, 1 << 20)
        if kind == "rope":
            Hq, Hkv, d = rng.choice(HEADS)
            case = _rope(None, R=log_int(1, 140000), Hq=Hq, Hkv=Hkv, d=d, dtype=rng.choice(("bf16", "bf16", "f32")),
                         rot=8 * rng.randint(1, d // 8), norm=rng.random() < 0.6, backward=rng.random() < 0.5,
                         far=log_int(16, 1000000), pad=8 * rng.choice((0, 0, 1, 5)), shape=shape)
            if case["R"] * (Hq + 2 * Hkv) * d * (2 if case["dtype"] == "f32" else 1) <= MOST_ROPE_ELEMENTS:
                return case
        elif kind == "prompt":
            Hq, Hkv, d = rng.choice(HEADS)
            n, L = log_int(1, 4096), log_int(1, 32000)
            B = log_int(1, 64)
            case = _prompt(None, B=B, Hq=Hq, Hkv=Hkv, d=d, n_lo=n // rng.choice((1, 2, 10)), n_hi=n,
                           L_lo=L // rng.choice((1, 3, 20)), L_hi=L, idle=rng.choice((0, 0, B // 4)), shape=shape)
            if 0 < work(case)["flops"] <= MOST_PROMPT_FLOPS and B * (n + L) * Hkv * d <= 200e6 and B * n * Hq * d <= 40e6:
                return case
        else:
            B, V = log_int(1, 256), log_int(100, 152064)
            case = _sample(None, B=B, V=V, dtype=rng.choice(("bf16", "bf16", "f32")), peaked=rng.random() < 0.7,
                           t_lo=rng.uniform(0.3, 0.9), t_hi=rng.uniform(0.9, 1.5),
                           top_k=rng.choice((0, 0, log_int(1, 2000))), top_p=rng.choice((1.0, rng.uniform(0.5, 0.99))),
                           min_p=rng.choice((0.0, 0.0, rng.uniform(0.005, 0.2))), greedy=rng.choice((0.0, 0.0, 0.2)),
                           mixed=rng.random() < 0.5, pad=rng.choice((0, 0, 1, 8)), shape=shape)
            if B * V * (2 if case["dtype"] == "f32" else 1) <= MOST_LOGITS:
                return case


# ---------------------------------------------------------------------------
# shapes of a case, from the case alone
# ---------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case.get("dtype", "bf16") == "bf16" else torch.float32


def _spans(case):
    """(resident rows, new rows, takes part, capacity) of every sequence, all [B]."""
    r = np.random.default_rng([case["shape"], 3])
    L = r.integers(case["L_lo"], case["L_hi"] + 1, size=case["B"])
    n = r.integers(case["n_lo"], case["n_hi"] + 1, size=case["B"])
    active = np.ones(case["B"], dtype=np.uint8)
    active[r.permutation(case["B"])[:case["idle"]]] = 0
    return L.astype(np.int64), n.astype(np.int64), active, (L + n + 40).astype(np.int64)


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    return {"rope": _prepare_rope, "prompt": _prepare_prompt, "sample": _prepare_sample}[case["kind"]](case, dev, gen)


def _prepare_rope(case, dev, gen):
    R, Hq, Hkv, d = case["R"], case["Hq"], case["Hkv"], case["d"]
    width = (Hq + 2 * Hkv) * d
    # the projections' output, a slice of wider rows where other projections lie beside it
    qkv = torch.empty(R, width + case["pad"], dtype=_dtype(case), device=dev)
    for at in range(0, R, 16384):
        qkv[at:at + 16384] = torch.randn(qkv[at:at + 16384].shape, generator=gen, device=dev)
    state = dict(case=case, qkv=qkv[:, :width],
                 positions=torch.randint(0, case["far"], (R,), generator=gen, device=dev, dtype=torch.int32),
                 inv_freq=torch.tensor([1e6 ** (-2.0 * i / case["rot"]) for i in range(case["rot"] // 2)],
                                       dtype=torch.float32, device=dev),
                 q_weight=None, k_weight=None)
    if case["norm"]:
        for name in ("q_weight", "k_weight"):
            state[name] = (1.0 + 0.2 * torch.randn(d, generator=gen, device=dev)).to(_dtype(case))
    if case["backward"]:
        for name, heads in (("dq", Hq), ("dk", Hkv), ("dv", Hkv)):
            state[name] = torch.randn(R, heads, d, generator=gen, device=dev)
    return state


def _prepare_prompt(case, dev, gen):
    B, Hq, Hkv, d = case["B"], case["Hq"], case["Hkv"], case["d"]
    L, n, active, cap = _spans(case)
    r = np.random.default_rng([case["shape"], 4])
    # what is resident: prompt, beacons of a ratio of 16, part of a window
    w = np.minimum(r.integers(0, 17, size=B), L)
    nb = np.minimum(r.integers(0, 400, size=B), L - w)
    P = L - w - nb
    base = np.concatenate([[0], np.cumsum(cap)[:-1]])
    off = np.concatenate([[0], np.cumsum(n)])

    def rnd(*shape):
        return torch.randn(*shape, generator=gen, device=dev).to(torch.bfloat16)

    def table(x):
        return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(dev)

    total, rows = int(off[-1]), int(cap.sum())
    state = dict(case=case, L=L, n=n, off=off, base=base, cap=cap, active_host=active,
                 k_slab=rnd(rows * Hkv * d), v_slab=rnd(rows * Hkv * d), q=rnd(total, Hq, d), k=rnd(total, Hkv, d),
                 v=rnd(total, Hkv, d), out=torch.zeros(total, Hq, d, device=dev), active=torch.from_numpy(active).to(dev),
                 start=table(np.stack([P, nb, w])), tables=table(np.stack([P, nb, w])))
    if own:
        from paper_2510_13797_amd import bc
        rt = bc.Runtime(B, Hq, Hkv, d, "bf16", 1.0 / math.sqrt(d), np.maximum(P, 0), np.full(B, 16), cap, dev)
        rt.k_slab, rt.v_slab = state["k_slab"], state["v_slab"]
        rt.P, rt.nb, rt.w = state["tables"][0], state["tables"][1], state["tables"][2]
        rt.cache.k_slab, rt.cache.v_slab = rt.k_slab.data_ptr(), rt.v_slab.data_ptr()
        rt.cache.P, rt.cache.nb, rt.cache.w = rt.P.data_ptr(), rt.nb.data_ptr(), rt.w.data_ptr()
        state["rt"] = rt
    return state


def _prepare_sample(case, dev, gen):
    B, V = case["B"], case["V"]
    r = np.random.default_rng([case["shape"], 5])
    z = 2.0 * torch.randn(B, V + case["pad"], generator=gen, device=dev)
    if case["peaked"]:          # a few dozen continuations that make sense, far above the rest
        few = min(V, 48)
        at = torch.randint(0, V, (B, few), generator=gen, device=dev)
        z.scatter_add_(1, at, 5.0 + 9.0 * torch.rand(B, few, generator=gen, device=dev))
    state = dict(case=case, logits=z.to(_dtype(case))[:, :V], u=torch.rand(B, generator=gen, device=dev))

    def per_row(values, dtype):
        return torch.from_numpy(np.asarray(values)).to(device=dev, dtype=dtype)

    some = (lambda: r.random(B) < 0.6) if case["mixed"] else (lambda: np.ones(B, dtype=bool))
    t = r.uniform(case["t_lo"], case["t_hi"], size=B)
    t[r.random(B) < case["greedy"]] = 0.0
    state["temperature"] = per_row(t, torch.float32)
    state["top_k"] = per_row(np.where(some(), np.ceil(case["top_k"] * r.uniform(0.5, 1.0, size=B)), 0), torch.int32) \
        if case["top_k"] else None
    state["top_p"] = per_row(np.where(some(), case["top_p"], 1.0), torch.float32) if case["top_p"] < 1.0 else None
    state["min_p"] = per_row(np.where(some(), case["min_p"], 0.0), torch.float32) if case["min_p"] > 0.0 else None
    return state


# ---------------------------------------------------------------------------
def run(state):
    kind = state["case"]["kind"]
    if own:
        from paper_2510_13797_amd import bc
        return {"rope": _own_rope, "prompt": _own_prompt, "sample": _own_sample}[kind](state, bc)
    return {"rope": _plain_rope, "prompt": _plain_prompt, "sample": _plain_sample}[kind](state)


def _own_rope(s, bc):
    c = s["case"]
    how = (s["positions"], s["inv_freq"], c["Hq"], c["Hkv"], c["d"], s["q_weight"], s["k_weight"])
    q, k, v = bc.qk_norm_rope(s["qkv"], *how)
    if not c["backward"]:
        return q, k, v
    return (q, k, v) + tuple(bc.qk_norm_rope_bwd(s["qkv"], s["dq"], s["dk"], s["dv"], *how))


def _own_prompt(s, bc):
    torch.add(s["start"], 0, out=s["tables"])
    s["rt"].prompt_step(s["k"], s["v"], s["q"], s["off"], active=s["active"], out=s["out"])
    return s["out"], s["tables"], s["k_slab"], s["v_slab"]


def _own_sample(s, bc):
    return bc.sample_tokens(s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], want_logprob=True)


# --------------------------------------------------------------------------- plain: rope
def _angles(s):
    a = s["positions"].double()[:, None] * s["inv_freq"].double()
    return torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]


def _turn(y, cos, sin, rot):
    a, b = y[..., :rot // 2], y[..., rot // 2:rot]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, y[..., rot:]], dim=-1)


def _plain_rope(s):
    c = s["case"]
    R, Hq, Hkv, d, rot, dt = c["R"], c["Hq"], c["Hkv"], c["d"], c["rot"], _dtype(c)
    cos, sin = _angles(s)
    xq, xk, xv = s["qkv"].float().view(R, Hq + 2 * Hkv, d).split([Hq, Hkv, Hkv], dim=1)
    outs, grads, dws = [], [], []
    for x, weight, name in ((xq, s["q_weight"], "dq"), (xk, s["k_weight"], "dk")):
        y = x
        if weight is not None:
            w = weight.float()
            rstd = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + 1e-6)
            y = x * rstd * w
        outs.append(_turn(y, cos, sin, rot).to(dt))
        if not c["backward"]:
            continue
        dy = _turn(s[name], cos, -sin, rot)
        if weight is not None:
            dws.append((dy * x * rstd).double().sum(dim=(0, 1)).float())
            dy = rstd * (w * dy - x * rstd * rstd * (w * dy * x).mean(dim=-1, keepdim=True))
        else:
            dws.append(None)
        grads.append(dy)
    outs.append(xv.to(dt))
    if not c["backward"]:
        return tuple(outs)
    return tuple(outs) + (torch.cat(grads + [s["dv"]], dim=1).to(dt).view(R, -1),) + tuple(dws)


# --------------------------------------------------------------------------- plain: prompt
def _slab_rows(slab, s, b, first, rows):
    """Rows [first, first + rows) of sequence b, [Hkv, rows, d]."""
    c = s["case"]
    at, cap = int(s["base"][b]) * c["Hkv"] * c["d"], int(s["cap"][b])
    return slab[at:at + cap * c["Hkv"] * c["d"]].view(c["Hkv"], cap, c["d"])[:, first:first + rows]


def _plain_prompt(s):
    c = s["case"]
    d, g = c["d"], c["Hq"] // c["Hkv"]
    torch.add(s["start"], 0, out=s["tables"])
    for b in range(c["B"]):
        L, n, at = int(s["L"][b]), int(s["n"][b]), int(s["off"][b])
        if not s["active_host"][b] or n == 0:
            continue
        _slab_rows(s["k_slab"], s, b, L, n).copy_(s["k"][at:at + n].transpose(0, 1))
        _slab_rows(s["v_slab"], s, b, L, n).copy_(s["v"][at:at + n].transpose(0, 1))
        keys, values = (_slab_rows(x, s, b, 0, L + n).float() for x in (s["k_slab"], s["v_slab"]))
        hidden = torch.arange(L + n, device=keys.device) > torch.arange(L, L + n, device=keys.device)[:, None]
        for h in range(c["Hkv"]):
            q = s["q"][at:at + n, h * g:(h + 1) * g].float().transpose(0, 1).reshape(g * n, d)
            x = (q @ keys[h].t().contiguous()).view(g, n, L + n) * (1.0 / math.sqrt(d))
            x.masked_fill_(hidden, float("-inf"))
            x = torch.exp(x - x.amax(dim=-1, keepdim=True))
            x = (x.view(g * n, L + n) @ values[h]) / x.sum(dim=-1).view(g * n, 1)
            s["out"][at:at + n, h * g:(h + 1) * g] = x.view(g, n, d).transpose(0, 1)
        s["tables"][0, b] = L + n
        s["tables"][1:, b] = 0
    return s["out"], s["tables"], s["k_slab"], s["v_slab"]


# --------------------------------------------------------------------------- plain: sample
def _plain_sample(s):
    z, at = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True)
    B, V = z.shape
    greedy = s["temperature"] == 0
    t = torch.where(greedy, torch.ones_like(s["temperature"]), s["temperature"]).double()
    y = (z.double() - z[:, :1].double()) / t[:, None]
    w = torch.exp(y)
    upto = torch.cumsum(w, dim=1)
    before = torch.cat([torch.zeros_like(w[:, :1]), upto[:, :-1]], dim=1)
    count = torch.full((B,), V, dtype=torch.int64, device=z.device)
    if s["top_k"] is not None:
        count = torch.where(s["top_k"] > 0, s["top_k"].long().clamp(max=V), count)
    count = torch.where(greedy, torch.ones_like(count), count)
    keep = torch.arange(V, device=z.device) < count[:, None]
    if s["top_p"] is not None:
        mass = s["top_p"].double()[:, None] * upto.gather(1, count[:, None] - 1)
        keep &= (before < mass) | (s["top_p"] >= 1.0)[:, None]
    if s["min_p"] is not None:
        keep &= y >= torch.log(s["min_p"].double())[:, None]
    keep[:, 0] = True
    last = keep.sum(dim=1, keepdim=True) - 1
    mass = upto.gather(1, last)
    pick = torch.minimum((upto <= s["u"].double()[:, None] * mass).sum(dim=1, keepdim=True), last)
    return at.gather(1, pick)[:, 0].int(), torch.log(w.gather(1, pick) / mass)[:, 0].float()


# ---------------------------------------------------------------------------
def work(case):
    es = 2 if case.get("dtype", "bf16") == "bf16" else 4
    if case["kind"] == "rope":
        R, d, qk, v = case["R"], case["d"], case["Hq"] + case["Hkv"], case["Hkv"]
        # the packed rows in, q, k and v out, a position a row; the gradients (fp32) in, the packed gradient out, and with
        # norms the packed rows of q and k once more for the backward call
        byts, flops = R * ((qk + v) * d * 2 * es + 4), R * qk * d * (8 if case["norm"] else 4)
        if case["backward"]:
            byts += R * ((qk + v) * d * (4 + es) + (qk * d * es if case["norm"] else 0) + 4)
            flops += R * qk * d * (16 if case["norm"] else 4)
        return {"bytes": byts, "flops": flops}
    if case["kind"] == "prompt":
        L, n, active, _ = _spans(case)
        L, n = L[(active != 0) & (n > 0)], n[(active != 0) & (n > 0)]
        kv, qrow = case["Hkv"] * case["d"], case["Hq"] * case["d"]
        pairs = int((n * L + n * (n + 1) // 2).sum())
        # resident K and V in, new rows in and out, the queries in, the output (fp32) out
        return {"bytes": int(L.sum()) * 4 * kv + int(n.sum()) * (8 * kv + 6 * qrow), "flops": 4 * pairs * qrow}
    # the logits once; an exponential of every one
    return {"bytes": case["B"] * (case["V"] * es + 28), "flops": 2 * case["B"] * case["V"]}


# ---------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "prompt": _exact_prompt, "sample": _exact_sample}[case["kind"]](case, s)


def _exact_rope(case, s):
    Hq, Hkv, d, rot = case["Hq"], case["Hkv"], case["d"], case["rot"]
    half = rot // 2
    parts, weights = [], [s["q_weight"], s["k_weight"]]
    weights = [None if w is None else w.double().requires_grad_(case["backward"]) for w in weights]
    dw = [None, None]
    for at in range(0, case["R"], 8192):
        rows = slice(at, min(at + 8192, case["R"]))
        x = s["qkv"][rows].double().unflatten(1, (Hq + 2 * Hkv, d)).requires_grad_(case["backward"])
        phase = s["positions"][rows].double()[:, None, None] * s["inv_freq"].double()
        unit = torch.polar(torch.ones_like(phase), phase)
        got = []
        for first, heads, weight in ((0, Hq, weights[0]), (Hq, Hkv, weights[1])):
            y = x[:, first:first + heads]
            if weight is not None:
                y = weight * y / torch.sqrt(y.square().sum(dim=-1, keepdim=True) / d + 1e-6)
            turned = torch.complex(y[..., :half].contiguous(), y[..., half:rot].contiguous()) * unit
            got.append(torch.cat([turned.real, turned.imag, y[..., rot:]], dim=-1))
        got.append(x[:, Hq + Hkv:] * 1.0)
        if case["backward"]:
            leaves = [x] + [w for w in weights if w is not None]
            grads = torch.autograd.grad(got, leaves, [s[n][rows].double() for n in ("dq", "dk", "dv")])
            got.append(grads[0].flatten(1))
            if weights[0] is not None:
                dw = [g if a is None else a + g for a, g in zip(dw, grads[1:])]
        parts.append([g.detach() for g in got])
    outs = tuple(torch.cat([p[i] for p in parts]) for i in range(len(parts[0])))
    return outs + tuple(dw) if case["backward"] else outs


def _exact_prompt(case, s):
    d, g = case["d"], case["Hq"] // case["Hkv"]
    out, tables = s["out"].double(), s["start"].clone()
    k_slab, v_slab = s["k_slab"].clone(), s["v_slab"].clone()
    for b in range(case["B"]):
        L, n, at = int(s["L"][b]), int(s["n"][b]), int(s["off"][b])
        if not s["active_host"][b] or n == 0:
            continue
        tables[:, b] = torch.tensor([L + n, 0, 0], dtype=torch.int32)
        for h in range(case["Hkv"]):
            first = (int(s["base"][b]) * case["Hkv"] + h * int(s["cap"][b])) * d
            for slab, new in ((k_slab, s["k"]), (v_slab, s["v"])):
                slab[first + L * d:first + (L + n) * d] = new[at:at + n, h].flatten()
            keys, values = (x[first:first + (L + n) * d].view(L + n, d).double() for x in (k_slab, v_slab))
            for i in range(0, n, 512):          # query rows i .. see keys up to their own
                m = min(512, n - i)
                for head in range(h * g, (h + 1) * g):
                    x = s["q"][at + i:at + i + m, head].double() @ keys[:L + i + m].t().contiguous() / math.sqrt(d)
                    x.masked_fill_(torch.ones_like(x, dtype=torch.bool).triu(L + i + 1), -math.inf)
                    out[at + i:at + i + m, head] = torch.softmax(x, dim=1) @ values[:L + i + m]
    return out, tables, k_slab, v_slab


def _exact_sample(case, s):
    if case["B"] * case["V"] > 60e6:
        return None
    z = s["logits"].double().cpu().numpy()
    u, t = s["u"].double().cpu().numpy(), s["temperature"].double().cpu().numpy()
    k, p, m = (None if s[x] is None else s[x].double().cpu().numpy() for x in ("top_k", "top_p", "min_p"))
    tokens, logprob = np.zeros(case["B"], np.int32), np.zeros(case["B"])
    for b, row in enumerate(z):
        order = np.argsort(-row, kind="stable")
        if t[b] == 0.0:
            tokens[b] = order[0]
            continue
        x = row[order]
        weight = np.exp((x - x[0]) / t[b])
        if k is not None and k[b] > 0:
            weight = weight[:int(k[b])]
        total = np.cumsum(weight)
        kept = len(weight)
        if p is not None and p[b] < 1.0:
            kept = min(kept, int(np.searchsorted(total, p[b] * total[-1], side="left")) + 1)
        if m is not None and m[b] > 0.0:
            kept = min(kept, max(1, int(((x[:len(weight)] - x[0]) / t[b] >= math.log(m[b])).sum())))
        pick = min(int(np.searchsorted(total[:kept], u[b] * total[kept - 1], side="right")), kept - 1)
        tokens[b], logprob[b] = order[pick], math.log(weight[pick] / total[kept - 1])
    return torch.from_numpy(tokens), torch.from_numpy(logprob)
