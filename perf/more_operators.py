"""A cache in pages of 8-bit entries, and the attention that reads it, as cases that can be timed.

Two kinds:

  append   rows of a layer's packed projections: norms of the heads, rotation by position, queries out in bf16, keys and values
           into the pages in 8 bits, with a scale for each block of 16 entries and head
  attend   the attention of a sequence's newest rows over its pages: one row (a decode step), a few (drafted tokens that are
           checked), many (a chunk of a prompt)

A page holds `page` entries of every KV head.  Entries are e4m3 values times their block's scale, a power of two: the least one for which
no entry written to the block since its first is beyond 448 times it.  Entries lie in groups of four: keys [d / 64][4][64], values
[d][4].

`own` chooses between the plain form, elementary torch operations, and the calls of `paper_2510_13797_amd.bc`.
"""
import math

import numpy as np
import torch

own = False

# (query heads, KV heads, head dimension)
HEADS = ((12, 2, 128), (32, 8, 128), (14, 2, 64), (4, 1, 64), (4, 1, 128), (16, 2, 128), (5, 1, 128), (12, 2, 64))
BLOCK = 16                     # entries that share a scale
E4M3 = torch.float8_e4m3fn
MOST_APPEND_ELEMENTS = 16 * 8688 * 16 * 128
MOST_FLOPS = 4.3e12
MOST_ENTRIES = 320e6           # elements of the keys


def _append(name, **kw):
    case = dict(kind="append", B=64, Hq=12, Hkv=2, d=128, dtype="bf16", rot=128, norm=True, n_lo=1, n_hi=1, L_lo=300, L_hi=1500,
                page=64, idle=0, evict=False, far=32768, pad=0, shape=1)
    case.update(kw)
    return dict(name=name, **case) if name else case


def _attend(name, **kw):
    case = dict(kind="attend", B=64, Hq=12, Hkv=2, d=128, n_lo=1, n_hi=1, L_lo=300, L_hi=1500, page=64, idle=0, share=1, shape=1)
    case.update(kw)
    return dict(name=name, **case) if name else case


def listed():
    return [
        # one user's next token in one layer: the latency of the call
        _append("append_one_token", B=1, Hq=32, Hkv=8, L_lo=3003, L_hi=3003),
        # a server's batch of 64 tokens
        _append("append_batch64"),
        # beacons take the place of their windows: entries behind the kept ones are dropped, half of the batch is due
        _append("append_beacons", L_lo=200, L_hi=700, idle=32, evict=True, page=16),
        # prompts at the training step's size: 16 of 8688 rows into empty pages
        _append("append_prompts_full", B=16, n_lo=8688, n_hi=8688, L_lo=0, L_hi=0, far=8192),
        # a small fp32 model's ragged chunks over sequences of all ages; half of the head rotated, rows that lie apart in memory
        _append("append_f32_ragged", B=24, Hq=14, Hkv=2, d=64, dtype="f32", rot=32, n_lo=0, n_hi=130, L_lo=0, L_hi=900, idle=3, pad=24,
                page=32),
        # one user's next token over a long conversation: latency
        _attend("attend_one_stream", B=1, Hq=32, Hkv=8, L_lo=16000, L_hi=16000),
        # rollouts, eight to a prompt whose pages they share
        _attend("attend_rollouts64", share=8),
        # the same batch without compression, far into its generations: the bytes of the cache
        _attend("attend_uncompressed64", L_lo=4352, L_hi=8704),
        # a small model's ragged batch in small pages
        _attend("attend_d64_ragged", B=24, Hq=14, Hkv=2, d=64, L_lo=1, L_hi=3500, page=16, idle=2),
        # eight drafted tokens a sequence are checked
        _attend("attend_drafts8", B=16, Hq=32, Hkv=8, n_lo=1, n_hi=8, L_lo=900, L_hi=6000),
        # one chunk of a long prompt, server's ordinary size
        _attend("attend_chunk512", B=1, Hq=32, Hkv=8, n_lo=512, n_hi=512, L_lo=7680, L_hi=7680),
        # chunks of 2048 rows far into four long documents
        _attend("attend_chunks_long", B=4, Hq=32, Hkv=8, n_lo=2048, n_hi=2048, L_lo=30000, L_hi=30000, page=128),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("append", "attend"))
    while True:
        Hq, Hkv, d = rng.choice(HEADS)
        B, n, L = log_int(1, 128), rng.choice((1, 1, log_int(1, 16), log_int(1, 4096))), log_int(1, 32000)
        how = dict(B=B, Hq=Hq, Hkv=Hkv, d=d, n_lo=max(n // rng.choice((1, 1, 2, 10)), 1 if n == 1 else 0), n_hi=n,
                   L_lo=L // rng.choice((1, 3, 20)), L_hi=L, page=1 << rng.randint(4, 8), idle=rng.choice((0, 0, B // 4)),
                   shape=rng.randrange(1, 1 << 20))
        if kind == "append":
            case = _append(None, dtype=rng.choice(("bf16", "bf16", "f32")), rot=8 * rng.randint(1, d // 8), norm=rng.random() < 0.6,
                           evict=rng.random() < 0.2, far=log_int(16, 1000000), pad=8 * rng.choice((0, 0, 1, 5)), **how)
            if (0 < int(_spans(case)[1].sum()) and B * n * (Hq + 2 * Hkv) * d * (2 if case["dtype"] == "f32" else 1) <= MOST_APPEND_ELEMENTS
                    and B * (n + L) * Hkv * d <= MOST_ENTRIES):
                return case
        else:
            case = _attend(None, share=rng.choice((1, 1, 4)), **how)
            if 0 < work(case)["flops"] <= MOST_FLOPS and B * (n + L) * Hkv * d <= MOST_ENTRIES and B * n * Hq * d <= 40e6:
                return case


# ---------------------------------------------------------------------------
# shapes of a case, from the case alone
# ---------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case.get("dtype", "bf16") == "bf16" else torch.float32


def _spans(case):
    """(entries in the cache, new rows, takes part, entries that are kept of those) of every sequence, all [B]."""
    r = np.random.default_rng([case["shape"], 3])
    B = case["B"]
    L = r.integers(case["L_lo"], case["L_hi"] + 1, size=B)
    n = r.integers(case["n_lo"], case["n_hi"] + 1, size=B)
    active = np.ones(B, dtype=np.uint8)
    active[r.permutation(B)[:case["idle"]]] = 0
    kept = np.maximum(L - 16, 0) if case.get("evict") else L
    return L.astype(np.int64), n.astype(np.int64), active, kept.astype(np.int64)


def _places(case):
    """(pages in the pool, table [B, pages of a sequence]): the pool's pages in no order; groups of `share` sequences have the whole pages of
    half of the shortest one's entries in common."""
    L, n, _, _ = _spans(case)
    r = np.random.default_rng([case["shape"], 4])
    B, page, share = case["B"], case["page"], case.get("share", 1)
    total = L + n if case["kind"] == "append" else np.maximum(L, n)
    pages = np.maximum(-(-total // page), 1)
    table = np.zeros((B, int(pages.max()) + 1), dtype=np.int64)
    common = np.zeros(B, dtype=np.int64)
    at = 0
    for b in range(B):
        first = b - b % share
        if b == first:
            common[b:b + share] = int(total[b:b + share].min()) // 2 // page if share > 1 else 0
        same = int(common[b]) if b > first else 0
        table[b, :same] = table[first, :same]
        table[b, same:pages[b]] = np.arange(at, at + pages[b] - same)
        at += int(pages[b]) - same
    order = r.permutation(at + 2)                    # (two pages that nobody has)
    used = np.arange(table.shape[1]) < pages[:, None]
    return at + 2, np.where(used, order[table], 0).astype(np.int32)


def _scale_of(most):
    """The least power of two s (2^-120 and up) with most <= 448 s."""
    m, e = torch.frexp(most.double().clamp(min=448.0 * 2.0 ** -120) / 448.0)
    return torch.ldexp(torch.ones_like(m), e - (m == 0.5).int()).float()


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    B, Hq, Hkv, d, page = case["B"], case["Hq"], case["Hkv"], case["d"], case["page"]
    L, n, active, kept = _spans(case)
    pool, table = _places(case)
    off = np.concatenate([[0], np.cumsum(n)])
    rows = int(off[-1])

    def there(x, dtype):
        return torch.from_numpy(np.ascontiguousarray(x)).to(device=dev, dtype=dtype)

    length = L if case["kind"] == "append" else np.maximum(L, n)          # (the newest n rows are in the cache when they attend)
    state = dict(case=case, rows=rows, n=n, length=length, table=there(table, torch.int32), start=there(length, torch.int32),
                 lengths=there(length, torch.int32), offsets=None if n.min() == n.max() == 1 else there(off, torch.int64), max_new=int(n.max()),
                 max_len=int(max(1, length.max())), active=there(active, torch.uint8) if case["idle"] else None, active_host=active, off=off)
    for name in ("k", "v"):                          # what is in the pages: entries of unit size, in blocks with their scales
        values = torch.empty(pool, Hkv, page // BLOCK, BLOCK * d, dtype=torch.uint8, device=dev)
        scales = torch.empty(pool, Hkv, page // BLOCK, device=dev)
        step = max(1, (1 << 26) // (Hkv * page * d))
        for at in range(0, pool, step):
            x = torch.randn(values[at:at + step].shape, generator=gen, device=dev)
            s = _scale_of(x.abs().amax(dim=-1))
            values[at:at + step] = (x / s[..., None]).to(E4M3).view(torch.uint8)
            scales[at:at + step] = s
        state[name + "_pages"], state[name + "_scale"] = values.view(pool, Hkv, page, d).view(E4M3), scales
    if case["kind"] == "append":
        width = (Hq + 2 * Hkv) * d
        # the projections' output, a slice of wider rows where other projections lie beside it
        qkv = torch.empty(rows, width + case["pad"], dtype=_dtype(case), device=dev)
        for at in range(0, rows, 16384):
            qkv[at:at + 16384] = torch.randn(qkv[at:at + 16384].shape, generator=gen, device=dev)
        state.update(qkv=qkv[:, :width], positions=torch.randint(0, case["far"], (rows,), generator=gen, device=dev, dtype=torch.int32),
                     inv_freq=torch.tensor([1e6 ** (-2.0 * i / case["rot"]) for i in range(case["rot"] // 2)], dtype=torch.float32, device=dev),
                     q_weight=None, k_weight=None, q=torch.zeros(rows, Hq, d, dtype=torch.bfloat16, device=dev),
                     keep=there(kept, torch.int32) if case["evict"] else None)
        if case["norm"]:
            for name in ("q_weight", "k_weight"):
                state[name] = (1.0 + 0.2 * torch.randn(d, generator=gen, device=dev)).to(_dtype(case))
    else:
        state["q"] = torch.randn(rows, Hq, d, generator=gen, device=dev).to(torch.bfloat16)
        state["out"] = torch.zeros(rows, Hq, d, device=dev)
    if own:
        from paper_2510_13797_amd import bc
        cache = bc.PagedCache(B, Hq, Hkv, d, pool, page, table.shape[1], dev, dtype=case.get("dtype", "bf16"))
        for name in ("k_pages", "v_pages", "k_scale", "v_scale", "table", "lengths"):
            getattr(cache, name).copy_(state[name])
            state[name] = getattr(cache, name)
        state["cache"] = cache
    return state


# ---------------------------------------------------------------------------
def run(state):
    append = state["case"]["kind"] == "append"
    if append:
        torch.add(state["start"], 0, out=state["lengths"])
    if own:
        (_own_append if append else _own_attend)(state)
    else:
        (_plain_append if append else _plain_attend)(state)
    if append:
        return tuple(state[x] for x in ("q", "k_pages", "v_pages", "k_scale", "v_scale", "lengths"))
    return state["out"]


def _own_append(s):
    s["cache"].append(s["qkv"], s["positions"], s["inv_freq"], row_offsets=s["offsets"], max_new=s["max_new"], q_weight=s["q_weight"],
                      k_weight=s["k_weight"], keep=s["keep"], active=s["active"], q=s["q"])


def _own_attend(s):
    s["cache"].attend(s["q"], row_offsets=s["offsets"], max_new=s["max_new"], max_len=s["max_len"], active=s["active"], out=s["out"])


# --------------------------------------------------------------------------- plain: entries of the pages
def _entries(s, name):
    """The bytes of the pages, and the dimensions a row number takes: keys [page, head, group, d / 64, 4, 64], values [page, head, group, d, 4]."""
    x = s[name + "_pages"].view(torch.uint8)
    pool, heads, page, d = x.shape
    return x.view(pool, heads, page // 4, d // 64, 4, 64) if name == "k" else x.view(pool, heads, page // 4, d, 4)


def _get(s, name, page, r):
    """Entries r of these pages (index tensors of one shape) as bytes [..., head, d]."""
    x = _entries(s, name)
    got = x[page, :, r // 4, :, r % 4, :] if name == "k" else x[page, :, r // 4, :, r % 4]
    return got.flatten(-2) if name == "k" else got


def _put(s, name, page, r, values):
    x = _entries(s, name)
    if name == "k":
        x[page, :, r // 4, :, r % 4, :] = values.unflatten(-1, (-1, 64))
    else:
        x[page, :, r // 4, :, r % 4] = values


def _scales_at(s, name, page, r):
    return s[name + "_scale"][page, :, r // BLOCK]


def _floats(values):
    return values.view(E4M3).float()


# --------------------------------------------------------------------------- plain: append
def _angles(s):
    a = s["positions"].double()[:, None] * s["inv_freq"].double()
    return torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]


def _turn(y, cos, sin, rot):
    a, b = y[..., :rot // 2], y[..., rot // 2:rot]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, y[..., rot:]], dim=-1)


def _plain_append(s):
    c = s["case"]
    R, B, Hq, Hkv, d, page = s["rows"], c["B"], c["Hq"], c["Hkv"], c["d"], c["page"]
    dev = s["qkv"].device
    # where every row goes
    n = torch.ones(B, dtype=torch.int64, device=dev) if s["offsets"] is None else s["offsets"][1:] - s["offsets"][:-1]
    first = torch.cumsum(n, 0) - n
    start = (s["lengths"] if s["keep"] is None else s["keep"]).long()
    taking = (n > 0) if s["active"] is None else (n > 0) & (s["active"] != 0)
    seq = torch.repeat_interleave(torch.arange(B, device=dev), n, output_size=R)
    slot = start[seq] + torch.arange(R, device=dev) - first[seq]
    rows = torch.nonzero(taking[seq])[:, 0]
    seq, slot = seq[rows], slot[rows]
    at, r = s["table"][seq, slot // page].long(), slot % page
    # norms and rotation
    cos, sin = _angles(s)
    xq, xk, xv = s["qkv"].float().view(R, Hq + 2 * Hkv, d).split([Hq, Hkv, Hkv], dim=1)
    turned = []
    for x, weight in ((xq, s["q_weight"]), (xk, s["k_weight"])):
        if weight is not None:
            x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + 1e-6) * weight.float()
        turned.append(_turn(x, cos, sin, c["rot"]))
    s["q"][rows] = turned[0][rows].to(torch.bfloat16)
    # entries that stay in the blocks where the rows begin
    begun = torch.nonzero(taking & (start % BLOCK != 0))[:, 0]
    old = start[begun, None] // BLOCK * BLOCK + torch.arange(BLOCK, device=dev)
    old_at, old_r = s["table"][begun[:, None], old // page].long(), old % page
    stays = old < start[begun, None]
    for name, x in (("k", turned[1][rows]), ("v", xv[rows])):
        scale = s[name + "_scale"]
        blocks = scale.shape[0] * scale.shape[2]
        block = at * scale.shape[2] + r // BLOCK
        most = torch.zeros(blocks, Hkv, device=dev).scatter_reduce_(0, block[:, None].expand(-1, Hkv), x.abs().amax(dim=-1), "amax")
        new = torch.zeros(blocks, device=dev).scatter_reduce_(0, block, torch.where(r % BLOCK == 0, 2.0, 1.0), "amax")[:, None]
        was = scale.transpose(1, 2).reshape(blocks, Hkv)
        need = _scale_of(most)
        now = torch.where(new == 2.0, need, torch.where(new == 1.0, torch.maximum(need, was), was))
        staying = _floats(_get(s, name, old_at, old_r)) * _scales_at(s, name, old_at, old_r)[..., None]
        scale.copy_(now.view(scale.shape[0], scale.shape[2], Hkv).transpose(1, 2))
        staying = (staying / _scales_at(s, name, old_at, old_r)[..., None]).to(E4M3).view(torch.uint8)
        _put(s, name, old_at[stays], old_r[stays], staying[stays])
        _put(s, name, at, r, (x / _scales_at(s, name, at, r)[..., None]).to(E4M3).view(torch.uint8))
    s["lengths"].copy_(torch.where(taking, start + n, s["lengths"].long()))


# --------------------------------------------------------------------------- plain: attend
def _plain_attend(s):
    c = s["case"]
    d, page, Hq, Hkv = c["d"], c["page"], c["Hq"], c["Hkv"]
    g = Hq // Hkv
    dev = s["q"].device
    takes = np.nonzero((s["active_host"] != 0) & (s["n"] > 0))[0]
    # as many sequences at a time as their scores fit a gigabyte
    most = int(s["n"][takes].max()), int(s["length"][takes].max())
    some = max(1, (1 << 28) // (Hq * most[0] * most[1] + 2 * Hkv * d * most[1]))
    for at in range(0, len(takes), some):
        b = takes[at:at + some]
        n, L = s["n"][b], s["length"][b]
        nm, Lm = int(n.max()), int(L.max())
        seq, L_dev, n_dev = (torch.from_numpy(x).to(dev) for x in (b, L, n))
        r = torch.arange(Lm, device=dev)
        there = r < L_dev[:, None]
        pages = torch.where(there, s["table"][seq][:, r // page].long(), 0)
        keys, values = (torch.where(there[..., None, None], _floats(_get(s, x, pages, (r % page).expand_as(pages)))
                                    * _scales_at(s, x, pages, (r % page).expand_as(pages))[..., None], 0.0).transpose(1, 2) for x in ("k", "v"))
        i = np.arange(nm)
        row = torch.from_numpy(s["off"][b][:, None] + np.minimum(i, np.maximum(n[:, None] - 1, 0))).to(dev)
        q = s["q"][row].float().view(len(b), nm, Hkv, g, d).permute(0, 2, 3, 1, 4).reshape(len(b) * Hkv, g * nm, d)
        x = (q @ keys.transpose(2, 3).reshape(len(b) * Hkv, d, Lm).contiguous()).view(len(b), Hkv * g, nm, Lm)
        x *= 1.0 / math.sqrt(d)
        hidden = r > (L_dev - n_dev)[:, None, None] + torch.arange(nm, device=dev)[:, None]
        x.masked_fill_(hidden[:, None], float("-inf"))
        x -= x.amax(dim=-1, keepdim=True)
        x.exp_()
        total = x.sum(dim=-1)
        o = x.view(len(b) * Hkv, g * nm, Lm) @ values.reshape(len(b) * Hkv, Lm, d).contiguous()
        o = (o.view(len(b), Hq, nm, d) / total[..., None]).transpose(1, 2)
        real = torch.from_numpy(i < n[:, None]).to(dev)
        s["out"][row[real]] = o[real]


# ---------------------------------------------------------------------------
def work(case):
    L, n, active, _ = _spans(case)
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    takes = (active != 0) & (n > 0)
    if case["kind"] == "append":
        # the packed rows and a position a row in; queries in bf16, keys and values in a byte out, a scale a block
        es, rows = 2 if case["dtype"] == "bf16" else 4, int(n[takes].sum())
        return {"bytes": rows * ((Hq + 2 * Hkv) * d * es + 4 + 2 * Hq * d + 2 * Hkv * d + 8 * Hkv // BLOCK),
                "flops": rows * (Hq + Hkv) * d * (8 if case["norm"] else 4)}
    length = np.maximum(L, n)
    _, table = _places(case)
    # keys and values of every entry once, however many sequences have it; queries in, outputs (fp32) out
    own_pages = np.zeros(int(table.max()) + 1, dtype=np.int64)
    for b in np.nonzero(takes)[0]:
        full = np.clip(length[b] - np.arange(table.shape[1]) * case["page"], 0, case["page"])
        np.maximum.at(own_pages, table[b][full > 0], full[full > 0])
    pairs = int((n * (length - n) + n * (n + 1) // 2)[takes].sum())
    return {"bytes": int(own_pages.sum()) * 2 * Hkv * (d + 4 / BLOCK) + int(n[takes].sum()) * 6 * Hq * d, "flops": 4 * pairs * Hq * d}


# ---------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return _exact_append(case, s) if case["kind"] == "append" else _exact_attend(case, s)


def _rows_of(s, name, b, count):
    """Entries [0, count) of a sequence: (values in 64 bits [head, count, d], scales [head, count])."""
    page, pool = s["case"]["page"], s[name + "_pages"]
    pages = s["table"][b, :-(-count // page)].long()
    x = pool.view(torch.uint8)[pages].view(E4M3).double()
    P, H, _, d = x.shape
    if name == "k":
        x = x.view(P, H, page // 4, d // 64, 4, 64).permute(1, 0, 2, 4, 3, 5)
    else:
        x = x.view(P, H, page // 4, d, 4).permute(1, 0, 2, 4, 3)
    scale = s[name + "_scale"][pages].double().repeat_interleave(BLOCK, dim=2).transpose(0, 1)
    return x.reshape(H, P * page, d)[:, :count], scale.reshape(H, P * page)[:, :count]


def _exact_append(case, s):
    """Values in the pages without their last rounding."""
    Hq, Hkv, d, rot, page = case["Hq"], case["Hkv"], case["d"], case["rot"], case["page"]
    half, eps = rot // 2, 1e-6
    x = s["qkv"].double().unflatten(1, (Hq + 2 * Hkv, d))
    phase = s["positions"].double()[:, None, None] * s["inv_freq"].double()
    unit = torch.polar(torch.ones_like(phase), phase)
    heads = []
    for lo, hi, weight in ((0, Hq, s["q_weight"]), (Hq, Hq + Hkv, s["k_weight"])):
        y = x[:, lo:hi]
        if weight is not None:
            y = weight.double() * y / torch.sqrt(y.square().sum(dim=-1, keepdim=True) / d + eps)
        z = torch.complex(y[..., :half].contiguous(), y[..., half:rot].contiguous()) * unit
        heads.append(torch.cat([z.real, z.imag, y[..., rot:]], dim=-1))
    _, n, active, kept = _spans(case)
    q, lengths = s["q"].double(), s["start"].clone()
    pages = {name: s[name + "_pages"].double() for name in ("k", "v")}
    scales = {name: s[name + "_scale"].double() for name in ("k", "v")}
    # row numbers that are written, of all sequences together: (page, row of the page), from where in the batch, and the entries that stay
    to, source, stay = [], [], []
    table = s["table"].cpu().numpy()
    for b in np.nonzero((active != 0) & (n > 0))[0]:
        a, e = int(kept[b]), int(kept[b] + n[b])
        lengths[b] = e
        for entries, into in ((np.arange(a, e), to), (np.arange(a // BLOCK * BLOCK, a), stay)):
            into.append(np.stack([table[b, entries // page], entries % page]))
        source.append(np.arange(int(s["off"][b]), int(s["off"][b + 1])))
    if to:
        (tp, tr), (sp, sr) = (torch.from_numpy(np.concatenate(x, axis=1)).long().to(q.device) for x in (to, stay))
        rows = torch.from_numpy(np.concatenate(source)).to(q.device)
        q[rows] = heads[0][rows]
        for name, new in (("k", heads[1][rows]), ("v", x[rows, Hq + Hkv:])):
            per = page // BLOCK
            old = scales[name].transpose(1, 2).reshape(-1, Hkv)
            base = torch.zeros_like(old)
            base[sp * per + sr // BLOCK] = old[sp * per + sr // BLOCK]          # blocks that hold entries already
            most = torch.zeros_like(old).index_reduce_(0, tp * per + tr // BLOCK, new.abs().amax(dim=-1), "amax")
            touched = torch.zeros(len(old), 1, dtype=torch.bool, device=q.device)
            touched[tp * per + tr // BLOCK] = True
            least = torch.exp2(torch.ceil(torch.log2(most.clamp(min=2.0 ** -130) / 448.0)).clamp(min=-120.0))
            now = torch.where(touched, torch.maximum(base, least), old)
            if name == "k":
                view = pages[name].view(-1, Hkv, page // 4, d // 64, 4, 64)
                view[sp, :, sr // 4, :, sr % 4, :] *= (old / now)[sp * per + sr // BLOCK][..., None, None]
                view[tp, :, tr // 4, :, tr % 4, :] = (new / now[tp * per + tr // BLOCK][..., None]).unflatten(-1, (d // 64, 64))
            else:
                view = pages[name].view(-1, Hkv, page // 4, d, 4)
                view[sp, :, sr // 4, :, sr % 4] *= (old / now)[sp * per + sr // BLOCK][..., None]
                view[tp, :, tr // 4, :, tr % 4] = new / now[tp * per + tr // BLOCK][..., None]
            scales[name] = now.view(-1, per, Hkv).transpose(1, 2).contiguous()
    return q, pages["k"], pages["v"], scales["k"], scales["v"], lengths


def _exact_attend(case, s):
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    out = s["out"].double()
    for b in range(case["B"]):
        n, L, at = int(s["n"][b]), int(s["length"][b]), int(s["off"][b])
        if n == 0 or not s["active_host"][b]:
            continue
        (K, ks), (V, vs) = _rows_of(s, "k", b, L), _rows_of(s, "v", b, L)
        K, V = K * ks[..., None], V * vs[..., None]
        for i in range(0, n, 512):                  # query rows i .. see entries up to their own
            m = min(512, n - i)
            seen = L - n + i + m
            for h in range(Hkv):
                q = s["q"][at + i:at + i + m, h * (Hq // Hkv):(h + 1) * (Hq // Hkv)].double().transpose(0, 1)
                x = torch.matmul(q.reshape(-1, d), K[h, :seen].t().contiguous()).view(-1, m, seen) / math.sqrt(d)
                x.masked_fill_(torch.ones(m, seen, dtype=torch.bool, device=x.device).triu(L - n + i + 1), -math.inf)
                o = torch.matmul(torch.softmax(x, dim=-1).view(-1, seen), V[h, :seen].contiguous())
                out[at + i:at + i + m, h * (Hq // Hkv):(h + 1) * (Hq // Hkv)] = o.view(-1, m, d).transpose(0, 1)
    return out
