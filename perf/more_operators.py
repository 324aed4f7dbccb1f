"""Measured calls of the attention with a sliding window and first tokens that stay visible, in
training and over a paged bf16 cache, and of what fills that cache.

``append``  new tokens of a step or a prompt: norms of queries and keys for each head where there
            are weights, the rotation by position, keys and values into the cache's pages.
``attend``  attention of new queries over the paged cache: single tokens, a few drafted tokens, a
            chunk of a prompt; with and without a window.
``window``  attention inside a window on whole sequences, query heads sharing key/value heads; with
            ``train`` the gradients of queries, keys and values too.

``run()`` makes one such call, in plain torch or, where ``own`` is set, through the public entry
points; ``exact()`` is the same from the definitions in fp64.

A query at position p sees the keys j <= p + right (right < 0: any) with j >= p - left (left < 0:
any) or j < sinks.  The cache is two pools [pages, heads, page, d]; token t of a sequence is row
t % page of the page that its row of the table names at t // page.
"""
import math

import torch

own = False

BF16, F32 = "bf16", "f32"
_TORCH = {BF16: torch.bfloat16, F32: torch.float32}
_BYTES = {BF16: 2, F32: 4}
_EPS = 1e-6


def _append(B, Hq, Hk, N, lo, hi, page, d, rot=None, dtype=BF16, norm=False, interleaved=False,
            far=0, ragged=False, name=None):
    """Sequences of lo..hi tokens, the last N of them new (ragged: from 1 to N)."""
    c = {"op": "append", "B": B, "Hq": Hq, "Hk": Hk, "N": N, "lo": lo, "hi": hi, "page": page, "d": d,
         "rot": d if rot is None else rot, "dtype": dtype, "norm": norm, "interleaved": interleaved,
         "far": far, "ragged": ragged}
    return dict(c, name=name) if name else c


def _attend(B, Hq, Hk, N, lo, hi, page, d, left=-1, sinks=0, out=BF16, name=None):
    """N queries of each sequence over the sequence's lo..hi stored tokens, theirs the last."""
    c = {"op": "attend", "B": B, "Hq": Hq, "Hk": Hk, "N": N, "lo": lo, "hi": hi, "page": page, "d": d,
         "left": left, "right": 0, "sinks": sinks, "out": out}
    return dict(c, name=name) if name else c


def _window(B, Hq, Hk, N, d, left, right=0, sinks=0, out=BF16, train=False, packed=False, name=None):
    c = {"op": "window", "B": B, "Hq": Hq, "Hk": Hk, "N": N, "d": d, "left": left, "right": right,
         "sinks": sinks, "out": out, "train": train, "packed": packed}
    return dict(c, name=name) if name else c


def listed():
    return [
        # One token of one conversation: launch and latency.
        _append(1, 32, 8, 1, 4097, 4097, 16, 128, name="append_b1"),
        # Decode step of a serving batch, heads normed before they turn.
        _append(64, 32, 8, 1, 200, 1000, 16, 128, norm=True, name="append_b64"),
        # A prompt of 4K tokens, slices of a packed projection output.
        _append(2, 16, 16, 4096, 4096, 4096, 64, 128, name="append_prompt_4k"),
        # Ragged prompts in fp32, half of each head rotated, neighbouring elements as pairs.
        _append(8, 12, 4, 777, 777, 1500, 32, 64, rot=32, dtype=F32, norm=True, interleaved=True,
                far=100000, ragged=True, name="append_ragged_777"),
        # Decode step of a single conversation.
        _attend(1, 32, 8, 1, 4097, 4097, 16, 128, name="attend_b1_4k"),
        # Decode step of a large serving batch.
        _attend(64, 32, 8, 1, 8192, 8192, 64, 128, name="attend_b64_8k"),
        # Four drafted tokens of each of 16 sequences of very different lengths, in a window.
        _attend(16, 12, 4, 4, 100, 16384, 32, 64, left=1023, sinks=4, name="draft_window"),
        # Chunked prefill: a few hundred new tokens against a long cache, ragged on both sides.
        _attend(1, 32, 8, 200, 20011, 20011, 16, 128, name="chunk_200_of_20k"),
        # An encoder's local attention, both ways, packed projections, a length that divides by
        # nothing, fp32 output.
        _window(8, 12, 12, 777, 64, 64, 64, out=F32, packed=True, name="local_777"),
        # Prompt of a decoder layer with a window and four first tokens.
        _window(2, 32, 8, 4096, 128, 511, sinks=4, name="window_4k"),
        # Training step of a causal layer without a window on a ragged length, heads shared by four.
        _window(4, 8, 2, 1000, 64, -1, train=True, name="train_1000"),
        # Training step of a long-context layer.
        _window(1, 32, 8, 8192, 128, 1023, sinks=4, train=True, name="train_8k"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "attend", "attend", "chunk", "window", "window", "train", "train"])
    d, page, Hk = rng.choice([64, 128]), 16 * rng.choice([1, 1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 8, 16])
    Hq = Hk * rng.choice([1, 2, 3, 4, 8])
    left, sinks = rng.choice([-1, _log_int(rng, 8, 8192)]), rng.choice([0, 0, 1, 4, 100])
    if op == "append":
        B, N = _log_int(rng, 1, 64), rng.choice([1, _log_int(rng, 1, 8192)])
        while B * N * (Hq + 2 * Hk) > 2 * 4096 * 48:
            N = (N + 1) // 2
        more = _log_int(rng, 1, 1000)
        return _append(B, Hq, Hk, N, N, N + more, page, d, rot=rng.choice([0, 16, d // 2, d, d]),
                       dtype=rng.choice([BF16, BF16, F32]), norm=rng.random() < 0.4,
                       interleaved=rng.random() < 0.3, far=rng.choice([0, _log_int(rng, 1, 1000000)]),
                       ragged=rng.random() < 0.4)
    if op == "chunk":
        B, N, hi = rng.randint(1, 2), _log_int(rng, 9, 1024), _log_int(rng, 1024, 32768)
        while B * Hq * N * hi > 32 * 200 * 20011:
            N = (N + 1) // 2
        return _attend(B, Hq, Hk, N, max(N, hi * 2 // 3), max(N, hi), page, d, left, sinks if left >= 0 else 0)
    if op == "attend":
        B, N, hi = _log_int(rng, 1, 64), rng.choice([1, 1, 1, 2, 4, 7]), _log_int(rng, 40, 32768)
        while B * Hk * hi > 64 * 8 * 8192 or B * Hq * N * hi > 64 * 32 * 8192:
            hi = (hi + 1) // 2
        return _attend(B, Hq, Hk, N, max(N, rng.choice([hi, hi // 20])), max(N, hi), page, d, left,
                       sinks if left >= 0 else 0, out=rng.choice([BF16, BF16, F32]))
    B, N, right = rng.randint(1, 8), _log_int(rng, 64, 8192), rng.choice([0, 0, 0, -1, left])
    while B * Hq * N * N > 32 * 8192 * 8192 * (0.5 if op == "train" else 1):
        N = (N + 1) // 2
    return _window(B, Hq, Hk, N, d, left, right, sinks if left >= 0 else 0, out=rng.choice([BF16, F32]) if op == "window" else BF16,
                   train=op == "train", packed=rng.random() < 0.5)


def _lens(c):
    """The lengths of a case's sequences: lo to hi, in no order."""
    B, lo, hi = c["B"], c["lo"], c["hi"]
    return [hi if i == 0 else lo + (hi - lo) * (i * 37 % B) // B for i in range(B)]


def _news(c):
    """New tokens of each sequence."""
    return [c["N"] - (i * 29 % c["B"]) * (c["N"] - 1) // c["B"] if c.get("ragged") else c["N"] for i in range(c["B"])]


# ---- inputs -----------------------------------------------------------------------------------


def _normal(g, shape, dtype, std=1.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _heads(g, B, N, sizes, d, dtype, packed, std=1.0):
    """Tensors [B, heads, N, d]: slices of one projection output [B, N, all heads, d], or apart."""
    if packed:
        return [x.transpose(1, 2) for x in _normal(g, (B, N, sum(sizes), d), dtype, std).split(sizes, 2)]
    return [_normal(g, (B, h, N, d), dtype, std) for h in sizes]


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    B, Hq, Hk, N, d = c["B"], c["Hq"], c["Hk"], c["N"], c["d"]
    if c["op"] == "window":
        s["q"], s["k"], s["v"] = _heads(g, B, N, [Hq, Hk, Hk], d, torch.bfloat16, c["packed"], 1.2)
        if c["train"]:
            s["do"], = _heads(g, B, N, [Hq], d, torch.bfloat16, c["packed"])
        return s
    # The pools, what they hold, and every sequence's pages in no order.
    P, lens = c["page"], _lens(c)
    pages = [-(-n // P) for n in lens]
    order = torch.randperm(sum(pages), generator=g, device="cuda").int()
    table = torch.zeros((B, max(pages)), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    s["table"] = table
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for name in ("k_pool", "v_pool"):
        s[name] = _normal(g, (sum(pages), Hk, P, d), torch.bfloat16)
    if c["op"] == "attend":
        s["q"] = _normal(g, (B, N, Hq, d), torch.bfloat16, 1.5).transpose(1, 2)
        if c["left"] >= 0:
            # Pages that the window has left behind have gone to other sequences.
            for b, n in enumerate(lens):
                first = max(0, n - N - c["left"]) // P
                table[b, -(-c["sinks"] // P):first] = -1
        return s
    dt = _TORCH[c["dtype"]]
    s["q"], s["k"], s["v"] = _heads(g, B, N, [Hq, Hk, Hk], d, dt, True, 1.5)
    s["wq"], s["wk"] = ((1 + _normal(g, (d,), torch.float32, 0.3)).to(dt) if c["norm"] else None for _ in range(2))
    s["inv_freq"] = None
    if c["rot"]:
        s["inv_freq"] = (10000.0 ** (-torch.arange(c["rot"] // 2, device="cuda", dtype=torch.float64) * 2 / c["rot"])).float()
    s["new"] = torch.tensor(_news(c), dtype=torch.int32, device="cuda") if c["ragged"] else None
    s["positions"] = None
    if c["far"]:
        s["positions"] = c["far"] + 3 * torch.arange(B, device="cuda")[:, None] + torch.arange(N, device="cuda")
    # Rows behind a sequence's new tokens stay as they are in the caller's buffer.
    s["q_out"] = torch.zeros((B, Hq, N, d), dtype=torch.bfloat16, device="cuda")
    return s


# ---- one pass, plain --------------------------------------------------------------------------


def _turn(x, cos, sin, c):
    """x [B, H, N, d] with its first rot elements rotated in pairs."""
    r = c["rot"]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _rows(s):
    """Of every row of a call [B, N]: its token's place in the sequence, and whether it is one."""
    c = s["case"]
    new = s["lens"].new_full((c["B"],), c["N"]) if s.get("new") is None else s["new"]
    i = torch.arange(c["N"], device="cuda")
    return (s["lens"] - new).long()[:, None] + i, i < new[:, None]


def _plain_append(s):
    c = s["case"]
    at, real = _rows(s)
    pos = at if s["positions"] is None else s["positions"]
    cos, sin = torch.ones((), device="cuda"), torch.zeros((), device="cuda")
    if c["rot"]:
        a = (pos.double()[..., None] * s["inv_freq"].double())[:, None]
        cos, sin = a.cos().float(), a.sin().float()
    out = []
    for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"])):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + _EPS) * w.float()
        out.append(_turn(y, cos, sin, c).to(torch.bfloat16))
    s["q_out"].copy_(torch.where(real[:, None, :, None], out[0], s["q_out"]))
    b, i = real.nonzero(as_tuple=True)
    page, row = s["table"][b, at[b, i] // c["page"]].long(), at[b, i] % c["page"]
    s["k_pool"][page, :, row] = out[1][b, :, i]
    s["v_pool"][page, :, row] = s["v"][b, :, i].to(torch.bfloat16)
    return {"q": s["q_out"], "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _stored(s, name):
    """fp32 [B, Hk, tokens, d] of every sequence's pages."""
    x = s[name][s["table"].long().clamp(min=0)]                     # [B, pages, Hk, page, d]
    return x.transpose(1, 2).flatten(2, 3).float()


def _hidden(at, keys, last, c):
    """[B, N, keys]: what the query at place at [B, N] does not see; last [B]: tokens there are."""
    j, p = torch.arange(keys, device="cuda"), at[..., None]
    hide = j >= last[:, None, None]
    if c["right"] >= 0:
        hide = hide | (j > p + c["right"])
    if c["left"] >= 0:
        hide = hide | ((j < p - c["left"]) & (j >= c["sinks"]))
    return hide


def _weights(q, K, hide, c):
    """Softmax weights [B, Hk, G * N, keys] in fp32 (0 in rows that see nothing) and their log sums."""
    B, Hq, N, d = q.shape
    w = torch.matmul(q.float().reshape(B, c["Hk"], -1, d), K.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(d))
    w.view(B, c["Hk"], -1, N, K.shape[2]).masked_fill_(hide[:, None, None], -math.inf)
    m = w.amax(-1, keepdim=True).clamp(min=-3e38)
    w = torch.exp(w.sub_(m))
    l = w.sum(-1, keepdim=True)
    w = w / torch.where(l > 0, l, 1.0)
    return w, (m + torch.log(l)).view(B, Hq, N)


def _plain(s):
    c = s["case"]
    if c["op"] == "append":
        return _plain_append(s)
    B, Hq, N, d = s["q"].shape
    if c["op"] == "attend":
        K, V = _stored(s, "k_pool"), _stored(s, "v_pool")
        w, lse = _weights(s["q"], K, _hidden(_rows(s)[0], K.shape[2], s["lens"], c), c)
        return {"o": torch.matmul(w, V).view(B, Hq, N, d).to(_TORCH[c["out"]]), "lse": lse}
    K, V = s["k"].float().contiguous(), s["v"].float().contiguous()
    at = torch.arange(N, device="cuda").expand(B, N)
    w, lse = _weights(s["q"], K, _hidden(at, N, torch.full((B,), N, device="cuda"), c), c)
    o = torch.matmul(w, V)
    out = {"o": o.view(B, Hq, N, d).to(_TORCH[c["out"]]), "lse": lse}
    if c["train"]:
        g, q = (s[x].float().reshape(B, c["Hk"], -1, d) for x in ("do", "q"))
        out["dv"] = torch.matmul(w.transpose(2, 3), g).to(torch.bfloat16)
        ds = torch.matmul(g, V.transpose(2, 3).contiguous())
        ds = ds.sub_((g * o).sum(-1, keepdim=True)).mul_(w).mul_(1.0 / math.sqrt(d))
        out["dq"] = torch.matmul(ds, K).view(B, Hq, N, d).to(torch.bfloat16)
        out["dk"] = torch.matmul(ds.transpose(2, 3), q).to(torch.bfloat16)
    return out


def run(state):
    if not own:
        return _plain(state)
    import paper_2606_07713_amd as moa
    s, c = state, state["case"]
    if c["op"] == "append":
        moa.paged_append(s["q"], s["k"], s["v"], s["k_pool"], s["v_pool"], s["lens"], page_table=s["table"],
                         new_lens=s["new"], positions=s["positions"], inv_freq=s["inv_freq"], q_weight=s["wq"],
                         k_weight=s["wk"], eps=_EPS, interleaved=c["interleaved"], q_out=s["q_out"])
        return {"q": s["q_out"], "k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    how = dict(left=c["left"], right=c["right"], sinks=c["sinks"])
    if c["op"] == "attend":
        o, lse = moa.paged_attn_fwd(s["q"], s["k_pool"], s["v_pool"], s["lens"], page_table=s["table"],
                                    out_dtype=_TORCH[c["out"]], return_lse=True, **how)
        return {"o": o, "lse": lse}
    o, lse = moa.win_attn_fwd(s["q"], s["k"], s["v"], out_dtype=_TORCH[c["out"]], return_lse=True, **how)
    out = {"o": o, "lse": lse}
    if c["train"]:
        out["dq"], out["dk"], out["dv"] = moa.win_attn_bwd(s["q"], s["k"], s["v"], o, s["do"], lse, **how)
    return out


# ---- the work of one pass ---------------------------------------------------------------------


def _seen(c, at, n):
    """How many of n keys the query at place `at` sees, and the first of them behind the sinks."""
    end = n if c["right"] < 0 else min(n, at + c["right"] + 1)
    first = 0 if c["left"] < 0 else max(0, at - c["left"])
    sinks = min(c["sinks"], first, end)
    return max(0, end - first) + sinks, max(first, sinks)


def work(case):
    c = case
    B, Hq, Hk, N, d = c["B"], c["Hq"], c["Hk"], c["N"], c["d"]
    if c["op"] == "append":
        n = sum(_news(c)) * d
        flops = (Hq + Hk) * n * ((4 if c["rot"] else 0) + (4 if c["norm"] else 0))
        return {"bytes": (Hq + 2 * Hk) * n * (_BYTES[c["dtype"]] + 2), "flops": max(flops, n)}
    pairs = keys = 0
    for n in _lens(c) if c["op"] == "attend" else [N] * B:
        pairs += sum(_seen(c, n - N + i, n)[0] for i in range(N))
        seen, first = _seen(c, n - N, n)                            # the first query's window goes furthest back
        keys += n - first + min(c["sinks"], first) if c["left"] >= 0 else n
    qo = B * Hq * N * (d * (2 + _BYTES[c["out"]]) + 4)
    if c["op"] == "window" and c["train"]:
        # forward: q, k, v in, o, lse out; gradients: q, k, v, o, do, lse in, dq, dk, dv out
        return {"bytes": qo + keys * Hk * d * 4 + B * Hq * N * (d * 8 + 4) + keys * Hk * d * 8, "flops": 14 * d * Hq * pairs}
    return {"bytes": qo + keys * Hk * d * 4, "flops": 4 * d * Hq * pairs}


# ---- the definitions in 64 bits ---------------------------------------------------------------


def _head64(x, w, angle, c):
    """One sequence's heads [H, n, d] normed and turned, pairs as complex numbers."""
    x, r = x.double(), c["rot"]
    if w is not None:
        x = x / (x.pow(2).sum(-1, keepdim=True) / c["d"] + _EPS).sqrt() * w.double()
    if not r:
        return x
    pairs = x[..., :r].unflatten(-1, (-1, 2)) if c["interleaved"] else x[..., :r].unflatten(-1, (2, -1)).transpose(-1, -2)
    z = torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.ones_like(angle), angle)
    z = torch.view_as_real(z)
    z = z.flatten(-2) if c["interleaved"] else z.transpose(-1, -2).flatten(-2)
    return torch.cat([z, x[..., r:]], -1)


def _exact_append(s):
    c = s["case"]
    out = {"q": s["q_out"].double(), "k_pool": s["k_pool"].double(), "v_pool": s["v_pool"].double()}
    for b, (n, new) in enumerate(zip(_lens(c), _news(c))):
        at = torch.arange(n - new, n, device="cuda")
        pos = at if s["positions"] is None else s["positions"][b, :new]
        angle = pos.double()[:, None] * s["inv_freq"].double() if c["rot"] else None
        out["q"][b, :, :new] = _head64(s["q"][b, :, :new], s["wq"], angle, c)
        k = _head64(s["k"][b, :, :new], s["wk"], angle, c)
        page = s["table"][b].long()[torch.div(at, c["page"], rounding_mode="floor")]
        out["k_pool"][page, :, at % c["page"]] = k.transpose(0, 1)
        out["v_pool"][page, :, at % c["page"]] = s["v"][b, :, :new].double().transpose(0, 1)
    return out


def _exact_head(q, k, v, at, c, do=None):
    """One head: o, lse and, with do, the gradients (dq, dk, dv)."""
    n = k.shape[0]
    gap = torch.arange(n, device="cuda")[None] - at[:, None]        # key's place less the query's
    see = torch.ones_like(gap, dtype=torch.bool)
    if c["left"] >= 0:
        see = (gap >= -c["left"]) | (torch.arange(n, device="cuda")[None] < c["sinks"])
    if c["right"] >= 0:
        see &= gap <= c["right"]
    z = (q @ k.t().contiguous()) / math.sqrt(c["d"])
    z = torch.where(see, z, -math.inf)
    lse = torch.logsumexp(z, -1)
    p = torch.where(see, torch.exp(z - lse[:, None]), 0.0)
    o = p @ v
    if do is None:
        return o, lse
    dp = do @ v.t().contiguous()
    dz = p * (dp - (p * dp).sum(-1, keepdim=True)) / math.sqrt(c["d"])
    return o, lse, dz @ k, dz.t().contiguous() @ q, p.t().contiguous() @ do


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "append":
        return _exact_append(s)
    B, Hq, N, d = s["q"].shape
    G = Hq // c["Hk"]
    new = lambda *n: torch.zeros(n, dtype=torch.float64, device="cuda")  # noqa: E731
    out = {"o": new(B, Hq, N, d), "lse": new(B, Hq, N)}
    train = c["op"] == "window" and c["train"]
    if train:
        out.update(dq=new(B, Hq, N, d), dk=new(B, c["Hk"], N, d), dv=new(B, c["Hk"], N, d))
    lens = _lens(c) if c["op"] == "attend" else [N] * B
    for b, n in enumerate(lens):
        at = torch.arange(n - N, n, device="cuda")
        if c["op"] == "attend":
            j = torch.arange(n, device="cuda")
            page = s["table"][b].long()[torch.div(j, c["page"], rounding_mode="floor")].clamp(min=0)
            k, v = (s[x][page, :, j % c["page"]].transpose(0, 1) for x in ("k_pool", "v_pool"))
        else:
            k, v = s["k"][b], s["v"][b]
        for h in range(Hq):
            r = _exact_head(s["q"][b, h].double(), k[h // G].double(), v[h // G].double(), at, c,
                            s["do"][b, h].double() if train else None)
            out["o"][b, h], out["lse"][b, h] = r[0], r[1]
            if train:
                out["dq"][b, h] = r[2]
                out["dk"][b, h // G] += r[3]
                out["dv"][b, h // G] += r[4]
    return out
