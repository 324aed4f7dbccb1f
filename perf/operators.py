"""Measured calls of the operators around a four-bit key/value cache and of the head norms with
position rotation, over the range their users call them with.

``rope``   RMS norm of every query and key head, then the rotation by position (a step's tokens,
           a prompt, positions with several axes); with ``train`` its gradients too.
``write``  new keys and values quantised into the pages of a four-bit cache and read back, as a
           prompt does whose attention shall see what later steps will see.
``read``   a stored context read back from its pages.
``attn``   attention of new queries over the four-bit cache: single tokens, a few drafted tokens,
           a chunk of a prompt.

``run()`` makes one such call, in plain torch or, where ``own`` is set, through the public entry
points; ``exact()`` is the same from the definitions in fp64.

A page of the cache holds P tokens (a multiple of 64) of one head: key codes, key scales, value
codes, value scales.  A code is a four-bit float (sign, two exponent bits, one mantissa bit: 0,
0.5, 1, 1.5, 2, 3, 4, 6), 32 successive elements of a row share a power of two 2^(byte - 127).
  key codes     [P][d/2]                        byte i: elements 2i (low half) and 2i + 1
  key scales    [P/64][d/32][16][4]             of token 64 a + 16 t + r at [a][block][r][t]
  value codes   [P/4][d/4][4][2]                of token 4 q + j, elements 4 c .. 4 c + 3 at [q][c][j]
  value scales  [P/64][d/32][4][4][4]           of token 64 a + 16 t + 4 g + j at [a][block][g][t][j]
"""
import math

import torch

own = False

BF16, F32 = "bf16", "f32"
_TORCH = {BF16: torch.bfloat16, F32: torch.float32}
_BYTES = {BF16: 2, F32: 4}
_EPS = 1e-6


def _rope(B, Hq, Hk, N, d, rot=None, dtype=BF16, axes=1, interleaved=False, train=False, packed=False,
          norm=True, far=0, name=None):
    c = {"op": "rope", "B": B, "Hq": Hq, "Hk": Hk, "N": N, "d": d, "rot": d if rot is None else rot,
         "dtype": dtype, "axes": axes, "interleaved": interleaved, "train": train, "packed": packed,
         "norm": norm, "far": far}
    return dict(c, name=name) if name else c


def _cache(op, B, Hk, N, lo, hi, page, d, name=None):
    """Sequences of lo..hi tokens, the last N of them written (or read) by the call."""
    c = {"op": op, "B": B, "Hk": Hk, "N": N, "lo": lo, "hi": hi, "page": page, "d": d}
    return dict(c, name=name) if name else c


def _attn(B, Hq, Hk, N, lo, hi, page, d, causal=True, name=None):
    """N queries of each sequence over the sequence's lo..hi stored tokens, theirs the last."""
    c = {"op": "attn", "B": B, "Hq": Hq, "Hk": Hk, "N": N, "lo": lo, "hi": hi, "page": page, "d": d,
         "causal": causal}
    return dict(c, name=name) if name else c


def listed():
    return [
        # One token of one conversation, far into it: launch and latency.
        _rope(1, 32, 8, 1, 128, far=100000, name="rope_step"),
        # A decoder layer's prompt, q and k slices of a packed projection output.
        _rope(2, 16, 16, 4096, 128, packed=True, name="rope_prompt_4k"),
        # Image and text tokens with (time, height, width) positions, half of each head rotated,
        # fp32, a token count that divides by nothing.
        _rope(8, 12, 12, 777, 64, rot=32, dtype=F32, axes=3, name="rope_axes_777"),
        # Training step of a decoder layer's norms and rotation.
        _rope(2, 16, 16, 4096, 128, train=True, name="rope_train_4k"),
        # Training step in fp32 on a ragged length, neighbouring elements as pairs.
        _rope(4, 8, 8, 1000, 64, dtype=F32, axes=2, interleaved=True, train=True, name="rope_train_1000"),
        # Decode step of a serving batch: one new token of each of 64 sequences.
        _cache("write", 64, 8, 1, 8000, 8192, 64, 128, name="write_step_b64"),
        # A prompt of 4K tokens.
        _cache("write", 2, 16, 4096, 4096, 4096, 256, 128, name="write_prompt_4k"),
        # A stored context of up to 16K tokens, read back whole.
        _cache("read", 4, 8, 16384, 9000, 16384, 128, 128, name="read_16k"),
        # Decode step of a single conversation.
        _attn(1, 32, 8, 1, 4097, 4097, 64, 128, name="decode_b1_4k"),
        # Decode step of a large serving batch.
        _attn(64, 32, 8, 1, 8192, 8192, 64, 128, name="decode_b64_8k"),
        # Four drafted tokens of each of 16 sequences of very different lengths.
        _attn(16, 12, 4, 4, 100, 16384, 128, 64, name="draft_ragged"),
        # Chunked prefill: a few hundred new tokens against a long cache, ragged on both sides.
        _attn(1, 32, 8, 200, 20011, 20011, 256, 128, name="chunk_200_of_20k"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "rope", "train", "write", "read", "attn", "attn", "chunk"])
    d, page = rng.choice([64, 128]), 64 * rng.choice([1, 1, 2, 3, 4])
    Hk = rng.choice([1, 2, 4, 5, 8, 16])
    if op in ("rope", "train"):
        B, N = rng.randint(1, 8), _log_int(rng, 1 if op == "rope" else 64, 8192)
        Hq, dtype = Hk * rng.choice([1, 2, 4]), rng.choice([BF16, BF16, F32])
        while B * N * (Hq + Hk) > 2 * 8192 * 32:
            N = (N + 1) // 2
        return _rope(B, Hq, Hk, N, d, rot=rng.choice([16, 32, d // 2, d, d]), dtype=dtype,
                     axes=rng.choice([1, 1, 2, 3]), interleaved=rng.random() < 0.3,
                     train=op == "train", packed=op == "rope" and rng.random() < 0.5,
                     norm=rng.random() < 0.8, far=_log_int(rng, 1, 1000000))
    if op in ("write", "read"):
        B, N = _log_int(rng, 1, 64), _log_int(rng, 1, 16384)
        while B * N * Hk > 4 * 8 * 16384:
            N = (N + 1) // 2
        lo = N if op == "write" else max(1, N * 2 // 3)
        return _cache(op, B, Hk, N, lo, max(lo, N) + (_log_int(rng, 1, 2000) if op == "write" else 0), page, d)
    Hq = Hk * rng.choice([1, 2, 4, 8])
    if op == "chunk":
        B, N, hi = rng.randint(1, 2), _log_int(rng, 9, 1024), _log_int(rng, 1024, 32768)
        while B * Hq * N * hi > 40 * 200 * 20011:
            N = (N + 1) // 2
        return _attn(B, Hq, Hk, N, max(N, hi * 2 // 3), max(N, hi), page, d, causal=rng.random() < 0.8)
    B, N, hi = _log_int(rng, 1, 64), rng.choice([1, 1, 1, 2, 4, 7]), _log_int(rng, 40, 32768)
    while B * Hk * hi > 64 * 8 * 8192 or B * Hq * N * hi > 64 * 32 * 8192:
        hi = (hi + 1) // 2
    return _attn(B, Hq, Hk, N, max(N, rng.choice([hi, hi // 20])), max(N, hi), page, d)


def _lens(c):
    """The lengths of a case's sequences: lo to hi, in no order."""
    B, lo, hi = c["B"], c["lo"], c["hi"]
    return [hi if i == 0 else lo + (hi - lo) * (i * 37 % B) // B for i in range(B)]


def _sections(c):
    """Rotated pairs of each axis: the first axis has what the others leave."""
    pairs, axes = c["rot"] // 2, c["axes"]
    return [pairs - (axes - 1) * (pairs // axes)] + [pairs // axes] * (axes - 1)


# ---- the four-bit format, in 32 bits ----------------------------------------------------------


def _quantise(x):
    """Codes (0..15, uint8) and scale bytes of x [..., d], blocks of 32: the smallest power of two
    under which no element of the block lies above 7, then the nearest code, ties to even."""
    b = x.float().unflatten(-1, (-1, 32))
    m, k = torch.frexp(b.abs().amax(-1))
    byte = (k - 3 + (m > 0.875).int() + 127).clamp(2, 252).int()
    y = b * ((254 - byte) << 23).view(torch.float32)[..., None]
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5)
            + (a > 5)) + 8 * (y < 0).to(torch.uint8)
    return code.flatten(-2), byte.to(torch.uint8)


def _values(code, byte):
    """fp32 values of codes [..., d] and scale bytes [..., d/32]."""
    t = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=code.device)
    v = torch.cat([t, -t])[code.int()].unflatten(-1, (-1, 32))
    return (v * (byte.int() << 23).view(torch.float32)[..., None]).flatten(-2)


def _to_pages(kc, ks, vc, vs):
    """Codes [n, P, d] and scale bytes [n, P, d/32] of keys and values -> pages [n, bytes]."""
    n, P, d = kc.shape
    kb, vb = (c[..., 0::2] | (c[..., 1::2] << 4) for c in (kc, vc))
    parts = (kb, ks.view(n, P // 64, 4, 16, d // 32).permute(0, 1, 4, 3, 2),
             vb.view(n, P // 4, 4, d // 4, 2).transpose(2, 3),
             vs.view(n, P // 64, 4, 4, 4, d // 32).permute(0, 1, 5, 3, 2, 4))
    return torch.cat([p.reshape(n, -1) for p in parts], 1)


def _from_pages(pages, P, d):
    """The reverse, on pages [..., bytes]."""
    lead = pages.shape[:-1]
    kb, ks, vb, vs = pages.split([P * d // 2, P * d // 32, P * d // 2, P * d // 32], -1)
    ks = ks.reshape(-1, P // 64, d // 32, 16, 4).permute(0, 1, 4, 3, 2).reshape(*lead, P, d // 32)
    vb = vb.reshape(-1, P // 4, d // 4, 4, 2).transpose(2, 3).reshape(*lead, P, d // 2)
    vs = vs.reshape(-1, P // 64, d // 32, 4, 4, 4).permute(0, 1, 4, 3, 5, 2).reshape(*lead, P, d // 32)
    kb = kb.reshape(*lead, P, d // 2)
    kc, vc = (torch.stack([b & 15, b >> 4], -1).flatten(-2) for b in (kb, vb))
    return kc, ks, vc, vs


def _stored(s):
    """fp32 keys and values [B, Hk, tokens, d] of every sequence's pages."""
    c = s["case"]
    pages = s["cache"][s["table"].long()].transpose(1, 2)          # [B, Hk, pages, bytes]
    kc, ks, vc, vs = _from_pages(pages, c["page"], c["d"])
    return _values(kc, ks).flatten(2, 3), _values(vc, vs).flatten(2, 3)


# ---- inputs -----------------------------------------------------------------------------------


def _normal(g, shape, dtype, std=1.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["op"] == "rope":
        B, N, d, dt = c["B"], c["N"], c["d"], _TORCH[c["dtype"]]
        shape = [(B, N, h, d) for h in (c["Hq"], c["Hk"])]
        if c["packed"]:
            # The projections' output [B, N, Hq + 2 Hk, d]: queries, keys, values.
            x = _normal(g, (B, N, c["Hq"] + 2 * c["Hk"], d), dt, 2.0)
            q, k = x[:, :, :c["Hq"]], x[:, :, c["Hq"]:c["Hq"] + c["Hk"]]
            s["q"], s["k"] = q.transpose(1, 2), k.transpose(1, 2)
        else:
            s["q"], s["k"] = (_normal(g, (b, h, n, e), dt, 2.0) for b, n, h, e in shape)
        if c["train"]:
            s["dq"], s["dk"] = (_normal(g, (b, h, n, e), dt) for b, n, h, e in shape)
        s["wq"], s["wk"] = ((1 + _normal(g, (d,), torch.float32, 0.3)).to(dt) if c["norm"] else None
                            for _ in range(2))
        s["inv_freq"] = (10000.0 ** (-torch.arange(c["rot"] // 2, device="cuda", dtype=torch.float64)
                                     * 2 / c["rot"])).float()
        pos = c["far"] + torch.arange(N, device="cuda").expand(c["axes"], B, N).clone()
        if c["axes"] > 1:                   # frames of 16 by 16 patches
            pos[1:] = torch.stack([pos[0] // 16 % 16, pos[0] % 16])[: c["axes"] - 1]
            pos[0] //= 256
        s["positions"] = pos if c["axes"] > 1 else pos[0]
        return s

    # The pool of pages, what it holds, and every sequence's pages in no order.
    B, Hk, P, d, lens = c["B"], c["Hk"], c["page"], c["d"], _lens(c)
    each = -(-max(lens) // P)
    pages = [-(-n // P) for n in lens]
    pool = sum(pages)
    order = torch.randperm(pool, generator=g, device="cuda").int()
    table = torch.zeros((B, each), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    cache = torch.empty((pool * Hk, P * (d + d // 16)), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // (P * d))
    for i in range(0, pool * Hk, step):
        n = min(step, pool * Hk - i)
        cache[i:i + n] = _to_pages(*_quantise(_normal(g, (n, P, d), torch.bfloat16)),
                                   *_quantise(_normal(g, (n, P, d), torch.bfloat16)))
    s["cache"] = cache.view(pool, Hk, -1)
    s["table"] = table
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if c["op"] == "write":
        s["k"], s["v"] = (_normal(g, (B, c["N"], Hk, d), torch.bfloat16).transpose(1, 2) for _ in range(2))
    elif c["op"] == "read":
        # Rows behind a sequence stay as they are in the caller's buffers.
        s["out"] = [torch.zeros((B, Hk, c["N"], d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    else:
        s["q"] = _normal(g, (B, c["N"], c["Hq"], d), torch.bfloat16, 1.5).transpose(1, 2)
    return s


# ---- one pass ---------------------------------------------------------------------------------


def _angles(s):
    """cos and sin [B, 1, N, rot/2] of every rotated pair, from angles in 64 bits."""
    c = s["case"]
    axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"),
                                   torch.tensor(_sections(c), device="cuda"), output_size=c["rot"] // 2)
    pos = s["positions"].view(c["axes"], c["B"], c["N"])[axis].permute(1, 2, 0)
    a = (pos.double() * s["inv_freq"].double())[:, None]
    return a.cos().float(), a.sin().float()


def _turn(x, cos, sin, c, back=False):
    """x [B, H, N, d] with its first rot elements rotated in pairs (back: by the opposite angles)."""
    r = c["rot"]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
    if back:
        sin = -sin
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _norm_rope(x, w, cos, sin, c):
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + _EPS) * w.float()
    return _turn(y, cos, sin, c).to(x.dtype)


def _norm_rope_bwd(x, dy, w, cos, sin, c):
    g = _turn(dy.float(), cos, sin, c, back=True)
    if w is None:
        return g.to(x.dtype), None
    x32 = x.float()
    r = torch.rsqrt(x32.square().mean(-1, keepdim=True) + _EPS)
    n, gw = x32 * r, g * w.float()
    dx = r * (gw - n * (gw * n).mean(-1, keepdim=True))
    return dx.to(x.dtype), (g * n).sum((0, 1, 2))


def _put(s):
    """The new tokens' codes and scales into the cache's pages; the values that they stand for."""
    c = s["case"]
    B, Hk, N, P, d = c["B"], c["Hk"], c["N"], c["page"], c["d"]
    (kc, ks), (vc, vs) = _quantise(s["k"]), _quantise(s["v"])
    pos = s["lens"].long()[:, None] - N + torch.arange(N, device="cuda")               # [B, N]
    page = torch.gather(s["table"].long(), 1, pos // P)[:, None, :, None]
    head = torch.arange(Hk, device="cuda")[None, :, None, None]
    r = (pos % P)[:, None, :, None]
    e, f = torch.arange(d // 2, device="cuda"), torch.arange(d // 32, device="cuda")
    cache, vo = s["cache"], P * d // 2 + P * d // 32
    cache[page, head, r * (d // 2) + e] = kc[..., 0::2] | (kc[..., 1::2] << 4)
    cache[page, head, P * d // 2 + r // 64 * (2 * d) + f * 64 + r % 16 * 4 + r // 16 % 4] = ks
    cache[page, head, vo + ((r // 4 * (d // 4) + e // 2) * 4 + r % 4) * 2 + e % 2] = vc[..., 0::2] | (vc[..., 1::2] << 4)
    cache[page, head, vo + P * d // 2 + r // 64 * (2 * d) + f * 64 + r // 4 % 4 * 16 + r // 16 % 4 * 4 + r % 4] = vs
    return _values(kc, ks).to(torch.bfloat16), _values(vc, vs).to(torch.bfloat16)


def _plain(s):
    c = s["case"]
    if c["op"] == "rope":
        cos, sin = _angles(s)
        out = {k + "o": _norm_rope(s[k], s["w" + k], cos, sin, c) for k in ("q", "k")}
        if c["train"]:
            out["dq"], out["dwq"] = _norm_rope_bwd(s["q"], s["dq"], s["wq"], cos, sin, c)
            out["dk"], out["dwk"] = _norm_rope_bwd(s["k"], s["dk"], s["wk"], cos, sin, c)
        return out
    if c["op"] == "write":
        return _put(s)
    K, V = _stored(s)
    if c["op"] == "read":
        seen = (torch.arange(c["N"], device="cuda") < s["lens"][:, None])[:, None, :, None]
        for out, x in zip(s["out"], (K, V)):
            out.copy_(torch.where(seen, x[:, :, :c["N"]].to(torch.bfloat16), out))
        return s["out"]
    B, Hq, N, d = s["q"].shape
    q = s["q"].float().reshape(B, c["Hk"], -1, d)
    w = torch.matmul(q, K.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(d))
    at = s["lens"][:, None] - N + torch.arange(N, device="cuda") if c["causal"] else s["lens"][:, None].expand(B, N) - 1
    hide = torch.arange(K.shape[2], device="cuda") > at[..., None]
    w = w.view(B, c["Hk"], -1, N, K.shape[2]).masked_fill(hide[:, None, None], -math.inf).view_as(w)
    m = w.amax(-1, keepdim=True)
    w = torch.exp(w - m)
    l = w.sum(-1, keepdim=True)
    o = torch.matmul(w, V) / l
    return o.view(B, Hq, N, d).to(torch.bfloat16), (m + torch.log(l)).view(B, Hq, N)


def run(state):
    if not own:
        return _plain(state)
    import paper_2606_07713_amd as moa
    s, c = state, state["case"]
    if c["op"] == "rope":
        how = dict(positions=s["positions"], inv_freq=s["inv_freq"], q_weight=s["wq"], k_weight=s["wk"],
                   eps=_EPS, interleaved=c["interleaved"], sections=_sections(c) if c["axes"] > 1 else None)
        q, k = moa.qk_norm_rope(s["q"], s["k"], **how)
        out = {"qo": q, "ko": k}
        if c["train"]:
            out["dq"], out["dk"], out["dwq"], out["dwk"] = moa.qk_norm_rope_bwd(s["q"], s["k"], s["dq"], s["dk"], **how)
        return out
    if c["op"] == "write":
        moa.kv4_write(s["k"], s["v"], s["cache"], s["lens"], page_table=s["table"])
        return moa.kv4_read(s["cache"], c["N"], c["d"], s["lens"], page_table=s["table"])
    if c["op"] == "read":
        # Token i of a sequence is row i: every sequence's new tokens are all that it has.
        return moa.kv4_read(s["cache"], c["N"], c["d"], s["lens"], page_table=s["table"], new_lens=s["lens"],
                            k_out=s["out"][0], v_out=s["out"][1])
    return moa.kv4_attn_fwd(s["q"], s["cache"], s["lens"], page_table=s["table"], causal=c["causal"],
                            return_lse=True)


# ---- the work of one pass ---------------------------------------------------------------------


def work(case):
    c = case
    d = c["d"]
    if c["op"] == "rope":
        n, es = c["B"] * c["N"] * (c["Hq"] + c["Hk"]) * d, _BYTES[c["dtype"]]
        # forward: read, write; backward: read the gradient (and the input again), write
        more = (3 if c["norm"] else 2) if c["train"] else 0
        return {"bytes": (2 + more) * n * es + 8 * c["axes"] * c["B"] * c["N"], "flops": (8 + 8 * more) * n}
    lens, Hk = _lens(c), c["Hk"]
    if c["op"] == "write":
        n = c["B"] * c["N"] * Hk * 2 * d
        return {"bytes": n * 2 + n * 17 // 32 + n * 2, "flops": 12 * n}
    if c["op"] == "read":
        n = sum(min(x, c["N"]) for x in lens) * Hk * 2 * d
        return {"bytes": n * 17 // 32 + n * 2, "flops": 2 * n}
    B, Hq, N = c["B"], c["Hq"], c["N"]
    pairs = sum(N * x - (N * (N - 1) // 2 if c["causal"] else 0) for x in lens)
    return {"bytes": sum(lens) * Hk * (d + d // 16) + B * Hq * N * (4 * d + 4), "flops": 4 * d * Hq * pairs}


# ---- the definitions in 64 bits ---------------------------------------------------------------


def _round4(x):
    """Rows of 32 in fp64 -> the values that the format holds for them."""
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(top / 7)).clamp(-125, 125))
    a = x.abs() / scale
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=1))) - 1)
    return torch.sign(x) * (torch.round(a / step) * step).clamp(max=6) * scale


def _rows64(s, b, n):
    """The first n stored keys and values [Hk, n, d] of sequence b in fp64, each element by its place."""
    c = s["case"]
    P, d = c["page"], c["d"]
    j = torch.arange(n, device="cuda")
    pages = s["cache"][s["table"][b].long()]                        # [pages, Hk, bytes]
    page, r = (j // P)[:, None], (j % P)[:, None]
    e = torch.arange(d, device="cuda")[None]
    level = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], dtype=torch.float64, device="cuda") / 2
    half = P * d // 2 + P * d // 32
    kat = r * (d // 2) + e // 2
    vat = half + (r // 4) * 2 * d + (e // 4) * 8 + (r % 4) * 2 + e % 4 // 2
    ksat = P * d // 2 + (r // 64) * 2 * d + (e // 32) * 64 + (r % 16) * 4 + r % 64 // 16
    vsat = half + P * d // 2 + (r // 64) * 2 * d + (e // 32) * 64 + (r % 16 // 4) * 16 + (r % 64 // 16) * 4 + r % 4
    out = []
    for code_at, scale_at in ((kat, ksat), (vat, vsat)):
        byte = pages[page, :, code_at].permute(2, 0, 1)
        code = torch.where(e % 2 == 1, byte // 16, byte % 16).long()
        power = torch.exp2(pages[page, :, scale_at].permute(2, 0, 1).double() - 127)
        out.append(torch.where(code >= 8, -1.0, 1.0) * level[code % 8] * power)
    return out


def _head64(x, w, ang, c, dy=None):
    """The norm and rotation of x [B, H, N, d] through complex numbers, and the gradients of dy."""
    r = c["rot"]
    x = x.double()
    rms = (x.pow(2).sum(-1, keepdim=True) / c["d"] + _EPS).sqrt()
    unit = x / rms if w is not None else x
    wd = w.double() if w is not None else 1.0

    def turn(v, a):
        pairs = v[..., :r].unflatten(-1, (-1, 2)) if c["interleaved"] else v[..., :r].unflatten(-1, (2, -1)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.ones_like(a), a))
        z = z.flatten(-2) if c["interleaved"] else z.transpose(-1, -2).flatten(-2)
        return torch.cat([z, v[..., r:]], -1)

    y = turn(unit * wd, ang)
    if dy is None:
        return y
    g = turn(dy.double(), -ang)
    if w is None:
        return y, g, None
    t = g * wd
    return y, t / rms - x * (t * x).sum(-1, keepdim=True) / (c["d"] * rms ** 3), (g * unit).sum((0, 1, 2))


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "rope":
        ax = [a for a, n in enumerate(_sections(c)) for _ in range(n)]
        pos = s["positions"].view(c["axes"], c["B"], c["N"]).double()
        ang = torch.stack([pos[a] * s["inv_freq"][i].double() for i, a in enumerate(ax)], -1)[:, None]
        out = {}
        for k in ("q", "k"):
            if c["train"]:
                out[k + "o"], out["d" + k], out["dw" + k] = _head64(s[k], s["w" + k], ang, c, s["d" + k])
            else:
                out[k + "o"] = _head64(s[k], s["w" + k], ang, c)
        return out
    if c["op"] == "write":
        return tuple(_round4(x.double().unflatten(-1, (-1, 32))).flatten(-2) for x in (s["k"], s["v"]))
    lens = _lens(c)
    if c["op"] == "read":
        out = [torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in s["out"]]
        for b, n in enumerate(lens):
            n = min(n, c["N"])
            for o, x in zip(out, _rows64(s, b, n)):
                o[b, :, :n] = x
        return out
    N, G = c["N"], c["Hq"] // c["Hk"]
    os, ls = [], []
    for b, n in enumerate(lens):
        k, v = _rows64(s, b, n)
        q = s["q"][b].double()
        at = torch.arange(N, device="cuda") + (n - N if c["causal"] else n)
        hide = torch.arange(n, device="cuda")[None] > at[:, None]
        o, l = [], []
        for h in range(c["Hq"]):
            w = (q[h] @ k[h // G].t().contiguous()) / math.sqrt(c["d"])
            w = w.masked_fill(hide, -math.inf)
            l.append(torch.logsumexp(w, -1))
            o.append(torch.softmax(w, -1) @ v[h // G])
        os.append(torch.stack(o))
        ls.append(torch.stack(l))
    return torch.stack(os), torch.stack(ls)
