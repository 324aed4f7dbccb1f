"""The attention with a window from its definition in fp64, its gradients, and how far the kernels may
be from them: bounds of the roundings that they make, element by element."""
import math

import torch

EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}   # half a step, relative


def visible(pos, n_keys, end, left, right, sinks):
    """[B, N, keys]: which keys the queries at pos [B, N] see of sequences with end [B] keys."""
    j = torch.arange(n_keys, device=pos.device)
    p = pos[..., None]
    see = (j < end[:, None, None]).expand(pos.shape[0], pos.shape[1], n_keys).clone()
    if right >= 0:
        see &= j <= p + right
    if left >= 0:
        see &= (j >= p - left) | (j < sinks)
    return see


def spread(x, heads):
    """Key/value heads [B, Hk, ...] for each of the query heads."""
    return x.repeat_interleave(heads // x.shape[1], 1)


class Exact:
    """q [B, Hq, N, d], k, v [B, Hk, M, d], see [B, N, M]; everything in fp64.  Keys and values that a
    row does not see have no part in it, whatever they hold."""

    def __init__(self, q, k, v, see, scale, do=None):
        q, k, v = q.double(), spread(k.double(), q.shape[1]), spread(v.double(), q.shape[1])
        see = see[:, None]
        self.see, self.scale, self.d, self.M = see, scale, q.shape[3], k.shape[2]
        s = torch.where(see, q @ k.transpose(2, 3) * scale, -math.inf)
        self.size = torch.where(see, (q.abs() @ k.abs().transpose(2, 3)) * abs(scale), 0.0).nan_to_num(0, posinf=0)   # of a score's terms
        self.lse = torch.logsumexp(s, -1)
        p = torch.where(see, torch.exp(s - torch.where(self.lse == -math.inf, 0.0, self.lse)[..., None]), 0.0)
        bad = ~v.isfinite()
        clean = torch.where(bad, 0.0, v)
        self.p, self.o = p, p @ clean
        self.bound = p @ clean.abs()
        # rows that see something that is not finite: no value is expected of these elements
        seen = see.double().expand(p.shape)
        self.odd = ((seen @ bad.double()) > 0) | p.isnan().any(-1, keepdim=True)
        if do is None:
            return
        do = do.double()
        Hk = v.shape[1]
        self.dp = dp = torch.where(see, do @ v.transpose(2, 3), 0.0)
        self.delta = (p * dp).sum(-1, keepdim=True)
        ds = p * (dp - self.delta)
        self.q, self.k, self.v, self.do, self.ds = q, k, v, do, ds
        self.dq = ds @ k * scale
        self.dk, self.dv = ds.transpose(2, 3) @ q * scale, p.transpose(2, 3) @ do

    def weight_error(self):
        """Of a weight, relative: the score's fp32 products and sum, its product with scale * log2(e), the
        exponential's own error; of the sum of the weights the same again and its additions."""
        top = self.size.amax(-1, keepdim=True)
        return 2 * ((self.d + 6) * 2.0 ** -24 * top + 2.0 ** -21) + self.M * 2.0 ** -24

    def o_bound(self, dtype, terms):
        return self.bound * (2.0 ** (-8 * terms) + self.weight_error()) + self.o.abs() * EPS[dtype] + 1e-30

    def lse_bound(self):
        return self.weight_error()[..., 0] + 2.0 ** -21 * self.lse.abs().nan_to_num(0, posinf=0) + 2.0 ** -22

    def grad_bounds(self, o_dtype, heads_k, few_keys=False):
        """Of dq, dk, dv in bf16: P and dS as one bf16 number each, D from O as it is stored, or with few
        keys as the sum of P dP over them, with a weight's error on each and one for every addition."""
        e = self.weight_error()
        r = 2.0 ** -8
        sd = (self.d + 6) * 2.0 ** -24
        terms = torch.where(self.see, self.do.abs() @ self.v.abs().transpose(2, 3), 0.0)
        o_off = (self.do.abs() * (self.o.abs() * EPS[o_dtype] + self.bound * (r + e))).sum(-1, keepdim=True)
        sum_off = sd * (self.do.abs() * self.o.abs()).sum(-1, keepdim=True)
        if few_keys:
            o_off = (self.p * (e + self.M * 2.0 ** -24) * self.dp.abs()).sum(-1, keepdim=True)
            sum_off = (self.p * sd * terms).sum(-1, keepdim=True)
        ds_off = self.p * ((2 * r + r * r + e) * (self.dp - self.delta).abs() + (1 + 2 * r) * (o_off + sum_off + sd * terms))
        s = abs(self.scale)
        dq = s * (ds_off @ self.k.abs()) + self.dq.abs() * r * (1 + r)
        dk = s * (ds_off.transpose(2, 3) @ self.q.abs()) + 1e-30
        dv = (self.p * (r + e)).transpose(2, 3) @ self.do.abs() + 1e-30
        n = self.p.shape[2] * self.p.shape[1]

        def fold(x):
            B, H = x.shape[:2]
            return x.view(B, heads_k, H // heads_k, *x.shape[2:]).sum(2)

        dk_all, dv_all = fold(self.dk), fold(self.dv)
        dk = fold(dk + (n * 2.0 ** -24) * (self.ds.abs().transpose(2, 3) @ self.q.abs() * s)) + dk_all.abs() * r
        dv = fold(dv + (n * 2.0 ** -24) * (self.p.transpose(2, 3) @ self.do.abs())) + dv_all.abs() * r
        return (self.dq, dq + 1e-30), (dk_all, dk), (dv_all, dv)


def close(got, want, bound, odd=None):
    """Asserts |got - want| <= bound wherever a value is expected (odd: where none is finite)."""
    got = got.double()
    if not got.numel():
        return
    if odd is not None:
        odd = odd.expand(got.shape)
        got, want, bound = torch.where(odd, 0.0, got), torch.where(odd, 0.0, want), torch.where(odd, 1.0, bound)
    assert got.isfinite().all(), f"{int((~got.isfinite()).sum())} values that are not finite"
    off = (got - want).abs() / bound
    i = int(off.argmax())
    assert off.max() <= 1, (f"off by {float(off.max()):.3g} of the bound at {i}: "
                            f"{float(got.flatten()[i])} for {float(want.flatten()[i])}")


def close_lse(got, want, bound, odd):
    empty = want == -math.inf
    assert torch.equal(got == -math.inf, empty) or bool(odd.any())
    hide = empty | odd
    close(torch.where(hide, 0.0, got.double()), torch.where(hide, 0.0, want), bound)
