"""Attention under score rules and rotary positions in 64 bits on the CPU, written from their definitions, and how far a
result of the library may be from them.

The bounds count roundings.  A rounding to type t is off by at most eps(t) / 2 of the value.  With u = 2^-24 (fp32):
  score   a dot product of H terms in fp32 and the few operations behind it: e_s = (H + 16) u scale sum |q k| + 16 u (|y| + |bias| + 1),
          absolute, so a probability is off by that, relative (twice e_s: against its row's maximum or lse), and by e_p = r + 16 u
          where probabilities are rounded to the inputs' type (r = 2^-8 for bf16, 0 for fp32) and 2^x is the hardware's
  sums    of n terms: (n + 16) u of the sum of their sizes
  outputs rounded once: r of the value"""
import math

import torch

U = 2.0 ** -24


def half_step(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else 0.0


def tokens(off, n, step):
    return off + torch.arange(n, dtype=torch.float64) * step


class Scored:
    """P, its sizes and errors for every query head, from CPU fp64 copies of the inputs."""

    def __init__(self, Q, K, V, q_off=0, kv_off=0, causal=False, scale=None, softcap=0.0, slopes=None, ranges=None, token_step=1):
        self.dtype = Q.dtype
        self.Q, self.K, self.V = (t.detach().cpu().double() for t in (Q, K, V))
        self.heads, self.nq, self.H = Q.shape
        self.nkv, self.group = K.shape[1], Q.shape[0] // K.shape[0]
        self.scale = 1.0 / math.sqrt(self.H) if scale is None else scale
        self.K, self.V = (t.repeat_interleave(self.group, 0) for t in (self.K, self.V))
        t, u = tokens(q_off, self.nq, token_step), tokens(kv_off, self.nkv, token_step)
        see = torch.ones(1, self.nq, self.nkv, dtype=torch.bool)
        if causal:
            see = see & (t.unsqueeze(1) >= u)
        if ranges is not None:
            r = ranges.cpu().double().reshape(-1, self.nq, 1, 2)
            see = see & (u >= r[..., 0]) & (u < r[..., 1])
        self.see = see.repeat_interleave(self.heads // see.shape[0], 0)
        hide = lambda x: torch.where(self.see, x, torch.zeros_like(x))
        z = hide(self.scale * self.Q @ self.K.transpose(1, 2))
        size = hide(self.scale * self.Q.abs() @ self.K.abs().transpose(1, 2))
        self.dy = torch.ones_like(z)
        y = z
        if softcap:
            y = softcap * torch.tanh(z / softcap)
            self.dy = 1.0 - (y / softcap) ** 2
        bias = torch.zeros_like(y)
        if slopes is not None:
            bias = slopes.cpu().double().view(-1, 1, 1) * (t.unsqueeze(1) - u).abs()
        self.s = (y - bias).masked_fill(~self.see, -math.inf)
        self.e_s = hide((self.H + 16) * U * size + 16 * U * (y.abs() + bias.abs() + 1.0))

    # ---- forward
    def partial(self):
        """(O, lse, m, l), and the bounds of O (normalised, before its own rounding), lse and m"""
        m = self.s.amax(2)
        m0 = torch.where(m == -math.inf, torch.zeros_like(m), m).unsqueeze(2)
        w = torch.exp(self.s - m0)
        l = w.sum(2)
        some = l > 0
        l1 = torch.where(some, l, torch.ones_like(l)).unsqueeze(2)
        p = w / l1
        O = p @ self.V
        lse = torch.where(some, m0.squeeze(2) + torch.log(l1.squeeze(2)), torch.full_like(l, -math.inf))
        e = 2 * self.e_s + 16 * U + (self.nkv + 16) * U
        row = (p * (e + half_step(self.dtype))) @ self.V.abs()
        row = row + (p * e).sum(2, keepdim=True) * O.abs()
        e_lse = (p * e).sum(2) + 8 * U * lse.abs().nan_to_num(0, 0, 0) + 8 * U
        e_m = self.e_s.amax(2) + 8 * U * m0.squeeze(2).abs()
        return {"O": O, "lse": lse, "m": m, "l": l, "e_O": row, "e_lse": e_lse, "e_m": e_m}

    # ---- backward, from the O and lse that the call was given
    def gradients(self, O, dO, lse):
        O, g, lse = (x.detach().cpu().double() for x in (O, dO, lse))
        r = half_step(self.dtype)
        # rows that see nothing have no part in anything
        some = self.see.any(2, keepdim=True)
        clean = lambda x: torch.where(some, x, torch.zeros_like(x))
        Q, O, g = clean(self.Q), clean(O), clean(g)
        keys = self.see.any(1).unsqueeze(2)
        K, V = (torch.where(keys, x, torch.zeros_like(x)) for x in (self.K, self.V))
        L = lse.unsqueeze(2)
        p = torch.where(self.see & (L > -math.inf), torch.exp(self.s - torch.where(L > -math.inf, L, torch.zeros_like(L))),
                        torch.zeros_like(self.s))
        dp, delta = g @ V.transpose(1, 2), (g * O).sum(2, keepdim=True)
        dz = p * (dp - delta) * self.dy
        e_p = 2 * self.e_s + 16 * U + 4 * U * torch.where(L > -math.inf, L.abs(), torch.zeros_like(L))
        e_dz = dz.abs() * (r + e_p + 16 * U) + p * (self.H + 16) * U * (g.abs() @ V.abs().transpose(1, 2) + (g * O).abs().sum(2, keepdim=True))
        # (dy = 1 - tanh^2 = 1 - (y / cap)^2: absolute errors of some steps of 1, and the score's error through tanh)
        e_dz = e_dz + (p * (dp - delta)).abs() * (16 * U + 2 * self.e_s)
        n_q, n_k = (self.nq * self.group + 16) * U, (self.nkv + 16) * U
        sc = self.scale
        by_kv = lambda x: x.view(-1, self.group, *x.shape[1:]).sum(1)
        out = {"dQ": sc * dz @ K, "dK": by_kv(sc * dz.transpose(1, 2) @ Q), "dV": by_kv(p.transpose(1, 2) @ g)}
        out["e_dQ"] = sc * (e_dz + n_k * dz.abs()) @ K.abs()
        out["e_dK"] = by_kv(sc * (e_dz + n_q * dz.abs()).transpose(1, 2) @ Q.abs())
        out["e_dV"] = by_kv((p * (r + e_p + n_q)).transpose(1, 2) @ g.abs())
        return out


def within(got, want, bound, what, rounded=0.0):
    """Every element within its bound (and its own rounding); infinities where they belong, no NaN."""
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert not torch.isnan(got).any(), "%s: NaN" % what
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine], want[~fine]), "%s: infinities" % what
    off = (got - want)[fine].abs()
    allowed = (bound * (1 + rounded) + rounded * want.abs() + 1e-30)[fine]
    if off.numel():
        worst = (off / allowed).max().item()
        assert worst <= 1.0, "%s: %.2f times its bound (off %.3g)" % (what, worst, off.max().item())
