"""Plain forms in 64 bits of what a layer does around the sparse attention (norm and rotation of query and key heads, cross attention
to encoder states), with bounds on how far a kernel that rounds as documented may be from them.  Written from the formulas; none of
the library's code."""
from __future__ import annotations

import math

import torch

U16 = 2.0 ** -8            # half a step of bf16, relative
U32 = 2.0 ** -24           # of fp32


# ---- norm and rotation
def pair_channels(n_pairs, halves):
    j = torch.arange(n_pairs)
    return (j, j + n_pairs) if halves else (2 * j, 2 * j + 1)


def _turn(x, a, b, cos, sin):
    y = x.clone()
    y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., b] * cos + x[..., a] * sin
    return y


def _pair_size(x, a, b):
    """|x_a| + |x_b| in both places of a turned pair, |x| elsewhere."""
    y = x.abs()
    y[..., a] = y[..., b] = x[..., a].abs() + x[..., b].abs()
    return y


def angles(pos, axis, freq):
    if len(axis) == 0:
        return torch.zeros((pos.shape[0], 0), dtype=torch.float64)
    return pos.double()[:, list(axis)] * torch.tensor(freq, dtype=torch.float64)


def norm_rope(x, w, pos, axis, freq, halves, eps):
    """y and its bound; x: [heads][tokens][d] float64."""
    a, b = pair_channels(len(axis), halves)
    t = angles(pos, axis, freq)
    u = x
    if w is not None:
        u = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
    y = _turn(u, a, b, t.cos(), t.sin())
    # one rounding to bf16; in fp32: the norm (a sum of d squares whose relative error is d u / 2 at most in the root), two products, the
    # rotation's two products and sum, cos and sin to a few units
    size = _pair_size(u, a, b)
    return y, U16 * y.abs() * (1 + U16) + (x.shape[-1] / 2 + 16) * U32 * size


def norm_rope_bwd(x, w, pos, axis, freq, halves, eps, dy, out_bits):
    """(dx, bound), (dw, bound); out_bits: half a step of dx's type."""
    a, b = pair_channels(len(axis), halves)
    t = angles(pos, axis, freq)
    g = _turn(dy, a, b, t.cos(), -t.sin())
    gs = _pair_size(dy, a, b)
    d, k = x.shape[-1], 8 * U32
    if w is None:
        return (g, out_bits * g.abs() * (1 + out_bits) + k * gs), (None, None)
    w = w.double()
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    xh = x * r
    dw = (g * xh).sum((0, 1))
    n = x.shape[0] * x.shape[1]
    dw_tol = (d / 2 + n + 16) * U32 * (gs * xh.abs()).sum((0, 1))                     # fp32 sums in any order
    m = (w * g * xh).mean(-1, keepdim=True)
    dx = r * (w * g - xh * m)
    size = r * (w.abs() * gs + xh.abs() * (w.abs() * gs * xh.abs()).mean(-1, keepdim=True))
    return (dx, out_bits * dx.abs() * (1 + out_bits) + (2 * d + 32) * U32 * size), (dw, dw_tol)


# ---- cross attention
class CrossRef:
    """Outputs, gradients and bounds of all segments; q, dO: [H][Lq][d], k, v: [Hkv][Lk][d], float64 on any device."""

    def __init__(self, q, k, v, q_len, k_len, k_off, scale, d_o=None):
        H, d = q.shape[0], q.shape[2]
        g = H // k.shape[0]
        zeros = torch.zeros_like
        lq = q.shape[:2]
        self.o, self.o_tol = zeros(q), zeros(q)
        self.lse = torch.full(lq, -math.inf, dtype=torch.float64, device=q.device)
        self.lse_tol = torch.zeros(lq, dtype=torch.float64, device=q.device)
        if d_o is not None:
            self.dq, self.dq_tol = zeros(q), zeros(q)
            self.dk, self.dk_tol, self.dv, self.dv_tol = zeros(k), zeros(k), zeros(k), zeros(k)
        r0 = 0
        for nq, nk, k0 in zip(q_len, k_len, k_off):
            rows, cols = slice(r0, r0 + nq), slice(k0, k0 + nk)
            r0 += nq
            if nq == 0 or nk == 0:
                continue
            for h in range(H):
                hk = h // g
                Q, K, V = q[h, rows], k[hk, cols], v[hk, cols]
                s = scale * Q @ K.T
                # the score's error: d products summed in fp32, the scaling, and the exponential's argument
                e_s = (scale * (d + 8) * U32 * (Q.abs() @ K.abs().T)).max().item()
                lse = torch.logsumexp(s, 1)
                p = torch.exp(s - lse[:, None])
                o = p @ V
                # P: rounded to bf16 once; exp2 to a few units, the sum of nk terms
                e_p = 2 * e_s + (nk + 64) * U32
                o_tol = (U16 * (1 + U16) + e_p) * (p @ V.abs()) * 1.01 + U16 * o.abs()
                self.o[h, rows], self.o_tol[h, rows] = o, o_tol
                l_tol = e_s + (nk + 64) * U32 + 8 * U32 * lse.abs()
                self.lse[h, rows], self.lse_tol[h, rows] = lse, l_tol
                if d_o is None:
                    continue
                G = d_o[h, rows]
                e_q = e_s + l_tol.max().item() + 64 * U32                # P of the backward: from the scores and lse again
                dp, delta = G @ V.T, (G * o).sum(1, keepdim=True)
                ds = p * (dp - delta)
                # delta is formed of the rounded O; dP and delta are sums of d products in fp32
                e_delta = (G.abs() * (o_tol + (d + 8) * U32 * o.abs())).sum(1, keepdim=True)
                ds_tol = (U16 * (1 + U16) + e_q) * ds.abs() + p * (1 + U16) * (e_delta + (d + 8) * U32 * (G.abs() @ V.abs().T))
                n_q = (nq + 8) * U32                                     # sums over the queries in fp32
                self.dq[h, rows] = dq = scale * ds @ K
                self.dq_tol[h, rows] = scale * (ds_tol + (nk + 8) * U32 * ds.abs()) @ K.abs() * 1.01 + U16 * dq.abs()
                self.dk[hk, cols] += scale * ds.T @ Q
                self.dk_tol[hk, cols] += scale * (ds_tol + g * n_q * ds.abs()).T @ Q.abs() * 1.01
                self.dv[hk, cols] += p.T @ G
                self.dv_tol[hk, cols] += ((U16 * (1 + U16) + e_q + g * n_q) * p).T @ G.abs() * 1.01
        if d_o is not None:
            self.dk_tol += U16 * self.dk.abs()
            self.dv_tol += U16 * self.dv.abs()


def check(name, got, want, tol, floor=1e-30):
    """got within tol of want, elementwise; infinities equal."""
    got = got.double().to(want.device)
    same = torch.isinf(want) & (got == want)
    off = torch.where(same, 0.0, (got - want).abs())
    bad = ~(off <= tol + floor)
    assert not bool(bad.any()), (f"{name}: {int(bad.sum())} of {bad.numel()} off, first at {tuple(bad.nonzero()[0].tolist())}: "
                                 f"{got[bad][0].item()} for {want[bad][0].item()}, allowed {tol[bad][0].item() if tol.dim() else tol}")
