"""The operators as a layer of a video transformer runs them: a fused projection -> norm and (time, height, width) rotation ->
pool -> route -> sparse attention -> cross attention of every shot to its own prompt, and back to the projection's gradient; against
64-bit autograd through the same chain with the selection held constant."""
import math

import numpy as np
import pytest
import torch

import layer_ref as R
from paper_2508_21058_b200 import MocCross, MocPlan, MocRope
from paper_2508_21058_b200 import workloads as W

pytestmark = pytest.mark.gpu


def _shots(lay):
    shot = np.repeat(lay.chunk_shot, np.diff(lay.chunk_off))
    return [0] + [int(np.nonzero(shot == s)[0][-1]) + 1 for s in np.unique(shot)]


def _mask(wl, sel, L):
    """[head][query][key] of the selection: anchors by the rule, and the picks."""
    lay = wl.layout
    chunk = torch.from_numpy(lay.token_chunk().astype(np.int64)).cuda()
    shot, text = (torch.from_numpy(np.asarray(x).astype(np.int64)).cuda() for x in (lay.chunk_shot, lay.chunk_mod))
    C = lay.n_chunks
    i, j = torch.arange(C, device="cuda")[:, None], torch.arange(C, device="cuda")[None, :]
    anchor = (text[None, :] == 1) | ((shot[:, None] == shot[None, :]) & (j >= i - wl.win_back) & (j <= i + wl.win_fwd))
    mask = anchor[chunk][:, chunk][None].repeat(wl.n_heads, 1, 1)
    for s in range(sel.shape[2]):
        pick = sel[:, :, s].long()
        mask |= (pick[:, :, None] == chunk[None, None, :]) & (pick >= 0)[:, :, None]
    return mask


@pytest.mark.parametrize("name,halves", [("mini2", False), ("cfg0", True)])
def test_layer_forward_and_backward(name, halves):
    wl = W.workload(name)
    H, L, d = wl.n_heads, wl.n_tokens, wl.head_dim
    gen = torch.Generator("cuda").manual_seed(11)
    bf = torch.bfloat16
    qkv = torch.randn(L, 3 * H, d, generator=gen, device="cuda").to(bf)
    w = [1 + 0.1 * torch.randn(d, generator=gen, device="cuda") for _ in range(2)]
    q_off = _shots(wl.layout)
    k_len = [33 + 20 * s for s in range(len(q_off) - 1)]
    k_off = [64 * s for s in range(len(q_off))] if max(k_len) <= 64 else [128 * s for s in range(len(q_off))]
    states = torch.randn(k_off[-1], 2, H, d, generator=gen, device="cuda").to(bf)
    d_out = torch.randn(H, L, d, generator=gen, device="cuda").to(bf)
    pos = torch.stack([torch.arange(L, device="cuda") // 200, torch.arange(L, device="cuda") % 200 // 20, torch.arange(L, device="cuda") % 20], 1).to(torch.int32)
    axes = (16, 24, 24) if d == 64 else (44, 42, 42)
    if halves:
        axes = (16, 16, 16)
    rope, plan, cross = MocRope.from_axes(d, axes, halves=halves), MocPlan.from_workload(wl), MocCross(H, H, d, q_off, k_off, k_len=k_len)
    ws, ws_r, ws_c = plan.new_workspace(with_bwd=True), rope.new_workspace(), cross.new_workspace(with_bwd=True)

    heads = qkv.transpose(0, 1)
    q, k, o, out = (torch.empty(H, L, d, dtype=bf, device="cuda") for _ in range(4))
    v = heads[2 * H:].contiguous()
    rope.moc_norm_rope(pos, heads[:H], w[0], q, heads[H:2 * H], w[1], k)
    desc, sel, o, lse, _ = plan.forward(q, k, v, ws)
    ek, ev = states[:, 0].transpose(0, 1), states[:, 1].transpose(0, 1)
    lse_c = torch.empty(H, L, device="cuda")
    cross.moc_cross_attend(o, ek, ev, out, lse_c, ws_c)
    d_o, dq, dk, dv = (torch.empty(H, L, d, dtype=bf, device="cuda") for _ in range(4))
    d_states = torch.empty_like(states)
    cross.moc_cross_attend_bwd(o, ek, ev, out, lse_c, d_out, d_o, d_states[:, 0].transpose(0, 1), d_states[:, 1].transpose(0, 1), ws_c)
    plan.moc_attend_bwd(q, k, v, o, lse, d_o, sel, dq, dk, dv, ws)
    d_qkv = torch.empty_like(qkv)
    dh = d_qkv.transpose(0, 1)
    dw = [torch.empty(d, device="cuda") for _ in range(2)]
    rope.moc_norm_rope_bwd(pos, heads[:H], w[0], dq, dh[:H], dw[0], ws_r, heads[H:2 * H], w[1], dk, dh[H:2 * H], dw[1])
    dh[2 * H:] = dv
    torch.cuda.synchronize()
    assert plan.moc_get_status(ws)[0] == 0 and cross.moc_cross_get_status(ws_c)[0] == 0

    # the same in 64 bits
    x, e = qkv.double().requires_grad_(), states.double().requires_grad_()
    w64 = [t.double().requires_grad_() for t in w]
    axis = [a for a, n in enumerate(axes) for _ in range(n // 2)]
    freq = torch.tensor([10000.0 ** (-2.0 * m / n) for n in axes for m in range(n // 2)], dtype=torch.float64, device="cuda")
    a, b = (t.cuda() for t in R.pair_channels(len(axis), halves))
    unit = torch.polar(torch.ones(L, len(axis), dtype=torch.float64, device="cuda"), pos.double()[:, axis] * freq)

    def turned(t, wt):
        t = t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6) * wt
        z = torch.complex(t[..., a], t[..., b]) * unit
        y = t.clone()
        y[..., a], y[..., b] = z.real, z.imag
        return y

    xt = x.transpose(0, 1)
    s = turned(xt[:H], w64[0]) @ turned(xt[H:2 * H], w64[1]).transpose(1, 2) / math.sqrt(d)
    o64 = torch.softmax(s.masked_fill(~_mask(wl, sel, L), -math.inf), -1) @ xt[2 * H:]
    outs = []
    for i in range(len(q_off) - 1):
        c = slice(k_off[i], k_off[i] + k_len[i])
        kk, vv = e[c, 0].transpose(0, 1), e[c, 1].transpose(0, 1)
        outs.append(torch.softmax(o64[:, q_off[i]:q_off[i + 1]] @ kk.transpose(1, 2) / math.sqrt(d), -1) @ vv)
    want = torch.cat(outs, 1)
    want.backward(d_out.double())
    # Every bf16 tensor between two operators, and P and dS inside them, is off by up to 2^-8 of itself: q, k, P, o, P' on the way to the
    # output, and besides dS', d_o, dS, dq or dk on the way back.  Five, then nine roundings, each of which moves what follows by about as much of
    # its size (in the 2-norm, where errors of single values average out; a score's error counts once more through the softmax).
    for what, got, ref, roundings in (("out", out, want.detach(), 6), ("d_qkv", d_qkv, x.grad, 12), ("d_states", d_states, e.grad, 12),
                                      ("dw_q", dw[0], w64[0].grad, 12), ("dw_k", dw[1], w64[1].grad, 12)):
        rel = float((got.double() - ref).norm() / ref.norm())
        assert rel <= roundings * 2.0 ** -8, (what, rel)
