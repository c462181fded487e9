"""The 64-bit plain forms that the operators around the sparse attention are held to, themselves: against autograd, central
differences, and closed forms."""
import math

import pytest
import torch

import layer_ref as R


@pytest.mark.parametrize("halves", [False, True])
def test_norm_and_rotation_against_autograd_and_differences(halves):
    g = torch.Generator().manual_seed(3)
    x = torch.randn(2, 5, 64, generator=g, dtype=torch.float64)
    w = 1 + 0.3 * torch.randn(64, generator=g, dtype=torch.float64)
    dy = torch.randn(2, 5, 64, generator=g, dtype=torch.float64)
    pos = torch.randint(-50, 5000, (5, 3), generator=g, dtype=torch.int32)
    axis = [0] * 6 + [1] * 10 + [2] * 8
    freq = [10000.0 ** (-m / 11) for m in range(24)]
    xa, wa = x.clone().requires_grad_(), w.clone().requires_grad_()
    # the rotation as complex numbers
    u = xa * torch.rsqrt((xa * xa).mean(-1, keepdim=True) + 1e-5) * wa
    a, b = R.pair_channels(24, halves)
    turned = torch.complex(u[..., a], u[..., b]) * torch.polar(torch.ones(5, 24, dtype=torch.float64), pos[:, axis].double() * torch.tensor(freq, dtype=torch.float64))
    y = u.clone()
    y[..., a], y[..., b] = turned.real, turned.imag
    y.backward(dy)
    got, _ = R.norm_rope(x, w, pos, axis, freq, halves, 1e-5)
    assert torch.allclose(got, y.detach(), atol=1e-12)
    (dx, _), (dw, _) = R.norm_rope_bwd(x, w, pos, axis, freq, halves, 1e-5, dy, 0.0)
    assert torch.allclose(dx, xa.grad, atol=1e-12) and torch.allclose(dw, wa.grad, atol=1e-12)
    e = 1e-6
    for h, t, c in [(0, 0, 0), (1, 4, 63), (0, 2, 30)]:
        lo, hi = x.clone(), x.clone()
        lo[h, t, c] -= e
        hi[h, t, c] += e
        num = ((R.norm_rope(hi, w, pos, axis, freq, halves, 1e-5)[0] - R.norm_rope(lo, w, pos, axis, freq, halves, 1e-5)[0]) * dy).sum() / (2 * e)
        assert abs(float(num - dx[h, t, c])) < 1e-8


def test_cross_attention_against_autograd_and_differences():
    g = torch.Generator().manual_seed(4)
    q_len, k_len, k_off, scale = [3, 0, 4, 2], [5, 2, 0, 7], [0, 6, 8, 9], 0.2
    q = torch.randn(4, 9, 16, generator=g, dtype=torch.float64)
    k, v = (torch.randn(2, 16, 16, generator=g, dtype=torch.float64) for _ in range(2))
    d_o = torch.randn(4, 9, 16, generator=g, dtype=torch.float64)
    ref = R.CrossRef(q, k, v, q_len, k_len, k_off, scale, d_o)
    mask = torch.zeros(9, 16, dtype=torch.bool)
    mask[0:3, 0:5] = mask[7:9, 9:16] = True
    qa, ka, va = (t.clone().requires_grad_() for t in (q, k, v))
    s = scale * qa @ ka.repeat_interleave(2, 0).transpose(1, 2)
    rows = mask.any(1)
    p = torch.softmax(s.masked_fill(~mask, -math.inf)[:, rows], -1)
    o = torch.zeros_like(q).index_copy(1, rows.nonzero()[:, 0], p @ va.repeat_interleave(2, 0))
    o.backward(d_o)
    assert torch.allclose(ref.o, o.detach(), atol=1e-12)
    for got, want in ((ref.dq, qa.grad), (ref.dk, ka.grad), (ref.dv, va.grad)):
        assert torch.allclose(got, want, atol=1e-12)
    assert bool((ref.lse[:, 3:7] == -math.inf).all()) and bool((ref.o[:, 3:7] == 0).all())
    e = 1e-6
    for t, grad in ((k, ref.dk), (v, ref.dv)):
        lo, hi = t.clone(), t.clone()
        lo[1, 10, 3] -= e
        hi[1, 10, 3] += e
        f = lambda x: (R.CrossRef(q, x if t is k else k, x if t is v else v, q_len, k_len, k_off, scale).o * d_o).sum()  # noqa: E731, B023
        assert abs(float((f(hi) - f(lo)) / (2 * e) - grad[1, 10, 3])) < 1e-8
