"""Norm of query and key heads with the position rotation in one pass, and its backward pass, through the C ABI against the 64-bit
plain form: both pairings, types, head sizes, layouts, missing norm, missing rotation, missing keys, far positions, one token."""
import pytest
import torch

import layer_ref as R
import parity_utils as PU
from paper_2508_21058_b200 import MocError, MocRope

pytestmark = pytest.mark.gpu

# tokens, query heads, key heads, d, channels per axis, halves, type, norm
CASES = [
    (1, 1, 0, 64, (), False, "bf16", True),
    (1, 24, 24, 128, (44, 42, 42), False, "bf16", True),
    (3, 5, 1, 64, (16, 24, 24), True, "bf16", True),
    (257, 4, 4, 64, (16, 24, 24), False, "fp32", True),
    (130, 24, 8, 128, (32, 24, 24), True, "fp32", True),
    (77, 3, 2, 128, (128,), True, "bf16", True),
    (33, 2, 2, 128, (6, 2, 0, 4), False, "bf16", True),
    (33, 9, 3, 64, (16,), True, "bf16", False),
    (40, 2, 7, 128, (), False, "fp32", True),
    (40, 2, 1, 64, (10, 2), False, "fp32", False),
    (5000, 2, 1, 64, (20, 20, 24), False, "bf16", True),
]


def _make(L, hq, hk, d, ax, halves, dtype, norm, seed=0):
    gen = torch.Generator().manual_seed(seed)
    t = torch.float32 if dtype == "fp32" else torch.bfloat16
    x = (3 * torch.randn(L, hq + hk, d, generator=gen)).to(t)
    w = [1 + 0.3 * torch.randn(d, generator=gen) if norm else None for _ in range(2)]
    pos = torch.randint(-2**31, 2**31 - 1, (L, len(ax)), generator=gen, dtype=torch.int64).to(torch.int32)
    pos[::2] = pos[::2] % 100
    dy = torch.randn(hq + hk, L, d, generator=gen).to(torch.bfloat16)
    axis = [a for a, n in enumerate(ax) for _ in range(n // 2)]
    freq = [10000.0 ** (-2.0 * m / n) for n in ax for m in range(n // 2)]
    return x, w, pos, dy, axis, freq


@pytest.mark.parametrize("case", CASES)
def test_forward_and_backward_against_64_bits(case):
    L, hq, hk, d, ax, halves, dtype, norm = case
    x, w, pos, dy, axis, freq = _make(*case)
    eps = 1e-6
    op = MocRope.from_axes(d, ax, eps=eps, halves=halves)
    g = PU.Guarded()
    xd = x.cuda().transpose(0, 1)                              # [head][token][d], strided
    wd = [None if v is None else v.cuda() for v in w]
    y = g.empty((hq + hk, L, d), torch.bfloat16)
    k = (xd[hq:], wd[1], y[hq:]) if hk else ()
    op.moc_norm_rope(pos.cuda(), xd[:hq], wd[0], y[:hq], *k)
    dx = g.empty((L, hq + hk, d), x.dtype)
    dxv = dx.transpose(0, 1)
    dw = [g.empty((d,), torch.float32) if norm else None for _ in range(2)]
    ws = g.empty((op.workspace_bytes(),), torch.uint8)
    dyd = dy.cuda()
    k = (xd[hq:], wd[1], dyd[hq:], dxv[hq:], dw[1]) if hk else ()
    op.moc_norm_rope_bwd(pos.cuda(), xd[:hq], wd[0], dyd[:hq], dxv[:hq], dw[0], ws, *k)
    torch.cuda.synchronize()
    g.check()
    x64 = x.double().transpose(0, 1)
    for z, heads in ((0, slice(0, hq)), (1, slice(hq, hq + hk))):
        if heads.start == heads.stop:
            continue
        want, tol = R.norm_rope(x64[heads], w[z], pos, axis, freq, halves, eps)
        R.check("y", y[heads], want, tol)
        (want, tol), (want_w, tol_w) = R.norm_rope_bwd(x64[heads], w[z], pos, axis, freq, halves, eps, dy[heads].double(),
                                                       R.U32 if dtype == "fp32" else R.U16)
        R.check("dx", dxv[heads], want, tol)
        if norm:
            R.check("dw", dw[z], want_w, tol_w)
    # again, bit for bit
    dw2 = [None if v is None else torch.empty_like(v) for v in dw]
    dx2 = torch.empty_like(dx)
    d2v = dx2.transpose(0, 1)
    k = (xd[hq:], wd[1], dyd[hq:], d2v[hq:], dw2[1]) if hk else ()
    op.moc_norm_rope_bwd(pos.cuda(), xd[:hq], wd[0], dyd[:hq], d2v[:hq], dw2[0], ws, *k)
    assert torch.equal(dx2, dx) and all(a is None or torch.equal(a, b) for a, b in list(zip(dw, dw2))[:2 if hk else 1])


def test_part_of_a_fused_projection_in_place_and_no_tokens():
    """Queries and keys inside a fused projection whose values stay as they are; the output over the input; no tokens."""
    L, hq, hk, d = 19, 4, 2, 64
    gen = torch.Generator().manual_seed(1)
    qkv = torch.randn(L, hq + 2 * hk, d, generator=gen).to(torch.bfloat16)
    w = 1 + 0.1 * torch.randn(d, generator=gen)
    pos = torch.randint(0, 50, (L, 3), generator=gen, dtype=torch.int32)
    op = MocRope.from_axes(d, (16, 24, 24))
    dev, v = qkv.cuda(), qkv.cuda().transpose(0, 1)
    q_out, k_out = torch.empty(hq, L, d, dtype=torch.bfloat16, device="cuda"), torch.empty(hk, L, d, dtype=torch.bfloat16, device="cuda")
    op.moc_norm_rope(pos.cuda(), v[:hq], w.cuda(), q_out, v[hq:hq + hk], w.cuda(), k_out)
    t = dev.transpose(0, 1)
    op.moc_norm_rope(pos.cuda(), t[:hq], w.cuda(), t[:hq], t[hq:hq + hk], w.cuda(), t[hq:hq + hk])
    assert torch.equal(t[:hq], q_out) and torch.equal(t[hq:hq + hk], k_out) and torch.equal(dev[:, hq + hk:].cpu(), qkv[:, hq + hk:])
    none = torch.empty(hq, 0, d, dtype=torch.bfloat16, device="cuda")
    dw = torch.full((d,), 7.0, device="cuda")
    op.moc_norm_rope(pos[:0].cuda(), none, w.cuda(), none)
    op.moc_norm_rope_bwd(pos[:0].cuda(), none, w.cuda(), none, none, dw, op.new_workspace())
    assert bool((dw == 0).all())


def test_rows_far_apart():
    """Offsets beyond 32 bits: two heads more than 2^31 values apart."""
    d, L, gap = 64, 3, 2**31 + 64
    buf = torch.empty(gap + L * d, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((2, L, d), (gap, d, 1))
    gen = torch.Generator().manual_seed(2)
    h = torch.randn(2, L, d, generator=gen).to(torch.bfloat16)
    x.copy_(h)
    pos = torch.randint(0, 50, (L, 1), generator=gen, dtype=torch.int32)
    op = MocRope.from_axes(d, (64,))
    w = torch.ones(d, device="cuda")
    op.moc_norm_rope(pos.cuda(), x, w, x)
    want, tol = R.norm_rope(h.double(), w.cpu(), pos, [0] * 32, [10000.0 ** (-m / 32) for m in range(32)], False, 1e-6)
    R.check("y", x, want, tol)


def test_special_values_stay_in_their_rows():
    """An infinity or NaN makes its own row's output what the formula gives and touches no other row; without norm, channels that are
    not turned pass through."""
    L, d = 6, 64
    gen = torch.Generator().manual_seed(5)
    x = torch.randn(3, L, d, generator=gen).to(torch.bfloat16)
    pos = torch.randint(0, 50, (L, 1), generator=gen, dtype=torch.int32)
    op = MocRope.from_axes(d, (32,))
    clean = torch.empty(3, L, d, dtype=torch.bfloat16, device="cuda")
    op.moc_norm_rope(pos.cuda(), x.cuda(), None, clean)
    x[1, 2, 50] = float("inf")
    x[2, 4, 60] = float("nan")
    y = torch.empty_like(clean)
    op.moc_norm_rope(pos.cuda(), x.cuda(), None, y)
    clean[1, 2, 50], clean[2, 4, 60] = float("inf"), float("nan")
    assert torch.equal(torch.nan_to_num(y, nan=123.0), torch.nan_to_num(clean, nan=123.0))
    w = torch.ones(d, device="cuda")
    op.moc_norm_rope(pos.cuda(), x.cuda(), w, y)
    bad = ~torch.isfinite(y).all(-1)
    assert bad.nonzero().tolist() == [[1, 2], [2, 4]]


@pytest.mark.parametrize("case", [(6, 5, 3, 128, (44, 42, 42), False, "bf16", True), (9, 5, 1, 64, (16, 24, 24), True, "fp32", True),
                                  (7, 11, 12, 128, (44, 42, 42), False, "bf16", True), (1, 23, 7, 64, (64,), True, "bf16", True)])
def test_no_eps_and_heads_that_leave_lanes_without_a_row(case):
    L, hq, hk, d, ax, halves, dtype, norm = case
    x, w, pos, dy, axis, freq = _make(*case, seed=7)
    op = MocRope.from_axes(d, ax, eps=0.0, halves=halves)
    xd, dyd = x.cuda().transpose(0, 1), dy.cuda()
    dx = torch.empty(hq + hk, L, d, dtype=x.dtype, device="cuda")
    dw = [torch.empty(d, device="cuda") for _ in range(2)]
    op.moc_norm_rope_bwd(pos.cuda(), xd[:hq], w[0].cuda(), dyd[:hq], dx[:hq], dw[0], op.new_workspace(), xd[hq:], w[1].cuda(), dyd[hq:],
                         dx[hq:], dw[1])
    x64 = x.double().transpose(0, 1)
    for z, heads in ((0, slice(0, hq)), (1, slice(hq, hq + hk))):
        (want, tol), (want_w, tol_w) = R.norm_rope_bwd(x64[heads], w[z], pos, axis, freq, halves, 0.0, dy[heads].double(),
                                                       R.U32 if dtype == "fp32" else R.U16)
        R.check("dx", dx[heads], want, tol)
        R.check("dw", dw[z], want_w, tol_w)


def test_graph_other_stream_and_refusals_of_the_binding():
    L, h, d = 64, 4, 128
    gen = torch.Generator().manual_seed(6)
    op = MocRope.from_axes(d, (44, 42, 42))
    x = torch.randn(h, L, d, generator=gen).to(torch.bfloat16).cuda()
    dy = torch.randn(h, L, d, generator=gen).to(torch.bfloat16).cuda()
    pos = torch.randint(0, 50, (L, 3), generator=gen, dtype=torch.int32).cuda()
    w = torch.ones(d, device="cuda")
    y, dx, dw, ws = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), op.new_workspace()

    def step():
        op.moc_norm_rope(pos, x, w, y)
        op.moc_norm_rope_bwd(pos, x, w, dy, dx, dw, ws)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    x.copy_(torch.randn(h, L, d, generator=gen))
    graph.replay()
    got = [t.clone() for t in (y, dx, dw)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, (y, dx, dw)))
    for bad in (lambda: op.moc_norm_rope(pos, x, w, y.float()), lambda: op.moc_norm_rope(pos.long(), x, w, y),
                lambda: op.moc_norm_rope(pos[:-1], x, w, y), lambda: op.moc_norm_rope(pos, x.half(), w, y),
                lambda: op.moc_norm_rope(pos, x, w.bfloat16(), y), lambda: op.moc_norm_rope(pos, x, w, y[:, :, ::2]),
                lambda: op.moc_norm_rope(pos, x[:1].expand(4, L, d), w, y), lambda: op.moc_norm_rope(pos.cpu(), x, w, y),
                lambda: op.moc_norm_rope(pos, x.cpu(), w, y), lambda: op.moc_norm_rope_bwd(pos, x, w, dy, dx, dw, ws[:-256]),
                lambda: op.moc_norm_rope(pos, x, w, y[:, :-1])):
        with pytest.raises(MocError):
            bad()
