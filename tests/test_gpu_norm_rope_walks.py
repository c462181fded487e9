"""Norm and rotation of streams with more tokens than warps, where a warp walks several batches of heads of a token, goes on from its
queries to its keys, and takes a second and third token; and the outputs that may lie over inputs.  Against the 64-bit plain form."""
import pytest
import torch

import layer_ref as R
from paper_2508_21058_b200 import MocRope
from paper_2508_21058_b200.binding import debug_rope_split

pytestmark = pytest.mark.gpu

# tokens, query heads, key heads, d, channels per axis, halves, fp32; a token for each lane group
CASES = [
    (8001, 24, 24, 128, (44, 42, 42), False, False, False),
    (8001, 24, 8, 128, (32, 24, 24), True, False, False),
    (8001, 24, 8, 128, (44, 42, 42), False, True, False),
    (7500, 16, 16, 64, (16, 16, 16), True, True, False),
    (20001, 20, 20, 64, (16, 24, 24), True, True, True),
    (9003, 24, 0, 128, (64,), False, False, False),
    (20001, 9, 7, 64, (16, 24, 24), False, False, True),
    (20002, 9, 7, 64, (16, 16, 16), True, False, True),
    (12001, 5, 3, 128, (44, 42, 42), False, True, True),
    (20003, 12, 4, 64, (20, 20, 24), False, False, True),
]


def _inputs(case, seed):
    L, hq, hk, d, ax, halves, fp32, _ = case
    gen = torch.Generator("cuda").manual_seed(seed)
    t = torch.float32 if fp32 else torch.bfloat16
    x = (2 * torch.randn(L, hq + hk, d, generator=gen, device="cuda")).to(t)
    w = [1 + 0.3 * torch.randn(d, generator=gen, device="cuda") for _ in range(2)]
    pos = torch.randint(0, 3000, (L, len(ax)), generator=gen, device="cuda", dtype=torch.int32)
    dy = torch.randn(hq + hk, L, d, generator=gen, device="cuda")
    # rows whose part of dw is far above what sums of fp32 may be off by: the stream's first and last ones and some between
    for tok in (0, 1, L // 3, L // 2 + 1, L - 2, L - 1):
        dy[:, tok] *= 256
    axis = [a for a, n in enumerate(ax) for _ in range(n // 2)]
    freq = [10000.0 ** (-2.0 * m / n) for n in ax for m in range(n // 2)]
    return x, w, pos, dy.to(torch.bfloat16), axis, freq


def _ref(f, case, x, w, pos, axis, freq, *rest):
    """The plain form head by head on the GPU: it holds several 64-bit copies of what it is given."""
    a, b = (t.cuda() for t in R.pair_channels(len(axis), case[5]))
    t = pos.double()[:, axis] * torch.tensor(freq, dtype=torch.float64, device="cuda")
    return f(x, w.double(), a, b, t.cos(), t.sin(), *rest)


def _forward(x, w, a, b, cos, sin):
    u = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w
    return R._turn(u, a, b, cos, sin), R._pair_size(u, a, b)


def _backward(x, w, a, b, cos, sin, dy):
    g, gs = R._turn(dy, a, b, cos, -sin), R._pair_size(dy, a, b)
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)
    xh = x * r
    m = (w * g * xh).mean(-1, keepdim=True)
    size = r * (w.abs() * gs + xh.abs() * (w.abs() * gs * xh.abs()).mean(-1, keepdim=True))
    return r * (w * g - xh * m), size, (g * xh).sum(0), (gs * xh.abs()).sum(0)


# the same of streams whose tokens several warps share, each with more than one batch: some with queries and keys
SHARED = [
    (2003, 24, 24, 128, (44, 42, 42), False, False, False),
    (1999, 12, 24, 128, (32, 24, 24), True, False, False),
    (1500, 24, 8, 128, (44, 42, 42), False, True, False),
    (9001, 12, 12, 64, (16, 24, 24), False, False, True),
    (6402, 12, 4, 64, (16, 16, 16), True, False, True),
    (4001, 5, 9, 128, (44, 42, 42), False, True, True),
]


def _split(case, bwd):
    L, hq, hk, d, _, _, fp32, _ = case
    return debug_rope_split(fp32, bwd, d, L, hq, hk, torch.cuda.get_device_properties(0).multi_processor_count)


@pytest.mark.parametrize("case", CASES)
def test_walks_of_several_tokens(case):
    split = [_split(case, bwd) for bwd in (0, 1)]
    for s in split:
        assert s["by_token"] == case[-1] and s["per_warp"] > 1 and s["items"] > s["warps"]
    assert split[1]["items"] > 2 * split[1]["warps"]                     # a third token
    _check(case, split[1])


@pytest.mark.parametrize("case", SHARED)
def test_tokens_that_several_warps_share(case):
    split = [_split(case, bwd) for bwd in (0, 1)]
    assert all(s["by_token"] == case[-1] for s in split) and any(s["n_split"] > 1 and s["per_warp"] > 1 for s in split)
    _check(case, split[1])


def _check(case, s):
    """Both directions; s: the backward's split."""
    L, hq, hk, d, ax, halves, fp32, _ = case
    x, w, pos, dy, axis, freq = _inputs(case, 1)
    op = MocRope.from_axes(d, ax, halves=halves)
    xv = x.transpose(0, 1)
    y, dx, ws = torch.empty_like(dy), torch.empty_like(x), op.new_workspace()
    dxv, dw = dx.transpose(0, 1), [torch.empty(d, device="cuda") for _ in range(2)]
    k = (xv[hq:], w[1], y[hq:]) if hk else ()
    op.moc_norm_rope(pos, xv[:hq], w[0], y[:hq], *k)
    k = (xv[hq:], w[1], dy[hq:], dxv[hq:], dw[1]) if hk else ()
    op.moc_norm_rope_bwd(pos, xv[:hq], w[0], dy[:hq], dxv[:hq], dw[0], ws, *k)
    torch.cuda.synchronize()
    half = R.U32 if fp32 else R.U16
    # A term of dw is off by the norm and the rotation's roundings, and goes through one sum after another: a lane's rows, a warp's lane
    # groups, eight warps, the blocks in 32 strands of eight at a time, and 32 strands.
    rows = -(-s["items"] // s["warps"]) * s["per_warp"] * 6
    steps = rows + 2 + 8 + s["warps"] // 8 // 32 + 8 + 32
    for z, heads in ((0, range(hq)), (1, range(hq, hq + hk))):
        want_w, size_w = (torch.zeros(d, dtype=torch.float64, device="cuda") for _ in range(2))
        for h in heads:
            x64 = xv[h].double()
            want, size = _ref(_forward, case, x64, w[z], pos, axis, freq)
            R.check("y", y[h], want, R.U16 * want.abs() * (1 + R.U16) + (d / 2 + 16) * R.U32 * size)
            want, size, part, part_size = _ref(_backward, case, x64, w[z], pos, axis, freq, dy[h].double())
            R.check("dx", dxv[h], want, half * want.abs() * (1 + half) + (2 * d + 32) * R.U32 * size)
            want_w += part
            size_w += part_size
        if len(heads):
            R.check("dw", dw[z], want_w, (steps + d / 2 + 16) * R.U32 * size_w)


@pytest.mark.parametrize("fp32,over", [(False, "dq_out"), (False, "q"), (True, "q")])
@pytest.mark.parametrize("L,hq,hk,d,halves", [(37, 5, 2, 64, False), (300, 24, 8, 128, True), (5000, 24, 24, 128, False), (9000, 3, 1, 64, True)])
def test_gradients_over_an_input(fp32, over, L, hq, hk, d, halves):
    """dq, dk over dq_out, dk_out, or over q, k, give what they give elsewhere, bit for bit."""
    ax = (16, 24, 24) if d == 64 else (44, 42, 42)
    if halves:
        ax = (16, 16, 16)
    case = (L, hq, hk, d, ax, halves, fp32, None)
    x, w, pos, dy, axis, freq = _inputs(case, 2)
    op = MocRope.from_axes(d, ax, halves=halves)
    ws = op.new_workspace()
    xv = x.transpose(0, 1)
    if over == "dq_out":
        dy = dy.transpose(0, 1).contiguous().transpose(0, 1)             # the projection's strides
    dx, dw = torch.empty_like(x).transpose(0, 1), [torch.empty(d, device="cuda") for _ in range(4)]
    op.moc_norm_rope_bwd(pos, xv[:hq], w[0], dy[:hq], dx[:hq], dw[0], ws, xv[hq:], w[1], dy[hq:], dx[hq:], dw[1])
    out = dy if over == "dq_out" else xv
    op.moc_norm_rope_bwd(pos, xv[:hq], w[0], dy[:hq], out[:hq], dw[2], ws, xv[hq:], w[1], dy[hq:], out[hq:], dw[3])
    assert torch.equal(out, dx) and torch.equal(dw[0], dw[2]) and torch.equal(dw[1], dw[3])


@pytest.mark.parametrize("L,h,d", [(40, 4, 64), (9000, 24, 128)])
def test_a_rotation_alone_over_its_input_and_back(L, h, d):
    """Without a norm, forward and backward over the same tensor; the rotation keeps every row's length."""
    x, _, pos, _, _, _ = _inputs((L, h, 0, d, (d,), False, False, None), 3)
    op = MocRope.from_axes(d, (d,))
    v = x.transpose(0, 1)
    before, want, back = v.clone(), torch.empty_like(v), torch.empty_like(v)
    op.moc_norm_rope(pos, v, None, want)
    op.moc_norm_rope(pos, v, None, v)
    assert torch.equal(v, want)
    op.moc_norm_rope_bwd(pos, v, None, want, back, None, op.new_workspace())
    op.moc_norm_rope_bwd(pos, v, None, v, v, None, op.new_workspace())
    assert torch.equal(v, back)
    # two roundings to bf16 of channels no larger than their pair, sqrt(2) each at most
    err = (back.double() - before.double()).abs()
    size = R._pair_size(before.double(), *(t.cuda() for t in R.pair_channels(d // 2, False)))
    assert bool((err <= (2 * R.U16 * (1 + R.U16) + 64 * R.U32) * 1.5 * size).all())
