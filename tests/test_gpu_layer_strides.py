"""Strides that the header allows and no other test has: of dimensions of extent one, which are not looked at, and of parts of fused
tensors far apart; norm and rotation, and cross attention with its backward pass, against the same on contiguous tensors, bit for bit."""
import pytest
import torch

from paper_2508_21058_b200 import MocCross, MocRope

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _filled(shape, gen):
    return torch.randn(shape, generator=gen, device="cuda").to(BF)


def _cross(op, q, k, v, do, o, dq, dk, dv):
    lse, ws = torch.empty(op.H, op.n_queries, device="cuda"), op.new_workspace(with_bwd=True)
    op.moc_cross_attend(q, k, v, o, lse, ws)
    op.moc_cross_attend_bwd(q, k, v, o, lse, do, dq, dk, dv, ws)
    torch.cuda.synchronize()
    assert op.moc_cross_get_status(ws) == (0, 0)
    return [t.clone() for t in (o, lse, dq, dk, dv)]


def _one(t, dim, stride):
    """t with another stride of a dimension of extent one."""
    strides = list(t.stride())
    strides[dim] = stride
    return t.as_strided(t.shape, strides, t.storage_offset())


@pytest.mark.parametrize("stride", [0, 3, 1 << 45])
@pytest.mark.parametrize("d,q_len,k_len", [(64, [300], [200]), (128, [1], [500]), (128, [70], [1]), (64, [1], [1]), (128, [600] * 3, [400] * 3)])
def test_strides_of_an_extent_of_one(stride, d, q_len, k_len):
    gen = torch.Generator("cuda").manual_seed(1)
    nq, nk = sum(q_len), sum(k_len)
    op = MocCross(1, 1, d, [sum(q_len[:i]) for i in range(len(q_len) + 1)], [sum(k_len[:i]) for i in range(len(k_len) + 1)])
    q, k, v, do = _filled((1, nq, d), gen), _filled((1, nk, d), gen), _filled((1, nk, d), gen), _filled((1, nq, d), gen)
    want = _cross(op, q, k, v, do, *(torch.empty_like(t) for t in (q, q, k, v)))

    def odd(t):
        t = _one(t, 0, stride)
        return _one(t, 1, stride) if t.shape[1] == 1 else t

    outs = [torch.empty_like(t) for t in (q, q, k, v)]
    got = _cross(op, *(odd(t) for t in (q, k, v, do, *outs)))
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("heads,kv,d,q_len,k_len", [(6, 2, 128, [300, 17], [333, 64]), (4, 4, 64, [700], [129]), (6, 2, 64, [1, 1, 1], [400, 3, 900]),
                                                    (24, 8, 128, [2400, 100], [333, 200])])
def test_parts_of_fused_tensors(heads, kv, d, q_len, k_len):
    """Queries inside a fused projection, keys and values interleaved [state][2][kv head][d] inside wider rows, outputs and gradients likewise;
    what lies between them stays."""
    gen = torch.Generator("cuda").manual_seed(2)
    nq, nk = sum(q_len), sum(k_len)
    op = MocCross(heads, kv, d, [sum(q_len[:i]) for i in range(len(q_len) + 1)], [sum(k_len[:i]) for i in range(len(k_len) + 1)])
    q, k, v, do = _filled((heads, nq, d), gen), _filled((kv, nk, d), gen), _filled((kv, nk, d), gen), _filled((heads, nq, d), gen)
    want = _cross(op, q, k, v, do, *(torch.empty_like(t) for t in (q, q, k, v)))
    wide_q = torch.full((4, nq, 3 * heads, d + 8), 5.0, dtype=BF, device="cuda")        # q, do, o, dq
    wide_k = torch.full((2, nk, 2 * kv + 1, d + 24), 5.0, dtype=BF, device="cuda")      # k and v; dk and dv
    pq = [w[:, heads:2 * heads, 8:].transpose(0, 1) for w in wide_q]
    pk = [w[:, i * kv:(i + 1) * kv, 16:16 + d].transpose(0, 1) for w in wide_k for i in range(2)]
    for t, s in zip((*pq[:2], *pk[:2]), (q, do, k, v)):
        t.copy_(s)
    got = _cross(op, pq[0], pk[0], pk[1], pq[1], pq[2], pq[3], pk[2], pk[3])
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    for t in (*pq, *pk):
        t.fill_(5.0)
    assert bool((wide_q == 5.0).all()) and bool((wide_k == 5.0).all())


@pytest.mark.parametrize("stride", [0, 3, 1 << 45])
@pytest.mark.parametrize("L,h,fp32", [(1, 5, False), (40, 1, False), (1, 1, True), (300, 1, True)])
def test_strides_of_an_extent_of_one_in_norm_and_rotation(stride, L, h, fp32):
    gen = torch.Generator("cuda").manual_seed(3)
    d = 128
    op = MocRope.from_axes(d, (44, 42, 42))
    x, dy = _filled((h, L, d), gen), _filled((h, L, d), gen)
    x = x.float() if fp32 else x
    pos = torch.randint(0, 50, (L, 3), generator=gen, device="cuda", dtype=torch.int32)
    w = 1 + 0.1 * torch.randn(d, generator=gen, device="cuda")

    def odd(t):
        t = _one(t, 0, stride) if h == 1 else t
        return _one(t, 1, stride) if L == 1 else t

    res = []
    for f in (lambda t: t, odd):
        y, dx, dw = torch.empty_like(dy), torch.empty_like(x), torch.empty(d, device="cuda")
        op.moc_norm_rope(pos, f(x), w, f(y))
        op.moc_norm_rope_bwd(pos, f(x), w, f(dy), f(dx), dw, op.new_workspace())
        res.append((y, dx, dw))
    assert all(torch.equal(a, b) for a, b in zip(*res))
