"""Operators beside the sparse attention, as a layer of a video transformer uses them: the norm of every query and key head with
the (time, height, width) rotation in one pass, forward and backward, and cross attention of a stream's shots to their prompts'
encoder states, forward and training step.  `run` computes them with elementary torch operations, or, where `own` is set, through
the library.

A case is a dict of plain values.
  task "rope", "rope-bwd": a fused projection [token][q heads + 2 k heads][dim]; the stream has `shots` shots of `caption` text tokens and
      `frames` frames of `height` x `width` tokens.  `ax_t`, `ax_h`, `ax_w`: channels that each axis turns; `halves`: channel j is
      turned with channel j + (ax_t + ax_h + ax_w) / 2, else with its neighbour; `norm`: with the norm; `fp32`: the projection's type
  task "cross", "cross-train": `segments` sequences of up to `q_len` queries and `k_len` encoder states, `heads` query heads on
      `kv_heads` key heads; `ragged`: the lengths differ; `padded`: the states lie `k_len` apart, else packed
"""
from __future__ import annotations

import math

import torch

own = False
THETA, EPS = 10000.0, 1e-6


def _rope(task, shots, caption, frames, height, width, q_heads, k_heads, dim, ax, halves=False, norm=True, fp32=False, **name):
    return dict(name, task=task, shots=shots, caption=caption, frames=frames, height=height, width=width, q_heads=q_heads, k_heads=k_heads,
                dim=dim, ax_t=ax[0], ax_h=ax[1], ax_w=ax[2], halves=halves, norm=norm, fp32=fp32)


def _cross(task, segments, q_len, k_len, heads, kv_heads, dim, ragged=False, padded=False, **name):
    return dict(name, task=task, segments=segments, q_len=q_len, k_len=k_len, heads=heads, kv_heads=kv_heads, dim=dim, ragged=ragged,
                padded=padded)


def listed():
    return [
        # the smallest stream, 576 tokens of four small heads: launches and latency
        _rope("rope", 1, 64, 8, 8, 8, 4, 4, 64, (16, 24, 24), name="rope-small"),
        # a clip of 33k tokens, all heads
        _rope("rope", 1, 256, 21, 30, 52, 24, 24, 128, (44, 42, 42), name="rope-clip"),
        # an fp32 projection with shared key heads, halves turned, a part of the channels not turned; an odd frame
        _rope("rope", 2, 77, 5, 27, 47, 24, 8, 128, (32, 24, 24), halves=True, fp32=True, name="rope-fp32-halves"),
        # eight shots, 264k tokens: the largest stream
        _rope("rope", 8, 256, 21, 30, 52, 24, 24, 128, (44, 42, 42), name="rope-scenes"),
        # the clip's backward pass
        _rope("rope-bwd", 1, 256, 21, 30, 52, 24, 24, 128, (44, 42, 42), name="rope-clip-bwd"),
        # a small training stream of odd sizes, small heads
        _rope("rope-bwd", 3, 41, 7, 13, 23, 12, 4, 64, (16, 24, 24), halves=True, name="rope-odd-bwd"),
        # a small clip to a short prompt: latency
        _cross("cross", 1, 576, 77, 4, 4, 64, name="cross-small"),
        # the clip to a prompt of 512 states
        _cross("cross", 1, 33016, 512, 24, 24, 128, name="cross-clip"),
        # few rows to many states: a caption's tokens read a clip's latents
        _cross("cross", 1, 257, 32760, 24, 24, 128, name="cross-few-rows"),
        # one query token a sequence (a step of generation token by token), encoder states of many lengths, shared key heads
        _cross("cross", 64, 1, 1500, 24, 8, 128, ragged=True, padded=True, name="cross-single-tokens"),
        # the clip's training step
        _cross("cross-train", 1, 33016, 512, 24, 24, 128, name="cross-clip-train"),
        # shots of many lengths, each to its own prompt, shared key heads
        _cross("cross-train", 8, 33016, 512, 6, 2, 128, ragged=True, padded=True, name="cross-scenes-train"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Streams of 6 to 264k tokens, 1 to 24 heads of 64 or 128 channels; prompts of 1 to 32k states."""
    top = max(max(work(c)["bytes"], work(c)["flops"] / 250) for c in listed())
    while True:
        dim = 64 if rng.random() < 0.3 else 128
        kv = _log_int(rng, 1, 24)
        heads = kv * rng.choice([g for g in (1, 1, 2, 3, 4, 8) if g * kv <= 24])
        if rng.random() < 0.5:
            half = [2 * rng.randint(0, dim // 6) for _ in range(3)]
            halves = rng.random() < 0.5
            if halves:                                # a multiple of 16 channels is turned
                half[0] += -sum(half) % 16
            if sum(half) > dim:
                continue
            c = _rope(rng.choice(["rope", "rope-bwd"]), _log_int(rng, 1, 8), _log_int(rng, 1, 300), _log_int(rng, 1, 24), _log_int(rng, 1, 32),
                      _log_int(rng, 1, 56), heads, kv, dim, half, halves, rng.random() < 0.85, rng.random() < 0.3)
        else:
            seg = 1 if rng.random() < 0.4 else _log_int(rng, 2, 64)
            task = rng.choice(["cross", "cross", "cross-train"])
            least = 16 if task == "cross-train" else 1       # with one state the gradients of queries and keys are zero: nothing to compare
            c = _cross(task, seg, 1 if rng.random() < 0.15 else _log_int(rng, 2, 33000 if seg < 10 else 3000),
                       _log_int(rng, least, 32000 if rng.random() < 0.2 else 1600), heads, kv, dim, rng.random() < 0.5, rng.random() < 0.4)
            if heads * seg * c["q_len"] * c["k_len"] > 8e8:      # of what the plain form holds in 32 bits
                continue
        w = work(c)
        if max(w["bytes"], w["flops"] / 250) <= top:
            return c


def _tokens(c):
    return c["shots"] * (c["caption"] + c["frames"] * c["height"] * c["width"])


def _lengths(c):
    """Queries and encoder states of every segment, and where its states begin."""
    n = c["segments"]
    q = [max(1, c["q_len"] - (i * 7919 % (c["q_len"] // 2 + 1) if c["ragged"] else 0)) for i in range(n)]
    k = [max(1, c["k_len"] - (i * 104729 % (c["k_len"] * 3 // 4 + 1) if c["ragged"] else 0)) for i in range(n)]
    at = [0]
    for x in k:
        at.append(at[-1] + (c["k_len"] if c["padded"] else x))
    return q, k, at


def work(c):
    d = c["dim"]
    if c["task"].startswith("rope"):
        values = float(_tokens(c)) * (c["q_heads"] + c["k_heads"]) * d
        x = 4 if c["fp32"] else 2
        if c["task"] == "rope":
            return {"bytes": values * (x + 2) + 12.0 * _tokens(c), "flops": 10 * values}
        reads_x = x if c["norm"] else 0
        return {"bytes": values * (2 + x + reads_x) + 12.0 * _tokens(c), "flops": 20 * values}
    q, k, _ = _lengths(c)
    pairs = float(c["heads"]) * sum(a * b for a, b in zip(q, k))
    rows, keys = 2.0 * c["heads"] * sum(q) * d, 2.0 * c["kv_heads"] * sum(k) * d
    if c["task"] == "cross":
        return {"bytes": 2 * rows + 2 * keys + 4.0 * c["heads"] * sum(q), "flops": 4 * d * pairs}
    # forward, then dO read and dQ, dK, dV written (the forward's operands counted once)
    return {"bytes": 4 * rows + 4 * keys + 4.0 * c["heads"] * sum(q), "flops": 14 * d * pairs}


# ---- inputs
def _positions(c, first):
    """int32 [token][3]: the frame's number in the stream and the place in the frame; a caption's tokens stand one after another in time."""
    cap, f, h, w = c["caption"], c["frames"], c["height"], c["width"]
    dev = "cuda"
    z = torch.zeros(cap, dtype=torch.int32, device=dev)
    text = torch.stack([torch.arange(cap, dtype=torch.int32, device=dev), z, z], 1)
    grid = torch.stack(torch.meshgrid(torch.arange(f, device=dev), torch.arange(h, device=dev), torch.arange(w, device=dev), indexing="ij"), -1)
    shot = torch.cat([text, grid.reshape(-1, 3).to(torch.int32) + torch.tensor([cap, 0, 0], dtype=torch.int32, device=dev)])
    step = torch.arange(c["shots"], dtype=torch.int32, device=dev) * (cap + f) + first
    pos = shot[None].repeat(c["shots"], 1, 1)
    pos[:, :, 0] += step[:, None]
    return pos.reshape(-1, 3).contiguous()


def prepare(c, seed):
    gen = torch.Generator("cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=gen)

    if c["task"].startswith("rope"):
        L, hq, hk, d = _tokens(c), c["q_heads"], c["k_heads"], c["dim"]
        s = {"case": c, "pos": _positions(c, seed % 1000)}
        s["qkv"] = normal(L, hq + 2 * hk, d, dtype=torch.float32 if c["fp32"] else torch.bfloat16)
        for n in ("w_q", "w_k"):
            s[n] = 1 + 0.2 * normal(d, dtype=torch.float32) if c["norm"] else None
        if c["task"] == "rope-bwd":
            s["d_q"], s["d_k"] = normal(hq, L, d), normal(hk, L, d)
        if own:
            from paper_2508_21058_b200 import MocRope
            s["op"] = MocRope.from_axes(d, (c["ax_t"], c["ax_h"], c["ax_w"]), theta=THETA, eps=EPS, halves=c["halves"])
            s["ws"] = s["op"].new_workspace()
        return s
    q, k, at = _lengths(c)
    H, kv, d = c["heads"], c["kv_heads"], c["dim"]
    s = {"case": c, "q": normal(H, sum(q), d), "kv": normal(at[-1], 2, kv, d)}
    s["q_len"], s["k_len"] = torch.tensor(q, device="cuda"), torch.tensor(k, device="cuda")
    s["k_at"] = torch.tensor(at[:-1], device="cuda")
    s["q_at"] = torch.cumsum(s["q_len"], 0) - s["q_len"]
    if c["task"] == "cross-train":
        s["d_o"] = normal(H, sum(q), d)
    if own:
        from paper_2508_21058_b200 import MocCross
        q_off = [sum(q[:i]) for i in range(len(q) + 1)]
        s["op"] = MocCross(H, kv, d, q_off, at, k_len=k)
        s["ws"] = s["op"].new_workspace(with_bwd=c["task"] == "cross-train")
    return s


def _q_k(s):
    """The projection's queries and keys, [head][token][dim] (the values behind them are not looked at)."""
    c, x = s["case"], s["qkv"].transpose(0, 1)
    return x[:c["q_heads"]], x[c["q_heads"]:c["q_heads"] + c["k_heads"]]


def _kv(s):
    return s["kv"][:, 0].transpose(0, 1), s["kv"][:, 1].transpose(0, 1)


def run(s):
    c = s["case"]
    if c["task"].startswith("rope"):
        return (_rope_own if own else _rope_plain)(s)
    return (_cross_own if own else _cross_plain)(s)


# ---- through the library
def _rope_own(s):
    c, op = s["case"], s["op"]
    q, k = _q_k(s)
    if c["task"] == "rope":
        q_out, k_out = (torch.empty(x.shape, dtype=torch.bfloat16, device="cuda") for x in (q, k))
        op.moc_norm_rope(s["pos"], q, s["w_q"], q_out, k, s["w_k"], k_out)
        return {"q": q_out, "k": k_out}
    grad = torch.empty_like(s["qkv"])                      # the projection's gradient; its values' part comes of the attention
    dq, dk = _q_k({"case": c, "qkv": grad})
    dw_q, dw_k = (torch.empty_like(s["w_q"]) if c["norm"] else None for _ in range(2))
    op.moc_norm_rope_bwd(s["pos"], q, s["w_q"], s["d_q"], dq, dw_q, s["ws"], k, s["w_k"], s["d_k"], dk, dw_k)
    return {"dq": dq, "dk": dk, "dw_q": dw_q, "dw_k": dw_k}


def _cross_own(s):
    op, q = s["op"], s["q"]
    k, v = _kv(s)
    o, lse = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
    op.moc_cross_attend(q, k, v, o, lse, s["ws"])
    if s["case"]["task"] == "cross":
        return {"o": o, "lse": lse}
    dq, dkv = torch.empty_like(q), torch.empty_like(s["kv"])
    dk, dv = _kv({"kv": dkv})
    op.moc_cross_attend_bwd(q, k, v, o, lse, s["d_o"], dq, dk, dv, s["ws"])
    return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


# ---- plain forms
def _turns(c, pos):
    """cos and sin of every token's angles, [token][pair]: the angle in 64 bits."""
    parts = []
    parts += [pos[:, 0:1].double() * THETA ** (-torch.arange(c["ax_t"] // 2, dtype=torch.float64, device="cuda") * 2 / max(1, c["ax_t"]))]
    parts += [pos[:, 1:2].double() * THETA ** (-torch.arange(c["ax_h"] // 2, dtype=torch.float64, device="cuda") * 2 / max(1, c["ax_h"]))]
    parts += [pos[:, 2:3].double() * THETA ** (-torch.arange(c["ax_w"] // 2, dtype=torch.float64, device="cuda") * 2 / max(1, c["ax_w"]))]
    angle = torch.cat(parts, 1)
    return angle.cos().float(), angle.sin().float()


def _turn(c, x, cos, sin):
    """The rotation by (cos, sin) of the channels that are turned."""
    n = cos.shape[1]
    if c["halves"]:
        a, b = x[..., :n], x[..., n:2 * n]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * n:]], -1)
    a, b = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., 2 * n:]], -1)


def _rope_plain(s):
    c = s["case"]
    cos, sin = _turns(c, s["pos"])

    def forward(x, w):
        x = x.float()
        if w is not None:
            x = x * ((x * x).mean(-1, keepdim=True) + EPS).rsqrt() * w
        return _turn(c, x, cos, sin).to(torch.bfloat16).contiguous()

    def backward(x, w, dy):
        g = _turn(c, dy.float(), cos, -sin)
        if w is None:
            return g.to(x.dtype), None
        x = x.float()
        r = ((x * x).mean(-1, keepdim=True) + EPS).rsqrt()
        xh = x * r
        dw = (g * xh).sum((0, 1), dtype=torch.float64).float()
        g = g * w
        return (r * (g - xh * (g * xh).mean(-1, keepdim=True))).to(s["qkv"].dtype), dw

    q, k = _q_k(s)
    if c["task"] == "rope":
        return {"q": forward(q, s["w_q"]), "k": forward(k, s["w_k"])}
    dq, dw_q = backward(q, s["w_q"], s["d_q"])
    dk, dw_k = backward(k, s["w_k"], s["d_k"])
    return {"dq": dq, "dk": dk, "dw_q": dw_q, "dw_k": dw_k}


def _cross_plain(s):
    """Every segment's queries and states in a batch of equal lengths; what a segment does not have is masked."""
    c = s["case"]
    n, lq, lk, kv, d = c["segments"], int(c["q_len"]), int(c["k_len"]), c["kv_heads"], c["dim"]
    g, scale = c["heads"] // kv, 1 / math.sqrt(d)
    i, j = torch.arange(lq, device="cuda"), torch.arange(lk, device="cuda")
    has_q, has_k = i[None] < s["q_len"][:, None], j[None] < s["k_len"][:, None]
    at_q = torch.where(has_q, s["q_at"][:, None] + i, 0)
    at_k = torch.where(has_k, s["k_at"][:, None] + j, 0)

    def rows(x):                                           # [kv head, segment, group, query, dim]
        return x.float()[:, at_q.flatten()].view(kv, g, n, lq, d).transpose(1, 2)

    def keys(x):                                           # [kv head, segment, 1, state, dim]; states that are not there are zero
        return torch.where(has_k[None, :, :, None], x.float()[:, at_k.flatten()].view(kv, n, lk, d), 0).unsqueeze(2)

    def packed(x):                                         # back to [head, query, ...]
        return x.transpose(1, 2).flatten(0, 1)[:, has_q]

    q, (k, v) = rows(s["q"]), map(keys, _kv(s))
    p = torch.matmul(q, k.transpose(-1, -2)).mul_(scale).masked_fill_(~has_k[None, :, None, None], -math.inf)
    top = p.amax(-1, keepdim=True)
    p = p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (total.log() + top).squeeze(-1)
    p = p.div_(total)
    o = torch.matmul(p, v)
    out = {"o": packed(o).to(torch.bfloat16), "lse": packed(lse)}
    if c["task"] == "cross":
        return out
    do = torch.where(has_q[None, :, None, :, None], rows(s["d_o"]), 0)
    dv = torch.matmul(p.transpose(-1, -2), do).sum(2)
    ds = torch.matmul(do, v.transpose(-1, -2)).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    del p
    dk = torch.matmul(ds.transpose(-1, -2), q).sum(2)
    dq = torch.matmul(ds, k)
    out["dq"] = packed(dq).to(torch.bfloat16)

    def states(x):                                         # gradients of the states; those behind a sequence's last get zero
        full = torch.zeros((kv, s["kv"].shape[0], d), dtype=torch.bfloat16, device="cuda")
        full[:, at_k[has_k]] = x[:, has_k].to(torch.bfloat16)
        return full

    out["dk"], out["dv"] = states(dk), states(dv)
    return out


# ---- from the definition, in 64 bits
def exact(c, seed):
    s = prepare(c, seed)
    return _rope_exact(c, s) if c["task"].startswith("rope") else _cross_exact(c, s)


def _rope_exact(c, s):
    """Every head by itself: the norm, then each turned pair of channels as the product of complex numbers."""
    L, d, hq, hk = _tokens(c), c["dim"], c["q_heads"], c["k_heads"]
    freq, axis = [], []
    for a, width in enumerate((c["ax_t"], c["ax_h"], c["ax_w"])):
        for m in range(width // 2):
            freq.append(math.exp(-math.log(THETA) * 2 * m / width))
            axis.append(a)
    n = len(freq)
    first = list(range(n)) if c["halves"] else [2 * m for m in range(n)]
    second = [m + n for m in first] if c["halves"] else [m + 1 for m in first]
    first, second, axis = (torch.tensor(x, dtype=torch.int64, device="cuda") for x in (first, second, axis))
    phase = s["pos"][:, axis].to(torch.float64) * torch.tensor(freq, dtype=torch.float64, device="cuda")
    unit = torch.polar(torch.ones_like(phase), phase)

    def turned(x, by):
        z = torch.complex(x[:, first], x[:, second]) * by
        y = x.clone()
        y[:, first], y[:, second] = z.real, z.imag
        return y

    out = {}
    for name, h0, heads in (("q", 0, hq), ("k", hq, hk)):
        w = None if s["w_" + name] is None else s["w_" + name].double()
        y = torch.empty((heads, L, d), dtype=torch.float64, device="cuda")
        dw = torch.zeros(d, dtype=torch.float64, device="cuda")
        for h in range(heads):
            x = s["qkv"][:, h0 + h].double()
            size = torch.sqrt(x.pow(2).sum(1, keepdim=True) / d + EPS)
            if c["task"] == "rope":
                y[h] = turned(x if w is None else x / size * w, unit)
                continue
            g = turned(s["d_" + name][h].double(), unit.conj())
            if w is None:
                y[h] = g
            else:
                dw += (g * x / size).sum(0)
                y[h] = g * w / size - x * ((g * w * x).sum(1, keepdim=True) / (d * size ** 3))
        if c["task"] == "rope":
            out[name] = y
        else:
            out["d" + name], out["dw_" + name] = y, None if w is None else dw
    return out


def _cross_exact(c, s):
    """Every segment and head by itself."""
    q_len, k_len, at = _lengths(c)
    H, kv, d = c["heads"], c["kv_heads"], c["dim"]
    train, Lq = c["task"] == "cross-train", sum(q_len)
    zeros = lambda *shape: torch.zeros(shape, dtype=torch.float64, device="cuda")  # noqa: E731
    out = {"o": zeros(H, Lq, d), "lse": zeros(H, Lq)}
    if train:
        out.update(dq=zeros(H, Lq, d), dk=zeros(kv, at[-1], d), dv=zeros(kv, at[-1], d))
    r0 = 0
    for seg, (nq, nk) in enumerate(zip(q_len, k_len)):
        rows, cols = slice(r0, r0 + nq), slice(at[seg], at[seg] + nk)
        r0 += nq
        for h in range(H):
            q, k, v = s["q"][h, rows].double(), s["kv"][cols, 0, h * kv // H].double(), s["kv"][cols, 1, h * kv // H].double()
            score = q @ k.T / math.sqrt(d)
            out["lse"][h, rows] = torch.logsumexp(score, 1)
            p = torch.exp(score - out["lse"][h, rows][:, None])
            del score
            out["o"][h, rows] = p @ v
            if train:
                g = s["d_o"][h, rows].double()
                out["dv"][h * kv // H, cols] += p.T @ g
                p *= g @ v.T - (g * out["o"][h, rows]).sum(1, keepdim=True)
                out["dq"][h, rows] = p @ k / math.sqrt(d)
                out["dk"][h * kv // H, cols] += p.T @ q / math.sqrt(d)
    return out
