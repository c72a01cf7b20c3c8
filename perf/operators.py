"""Timed cases of the operators of a denoiser block around the hybrid attention: layer norm, rotary positions with several axes, gated
feed-forward.

A case is a plain dict; `op` and `direction` name the call:

  norm  y = (x - mean) * rstd * (offset + w) + b over the rows of x [rows, width]; w, b one row for all rows, or one for each
        group of `group` rows (a denoiser's modulation, one scale and shift per latent frame).  backward: dx, dw, db
  rope  the rows of a fused projection [batch, tokens, (heads + 2 kv_heads) * head_dim] -> q, k, v [batch, heads, tokens, head_dim], q and k
        rotated by their positions in time, height and width.  backward: dq, dk, dv -> the gradient of the rows
  ff    y = (act(x Wg^T) * (x Wu^T)) Wd^T; `save` also returns the two projections for the backward pass.  backward: from dy and
        the saved projections dx, dWg, dWu, dWd

Where `own` is false `run` is the plain form in 32 bits; where it is true, the calls of `paper_2604_10103_b200.layers`.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

# the 832x480 layer of the repository's workloads: 12 heads of 128, a latent frame of 30 x 52 tokens, chunks of 3 frames
HEADS, DIM, HIGH, WIDE, CHUNK = 12, 128, 30, 52, 3
FRAME, WIDTH = HIGH * WIDE, HEADS * DIM
CLIP = 21 * FRAME           # a training clip: 21 latent frames
HIDDEN = 4096               # about 8/3 of the width: a gated block has three matrices


def _norm(name, direction, rows, width, **kw):
    return dict(dict(op="norm", direction=direction, type="bf16", rows=rows, width=width, group=0, offset=0.0, eps=1e-6), name=name, **kw)


def _rope(name, direction, frames, high, wide, **kw):
    return dict(dict(op="rope", direction=direction, type="bf16", batch=1, frames=frames, high=high, wide=wide, heads=HEADS, kv_heads=HEADS,
                     head_dim=DIM, pairing="adjacent"), name=name, **kw)


def _ff(name, direction, rows, **kw):
    return dict(dict(op="ff", direction=direction, type="bf16", rows=rows, width=WIDTH, hidden=HIDDEN, act="silu", save=False), name=name, **kw)


def listed():
    return [
        # the `tiny` workload's chunk (one 8x8 frame, two heads of 64): a call whose time is its launch
        _rope("rope_tiny", "forward", 1, 8, 8, heads=2, kv_heads=2, head_dim=64),
        # one layer of one denoising step at 832x480: a chunk's projections to the tensors the hybrid attention reads
        _rope("rope_chunk_832x480", "forward", CHUNK, HIGH, WIDE),
        # the same for a whole training clip, backward
        _rope("rope_clip_backward", "backward", 21, HIGH, WIDE),
        # the modulated norm before attention and feed-forward: scale and shift per latent frame of the chunk
        _norm("norm_chunk_modulated", "forward", CHUNK * FRAME, WIDTH, group=FRAME, offset=1.0),
        # a short sequence of conditioning vectors in float32, odd in both sizes, backward
        _norm("norm_short_odd_backward", "backward", 333, 1027, type="f32"),
        # a training clip's norm, backward: dx and the weight's and bias's gradient over 32760 rows
        _norm("norm_clip_backward", "backward", CLIP, WIDTH),
        # feed-forward of a single token: the weights are read once
        _ff("ff_one_token", "forward", 1),
        # a prompt's tokens (odd, less than one row tile) in float16
        _ff("ff_77_tokens", "forward", 77, type="f16", act="gelu_tanh"),
        # one latent frame, with the projections kept for the backward pass
        _ff("ff_frame_saved", "forward", FRAME, save=True),
        # one denoising step's chunk
        _ff("ff_chunk", "forward", CHUNK * FRAME),
        # the step with gradient of the training rollout: one chunk, backward
        _ff("ff_chunk_backward", "backward", CHUNK * FRAME),
        # a training clip, backward
        _ff("ff_clip_backward", "backward", CLIP),
    ]


def _spread(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n if n != 3 << 10 else n + 1


def draw(rng):
    op = rng.choice(["norm", "rope", "ff", "ff"])
    direction = rng.choice(["forward", "backward"])
    if op == "norm":
        rows = _spread(rng, 1, CLIP)
        modulated = rng.random() < 0.5
        width = _spread(rng, 32, 8192)
        while rows * width > CLIP * WIDTH:
            rows = max(1, rows // 2)
        return dict(op=op, direction=direction, type=rng.choice(["bf16", "bf16", "f16", "f32"]), rows=rows, width=width,
                    group=max(1, rows // rng.randint(1, 8)) if modulated else 0, offset=1.0 if modulated else 0.0, eps=1e-6)
    if op == "rope":
        heads, dim = rng.choice([(2, 64), (5, 64), (12, 128), (12, 64), (16, 128), (24, 128), (10, 96)])
        case = dict(op=op, direction=direction, type=rng.choice(["bf16", "bf16", "f16", "f32"]), batch=rng.choice([1, 1, 2]),
                    frames=_spread(rng, 1, 21), high=_spread(rng, 1, 45), wide=_spread(rng, 1, 80), heads=heads,
                    kv_heads=heads if heads % 4 or rng.random() < 0.6 else heads // 4, head_dim=dim, pairing=rng.choice(["adjacent", "adjacent", "halves"]))
        while case["batch"] * case["frames"] * case["high"] * case["wide"] * heads * dim > CLIP * WIDTH // 2:
            case["frames"], case["high"] = max(1, case["frames"] // 2), max(1, case["high"] // 2)
        return case
    case = dict(op=op, direction=direction, type=rng.choice(["bf16", "bf16", "bf16", "f16"]), rows=_spread(rng, 1, CLIP),
                width=8 * rng.choice([64, 81, 96, 128, 160, 192, 256]), hidden=8 * _spread(rng, 32, 1024), act=rng.choice(["silu", "silu", "gelu_tanh"]),
                save=direction == "forward" and rng.random() < 0.4)
    if case["hidden"] == 3 << 10:
        case["hidden"] += 8
    while case["rows"] * case["hidden"] * case["width"] > CLIP * HIDDEN * WIDTH:
        case["rows"] //= 2
    return case


def _pairs(head_dim):
    n = head_dim // 2                   # a third each for height and width, the rest for time
    return (n - 2 * (n // 3), n // 3, n // 3)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 2654435761 % (1 << 62) + 17)
    t = TYPES[case["type"]]

    def normal(*shape, scale=1.0, shift=0.0, dtype=t):
        return torch.randn(shape, generator=g, device="cuda").mul_(scale).add_(shift).to(dtype)

    s = dict(case)
    if case["op"] == "norm":
        rows, width, group = case["rows"], case["width"], case["group"]
        groups = -(-rows // group) if group else 1
        # activations of a residual stream: channels of different size, a mean of their own in each row
        s["x"] = (torch.randn(rows, width, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(width, generator=g, device="cuda"))
                  + 0.3 * torch.randn(rows, 1, generator=g, device="cuda")).to(t)
        if group:               # slices of one modulation tensor: scale and shift beside the block's four others
            m = normal(groups, 6, width, scale=0.3)
            s["w"], s["b"] = m[:, 1], m[:, 0]
        else:
            s["w"], s["b"] = normal(1, width, scale=0.2, shift=1.0), normal(1, width, scale=0.2)
        if case["direction"] == "backward":
            xf = s["x"].float()
            s["mean"] = xf.mean(1)
            s["rstd"] = 1.0 / torch.sqrt((xf - s["mean"][:, None]).square().mean(1) + case["eps"])
            s["dy"] = normal(rows, width)
    elif case["op"] == "rope":
        B, F, Y, X, H, KV, d = (case[k] for k in ("batch", "frames", "high", "wide", "heads", "kv_heads", "head_dim"))
        T, pairs = F * Y * X, _pairs(d)
        start = torch.randint(0, 200, (1,), generator=g, device="cuda")          # where in the stream the chunk stands
        grid = torch.meshgrid(torch.arange(F, device="cuda") + start, torch.arange(Y, device="cuda"), torch.arange(X, device="cuda"), indexing="ij")
        s["pos"] = torch.stack([p.reshape(-1) for p in grid], dim=1).to(torch.int32)[None].contiguous()         # [1, T, 3]
        extents = (256, 64, 96)
        tabs = [torch.arange(e, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(n, dtype=torch.float64) / n) for e, n in zip(extents, pairs)]
        angles = torch.cat([a.reshape(-1) for a in tabs])
        s["tables"] = (angles.cos().float().cuda(), angles.sin().float().cuda(), extents, pairs)
        # where pair p of the plain form finds its table: axis, first entry, entries in a row
        axis = torch.repeat_interleave(torch.arange(3), torch.tensor(pairs))
        first = torch.tensor([sum(e * n for e, n in zip(extents[:a], pairs[:a])) - sum(pairs[:a]) for a in range(3)])
        s["axis"], s["first"], s["row"] = axis.cuda(), (first[axis] + torch.arange(d // 2)).cuda(), torch.tensor(pairs)[axis].cuda()
        if case["direction"] == "forward":
            s["rows_in"] = normal(B, T, (H + 2 * KV) * d)
        else:
            s["dq"], s["dk"], s["dv"] = normal(B, H, T, d), normal(B, KV, T, d), normal(B, KV, T, d)
    else:
        M, K, N = case["rows"], case["width"], case["hidden"]
        s["x"] = normal(M, K)
        s["wg"], s["wu"] = normal(N, K, scale=1.5 / math.sqrt(K)), normal(N, K, scale=1.0 / math.sqrt(K))
        s["wd"] = normal(K, N, scale=1.0 / math.sqrt(N))
        if case["direction"] == "backward":
            xf = s["x"].float()
            s["gate"], s["up"] = (xf @ s["wg"].float().t()).to(t), (xf @ s["wu"].float().t()).to(t)
            s["dy"] = normal(M, K)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _by_rows(p, s):
    """One row of the parameter for each row of x."""
    return p.float() if not s["group"] else p.float().repeat_interleave(s["group"], dim=0)[:s["rows"]]


def _group_sums(v, s):
    if not s["group"]:
        return v.sum(0, keepdim=True)
    groups = -(-s["rows"] // s["group"])
    full = torch.zeros(groups * s["group"], v.shape[1], device=v.device)
    full[:s["rows"]] = v
    return full.view(groups, s["group"], -1).sum(1)


def _norm_forward(s):
    x = s["x"].float()
    mean = x.mean(1)
    xc = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((xc * xc).mean(1) + s["eps"])
    y = xc * rstd[:, None] * (_by_rows(s["w"], s) + s["offset"]) + _by_rows(s["b"], s)
    return y.to(s["x"].dtype), mean, rstd


def _norm_backward(s):
    xhat = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    dy = s["dy"].float()
    gh = dy * (_by_rows(s["w"], s) + s["offset"])
    dx = s["rstd"][:, None] * (gh - gh.mean(1, keepdim=True) - xhat * (gh * xhat).mean(1, keepdim=True))
    return dx.to(s["x"].dtype), _group_sums(dy * xhat, s), _group_sums(dy, s)


def _turn(x, cos, sin, pairing):
    """x [B, T, H, d] by the angles [., T, d/2]."""
    if pairing == "adjacent":
        x0, x1 = x[..., 0::2], x[..., 1::2]
        return torch.stack([x0 * cos - x1 * sin, x0 * sin + x1 * cos], dim=-1).flatten(-2)
    x0, x1 = x.chunk(2, dim=-1)
    return torch.cat([x0 * cos - x1 * sin, x0 * sin + x1 * cos], dim=-1)


def _angles(s):
    at = s["first"] + s["pos"].long()[..., s["axis"]] * s["row"]
    return s["tables"][0][at][:, :, None], s["tables"][1][at][:, :, None]


def _rope_forward(s):
    B, T = s["rows_in"].shape[:2]
    H, KV, d, t = s["heads"], s["kv_heads"], s["head_dim"], s["rows_in"].dtype
    cos, sin = _angles(s)
    x = s["rows_in"].view(B, T, H + 2 * KV, d).float()
    q, k, v = x[:, :, :H], x[:, :, H:H + KV], x[:, :, H + KV:]
    return tuple(p.transpose(1, 2).to(t).contiguous() for p in (_turn(q, cos, sin, s["pairing"]), _turn(k, cos, sin, s["pairing"]), v))


def _rope_backward(s):
    cos, sin = _angles(s)
    dq, dk, dv = s["dq"].transpose(1, 2).float(), s["dk"].transpose(1, 2).float(), s["dv"].transpose(1, 2).float()
    return torch.cat([_turn(dq, cos, -sin, s["pairing"]), _turn(dk, cos, -sin, s["pairing"]), dv], dim=2).flatten(2).to(s["dq"].dtype)


GELU_A, GELU_B = math.sqrt(2.0 / math.pi), 0.044715


def _act(g, name):
    """The activation and its derivative."""
    if name == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return g * p, p * (1.0 + g * (1.0 - p))
    # 0.5 (1 + tanh v) = 1 / (1 + exp(-2 v))
    p = 1.0 / (1.0 + torch.exp(-2.0 * GELU_A * (g + GELU_B * g * g * g)))
    return g * p, p + g * p * (1.0 - p) * 2.0 * GELU_A * (1.0 + 3.0 * GELU_B * g * g)


def _ff_forward(s):
    x, t = s["x"].float(), s["x"].dtype
    g, u = x @ s["wg"].float().t(), x @ s["wu"].float().t()
    y = ((_act(g, s["act"])[0] * u) @ s["wd"].float().t()).to(t)
    return (y, g.to(t), u.to(t)) if s["save"] else y


def _ff_backward(s):
    x, t, g, u, dy = s["x"].float(), s["x"].dtype, s["gate"].float(), s["up"].float(), s["dy"].float()
    a, da = _act(g, s["act"])
    dh = dy @ s["wd"].float()
    dg, du = dh * u * da, dh * a
    dx = dg @ s["wg"].float() + du @ s["wu"].float()
    return dx.to(t), (dg.t() @ x).to(t), (du.t() @ x).to(t), (dy.t() @ (a * u)).to(t)


# ------------------------------------------------------------------------------------------------ the library's calls
def _run_own(s):
    from paper_2604_10103_b200 import layers
    forward = s["direction"] == "forward"
    if s["op"] == "norm":
        if forward:
            return layers.layer_norm(s["x"], s["w"], s["b"], eps=s["eps"], weight_offset=s["offset"], rows_per_group=s["group"])
        return layers.layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["w"], weight_offset=s["offset"], rows_per_group=s["group"])
    if s["op"] == "rope":
        if forward:
            return layers.split_heads_rope(s["rows_in"], s["heads"], s["kv_heads"], s["pos"], s["tables"], pairing=s["pairing"])
        return layers.split_heads_rope_backward(s["dq"], s["dk"], s["dv"], s["pos"], s["tables"], pairing=s["pairing"])
    if forward:
        return layers.gated_ff(s["x"], s["wg"], s["wu"], s["wd"], act=s["act"], save=s["save"])
    return layers.gated_ff_backward(s["dy"], s["x"], s["wg"], s["wu"], s["wd"], s["gate"], s["up"], act=s["act"])


def run(state):
    if own:
        return _run_own(state)
    return {("norm", "forward"): _norm_forward, ("norm", "backward"): _norm_backward, ("rope", "forward"): _rope_forward,
            ("rope", "backward"): _rope_backward, ("ff", "forward"): _ff_forward, ("ff", "backward"): _ff_backward}[state["op"], state["direction"]](state)


def work(case):
    e = 4 if case["type"] == "f32" else 2
    forward = case["direction"] == "forward"
    if case["op"] == "norm":
        R, D = case["rows"], case["width"]
        G = -(-R // case["group"]) if case["group"] else 1
        if forward:             # x, w, b -> y, mean, rstd
            return {"bytes": 2 * R * D * e + 2 * G * D * e + 8 * R, "flops": 8 * R * D}
        return {"bytes": 3 * R * D * e + G * D * e + 8 * G * D + 8 * R, "flops": 14 * R * D}         # dy, x, w, mean, rstd -> dx, dw, db
    if case["op"] == "rope":
        T = case["frames"] * case["high"] * case["wide"]
        rows = case["batch"] * T * case["head_dim"]
        return {"bytes": 2 * rows * (case["heads"] + 2 * case["kv_heads"]) * e + 12 * T, "flops": 3 * rows * (case["heads"] + case["kv_heads"])}
    M, K, N = case["rows"], case["width"], case["hidden"]
    if forward:                 # x, three weights -> y (and the two projections)
        return {"bytes": e * (2 * M * K + 3 * N * K + (2 * M * N if case["save"] else 0)), "flops": 6 * M * N * K}
    return {"bytes": e * (3 * M * K + 6 * N * K + 2 * M * N), "flops": 12 * M * N * K}               # dy, x, weights, projections -> dx, dW


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """From the definitions in float64: gradients by differentiating them, rotations as products of complex numbers."""
    s = prepare(case, seed)
    forward = case["direction"] == "forward"
    F = torch.nn.functional
    if case["op"] == "norm":
        x, w, b = s["x"].double(), s["w"].double(), s["b"].double()
        of = torch.arange(case["rows"], device="cuda") // case["group"] if case["group"] else torch.zeros(case["rows"], dtype=torch.long, device="cuda")
        if forward:
            var, mean = torch.var_mean(x, dim=1, correction=0)
            rstd = (var + case["eps"]) ** -0.5
            return ((x - mean[:, None]) * rstd[:, None]) * (case["offset"] + w)[of] + b[of], mean, rstd
        # the saved mean and rstd stand for functions of x: dx by the chain rule through both, at the saved values
        mean, rstd, dy = s["mean"].double()[:, None], s["rstd"].double()[:, None], s["dy"].double()
        up = dy * (case["offset"] + w)[of]
        d_rstd = (up * (x - mean)).sum(1, keepdim=True)
        d_var = -0.5 * rstd ** 3 * d_rstd
        dx = up * rstd - (up * rstd).mean(1, keepdim=True) + 2.0 * d_var * (x - mean) / case["width"]
        dw = torch.zeros_like(w).index_add_(0, of, dy * ((x - mean) * rstd))
        return dx, dw, torch.zeros_like(w).index_add_(0, of, dy)
    if case["op"] == "rope":
        cos, sin, extents, pairs = s["tables"]
        starts = [sum(e * n for e, n in zip(extents[:a], pairs[:a])) for a in range(3)]
        z = torch.complex(cos.double(), sin.double())
        unit = torch.cat([z[o:o + e * n].view(e, n)[s["pos"][..., a].long()] for a, (o, e, n) in enumerate(zip(starts, extents, pairs))], dim=-1)   # [1, T, d/2]
        if not forward:
            unit = unit.conj()
        adjacent = case["pairing"] == "adjacent"

        def turn(x):            # [B, H, T, d]
            v = x.double().unflatten(-1, (-1, 2) if adjacent else (2, -1)).movedim(-1 if adjacent else -2, -1).contiguous()
            r = torch.view_as_real(torch.view_as_complex(v) * unit[:, None])
            return (r if adjacent else r.movedim(-1, -2)).flatten(-2)

        if forward:
            x = s["rows_in"].unflatten(-1, (-1, case["head_dim"])).movedim(2, 1)
            q, k, v = x.split([case["heads"], case["kv_heads"], case["kv_heads"]], dim=1)
            return turn(q), turn(k), v.double()
        return torch.cat([turn(s["dq"]), turn(s["dk"]), s["dv"].double()], dim=1).movedim(1, 2).flatten(2)
    act = F.silu if case["act"] == "silu" else lambda g: F.gelu(g, approximate="tanh")
    x, wg, wu, wd = (s[k].double() for k in ("x", "wg", "wu", "wd"))
    if forward:
        gate, up = F.linear(x, wg), F.linear(x, wu)
        y = F.linear(act(gate) * up, wd)
        return (y, gate, up) if case["save"] else y
    with torch.enable_grad():
        gate, up, wd = s["gate"].double().requires_grad_(), s["up"].double().requires_grad_(), wd.requires_grad_()
        d_gate, d_up, d_wd = torch.autograd.grad(F.linear(act(gate) * up, wd), (gate, up, wd), s["dy"].double())
    return d_gate.matmul(wg) + d_up.matmul(wu), torch.einsum("mn,mk->nk", d_gate, x), torch.einsum("mn,mk->nk", d_up, x), d_wd
