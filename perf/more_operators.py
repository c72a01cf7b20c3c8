"""Timed cases of what a denoiser block with biases and its training step need: linear layers with their epilogue, q/k norms with the rotation,
the gradients' norm, the optimizer.

A case is a plain dict; `op` and `direction` name the call:

  linear  y = residual + gate * act(x W^T + b) over the rows of x; gate: one row for each group of `group` rows (a modulation, one per latent
          frame); `save` also returns x W^T + b for the backward pass.  backward: from dy (and the saved sums) dx, dW, db, dgate
  heads   the rows of a fused projection [batch, tokens, (heads + 2 kv_heads) * head_dim] -> q, k, v [batch, heads, tokens, head_dim], q and k
          scaled by 1 / rms (over a head, or over all heads of the token) and a weight, then rotated by the token's position in time, height and
          width.  backward: dq, dk, dv and the rows -> the gradient of the rows, of both weights
  norm    the 2-norm of many gradients together, and the factor that brings it to `most` at most
  adamw   one step of AdamW over many tensors: states in 32 bits, or in 8 (m in e4m3, v in e5m2, a scale for each 256 elements, rounded up or down
          at random, from a hash of seed, step and place)

Where `own` is false `run` is the plain form; where it is true, the calls of `paper_2604_10103_b200`.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

# the 832x480 layer of the repository's workloads: 12 heads of 128, a latent frame of 30 x 52 tokens, chunks of 3 frames
HEADS, DIM, HIGH, WIDE, CHUNK = 12, 128, 30, 52, 3
FRAME, WIDTH = HIGH * WIDE, HEADS * DIM
CLIP = 21 * FRAME           # a training clip: 21 latent frames
HIDDEN = 4 * WIDTH          # a feed-forward of two matrices
BLOCK = 256                 # elements that share a scale; tensors start at multiples of it in the flat buffers
LARGEST_STEP = 4 * 28_400_000       # elements of the largest step


def _linear(name, direction, rows, width, out, **kw):
    return dict(dict(op="linear", direction=direction, type="bf16", rows=rows, width=width, out=out, bias=True, act="none", group=0, residual=False,
                     save=False), name=name, **kw)


def _heads(name, direction, frames, high, wide, **kw):
    return dict(dict(op="heads", direction=direction, type="bf16", batch=1, frames=frames, high=high, wide=wide, heads=HEADS, kv_heads=HEADS,
                     head_dim=DIM, over="width", pairing="adjacent", eps=1e-6), name=name, **kw)


def _step(op, name, layers, width, hidden, **kw):
    more = dict(most=1.0) if op == "norm" else dict(bits=32, master=True, lr=1e-4, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.01)
    return dict(dict(op=op, direction="forward", type="bf16", layers=layers, width=width, hidden=hidden, **more), name=name, **kw)


def listed():
    return [
        # the modulation of a block from one time embedding: a single row, six rows of output
        _linear("linear_one_row", "forward", 1, WIDTH, 6 * WIDTH, act="silu"),
        # a prompt's tokens (odd, less than a tile) in float16 through the feed-forward's first matrix, its sums kept for the backward pass
        _linear("linear_prompt_saved", "forward", 77, WIDTH, HIDDEN, type="f16", act="gelu_tanh", save=True),
        # the feed-forward's second matrix for a chunk, with the gate per frame and the residual stream
        _linear("linear_chunk_gated", "forward", CHUNK * FRAME, HIDDEN, WIDTH, group=FRAME, residual=True),
        # the feed-forward's first matrix for a training clip, backward
        _linear("linear_clip_backward", "backward", CLIP, WIDTH, HIDDEN, act="gelu_tanh"),
        # norms of each head, shared key heads, a small odd picture in float32: a call whose time is its launch
        _heads("heads_small_odd", "forward", 1, 7, 9, heads=8, kv_heads=2, head_dim=64, type="f32", over="head", pairing="halves"),
        # one layer of one denoising step at 832x480: a chunk's projections to the tensors the hybrid attention reads
        _heads("heads_chunk", "forward", CHUNK, HIGH, WIDE),
        # the same for a training clip, backward
        _heads("heads_clip_backward", "backward", 21, HIGH, WIDE),
        # all gradients of a small model in float32; of one layer of the 832x480 model
        _step("norm", "norm_small", 2, 128, 512, type="f32"),
        _step("norm", "norm_layer", 1, WIDTH, HIDDEN),
        # a step of the small model: many small tensors, a call whose time is its launch
        _step("adamw", "adamw_small", 2, 128, 512, type="f32", master=False),
        # four layers of the 832x480 model, states and master weights in float32
        _step("adamw", "adamw_layers", 4, WIDTH, HIDDEN),
        # two layers of it, states in 8 bits
        _step("adamw", "adamw_layers_8bit", 2, WIDTH, HIDDEN, bits=8),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "heads", "norm", "adamw"])
    direction = rng.choice(["forward", "backward"])
    if op == "linear":
        case = dict(op=op, direction=direction, type=rng.choice(["bf16", "bf16", "bf16", "f16"]), rows=_spread(rng, 1, CLIP),
                    width=8 * _spread(rng, 8, 768), out=8 * _spread(rng, 8, 1152), bias=rng.random() < 0.8, act=rng.choice(["none", "silu", "gelu_tanh"]),
                    group=0, residual=rng.random() < 0.5, save=direction == "forward" and rng.random() < 0.4)
        while case["rows"] * case["width"] * case["out"] > CLIP * WIDTH * HIDDEN:
            case["rows"] //= 2
        if rng.random() < 0.5:
            case["group"] = max(1, case["rows"] // rng.randint(1, 8))
        return case
    if op == "heads":
        heads, dim = rng.choice([(2, 64), (5, 64), (12, 128), (12, 64), (16, 128), (24, 128), (10, 96)])
        case = dict(op=op, direction=direction, type=rng.choice(["bf16", "bf16", "f16", "f32"]), batch=rng.choice([1, 1, 2]),
                    frames=_spread(rng, 1, 21), high=_spread(rng, 1, 45), wide=_spread(rng, 1, 80), heads=heads,
                    kv_heads=heads if heads % 4 or rng.random() < 0.6 else heads // 4, head_dim=dim, over=rng.choice(["width", "head"]),
                    pairing=rng.choice(["adjacent", "adjacent", "halves"]), eps=rng.choice([1e-6, 1e-5]))
        while case["batch"] * case["frames"] * case["high"] * case["wide"] * heads * dim > CLIP * WIDTH // 2:
            case["frames"], case["high"] = max(1, case["frames"] // 2), max(1, case["high"] // 2)
        return case
    width = 8 * _spread(rng, 8, 256)
    case = dict(op=op, direction="forward", type=rng.choice(["bf16", "bf16", "f32"]), layers=rng.randint(1, 12), width=width, hidden=width * rng.randint(2, 4))
    while case["layers"] > 1 and case["layers"] * width * (4 * width + 2 * case["hidden"]) > LARGEST_STEP // 2:
        case["layers"] -= 1
    if op == "norm":
        return dict(case, most=rng.choice([0.1, 1.0, 10.0]))
    bits = rng.choice([32, 8])
    return dict(case, bits=bits, master=case["type"] == "bf16" and rng.random() < 0.7, lr=rng.choice([1e-3, 1e-4, 2e-5]), beta1=0.9,
                beta2=rng.choice([0.99, 0.999]), eps=1e-8, decay=rng.choice([0.0, 0.01, 0.1]))


def _pairs(head_dim):
    n = head_dim // 2                   # a third each for height and width, the rest for time
    return (n - 2 * (n // 3), n // 3, n // 3)


def _shapes(case):
    """The parameters of a block, layer after layer: matrices and vectors."""
    w, h = case["width"], case["hidden"]
    return [(3 * w, w), (3 * w,), (w, w), (w,), (h, w), (h,), (w, h), (w,), (w,), (w,), (6, w)] * case["layers"]


def _places(shapes):
    """Where each tensor starts in a flat buffer, and the buffer's length."""
    starts, at = [], 0
    for shape in shapes:
        starts.append(at)
        at += -(-math.prod(shape) // BLOCK) * BLOCK
    return starts, at


def _views(flat, shapes):
    return [flat[a:a + math.prod(shape)].view(shape) for a, shape in zip(_places(shapes)[0], shapes)]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 2654435761 % (1 << 62) + 29)
    t = TYPES[case["type"]]

    def normal(*shape, scale=1.0, shift=0.0, dtype=t):
        return torch.randn(shape, generator=g, device="cuda").mul_(scale).add_(shift).to(dtype)

    s = dict(case)
    if case["op"] == "linear":
        M, K, N, group = case["rows"], case["width"], case["out"], case["group"]
        s["x"], s["w"] = normal(M, K), normal(N, K, scale=1.0 / math.sqrt(K))
        s["b"] = normal(N, scale=0.3) if case["bias"] else None
        # a slice of one modulation tensor: the gate beside the block's five others
        s["gate"] = normal(-(-M // group), 6, N, scale=0.5)[:, 2] if group else None
        if case["direction"] == "forward":
            s["res"] = normal(M, N) if case["residual"] else None
        else:
            pre = s["x"].float() @ s["w"].float().t()
            s["pre"] = (pre if s["b"] is None else pre + s["b"].float()).to(t) if case["act"] != "none" or group else None
            s["dy"] = normal(M, N)
        return s
    if case["op"] == "heads":
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
        # projections with heads of different size
        size = torch.exp(0.5 * torch.randn(H + 2 * KV, 1, generator=g, device="cuda")).expand(-1, d).reshape(-1)
        s["rows_in"] = (torch.randn(B, T, (H + 2 * KV) * d, generator=g, device="cuda") * size).to(t)
        n = 1 if case["over"] == "head" else H
        s["qw"], s["kw"] = normal(n * d, scale=0.2, shift=1.0), normal((1 if case["over"] == "head" else KV) * d, scale=0.2, shift=1.0)
        if case["direction"] == "backward":
            s["dq"], s["dk"], s["dv"] = normal(B, H, T, d), normal(B, KV, T, d), normal(B, KV, T, d)
        return s
    shapes = _shapes(case)
    starts, n = _places(shapes)
    inside = torch.zeros(n // BLOCK, BLOCK, dtype=torch.bool, device="cuda")            # (what lies between two tensors is 0 and stays 0)
    for view in _views(inside.view(-1), shapes):
        view.fill_(True)
    # gradients of different size from tensor to tensor and from element to element, a few far out
    size = torch.exp(torch.randn(n // BLOCK, 1, generator=g, device="cuda") - 6.0)
    grad = (torch.randn(n // BLOCK, BLOCK, generator=g, device="cuda") * size * inside)
    s["grad"], s["shapes"] = grad.to(t).view(-1), shapes
    s["grads"] = _views(s["grad"], shapes)
    if case["op"] == "norm":
        return s
    s["t"] = 10                         # steps taken before
    p = torch.randn(n // BLOCK, BLOCK, generator=g, device="cuda") * 0.02 * inside
    s["p"] = p.to(t).view(-1)
    s["master"] = p.view(-1) if case["master"] else None
    m = (0.3 * grad + 0.3 * size * torch.randn(n // BLOCK, BLOCK, generator=g, device="cuda")) * inside
    v = (0.01 * size * size * (0.1 + torch.rand(n // BLOCK, BLOCK, generator=g, device="cuda"))) * inside
    if case["bits"] == 8:
        ms, vs = (m.abs().amax(1, keepdim=True) / 448.0).clamp_min(2.0 ** -126), (v.amax(1, keepdim=True) / 57344.0).clamp_min(2.0 ** -126)
        s["m"], s["v"] = (m / ms).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(-1), (v / vs).clamp(0.0, 57344.0).to(torch.float8_e5m2).view(-1)
        s["scales"] = torch.cat([ms, vs], dim=1).contiguous()
    else:
        s["m"], s["v"], s["scales"] = m.view(-1), v.view(-1), None
    s["factor"] = torch.rand((), generator=g, device="cuda") * 0.5 + 0.5
    s["decay_of"] = torch.zeros(n // BLOCK, 1, device="cuda")                           # matrices decay, vectors do not
    for a, shape in zip(starts, shapes):
        if len(shape) > 1:
            s["decay_of"][a // BLOCK:(a + math.prod(shape) + BLOCK - 1) // BLOCK] = case["decay"]
    s["seed"] = int(seed) & 0x7fffffff
    if own:                             # the optimizer that a training program keeps, in the middle of its training
        from paper_2604_10103_b200 import optim
        params = [torch.nn.Parameter(view) for view in _views(s["p"], shapes)]
        for q, grad_of in zip(params, s["grads"]):
            q.grad = grad_of
        groups = [dict(params=[q], weight_decay=case["decay"] if q.dim() > 1 else 0.0) for q in params]
        s["opt"] = optim.AdamW(groups, lr=case["lr"], betas=(case["beta1"], case["beta2"]), eps=case["eps"], state_bits=case["bits"],
                               master_weights=case["master"], seed=s["seed"])
        for name in ("master", "m", "v", "scales"):
            if s[name] is not None:
                s["opt"].buffers[name].copy_(s[name])
                s[name] = s["opt"].buffers[name]
        s["opt"].buffers["steps"].fill_(s["t"])
    return s


# ------------------------------------------------------------------------------------------------ plain forms
GELU_A, GELU_B = math.sqrt(2.0 / math.pi), 0.044715


def _act(g, name):
    """The activation and its derivative."""
    if name == "none":
        return g, torch.ones_like(g)
    if name == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return g * p, p * (1.0 + g * (1.0 - p))
    # 0.5 (1 + tanh v) = 1 / (1 + exp(-2 v))
    p = 1.0 / (1.0 + torch.exp(-2.0 * GELU_A * (g + GELU_B * g * g * g)))
    return g * p, p + g * p * (1.0 - p) * 2.0 * GELU_A * (1.0 + 3.0 * GELU_B * g * g)


def _by_rows(s):
    """One row of the gate for each row of x."""
    return s["gate"].float().repeat_interleave(s["group"], dim=0)[:s["rows"]]


def _group_sums(v, s):
    groups = -(-s["rows"] // s["group"])
    full = torch.zeros(groups * s["group"], v.shape[1], device=v.device, dtype=v.dtype)
    full[:s["rows"]] = v
    return full.view(groups, s["group"], -1).sum(1)


def _linear_forward(s):
    t = s["x"].dtype
    pre = s["x"].float() @ s["w"].float().t()
    if s["b"] is not None:
        pre = pre + s["b"].float()
    y = _act(pre, s["act"])[0]
    if s["gate"] is not None:
        y = y * _by_rows(s)
    if s["res"] is not None:
        y = y + s["res"].float()
    return (y.to(t), pre.to(t)) if s["save"] else y.to(t)


def _linear_backward(s):
    t, dp, dgate = s["x"].dtype, s["dy"].float(), None
    if s["pre"] is not None:
        a, da = _act(s["pre"].float(), s["act"])
        if s["gate"] is not None:
            dgate = _group_sums((dp * a).double(), s).float()
            dp = dp * _by_rows(s)
        dp = dp * da
    db = dp.double().sum(0).float() if s["b"] is not None else None
    return (dp @ s["w"].float()).to(t), (dp.t() @ s["x"].float()).to(t), db, dgate


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


def _mean(v, over):
    return v.mean((-2, -1) if over == "width" else -1, keepdim=True)


def _heads_forward(s):
    B, T = s["rows_in"].shape[:2]
    H, KV, d, t = s["heads"], s["kv_heads"], s["head_dim"], s["rows_in"].dtype
    cos, sin = _angles(s)
    x = s["rows_in"].view(B, T, H + 2 * KV, d).float()
    q, k, v = x[:, :, :H], x[:, :, H:H + KV], x[:, :, H + KV:]
    q = q / torch.sqrt(_mean(q * q, s["over"]) + s["eps"]) * s["qw"].float().view(-1, d)
    k = k / torch.sqrt(_mean(k * k, s["over"]) + s["eps"]) * s["kw"].float().view(-1, d)
    return tuple(p.transpose(1, 2).to(t).contiguous() for p in (_turn(q, cos, sin, s["pairing"]), _turn(k, cos, sin, s["pairing"]), v))


def _heads_part_backward(x, dy, w, s):
    r = 1.0 / torch.sqrt(_mean(x * x, s["over"]) + s["eps"])
    xh, gw = x * r, dy * w.float().view(-1, x.shape[-1])
    dw = (dy * xh).double().sum((0, 1) if s["over"] == "width" else (0, 1, 2)).float()
    return r * (gw - xh * _mean(gw * xh, s["over"])), dw.reshape(-1)


def _heads_backward(s):
    B, T = s["rows_in"].shape[:2]
    H, KV, d = s["heads"], s["kv_heads"], s["head_dim"]
    cos, sin = _angles(s)
    x = s["rows_in"].view(B, T, H + 2 * KV, d)
    dq, dk = _turn(s["dq"].transpose(1, 2).float(), cos, -sin, s["pairing"]), _turn(s["dk"].transpose(1, 2).float(), cos, -sin, s["pairing"])
    dq, dqw = _heads_part_backward(x[:, :, :H].float(), dq, s["qw"], s)
    dk, dkw = _heads_part_backward(x[:, :, H:H + KV].float(), dk, s["kw"], s)
    return torch.cat([dq, dk, s["dv"].transpose(1, 2).float()], dim=2).flatten(2).to(s["dq"].dtype), dqw, dkw


def _norm(s):
    norm = s["grad"].double().square().sum().sqrt()
    return norm.float(), torch.clamp(s["most"] / norm, max=1.0).float()


MASK = 0xffffffff


def _mix(x):
    """A mix of 32 bits (held in 64)."""
    x = ((x ^ (x >> 16)) * 0x7feb352d) & MASK
    x = ((x ^ (x >> 15)) * 0x846ca68b) & MASK
    return x ^ (x >> 16)


def _random(s, n, t):
    """32 bits for each element: of the seed, the step and the element's place in the flat buffer."""
    step = _mix(torch.full((), (s["seed"] + 0x9e3779b9 * t) & MASK, dtype=torch.int64, device="cuda"))
    return _mix((_mix(torch.arange(n // BLOCK, device="cuda") ^ step)[:, None] + torch.arange(BLOCK, device="cuda")) & MASK)


def _up_or_down(y, bits16, drop, least):
    """y >= 0 with the last `drop` bits of its float32 mantissa rounded away (of numbers below `least` as if they were next to it): up with
    the probability of what is cut off."""
    small = y < least
    z = torch.where(small, y + least, y)
    z = ((z.view(torch.int32) + (bits16 << (drop - 16)).int()) & -(1 << drop)).view(torch.float32)
    return torch.where(small, z - least, z)


def _adamw(s):
    s["t"] += 1
    t, b1, b2, bits8 = s["t"], s["beta1"], s["beta2"], s["bits"] == 8
    g = s["grad"].float().view(-1, BLOCK) * s["factor"]
    p = (s["p"] if s["master"] is None else s["master"]).float().view(-1, BLOCK)
    m, v = s["m"].float().view(-1, BLOCK), s["v"].float().view(-1, BLOCK)
    if bits8:
        m, v = m * s["scales"][:, :1], v * s["scales"][:, 1:]
    m = b1 * m + (1.0 - b1) * g
    v = b2 * v + (1.0 - b2) * g * g
    step = (m / (1.0 - b1 ** t)) / (torch.sqrt(v / (1.0 - b2 ** t)) + s["eps"])
    p = p - s["lr"] * (step + s["decay_of"] * p)
    if bits8:
        r = _random(s, p.numel(), t)
        ms = (m.abs().amax(1, keepdim=True) / 448.0).clamp_min(2.0 ** -126)
        vs = (v.amax(1, keepdim=True) / 57344.0).clamp_min(2.0 ** -126)
        y = torch.copysign(_up_or_down((m.abs() / ms).clamp_max(448.0), r & 0xffff, 20, 2.0 ** -6), m)
        z = _up_or_down((v / vs).clamp_max(57344.0), r >> 16, 21, 2.0 ** -14)
        z = torch.where(v > 0.0, z.clamp_min(2.0 ** -16), z)                # (a second moment that is there does not become 0)
        m, v = y, z
        s["scales"].copy_(torch.cat([ms, vs], dim=1))
    s["m"].copy_(m.view(-1))
    s["v"].copy_(v.view(-1))
    s["p"].copy_(p.view(-1))
    if s["master"] is not None:
        s["master"].copy_(p.view(-1))
    return s["p"], s["master"], s["m"], s["v"], s["scales"]


# ------------------------------------------------------------------------------------------------ the library's calls
def _run_own(s):
    from paper_2604_10103_b200 import layers, optim
    forward = s["direction"] == "forward"
    if s["op"] == "linear":
        act = None if s["act"] == "none" else s["act"]
        if forward:
            return layers.linear(s["x"], s["w"], s["b"], act=act, gate=s["gate"], residual=s["res"], rows_per_group=s["group"], save=s["save"])
        return layers.linear_backward(s["dy"], s["x"], s["w"], s["pre"], act=act, gate=s["gate"], rows_per_group=s["group"], dbias=s["b"] is not None)
    if s["op"] == "heads":
        how = dict(eps=s["eps"], over=s["over"], pairing=s["pairing"])
        if forward:
            return layers.split_heads_norm_rope(s["rows_in"], s["heads"], s["kv_heads"], s["qw"], s["kw"], s["pos"], s["tables"], **how)
        return layers.split_heads_norm_rope_backward(s["dq"], s["dk"], s["dv"], s["rows_in"], s["qw"], s["kw"], s["pos"], s["tables"], **how)
    if s["op"] == "norm":
        return optim.gradient_norm(s["grads"], s["most"])
    s["opt"].step(grad_factor=s["factor"])
    return s["p"], s["master"], s["m"], s["v"], s["scales"]


def run(state):
    if own:
        return _run_own(state)
    return {("linear", "forward"): _linear_forward, ("linear", "backward"): _linear_backward, ("heads", "forward"): _heads_forward,
            ("heads", "backward"): _heads_backward, ("norm", "forward"): _norm, ("adamw", "forward"): _adamw}[state["op"], state["direction"]](state)


def work(case):
    e = 4 if case["type"] == "f32" else 2
    forward = case["direction"] == "forward"
    if case["op"] == "linear":
        M, K, N = case["rows"], case["width"], case["out"]
        G = -(-M // case["group"]) if case["group"] else 0
        params = N * K + (N if case["bias"] else 0) + G * N
        if forward:             # x, W, b, gate, residual -> y (and the sums)
            return {"bytes": e * (M * K + params + M * N * (1 + case["residual"] + case["save"])), "flops": 2 * M * N * K}
        saved = case["act"] != "none" or case["group"] > 0
        return {"bytes": e * (2 * M * K + 2 * N * K + G * N + M * N * (1 + saved)) + 4 * N * (G + case["bias"]), "flops": 4 * M * N * K}
    if case["op"] == "heads":
        T, H, KV, d = case["frames"] * case["high"] * case["wide"], case["heads"], case["kv_heads"], case["head_dim"]
        rows = case["batch"] * T * d
        if forward:
            return {"bytes": 2 * rows * (H + 2 * KV) * e + 12 * T, "flops": 7 * rows * (H + KV)}
        return {"bytes": rows * (2 * (H + 2 * KV) + H + KV) * e + 12 * T, "flops": 16 * rows * (H + KV)}      # dq, dk, dv, q's and k's rows -> rows
    n = sum(math.prod(shape) for shape in _shapes(case))
    if case["op"] == "norm":
        return {"bytes": n * e, "flops": 2 * n}
    state = 16.0 if case["bits"] == 32 else 4.0 + 16.0 / BLOCK
    return {"bytes": n * (e + (8 + e if case["master"] else 2 * e) + state), "flops": 20 * n}


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """From the definitions in float64: gradients by differentiating them, rotations as products of complex numbers, states in 8 bits as multiples
    of the distance between their neighbours."""
    s = prepare(case, seed)
    forward = case["direction"] == "forward"
    F = torch.nn.functional
    if case["op"] == "linear":
        act = {"none": lambda a: a, "silu": F.silu, "gelu_tanh": lambda a: F.gelu(a, approximate="tanh")}[case["act"]]
        x, w = s["x"].double(), s["w"].double()
        b, gate = None if s["b"] is None else s["b"].double(), None if s["gate"] is None else s["gate"].double()
        of = torch.arange(case["rows"], device="cuda") // case["group"] if case["group"] else None
        if forward:
            pre = F.linear(x, w, b)
            y = act(pre)
            if gate is not None:
                y.mul_(gate[of])
            if s["res"] is not None:
                y.add_(s["res"].double())
            return (y, pre) if case["save"] else y
        dy = s["dy"].double()
        if s["pre"] is None:
            return dy.matmul(w), torch.einsum("mn,mk->nk", dy, x), None if b is None else torch.einsum("mn->n", dy), None
        with torch.enable_grad():
            pre = s["pre"].double().requires_grad_()
            out, wrt = act(pre), [pre]
            if gate is not None:
                wrt.append(gate.requires_grad_())
                out = out * gate[of]
            dp, *dgate = torch.autograd.grad(out, wrt, dy)
        return dp.matmul(w), torch.einsum("mn,mk->nk", dp, x), None if b is None else torch.einsum("mn->n", dp), dgate[0] if dgate else None
    if case["op"] == "heads":
        cos, sin, extents, pairs = s["tables"]
        starts = [sum(e * n for e, n in zip(extents[:a], pairs[:a])) for a in range(3)]
        z = torch.complex(cos.double(), sin.double())
        unit = torch.cat([z[o:o + e * n].view(e, n)[s["pos"][..., a].long()] for a, (o, e, n) in enumerate(zip(starts, extents, pairs))], dim=-1)   # [1, T, d/2]
        adjacent, H, KV, d = case["pairing"] == "adjacent", case["heads"], case["kv_heads"], case["head_dim"]

        def made(x, w):         # [B, h, T, d]
            square = x.square().mean(-1, keepdim=True)
            if case["over"] == "width":
                square = square.mean(1, keepdim=True)
            x = x * (square + case["eps"]) ** -0.5 * w.view(-1, 1, d)
            v = x.unflatten(-1, (-1, 2) if adjacent else (2, -1)).movedim(-1 if adjacent else -2, -1).contiguous()
            r = torch.view_as_real(torch.view_as_complex(v) * unit[:, None])
            return (r if adjacent else r.movedim(-1, -2)).flatten(-2)

        x = s["rows_in"].double().unflatten(-1, (-1, d)).movedim(2, 1)
        q, k, v = x.split([H, KV, KV], dim=1)
        qw, kw = s["qw"].double(), s["kw"].double()
        if forward:
            return made(q, qw), made(k, kw), v
        with torch.enable_grad():
            q, k, qw, kw = (a.detach().clone().requires_grad_() for a in (q, k, qw, kw))
            dq, dqw = torch.autograd.grad(made(q, qw), (q, qw), s["dq"].double())
            dk, dkw = torch.autograd.grad(made(k, kw), (k, kw), s["dk"].double())
        return torch.cat([dq, dk, s["dv"].double()], dim=1).movedim(1, 2).flatten(2), dqw, dkw
    if case["op"] == "norm":
        norm = torch.linalg.vector_norm(s["grad"].double())
        return norm, torch.minimum(case["most"] / norm, torch.ones_like(norm))
    t, b1, b2 = s["t"] + 1, case["beta1"], case["beta2"]
    p = (s["p"] if s["master"] is None else s["master"]).double()
    g, m, v = s["grad"].double().mul_(s["factor"].double()), s["m"].double(), s["v"].double()
    if case["bits"] == 8:
        m, v = (q.view(-1, BLOCK).mul(s["scales"][:, i, None].double()).view(-1) for i, q in enumerate((m, v)))
    m.lerp_(g, 1.0 - b1)
    v.lerp_(g.square(), 1.0 - b2)
    decay = s["decay_of"].double().expand(-1, BLOCK).reshape(-1)
    p = p * (1.0 - case["lr"] * decay) - (case["lr"] / (1.0 - b1 ** t)) * m / (v.sqrt() * (1.0 - b2 ** t) ** -0.5 + case["eps"])
    scales = None
    if case["bits"] == 8:
        scales = torch.stack([m.view(-1, BLOCK).abs().amax(1) / 448.0, v.view(-1, BLOCK).amax(1) / 57344.0], dim=1).clamp_min(2.0 ** -126)
        r = _random(s, p.numel(), t)

        def rounded(y, bits16, mantissa, lowest):
            apart = torch.exp2(y.clamp_min(2.0 ** lowest).log2().floor() - mantissa)
            return torch.floor(y / apart + bits16.double() / 65536.0) * apart
        y, z = (m.view(-1, BLOCK) / scales[:, :1]).clamp(-448.0, 448.0), (v.view(-1, BLOCK) / scales[:, 1:]).clamp_max(57344.0)
        m = (y.sign() * rounded(y.abs(), r & 0xffff, 3, -6)).view(-1)
        v = torch.maximum(rounded(z, r >> 16, 2, -14), (z > 0.0) * 2.0 ** -16).view(-1)
    return p, None if s["master"] is None else p, m, v, scales
