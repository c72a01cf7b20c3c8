"""AdamW over many tensors and the gradients' norm against the definitions in 64 bits.

Bounds.  m is a sum of two products, each factor and the sum rounded to float32: at most 5 2^-24 of the absolute terms A = |b1 m| + |(1 - b1) g|; v
likewise 6 2^-24 of itself.  The step's quotient takes those, the two corrections (an exponential's 2 ulp and its argument's rounding), a root, a
division: below 40 2^-24 of A / (c1 den).  The parameter adds two roundings of its own: 4 2^-24 |p|.  A bf16 parameter is rounded once more: U |p|.
States in 8 bits: the code is the lower or the upper neighbour of value / scale, and the one that the hash says, unless the two lie within the
float32 error of that quotient (8 2^-24 of it, against neighbours 2^-3 apart: 2^-15 of a step, and 2^-16 is the random number's own step)."""
import math

import pytest
import torch

from tests import layer_forms as lf

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
E = 2.0 ** -24
MASK = 0xffffffff


def mix(x):
    x = ((x ^ (x >> 16)) * 0x7feb352d) & MASK
    x = ((x ^ (x >> 15)) * 0x846ca68b) & MASK
    return x ^ (x >> 16)


def random_bits(seed, t, blocks):
    step = mix(torch.tensor((seed + 0x9e3779b9 * t) & MASK))
    return mix((mix(blocks ^ step)[:, None] + torch.arange(256)) & MASK)


def definition(p, g, m, v, t, lr, betas, eps, wd, factor=1.0):
    """(p, m, v, absolute terms of m, of the quotient)."""
    b1, b2 = betas
    g = g * factor
    m2, v2 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    den = torch.sqrt(v2 / (1 - b2 ** t)) + eps
    a = b1 * m.abs() + (1 - b1) * g.abs()
    return p - lr * (m2 / (1 - b1 ** t) / den + wd * p), m2, v2, a, a / (1 - b1 ** t) / den


def make(sizes, dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)
    params = [torch.nn.Parameter((0.1 * torch.randn(s, generator=gen)).to(dtype).cuda()) for s in sizes]
    for p in params:
        p.grad = (torch.randn(p.shape, generator=gen) * math.exp(torch.randn((), generator=gen))).to(dtype).cuda()
    return params, gen


SIZES = [(3, 5), (1,), (256,), (255,), (257,), (0,), (40, 33), (8192,), (8193,), (2, 8200), (131, 127), (20000,)]


def run_steps(dtype, bits, masters, steps=3, sizes=SIZES, lr=0.01, betas=(0.9, 0.99), eps=1e-6, wd=0.1):
    from paper_2604_10103_b200 import optim
    params, gen = make(sizes, dtype, bits)
    opt = optim.AdamW(params, lr=lr, betas=betas, eps=eps, weight_decay=wd, state_bits=bits, master_weights=masters, seed=77)
    factor = torch.tensor(0.75, device="cuda")
    for t in range(1, steps + 1):
        before = [{k: x.clone() for k, x in opt.state[p].items()} | dict(p=p.detach().clone()) for p in params]
        opt.step(grad_factor=factor)
        for i, (p, old) in enumerate(zip(params, before)):
            new, g = opt.state[p], lf.f64(p.grad)
            assert int(new["step"]) == t
            if p.numel() == 0:
                continue
            start = lf.f64(old.get("master", old["p"]))
            m, v = lf.f64(old["m"].float()), lf.f64(old["v"].float())
            if bits == 8:
                by = lf.f64(old["scales"]).repeat_interleave(256, dim=0)[:p.numel()]
                m, v = m * by[:, 0].view(p.shape), v * by[:, 1].view(p.shape)
            rp, rm, rv, a, q = definition(start, g, m, v, t, lr, betas, eps, wd, 0.75)
            bound = E * (4 * rp.abs() + 4 * start.abs() + 40 * lr * (q + wd * start.abs()))
            if masters and dtype is BF:
                lf.close(new["master"], rp, bound, f"master {i}")
                assert torch.equal(p.detach(), new["master"].to(BF))
            else:
                lf.close(p, rp, bound + (lf.U[BF] * rp.abs() if dtype is BF else 0.0), f"p {i}")
            if bits == 32:
                lf.close(new["m"], rm, 5 * E * a + 1e-45, f"m {i}")
                lf.close(new["v"], rv, 6 * E * rv + 1e-45, f"v {i}")
                continue
            n = p.numel()
            blocks = torch.arange(-(-n // 256)) + opt._first_block[i]
            r = random_bits(77, t, blocks).view(-1)[:n].view(p.shape)
            scales = lf.f64(new["scales"])
            for k, (ref, err, top, mantissa, lowest, drawn) in enumerate(((rm, 5 * E * a, 448.0, 3, -6, r & 0xffff), (rv, 6 * E * rv, 57344.0, 2, -14, r >> 16))):
                code = lf.f64(new["m" if k == 0 else "v"].float())
                largest = torch.stack([c.abs().max() for c in ref.reshape(-1).split(256)])
                slack = torch.stack([c.max() for c in err.reshape(-1).split(256)])
                want = (largest / top).clamp_min(2.0 ** -126)
                assert ((scales[:, k] - want).abs() <= slack / top + 2 * E * want).all()
                s = scales[:, k].repeat_interleave(256)[:n].view(p.shape)
                y = (ref / s).abs().clamp_max(top)
                apart = 2.0 ** (torch.floor(torch.log2(y.clamp_min(2.0 ** lowest))) - mantissa)
                off = (code.abs() - y).abs() / apart
                least = (y > 0) & (code.abs() == 2.0 ** (lowest - mantissa)) if k else torch.zeros_like(y, dtype=torch.bool)
                assert ((off < 1 + 2.0 ** -15) | least).all()
                assert (code * ref >= 0).all()
                u = y / apart + drawn.double() / 65536
                clear = (u - u.round()).abs() > (err / s + 4 * E * y) / apart + 1e-12
                assert clear.double().mean() > 0.999 or n < 5000
                want = torch.floor(u) * apart
                if k:
                    want = torch.maximum(want, (ref > 0) * 2.0 ** -16)
                assert torch.equal(code.abs()[clear], want[clear])
    return opt


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,masters", [(F32, True), (BF, True), (BF, False)])
def test_steps(dtype, masters, bits):
    run_steps(dtype, bits, masters)


@pytest.mark.parametrize("bits", [32, 8])
def test_more_tensors_than_a_table_holds(bits):
    run_steps(BF, bits, True, steps=2, sizes=[(5 + i % 7, 9) for i in range(700)])


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_parameters_off_16_bytes_and_what_lies_between(bits, dtype):
    from paper_2604_10103_b200 import optim
    flat = torch.full((9000,), 7.0, dtype=dtype, device="cuda")
    grads = torch.randn(9000, device="cuda").to(dtype)
    at = [(1, 300), (302, 8200), (8503, 1)]
    params = [torch.nn.Parameter(flat[a:a + n]) for a, n in at]
    twins = [torch.nn.Parameter(flat[a:a + n].clone()) for a, n in at]
    for (a, n), p, q in zip(at, params, twins):
        p.grad, q.grad = grads[a:a + n], grads[a:a + n].clone()
    kw = dict(lr=0.1, state_bits=bits)
    one, two = optim.AdamW(params, **kw), optim.AdamW(twins, **kw)
    for _ in range(2):
        one.step()
        two.step()
    for p, q in zip(params, twins):
        assert torch.equal(p, q)
    for k in ("m", "v", "scales", "master"):
        assert one.buffers[k] is None or torch.equal(one.buffers[k].view(torch.uint8), two.buffers[k].view(torch.uint8))
    held = torch.ones(9000, dtype=torch.bool, device="cuda")
    for a, n in at:
        held[a:a + n] = False
    assert (flat[held] == 7.0).all()
    for p, q in zip(params, at):
        n = q[1]
        a = one._first_block[[id(x) for x in params].index(id(p))] * 256
        rest = one.buffers["m"][a + n:a + -(-n // 256) * 256].float()
        assert (rest == 0).all()


def test_groups_rates_on_the_device_and_missing_gradients():
    from paper_2604_10103_b200 import optim
    params, _ = make([(300,), (20, 20), (77,)], F32)
    rate = torch.tensor(0.02, device="cuda")
    opt = optim.AdamW([dict(params=params[:1], lr=rate, weight_decay=0.0), dict(params=params[1:], betas=(0.5, 0.9), lr=0.3)], eps=1e-3, weight_decay=0.2)
    missing, params[1].grad = params[1].grad, None
    start = [lf.f64(p) for p in params]
    opt.step()
    assert torch.equal(lf.f64(params[1]), start[1]) and [int(opt.state[p]["step"]) for p in params] == [1, 0, 1]
    z = [torch.zeros_like(s) for s in start]
    for i, (lr, betas, wd) in ((0, (0.02, (0.9, 0.999), 0.0)), (2, (0.3, (0.5, 0.9), 0.2))):
        rp, *_, q = definition(start[i], lf.f64(params[i].grad), z[i], z[i], 1, lr, betas, 1e-3, wd)
        lf.close(params[i], rp, E * (8 * start[i].abs() + 4 * rp.abs() + 42 * lr * (q + wd * start[i].abs())), f"p {i}")
    params[1].grad = missing
    opt.param_groups[1]["lr"] = 0.1
    rate.fill_(0.0)
    first = params[0].detach().clone()
    opt.step()
    assert torch.equal(params[0], first) and [int(opt.state[p]["step"]) for p in params] == [2, 1, 2]
    rp, *_, q = definition(start[1], lf.f64(missing), z[1], z[1], 1, 0.1, (0.5, 0.9), 1e-3, 0.2)
    lf.close(params[1], rp, E * (8 * start[1].abs() + 4 * rp.abs() + 42 * 0.1 * (q + 0.2 * start[1].abs())), "p 1")


@pytest.mark.parametrize("bits", [32, 8])
def test_a_factor_that_is_not_finite_leaves_the_step_out(bits):
    from paper_2604_10103_b200 import optim
    params, _ = make([(3000,), (7, 7)], BF)
    opt = optim.AdamW(params, lr=0.1, state_bits=bits)
    opt.step()
    before = {k: v.clone() for k, v in opt.buffers.items() if v is not None}, [p.detach().clone() for p in params]
    params[0].grad[17] = float("inf")
    norm, factor = optim.gradient_norm([p.grad for p in params], 1.0)
    assert math.isinf(float(norm)) and math.isnan(float(factor))
    opt.step(grad_factor=factor)
    assert all(torch.equal(opt.buffers[k].view(torch.uint8), v.view(torch.uint8)) for k, v in before[0].items())
    assert all(torch.equal(p, q) for p, q in zip(params, before[1]))


def test_values_that_are_not_finite_stay_in_their_block():
    from paper_2604_10103_b200 import optim
    for bits in (32, 8):
        params, _ = make([(1024,)], F32)
        params[0].grad[300] = float("nan")
        params[0].grad[600] = float("-inf")
        opt = optim.AdamW(params, lr=0.1, state_bits=bits)
        opt.step()
        bad = ~torch.isfinite(params[0].detach())
        assert bad.nonzero().view(-1).tolist() == [300, 600]
        opt.step()
        bad = ~torch.isfinite(params[0].detach())
        assert not bad[:256].any() and not bad[768:].any() and bad[300] and bad[600]
        assert (int(bad.sum()) == 2) == (bits == 32)


def test_gradients_of_zero_and_tiny_ones():
    from paper_2604_10103_b200 import optim
    for bits in (32, 8):
        p = torch.nn.Parameter(torch.ones(512, device="cuda"))
        p.grad = torch.zeros(512, device="cuda")
        p.grad[256:] = 1e-21                # (its square leaves float32's normal range)
        opt = optim.AdamW([p], lr=0.1, weight_decay=0.0, state_bits=bits)
        for _ in range(3):
            opt.step()
        assert (p[:256] == 1).all() and torch.isfinite(p).all() and (p[256:] <= 1).all()


def test_the_mean_of_many_roundings_is_right():
    """v and m of constant gradients after many steps, blocks that hold one large value: each element's mean over the block of its error stays within
    6 standard deviations (a step's rounding is at most one spacing, 2^-3 of m and 2^-2 of v, and the later ones halve what the first left)."""
    from paper_2604_10103_b200 import optim
    n = 256 * 64
    p = torch.nn.Parameter(torch.zeros(n, device="cuda"))
    p.grad = torch.full((n,), 0.3, device="cuda")
    p.grad[::256] = 1.0
    opt = optim.AdamW([p], lr=0.0, betas=(0.9, 0.99), state_bits=8)
    for t in range(1, 41):
        opt.step()
    s = opt.state[p]
    small = torch.ones(n, dtype=torch.bool, device="cuda")
    small[::256] = False
    for k, (name, want, apart, beta) in enumerate((("m", 0.3 * (1 - 0.9 ** 40), 2.0 ** -3, 0.9), ("v", 0.09 * (1 - 0.99 ** 40), 2.0 ** -2, 0.99))):
        got = (s[name].float() * s["scales"][:, k].repeat_interleave(256))[small].double()
        # variance of the sum of independent roundings: at most (apart / 2)^2 each (of values up to the final one), weighted by beta^2j
        sd = apart / 2 * want * math.sqrt(sum(beta ** (2 * j) for j in range(40)) / got.numel())
        assert abs(float(got.mean()) - want) < 6 * sd


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_steps_count_and_follow_the_rate(bits):
    from paper_2604_10103_b200 import optim
    one, _ = make([(5000,), (33, 3)], BF)
    two = [torch.nn.Parameter(p.detach().clone()) for p in one]
    for p, q in zip(one, two):
        q.grad = p.grad.clone()
    rates = [torch.tensor(0.1, device="cuda") for _ in range(2)]
    a, b = (optim.AdamW(ps, lr=r, state_bits=bits) for ps, r in zip((one, two), rates))

    def step(ps, opt):
        norm, factor = optim.gradient_norm([p.grad for p in ps], 0.5)
        opt.step(grad_factor=factor)
    step(one, a)
    step(two, b)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(two, b)
    for t in range(4):
        for p, q in zip(one, two):
            fresh = torch.randn_like(p)
            p.grad.copy_(fresh)
            q.grad.copy_(fresh)
        for r in rates:
            r.fill_(0.1 / (t + 1))
        step(one, a)
        g.replay()
    assert all(torch.equal(p, q) for p, q in zip(one, two))
    assert all(torch.equal(a.buffers[k].view(torch.uint8), b.buffers[k].view(torch.uint8)) for k in a.buffers if a.buffers[k] is not None)


def test_two_streams_at_once():
    from paper_2604_10103_b200 import optim
    sets = [make([(40000,), (300, 300)], BF, seed=i)[0] for i in range(2)]
    twins = [[torch.nn.Parameter(p.detach().clone()) for p in ps] for ps in sets]
    for ps, qs in zip(sets, twins):
        for p, q in zip(ps, qs):
            q.grad = p.grad.clone()
    opts = [optim.AdamW(ps, lr=0.1, state_bits=8) for ps in sets]
    refs = [optim.AdamW(ps, lr=0.1, state_bits=8) for ps in twins]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, ps, o in zip(streams, sets, opts):
            with torch.cuda.stream(s):
                _, factor = optim.gradient_norm([p.grad for p in ps], 1.0)
                o.step(grad_factor=factor)
    torch.cuda.synchronize()
    for ps, o in zip(twins, refs):
        for _ in range(10):
            _, factor = optim.gradient_norm([p.grad for p in ps], 1.0)
            o.step(grad_factor=factor)
    assert all(torch.equal(p, q) for ps, qs in zip(sets, twins) for p, q in zip(ps, qs))


@pytest.mark.parametrize("bits", [32, 8])
def test_state_goes_out_and_comes_back(bits, tmp_path):
    from paper_2604_10103_b200 import optim
    params, _ = make([(500,), (3, 400)], BF)
    opt = optim.AdamW(params, lr=0.1, state_bits=bits)
    opt.step()
    torch.save(dict(opt=opt.state_dict(), params=[p.detach() for p in params]), tmp_path / "s.pt")
    opt.step()
    saved = torch.load(tmp_path / "s.pt")
    other = [torch.nn.Parameter(p) for p in saved["params"]]
    for p, q in zip(params, other):
        q.grad = p.grad.clone()
    again = optim.AdamW(other, lr=0.5, state_bits=bits)
    again.load_state_dict(saved["opt"])
    assert again.param_groups[0]["lr"] == 0.1
    again.step()
    assert all(torch.equal(p, q) for p, q in zip(params, other))
    with pytest.raises(ValueError):
        optim.AdamW(other, state_bits=40 - bits).load_state_dict(saved["opt"])
    with pytest.raises(ValueError):
        optim.AdamW(other[:1], state_bits=bits).load_state_dict(saved["opt"])


def test_a_backward_pass_over_a_stepped_parameter_raises():
    from paper_2604_10103_b200 import optim
    params, _ = make([(50,)], F32)
    opt = optim.AdamW(params)
    y = (params[0] * params[0]).sum()
    opt.step()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_a_copy_goes_by_the_state():
    import copy

    from paper_2604_10103_b200 import optim
    params, _ = make([(50,)], F32)
    opt = optim.AdamW(params)
    with pytest.raises(TypeError, match="state_dict"):
        copy.deepcopy(opt)
    with pytest.raises(ValueError, match="construction"):
        opt.add_param_group(dict(params=[torch.nn.Parameter(torch.zeros(3, device="cuda"))]))


def test_what_a_step_refuses():
    from paper_2604_10103_b200 import optim
    params, _ = make([(50,), (4, 6)], F32)
    opt = optim.AdamW(params, lr=0.1)
    before = [p.detach().clone() for p in params]
    for factor in (torch.tensor(1.0), torch.ones(2, device="cuda"), torch.tensor(1.0, device="cuda", dtype=torch.float64)):
        with pytest.raises(ValueError):
            opt.step(grad_factor=factor)
    params[1].grad = torch.randn(6, 4, device="cuda").t()
    with pytest.raises(ValueError, match="gradient"):
        opt.step()
    params[1].grad = None
    params[0].data = torch.zeros(3, device="cuda")
    params[0].grad = torch.zeros(3, device="cuda")
    with pytest.raises(ValueError):
        opt.step()
    assert torch.equal(params[1].detach(), before[1]) and int(opt.state[params[1]]["step"]) == 0
    for bad in (torch.nn.Parameter(torch.zeros(3, device="cuda").half()), torch.nn.Parameter(torch.zeros(4, 6, device="cuda").t())):
        with pytest.raises(ValueError):
            optim.AdamW([bad])
    with pytest.raises(ValueError):
        optim.gradient_norm([torch.zeros(4, 6, device="cuda").t()])
    with pytest.raises(ValueError):
        optim.gradient_norm([torch.zeros(4, device="cuda"), torch.zeros(4)])
    with pytest.raises(ValueError):
        optim.gradient_norm([torch.zeros(4, device="cuda", dtype=torch.float64)])


def test_a_scheduler_drives_it():
    from paper_2604_10103_b200 import optim
    params, _ = make([(50,)], F32)
    opt = optim.AdamW(params, lr=1.0, weight_decay=0.0)
    schedule = torch.optim.lr_scheduler.StepLR(opt, 1, 0.5)
    moves = []
    for _ in range(3):
        old = params[0].detach().clone()
        opt.step()
        schedule.step()
        moves.append(float((params[0].detach() - old).abs().max()))
    # (a constant gradient's quotient is 1 in each step, up to eps and float32)
    assert all(abs(m - want) < 1e-4 for m, want in zip(moves, (1.0, 0.5, 0.25)))


# ------------------------------------------------------------------------------------------------ norm
@pytest.mark.parametrize("sizes", [[1], [0, 3], [255, 257, 1], [4096, 16384, 16385], [3] * 40, [1000] * 1300, [3_000_001, 17]])
@pytest.mark.parametrize("dtype", [F32, BF, torch.float16])
def test_norm(sizes, dtype):
    """Squares of float32 rounded once (E), summed in float32 over at most 64 elements of a thread's chunk (64 E), then in double; a root halves the
    relative error, the result is rounded (E)."""
    from paper_2604_10103_b200 import optim
    g = torch.Generator().manual_seed(sum(sizes))
    ts = [(torch.randn(n, generator=g) * 3).to(dtype).cuda() for n in sizes]
    want = math.sqrt(sum(float(lf.f64(t).square().sum()) for t in ts))
    for most in (float("inf"), 2 * want + 1, 0.5 * want, 0.0):
        norm, factor = optim.gradient_norm(ts, most)
        assert norm.shape == factor.shape == () and abs(float(norm) - want) <= 40 * E * want
        assert abs(float(factor) - (1.0 if want == 0 else min(1.0, most / want))) <= 42 * E
    again, _ = optim.gradient_norm(ts)
    assert torch.equal(norm, again)


def test_norm_off_16_bytes_of_mixed_types_and_of_nothing():
    from paper_2604_10103_b200 import optim
    x = torch.randn(100000, device="cuda")
    ts = [x[1:50000], x.to(BF)[3:], x.half()[1:8], x[:0]]
    want = math.sqrt(sum(float(lf.f64(t).square().sum()) for t in ts))
    assert abs(float(optim.gradient_norm(ts)[0]) - want) <= 40 * E * want
    norm, factor = optim.gradient_norm([x[:0]], 1.0)
    assert float(norm) == 0.0 and float(factor) == 1.0
    norm, factor = optim.gradient_norm([torch.zeros(5, device="cuda")], 0.0)
    assert float(norm) == 0.0 and float(factor) == 1.0
    norm, factor = optim.gradient_norm([torch.full((3,), 1e20, device="cuda")], 1.0)
    assert math.isinf(float(norm)) and math.isnan(float(factor))
    bad = torch.ones(5000, device="cuda")
    bad[4321] = float("nan")
    assert math.isnan(float(optim.gradient_norm([bad], 1.0)[1]))
