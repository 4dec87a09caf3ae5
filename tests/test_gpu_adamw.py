"""AdamW over many tensors (moments in fp32 and in 8 bits) and the norm of many gradients, against the formulas in 64 bits."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS32 = 2.0 ** -24                                  # half a step of fp32, relative
HYPER = dict(lr=2e-3, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)

# lengths around the kernel's 8, 128, 2048 and 4096 elements; a list longer than one launch's table is test_many
LENGTHS = [1, 7, 8, 127, 128, 129, 1000, 2048, 4095, 4096, 4097, 12345]


def _tensors(lengths, grad_dtype, seed, odd=False):
    """One long buffer's views, at odd places (element by element) or at multiples of 128."""
    g = torch.Generator().manual_seed(seed)
    out = {}
    for name, dtype in (("p", torch.float32), ("g", grad_dtype), ("m", torch.float32), ("v", torch.float32)):
        views = []
        for n in lengths:
            x = torch.randn(n, generator=g) * 10.0 ** torch.randint(-4, 1, (n,), generator=g).float()
            x = x.abs() if name == "v" else x
            buf = torch.zeros(n + 128, dtype=dtype, device=DEV)
            views.append(buf[1:n + 1] if odd else buf[:n])
            views[-1].copy_(x.to(dtype))
        out[name] = views
    out["step"] = torch.tensor([3], dtype=torch.int32, device=DEV)
    return out


def _formula(p, g, m, v, t, lr, betas, eps, weight_decay, scale=1.0):
    """One step in 64 bits (numpy), betas as the fp32 numbers that the call takes."""
    b1, b2 = (float(np.float32(b)) for b in betas)
    lr, eps, wd = (float(np.float32(x)) for x in (lr, eps, weight_decay))
    g = g * scale
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    move = m / (1 - b1 ** t) / (np.sqrt(v / (1 - b2 ** t)) + eps)
    return p - lr * (move + wd * p), m, v, move


def _np(ts):
    return [t.double().cpu().numpy() for t in ts]


def _close(got, want, allow, what):
    err = np.abs(got - want)
    worst = float((err / allow).max()) if err.size else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3g} x the allowance"


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("odd", [False, True])
def test_steps_with_fp32_moments(grad, odd):
    import paper_1511_08486_amd as sfb
    x = _tensors(LENGTHS, grad, 1, odd)
    copies = [torch.zeros_like(p, dtype=torch.bfloat16) for p in x["p"]]
    opt = sfb.AdamW(x["p"], x["g"], x["m"], x["v"], x["step"], copies=copies)
    for t in (4, 5):
        p0, g0, m0, v0 = (_np(x[k]) for k in "pgmv")
        opt.step(**HYPER)
        opt.sync()
        for i, n in enumerate(LENGTHS):
            p, m, v, move = _formula(p0[i], g0[i], m0[i], v0[i], t, **HYPER)
            # m: two products and a sum; v: three products and a sum (all positive)
            _close(x["m"][i].double().cpu().numpy(), m, 3 * EPS32 * (np.abs(m0[i]) + np.abs(g0[i])) + 1e-44, f"m of {n}")
            _close(x["v"][i].double().cpu().numpy(), v, 5 * EPS32 * v + 1e-44, f"v of {n}")
            # p: its own rounding, and a dozen roundings of the move, whose numerator may have cancelled
            allow = 2 * EPS32 * np.abs(p) + HYPER["lr"] * 16 * EPS32 * (np.abs(move) * (np.abs(m0[i]) + np.abs(g0[i])) / np.maximum(np.abs(m), 1e-30) + np.abs(p))
            _close(x["p"][i].double().cpu().numpy(), p, allow, f"p of {n}")
            assert torch.equal(copies[i], x["p"][i].to(torch.bfloat16))
        assert int(x["step"]) == t


def test_first_step_moves_by_the_rate():
    """From zero moments m / (1 - b1) = g and v / (1 - b2) = g^2: every element moves by lr, whatever its gradient's size."""
    import paper_1511_08486_amd as sfb
    g = torch.tensor([1e-3, -5.0, 2e4, 0.0, -1e-6], device=DEV)
    p = torch.zeros(5, device=DEV)
    m, v = torch.zeros_like(p), torch.zeros_like(p)
    step = torch.zeros(1, dtype=torch.int32, device=DEV)
    opt = sfb.AdamW([p], [g], [m], [v], step)
    opt.step(lr=0.5, betas=(0.9, 0.999), eps=0.0 + 1e-30, weight_decay=0.0)
    opt.sync()
    want = torch.tensor([-0.5, 0.5, -0.5, 0.0, 0.5])
    # a dozen roundings; 1 - b2 as fp32 differences: the factors' own rounding, 2^-24 of numbers near 1, over 0.001
    assert torch.allclose(p.cpu(), want, rtol=2e-4, atol=0), p
    assert int(step) == 1


def test_many_tensors_are_what_one_by_one_gives():
    """More tensors than one launch's table holds, empty ones among them, equal the same call on each alone."""
    import paper_1511_08486_amd as sfb
    lengths = [(37 * i) % 300 for i in range(150)]
    x = _tensors(lengths, torch.float32, 5)
    want = []
    for i in range(len(lengths)):
        y = {k: [x[k][i].clone()] for k in "pgmv"}
        step = x["step"].clone()
        o = sfb.AdamW(y["p"], y["g"], y["m"], y["v"], step)
        o.step(**HYPER)
        o.sync()
        want.append((y["p"][0], y["m"][0], y["v"][0]))
    opt = sfb.AdamW(x["p"], x["g"], x["m"], x["v"], x["step"])
    opt.step(**HYPER)
    opt.sync()
    for i in range(len(lengths)):
        for a, b in zip((x["p"][i], x["m"][i], x["v"][i]), want[i]):
            assert torch.equal(a, b), i
    assert int(x["step"]) == 4


def _values(codes, scales, second):
    """What 8-bit moments stand for, by the header's definition (numpy, 64 bits)."""
    table = np.zeros(256)
    for c in range(256):
        e, f = (c >> 3) & (31 if second else 15), c & 7
        bias = 15 if second else 7
        v = math.ldexp(f, -2 - bias) if e == 0 else math.ldexp(8 + f, e - 3 - bias)
        table[c] = v if second else math.copysign(v, -1.0 if c & 128 else 1.0)
    c, s = codes.cpu().numpy(), scales.cpu().numpy().astype(np.float64)
    return table[c] * np.repeat(np.exp2(s - 127.0), 128)[:len(c)]


def _state8(lengths):
    z = lambda n: torch.zeros(n, dtype=torch.uint8, device=DEV)  # noqa: E731
    return ([z(n) for n in lengths], [z(n) for n in lengths], [z((n + 127) // 128) for n in lengths], [z((n + 127) // 128) for n in lengths])


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("odd", [False, True])
def test_steps_with_moments_in_8_bits(grad, odd):
    import paper_1511_08486_amd as sfb
    x = _tensors(LENGTHS, grad, 2, odd)
    x["step"].zero_()
    m8, v8, ms, vs = _state8(LENGTHS)
    opt = sfb.AdamW(x["p"], x["g"], m8, v8, x["step"], m_scales=ms, v_scales=vs)
    outs = [[torch.full((n,), 7.0, dtype=torch.bfloat16, device=DEV) for n in LENGTHS] for _ in range(2)]
    for t in (1, 2, 3):
        p0, g0 = _np(x["p"]), _np(x["g"])
        m0 = [_values(a, b, False) for a, b in zip(m8, ms)]
        v0 = [_values(a, b, True) for a, b in zip(v8, vs)]
        opt.step(**HYPER, seed=11)
        opt.unpack(*outs)
        opt.sync()
        for i, n in enumerate(LENGTHS):
            p, m, v, move = _formula(p0[i], g0[i], m0[i], v0[i], t, **HYPER)
            allow = 2 * EPS32 * np.abs(p) + HYPER["lr"] * 16 * EPS32 * (np.abs(move) * (np.abs(m0[i]) + np.abs(g0[i])) / np.maximum(np.abs(m), 1e-30) + np.abs(p))
            _close(x["p"][i].double().cpu().numpy(), p, allow, f"p of {n}")         # by the moments before rounding
            got_m, got_v = _values(m8[i], ms[i], False), _values(v8[i], vs[i], True)
            top = lambda z: np.repeat([np.abs(z[k:k + 128]).max() for k in range(0, n, 128)], 128)[:n]  # noqa: E731
            # one step of the code: an eighth (of the binade's lower end), or the smallest code (2^-9 and 2^-17 of the scale,
            # which is 2^-7 and 2^-14 of the block's largest power of two at least); the random part may land just over a whole code
            _close(got_m, m, np.abs(m) / 8 * (1 + 1e-4) + top(m) * 2.0 ** -16 * (1 + 1e-4) + 1e-30, f"m of {n}")
            _close(got_v, v, np.abs(v) / 8 * (1 + 1e-4) + top(v) * 2.0 ** -31 * (1 + 1e-4) + 1e-30, f"v of {n}")
            assert ((got_v > 0) == (v > 0)).all()
            assert (outs[0][i].double().cpu().numpy() == got_m).all() and (outs[1][i].double().cpu().numpy() == got_v).all()


def test_rounding_to_8_bits_keeps_the_mean():
    """What is rounded at random averages to what was rounded: with b1 = 0.5 and zero moments m = g / 2, v = g^2 / 2."""
    import paper_1511_08486_amd as sfb
    n, steps = 1 << 16, 8
    for value in (0.7, 0.0131, 1.0):
        sums = np.zeros(2)
        for seed in range(steps):
            p, g = torch.zeros(n, device=DEV), torch.full((n,), value, device=DEV)
            g[::128] = 1.0                                                # the block's largest
            m8, v8, ms, vs = _state8([n])
            step = torch.zeros(1, dtype=torch.int32, device=DEV)
            opt = sfb.AdamW([p], [g], m8, v8, step, m_scales=ms, v_scales=vs)
            opt.step(lr=0.0, betas=(0.5, 0.5), seed=seed)
            opt.sync()
            keep = np.arange(n) % 128 != 0
            sums += [_values(m8[0], ms[0], False)[keep].mean(), _values(v8[0], vs[0], True)[keep].mean()]
        want = np.array([0.5 * value, 0.5 * value * value])
        # n draws of at most a code's distance (an eighth): six deviations, and 2^-16 of a code for the 16 bits
        allow = want / 8 * (6 * 0.5 / math.sqrt(n * steps) + 2.0 ** -16) + want * 1e-6
        assert (np.abs(sums / steps - want) <= allow).all(), (value, sums / steps, want)


def test_second_moment_follows_gradients_that_vanish():
    """(1 - b2) of v is far below a code's distance; the drawn rounding follows the decay all the same."""
    import paper_1511_08486_amd as sfb
    n, steps = 8192, 400
    p, g = torch.zeros(n, device=DEV), torch.ones(n, device=DEV)
    m8, v8, ms, vs = _state8([n])
    step = torch.zeros(1, dtype=torch.int32, device=DEV)
    opt = sfb.AdamW([p], [g], m8, v8, step, m_scales=ms, v_scales=vs)
    opt.step(lr=0.0, betas=(0.9, 0.5))
    g.zero_()
    for _ in range(steps):
        opt.step(lr=0.0, betas=(0.9, 0.995))
    opt.sync()
    got, want = _values(v8[0], vs[0], True).mean(), 0.5 * 0.995 ** steps
    # each step's rounding adds at most (code distance d = v / 8)^2 f (1 - f) <= (v^2 / 64) 0.04 of variance, 400 of them: a deviation
    # below 0.5 of v for one element, 0.5 / sqrt(8192) = 0.0055 for the mean: six of them
    assert abs(got / want - 1.0) < 0.033, (got, want)


def test_values_that_are_not_finite_stay_apart():
    """A NaN or an infinity in a gradient spoils its own element only, in both kinds of state."""
    import paper_1511_08486_amd as sfb
    n = 400
    for bits in (32, 8):
        p, g = torch.zeros(n, device=DEV), torch.full((n,), 0.25, device=DEV)
        g[5], g[200], g[399] = float("nan"), float("inf"), float("-inf")
        step = torch.zeros(1, dtype=torch.int32, device=DEV)
        m8, v8, ms, vs = _state8([n])
        if bits == 8:
            opt = sfb.AdamW([p], [g], m8, v8, step, m_scales=ms, v_scales=vs)
        else:
            opt = sfb.AdamW([p], [g], [torch.zeros(n, device=DEV)], [torch.zeros(n, device=DEV)], step)
        opt.step(lr=0.5, weight_decay=0.0)
        out = [torch.zeros(n, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        if bits == 8:
            opt.unpack([out[0]], [out[1]])
        opt.sync()
        bad = torch.zeros(n, dtype=torch.bool)
        bad[[5, 200, 399]] = True
        assert torch.equal(torch.isnan(p.cpu()), bad)
        assert torch.allclose(p.cpu()[~bad], torch.tensor(-0.5), rtol=2e-4)
        if bits == 8:
            assert torch.equal(torch.isnan(out[0].float().cpu()), bad) and torch.equal(torch.isnan(out[1].float().cpu()), bad)


def test_scale_rate_and_skip_on_the_device():
    import paper_1511_08486_amd as sfb
    x = _tensors([1000], torch.float32, 9)
    p0, g0, m0, v0 = (_np(x[k])[0] for k in "pgmv")
    opt = sfb.AdamW(x["p"], x["g"], x["m"], x["v"], x["step"])
    scale = torch.tensor([float("nan")], device=DEV)
    before = [x[k][0].clone() for k in "pmv"]
    opt.step(**HYPER, grad_scale=scale)
    opt.sync()
    assert int(x["step"]) == 3 and all(torch.equal(a, x[k][0]) for a, k in zip(before, "pmv"))
    scale.fill_(0.25)
    rate = torch.tensor([0.5], device=DEV)
    opt.step(**HYPER, grad_scale=scale, lr_scale=rate)
    opt.sync()
    want = _formula(p0, g0, m0, v0, 4, HYPER["lr"] * 0.5, HYPER["betas"], HYPER["eps"], HYPER["weight_decay"], 0.25)
    assert np.allclose(x["p"][0].cpu().numpy(), want[0], rtol=1e-5, atol=1e-7)
    assert np.allclose(x["v"][0].cpu().numpy(), want[2], rtol=5 * EPS32, atol=1e-40)


def test_step_recorded_in_a_graph_counts_on():
    """A replayed call takes the next step each time (the counter is on the device), draws anew, and follows rate and factor there."""
    import paper_1511_08486_amd as sfb
    side = torch.cuda.Stream(device=DEV)
    with torch.cuda.stream(side):
        runs = []
        for _ in range(2):
            x = _tensors([3000, 129, 5], torch.bfloat16, 21)
            x["step"].zero_()
            m8, v8, ms, vs = _state8([3000, 129, 5])
            out = torch.zeros(2, device=DEV)
            opt = sfb.AdamW(x["p"], x["g"], m8, v8, x["step"], m_scales=ms, v_scales=vs)
            norm = sfb.GradNorm(x["g"])
            runs.append((x, m8, v8, ms, vs, out, opt, norm))
        side.synchronize()

    def go(r):
        r[7](0.5, r[5])
        r[6].step(**HYPER, seed=3, grad_scale=r[5][1:])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        go(runs[1])
    scratch = torch.zeros(1 << 16, device=DEV)
    for _ in range(4):
        with torch.cuda.stream(side):
            go(runs[0])
        graph.replay()
        torch.cuda.synchronize()
        a, b = runs
        assert torch.equal(a[5], b[5]) and int(a[0]["step"]) == int(b[0]["step"])
        for i in range(3):
            for u, w in ((a[0]["p"], b[0]["p"]), (a[1], b[1]), (a[2], b[2]), (a[3], b[3]), (a[4], b[4])):
                assert torch.equal(u[i], w[i])
        scratch.add_(1.0)
        torch.cuda.synchronize()
    assert int(runs[0][0]["step"]) == 4


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lengths", [[1], [16384], [16385, 0, 3], [5] * 300, [100000, 1, 70001]])
def test_norm_of_many_gradients(dtype, lengths):
    import paper_1511_08486_amd as sfb
    x = _tensors(lengths, dtype, 4, odd=len(lengths) == 3)
    out = torch.zeros(2, device=DEV)
    norm = sfb.GradNorm(x["g"])
    want = math.sqrt(sum(float((g ** 2).sum()) for g in _np(x["g"])))
    for limit in (want * 3, want / 7, math.inf):
        norm(limit, out)
        norm.sync()
        assert abs(float(out[0]) - want) <= 2 * EPS32 * want
        assert abs(float(out[1]) - min(1.0, float(np.float32(limit)) / want)) <= 3 * EPS32


def test_norm_of_extreme_gradients():
    import paper_1511_08486_amd as sfb
    out = torch.zeros(2, device=DEV)
    big = torch.full((1000,), 1e30, device=DEV)                         # squares beyond fp32
    sfb.GradNorm([big])(1.0, out)
    torch.cuda.synchronize()
    assert abs(float(out[0]) / (float(np.float32(1e30)) * math.sqrt(1000)) - 1) < 1e-6 and 0 < float(out[1]) < 1e-30
    sfb.GradNorm([torch.zeros(10, device=DEV)])(1.0, out)
    torch.cuda.synchronize()
    assert out.tolist() == [0.0, 1.0]
    for bad in (float("nan"), float("inf")):
        big[500] = bad
        sfb.GradNorm([big])(1.0, out)
        torch.cuda.synchronize()
        assert math.isnan(float(out[1])) and not math.isfinite(float(out[0]))
    sfb.GradNorm([])(1.0, out)
    torch.cuda.synchronize()
    assert out.tolist() == [0.0, 1.0]


def test_lists_that_do_not_fit_are_refused():
    import paper_1511_08486_amd as sfb
    x = _tensors([10, 20], torch.float32, 1)
    args = lambda **kw: dict(dict(params=x["p"], grads=x["g"], m=x["m"], v=x["v"], step=x["step"]), **kw)  # noqa: E731
    for bad in (dict(grads=x["g"][:1]), dict(m=[t.bfloat16() for t in x["m"]]), dict(v=[x["v"][1], x["v"][0]]), dict(step=x["step"].float()),
                dict(params=[t.cpu() for t in x["p"]]), dict(m_scales=[torch.zeros(1, dtype=torch.uint8, device=DEV)] * 2),
                dict(grads=[x["g"][0], x["g"][1].bfloat16()]), dict(copies=x["p"])):
        with pytest.raises(ValueError):
            sfb.AdamW(**args(**bad))
    opt = sfb.AdamW(**args())
    with pytest.raises(ValueError):
        opt.unpack(x["p"], x["p"])
    for bad in (dict(lr=-1.0), dict(lr=math.nan), dict(lr=1e-3, betas=(1.0, 0.9)), dict(lr=1e-3, betas=(0.9, -0.1)), dict(lr=1e-3, eps=math.inf)):
        with pytest.raises(sfb.SfbError):
            opt.step(**bad)
    opt.sync()
    assert int(x["step"]) == 3


def test_elements_beyond_32_bit_offsets():
    """One tensor of 2^31 + 5000 elements, its norm and its step: the formulas at both ends."""
    import paper_1511_08486_amd as sfb
    n = (1 << 31) + 5000
    p, m, v = (torch.zeros(n, device=DEV) for _ in range(3))
    g = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    p.add_(0.5)
    ends = [slice(0, 3000), slice(n - 3000, n)]
    for e in ends:
        g[e].normal_(generator=torch.Generator(device=DEV).manual_seed(1))
    step, out = torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros(2, device=DEV)
    sfb.GradNorm([g])(1.0, out)
    opt = sfb.AdamW([p], [g], [m], [v], step)
    opt.step(**HYPER, grad_scale=out[1:])
    opt.sync()
    want = math.sqrt(sum(float((g[e].double() ** 2).sum()) for e in ends))
    assert abs(float(out[0]) - want) <= 2 * EPS32 * want
    for e in ends:
        x = g[e].double().cpu().numpy()
        w, wm, wv, _ = _formula(np.full(3000, 0.5), x, 0.0 * x, 0.0 * x, 1, scale=float(out[1]), **HYPER)
        _close(p[e].double().cpu().numpy(), w, 4 * EPS32 + HYPER["lr"] * 16 * EPS32 + 0 * w, "p")
        _close(m[e].double().cpu().numpy(), wm, 4 * EPS32 * np.abs(wm) + 1e-44, "m")
        _close(v[e].double().cpu().numpy(), wv, 6 * EPS32 * wv + 1e-44, "v")
    middle = p[n // 2:n // 2 + 1000]
    assert torch.allclose(middle, torch.full_like(middle, 0.5 * (1 - HYPER["lr"] * HYPER["weight_decay"])), rtol=1e-6)
