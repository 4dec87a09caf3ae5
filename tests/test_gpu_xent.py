"""Softmax cross entropy of a linear head without the scores in memory, and its gradients, against the formulas in 64 bits."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -9, "f32": 2.0 ** -24}       # half a step, relative to the binade's upper end; twice that to its lower end


def _inputs(n, J, D, dtype, w_dtype, seed, spread=2.0, pad=0, offset=0, padded=0.0, sure=1.0):
    g = torch.Generator().manual_seed(seed)

    def place(x, t):
        rows, cols = x.shape
        buf = torch.full((rows * (cols + pad) + offset + 8,), float("nan"), dtype=t, device=DEV)
        view = buf[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
        view.copy_(x)
        return view
    W = torch.randn(J, D, generator=g) * spread / math.sqrt(D)
    y = torch.randint(0, J, (n,), generator=g, dtype=torch.int32)
    lean = torch.rand(n, 1, generator=g) * sure * (math.log(J) + 0.5 * spread ** 2) / spread ** 2
    a = torch.randn(n, D, generator=g) + lean * W[y.long()]
    out = torch.rand(n, generator=g) < padded
    y[out] = torch.where(torch.rand(n, generator=g) < 0.5, -100, J).to(torch.int32)[out]
    a[out] = torch.tensor(float("nan"))              # what stands in rows that take no part is not looked at
    return place(W, TYPES[w_dtype]), place(a, TYPES[dtype]), y.to(DEV)


def _formula(W, a, y, weight=None, scale=1.0, mean=False):
    """64 bits, with what each entry of dA and dW adds up in magnitude, squared and summed."""
    W, a, y = W.double(), a.double(), y.long()
    n, J = a.shape[0], W.shape[0]
    keep = (y >= 0) & (y < J)
    a = torch.where(keep[:, None], a, 0.0)
    z = a @ W.T
    lse = torch.logsumexp(z, 1)
    at = torch.where(keep, y, 0)
    loss = torch.where(keep, lse - z.gather(1, at[:, None])[:, 0], 0.0)
    f = torch.full((n,), float(scale), dtype=torch.float64, device=W.device) * (weight.double() if weight is not None else 1.0)
    if mean:
        f = f / max(1, int(keep.sum()))
    f = torch.where(keep, f, 0.0)
    p = torch.exp(z - lse[:, None])
    u = p.clone()
    u[torch.arange(n), at] -= 1.0
    u, p = u * f[:, None], p * f[:, None].abs()
    zmax = a.abs() @ W.abs().T
    return dict(loss=loss, lse=torch.where(keep, lse, 0.0), total=(f * loss).sum().reshape(1), dA=u @ W, dW=u.T @ a,
                dA_sq=((u * u) @ (W * W)).sqrt(), dW_sq=((u * u).T @ (a * a)).sqrt(), p=p, z_sum=zmax,
                dA_abs=(u.abs() @ W.abs()), dW_abs=(u.abs().T @ a.abs()), p_dA=p @ W.abs(), p_dW=p.T @ a.abs(),
                l_dA=f.abs()[:, None] * W.abs()[at], keep=keep)


def _check(got, want, dtype, w_dtype, D, what):
    """Errors that the arithmetic allows.  A score: products exact (or three bf16 terms, 2^-24 of each left out), D of them added in fp32 in
    blocks: (sqrt(D) + 8) roundings of the sum of magnitudes, as independent ones; six deviations of them at most."""
    ez = 6 * 2.0 ** -24 * (math.sqrt(D) * 0.25 + 4) * float(want["z_sum"].max())
    fine = lambda x: torch.isfinite(x).all()  # noqa: E731
    for k in ("loss", "lse", "total", "dA", "dW"):
        if k in got:
            assert fine(got[k].float()), f"{what}: {k} is not finite"
    if "lse" in got:
        err = (got["lse"].double() - want["lse"]).abs().max()
        assert err <= ez + 4 * 2.0 ** -24 * want["lse"].abs().max() + 1e-6, f"{what}: lse {err:.3g} of {ez:.3g}"
    if "loss" in got:
        err = (got["loss"].double() - want["loss"]).abs().max()
        assert err <= 2 * ez + 8 * 2.0 ** -24 * want["lse"].abs().max() + 1e-6, f"{what}: loss {err:.3g} of {ez:.3g}"
    if "total" in got:
        err, most = (got["total"].double() - want["total"]).abs().max(), (2 * ez + 1e-6) * float(want["p"].sum()) + 2.0 ** -23 * want["total"].abs().max()
        assert err <= most, f"{what}: total {err:.3g} of {most:.3g}"
    both = dtype == "bf16" and w_dtype == "bf16"
    for k, t in (("dA", dtype), ("dW", w_dtype)):
        if k not in got or got[k] is None:
            continue
        x, w = got[k].double(), want[k]
        # the result's rounding; U's (bf16 where both are, else three terms) as independent errors, six deviations and the largest single
        # one; an error ez of the scores moves every p by ez p; sums in fp32
        allow = 2 * HALF[t] * w.abs() + 2.0 ** -22 * 8 * want[k + "_abs"] + 2 * ez * (want["p_" + k] + (want["l_dA"] if k == "dA" else want["dW_abs"]))
        if both:
            allow = allow + 6 * 2 * HALF["bf16"] * want[k + "_sq"]
        elif t == "bf16" and k == "dW":
            allow = allow + 6 * 2.0 ** -17 * want[k + "_abs"]         # second terms' own products left out
        elif t == "bf16":
            # one fp16 term of U and of W, 11 bits each: at most half a step off, 2^-11 of a value, so a product 2^-10 (1 + 2^-12)
            allow = allow + (2.0 ** -10 + 2.0 ** -22) * want[k + "_abs"]
        allow = allow + 1e-30
        worst = float(((x - w).abs() / allow).max())
        assert worst <= 1.0, f"{what}: {k} {worst:.3g} x the allowance"


def _outputs(n, J, D, dtype, w_dtype, pad=0, offset=0, rows_behind=3):
    def mat(r, t):
        buf = torch.full((r * (D + pad) + offset + 8,), 77.0, dtype=TYPES[t], device=DEV)
        return buf[offset:offset + r * (D + pad)].view(r, D + pad)
    vec = lambda: torch.full((n + rows_behind,), 77.0, device=DEV)  # noqa: E731
    return dict(loss=vec(), lse=vec(), total=torch.full((2,), 77.0, device=DEV), dA=mat(n + rows_behind, dtype), dW=mat(J, w_dtype))


def _run(n, J, D, dtype, w_dtype, seed, pad=0, offset=0, out_pad=0, out_offset=0, weighted=False, mean=True, scale=1.0, rows=None, ws=None, two=False, **kw):
    import paper_1511_08486_amd as sfb
    W, a, y = _inputs(n, J, D, dtype, w_dtype, seed, pad=pad, offset=offset, **kw)
    weight = torch.rand(n, generator=torch.Generator().manual_seed(seed + 1)).add_(0.1).to(DEV) if weighted else None
    head = sfb.SoftmaxHead(J, D, rows or n, dtype=dtype, w_dtype=w_dtype)
    if ws:
        head = sfb.SoftmaxHead(J, D, rows or n, dtype=dtype, w_dtype=w_dtype, workspace_bytes=max(head.least_bytes, int(ws * head.best_bytes)))
    head._ws.fill_(255)                              # NaN in every type: nothing may be taken from it that the call has not written
    o = _outputs(n, J, D, dtype, w_dtype, out_pad, out_offset)
    more = dict(weight=weight, scale=scale, mean=mean)
    dA, dW = o["dA"][:n, :D], o["dW"][:, :D]
    if two:
        head.loss(W, a, y, o["loss"][:n], o["lse"][:n], o["total"][:1], **more)
        head._ws.fill_(255)
        head.gradients(W, a, y, o["lse"][:n], dA, dW, **more)
    else:
        head.loss_and_gradients(W, a, y, o["loss"][:n], o["lse"][:n], dA, dW, o["total"][:1], **more)
    head.sync()
    want = _formula(W, a, y, weight, scale, mean)
    got = dict(loss=o["loss"][:n], lse=o["lse"][:n], total=o["total"][:1], dA=dA, dW=dW)
    _check(got, want, dtype, w_dtype, D, f"n {n} J {J} D {D} {dtype}/{w_dtype}")
    keep = want["keep"]
    assert (got["loss"][~keep] == 0).all() and (got["lse"][~keep] == 0).all() and (dA[~keep] == 0).all()
    # what lies behind the rows and columns stays
    assert (o["loss"][n:] == 77).all() and (o["lse"][n:] == 77).all() and o["total"][1] == 77 and (o["dA"][n:] == 77).all()
    assert (o["dA"][:, D:] == 77).all() and (o["dW"][:, D:] == 77).all()
    return got, want


PAIRS = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")]


@pytest.mark.parametrize("dtype,w_dtype", PAIRS)
@pytest.mark.parametrize("n,J,D", [(1, 500, 64), (1, 1, 1), (3, 2, 7), (31, 300, 72), (33, 1000, 128), (64, 257, 200), (65, 511, 65), (130, 1000, 320),
                                   (257, 700, 136), (300, 5000, 256)])
def test_small_and_odd_sizes(n, J, D, dtype, w_dtype):
    _run(n, J, D, dtype, w_dtype, seed=n)


@pytest.mark.parametrize("dtype,w_dtype", PAIRS)
def test_large_tiles(dtype, w_dtype):
    _run(1000, 12345, 520, dtype, w_dtype, seed=3, padded=0.1)


@pytest.mark.parametrize("dtype,w_dtype", PAIRS)
@pytest.mark.parametrize("two", [False, True])
def test_long_features(two, dtype, w_dtype):
    """Few tiles and a long contraction: the scores in slices of D."""
    _run(130, 1001, 1607, dtype, w_dtype, seed=30, padded=0.1, two=two)
    _run(65, 300, 4096, dtype, w_dtype, seed=31, weighted=True, two=two, spread=4.0)


@pytest.mark.parametrize("dtype,w_dtype", PAIRS)
@pytest.mark.parametrize("n,J,D", [(1, 1000, 2048), (40, 5000, 1600), (64, 300, 4096), (33, 70000, 1536)])
def test_few_rows_of_long_features(n, J, D, dtype, w_dtype):
    _run(n, J, D, dtype, w_dtype, seed=32, padded=0.1 if n > 1 else 0.0)
    _run(n, J, D, dtype, w_dtype, seed=32, padded=0.1 if n > 1 else 0.0, two=True)


@pytest.mark.parametrize("dtype,w_dtype", PAIRS)
def test_rows_and_words_of_very_different_size(dtype, w_dtype):
    """Rows of a and of W 2^-20 to 2^20 of their neighbours', scores of ordinary size all the same."""
    import paper_1511_08486_amd as sfb
    n, J, D = 96, 520, 640
    W, a, y = _inputs(n, J, D, dtype, w_dtype, 33)
    W[::3] *= 2.0 ** -20
    W[1::3, :8] *= 2.0 ** 10
    a[::2, :8] *= 2.0 ** -12
    W = torch.where(torch.rand(J, 1, generator=torch.Generator().manual_seed(5)).to(DEV) < 0.1, torch.zeros_like(W), W)
    weight = (2.0 ** torch.randint(-20, 20, (n,), generator=torch.Generator().manual_seed(6)).float()).to(DEV)
    o = dict(loss=torch.empty(n, device=DEV), lse=torch.empty(n, device=DEV), total=torch.empty(1, device=DEV), dA=torch.empty_like(a), dW=torch.empty_like(W))
    head = sfb.SoftmaxHead(J, D, n, dtype=dtype, w_dtype=w_dtype)
    head.loss_and_gradients(W, a, y, **o, weight=weight)
    head.sync()
    _check(o, _formula(W, a, y, weight), dtype, w_dtype, D, f"{dtype}/{w_dtype}")


def test_many_rows():
    _run(3000, 4100, 1032, "bf16", "bf16", seed=4, padded=0.2)


@pytest.mark.parametrize("dtype,w_dtype", PAIRS)
@pytest.mark.parametrize("pad,offset,out_pad,out_offset", [(8, 0, 8, 0), (1, 0, 3, 0), (0, 1, 0, 1), (5, 3, 1, 1)])
def test_strides_and_alignment(pad, offset, out_pad, out_offset, dtype, w_dtype):
    _run(70, 600, 136, dtype, w_dtype, 5, pad=pad, offset=offset, out_pad=out_pad, out_offset=out_offset)


@pytest.mark.parametrize("dtype,w_dtype", PAIRS)
@pytest.mark.parametrize("padded", [0.5, 0.97])
def test_padded_batches_weights_and_scale(padded, dtype, w_dtype):
    _run(200, 900, 192, dtype, w_dtype, 6, padded=padded, weighted=True, scale=3.5)
    _run(200, 900, 192, dtype, w_dtype, 7, padded=padded, mean=False, scale=-0.25)


@pytest.mark.parametrize("dtype,w_dtype", PAIRS)
def test_batches_without_a_row(dtype, w_dtype):
    _run(40, 300, 128, dtype, w_dtype, 8, padded=1.1)
    import paper_1511_08486_amd as sfb
    W, a, y = _inputs(1, 300, 128, dtype, w_dtype, 9)
    head = sfb.SoftmaxHead(300, 128, 16, dtype=dtype, w_dtype=w_dtype)
    dW, total = torch.full((300, 128), 5.0, dtype=TYPES[w_dtype], device=DEV), torch.full((1,), 5.0, device=DEV)
    e = torch.empty(0, device=DEV)
    head.loss_and_gradients(W, a[:0], y[:0], e, e, a[:0].clone(), dW, total, mean=True)
    head.sync()
    assert (dW == 0).all() and float(total) == 0.0


@pytest.mark.parametrize("dtype,w_dtype", PAIRS)
def test_pieces_of_the_vocabulary(dtype, w_dtype):
    """Any workspace from the least on gives the same results (to rounding), whatever it held."""
    for ws in (1e-9, 0.3, 1.0):
        _run(90, 3000, 200, dtype, w_dtype, 10, ws=ws, padded=0.1)


@pytest.mark.parametrize("dtype,w_dtype", PAIRS)
@pytest.mark.parametrize("two", [False, True])
def test_pieces_of_long_features(two, dtype, w_dtype):
    """The same where the scores are kept as long as the workspace holds them, in several pieces of U."""
    for ws in (1e-9, 0.2, 0.35, 0.5, 0.7, 0.9, 1.0):
        _run(150, 3000, 1600, dtype, w_dtype, 18, ws=ws, padded=0.1, two=two)


@pytest.mark.parametrize("dtype,w_dtype", PAIRS)
def test_two_calls_and_fewer_rows_than_the_head_takes(dtype, w_dtype):
    _run(77, 1500, 264, dtype, w_dtype, 11, rows=400, two=True, padded=0.2, weighted=True)


@pytest.mark.parametrize("dtype,w_dtype", PAIRS)
def test_models_that_are_sure_and_scores_that_are_large(dtype, w_dtype):
    _run(60, 700, 128, dtype, w_dtype, 12, spread=1.0, sure=3.0)        # losses of 1e-6 and below
    _run(60, 700, 128, dtype, w_dtype, 13, spread=30.0)                 # scores of +-100


def test_one_output_at_a_time():
    import paper_1511_08486_amd as sfb
    W, a, y = _inputs(50, 800, 128, "bf16", "bf16", 14)
    head = sfb.SoftmaxHead(800, 128, 50)
    full = dict(dA=torch.empty(50, 128, dtype=torch.bfloat16, device=DEV), dW=torch.empty(800, 128, dtype=torch.bfloat16, device=DEV))
    lse = torch.empty(50, device=DEV)
    head.loss_and_gradients(W, a, y, lse=lse, **full)
    for k in full:
        one = torch.empty_like(full[k])
        head.gradients(W, a, y, lse, **{k: one})
        head.sync()
        assert torch.equal(one, full[k])
    loss = torch.empty(50, device=DEV)
    head.loss(W, a, y, loss=loss)
    head.sync()
    assert torch.allclose(loss.double(), _formula(W, a, y)["loss"], atol=1e-4)


def test_results_do_not_depend_on_the_run():
    import paper_1511_08486_amd as sfb
    W, a, y = _inputs(500, 6000, 384, "bf16", "bf16", 15, padded=0.1)
    head = sfb.SoftmaxHead(6000, 384, 500)
    runs = []
    for _ in range(3):
        o = dict(loss=torch.empty(500, device=DEV), lse=torch.empty(500, device=DEV), dA=torch.empty_like(a), dW=torch.empty(6000, 384, dtype=torch.bfloat16, device=DEV),
                 total=torch.empty(1, device=DEV))
        head.loss_and_gradients(W, a, y, **o, mean=True)
        head.sync()
        runs.append(o)
    for r in runs[1:]:
        assert all(torch.equal(r[k], runs[0][k]) for k in r)


def test_gradients_against_differences():
    """(total(W + h V) - total(W - h V)) / 2h = <dW, V>, and the same for a, in fp32."""
    import paper_1511_08486_amd as sfb
    n, J, D = 40, 300, 96
    W, a, y = _inputs(n, J, D, "f32", "f32", 16, padded=0.1, spread=1.0)
    a = torch.nan_to_num(a)
    head = sfb.SoftmaxHead(J, D, n, dtype="f32", w_dtype="f32")
    lse, total = torch.empty(n, device=DEV), torch.empty(1, device=DEV)
    dA, dW = torch.empty(n, D, device=DEV), torch.empty(J, D, device=DEV)
    head.loss_and_gradients(W.contiguous(), a, y, lse=lse, dA=dA, dW=dW, mean=True)
    g = torch.Generator().manual_seed(1)
    for which, grad in (("W", dW), ("a", dA)):
        V = torch.randn(grad.shape, generator=g).to(DEV)
        V = V * grad.abs().mean() + grad                                 # a direction with a slope
        h = 0.02 / float(V.abs().max())
        ends = []
        for s in (h, -h):
            head.loss(W + s * V if which == "W" else W.contiguous(), a + s * V if which == "a" else a, y, total=total, mean=True)
            head.sync()
            ends.append(float(total))
        slope, want = (ends[0] - ends[1]) / (2 * h), float((grad.double() * V.double()).sum())
        # total's rounding over 2h, and the third derivative: at most (h |V a|)^2 of the slope
        move = h * float((V @ a.T if which == "W" else V @ W.T).abs().max())
        assert abs(slope - want) <= 8 * 2.0 ** -24 * abs(ends[0]) / h + move ** 2 * float((grad.abs() * V.abs()).sum()), (which, slope, want)


def test_recorded_in_a_graph():
    import paper_1511_08486_amd as sfb
    side = torch.cuda.Stream(device=DEV)
    W, a, y = _inputs(100, 2000, 256, "bf16", "bf16", 17, padded=0.2)
    a = torch.nan_to_num(a)
    torch.cuda.synchronize()

    def outs():
        return dict(loss=torch.zeros(100, device=DEV), lse=torch.zeros(100, device=DEV), dA=torch.zeros_like(a),
                    dW=torch.zeros(2000, 256, dtype=torch.bfloat16, device=DEV), total=torch.zeros(1, device=DEV))
    with torch.cuda.stream(side):
        eager, taken = sfb.SoftmaxHead(2000, 256, 100), sfb.SoftmaxHead(2000, 256, 100)
        e, t = outs(), outs()
        side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        taken.loss_and_gradients(W, a, y, **t, mean=True)
    scratch = torch.zeros(1 << 16, device=DEV)
    for k in range(4):
        y.copy_(torch.where(torch.arange(100, device=DEV) % 3 == k % 3, -1, (y.clamp(min=0) * 7 + k) % 2000))   # other rows take part
        a.mul_(-1.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            eager.loss_and_gradients(W, a, y, **e, mean=True)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(e[n], t[n]) for n in e), k
        scratch.add_(1.0)
        torch.cuda.synchronize()


def test_a_training_run_of_head_norm_and_adamw():
    """The operators as they are used: gradients of the head, clipped by their norm, AdamW with moments in 8 bits and a bf16 copy that the
    next step's head reads; every step against the same formulas in 64 bits from the state it began with."""
    import paper_1511_08486_amd as sfb
    n, J, D = 96, 1200, 128
    master = torch.randn(J, D, generator=torch.Generator().manual_seed(2)).to(DEV) * 0.05
    W = master.to(torch.bfloat16)
    head = sfb.SoftmaxHead(J, D, n)
    dW = torch.empty(J, D, dtype=torch.bfloat16, device=DEV)
    m8, v8 = (torch.zeros(J * D, dtype=torch.uint8, device=DEV) for _ in range(2))
    ms, vs = (torch.zeros(J * D // 128, dtype=torch.uint8, device=DEV) for _ in range(2))
    step, out, total = torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros(2, device=DEV), torch.zeros(1, device=DEV)
    norm = sfb.GradNorm([dW])
    opt = sfb.AdamW([master], [dW], [m8], [v8], step, m_scales=[ms], v_scales=[vs], copies=[W])
    mo, vo = (torch.zeros(J * D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for t in range(1, 6):
        _, a, y = _inputs(n, J, D, "bf16", "bf16", 100 + t, padded=0.2)
        opt.unpack([mo], [vo])
        opt.sync()
        W0, p0, m0, v0 = W.clone(), master.double(), mo.double().view(J, D), vo.double().view(J, D)
        head.loss_and_gradients(W, a, y, total=total, dW=dW, mean=True)
        norm(0.01, out)
        opt.step(lr=1e-2, betas=(0.9, 0.95), weight_decay=0.1, grad_scale=out[1:], seed=t)
        opt.sync()
        want = _formula(W0, a, y, mean=True)
        _check(dict(total=total, dW=dW), want, "bf16", "bf16", D, f"step {t}")
        g = dW.double()
        assert abs(float(out[0]) / float(g.norm()) - 1) < 1e-6 and abs(float(out[1]) / min(1.0, 0.01 / float(g.norm())) - 1) < 1e-6
        g = g * float(out[1])
        m, v = 0.9 * m0 + 0.1 * g, 0.95 * v0 + 0.05 * g * g
        p = p0 - 1e-2 * (m / (1 - 0.9 ** t) / ((v / (1 - 0.95 ** t)).sqrt() + 1e-8) + 0.1 * p0)
        assert float((master.double() - p).abs().max()) <= 1e-2 * 1e-4   # fp32 betas (1 - b2 to 1e-6) and a dozen roundings of moves of 1e-2
        assert torch.equal(W, master.to(torch.bfloat16)) and int(step) == t


def test_refusals():
    import paper_1511_08486_amd as sfb
    W, a, y = _inputs(10, 200, 64, "bf16", "bf16", 1)
    head = sfb.SoftmaxHead(200, 64, 10)
    v, dA, dW = torch.empty(10, device=DEV), torch.empty_like(a), torch.empty_like(W)
    for bad in (dict(W=W.float()), dict(W=W[:100]), dict(a=a.float()), dict(a=a[:, :32]), dict(y=y.long()), dict(y=y[:5]), dict(loss=v[:5]), dict(loss=v.double()),
                dict(dA=dA[:5]), dict(dW=dW.t()), dict(a=a.cpu()), dict(weight=v[:3])):
        with pytest.raises(ValueError):
            head.loss_and_gradients(**dict(dict(W=W, a=a, y=y, loss=v, lse=v.clone(), dA=dA, dW=dW), **bad))
    with pytest.raises(sfb.SfbError):
        head.loss(W, torch.cat([a, a]), torch.cat([y, y]))               # more rows than the head takes
    small = sfb.SoftmaxHead(200, 64, 10, workspace_bytes=head.least_bytes - 256)
    with pytest.raises(sfb.SfbError):
        small.loss_and_gradients(W, a, y, dA=dA, dW=dW)
    head.sync()


def test_heads_on_streams_of_their_own():
    """Two heads at once on two streams, each with its workspace, give what they give one after the other; "cuda" names the current GPU."""
    import paper_1511_08486_amd as sfb
    W, a, y = _inputs(300, 4000, 512, "bf16", "bf16", 40, padded=0.1)
    W2, a2, y2 = _inputs(200, 3000, 640, "f32", "f32", 41)

    def outs(n, J, D, t):
        return dict(lse=torch.zeros(n, device=DEV), dA=torch.zeros(n, D, dtype=t, device=DEV), dW=torch.zeros(J, D, dtype=t, device=DEV))
    sides = [torch.cuda.Stream(device=DEV) for _ in range(2)]
    heads = [sfb.SoftmaxHead(4000, 512, 300, stream=sides[0].cuda_stream, device="cuda"),
             sfb.SoftmaxHead(3000, 640, 200, dtype="f32", w_dtype="f32", stream=sides[1].cuda_stream, device="cuda")]
    want, got = [[outs(300, 4000, 512, torch.bfloat16), outs(200, 3000, 640, torch.float32)] for _ in range(2)]
    torch.cuda.synchronize()
    for h, o, x in zip(heads, want, ((W, a, y), (W2, a2, y2))):
        h.loss_and_gradients(*x, **o)
        h.sync()
    for _ in range(3):
        for h, o, x in zip(heads, got, ((W, a, y), (W2, a2, y2))):
            h.loss_and_gradients(*x, **o)
    torch.cuda.synchronize()
    for o, w in zip(got, want):
        assert all(torch.equal(o[k], w[k]) for k in o)


def test_words_beyond_32_bit_offsets():
    """W of 2.2e9 entries: the rows at its end, as words, labels and gradients."""
    import paper_1511_08486_amd as sfb
    n, J, D = 40, 140000, 16000
    W = torch.empty(J, D, dtype=torch.bfloat16, device=DEV)
    W.normal_(0.0, 0.02, generator=torch.Generator(device=DEV).manual_seed(3))
    a = torch.randn(n, D, generator=torch.Generator().manual_seed(4)).to(DEV).to(torch.bfloat16)
    y = torch.randint(J - 3000, J, (n,), generator=torch.Generator().manual_seed(5), dtype=torch.int32).to(DEV)
    o = dict(loss=torch.empty(n, device=DEV), lse=torch.empty(n, device=DEV), dA=torch.empty_like(a), dW=torch.empty_like(W))
    head = sfb.SoftmaxHead(J, D, n)
    head.loss_and_gradients(W, a, y, **o)
    head.sync()
    z = torch.cat([a.double() @ W[i:i + 10000].double().T for i in range(0, J, 10000)], 1)
    lse = torch.logsumexp(z, 1)
    u = torch.exp(z - lse[:, None])
    u[torch.arange(n), y.long()] -= 1.0
    dA = sum(u[:, i:i + 10000] @ W[i:i + 10000].double() for i in range(0, J, 10000))
    # scores of some +-2.5 from 16000 products: 1e-5 is twenty deviations of their rounding
    assert (o["lse"].double() - lse).abs().max() < 1e-5 and (o["loss"].double() - (lse - z[torch.arange(n), y.long()])).abs().max() < 2e-5
    # results' and U's rounding to bf16: 2^-8 each at most of the largest terms, by norm
    assert float((o["dA"].double() - dA).norm() / dA.norm()) < 2.0 ** -7
    for rows in (torch.arange(J - 3000, J, device=DEV), torch.arange(0, 500, device=DEV), torch.arange(134217, 134317, device=DEV)):
        dW = u[:, rows].T @ a.double()
        assert float((o["dW"][rows].double() - dW).norm() / dW.norm()) < 2.0 ** -7


@pytest.mark.parametrize("dtype,w_dtype", PAIRS)
@pytest.mark.parametrize("D", [1023, 1028, 4100, 8191, 8200, 25000])
def test_rows_of_every_length(D, dtype, w_dtype):
    _run(20, 70, D, dtype, w_dtype, 42, padded=0.2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,J,D,pad", [(1, 500, 64, 0), (1, 129, 68, 0), (7, 1000, 132, 4), (32, 300, 320, 0), (33, 257, 256, 8), (64, 5000, 1100, 0), (20, 700, 4096, 0),
                                       (20, 700, 100, 1), (64, 300, 66, 0), (5, 40, 60, 0)])
def test_loss_of_few_rows_with_fp32_words(n, J, D, pad, dtype):
    """W in fp32 read as it is (whole multiples of 4 features at 16-byte rows), and where it cannot be."""
    import paper_1511_08486_amd as sfb
    W, a, y = _inputs(n, J, D, dtype, "f32", 50 + n, pad=pad, padded=0.2 if n > 1 else 0.0, spread=3.0)
    weight = torch.rand(n, generator=torch.Generator().manual_seed(1)).to(DEV)
    head = sfb.SoftmaxHead(J, D, n, dtype=dtype, w_dtype="f32", gradients=False)
    head._ws.fill_(255)
    o = dict(loss=torch.full((n,), 7.0, device=DEV), lse=torch.full((n,), 7.0, device=DEV), total=torch.zeros(1, device=DEV))
    head.loss(W, a, y, **o, weight=weight, mean=True)
    head.sync()
    _check(o, _formula(W, a, y, weight, mean=True), dtype, "f32", D, f"{n} {J} {D}")


@pytest.mark.parametrize("n,J,D,pad,padded", [(1, 9000, 2048, 0, 0.0), (1, 300, 64, 0, 1.0), (7, 131, 128, 8, 0.4), (32, 40000, 1024, 0, 0.2),
                                              (33, 9001, 1984, 64, 0.5), (64, 2, 64, 0, 0.3), (64, 20000, 2048, 8, 1.0), (64, 8191, 704, 0, 0.0)])
def test_loss_of_few_rows_where_they_lie(n, J, D, pad, padded):
    """Features in bf16 at 16-byte places, whole stages: read in place, NaN in rows that take no part."""
    for weighted, mean in ((False, True), (True, False)):
        _run(n, J, D, "bf16", "bf16", seed=41, pad=pad, padded=padded, weighted=weighted, mean=mean, scale=0.75, two=True)
        _run(n, J, D, "bf16", "bf16", seed=41, pad=pad, padded=padded, weighted=weighted, mean=mean, rows=n + 100, ws=0.0, two=True)


def test_loss_of_few_rows_in_a_graph_with_other_labels():
    """Each replay of a captured loss follows the labels and features that are there then; labels as far out as their type goes."""
    import paper_1511_08486_amd as sfb
    n, J, D = 19, 5003, 256
    W, a, y = _inputs(n, J, D, "bf16", "bf16", seed=43)
    s = torch.cuda.Stream()
    head = sfb.SoftmaxHead(J, D, n, gradients=False, stream=s.cuda_stream)
    weight = torch.rand(n, device=DEV) + 0.1
    loss, lse, total = torch.full((n,), 77.0, device=DEV), torch.full((n,), 77.0, device=DEV), torch.full((1,), 77.0, device=DEV)
    call = lambda: head.loss(W, a, y, loss=loss, lse=lse, total=total, weight=weight, mean=True)  # noqa: E731
    torch.cuda.synchronize()
    call()
    head.sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call()
    for i, out in enumerate(([], [0, 5], [0, 1, 2, 18], list(range(n)), [7])):
        y.copy_(torch.randint(0, J, (n,), generator=torch.Generator().manual_seed(50 + i), dtype=torch.int32))
        a.copy_(torch.randn(n, D, generator=torch.Generator().manual_seed(60 + i)))
        for k, r in enumerate(out):
            y[r] = (-2 ** 31, 2 ** 31 - 1, -1, J)[k % 4]
            a[r] = (float("nan"), float("inf"), -float("inf"), 3e38)[k % 4]
        for x in (loss, lse, total):
            x.fill_(77.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        _check(dict(loss=loss, lse=lse, total=total), _formula(W, a, y, weight, mean=True), "bf16", "bf16", D, f"replay {i}")
        first = [x.clone() for x in (loss, lse, total)]
        call()
        head.sync()
        assert all(torch.equal(p, q) for p, q in zip(first, (loss, lse, total)))
