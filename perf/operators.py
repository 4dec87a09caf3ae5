"""The operators of a model's output layer and of its training step: softmax cross entropy of a linear head whose scores
are never held whole, with both gradients; the norm of many gradients; an AdamW step over many tensors with states in 32
or in 8 bits.  `listed` and `draw` say on what, `run` computes them in plain torch operations or, with `own`, through the
framework's entry points, `exact` says what should come out."""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda:0"

# What the 8-bit states are.  A block is 128 elements; its scale is a power of two, kept as exponent + 127 in a byte.
#   first moment   sign, 4 exponent bits of bias 7, 3 mantissa bits (torch.float8_e4m3fn's layout, NaN as 0x7f)
#   second moment  5 exponent bits of bias 15, 3 mantissa bits, no sign: the upper bits of an fp16 number
# Both are rounded at random, in proportion, with 16 bits each of a number made from (seed, step, element).
BLOCK = 128
M32 = 0xFFFFFFFF

_XENT = dict(op="xent", grads=True, n=1, J=1000, D=1024, dtype="bf16", w_dtype="bf16", spread=2.0, padded=0.0, weighted=False, pad_ld=0)
_MANY = dict(count=1, least=1, most=1, layout=0, grad="f32", max_norm=1.0)
_ADAMW = dict(op="adamw", bits=32, copy=False, clip=False, **_MANY)
_NORM = dict(op="norm", **_MANY)


def listed():
    return [
        # one token scored: W is read once, and nothing else costs
        dict(_XENT, name="xent_one_token", grads=False, n=1, J=32000, D=2048),
        # a few drafted tokens scored together against a large vocabulary
        dict(_XENT, name="xent_few_tokens", grads=False, n=24, J=65536, D=4096),
        # the ordinary fp32 model of this framework: 1000 classes on 4096 features, 512 samples
        dict(_XENT, name="xent_classes_f32", n=512, J=1000, D=4096, dtype="f32", w_dtype="f32"),
        # sizes off every grid, rows further apart than they are long, a fifth of the rows padding
        dict(_XENT, name="xent_ragged", n=999, J=50021, D=1100, padded=0.2, pad_ld=3),
        # 10000 classes on 21504 bf16 features with W in fp32
        dict(_XENT, name="xent_large_classes", n=512, J=10000, D=21504, w_dtype="f32", spread=1.0),
        # an fp32 language model's head, rows weighted, a padded batch
        dict(_XENT, name="xent_f32_weighted", n=2000, J=32000, D=1024, dtype="f32", w_dtype="f32", padded=0.3, weighted=True),
        # a training step's head at its largest: 4096 tokens, 131072 words, 4096 features
        dict(_XENT, name="xent_vocabulary", n=4096, J=131072, D=4096),
        # the gradients of a small model, fp32
        dict(_NORM, name="norm_small", count=20, least=64, most=40000, layout=1),
        # the gradients of a model of some hundred tensors, bf16
        dict(_NORM, name="norm_many", count=290, least=512, most=4000000, layout=2, grad="bf16"),
        # a small model's step: launches count
        dict(_ADAMW, name="adamw_small", count=20, least=64, most=40000, layout=1),
        # a model of some hundred tensors, bf16 gradients and a bf16 copy of the weights, clipped, states in 8 bits
        dict(_ADAMW, name="adamw_many_8bit", count=290, least=512, most=4000000, layout=2, grad="bf16", bits=8, copy=True, clip=True),
        # one W of 10000 x 21504 in fp32
        dict(_ADAMW, name="adamw_large", count=1, least=215040000, most=215040000),
    ]


def _size(rng, lo, hi):
    """Log-uniform in [lo, hi]; half as they fall (odd ones among them), half on a round size."""
    x = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    if rng.random() < 0.5:
        return max(lo, min(hi, int(round(x))))
    q = 8 if x < 256 else 64 if x < 4096 else 256
    return max(lo, min(hi, int(round(x / q)) * q or q))


def draw(rng):
    op = rng.choice(["xent", "xent", "xent", "adamw", "adamw", "norm"])
    if op == "xent":
        dtype, w_dtype = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
        while True:
            n, J, D = _size(rng, 1, 8192), _size(rng, 500, 131072), _size(rng, 64, 8192)
            if n * J * D <= (2.2e12 if w_dtype == "bf16" else 2.0e11) and J * D <= 5.4e8 and n * J <= 6e8:
                break
        return dict(_XENT, grads=rng.random() < 0.6, n=n, J=J, D=D, dtype=dtype, w_dtype=w_dtype, spread=round(rng.uniform(0.5, 3.0), 2),
                    padded=rng.choice([0.0, 0.0, 0.3]) if n >= 16 else 0.0, weighted=rng.random() < 0.3, pad_ld=rng.choice([0, 0, 1, 8]))
    while True:
        count, most = _size(rng, 1, 400), _size(rng, 2000, 50000000)
        c = dict(count=count, least=rng.choice([1, 100, 1000]), most=most, layout=rng.randrange(1000), grad=rng.choice(["f32", "bf16"]),
                 max_norm=round(rng.uniform(0.1, 2.0), 3))
        if sum(_sizes(c)) <= 150000000:
            break
    if op == "norm":
        return dict(_NORM, **c)
    return dict(_ADAMW, **c, bits=rng.choice([32, 8]), copy=rng.random() < 0.5, clip=rng.random() < 0.3)


# ---------------------------------------------------------------------------------------------------------------
# inputs


def _sizes(case):
    """The tensors' lengths: one of `most`, the others log-uniform in [least, most]."""
    r = random.Random(case["layout"])
    lo, hi = math.log(case["least"]), math.log(case["most"])
    return [case["most"]] + [max(1, int(round(math.exp(r.uniform(lo, hi))))) for _ in range(case["count"] - 1)]


def _places(sizes):
    """Where each tensor starts in one long buffer: at a multiple of 128 elements, as an allocator places them."""
    at, places = 0, []
    for n in sizes:
        places.append(at)
        at += (n + BLOCK - 1) // BLOCK * BLOCK
    return places, at


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 29)
    return g


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _rows(n, width, pad, dtype):
    """[n][width] whose rows lie width + pad elements apart."""
    return torch.empty((n, width + pad), dtype=dtype, device=DEV)[:, :width]


def prepare(case, seed):
    g = _gen(seed)
    randn = lambda *s: torch.randn(s, generator=g, device=DEV, dtype=torch.float32)  # noqa: E731
    rand = lambda *s: torch.rand(s, generator=g, device=DEV, dtype=torch.float32)  # noqa: E731
    s = dict(case=case)
    if case["op"] == "xent":
        n, J, D, t = case["n"], case["J"], case["D"], case["spread"]
        W = _rows(J, D, case["pad_ld"], _type(case["w_dtype"]))
        W.copy_(randn(J, D).mul_(t / math.sqrt(D)))
        y = torch.randint(0, J, (n,), generator=g, device=DEV, dtype=torch.int32)
        # normalised features that lean towards their word's row of W: from rows the model knows nothing of to sure ones
        lean = rand(n, 1).mul_(1.1 * (math.log(J) + 0.5 * t * t) / (t * t))
        a = _rows(n, D, case["pad_ld"], _type(case["dtype"]))
        a.copy_(randn(n, D) + lean * W[y.long()].float())
        y[rand(n) < case["padded"]] = -1
        s.update(W=W, a=a, y=y, weight=rand(n).add_(0.5) if case["weighted"] else None)
        s.update(loss=torch.zeros(n, device=DEV), lse=torch.zeros(n, device=DEV), total=torch.zeros(1, device=DEV))
        if case["grads"]:
            s.update(dA=_rows(n, D, 0, a.dtype), dW=_rows(J, D, 0, W.dtype))
        return s
    sizes = _sizes(case)
    places, total = _places(sizes)
    inside = torch.zeros(total, dtype=torch.bool, device=DEV)
    views = lambda x: [x[p:p + n] for p, n in zip(places, sizes)]  # noqa: E731
    for v in views(inside):
        v.fill_(True)
    # gradients whose size differs from place to place by a factor of some hundreds, as layers' do
    grad = randn(total).mul_(torch.exp(2.0 * randn(total // BLOCK)).repeat_interleave(BLOCK)).mul_(1e-3).mul_(inside).to(_type(case["grad"]))
    s.update(grad=grad, grads=views(grad), out=torch.zeros(2, device=DEV))
    if case["op"] == "norm":
        return s
    # a run under way: some steps taken, moments of gradients like today's
    p = randn(total).mul_(0.05).mul_(inside)
    m = grad.float().mul(0.3).add_(randn(total).mul_(grad.float().abs()).mul_(0.2)).mul_(inside)
    v = grad.float().square().mul_(0.8).add_(1e-12).mul_(inside)
    s.update(p=p, ps=views(p), step=torch.full((1,), 100, dtype=torch.int32, device=DEV))
    s.update(lr=3e-4, beta1=0.9, beta2=0.95, eps=1e-8, decay=0.1, seed=12345)
    if case["bits"] == 8:
        m, ms = _pack_first(m, torch.full_like(m, 0.5))
        v, vs = _pack_second(v, torch.full_like(v, 0.5))
        starts = [(q // BLOCK, (q + n + BLOCK - 1) // BLOCK) for q, n in zip(places, sizes)]
        s.update(ms=ms, vs=vs, mss=[ms[i:j] for i, j in starts], vss=[vs[i:j] for i, j in starts])
        s.update(m_out=torch.zeros(total, dtype=torch.bfloat16, device=DEV), v_out=torch.zeros(total, dtype=torch.bfloat16, device=DEV))
        s.update(m_outs=views(s["m_out"]), v_outs=views(s["v_out"]))
    s.update(m=m, v=v, mv=views(m), vv=views(v))
    if case["copy"]:
        s["copy"] = p.to(torch.bfloat16)
        s["copies"] = views(s["copy"])
    return s


# ---------------------------------------------------------------------------------------------------------------
# the plain forms


def _xent(s):
    c, W, a, y = s["case"], s["W"].float(), s["a"].float(), s["y"]
    keep = (y >= 0) & (y < c["J"])
    at = torch.where(keep, y, 0).long()[:, None]
    a = torch.where(keep[:, None], a, 0.0)
    z = a @ W.T
    top = z.amax(1, keepdim=True)
    zy = z.gather(1, at)
    e = z.sub_(top).exp_()
    sums = e.sum(1, keepdim=True)
    lse = top + sums.log()
    loss = torch.where(keep, (sums.log() + (top - zy))[:, 0], 0.0)
    lse = torch.where(keep, lse[:, 0], 0.0)
    g = keep.float() / keep.sum().clamp(min=1)
    if s["weight"] is not None:
        g = g * s["weight"]
    out = {"loss": loss, "lse": lse, "total": (g * loss).sum().reshape(1)}
    if c["grads"]:
        u = e.div_(sums)
        u.scatter_add_(1, at, torch.full_like(zy, -1.0))
        u.mul_(g[:, None])
        out["dA"] = (u @ W).to(s["a"].dtype)
        out["dW"] = (u.T @ a).to(s["W"].dtype)
    return out


def _norm(s):
    norm = s["grad"].double().square().sum().sqrt()
    factor = torch.where(torch.isfinite(norm), torch.clamp(s["case"]["max_norm"] / norm, max=1.0), math.nan)
    return torch.stack([norm, factor]).float()


def _mix(x):
    """32 bits stirred; int64 tensors or numbers in [0, 2^32)."""
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & M32
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & M32
    return x ^ (x >> 16)


def _noise(s, n, step):
    """(first, second) in [0, 1): 16 random bits each for n elements, below 2^32 of them."""
    key = _mix((s["seed"] + step.long() * 0x9E3779B9) & M32)
    h = _mix(torch.arange(n, device=DEV) ^ key)
    return (h & 0xFFFF).float() * 2.0 ** -16, (h >> 16).float() * 2.0 ** -16


def _scale_of(x, below):
    """Exponent of every block's scale: that of its largest finite magnitude, less `below`, within [-100, 120]."""
    x = torch.where(torch.isfinite(x), x.abs(), 0.0).reshape(-1, BLOCK).amax(1)
    return ((x.view(torch.int32) >> 23) - 127 - below).clamp_(-100, 120)


def _pow2(k):
    """2^k exactly, k an int32 tensor within [-126, 127]."""
    return ((k + 127) << 23).view(torch.float32)


def _pack(x, noise, k, small, bias, nan):
    """Codes of x >= 0 with 3 mantissa bits, rounded up with the probability `noise` stands for."""
    x = (x.reshape(-1, BLOCK) * _pow2(-k)[:, None]).reshape(-1)
    bits = (x.view(torch.int32) + ((noise * 65536.0).to(torch.int32) << 4) >> 20) - ((127 - bias) << 3)
    low = (x * small + noise).floor().to(torch.int32)
    code = torch.where(x < 8.0 / small, low, bits)
    return torch.where(torch.isfinite(x), code, nan)


def _pack_first(m, noise):
    k = _scale_of(m, 7)
    code = _pack(m.abs(), noise, k, 512.0, 7, 0x7F)
    return (code | torch.where(torch.signbit(m), 128, 0)).to(torch.uint8), (k + 127).to(torch.uint8)


def _pack_second(v, noise):
    k = _scale_of(v, 14)
    code = _pack(v, noise, k, 131072.0, 15, 0xFF)
    return torch.where(v > 0, code.clamp(min=1), code).to(torch.uint8), (k + 127).to(torch.uint8)


def _unpack(codes, scales):
    x = codes.view(torch.float8_e4m3fn).float()
    return (x.reshape(-1, BLOCK) * _pow2(scales.to(torch.int32) - 127)[:, None]).reshape(-1)


def _unpack_second(codes, scales):
    x = (codes.to(torch.int16) << 7).view(torch.float16).float()
    return (x.reshape(-1, BLOCK) * _pow2(scales.to(torch.int32) - 127)[:, None]).reshape(-1)


def _adamw(s):
    c, p = s["case"], s["p"]
    out = {}
    if c["clip"]:
        out["norm"] = _norm(s)
    g = s["grad"].float()
    if c["clip"]:
        g = g * out["norm"][1]
    bits8 = c["bits"] == 8
    m = _unpack(s["m"], s["ms"]) if bits8 else s["m"]
    v = _unpack_second(s["v"], s["vs"]) if bits8 else s["v"]
    b1, b2 = torch.tensor(s["beta1"], dtype=torch.float32).item(), torch.tensor(s["beta2"], dtype=torch.float32).item()
    m = m * b1 + g * (1.0 - b1)
    v = v * b2 + g * g * (1.0 - b2)
    s["step"] += 1
    t = s["step"].double()
    c1, c2 = 1.0 - s["beta1"] ** t, 1.0 - s["beta2"] ** t
    move = (m / c1.float()) / ((v / c2.float()).sqrt() + s["eps"])
    p.copy_(p - s["lr"] * (move + s["decay"] * p))
    out.update(p=p, step=s["step"])
    if c["copy"]:
        s["copy"].copy_(p)
        out["copy"] = s["copy"]
    if bits8:
        first, second = _noise(s, p.numel(), s["step"])
        (mc, ms), (vc, vs) = _pack_first(m, first), _pack_second(v, second)
        for_now = ((s["m"], mc), (s["ms"], ms), (s["v"], vc), (s["vs"], vs))
        [x.copy_(y) for x, y in for_now]
        out["m"] = _unpack(mc, ms).to(torch.bfloat16)               # exact: four significant bits and a power of two
        out["v"] = _unpack_second(vc, vs).to(torch.bfloat16)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
        out["m"], out["v"] = s["m"], s["v"]
    return out


# ---------------------------------------------------------------------------------------------------------------
# the framework's calls


def _own(s):
    import paper_1511_08486_amd as sfb
    c = s["case"]
    if c["op"] == "xent":
        if "head" not in s:                         # what a program keeps for as long as it trains: sizes and a workspace
            s["head"] = sfb.SoftmaxHead(c["J"], c["D"], c["n"], dtype=c["dtype"], w_dtype=c["w_dtype"], device=DEV)
        h, more = s["head"], dict(total=s["total"], weight=s["weight"], mean=True)
        out = {"loss": s["loss"], "lse": s["lse"], "total": s["total"]}
        if c["grads"]:
            h.loss_and_gradients(s["W"], s["a"], s["y"], s["loss"], s["lse"], s["dA"], s["dW"], **more)
            return dict(out, dA=s["dA"], dW=s["dW"])
        h.loss(s["W"], s["a"], s["y"], s["loss"], s["lse"], **more)
        return out
    if "norm" not in s and (c["op"] == "norm" or c["clip"]):
        s["norm"] = sfb.GradNorm(s["grads"], device=DEV)
    if c["op"] == "norm":
        return s["norm"](c["max_norm"], s["out"])
    if "opt" not in s:                              # the tensors' table, made once
        s["opt"] = sfb.AdamW(s["ps"], s["grads"], s["mv"], s["vv"], s["step"], m_scales=s.get("mss"), v_scales=s.get("vss"),
                             copies=s.get("copies"), device=DEV)
    out = {"p": s["p"], "step": s["step"]}
    if c["clip"]:
        out["norm"] = s["norm"](c["max_norm"], s["out"])
    s["opt"].step(lr=s["lr"], betas=(s["beta1"], s["beta2"]), eps=s["eps"], weight_decay=s["decay"], seed=s["seed"],
                  grad_scale=s["out"][1:] if c["clip"] else None)
    if c["copy"]:
        out["copy"] = s["copy"]
    if c["bits"] == 8:
        s["opt"].unpack(s["m_outs"], s["v_outs"])
        return dict(out, m=s["m_out"], v=s["v_out"])
    return dict(out, m=s["m"], v=s["v"])


def run(s):
    if own:
        return _own(s)
    return {"xent": _xent, "norm": _norm, "adamw": _adamw}[s["case"]["op"]](s)


def work(case):
    if case["op"] == "xent":
        n, J, D = case["n"] * (1.0 - case["padded"]), case["J"], case["D"]
        wb, ab = J * D * (2 if case["w_dtype"] == "bf16" else 4), n * D * (2 if case["dtype"] == "bf16" else 4)
        rows = 12 * case["n"]
        if case["grads"]:
            return {"bytes": 2 * wb + 2 * ab + rows, "flops": 6.0 * n * J * D}
        return {"bytes": wb + ab + rows, "flops": 2.0 * n * J * D}
    n, gb = sum(_sizes(case)), 2 if case["grad"] == "bf16" else 4
    if case["op"] == "norm":
        return {"bytes": n * gb + 8, "flops": 2.0 * n}
    each = 8 + gb + (16 if case["bits"] == 32 else 4 + 4.0 / BLOCK + 4) + 2 * case["copy"]
    return {"bytes": n * each, "flops": 15.0 * n}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "xent":
        return _exact_xent(case, s)
    g = s["grad"].double()
    norm = torch.linalg.vector_norm(g)
    both = torch.stack([norm, (case["max_norm"] / norm).clamp(max=1.0)])
    if case["op"] == "norm":
        return both
    if case["clip"]:
        g.mul_(both[1])
    if case["bits"] == 8:
        m, v = _exact_values(s["m"], s["ms"], True), _exact_values(s["v"], s["vs"], False)
    else:
        m, v = s["m"].double(), s["v"].double()
    t = int(s["step"]) + 1
    m.lerp_(g, 1.0 - s["beta1"])
    v.lerp_(g.square_(), 1.0 - s["beta2"])
    p = s["p"].double()
    p = p * (1.0 - s["lr"] * s["decay"]) - s["lr"] / (1.0 - s["beta1"] ** t) * m / ((v / (1.0 - s["beta2"] ** t)).sqrt() + s["eps"])
    out = {"p": p, "step": torch.tensor([t], dtype=torch.int32)}
    if case["copy"]:
        out["copy"] = p
    if case["clip"]:
        out["norm"] = both
    # which way a state in 8 bits is rounded is drawn, and has no value of its own
    out.update(m=None, v=None) if case["bits"] == 8 else out.update(m=m, v=v)
    return out


def _exact_values(codes, scales, signed):
    """What 8-bit codes stand for, by the definition of their format."""
    table, bias = [], 7 if signed else 15
    for code in range(256):
        e, f = (code >> 3) & (15 if signed else 31), code & 7
        x = math.ldexp(f, -2 - bias) if e == 0 else math.ldexp(8 + f, e - 3 - bias)
        table.append(-x if signed and code & 128 else x)
    x = torch.tensor(table, dtype=torch.float64, device=DEV)[codes.long()]
    return x * torch.pow(2.0, scales.double() - 127.0).repeat_interleave(BLOCK)


def _exact_xent(case, s):
    n, J = case["n"], case["J"]
    W, rows = s["W"].double(), [i for i, k in enumerate(s["y"].tolist()) if 0 <= k < J]
    weight = s["weight"].double() if s["weight"] is not None else torch.ones(n, dtype=torch.float64, device=DEV)
    loss, lse = torch.zeros(n, dtype=torch.float64, device=DEV), torch.zeros(n, dtype=torch.float64, device=DEV)
    dA = torch.zeros((n, case["D"]), dtype=torch.float64, device=DEV) if case["grads"] else None
    dW = torch.zeros((J, case["D"]), dtype=torch.float64, device=DEV) if case["grads"] else None
    step = max(1, 200000000 // J)
    for i in range(0, len(rows), step):
        r = torch.tensor(rows[i:i + step], device=DEV)
        a, y = s["a"][r].double(), s["y"][r].long()
        z = torch.matmul(a, W.t())
        lse[r] = torch.logsumexp(z, dim=1)
        loss[r] = lse[r] - z[torch.arange(len(r), device=DEV), y]
        if case["grads"]:
            u = z.sub_(lse[r].unsqueeze(1)).exp_()
            u[torch.arange(len(r), device=DEV), y] -= 1.0
            u *= (weight[r] / len(rows)).unsqueeze(1)
            dA[r] = torch.matmul(u, W)
            dW.addmm_(u.t(), a)
    out = {"loss": loss, "lse": lse, "total": ((weight * loss).sum() / max(1, len(rows))).reshape(1)}
    if case["grads"]:
        out.update(dA=dA, dW=dW)
    return out
