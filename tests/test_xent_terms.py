"""How many 16-bit terms of fp32 operands the softmax head's products take, pinned entry by entry, and that the pins see a term that is missing.

Rows of features have three entries that are not 0, so that a score is a sum of three products and its error is small and known for
itself; the gradients are formed from a given log-sum-exp.  What is left of an error is the terms' arithmetic.  The emulation below
(64 bits, the terms as the header states them) stands in for the kernels here; the same checks run on them in the GPU tests."""
import pytest
import torch

CASES = [(24, 300, 1600), (96, 520, 640), (20, 70, 8200), (130, 1001, 192), (64, 2000, 256), (300, 900, 320)]
PAIRS = [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")]
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
E24 = 2.0 ** -24


def inputs(n, J, D, dtype, w_dtype, seed):
    """Words of sizes 2^-6 to 1 and rows' weights of 2^-12 to 2^12, all bits of the mantissas in use; scores of a few units."""
    g = torch.Generator().manual_seed(seed)
    W = torch.randn(J, D, generator=g) * 2.0 ** -torch.randint(0, 7, (J, 1), generator=g).float()
    a = torch.zeros(n, D)
    # neighbouring rows share features, so that dW adds up over rows
    at = (torch.randint(0, D, (n, 3), generator=g) % max(8, min(D, n // 2))) if n > 64 else torch.randint(0, D, (n, 3), generator=g)
    a.scatter_(1, at, torch.randn(n, 3, generator=g) * 1.3)
    y = torch.randint(0, J, (n,), generator=g, dtype=torch.int32)
    weight = (torch.rand(n, generator=g) + 0.5) * 2.0 ** torch.randint(-12, 13, (n,), generator=g).float()
    return W.to(TYPES[w_dtype]), a.to(TYPES[dtype]), y, weight


def scores(W, a):
    """64 bits, in rows' nonzero features only (the products of zeros are exact), with the sum of their magnitudes."""
    return a.double() @ W.double().T, a.double().abs() @ W.double().abs().T


def check_loss(got, W, a, y):
    """lse and loss: scores to 2^-20 of their products' magnitudes (two terms an operand leave 2^-22, three products and sums in
    fp32 a few 2^-24 each); exponentials and sums of J to a few 2^-24."""
    z, size = scores(W, a)
    lse = torch.logsumexp(z, 1)
    zy = z.gather(1, y.long()[:, None])[:, 0]
    p = torch.exp(z - lse[:, None])
    ez = 2.0 ** -20 * size
    moved = (p * ez).sum(1) + 2.0 ** -20 + 4 * E24 * lse.abs()          # (x of an exponential is rounded: |x| 2^-23 of it, |x| below 16)
    worst = {"lse": float(((got["lse"].double() - lse).abs() / moved).max()),
             "loss": float(((got["loss"].double() - (lse - zy)).abs() / (moved + ez.gather(1, y.long()[:, None])[:, 0] + 4 * E24 * zy.abs())).max())}
    assert max(worst.values()) <= 1.0, worst


def factors(W, a, y, weight, lse):
    """u of the given log-sum-exp, and how far off each may be before it is split: its score, the exponential's argument, the product with the weight."""
    z, size = scores(W, a)
    x = z - lse.double()[:, None]
    p, g = torch.exp(x), weight.double()[:, None]
    u = p.clone()
    u[torch.arange(len(y)), y.long()] -= 1.0
    off = p * (2.0 ** -20 * size + 2.0 ** -23 * (x.abs() + 2)) + 2 * E24 * u.abs()
    return u * g, off * g


def check_gradients(got, W, a, y, weight, lse):
    """dA in fp32: two fp16 terms of u and of W, 2^-22 of a product for each and for the product of second terms, and W's and U's smallest
    (2^-48 of the largest); dW: three bf16 terms, exact, 3 2^-24 for the products left out.  Both: the sums' roundings in fp32, sixteen half
    steps of the magnitudes' sum, and the result's own."""
    u, off = factors(W, a, y, weight, lse)
    Wd, ad = W.double(), a.double()
    worst = {}
    if got.get("dA") is not None and a.dtype == torch.float32:
        size = u.abs() @ Wd.abs()
        floor = weight.double()[:, None] * Wd.abs().max() * len(Wd) * 2.0 ** -48
        allow = off @ Wd.abs() + (3 * 2.0 ** -22 + 16 * E24) * size + floor
        worst["dA"] = float(((got["dA"].double() - u @ Wd).abs() / allow).max())
    if got.get("dW") is not None and W.dtype == torch.float32:
        size = u.abs().T @ ad.abs()
        allow = off.T @ ad.abs() + (3 * E24 + 16 * E24) * size + 1e-30
        worst["dW"] = float(((got["dW"].double() - u.T @ ad).abs() / allow).max())
    assert all(v <= 1.0 for v in worst.values()), worst
    return worst


# ---- the terms, emulated ------------------------------------------------------------------------------------------


def halves(x, terms):
    """fp16 terms of rows divided by their own power of two, put together again"""
    top = x.abs().amax(1, keepdim=True).clamp(min=1e-300)
    scale = 2.0 ** (torch.floor(torch.log2(top)) - 14)
    r, out = x / scale, []
    for t in range(terms):
        h = r.to(torch.float16).double()
        out.append(h * scale / 2048.0 ** t)
        r = (r - h) * 2048.0
    return out


def bf16s(x, terms):
    out = []
    for _ in range(terms):
        out.append(x.float().to(torch.bfloat16).double())
        x = x - out[-1]
    return out


def product(xs, ys, most):
    """sum over the pairs of terms whose numbers add up to `most` at most"""
    return sum(x @ y for i, x in enumerate(xs) for j, y in enumerate(ys) if i + j <= most)


def emulate(W, a, y, weight, lse, score=2, dA=2, dW=3):
    """The call with so many terms of an fp32 operand (a bf16 one is one term) in each product."""
    one = lambda t, k: 1 if t.dtype == torch.bfloat16 else k  # noqa: E731
    Wd, ad = W.double(), a.double()
    z = product(halves(ad, one(a, score)), [t.T for t in halves(Wd, one(W, score))], score - 1)
    if lse is None:
        v = torch.logsumexp(z, 1)
        return dict(lse=v.float(), loss=(v - z.gather(1, y.long()[:, None])[:, 0]).float())
    u = torch.exp(z - lse.double()[:, None])
    u[torch.arange(len(y)), y.long()] -= 1.0
    u = u * weight.double()[:, None]
    # (along a row of U the words' own powers of two are in it)
    top = 2.0 ** torch.floor(torch.log2(Wd.abs().amax(1)))
    us = [t / top for t in halves(u * top, dA)]
    return dict(dA=product(us, halves(Wd, one(W, dA)), dA - 1).to(a.dtype),
                dW=product([t.T for t in bf16s(u.float().double(), dW)], bf16s(ad, one(a, dW)), dW - 1).to(W.dtype))


@pytest.mark.parametrize("dtype,w_dtype", PAIRS)
@pytest.mark.parametrize("n,J,D", CASES)
def test_a_term_that_is_missing_is_seen(n, J, D, dtype, w_dtype):
    W, a, y, weight = inputs(n, J, D, dtype, w_dtype, n)
    whole = emulate(W, a, y, weight, None)
    check_loss(whole, W, a, y)
    with pytest.raises(AssertionError):
        check_loss(emulate(W, a, y, weight, None, score=1), W, a, y)
    lse = whole["lse"]
    check_gradients(emulate(W, a, y, weight, lse), W, a, y, weight, lse)
    if dtype == "f32":
        with pytest.raises(AssertionError, match="dA"):
            check_gradients(dict(dA=emulate(W, a, y, weight, lse, dA=1)["dA"]), W, a, y, weight, lse)
    if w_dtype == "f32":
        for terms in (1, 2):
            with pytest.raises(AssertionError, match="dW"):
                check_gradients(dict(dW=emulate(W, a, y, weight, lse, dW=terms)["dW"]), W, a, y, weight, lse)
