"""What sfb_adamw_* and sfb_grad_norm refuse, on the host: fake pointers are safe, nothing is launched."""
import ctypes as C

import pytest

P = 0x1000


@pytest.fixture()
def call():
    import paper_1511_08486_amd as sfb
    from paper_1511_08486_amd import binding as b
    ctx = C.c_void_p()
    assert b.lib.sfb_create(C.byref(ctx), sfb.SFB_MLR, 1, 1, 1, 1, sfb.SFB_F32, None) == 0

    def step(count=1, opt=True, tensors=True, tensor=(), **kw):
        t = (b.sfb_adamw_tensor * 1)(b.sfb_adamw_tensor(P, P, P, P, None, None, None, 8))
        for k, v in dict(tensor).items():
            setattr(t[0], k, v)
        o = b.sfb_adamw(1e-3, 0.9, 0.99, 1e-8, 0.1, 32, 0, 1, P, None, None)
        for k, v in kw.items():
            setattr(o, k, v)
        return b.lib.sfb_adamw_step(ctx, t if tensors else None, count, C.byref(o) if opt else None)

    yield b.lib, ctx, step
    b.lib.sfb_destroy(ctx)


def test_adamw_refuses(call):
    lib, ctx, step = call
    assert step(opt=False) == -1 and step(tensors=False) == -1 and step(count=-1) == -1 and step(step=None) == -1
    for name in ("lr", "eps", "weight_decay"):
        assert step(**{name: -1.0}) == -1 and step(**{name: float("nan")}) == -1 and step(**{name: float("inf")}) == -1
    for name in ("beta1", "beta2"):
        assert step(**{name: 1.0}) == -1 and step(**{name: -0.1}) == -1 and step(**{name: float("nan")}) == -1
    assert step(step=P + 2) == -1 and step(grad_scale=P + 1) == -1 and step(lr_scale=P + 2) == -1
    assert step(state_bits=16) == -1 and step(grad_dtype=7) == -3
    for name in ("p", "g", "m", "v"):
        assert step(tensor={name: None}) == -1
    assert step(tensor={"n": -1}) == -2 and step(tensor={"n": (1 << 40) + 1}) == -2
    assert step(state_bits=8) == -1                                     # no scales
    assert step(tensor={"p": P + 2}) == -1 and step(tensor={"g": P + 2}) == -1 and step(tensor={"copy": P + 1}) == -1
    assert step(tensor={"g": P + 1}, grad_dtype=1) == -1


def test_unpack_refuses(call):
    lib, ctx, _ = call
    from paper_1511_08486_amd import binding as b
    t = (b.sfb_adamw_tensor * 1)(b.sfb_adamw_tensor(None, None, P, P, P, P, None, 8))
    out, none = (C.c_void_p * 1)(P), (C.c_void_p * 1)(None)
    assert lib.sfb_adamw_unpack(None, t, 1, out, out) == -1 and lib.sfb_adamw_unpack(ctx, None, 1, out, out) == -1
    assert lib.sfb_adamw_unpack(ctx, t, 1, none, out) == -1 and lib.sfb_adamw_unpack(ctx, t, -1, out, out) == -1
    t[0].v_scale = None
    assert lib.sfb_adamw_unpack(ctx, t, 1, out, out) == -1


def test_grad_norm_refuses(call):
    lib, ctx, _ = call
    from paper_1511_08486_amd import binding as b
    g = (b.sfb_gradient * 1)(b.sfb_gradient(P, 100000))
    need = C.c_size_t()
    assert lib.sfb_grad_norm_bytes(g, 1, C.byref(need)) == 0 and need.value >= 16
    assert lib.sfb_grad_norm_bytes(g, 1, None) == -1 and lib.sfb_grad_norm_bytes(None, 1, C.byref(need)) == -1
    out = C.c_void_p(P)
    ok = dict(c=ctx, g=g, n=1, d=0, mx=1.0, out=out, ws=out, b=need.value)
    call_ = lambda **kw: (lambda a: lib.sfb_grad_norm(a["c"], a["g"], a["n"], a["d"], a["mx"], a["out"], a["ws"], a["b"]))({**ok, **kw})  # noqa: E731
    assert call_(c=None) == -1 and call_(g=None) == -1 and call_(n=-1) == -1 and call_(out=None) == -1
    assert call_(mx=0.0) == -1 and call_(mx=-1.0) == -1 and call_(mx=float("nan")) == -1
    assert call_(d=9) == -3 and call_(ws=None) == -5 and call_(b=need.value - 1) == -5
    g[0].n = -1
    assert call_() == -2
    g[0].n, g[0].g = 8, None
    assert call_() == -1
