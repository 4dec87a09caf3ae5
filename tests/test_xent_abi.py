"""What the sfb_xent_* entry points refuse, on the host: fake pointers are safe, nothing is launched."""
import ctypes as C

import pytest

P = 0x1000


@pytest.fixture()
def make():
    import paper_1511_08486_amd as sfb
    from paper_1511_08486_amd import binding as b
    made = []

    def ctx(model=sfb.SFB_MLR, J=1000, D=64, rows=32, dtype=sfb.SFB_BF16):
        c = C.c_void_p()
        assert b.lib.sfb_create(C.byref(c), model, J, D, 1, rows, dtype, None) == 0
        made.append(c)
        return c

    def args(**kw):
        x = b.sfb_xent(W=P, ldw=64, w_dtype=1, mean=0, a=P, lda=64, y=P, n=32, loss=P, lse=P, total=None, weight=None, scale=1.0, reserved=0,
                       dA=P, ldda=64, dW=P, lddw=64, ws=P, ws_bytes=1 << 40)
        for k, v in kw.items():
            setattr(x, k, v)
        return x

    yield b.lib, ctx, args
    for c in made:
        b.lib.sfb_destroy(c)


@pytest.mark.parametrize("name", ["sfb_xent_loss", "sfb_xent_gradients", "sfb_xent_loss_and_gradients"])
def test_calls_refuse(make, name):
    lib, ctx, args = make
    import paper_1511_08486_amd as sfb
    c = ctx()
    call = lambda **kw: getattr(lib, name)(c, C.byref(args(**kw)))  # noqa: E731
    assert getattr(lib, name)(None, C.byref(args())) == -1 and getattr(lib, name)(c, None) == -1
    for null in ("W", "a", "y"):
        assert call(**{null: None}) == -1
    assert call(scale=float("nan")) == -1 and call(scale=float("inf")) == -1
    assert call(w_dtype=5) == -3
    assert call(n=-1) == -2 and call(n=33) == -2
    assert call(ldw=63) == -2 and call(lda=63) == -2
    for off in ("y", "loss", "lse", "total", "weight"):
        assert call(**{off: P + 2}) == -1
    assert call(W=P + 1) == -1 and call(a=P + 1) == -1 and call(ws=P + 16) == -1
    assert call(ws=None) == -5 and call(ws_bytes=0) == -5
    grads = C.c_size_t()
    assert lib.sfb_xent_workspace_bytes(c, 1, 0 if name == "sfb_xent_loss" else 1, C.byref(grads), None) == 0
    assert call(ws_bytes=grads.value - 1) == -5
    if name != "sfb_xent_loss":
        assert call(ldda=63) == -2 and call(lddw=63) == -2 and call(dA=P + 1) == -1 and call(dW=P + 1) == -1
    if name == "sfb_xent_gradients":
        assert call(lse=None) == -1
        assert call(dA=None, dW=None) == 0                               # nothing is wanted, nothing is launched
    assert getattr(lib, name)(ctx(model=sfb.SFB_DML, dtype=sfb.SFB_F32), C.byref(args())) == -6


def test_workspace_bytes(make):
    lib, ctx, _ = make
    import paper_1511_08486_amd as sfb
    least, best = C.c_size_t(), C.c_size_t()
    assert lib.sfb_xent_workspace_bytes(None, 1, 1, C.byref(least), C.byref(best)) == -1
    assert lib.sfb_xent_workspace_bytes(ctx(), 1, 1, None, None) == -1
    assert lib.sfb_xent_workspace_bytes(ctx(), 7, 1, C.byref(least), C.byref(best)) == -3
    assert lib.sfb_xent_workspace_bytes(ctx(model=sfb.SFB_DML, dtype=sfb.SFB_F32), 1, 1, C.byref(least), C.byref(best)) == -6
    assert lib.sfb_xent_workspace_bytes(ctx(D=(1 << 22) + 1), 1, 1, C.byref(least), C.byref(best)) == -6
    assert lib.sfb_xent_workspace_bytes(ctx(rows=(1 << 22) + 1), 1, 1, C.byref(least), C.byref(best)) == -6
    # one piece of 256 words beyond the bounds that pieces are cut to
    for c, w in ((ctx(rows=1 << 22, dtype=sfb.SFB_F32, J=100000), 0), (ctx(D=1 << 22, rows=8, dtype=sfb.SFB_F32, J=100000), 0), (ctx(rows=1 << 22, J=100000), 1)):
        for grads in (0, 1):
            assert lib.sfb_xent_workspace_bytes(c, w, grads, C.byref(least), C.byref(best)) == 0 and 0 < least.value <= best.value
    # far below the scores and factors themselves: 131072 words, 4096 features, 8192 rows are 4.3 GB of fp32 scores
    big = ctx(J=131072, D=4096, rows=8192)
    for grads in (0, 1):
        assert lib.sfb_xent_workspace_bytes(big, 1, grads, C.byref(least), C.byref(best)) == 0
        assert 0 < least.value <= best.value < 1 << 30
