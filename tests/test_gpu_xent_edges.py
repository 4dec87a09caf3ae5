"""Calls of the softmax head where plans change: workspaces, places of W, tiles; against the formulas in 64 bits."""
import pytest
import torch

import test_xent_terms as terms
from test_gpu_xent import DEV, PAIRS, TYPES, _check, _formula, _inputs, _run

pytestmark = pytest.mark.gpu


def _loss(W, a, y, dtype, w_dtype, rows=None, weight=None, least=False):
    """loss, lse and total of a head that forms no gradients, on a workspace of NaN"""
    import paper_1511_08486_amd as sfb
    (J, D), n = W.shape, a.shape[0]
    head = sfb.SoftmaxHead(J, D, rows or n, dtype=dtype, w_dtype=w_dtype, gradients=False)
    if least:
        head = sfb.SoftmaxHead(J, D, rows or n, dtype=dtype, w_dtype=w_dtype, gradients=False, workspace_bytes=head.least_bytes)
        assert head._ws.numel() == max(head.least_bytes, 256)
    head._ws.fill_(255)
    o = dict(loss=torch.full((n,), 7.0, device=DEV), lse=torch.full((n,), 7.0, device=DEV), total=torch.zeros(1, device=DEV))
    head.loss(W, a, y, **o, weight=weight, mean=True)
    head.sync()
    return o


@pytest.mark.parametrize("n,J,D,pad,offset", [(1, 9000, 136, 1, 0), (24, 9000, 136, 3, 0), (64, 600, 1600, 1, 0), (33, 5000, 72, 0, 1), (70, 9000, 136, 1, 0),
                                              (200, 3000, 1608, 5, 3)])
def test_loss_alone_with_bf16_words_at_odd_places(n, J, D, pad, offset):
    """D % 8 = 0, so that W could be read as it is at other places; a head without gradients, whose best workspace is small then."""
    W, a, y = _inputs(n, J, D, "bf16", "bf16", 70 + n, pad=pad, offset=offset, padded=0.2 if n > 1 else 0.0)
    for least in (False, True):
        _check(_loss(W, a, y, "bf16", "bf16", least=least), _formula(W, a, y, mean=True), "bf16", "bf16", D, f"{n} {J} {D} least {least}")


def _product(head):
    """The kernel that the head's last call multiplied with first."""
    import ctypes as C
    from paper_1511_08486_amd import binding as b
    name = C.create_string_buffer(200)
    assert b.lib.sfb_last_kernel(head._ctx, 8, name, 200, None) == 0
    return name.value.decode()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 64])
def test_few_fp32_words_of_long_rows_are_cut_into_slices_of_features(n, dtype):
    """1000 words are eight workgroups where W is read as it is; more words of shorter rows fill the card that way."""
    import paper_1511_08486_amd as sfb
    for J, D, as_it_is in ((1000, 8192, False), (24000, 512, True), (8100, 12000, True)):
        W, a, y = _inputs(n, J, D, dtype, "f32", 80)
        head = sfb.SoftmaxHead(J, D, n, dtype=dtype, w_dtype="f32", gradients=False)
        loss = torch.empty(n, device=DEV)
        head.loss(W, a, y, loss=loss)
        head.sync()
        assert ("raw" in _product(head)) == as_it_is, _product(head)
        _check(dict(loss=loss), _formula(W, a, y), dtype, "f32", D, f"{n} {J} {D}")


@pytest.mark.parametrize("n,J,D,sliced", [(1, 8000, 1504, False), (1, 8000, 4096, False), (1, 1000, 4096, True), (64, 8000, 4096, True), (1, 500, 1024, False)])
def test_the_loss_alone_is_cut_into_slices_where_that_gains(n, J, D, sliced):
    import ctypes as C
    import paper_1511_08486_amd as sfb
    from paper_1511_08486_amd import binding as b
    W, a, y = _inputs(n, J, D, "bf16", "bf16", 81)
    head = sfb.SoftmaxHead(J, D, n, gradients=False)
    loss, grid = torch.empty(n, device=DEV), C.c_int32()
    head.loss(W, a, y, loss=loss)
    head.sync()
    assert b.lib.sfb_last_kernel(head._ctx, 8, None, 0, C.byref(grid)) == 0
    assert (grid.value > (J + 127) // 128) == sliced, grid.value         # tiles of 128 words at least: more workgroups are slices
    _check(dict(loss=loss), _formula(W, a, y), "bf16", "bf16", D, f"{n} {J} {D}")


def test_a_workspace_is_not_taken_from_another_streams_freed_memory():
    """What was freed on the current stream may still be in use there: an object of another stream must not be handed it."""
    import paper_1511_08486_amd as sfb
    side = torch.cuda.Stream(device=DEV)
    grads = [torch.ones(3 << 20, device=DEV)]
    kinds = ((lambda: sfb.SoftmaxHead(9000, 520, 200, stream=side.cuda_stream)), (lambda: sfb.GradNorm(grads, stream=side.cuda_stream)))
    for make in kinds:
        first = make()
        nbytes = first._ws.numel()
        torch.cuda.synchronize()
        freed = [torch.empty(nbytes, dtype=torch.uint8, device=DEV) for _ in range(4)]
        places = {t.data_ptr() for t in freed}
        del freed
        second = make()
        assert second._ws.data_ptr() not in places
        again = torch.empty(nbytes, dtype=torch.uint8, device=DEV)      # (they were there to be taken)
        assert again.data_ptr() in places
        with torch.cuda.stream(side):                                    # the stream's own freed memory is what it may take
            del first
    with torch.cuda.stream(side):                                        # and an object of the default stream made on another
        head = sfb.SoftmaxHead(300, 64, 8, stream=0)
        assert head.stream == 0 and head._ws.numel() >= 256
    torch.cuda.synchronize()


def test_loss_of_more_scores_than_a_launch_takes():
    """2^39 scores in fp32: the vocabulary goes in pieces, whatever the workspace holds."""
    import paper_1511_08486_amd as sfb
    n, J, D = 1 << 20, 1 << 19, 64
    g = torch.Generator(device=DEV).manual_seed(7)
    W, a = torch.randn(J, D, generator=g, device=DEV) * 0.25, torch.randn(n, D, generator=g, device=DEV)
    y = torch.randint(0, J, (n,), generator=g, device=DEV, dtype=torch.int32)
    y[5::1000] = -1
    loss, lse = torch.full((n,), 7.0, device=DEV), torch.full((n,), 7.0, device=DEV)
    head = sfb.SoftmaxHead(J, D, n, dtype="f32", w_dtype="f32", gradients=False)
    head.loss(W, a, y, loss=loss, lse=lse)
    head.sync()
    rows = torch.cat([torch.arange(0, 8), torch.tensor([1005]), torch.randint(0, n, (40,), generator=torch.Generator().manual_seed(1)), torch.arange(n - 8, n)]).to(DEV)
    assert (loss[5::1000] == 0).all() and torch.isfinite(loss).all()
    want = _formula(W, a[rows], y[rows])
    _check(dict(loss=loss[rows], lse=lse[rows]), want, "f32", "f32", D, "rows")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,J,D,pad,offset", [(1, 3000, 1, 0, 0), (2, 129, 3, 1, 1), (64, 5000, 63, 0, 2), (1, 20000, 64, 1, 0), (33, 20001, 65, 0, 0), (64, 30000, 66, 2, 1),
                                              (32, 40000, 127, 0, 3), (5, 40000, 130, 0, 0), (64, 20000, 193, 0, 0), (31, 20000, 254, 1, 1), (1, 24000, 259, 0, 0),
                                              (64, 16001, 321, 4, 1), (7, 16000, 383, 0, 0), (33, 16000, 447, 0, 0), (1, 16000, 511, 2, 3), (64, 33000, 1025, 0, 0),
                                              (20, 40000, 2047, 0, 1)])
def test_loss_of_few_rows_with_fp32_words_at_any_place(n, J, D, pad, offset, dtype):
    """W in fp32 with rows that neither start nor end at 16-byte places, one to thirty-two stages of 64 features; NaN between the rows."""
    import paper_1511_08486_amd as sfb
    W, a, y = _inputs(n, J, D, dtype, "f32", 90 + n, pad=pad, offset=offset, padded=0.2 if n > 2 else 0.0)
    weight = torch.rand(n, generator=torch.Generator().manual_seed(1)).to(DEV)
    want = _formula(W, a, y, weight, mean=True)
    for least in (False, True):
        _check(_loss(W, a, y, dtype, "f32", weight=weight, least=least), want, dtype, "f32", D, f"{n} {J} {D} least {least}")
    head = sfb.SoftmaxHead(J, D, n, dtype=dtype, w_dtype="f32", gradients=False)
    head.loss(W, a, y, loss=torch.empty(n, device=DEV))
    head.sync()
    assert "raw" in _product(head)


@pytest.mark.parametrize("dtype,w_dtype", terms.PAIRS)
@pytest.mark.parametrize("n,J,D", terms.CASES)
def test_every_term_of_an_fp32_operand_is_in(n, J, D, dtype, w_dtype):
    """Bounds that a product with a term less does not keep (tests/test_xent_terms.py shows that): losses, gradients alone and in one call."""
    import paper_1511_08486_amd as sfb
    cpu = terms.inputs(n, J, D, dtype, w_dtype, n)
    W, a, y, weight = (x.to(DEV) for x in cpu)
    back = lambda o: {k: v.cpu() for k, v in o.items()}  # noqa: E731
    head = sfb.SoftmaxHead(J, D, n, dtype=dtype, w_dtype=w_dtype)
    head._ws.fill_(255)
    o = dict(loss=torch.empty(n, device=DEV), lse=torch.empty(n, device=DEV))
    head.loss(W, a, y, **o)
    head.sync()
    terms.check_loss(back(o), *cpu[:3])
    grads = dict(dA=torch.empty_like(a), dW=torch.empty_like(W))
    head.gradients(W, a, y, o["lse"], **grads, weight=weight)
    head.sync()
    terms.check_gradients(back(grads), *cpu, o["lse"].cpu())
    both = dict(loss=torch.empty(n, device=DEV), lse=torch.empty(n, device=DEV), dA=torch.empty_like(a), dW=torch.empty_like(W))
    head.loss_and_gradients(W, a, y, **both, weight=weight)
    head.sync()
    both = back(both)
    terms.check_loss(both, *cpu[:3])
    terms.check_gradients(both, *cpu, both["lse"])


@pytest.mark.parametrize("n,J,D,pad,padded", [(1, 9000, 2048, 0, 0.0), (7, 131, 128, 8, 0.4), (33, 9001, 1984, 64, 0.5), (64, 20000, 2048, 8, 1.0)])
def test_loss_of_few_rows_where_they_lie_on_the_least_workspace(n, J, D, pad, padded):
    import paper_1511_08486_amd as sfb
    for rows in (n, n + 100):
        W, a, y = _inputs(n, J, D, "bf16", "bf16", 41, pad=pad, padded=padded)
        want = _formula(W, a, y, mean=True)
        _check(_loss(W, a, y, "bf16", "bf16", rows=rows, least=True), want, "bf16", "bf16", D, f"{n} {J} {D} rows {rows}")
        least = sfb.SoftmaxHead(J, D, rows).least_bytes
        head = sfb.SoftmaxHead(J, D, rows, workspace_bytes=least)
        assert head._ws.numel() == max(least, 256)
        head._ws.fill_(255)
        o = dict(loss=torch.empty(n, device=DEV), lse=torch.empty(n, device=DEV), total=torch.empty(1, device=DEV))
        head.loss(W, a, y, **o, mean=True)
        head._ws.fill_(255)
        grads = dict(dA=torch.empty_like(a), dW=torch.empty_like(W))
        head.gradients(W, a, y, o["lse"], **grads, mean=True)
        head.sync()
        _check(dict(o, **grads), want, "bf16", "bf16", D, f"{n} {J} {D} rows {rows}")


@pytest.mark.parametrize("dtype,w_dtype", PAIRS)
def test_rows_that_a_launch_of_their_own_lists(dtype, w_dtype):
    """More than 1024 rows, in every pair of types, some without a label, with room to spare and with the least."""
    for ws in (None, 1e-9):
        _run(1030, 700, 136, dtype, w_dtype, seed=61, padded=0.3, weighted=True, rows=1100, ws=ws)
        _run(2100, 300, 72, dtype, w_dtype, seed=62, padded=0.97, mean=False, scale=0.5, ws=ws, two=True)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("n,J,D,dtype,w_dtype,pad", [(5, 900, 128, "bf16", "bf16", 0), (70, 900, 136, "bf16", "bf16", 0), (40, 700, 1600, "bf16", "bf16", 0), (70, 600, 136, "f32", "f32", 0),
                                                     (40, 700, 1600, "f32", "f32", 0), (20, 24000, 192, "bf16", "f32", 0), (20, 24000, 192, "f32", "f32", 1), (20, 900, 72, "f32", "bf16", 0)])
def test_a_feature_that_is_not_finite_stays_in_its_row(n, J, D, dtype, w_dtype, pad, bad):
    """The row's own loss and gradient are not finite, and with it all of dW; the other rows' are what they are without it."""
    import paper_1511_08486_amd as sfb
    W, a, y = _inputs(n, J, D, dtype, w_dtype, 71, pad=pad)
    want, others = _formula(W, a, y), torch.arange(n, device=DEV) != 3
    a[3, D // 2] = bad
    o = dict(loss=torch.empty(n, device=DEV), lse=torch.empty(n, device=DEV), dA=torch.empty((n, D), dtype=a.dtype, device=DEV), dW=torch.empty((J, D), dtype=W.dtype, device=DEV))
    head = sfb.SoftmaxHead(J, D, n, dtype=dtype, w_dtype=w_dtype)
    for call in ("both", "loss"):
        if call == "both":
            head.loss_and_gradients(W, a, y, **o)
        else:
            o["loss"].zero_()
            head.loss(W, a, y, loss=o["loss"], lse=o["lse"])
        head.sync()
        assert not torch.isfinite(o["loss"][3]) and not torch.isfinite(o["lse"][3])
        assert not torch.isfinite(o["dA"][3].float()).any() and not torch.isfinite(o["dW"].float()).any()
        _check({k: o[k][others] for k in ("loss", "lse", "dA")}, {k: v[others] if v.shape[:1] == (n,) and k != "total" else v for k, v in want.items()},
               dtype, w_dtype, D, f"{call}: the other rows")


@pytest.mark.parametrize("n,J,D,dtype,w_dtype,pad", [(5, 900, 128, "bf16", "bf16", 0), (70, 900, 136, "bf16", "bf16", 0), (70, 600, 136, "f32", "f32", 0), (40, 700, 1600, "f32", "f32", 0),
                                                     (20, 24000, 192, "bf16", "f32", 0), (20, 24000, 192, "f32", "f32", 1)])
def test_a_word_that_is_nan_is_in_every_loss(n, J, D, dtype, w_dtype, pad):
    W, a, y = _inputs(n, J, D, dtype, w_dtype, 72, pad=pad)
    W[J // 2, D - 1] = float("nan")
    o = _loss(W, a, y, dtype, w_dtype)
    assert torch.isnan(o["loss"]).all() and torch.isnan(o["lse"]).all() and torch.isnan(o["total"]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,J,D,pad,offset", [(1, 500, 64, 0, 0), (64, 130, 65, 0, 1), (33, 1000, 67, 1, 0), (20, 3000, 130, 0, 2), (64, 257, 447, 0, 0), (5, 12000, 513, 2, 3),
                                              (32, 12000, 515, 0, 0), (40, 12001, 1022, 1, 1), (1, 20000, 1025, 0, 0), (64, 12000, 1540, 0, 0), (24, 12000, 2051, 3, 0)])
def test_gradients_of_few_rows_with_fp32_words_at_any_place(n, J, D, pad, offset, dtype):
    import paper_1511_08486_amd as sfb
    _run(n, J, D, dtype, "f32", seed=100 + n, pad=pad, offset=offset, padded=0.2 if n > 2 else 0.0, weighted=True, scale=1.5)
    _run(n, J, D, dtype, "f32", seed=100 + n, pad=pad, offset=offset, mean=False, out_pad=3, out_offset=1, two=True)
    W, a, y = _inputs(n, J, D, dtype, "f32", 1, pad=pad, offset=offset)
    head = sfb.SoftmaxHead(J, D, n, dtype=dtype, w_dtype="f32")
    head.loss_and_gradients(W, a, y, dA=torch.empty_like(a))
    head.sync()
    assert "raw" in _product(head)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,J,D", [(40, 20000, 520), (7, 15003, 1100)])
def test_gradients_of_few_rows_with_fp32_words_in_pieces(n, J, D, dtype):
    for ws in (1e-9, 0.1, 0.2, 0.3, 0.45, 0.6, 0.8):
        _run(n, J, D, dtype, "f32", seed=120, ws=ws, padded=0.1, two=ws == 0.45)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_gradient_of_few_rows_with_fp32_words_and_the_total(dtype):
    import paper_1511_08486_amd as sfb
    n, J, D = 30, 4000, 260
    W, a, y = _inputs(n, J, D, dtype, "f32", 121, padded=0.2)
    head, want = sfb.SoftmaxHead(J, D, n, dtype=dtype, w_dtype="f32"), _formula(W, a, y, mean=True)
    for k, like in (("dA", a), ("dW", W)):
        o = {"total": torch.zeros(1, device=DEV), k: torch.empty(like.shape, dtype=like.dtype, device=DEV)}
        head._ws.fill_(255)
        head.loss_and_gradients(W, a, y, **o, mean=True)
        head.sync()
        _check(o, want, dtype, "f32", D, k)


def test_few_rows_with_fp32_words_recorded_in_a_graph():
    import paper_1511_08486_amd as sfb
    n, J, D = 24, 6000, 322
    side = torch.cuda.Stream(device=DEV)
    W, a, y = _inputs(n, J, D, "f32", "f32", 122)
    outs = lambda: dict(loss=torch.zeros(n, device=DEV), lse=torch.zeros(n, device=DEV), dA=torch.zeros(n, D, device=DEV), dW=torch.zeros(J, D, device=DEV),  # noqa: E731
                        total=torch.zeros(1, device=DEV))
    eager, taken = (sfb.SoftmaxHead(J, D, n, dtype="f32", w_dtype="f32", stream=side.cuda_stream) for _ in range(2))
    e, t = outs(), outs()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        taken.loss_and_gradients(W, a, y, **t, mean=True)
    for k in range(4):
        y.copy_(torch.where(torch.arange(n, device=DEV) % 3 == k % 3, -1, (y.clamp(min=0) * 7 + k) % J))
        a.mul_(-1.0)
        torch.cuda.synchronize()
        eager.loss_and_gradients(W, a, y, **e, mean=True)
        eager.sync()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(e[x], t[x]) for x in e), k
        _check(t, _formula(W, a, y, mean=True), "f32", "f32", D, f"replay {k}")
