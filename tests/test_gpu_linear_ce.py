"""linear_ce_loss and its C entry points against the definition in 64 bits, on the GPU."""
import ctypes

import pytest
import torch

import paper_2512_19743_amd as apml

from . import _feature_oracle as oracle

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    apml.load()


def make(samples, rows, classes, dim, dtype, *, seed=1, ignored=0.0, index=torch.int64, lean=1.0):
    """x (.., rows, dim), w (.., classes, dim) and targets; samples 0: one set of classes."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    S = max(1, samples)
    w = torch.randn(S, classes, dim, device="cuda", generator=g) * (2.0 / dim ** 0.5)
    t = torch.randint(0, classes, (S, rows), device="cuda", generator=g)
    x = torch.randn(S, rows, dim, device="cuda", generator=g) + lean * torch.stack([w[s][t[s]] for s in range(S)])
    if ignored:
        t = t.masked_fill(torch.rand(S, rows, device="cuda", generator=g) < ignored, -100)
    x, w, t = x.to(dtype), w.to(dtype), t.to(index)
    return (x, w, t) if samples else (x[0], w[0], t[0])


def check(x, w, t, *, grad_loss=None, reduction="mean", **kw):
    x, w = x.detach().requires_grad_(True), w.detach().requires_grad_(True)
    loss = apml.linear_ce_loss(x, w, t, reduction=reduction, **kw)
    assert loss.dtype == F32
    gx, gw = torch.autograd.grad(loss, (x, w), grad_loss if grad_loss is not None else torch.ones_like(loss))
    assert gx.dtype == gw.dtype == x.dtype and gx.shape == x.shape and gw.shape == w.shape
    ref = oracle.linear_ce(x.detach(), w.detach(), t, reduction=reduction, grad_loss=grad_loss, **kw)
    oracle.within(loss.detach(), ref["loss"], ref["loss_tol"], "loss")
    oracle.within(gx, ref["grad_x"], ref["grad_x_tol"], "grad_x")
    oracle.within(gw, ref["grad_w"], ref["grad_w_tol"], "grad_w")
    return loss.detach(), gx, gw


SIZES = [(0, 1, 1, 1), (0, 1, 7, 3), (0, 2, 16, 8), (0, 3, 1000, 64), (0, 16, 128, 64), (0, 17, 130, 72),
         (0, 64, 256, 128), (0, 65, 257, 65), (0, 130, 129, 200), (0, 1, 3001, 512), (0, 300, 513, 256),
         (0, 257, 2500, 33), (1, 40, 50, 24), (2, 33, 100, 48), (3, 129, 300, 64), (5, 16, 16, 128), (7, 1, 1, 9)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_small_and_odd_sizes(size, dtype):
    x, w, t = make(*size, dtype)
    check(x, w, t)
    g = torch.rand(t.shape, device="cuda") + 0.5
    check(x, w, t, reduction="none", grad_loss=g, scale=1.7)


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("size", [(0, 4096, 4100, 64), (0, 4160, 17000, 40), (0, 90, 70001, 64), (0, 6000, 300, 1024),
                                  (4, 2000, 1999, 72), (40, 1024, 1100, 32), (0, 200, 131000, 255), (0, 5000, 700, 515),
                                  (0, 40000, 260, 96)], ids=lambda s: "x".join(map(str, s)))
def test_sizes_of_every_tile_piece_and_split(size, dtype):
    # whole tiles of the large shape; several pieces of the classes and of the
    # samples; sums split over classes and over rows
    x, w, t = make(*size, dtype, ignored=0.1)
    check(x, w, t, reduction="sum", z_weight=1e-3)


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("reduction", ["none", "sum", "mean"])
@pytest.mark.parametrize("z_weight", [0.0, 0.01, -0.5])
def test_options(dtype, reduction, z_weight):
    x, w, t = make(0, 100, 333, 96, dtype, ignored=0.3, index=torch.int32)
    g = torch.randn(t.shape if reduction == "none" else (), device="cuda")
    check(x, w, t, reduction=reduction, z_weight=z_weight, scale=-0.8, grad_loss=g)


@pytest.mark.parametrize("ignore", [0, 7, 2 ** 40])
def test_any_class_may_be_the_ignored_one(ignore):
    x, w, t = make(0, 100, 10, 32, F32)
    check(x, w, t, ignore_index=ignore, reduction="mean")


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
def test_rows_of_very_different_weight(dtype):
    x, w, t = make(0, 70, 200, 64, dtype)
    g = torch.logspace(-12, 3, 70, device="cuda") * torch.where(torch.arange(70, device="cuda") % 2 == 0, 1.0, -1.0)
    g[5] = 0.0
    check(x, w, t, reduction="none", grad_loss=g)


def test_leading_dimensions_are_rows():
    x, w, t = make(0, 60, 90, 64, BF16)
    a = apml.linear_ce_loss(x, w, t, reduction="none")
    b = apml.linear_ce_loss(x.view(3, 4, 5, 64), w, t.view(3, 4, 5), reduction="none")
    assert b.shape == (3, 4, 5) and torch.equal(a, b.flatten())


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
def test_every_row_ignored(dtype):
    x, w, t = make(0, 33, 50, 64, dtype)
    x[:] = float("nan")
    t[:] = -100
    for reduction in ("none", "sum", "mean"):
        a, b = x.clone().requires_grad_(True), w.clone().requires_grad_(True)
        loss = apml.linear_ce_loss(a, b, t, reduction=reduction, z_weight=0.1)
        assert (loss == 0).all()
        for grad in torch.autograd.grad(loss.sum(), (a, b)):
            assert (grad == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 72])
def test_nan_and_infinity_in_ignored_rows(dtype, dim):
    x, w, t = make(0, 50, 80, dim, dtype, ignored=0.4)
    gone = t == -100
    y = x.clone()
    y[gone] = torch.tensor([float("nan"), float("inf")], device="cuda").repeat(dim // 2).to(dtype)
    for a, b in zip(check(y, w, t), check(x, w, t)):
        assert torch.equal(a, b)


def test_a_target_outside_the_classes_is_loud():
    x, w, t = make(0, 40, 60, 64, BF16)
    for bad in (60, -1, 2 ** 40):
        u = t.clone()
        u[7] = bad
        a = x.clone().requires_grad_(True)
        b = w.clone().requires_grad_(True)
        loss = apml.linear_ce_loss(a, b, u, reduction="none")
        assert torch.isnan(loss[7]) and torch.isfinite(loss[:7]).all() and torch.isfinite(loss[8:]).all()
        gx, gw = torch.autograd.grad(loss.sum(), (a, b))
        assert torch.isnan(gx[7]).all() and torch.isfinite(gx[:7]).all() and torch.isfinite(gx[8:]).all()
        assert torch.isnan(gw).all()
        assert torch.isnan(apml.linear_ce_loss(x, w, u))


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
def test_certain_targets_keep_their_small_losses(dtype):
    # the target's probability is 1 - 1e-6 and nearer: the loss is what the other classes leave
    g = torch.Generator(device="cuda").manual_seed(3)
    w = torch.nn.functional.normalize(torch.randn(64, 64, device="cuda", generator=g), dim=-1).to(dtype)
    t = torch.arange(64, device="cuda")
    x = w.clone()
    ref = oracle.linear_ce(x, w, t, scale=24.0, reduction="none")
    assert ref["loss"].max() < 1e-3
    loss, state = apml.apml_linear_ce_forward(x, w, t, scale=24.0, reduction="none")
    # relative: 24 (dim + 16) 2^-24 sum |x||w| on both logits, and the exponentials
    sums = (x.double().abs() @ w.double().abs().T).amax(1)
    rel = 2 * 24.0 * (64 + 16) * 2.0 ** -24 * sums + 2 * oracle.EXP
    oracle.within(loss, ref["loss"], ref["loss"] * rel * 1.01, "loss")


def test_logits_beyond_the_exponentials_range():
    x, w, t = make(0, 40, 60, 64, F32)
    check(x * 100.0, w, t, reduction="none")
    check(x, w, t, reduction="none", scale=-3000.0)


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-40])
def test_scales_of_nothing(scale):
    x, w, t = make(0, 40, 61, 64, F32, ignored=0.2)
    loss, gx, gw = check(x, w, t, reduction="none", scale=scale)
    assert (gx.abs() <= 1e-30).all() and (gw.abs() <= 1e-30).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e6, 1e30])
def test_upstream_gradients_of_any_size(dtype, size):
    if dtype == F16 and size == 1e30:
        pytest.skip("every gradient is beyond half precision")
    x, w, t = make(0, 40, 61, 64, dtype)
    for reduction in ("none", "sum"):
        check(x, w, t, reduction=reduction, z_weight=0.3, grad_loss=torch.full(t.shape if reduction == "none" else (), size,
                                                                              device="cuda"))


def test_rows_and_classes_that_are_equal():
    x, w, t = make(0, 40, 300, 64, BF16)
    w[:] = w[0]
    check(x, w, t)
    x[:] = x[0]
    t[:] = 5
    check(x, w, t, reduction="none", grad_loss=torch.rand(40, device="cuda"))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shift", [1, 3, 8])
def test_pointers_off_a_vectors_alignment(dtype, shift):
    x, w, t = make(0, 70, 300, 64, dtype)
    off = lambda a: torch.cat([a.new_zeros(shift), a.flatten()])[shift:].view_as(a)  # noqa: E731
    a, b = check(x, w, t), check(off(x), off(w), t)
    if dtype == BF16:  # the same products; aligned float32 rows of one tile are multiplied as they are, others by planes
        for u, v in zip(a, b):
            assert torch.equal(u, v)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_gradients_off_a_vectors_alignment(dtype):
    from paper_2512_19743_amd import _lib
    lib = apml.load()
    for dim in (64, 75):
        x, w, t = make(0, 70, 300, dim, dtype)
        one = torch.ones((), device="cuda")
        _, state = apml.apml_linear_ce_forward(x, w, t)
        want = apml.apml_linear_ce_backward(state, x, w, t, one)
        d = _lib._linear_ce_desc(x, w, t, 1.0, 0.0, -100, "mean")
        ws = _lib._ce_workspace(d, x, w, True)
        out = [torch.full((v.numel() + 8,), 7.0, dtype=dtype, device="cuda") for v in (x, w)]
        size = x.element_size()
        torch.cuda.synchronize()
        st = lib.apml_linear_ce_backward(ctypes.byref(d), x.data_ptr(), w.data_ptr(), t.data_ptr(), state.data_ptr(),
                                         one.data_ptr(), out[0].data_ptr() + 3 * size, out[1].data_ptr() + size,
                                         ws.data_ptr(), ws.numel(), None)
        torch.cuda.synchronize()
        assert st == 0
        for o, at, v in zip(out, (3, 1), want):
            assert torch.equal(o[at:at + v.numel()].view_as(v), v)
            assert (o[:at] == 7.0).all() and (o[at + v.numel():] == 7.0).all()


@pytest.mark.parametrize("size", [(0, 1, 5000, 96), (0, 16, 300, 32), (0, 17, 300, 160), (0, 128, 1000, 64),
                                  (0, 129, 1000, 64), (3, 100, 257, 64), (2, 5, 130, 2048)], ids=lambda s: "x".join(map(str, s)))
def test_float32_rows_of_one_tile(size):
    x, w, t = make(*size, F32, ignored=0.1)
    check(x, w, t, reduction="none", z_weight=1e-3)
    x[t == -100] = float("nan")
    check(x, w, t, scale=-1.5)


def test_strided_inputs():
    x, w, t = make(0, 70, 300, 64, BF16)
    xs = torch.stack([x, x], 1)[:, 0]
    ws = w.t().contiguous().t()
    ts = torch.stack([t, t], 1)[:, 1]
    assert not (xs.is_contiguous() or ws.is_contiguous() or ts.is_contiguous())
    assert torch.equal(apml.linear_ce_loss(xs, ws, ts), apml.linear_ce_loss(x, w, t))


def test_broadcast_upstream_gradient_and_one_sided_gradients():
    x, w, t = make(0, 70, 300, 64, BF16)
    a, b = x.clone().requires_grad_(True), w.clone().requires_grad_(True)
    ga, gb = torch.autograd.grad(apml.linear_ce_loss(a, b, t, reduction="none").sum(), (a, b))
    assert torch.equal(torch.autograd.grad(apml.linear_ce_loss(a, w, t, reduction="sum"), a)[0], ga)
    assert torch.equal(torch.autograd.grad(apml.linear_ce_loss(x, b, t, reduction="sum"), b)[0], gb)
    # one set of classes for two batches: the gradients add up
    both = apml.linear_ce_loss(a, b, t, reduction="sum") + apml.linear_ce_loss(2 * a, b, t, reduction="sum")
    gw = torch.autograd.grad(both, b)[0]
    r = [oracle.linear_ce(k * x, w, t, reduction="sum") for k in (1, 2)]
    oracle.within(gw, r[0]["grad_w"] + r[1]["grad_w"],
                  r[0]["grad_w_tol"] + r[1]["grad_w_tol"] + 2.0 ** -8 * (r[0]["grad_w"] + r[1]["grad_w"]).abs(), "grad_w")


@pytest.mark.parametrize("samples", [0, 2])
def test_gradients_against_differences(samples):
    x, w, t = make(samples, 9, 20, 12, F32, lean=0.5)
    args = dict(z_weight=0.05, scale=1.3, reduction="sum")
    a, b = x.clone().requires_grad_(True), w.clone().requires_grad_(True)
    gx, gw = torch.autograd.grad(apml.linear_ce_loss(a, b, t, **args), (a, b))
    g = torch.Generator(device="cuda").manual_seed(5)
    dx, dw = (torch.randn(v.shape, device="cuda", generator=g) for v in (x, w))
    h = 2.0 ** -6
    up, down = (float(apml.linear_ce_loss(x + k * h * dx, w + k * h * dw, t, **args).double()) for k in (1, -1))
    want = float((gx.double() * dx.double()).sum() + (gw.double() * dw.double()).sum())
    # central differences: rounding 2^-20 |loss| / h, and h^2 / 6 of the third derivative, which the
    # same difference in 64 bits has as well
    f = lambda k: float(oracle.linear_ce((x + k * h * dx).double().float(), (w + k * h * dw).double().float(), t,
                                         **args)["loss"])  # noqa: E731
    curved = abs((f(1) - f(-1)) / (2 * h) - want)
    assert abs((up - down) / (2 * h) - want) <= curved + 2.0 ** -18 * (abs(up) + abs(down)) / h


def test_the_same_bits_every_time():
    x, w, t = make(0, 500, 9001, 256, BF16, ignored=0.1)
    runs = [check(x, w, t, z_weight=1e-3) for _ in range(3)]
    for r in runs[1:]:
        for a, b in zip(r, runs[0]):
            assert torch.equal(a, b)


def test_backward_twice_and_without_gradients():
    x, w, t = make(0, 50, 60, 64, BF16)
    a = x.clone().requires_grad_(True)
    loss = apml.linear_ce_loss(a, w, t)
    first = torch.autograd.grad(loss, a, retain_graph=True)[0]
    assert torch.equal(first, torch.autograd.grad(loss, a)[0])
    assert not apml.linear_ce_loss(x, w, t).requires_grad
    with torch.no_grad():
        assert torch.equal(apml.linear_ce_loss(a, w, t), loss.detach())
    assert apml.apml_linear_ce_forward(x, w, t, keep_state=False)[1] is None


def test_a_second_derivative_is_refused():
    x, w, t = make(0, 30, 40, 64, F32)
    a = x.clone().requires_grad_(True)
    first = torch.autograd.grad(apml.linear_ce_loss(a, w, t), a)[0]
    g = torch.autograd.grad(apml.linear_ce_loss(a, w, t), a, create_graph=True)[0]
    assert torch.equal(g.detach(), first)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g.sum(), a)


def test_no_rows():
    for shape in ((0, 64), (3, 0, 64)):
        x = torch.empty(shape, device="cuda", dtype=BF16, requires_grad=True)
        w = torch.randn(20, 64, device="cuda").to(BF16).requires_grad_(True)
        t = torch.empty(shape[:-1], device="cuda", dtype=torch.int64)
        assert apml.linear_ce_loss(x, w, t, reduction="none").shape == shape[:-1]
        loss = apml.linear_ce_loss(x, w, t)
        gx, gw = torch.autograd.grad(loss, (x, w))
        assert loss == 0 and gx.shape == x.shape and (gw == 0).all()


def test_on_another_stream():
    x, w, t = make(0, 300, 2000, 128, BF16)
    want, state = apml.apml_linear_ce_forward(x, w, t)
    g = torch.ones((), device="cuda")
    wx, ww = apml.apml_linear_ce_backward(state, x, w, t, g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for use in ("argument", "context"):
        if use == "argument":
            loss, st = apml.apml_linear_ce_forward(x, w, t, stream=side)
            gx, gw = apml.apml_linear_ce_backward(st, x, w, t, g, stream=side)
        else:
            with torch.cuda.stream(side):
                loss, st = apml.apml_linear_ce_forward(x, w, t)
                gx, gw = apml.apml_linear_ce_backward(st, x, w, t, g)
        side.synchronize()
        assert torch.equal(loss, want) and torch.equal(gx, wx) and torch.equal(gw, ww)


def test_two_streams_at_once():
    data = [make(0, 400 + 100 * k, 3000, 128, BF16, seed=k) for k in range(2)]
    g = torch.ones((), device="cuda")
    want = []
    for d in data:
        loss, st = apml.apml_linear_ce_forward(*d)
        want.append((loss, *apml.apml_linear_ce_backward(st, *d, g)))
    streams = [torch.cuda.Stream() for _ in data]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(4):
        for k, s in enumerate(streams):
            loss, st = apml.apml_linear_ce_forward(*data[k], stream=s)
            got[k].append((loss, *apml.apml_linear_ce_backward(st, *data[k], g, stream=s)))
    torch.cuda.synchronize()
    for k in range(2):
        for r in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(r, want[k]))


def test_captured_and_replayed():
    x, w, t = make(0, 200, 1500, 96, BF16, ignored=0.1)
    g = torch.full((), 0.5, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(stream):
        apml.apml_linear_ce_backward(apml.apml_linear_ce_forward(x, w, t)[1], x, w, t, g)
        stream.synchronize()
        for _ in range(2):  # two graphs of the same call, alive together
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                loss, st = apml.apml_linear_ce_forward(x, w, t)
                gx, gw = apml.apml_linear_ce_backward(st, x, w, t, g)
            graphs.append((graph, loss, gx, gw))
    torch.cuda.synchronize()
    for k in range(3):
        y, v, u = make(0, 200, 1500, 96, BF16, ignored=0.1, seed=10 + k)
        x.copy_(y), w.copy_(v), t.copy_(u)
        loss, st = apml.apml_linear_ce_forward(y, v, u)
        want = (loss, *apml.apml_linear_ce_backward(st, y, v, u, g))
        torch.cuda.synchronize()
        for graph, *_ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, *got in graphs:
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_training_steps_gradients_captured():
    # the public call and its backward pass in one graph, as a captured training step has them
    x, w, t = make(0, 200, 1500, 96, BF16, ignored=0.1)
    a, b = x.clone().requires_grad_(True), w.clone().requires_grad_(True)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(2):
            torch.autograd.grad(apml.linear_ce_loss(a, b, t), (a, b))
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            loss = apml.linear_ce_loss(a, b, t)
            ga, gb = torch.autograd.grad(loss, (a, b))
    torch.cuda.synchronize()
    for k in range(3):
        y, v, u = make(0, 200, 1500, 96, BF16, ignored=0.1, seed=30 + k)
        with torch.no_grad():
            a.copy_(y), b.copy_(v)
        t.copy_(u)
        want = check(y, v, u)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip((loss.detach(), ga, gb), want))


def test_calls_from_two_threads():
    import threading
    data = [make(0, 300, 2000 + 100 * k, 128, BF16, seed=k) for k in range(2)]
    want = [check(*d) for d in data]
    got, errors = [[], []], []

    def work(k):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(4):
                    a, b = data[k][0].clone().requires_grad_(True), data[k][1].clone().requires_grad_(True)
                    loss = apml.linear_ce_loss(a, b, data[k][2])
                    got[k].append((loss.detach(), *torch.autograd.grad(loss, (a, b))))
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    torch.cuda.synchronize()
    assert not errors, errors
    for k in range(2):
        for r in got[k]:
            assert all(torch.equal(p, q) for p, q in zip(r, want[k]))


def test_workspace_of_the_asked_size_and_no_less():
    x, w, t = make(0, 70, 300, 72, BF16)
    lib = apml.load()
    from paper_2512_19743_amd import _lib
    d = _lib.apml_linear_ce_desc()
    lib.apml_linear_ce_desc_default(ctypes.byref(d))
    d.dtype, d.rows, d.classes, d.dim = 1, 70, 300, 72
    fwd, bwd = ctypes.c_size_t(), ctypes.c_size_t()
    ptr = lambda v: ctypes.c_void_p(v.data_ptr())  # noqa: E731
    assert lib.apml_linear_ce_workspace(ctypes.byref(d), ptr(x), ptr(w), ctypes.byref(fwd), ctypes.byref(bwd)) == 0
    want_loss, want_state = apml.apml_linear_ce_forward(x, w, t)
    gx0, gw0 = apml.apml_linear_ce_backward(want_state, x, w, t, torch.ones((), device="cuda"))
    loss, state, one = torch.full((1,), 7.0, device="cuda"), torch.zeros(71, 4, device="cuda"), torch.ones(1, device="cuda")
    gx, gw = torch.full_like(x, 7.0), torch.full_like(w, 7.0)
    guard = 4096
    ws = torch.full((max(fwd.value, bwd.value) + guard,), 77, dtype=torch.uint8, device="cuda")
    call = lambda n: lib.apml_linear_ce_forward(ctypes.byref(d), ptr(x), ptr(w), ptr(t), ptr(loss), ptr(state), ptr(ws),  # noqa: E731
                                                n, None)
    back = lambda n: lib.apml_linear_ce_backward(ctypes.byref(d), ptr(x), ptr(w), ptr(t), ptr(state), ptr(one), ptr(gx),  # noqa: E731
                                                 ptr(gw), ptr(ws), n, None)
    torch.cuda.synchronize()
    assert call(fwd.value - 1) == 1 and back(bwd.value - 1) == 1
    torch.cuda.synchronize()
    assert (loss == 7.0).all() and (gx == 7.0).all() and (gw == 7.0).all()
    assert call(fwd.value) == 0
    torch.cuda.synchronize()
    assert (ws[fwd.value:] == 77).all()
    ws.fill_(77)
    torch.cuda.synchronize()
    assert back(bwd.value) == 0
    torch.cuda.synchronize()
    assert (ws[bwd.value:] == 77).all()
    assert torch.equal(loss[0], want_loss) and torch.equal(gx, gx0) and torch.equal(gw, gw0)


def test_binding_refuses():
    x, w, t = make(0, 20, 30, 64, BF16)
    bad = [
        (x.float(), w, t), (x, w.float(), t), (x.double(), w.double(), t), (x, w, t.float()), (x, w[:, :32].contiguous(), t),
        (x, w, t[:10]), (x, w[:0], t), (x[:, :0].contiguous(), w[:, :0].contiguous(), t), (x, w.cpu(), t), (x.cpu(), w, t),
        (x, w, t.cpu()), (x, w.expand(2, 30, 64).contiguous(), t), (x, w[0], t), (x[0], w, t[0]),
    ]
    for args in bad:
        with pytest.raises(ValueError):
            apml.linear_ce_loss(*args)
    with pytest.raises(ValueError):
        apml.linear_ce_loss(x, w, t, reduction="average")
    with pytest.raises(ValueError):
        apml.linear_ce_loss(x, w, t, ignore_index=2 ** 64 - 100)
    with pytest.raises(ValueError):
        apml.apml_linear_ce_forward(x.t(), w, t)
    with pytest.raises(apml.ApmlError):
        apml.linear_ce_loss(x, w, t, scale=float("nan"))
    loss, state = apml.apml_linear_ce_forward(x, w, t)
    with pytest.raises(ValueError):
        apml.apml_linear_ce_backward(state[:5].contiguous(), x, w, t, torch.ones((), device="cuda"))
    with pytest.raises(ValueError):
        apml.apml_linear_ce_backward(state, x, w, t, torch.ones(20, device="cuda"))


def test_a_scale_that_is_a_tensor_is_refused():
    """It would be read without its gradient."""
    x, w, t = make(0, 20, 30, 64, BF16)
    for kw in (dict(scale=torch.ones((), requires_grad=True)), dict(z_weight=torch.zeros(()))):
        with pytest.raises(ValueError, match="number"):
            apml.linear_ce_loss(x, w, t, **kw)
    learned = torch.tensor(1.5, device="cuda", requires_grad=True)
    xf, wf = x.float(), w.float()
    apml.linear_ce_loss(xf * learned, wf, t).backward()
    want = torch.tensor(1.5, dtype=torch.float64, requires_grad=True)
    torch.nn.functional.cross_entropy((xf.cpu().double() * want) @ wf.cpu().double().T, t.cpu()).backward()
    # a sum of rows * dim terms in float32, each off by 2^-16 at most
    size = (xf.abs().double().sum() * wf.abs().double().amax()).item()
    assert abs(learned.grad.item() - want.grad.item()) <= 2.0 ** -16 * size


@pytest.mark.parametrize("mode", [torch.no_grad, torch.inference_mode])
def test_scored_without_gradients(mode):
    x, w, t = make(0, 20, 300, 64, BF16)
    want = apml.linear_ce_loss(x, w, t, reduction="none")
    with mode():
        got = apml.linear_ce_loss(x, w.requires_grad_(), t, reduction="none")
    assert torch.equal(got, want) and not got.requires_grad


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", [(0, 64, 40000, 128), (0, 4100, 90, 200), (3, 333, 5001, 48), (0, 2000, 2000, 600)],
                         ids=lambda s: "x".join(map(str, s)))
def test_one_gradient_alone(size, dtype):
    """Alone a gradient is cut into parts of its own."""
    x, w, t = make(*size, dtype)
    one = torch.ones((), device="cuda")
    want = oracle.linear_ce(x, w, t)
    _, state = apml.apml_linear_ce_forward(x, w, t)
    gx, none = apml.apml_linear_ce_backward(state, x, w, t, one, want_grad_w=False)
    oracle.within(gx, want["grad_x"], want["grad_x_tol"], "grad_x")
    assert none is None
    none, gw = apml.apml_linear_ce_backward(state, x, w, t, one, want_grad_x=False)
    oracle.within(gw, want["grad_w"], want["grad_w_tol"], "grad_w")
    assert none is None


@pytest.mark.parametrize("size,dtype", [((5, 4096, 8192, 64), BF16), ((7, 2050, 8000, 33), F32), ((0, 5000, 30000, 64), F32)],
                         ids=["3+2 of 5 samples", "4+3 of 7 samples", "pieces of the classes"])
def test_pieces_of_unequal_size(size, dtype):
    x, w, t = make(*size, dtype, ignored=0.1)
    check(x, w, t, z_weight=1e-3)


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("size", [(2, 300, 1500, 64), (0, 64, 40000, 128), (3, 129, 2000, 67), (0, 700, 1000, 200)],
                         ids=lambda s: "x".join(map(str, s)))
def test_the_targets_entries_lose_nothing_in_x(size, dtype):
    """x's gradient is as near as one rounding of it: the roundings of the other classes' entries are
    independent and each far below the row's, so that their squares add up to little."""
    x, w, t = make(*size, dtype, ignored=0.1)
    x, w = (torch.nn.functional.normalize(v.float(), dim=-1).to(dtype) for v in (x, w))
    up = float(t.numel())  # float16: the gradient of a mean is below its normal range
    leaf = x.clone().requires_grad_(True)
    loss = apml.linear_ce_loss(leaf, w, t, scale=12.0)
    got = torch.autograd.grad(loss, leaf, torch.tensor(up, device="cuda"))[0].double()
    X, W, T = (v if w.dim() == 3 else v.unsqueeze(0) for v in (x.double(), w.double(), t))
    used = T >= 0
    at = T.clamp_min(0).unsqueeze(-1)
    G = torch.softmax(12.0 * X @ W.transpose(1, 2).contiguous(), -1)
    G = G.scatter(2, at, G.gather(2, at) - 1.0) * (12.0 * up / used.sum()) * used.unsqueeze(-1)
    want = (G @ W).reshape(x.shape)
    rounded = (want.to(dtype).double() - want).square().sum()
    # an entry's rounding is off by u of it at most, u^2 / 3 in the mean of squares
    others = (oracle.HALF[dtype] ** 2 / 3 * G.scatter(2, at, 0.0).square() * W.square().sum(-1).unsqueeze(1)).sum()
    assert (got - want).square().sum() <= 1.2 * (rounded + others)


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("low", [150.0, 1000.0])
@pytest.mark.parametrize("size", [(0, 70, 200, 64), (0, 70, 200, 72), (2, 40, 90, 64), (0, 2048, 2100, 136)],
                         ids=lambda s: "x".join(map(str, s)))
def test_rows_of_no_weight_with_logits_far_below_zero(size, low, dtype):
    """A row that counts and whose upstream gradient is 0 has a gradient of 0, wherever its logits lie."""
    x, w, t = make(*size, dtype)
    x[..., 0], w[..., 0] = 8.0, -low / 8.0
    g = torch.rand(t.shape, device="cuda") + 0.5
    g[..., ::3] = 0.0
    for z_weight in (0.0, 0.01):
        _, gx, _ = check(x, w, t, reduction="none", z_weight=z_weight, grad_loss=g)
        assert (gx[..., ::3, :] == 0).all()
        for reduction in ("none", "sum", "mean"):
            off = torch.zeros(t.shape if reduction == "none" else (), device="cuda")
            _, gx, gw = check(x, w, t, reduction=reduction, z_weight=z_weight, grad_loss=off)
            assert (gx == 0).all() and (gw == 0).all()
    check(x, w, t, z_weight=0.01)


@pytest.mark.parametrize("dim", [64, 75, 600])
@pytest.mark.parametrize("z_weight", [0.0, 1e-3])
def test_float16_rows_of_small_weight_keep_their_bits_in_w(dim, z_weight):
    """Half the rows weigh 2^-20 of the others and share no class with them, at upstream gradients under
    which all results are in float16's normal range, as a scaled loss has them."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    n = 32
    x, w = torch.zeros(2 * n, dim, device="cuda"), torch.zeros(2 * n, dim, device="cuda")
    x[:n, :n] = w[:n, :n] = 8.0 * torch.eye(n, device="cuda")  # sure of their classes: exp(-64) elsewhere
    x[n:, n:] = torch.randn(n, dim - n, device="cuda", generator=gen)
    w[n:, n:] = torch.randn(n, dim - n, device="cuda", generator=gen) * (2.0 / dim ** 0.5)
    t = torch.cat([torch.arange(n, device="cuda"), torch.randint(n, 2 * n, (n,), device="cuda", generator=gen)])
    up = torch.where(torch.arange(2 * n, device="cuda") < n, 2.0 ** 12, 2.0 ** -8)
    x, w = x.half(), w.half()
    _, _, gw = check(x, w, t, reduction="none", grad_loss=up, z_weight=z_weight)
    X, W, T, U = x.double(), w.double(), t.unsqueeze(1), up.double().unsqueeze(1)
    z = X @ W.T
    lse = torch.logsumexp(z, 1, keepdim=True)
    p = torch.softmax(z, 1)
    one = torch.zeros_like(p).scatter(1, T, 1.0)
    c = 1 + 2 * z_weight * lse
    want = (U * (c * p - one)).T @ X
    # an entry of the logits' gradient and the result are rounded once (2^-11), the logits' sums and the
    # exponentials are off by 2^-15; a feature by 2^-38 of the largest one times its row's weight
    size = U * (c * p * (1 - one) + (1 - p + 2 * z_weight * lse.abs()) * one)
    largest = float((U * (1 + 2 * z_weight * lse.abs()) * X.abs()).max())
    tol = size.T @ X.abs() * (2.0 ** -11 + 2.0 ** -14) + (size / U).sum(0).unsqueeze(1) * 2.0 ** -38 * largest
    tol = tol + 2.0 ** -11 * want.abs() + 2.0 ** -24
    oracle.within(gw[n:], want[n:], tol[n:], "grad_w")


@pytest.mark.parametrize("weights", ["even", "uneven", "penalty"])
def test_float16_features_next_to_the_largest(weights):
    """The rows times their weights stay within the type."""
    x, w, t = make(0, 40, 61, 64, F16)
    x, w = x * 16000.0, w / 16000.0
    x[3, 5] = 65504.0
    up = torch.full(t.shape, 2.0 ** -9, device="cuda")
    if weights == "uneven":
        up = up * torch.logspace(-3, 0, 40, device="cuda")
        up[3] = 2.0 ** -9
    check(x, w, t, reduction="none", grad_loss=up, z_weight=0.1 if weights == "penalty" else 0.0)
    x[:] = 0.0
    check(x, w, t, reduction="none", grad_loss=up)


@pytest.mark.parametrize("rows,dim", [(4, 1), (4, 33), (130, 64), (130, 1000)])
def test_float32_products_drop_less_than_a_rounding(rows, dim):
    """c c for c = 1 + 2^-7 - 2^-23, whose last 16 bits are all ones: cut into 8-bit pieces that are
    truncated, the pieces' products that are left out are 2^-21 of it."""
    c = 1 + 2.0 ** -7 - 2.0 ** -23
    x, w = torch.zeros(rows, dim, device="cuda"), torch.zeros(2, dim, device="cuda")
    x[:, dim // 2] = c * torch.tensor([1.0, 2.0, 4.0, -8.0], device="cuda").repeat(rows)[:rows]
    w[1, dim // 2] = c
    t = (x[:, dim // 2] < 0).long()
    # the loss is the larger logit, 16 c c and more, and log1p(exp(-16)) below 2^-23; float32: the scale in
    # other units, the product's last sum, the result
    loss = apml.linear_ce_loss(x, w, t, scale=16.0, reduction="none")
    ref = oracle.linear_ce(x, w, t, scale=16.0, reduction="none")["loss"]
    oracle.within(loss, ref, 3.25 * 2.0 ** -24 * ref, "loss")


@pytest.mark.parametrize("size,dtype", [((0, 530000, 300, 40), BF16), ((0, 530001, 270, 72), F16),
                                        ((0, 175000, 2600, 72), F32), ((0, 263001, 260, 24), F32),
                                        ((0, 2200000, 40, 8), BF16), ((2, 264000, 257, 16), F32)],
                         ids=lambda v: "x".join(map(str, v)) if isinstance(v, tuple) else str(v)[6:])
def test_pieces_of_the_rows(size, dtype):
    """So many rows that a piece of all of them would be too large at the fewest classes."""
    x, w, t = make(*size, dtype, ignored=0.1)
    up = torch.full((), 2.0 ** -6, device="cuda")
    _, gx, gw = check(x, w, t, reduction="sum", z_weight=1e-3, grad_loss=up)
    _, state = apml.apml_linear_ce_forward(x, w, t, reduction="sum", z_weight=1e-3)
    alone = dict(reduction="sum", z_weight=1e-3)
    a, none = apml.apml_linear_ce_backward(state, x, w, t, up, want_grad_w=False, **alone)
    assert none is None and (a.double() - gx.double()).abs().max() <= 2.0 ** -7 * gx.double().abs().max()
    none, b = apml.apml_linear_ce_backward(state, x, w, t, up, want_grad_x=False, **alone)
    assert none is None and (b.double() - gw.double()).abs().max() <= 2.0 ** -7 * gw.double().abs().max()


@pytest.mark.parametrize("size,dtype", [((0, 200, 1500, 100), F16), ((0, 263000, 260, 24), F32)],
                         ids=["float16 rows of unequal weight", "pieces of the rows"])
def test_captured_with_a_weight_a_row(size, dtype):
    def data(seed):
        x, w, t = make(*size, dtype, ignored=0.1, seed=seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        return x, w, t, torch.exp2(-12.0 * torch.rand(t.shape, device="cuda", generator=g))

    def step(x, w, t, up):
        loss, st = apml.apml_linear_ce_forward(x, w, t, reduction="none", z_weight=1e-3)
        return loss, *apml.apml_linear_ce_backward(st, x, w, t, up, reduction="none", z_weight=1e-3)

    held = data(1)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step(*held)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = step(*held)
    torch.cuda.synchronize()
    for k in range(3):
        new = data(20 + k)
        for a, b in zip(held, new):
            a.copy_(b)
        want = step(*new)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
