"""balance_loss, expert_counts and their C entry points against the definitions in 64 bits, on the GPU."""
import pytest
import torch

import paper_2512_19743_amd as apml

from . import _feature_oracle as oracle

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
INF = float("inf")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    apml.load()


def make(samples, tokens, experts, chosen, dtype, *, seed=1, dropped=0.0, padded=0.0, index=torch.int64):
    g = torch.Generator(device="cuda").manual_seed(seed)
    S = max(1, samples)
    logits = (1.5 * torch.randn(S, tokens, experts, device="cuda", generator=g)
              + torch.randn(experts, device="cuda", generator=g)).to(dtype)
    ids = logits.float().topk(chosen, -1).indices
    if dropped:
        ids = ids.masked_fill(torch.rand(ids.shape, device="cuda", generator=g) < dropped, -1)
    valid = torch.rand(S, tokens, device="cuda", generator=g) >= padded if padded else None
    ids = ids.to(index)
    return (logits, ids, valid) if samples else (logits[0], ids[0], valid[0] if valid is not None else None)


def check(logits, ids, valid, *, reduction="mean", z_weight=0.0, grad_loss=None, counts=None):
    a = logits.detach().requires_grad_(True)
    want = counts if counts is not None else oracle.counts(ids, logits.shape[-1], valid)
    loss, got = apml.balance_loss(a, ids if counts is None else None, counts=counts, valid=valid, z_weight=z_weight,
                                  reduction=reduction)
    assert got.dtype == torch.int64 and torch.equal(got.cpu(), want.cpu()) and not got.requires_grad
    if counts is None:
        assert torch.equal(apml.expert_counts(ids, logits.shape[-1], valid=valid), got)
    grad = torch.autograd.grad(loss, a, grad_loss if grad_loss is not None else torch.ones_like(loss))[0]
    assert loss.dtype == F32 and grad.dtype == a.dtype and grad.shape == a.shape
    ref = oracle.balance(logits, want, valid=valid, z_weight=z_weight, reduction=reduction, grad_loss=grad_loss)
    oracle.within(loss.detach(), ref["loss"], ref["loss_tol"], "loss")
    oracle.within(grad, ref["grad"], ref["grad_tol"], "grad")
    return loss.detach(), got, grad


SIZES = [(0, 1, 1, 1), (0, 1, 8, 2), (0, 2, 3, 3), (0, 255, 4, 1), (0, 1000, 8, 2), (0, 77, 16, 4), (2, 300, 12, 2),
         (3, 129, 64, 6), (1, 513, 65, 3), (0, 700, 128, 8), (5, 33, 161, 2), (2, 1, 256, 8), (0, 300, 500, 4),
         (0, 65, 1023, 2), (2, 40, 1024, 8), (70, 5, 7, 2)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_small_and_odd_sizes(size, dtype):
    up = torch.tensor(float(max(1, size[0]) * size[1]), device="cuda")  # keeps half precision's gradients in range
    check(*make(*size, dtype), grad_loss=up)
    check(*make(*size, dtype, seed=2, dropped=0.2, padded=0.3, index=torch.int32), z_weight=0.01, grad_loss=up)


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("size", [(0, 100001, 8, 2), (3, 20000, 64, 6), (2, 9999, 161, 3), (0, 30000, 256, 8)],
                         ids=lambda s: "x".join(map(str, s)))
def test_many_chunks(size, dtype):
    up = torch.tensor(float(max(1, size[0]) * size[1]), device="cuda")
    check(*make(*size, dtype, dropped=0.1, padded=0.2), z_weight=1e-3, grad_loss=up)


@pytest.mark.parametrize("reduction", ["none", "sum", "mean"])
@pytest.mark.parametrize("samples", [0, 1, 4])
def test_reductions_and_upstream_gradients(reduction, samples):
    logits, ids, valid = make(samples, 90, 24, 3, F32, padded=0.2)
    g = torch.randn((samples,) if samples and reduction == "none" else (), device="cuda")
    loss, counts, grad = check(logits, ids, valid, reduction=reduction, z_weight=0.2, grad_loss=g)
    assert loss.shape == g.shape and counts.shape == logits.shape[:-2] + logits.shape[-1:]
    # the counts of elsewhere give the same loss and gradient
    again = check(logits, None, valid, reduction=reduction, z_weight=0.2, grad_loss=g, counts=counts)
    assert torch.equal(loss, again[0]) and torch.equal(grad, again[2])
    check(logits, None, valid, reduction=reduction, grad_loss=g, counts=counts * 3 + 5)
    check(logits, None, valid, reduction=reduction, grad_loss=g, counts=torch.zeros_like(counts))
    check(logits, None, valid, reduction=reduction, grad_loss=g, counts=counts + 2 ** 40)


def test_even_routing_is_one():
    logits = torch.zeros(64, 16, device="cuda")
    ids = torch.arange(64, device="cuda").remainder(16).unsqueeze(1)
    loss, counts = apml.balance_loss(logits, ids)
    assert (counts == 4).all() and abs(float(loss) - 1.0) <= 2.0 ** -20


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("experts", [16, 21])
def test_padding_that_holds_anything(dtype, experts):
    logits, ids, valid = make(3, 70, experts, 2, dtype, padded=0.4)
    valid[1] = False  # a sample without tokens
    other = logits.clone()
    other[~valid] = torch.tensor(float("nan"), dtype=dtype, device="cuda")
    odd = ids.clone()
    odd[~valid] = 2 ** 50
    a = check(logits, ids, valid, reduction="none", z_weight=0.1)
    x = other.requires_grad_(True)
    loss, counts = apml.balance_loss(x, odd, valid=valid, reduction="none", z_weight=0.1)
    grad = torch.autograd.grad(loss.sum(), x)[0]
    assert torch.equal(loss, a[0]) and torch.equal(counts, a[1]) and torch.equal(grad, a[2])
    assert loss[1] == 0 and (grad[~valid] == 0).all() and (counts[1] == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("experts", [16, 21])
def test_experts_out_of_reach(dtype, experts):
    logits, ids, _ = make(2, 60, experts, 2, dtype)
    g = torch.Generator(device="cuda").manual_seed(4)
    logits = logits.masked_fill(torch.rand(logits.shape, device="cuda", generator=g) < 0.5, -INF)
    logits[0, 7] = -INF  # nothing left
    logits[1, 3, 1:] = -INF
    logits[1, 4, :-1] = torch.finfo(dtype).min
    check(logits, ids, None, z_weight=0.1)


def test_logits_at_the_types_ends():
    for dtype in (F32, BF16, F16):
        logits, ids, _ = make(0, 60, 16, 2, dtype)
        logits[::3] = torch.finfo(dtype).max
        logits[1::3, 4] = torch.finfo(dtype).max
        logits[1::3, 5] = torch.finfo(dtype).min
        check(logits, ids, None)


def test_indices_outside_the_experts_and_named_twice():
    logits, ids, _ = make(0, 50, 10, 3, F32)
    ids[::4, 0] = 10
    ids[1::4, 1] = -7
    ids[2::4, 2] = 2 ** 32 + 1
    ids[3::4, 2] = ids[3::4, 1]
    check(logits, ids, None)


@pytest.mark.parametrize("shift", [1, 2])
def test_pointers_off_a_vectors_alignment(shift):
    for dtype in (F32, BF16):
        logits, ids, valid = make(2, 60, 32, 2, dtype, padded=0.2)
        off = torch.cat([logits.new_zeros(shift), logits.flatten()])[shift:].view_as(logits)
        check(off, ids, valid)


def test_strided_inputs():
    logits, ids, valid = make(2, 60, 32, 4, BF16, padded=0.2)
    ls = logits.transpose(0, 1).contiguous().transpose(0, 1)
    es = torch.stack([ids, ids], -1)[..., 0]
    vs = torch.stack([valid, valid], -1)[..., 0]
    assert not (ls.is_contiguous() or es.is_contiguous() or vs.is_contiguous())
    a, b = apml.balance_loss(ls, es, valid=vs), apml.balance_loss(logits, ids, valid=valid)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.equal(apml.expert_counts(es, 32, valid=vs), b[1])


def test_gradients_against_differences():
    logits, ids, valid = make(2, 20, 9, 2, F32, padded=0.2)
    counts = apml.expert_counts(ids, 9, valid=valid)
    x = logits.clone().requires_grad_(True)
    loss, _ = apml.balance_loss(x, counts=counts, valid=valid, z_weight=0.1)
    grad = torch.autograd.grad(loss, x)[0]
    g = torch.Generator(device="cuda").manual_seed(5)
    d = torch.randn(logits.shape, device="cuda", generator=g)
    h = 2.0 ** -6
    want = float((grad.double() * d.double()).sum())
    f = lambda k: float(apml.balance_loss(logits + k * h * d, counts=counts, valid=valid, z_weight=0.1)[0].double())  # noqa: E731
    o = lambda k: float(oracle.balance(logits + k * h * d, counts, valid=valid, z_weight=0.1)["loss"])  # noqa: E731
    curved = abs((o(1) - o(-1)) / (2 * h) - want)
    assert abs((f(1) - f(-1)) / (2 * h) - want) <= curved + 2.0 ** -18 * (abs(f(1)) + abs(f(-1))) / h


def test_the_same_bits_every_time():
    d = make(4, 5000, 48, 4, BF16, padded=0.1)
    runs = [check(*d, z_weight=0.1) for _ in range(3)]
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, runs[0]))


def test_two_streams_at_once():
    data = [make(2, 6000 + 50 * k, 60, 3, BF16, seed=k, padded=0.2) for k in range(2)]
    want = [apml.apml_balance_forward(a, b, valid=c, z_weight=0.1)[:2] for a, b, c in data]
    streams = [torch.cuda.Stream() for _ in data]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(4):
        for k, s in enumerate(streams):
            a, b, c = data[k]
            got[k].append(apml.apml_balance_forward(a, b, valid=c, z_weight=0.1, stream=s)[:2])
    torch.cuda.synchronize()
    for k in range(2):
        for r in got[k]:
            assert torch.equal(r[0], want[k][0]) and torch.equal(r[1], want[k][1])


def test_a_second_derivative_is_refused():
    logits, ids, _ = make(0, 30, 8, 2, F32)
    a = logits.clone().requires_grad_(True)
    first = torch.autograd.grad(apml.balance_loss(a, ids)[0], a)[0]
    g = torch.autograd.grad(apml.balance_loss(a, ids)[0], a, create_graph=True)[0]
    assert torch.equal(g.detach(), first)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g.sum(), a)


def test_no_tokens():
    for shape in ((0, 8), (3, 0, 8)):
        x = torch.empty(shape, device="cuda", requires_grad=True)
        ids = torch.empty(*shape[:-1], 2, dtype=torch.int64, device="cuda")
        loss, counts = apml.balance_loss(x, ids)
        assert loss == 0 and (counts == 0).all() and counts.shape == shape[:-2] + shape[-1:]
        assert torch.autograd.grad(loss, x)[0].shape == x.shape
        assert torch.equal(apml.expert_counts(ids, 8), counts)


def test_on_another_stream():
    logits, ids, valid = make(2, 3000, 64, 4, BF16, padded=0.2)
    g = torch.ones((), device="cuda")
    want = apml.apml_balance_forward(logits, ids, valid=valid)
    grad = apml.apml_balance_backward(want[2], logits, g, valid=valid)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = apml.apml_balance_forward(logits, ids, valid=valid, stream=side)
    ggot = apml.apml_balance_backward(got[2], logits, g, valid=valid, stream=side)
    counts = apml.apml_expert_counts(ids, 64, valid=valid, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(ggot, grad)
    assert torch.equal(counts, want[1])


def test_captured_and_replayed():
    logits, ids, valid = make(2, 9000, 64, 4, BF16, padded=0.2)
    g = torch.ones((), device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        apml.apml_balance_forward(logits, ids, valid=valid)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            loss, counts, state = apml.apml_balance_forward(logits, ids, valid=valid, z_weight=0.1)
            grad = apml.apml_balance_backward(state, logits, g, valid=valid, z_weight=0.1)
            alone = apml.apml_expert_counts(ids, 64, valid=valid)
    torch.cuda.synchronize()
    for k in range(3):
        a, b, c = make(2, 9000, 64, 4, BF16, padded=0.2, seed=20 + k)
        logits.copy_(a), ids.copy_(b), valid.copy_(c)
        want = apml.apml_balance_forward(a, b, valid=c, z_weight=0.1)
        wgrad = apml.apml_balance_backward(want[2], a, g, valid=c, z_weight=0.1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want[0]) and torch.equal(counts, want[1]) and torch.equal(grad, wgrad)
        assert torch.equal(alone, want[1])


def test_binding_refuses():
    logits, ids, valid = make(2, 20, 8, 2, F32, padded=0.2)
    ok = dict(valid=valid)
    for args, kw in [((logits.double(), ids), ok), ((logits, ids.float()), ok), ((logits, ids[:, :10]), ok),
                     ((logits, ids), dict(valid=valid.float())), ((logits, ids), dict(valid=valid[0])),
                     ((logits, None), ok), ((logits, ids), dict(counts=torch.zeros(2, 8, dtype=torch.int64, device="cuda"))),
                     ((logits, None), dict(counts=torch.zeros(2, 7, dtype=torch.int64, device="cuda"))),
                     ((logits, None), dict(counts=torch.zeros(2, 8, device="cuda"))),
                     ((logits, ids[..., :0]), ok), ((logits[..., :0], ids), ok), ((logits.cpu(), ids), ok),
                     ((logits, ids.cpu()), ok), ((logits[0, 0], ids[0, 0]), {}), ((logits, ids), dict(reduction="all"))]:
        with pytest.raises(ValueError):
            apml.balance_loss(*args, **kw)
    with pytest.raises(apml.ApmlError):
        apml.balance_loss(torch.zeros(4, 1025, device="cuda"), torch.zeros(4, 1, dtype=torch.int64, device="cuda"))
    with pytest.raises(apml.ApmlError):
        apml.balance_loss(logits, ids, z_weight=float("inf"))
    for args in [(ids.float(), 8), (ids, 0), (ids[0, 0], 8), (ids.cpu(), 8)]:
        with pytest.raises(ValueError):
            apml.expert_counts(*args)
    with pytest.raises(apml.ApmlError):
        apml.expert_counts(ids, 1025)


def test_a_training_step_of_all_losses_together():
    """Predicted points, their descriptors matched to the reference's, tokens of a code book and a router:
    the losses add up, and each input's gradient is its own loss's."""
    g = torch.Generator(device="cuda").manual_seed(9)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    points, ref = rand(2, 256, 3).requires_grad_(True), rand(2, 256, 3)
    feats, feats_ref = rand(2, 256, 64).requires_grad_(True), rand(2, 256, 64).requires_grad_(True)
    match = torch.stack([torch.randperm(256, device="cuda", generator=g) for _ in range(2)])
    book = rand(500, 64).mul(0.25).requires_grad_(True)
    token = torch.randint(0, 500, (2, 256), device="cuda", generator=g)
    router = rand(2, 256, 16).requires_grad_(True)
    chosen = router.detach().topk(2, -1).indices

    def losses():
        shape = apml.apml_loss(points, ref)
        matching = apml.linear_ce_loss(feats, feats_ref, match, scale=0.3)
        tokens = apml.linear_ce_loss(feats, book, token, z_weight=1e-4)
        balance, counts = apml.balance_loss(router, chosen, z_weight=1e-3)
        return shape, matching, tokens, balance

    parts = losses()
    leaves = (points, feats, feats_ref, book, router)
    total = parts[0] + 0.5 * parts[1] + 2.0 * parts[2] + 0.01 * parts[3]
    got = torch.autograd.grad(total, leaves)
    a, b, c, d = losses()
    gp = torch.autograd.grad(a, points)[0]
    gm = torch.autograd.grad(b, (feats, feats_ref))
    gt = torch.autograd.grad(c, (feats, book))
    gr = torch.autograd.grad(d, router)[0]
    near = lambda u, v: torch.testing.assert_close(u, v, rtol=1e-5, atol=1e-9)  # noqa: E731
    near(got[0], gp)
    near(got[1], 0.5 * gm[0] + 2.0 * gt[0])
    near(got[2], 0.5 * gm[1])
    near(got[3], 2.0 * gt[1])
    near(got[4], 0.01 * gr)
    r = oracle.linear_ce(feats.detach(), feats_ref.detach(), match, scale=0.3)
    oracle.within(gm[0], r["grad_x"], r["grad_x_tol"], "descriptors")


@pytest.mark.parametrize("mode", [torch.no_grad, torch.inference_mode])
def test_measured_without_gradients(mode):
    logits, ids, valid = make(2, 100, 16, 2, BF16, padded=0.2)
    want, tokens = apml.balance_loss(logits, ids, valid=valid)
    with mode():
        got, count = apml.balance_loss(logits, ids, valid=valid)
        again, _ = apml.balance_loss(logits, counts=count, valid=valid)
    assert torch.equal(got, want) and torch.equal(again, want) and torch.equal(count, tokens)
    with pytest.raises(ValueError, match="number"):
        apml.balance_loss(logits, ids, valid=valid, z_weight=torch.zeros(()))


@pytest.mark.parametrize("slots_dropped", [0.0, 1e-3, 0.05])
@pytest.mark.parametrize("experts", [8, 21])
def test_shares_that_are_nearly_equal(experts, slots_dropped):
    """Every expert chosen by every token: the gradient is what is left of equal shares."""
    logits, ids, valid = make(2, 3001, experts, experts, F32, dropped=slots_dropped, padded=0.2)
    ids = torch.where(ids < 0, ids, torch.arange(experts, device="cuda"))
    leaf = logits.clone().requires_grad_(True)
    loss, counts = apml.balance_loss(leaf, ids, valid=valid)
    got = torch.autograd.grad(loss, leaf)[0].double()
    p = torch.where(valid.unsqueeze(-1), torch.softmax(logits.double(), -1), 0.0)
    c = counts.double()
    d = (experts * (c - c.amin(-1, keepdim=True)) / c.sum(-1, keepdim=True)).unsqueeze(1)
    g = 1.0 / (2 * valid.sum(-1).double()).view(2, 1, 1)
    dot = (p * d).sum(-1, keepdim=True)
    # p is off by 3 * 2^-17 at most, the sum over the experts by a step each
    tol = g * p * (d + dot) * (3 * 2.0 ** -17 + (experts + 16) * 2.0 ** -24) + 2.0 ** -149
    assert ((got - g * p * (d - dot)).abs() <= tol).all()
    if slots_dropped == 0.0:
        assert (counts == counts[:, :1]).all() and not got.any()


@pytest.mark.parametrize("experts,tokens,dtype,low", [(2, 524288, F16, -1.375), (2, 524288, F16, 2.25),
                                                      (8, 262144, BF16, -1.375), (4, 262144, F32, 2.25)],
                         ids=["2 f16", "2 f16 other", "8 bf16", "4 f32"])
def test_long_samples_of_equal_tokens(experts, tokens, dtype, low):
    """1024 samples, each a chunk of its own, whose tokens add the same number to a sum again and again."""
    row = torch.zeros(experts, device="cuda", dtype=dtype)
    row[0] = low
    logits = row.expand(1024, tokens, experts).contiguous()
    counts = torch.zeros(1024, experts, device="cuda", dtype=torch.int64)
    counts[:, 0] = 7
    z = row.double()
    want = experts * torch.softmax(z, 0)[0]
    # at most 128 such sums in float32, off by half as many half steps of the last; the exponentials,
    # the softmax's sum and quotient 2^-20
    rel = 64 * 2.0 ** -24 + 2.0 ** -20
    loss, _ = apml.balance_loss(logits, counts=counts, reduction="none")
    oracle.within(loss, want.expand(1024), want.expand(1024) * rel, "loss")
    loss, _ = apml.balance_loss(logits, counts=counts, reduction="none", z_weight=1.0)
    want = want + torch.logsumexp(z, 0).square()
    oracle.within(loss, want.expand(1024), want.expand(1024) * (rel + 2.0 ** -20), "loss")
