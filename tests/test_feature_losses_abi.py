"""The feature losses' C entry points answer bad arguments before any HIP call, so without a device."""
import ctypes

import pytest
import torch

import paper_2512_19743_amd as apml
from paper_2512_19743_amd import _lib

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x1001)


def ce_desc(**kw):
    d = _lib.apml_linear_ce_desc()
    _lib.load().apml_linear_ce_desc_default(ctypes.byref(d))
    d.rows, d.classes, d.dim = 8, 16, 32
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def balance_desc(**kw):
    d = _lib.apml_balance_desc()
    _lib.load().apml_balance_desc_default(ctypes.byref(d))
    d.tokens, d.experts = 8, 16
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def test_defaults():
    d, b = ce_desc(), balance_desc()
    assert d.struct_size == ctypes.sizeof(d) and b.struct_size == ctypes.sizeof(b)
    assert (d.dtype, d.target_type, d.samples, d.reduction, d.scale, d.z_weight, d.ignore_index) == (0, 0, 1, 2, 1, 0, -100)
    assert (b.dtype, b.index_type, b.samples, b.chosen, b.reduction, b.z_weight) == (0, 0, 1, 1, 2, 0)


BAD_CE = [(dict(struct_size=4), 1), (dict(dtype=3), 1), (dict(dtype=-1), 1), (dict(target_type=2), 1), (dict(reduction=3), 1),
          (dict(samples=0), 1), (dict(rows=0), 1), (dict(classes=0), 1), (dict(dim=0), 1), (dict(rows=-5), 1),
          (dict(scale=float("inf")), 1), (dict(z_weight=float("nan")), 1), (dict(dim=(1 << 20) + 1), 2),
          (dict(classes=(1 << 26) + 1), 2), (dict(samples=1 << 14, rows=1 << 13), 2), (dict(rows=1 << 26, classes=1 << 26), 2),
          (dict(classes=1 << 26, dim=1 << 20), 2)]


@pytest.mark.parametrize("kw,status", BAD_CE)
def test_linear_ce_refuses_sizes(kw, status):
    lib, d, n = _lib.load(), ce_desc(**kw), ctypes.c_size_t()
    big = 1 << 60
    assert lib.apml_linear_ce_workspace(ctypes.byref(d), None, None, ctypes.byref(n), ctypes.byref(n)) == status
    assert lib.apml_linear_ce_forward(ctypes.byref(d), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, big, None) == status
    assert lib.apml_linear_ce_backward(ctypes.byref(d), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, big, None) == status
    assert lib.apml_last_error()


def test_linear_ce_refuses_pointers_and_workspaces():
    lib, d = _lib.load(), ce_desc()
    ref, n = ctypes.byref(d), ctypes.c_size_t()
    assert lib.apml_linear_ce_workspace(None, None, None, ctypes.byref(n), None) == 1
    assert lib.apml_linear_ce_workspace(ref, None, None, None, None) == 1
    assert lib.apml_linear_ce_workspace(ref, None, None, ctypes.byref(n), None) == 0 and n.value > 0
    forward = lambda x=FAKE, w=FAKE, t=FAKE, loss=FAKE, state=FAKE, ws=FAKE, size=1 << 60: lib.apml_linear_ce_forward(  # noqa: E731
        ref, x, w, t, loss, state, ws, size, None)
    for kw in (dict(x=None), dict(w=None), dict(t=None), dict(loss=None), dict(ws=None), dict(x=ODD), dict(w=ODD),
               dict(t=ODD), dict(state=ODD), dict(ws=ctypes.c_void_p(0x1010)), dict(size=0), dict(size=n.value // 8)):
        assert forward(**kw) == 1, kw
    assert "workspace of" in lib.apml_last_error().decode()
    back = lambda x=FAKE, state=FAKE, g=FAKE, gx=FAKE, gw=FAKE, ws=FAKE, size=1 << 60: lib.apml_linear_ce_backward(  # noqa: E731
        ref, x, FAKE, FAKE, state, g, gx, gw, ws, size, None)
    for kw in (dict(x=None), dict(state=None), dict(g=None), dict(gx=None, gw=None), dict(ws=None), dict(gx=ODD),
               dict(gw=ODD), dict(state=ODD), dict(size=0)):
        assert back(**kw) == 1, kw


def test_workspace_covers_any_alignment():
    lib = _lib.load()
    for kw in (dict(dtype=1, dim=64), dict(dtype=2, dim=72), dict(dtype=0, dim=33), dict(dtype=1, rows=5000, classes=40000)):
        d = ce_desc(**kw)
        sizes = []
        for x, w in ((None, None), (FAKE, FAKE), (ODD, FAKE), (FAKE, ODD)):
            f, b = ctypes.c_size_t(), ctypes.c_size_t()
            assert lib.apml_linear_ce_workspace(ctypes.byref(d), x, w, ctypes.byref(f), ctypes.byref(b)) == 0
            sizes.append((f.value, b.value))
        assert all(s[0] <= sizes[0][0] and s[1] <= sizes[0][1] for s in sizes)


BAD_BALANCE = [(dict(struct_size=4), 1), (dict(dtype=3), 1), (dict(index_type=-1), 1), (dict(reduction=-1), 1),
               (dict(samples=0), 1), (dict(tokens=0), 1), (dict(experts=0), 1), (dict(chosen=0), 1),
               (dict(z_weight=float("nan")), 1), (dict(experts=1025), 2), (dict(samples=(1 << 20) + 1), 2),
               (dict(samples=1 << 11, tokens=1 << 20), 2), (dict(tokens=1 << 28, chosen=8), 2)]


@pytest.mark.parametrize("kw,status", BAD_BALANCE)
def test_balance_refuses_sizes(kw, status):
    lib, d, n = _lib.load(), balance_desc(**kw), ctypes.c_size_t()
    assert lib.apml_balance_workspace(ctypes.byref(d), ctypes.byref(n)) == status
    assert lib.apml_balance_forward(ctypes.byref(d), FAKE, FAKE, None, FAKE, FAKE, FAKE, FAKE, 1 << 60, None) == status
    assert lib.apml_balance_backward(ctypes.byref(d), FAKE, None, FAKE, FAKE, FAKE, None) == status


def test_balance_refuses_pointers_and_workspaces():
    lib, d = _lib.load(), balance_desc()
    ref, n = ctypes.byref(d), ctypes.c_size_t()
    assert lib.apml_balance_workspace(None, ctypes.byref(n)) == 1 and lib.apml_balance_workspace(ref, None) == 1
    assert lib.apml_balance_workspace(ref, ctypes.byref(n)) == 0
    forward = lambda logits=FAKE, index=FAKE, counts=FAKE, loss=FAKE, ws=FAKE, size=1 << 60: lib.apml_balance_forward(  # noqa: E731
        ref, logits, index, None, counts, loss, FAKE, ws, size, None)
    for kw in (dict(logits=None), dict(counts=None), dict(loss=None), dict(ws=None), dict(logits=ODD), dict(index=ODD),
               dict(ws=ctypes.c_void_p(0x1010)), dict(size=n.value - 1)):
        assert forward(**kw) == 1, kw
    back = lambda logits=FAKE, state=FAKE, g=FAKE, out=FAKE: lib.apml_balance_backward(ref, logits, None, state, g, out, None)  # noqa: E731
    for kw in (dict(logits=None), dict(state=None), dict(g=None), dict(out=None), dict(logits=ODD), dict(out=ODD)):
        assert back(**kw) == 1, kw
    counts = lambda index=FAKE, kind=0, s=1, t=8, k=2, e=4, out=FAKE: lib.apml_expert_counts(index, kind, None, s, t, k, e, out, None)  # noqa: E731
    for kw in (dict(index=None), dict(out=None), dict(index=ODD), dict(kind=2), dict(s=0), dict(t=0), dict(k=0), dict(e=0)):
        assert counts(**kw) == 1, kw
    assert counts(e=1025) == 2


def test_binding_refuses_cpu_tensors():
    x, t = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="GPU"):
        apml.linear_ce_loss(x, x, t)
    with pytest.raises(ValueError, match="GPU"):
        apml.balance_loss(x, t.unsqueeze(1))
    with pytest.raises(ValueError, match="GPU"):
        apml.expert_counts(t.unsqueeze(1), 8)


# a dispatch counts its threads in 32 bits
MANY = [dict(rows=1 << 20, classes=1 << 18, dim=64), dict(rows=1 << 26, classes=1 << 12, dim=64),
        dict(samples=1 << 15, rows=1 << 11, classes=1 << 13, dim=64), dict(rows=1 << 20, classes=256, dim=(1 << 15) + 1),
        dict(rows=16, classes=1 << 25, dim=1025), dict(rows=64, classes=1 << 26, dim=4096)]


@pytest.mark.parametrize("kw", MANY)
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_linear_ce_refuses_launches_of_too_many_threads(kw, dtype):
    lib, d, n = _lib.load(), ce_desc(dtype=dtype, **kw), ctypes.c_size_t()
    big = 1 << 62
    assert lib.apml_linear_ce_workspace(ctypes.byref(d), None, None, ctypes.byref(n), ctypes.byref(n)) == 2
    assert lib.apml_linear_ce_forward(ctypes.byref(d), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, big, None) == 2
    assert lib.apml_linear_ce_backward(ctypes.byref(d), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, big, None) == 2


@pytest.mark.parametrize("kw", [dict(rows=1 << 20, classes=1 << 17, dim=4096), dict(rows=1 << 26, classes=1000, dim=64),
                                dict(rows=1, classes=1 << 26, dim=512), dict(samples=1 << 20, rows=64, classes=64, dim=64)])
def test_large_calls_are_taken(kw):
    lib, d, n = _lib.load(), ce_desc(dtype=1, **kw), ctypes.c_size_t()
    assert lib.apml_linear_ce_workspace(ctypes.byref(d), FAKE, FAKE, ctypes.byref(n), ctypes.byref(n)) == 0 and n.value > 0


def test_results_off_their_elements_are_refused():
    lib, d, b = _lib.load(), ce_desc(), balance_desc()
    big = 1 << 60
    assert lib.apml_linear_ce_forward(ctypes.byref(d), FAKE, FAKE, FAKE, ODD, FAKE, FAKE, big, None) == 1
    for counts, loss, state in ((ctypes.c_void_p(FAKE.value + 4), FAKE, FAKE), (FAKE, ODD, FAKE), (FAKE, FAKE, ODD)):
        assert lib.apml_balance_forward(ctypes.byref(b), FAKE, FAKE, None, counts, loss, state, FAKE, big, None) == 1
    for state, g in ((ODD, FAKE), (FAKE, ODD)):
        assert lib.apml_balance_backward(ctypes.byref(b), FAKE, None, state, g, FAKE, None) == 1
    assert lib.apml_expert_counts(FAKE, 0, None, 1, 8, 2, 4, ctypes.c_void_p(FAKE.value + 4), None) == 1


@pytest.mark.parametrize("kw", [dict(dtype=1, rows=1 << 20, classes=40), dict(dtype=1, rows=1 << 22, classes=300),
                                dict(dtype=2, rows=1 << 26, classes=13), dict(dtype=0, rows=1 << 22, classes=300, dim=72),
                                dict(dtype=0, rows=1 << 21, classes=5000, dim=64), dict(dtype=1, rows=1 << 20, classes=1 << 17),
                                dict(dtype=1, samples=4, rows=1 << 20, classes=700), dict(dtype=1, rows=524289, classes=256),
                                dict(dtype=0, rows=8192, classes=131072, dim=1024), dict(dtype=1, samples=4096, rows=300, classes=300)],
                         ids=str)
def test_backward_workspace_keeps_to_its_piece(kw):
    """Beside copies of x and w, the rows' coefficients and sums of gradients in float32, all of the
    inputs' size, the backward pass has a piece of the logits' gradient of 256 MB (rows up to 192
    elements longer than the piece) at any sizes."""
    lib, d, n = _lib.load(), ce_desc(**{"dim": 64, **kw}), ctypes.c_size_t()
    assert lib.apml_linear_ce_workspace(ctypes.byref(d), FAKE, FAKE, None, ctypes.byref(n)) == 0
    up = lambda a: (a + 63) // 64 * 64  # noqa: E731
    size, dim = (6 if d.dtype == 0 else 2), up(d.dim)
    rows, classes = d.samples * up(d.rows), d.samples * d.classes
    copies = (2 * rows * dim + classes * dim) * size + 16 * rows
    sums = 4 * (rows + 2 * classes) * dim  # one for x's, two parts for w's
    parts = 64 << 20  # of small gradients, up to 64 each
    assert n.value <= copies + sums + parts + 1.2 * (256 << 20)


@pytest.mark.parametrize("scale,status", [(3e38, 1), (-3e38, 1), (2.3e38, 0), (-2.3e38, 0)])
def test_a_scale_beyond_float32_in_units_of_log_2_is_refused(scale, status):
    """The kernels multiply by scale / log 2, which would be infinite: NaN for a logit of 0."""
    lib, d, n = _lib.load(), ce_desc(scale=scale), ctypes.c_size_t()
    assert lib.apml_linear_ce_workspace(ctypes.byref(d), None, None, ctypes.byref(n), None) == status
    if status:
        assert lib.apml_linear_ce_forward(ctypes.byref(d), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 60, None) == status
        assert lib.apml_linear_ce_backward(ctypes.byref(d), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 60,
                                           None) == status
        assert "scale" in lib.apml_last_error().decode()
