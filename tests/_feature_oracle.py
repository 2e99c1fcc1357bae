"""The losses on features and on routed experts in 64 bits, by plain torch, with bounds on how far
single-precision sums and rounded gradients may be from them.

u is the half step of a type relative to a value (bf16 2^-8, fp16 2^-11, fp32 2^-24). A logit is a sum
of dim products in float32, off by at most (dim + 16) 2^-24 sum |x||w| |scale|: `tz` per row, with the
three planes' dropped products in the 16. Exponentials of arguments down to -40 add 40 * 1.45 * 2^-24
and a few steps of the argument's scaling and of the function itself: EXP = 2^-17 in all.
"""
import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
EXP = 2.0 ** -17


def linear_ce(x, w, target, *, scale=1.0, z_weight=0.0, ignore_index=-100, reduction="mean", grad_loss=None):
    """dict of loss, grad_x, grad_w and the bounds loss_tol, grad_x_tol, grad_w_tol, all float64."""
    dtype, shape = x.dtype, x.shape
    batched = w.dim() == 3
    X = x.double() if batched else x.double().reshape(1, -1, x.shape[-1])
    W = w.double() if batched else w.double().unsqueeze(0)
    T = target.long().reshape(X.shape[:2])
    S, R, D = X.shape
    V = W.shape[1]
    used = T != ignore_index
    n = max(1, int(used.sum()))
    up = torch.ones(S, R, dtype=torch.float64, device=x.device)
    if grad_loss is not None:
        up = grad_loss.double().reshape(S, R) if reduction == "none" else up * grad_loss.double()
    if reduction == "mean":
        up = up / n
    u = HALF[dtype]
    out = {k: [] for k in ("rows", "rows_tol", "gx", "gx_tol", "gw", "gw_tol")}
    for s in range(S):
        ok = used[s].unsqueeze(1)
        xs, ws = torch.where(ok, X[s], 0.0), W[s]
        z = (xs @ ws.T) * scale
        tz = (D + 16) * 2.0 ** -24 * abs(scale) * (xs.abs() @ ws.abs().T).amax(1)
        at = T[s].clamp(0, V - 1).unsqueeze(1)
        lse = torch.logsumexp(z, 1)
        p = torch.softmax(z, 1)
        others = p.scatter(1, at, 0.0)
        miss = others.sum(1)
        picked = z.gather(1, at).squeeze(1)
        loss = torch.where(miss < 0.5, -torch.log1p(-miss), lse - picked)
        loss = torch.where(used[s], loss + z_weight * lse.square(), 0.0)
        tol = 2 * tz * (1 + 2 * abs(z_weight) * lse.abs()) + (EXP + 2.0 ** -21) * (1 + loss.abs()) + 2.0 ** -21 * (
            lse.abs() + abs(z_weight) * lse.square())
        out["rows"].append(loss)
        out["rows_tol"].append(torch.where(used[s], tol, 0.0))
        b = torch.where(used[s], up[s] * scale, 0.0).unsqueeze(1)
        c = 2.0 * z_weight * lse.unsqueeze(1) * b
        mine = p.gather(1, at)
        G = ((b + c) * others).scatter(1, at, c * mine - b * miss.unsqueeze(1))
        A = ((b.abs() + c.abs()) * others).scatter(1, at, c.abs() * mine + b.abs() * miss.unsqueeze(1))
        m = 2 * (b.abs() + c.abs())  # at least the power of two that the row is scaled by
        rel = (4 * tz + 2 * EXP).unsqueeze(1) + u + 2.0 ** -20
        floor = m * 2.0 ** -39 if dtype == torch.float16 else m * 2.0 ** -120
        dG = A * rel + torch.where(used[s].unsqueeze(1), floor, 0.0)
        # scale, g / n and their product are float32: below 2^-126 each is off by up
        # to 2^-150, half a step of the subnormal numbers, whatever its size
        dG = dG + 2.0 ** -150 * (2 + up[s].abs().unsqueeze(1) + abs(scale)) * torch.where(used[s].unsqueeze(1), 1.0, 0.0)
        gx, gw = G @ ws, G.T @ xs
        out["gx"].append(gx)
        out["gx_tol"].append(dG @ ws.abs() + A @ ws.abs() * (V + 64) * 2.0 ** -24 + u * gx.abs() + SMALLEST[dtype])
        tw = dG.T @ xs.abs() + A.T @ xs.abs() * (R + 64) * 2.0 ** -24 + u * gw.abs() + SMALLEST[dtype]
        if dtype == torch.float16:  # rows far below the largest upstream gradient fall below the type's range
            tw = tw + (A / m.clamp_min(1e-300)).sum(0).unsqueeze(1) * m.max() * 2.0 ** -25
        out["gw"].append(gw)
        out["gw_tol"].append(tw)
    o = {k: torch.stack(v) for k, v in out.items()}
    rows, tol = o["rows"].reshape(target.shape), o["rows_tol"].reshape(target.shape)
    if reduction != "none":
        rows, tol = rows.sum(), tol.sum() + 2.0 ** -23 * rows.abs().sum()
        if reduction == "mean":
            rows, tol = rows / n, tol / n
    return {"loss": rows, "loss_tol": tol + 1e-37, "grad_x": o["gx"].reshape(shape), "grad_x_tol": o["gx_tol"].reshape(shape),
            "grad_w": o["gw"].reshape(w.shape), "grad_w_tol": o["gw_tol"].reshape(w.shape)}


def counts(experts, num, valid=None):
    ids = experts.long().reshape(-1, *experts.shape[-2:]).cpu()
    out = torch.zeros(ids.shape[0], num, dtype=torch.int64)
    for b in range(ids.shape[0]):
        e = ids[b] if valid is None else ids[b][valid.reshape(ids.shape[0], -1)[b].cpu()]
        e = e.reshape(-1)
        out[b] = torch.bincount(e[(e >= 0) & (e < num)], minlength=num)
    return out.reshape(*experts.shape[:-2], num)


def balance(logits, count, *, valid=None, z_weight=0.0, reduction="mean", grad_loss=None):
    """dict of loss, grad and the bounds loss_tol, grad_tol, all float64."""
    dtype = logits.dtype
    z = logits.double().reshape(-1, *logits.shape[-2:])
    S, T, E = z.shape
    ok = torch.ones(S, T, dtype=torch.bool, device=z.device) if valid is None else valid.reshape(S, T)
    z = torch.where(ok.unsqueeze(-1), z, 0.0)
    c = count.to(z.device).double().reshape(S, E)
    load = E * c / c.sum(1, keepdim=True).clamp_min(1)
    n = ok.sum(1).clamp_min(1).double()
    top = z.amax(-1, keepdim=True)
    none = torch.isneginf(top)
    e = torch.exp(z - torch.where(none, 0.0, top))
    p = torch.where(ok.unsqueeze(-1), e / e.sum(-1, keepdim=True).clamp_min(1e-300), 0.0)
    lse = torch.where(ok & ~none.squeeze(-1), torch.logsumexp(z, -1), 0.0)
    first = (p.sum(1) * load).sum(-1) / n
    loss = first + z_weight * lse.square().sum(1) / n
    off = 2 * EXP + (T + 16) * 2.0 ** -24
    loss_tol = first * off + abs(z_weight) * (lse.square().sum(1) / n) * (off + 2.0 ** -20) + 2.0 ** -23 * loss.abs()
    up = torch.ones(S, dtype=torch.float64, device=z.device)
    if grad_loss is not None:
        up = up * grad_loss.double().reshape(-1)
    if reduction == "mean":
        up = up / S
    g = (up / n).view(S, 1, 1)
    dot = (p * load.unsqueeze(1)).sum(-1, keepdim=True)
    zt = 2.0 * z_weight * lse.unsqueeze(-1)
    grad = g * p * (load.unsqueeze(1) - dot + zt)
    size = g.abs() * p * (load.unsqueeze(1) + dot + zt.abs())
    grad_tol = size * (3 * EXP + (E + 16) * 2.0 ** -24) + HALF[dtype] * grad.abs() + SMALLEST[dtype]
    if reduction == "none":
        loss, loss_tol = loss.reshape(logits.shape[:-2]), loss_tol.reshape(logits.shape[:-2])
    else:
        loss, loss_tol = loss.sum(), loss_tol.sum()
        if reduction == "mean":
            loss, loss_tol = loss / S, loss_tol / S
    return {"loss": loss, "loss_tol": loss_tol + 1e-37, "grad": grad.reshape(logits.shape),
            "grad_tol": grad_tol.reshape(logits.shape)}


def within(got, want, tol, what):
    assert got.shape == want.shape, (what, got.shape, want.shape)
    # a value past the type's largest by more than half a step rounds to infinity
    # (lse^2 of a row of float32's lowest value is 1e77)
    over = want.abs() > torch.finfo(got.dtype).max * (1 + HALF[got.dtype])
    want = torch.where(over, torch.sign(want) * float("inf"), want)
    got = got.double()
    bad = ~((got == want) | ((got - want).abs() <= tol))
    if bad.any():
        i = tuple(int(k) for k in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {float(got[i]):.9g}, "
                             f"oracle {float(want[i]):.9g}, bound {float(tol[i]):.3g}")
