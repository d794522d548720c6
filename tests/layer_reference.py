"""Plain 64-bit forms of the operators behind the router, with bounds on how far a 32-bit computation on bf16 operands may be from
them.  ``U`` is half a step of bf16 relative to the value; a 32-bit sum of K products is off by at most K 2^-23 times the sum of
their magnitudes (one truncation per addition), a 32-bit sigmoid and its neighbours by 2^-20 of the magnitudes that go in."""
import torch

U = 2.0 ** -8
F = 2.0 ** -20


def acc(terms, magnitude):
    return terms * 2.0 ** -23 * magnitude


def lists(idx, M):
    """offsets, pairs (in ascending order inside a run) of the ids that name an expert."""
    flat = idx.reshape(-1).long().cpu()
    place = torch.argsort(torch.where((flat < 0) | (flat >= M), M, flat), stable=True)
    counts = torch.bincount(flat[(flat >= 0) & (flat < M)], minlength=M)
    offsets = torch.zeros(M + 1, dtype=torch.int32)
    offsets[1:] = counts.cumsum(0)
    return offsets.to(idx.device), place.to(torch.int32).to(idx.device)


def runs(offsets, pairs):
    b = offsets.tolist()
    for e in range(len(b) - 1):
        if b[e + 1] > b[e]:
            yield e, b[e], b[e + 1], pairs[b[e]:b[e + 1]].long()


def experts(X, W1, W2, offsets, pairs, k, rounded=True):
    """y, hidden and their bounds.  ``rounded``: the activation is rounded to bf16 on the way."""
    T, h = X.shape
    s = W2.shape[1]
    z = lambda *n: torch.zeros(n, dtype=torch.float64, device=X.device)  # noqa: E731
    y, y_tol, hid, hid_tol = z(T * k, h), z(T * k, h), z(T * k, 2 * s), z(T * k, 2 * s)
    for e, a, b, p in runs(offsets, pairs):
        x, w1, w2 = X[p // k].double(), W1[e].double(), W2[e].double()
        u = x @ w1
        du = acc(h, x.abs() @ w1.abs())
        g, up = u[:, :s], u[:, s:]
        silu = g * torch.sigmoid(g)
        act = silu * up
        da = 1.1 * du[:, :s] * up.abs() + silu.abs() * du[:, s:] + 1.1 * du[:, :s] * du[:, s:] + F * act.abs()
        if rounded:
            da = da + U * (act.abs() + da)
        y[p] = act @ w2
        y_tol[p] = da @ w2.abs() + acc(s, (act.abs() + da) @ w2.abs())
        hid[a:b], hid_tol[a:b] = u, du
    y_tol += U * (y.abs() + y_tol) + 1e-30
    hid_tol += U * (hid.abs() + hid_tol) + 1e-30
    return y, y_tol, hid, hid_tol


def experts_backward(X, W1, W2, offsets, pairs, gate, hidden, dout):
    """dx, dgate, dw1, dw2, each with its bound."""
    T, h = X.shape
    M, s, _ = W2.shape
    k = gate.shape[1]
    z = lambda *n: torch.zeros(n, dtype=torch.float64, device=X.device)  # noqa: E731
    dx, dx_tol, dgate, dgate_tol = z(T, h), z(T, h), z(T * k), z(T * k)
    dw1, dw1_tol, dw2, dw2_tol = z(M, h, 2 * s), z(M, h, 2 * s), z(M, s, h), z(M, s, h)
    flat = gate.reshape(-1).double()
    for e, a, b, p in runs(offsets, pairs):
        x, d, w1, w2 = X[p // k].double(), dout[p // k].double(), W1[e].double(), W2[e].double()
        u, gt = hidden[a:b].double(), flat[p][:, None]
        g, up = u[:, :s], u[:, s:]
        sg = torch.sigmoid(g)
        silu = g * sg
        act = silu * up
        c = d @ w2.T
        dc = acc(h, d.abs() @ w2.abs().T)
        dgate[p] = (c * act).sum(-1)
        size = ((c.abs() + dc) * act.abs()).sum(-1)
        dgate_tol[p] = (dc * act.abs()).sum(-1) + (F + s * 2.0 ** -23) * size
        f = torch.cat((up * sg * (1 + g * (1 - sg)), silu), -1)
        size_f = torch.cat((up.abs() * (1 + g.abs()), silu.abs()), -1)
        cc, dcc = torch.cat((c, c), -1), torch.cat((dc, dc), -1)
        du = gt * cc * f
        du_tol = gt.abs() * (dcc * f.abs() + F * (cc.abs() + dcc) * size_f)
        du_tol = du_tol + U * (du.abs() + du_tol) + 1e-40
        rows = du @ w1.T
        rows_tol = du_tol @ w1.abs().T + acc(2 * s, (du.abs() + du_tol) @ w1.abs().T)
        # a slot's row in fp16 behind a power of two: half a step is 2^-11, or 2^-39 of the largest of the row's columns
        rows_tol = rows_tol + 2.0 ** -11 * (rows.abs() + rows_tol) + 2.0 ** -38 * (rows.abs() + rows_tol).amax(-1, keepdim=True)
        dx.index_add_(0, p // k, rows)
        dx_tol.index_add_(0, p // k, rows_tol)
        dw1[e] = x.T @ du
        dw1_tol[e] = x.abs().T @ du_tol + acc(b - a + 16, x.abs().T @ (du.abs() + du_tol))
        ga = gt * act
        ga_tol = (U + F) * ga.abs() + 1e-40
        dw2[e] = ga.T @ d
        dw2_tol[e] = ga_tol.T @ d.abs() + acc(b - a + 16, (ga.abs() + ga_tol).T @ d.abs())
    dx_tol += U * (dx.abs() + dx_tol) + k * 2.0 ** -23 * (dx.abs() + dx_tol) + 1e-30
    for v, tol in ((dw1, dw1_tol), (dw2, dw2_tol)):
        tol += U * (v.abs() + tol) + 1e-30
    return (dx, dx_tol), (dgate.view(T, k), dgate_tol.view(T, k) + 1e-30), (dw1, dw1_tol), (dw2, dw2_tol)


def rms(v, eps):
    return (v.square().mean(-1, keepdim=True) + eps).sqrt()


def combine(Y, gate, residual, w_post, scale, w_pre, eps, T, k, h):
    """residual, x, sum in 64 bits (any of the inputs may be None)."""
    like = next(t for t in (Y, residual) if t is not None)
    y = torch.zeros((T, h), dtype=torch.float64, device=like.device)
    if Y is not None:
        rows = Y.double().view(T, k, h)
        y = (rows * gate.double()[..., None]).nan_to_num(0.0).sum(1) if gate is not None else rows.sum(1)
    n = y
    if Y is not None:
        n = y / rms(y, eps) * w_post.double() if w_post is not None else y
        n = n * scale.double() if scale is not None else n
    r = n + residual.double() if residual is not None else n
    x = r / rms(r, eps) * w_pre.double() if w_pre is not None else None
    return r, x, y


def combine_backward(dres, dx, y, r, w_post, scale, w_pre, eps):
    """dresidual, dsum, dw_post, dscale, dw_pre in 64 bits."""
    like = dres if dres is not None else dx
    g = torch.zeros(like.shape, dtype=torch.float64, device=like.device) if dres is None else dres.double()
    dw_pre = None
    if dx is not None:
        rd, v = r.double(), dx.double() * w_pre.double()
        m = rms(rd, eps)
        g = g + (v - rd / m * (rd / m * v).mean(-1, keepdim=True)) / m
        dw_pre = (dx.double() * rd / m).sum(0)
    u = g * scale.double() if scale is not None else g
    dw_post = dscale = None
    hat = None
    if y is not None:
        yd = y.double()
        m = rms(yd, eps) if w_post is not None else torch.ones_like(yd[:, :1])
        hat = yd / m
        both = (g * hat).sum(0)
        dscale = both * (w_post.double() if w_post is not None else 1)
        dw_post = both * (scale.double() if scale is not None else 1)
    if w_post is not None:
        u = u * w_post.double()
        u = (u - hat * (hat * u).mean(-1, keepdim=True)) / m
    return g, u, dw_post, dscale, dw_pre


def within(got, want, tol, what):
    err = (got.double() - want).abs()
    bad = ~(err <= tol)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} values off; worst {float((err / tol).nan_to_num(9e9).max()):.3g} "
                           f"of the bound, first at {tuple(int(i) for i in bad.nonzero()[0])}")
