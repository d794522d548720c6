"""The joining of a token's rows with its norms, and its gradients, against their plain 64-bit forms.  Bounds: a 32-bit sum of squares
over a row (a few dozen additions per thread, then a tree) and the inverse root are good to R = 2^-18 relative; what is added up is
bounded by the magnitudes that go in; bf16 outputs add half a step."""
import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

binding = pytest.importorskip("paper_2609_36301_b200.binding")

R = 2.0 ** -18
EPS = 1e-6
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def randn(gen, *n):
    return torch.randn(n, generator=gen, device="cuda")


def weights(gen, h):
    return 1 + 0.1 * randn(gen, h), 0.3 + 0.05 * randn(gen, h), 1 + 0.1 * randn(gen, h)


def half_step(v, dtype):
    return (ref.U if dtype == torch.bfloat16 else 2.0 ** -23) * v.abs()


def forward_bounds(Y, gate, residual, w_post, scale, w_pre, T, k, h, dtype):
    """(residual, x, sum) and their bounds."""
    r, x, y = ref.combine(Y, gate, residual, w_post, scale, w_pre, EPS, T, k, h)
    ty = torch.zeros_like(y)
    n = torch.zeros_like(y)
    if Y is not None:
        g = gate.double()[..., None] if gate is not None else torch.ones((T, k, 1), device="cuda", dtype=torch.float64)
        ty = ref.acc(k + 1, (Y.double().view(T, k, h) * g).abs().nan_to_num(0.0).sum(1))
        n = r - residual.double() if residual is not None else r
    w = (w_post.double().abs() if w_post is not None else 1) * (scale.double().abs() if scale is not None else 1)
    m = ref.rms(y, EPS) if w_post is not None else 1
    spread = (ty.square().mean(-1, keepdim=True).sqrt() / m) if w_post is not None else 0
    tr = w * ty / m + n.abs() * (R + spread) + 2.0 ** -22 * (r.abs() + n.abs())
    tx = None
    if w_pre is not None:
        mr = ref.rms(r, EPS)
        tx = w_pre.double().abs() * (tr + r.abs() * (R + tr.square().mean(-1, keepdim=True).sqrt() / mr)) / mr
        tx = tx + half_step(x.abs() + tx, torch.bfloat16) + 1e-30
    return (r, tr + half_step(r.abs() + tr, dtype) + 1e-30), (x, tx), (y, ty + half_step(y.abs() + ty, torch.bfloat16) + 1e-30)


SHAPES = [(1, 8, 1), (1, 4096, 16), (3, 64, 2), (64, 4096, 16), (37, 2048, 8), (5, 8192, 3), (1183, 264, 4), (1185, 264, 4), (1500, 512, 4),
          (1300, 1000, 6), (1301, 1032, 5), (2000, 520, 1), (1200, 8192, 2), (1190, 8, 32), (1203, 2056, 7)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,h,k", SHAPES)
def test_forward(T, h, k, dtype):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T + h)
    Y, gate, res = randn(gen, T * k, h).bfloat16(), randn(gen, T, k).softmax(-1), (2 * randn(gen, T, h)).to(DT[dtype])
    w = weights(gen, h)
    got = binding.combine(Y, gate, res, *w, eps=EPS, want_sum=True)
    want = forward_bounds(Y, gate, res, *w, T, k, h, DT[dtype])
    for name, value, (exact, tol) in zip(("residual", "x", "sum"), (got.residual, got.x, got.sum), want):
        ref.within(value, exact, tol, name)
    assert got.residual.dtype == DT[dtype]


@pytest.mark.parametrize("have", ["gate", "residual", "w_post", "scale", "w_pre", "only_norm", "rows"])
@pytest.mark.parametrize("T,h,k", [(7, 256, 3), (1400, 256, 3), (1400, 1200, 2)])
def test_forward_without(T, h, k, have):
    """Each of the parts left out, the norm alone, and rows that are only added up."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    Y, gate, res = randn(gen, T * k, h).bfloat16(), randn(gen, T, k).softmax(-1), randn(gen, T, h).bfloat16()
    w_post, scale, w_pre = weights(gen, h)
    args = dict(Y=Y, gate=gate, residual=res, w_post=w_post, scale=scale, w_pre=w_pre)
    if have in args:
        args[have] = None
    if have == "only_norm":
        args.update(Y=None, gate=None)
    if have == "rows":
        args.update(gate=None, residual=None, w_post=None, scale=None, w_pre=None)
    got = binding.combine(**args, eps=EPS, k=k if args["Y"] is not None else 0)
    (r, tr), (x, tx), _ = forward_bounds(*[args[n] for n in ("Y", "gate", "residual", "w_post", "scale", "w_pre")], T, k, h, torch.bfloat16)
    ref.within(got.residual, r, tr, "residual")
    assert (got.x is None) == (args["w_pre"] is None)
    if got.x is not None:
        ref.within(got.x, x, tx, "x")


@pytest.mark.parametrize("T,h,k", [(30000, 4096, 1), (30000, 1024, 2), (9000, 8192, 1)])
def test_residual_and_sum_do_not_depend_on_the_next_norm(T, h, k):
    """Without the next block's norm a CTA goes from token to token with a sum over the row less."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T)
    Y, gate, res = randn(gen, T * k, h).bfloat16(), randn(gen, T, k).softmax(-1), randn(gen, T, h).bfloat16()
    Y *= torch.exp2(torch.randint(-9, 9, (T, 1, 1), generator=gen, device="cuda").float()).expand(T, k, 1).reshape(T * k, 1).bfloat16()
    w_post, scale, w_pre = weights(gen, h)
    full = binding.combine(Y, gate, res, w_post, scale, w_pre, eps=EPS, want_sum=True)
    for _ in range(5):
        got = binding.combine(Y, gate, res, w_post, scale, None, eps=EPS, want_sum=True)
        assert got.x is None and torch.equal(got.residual, full.residual) and torch.equal(got.sum, full.sum)


def test_slots_with_a_gate_of_zero_are_not_read():
    T, h, k = 40, 512, 4
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    Y, gate, res = randn(gen, T * k, h).bfloat16(), randn(gen, T, k).softmax(-1), randn(gen, T, h).bfloat16()
    gate[::3, 1] = 0
    gate[5] = 0                                              # a token without any expert
    w = weights(gen, h)
    want = forward_bounds(Y, gate, res, *w, T, k, h, torch.bfloat16)
    Y[(gate == 0).reshape(-1)] = float("nan")
    got = binding.combine(Y, gate, res, *w, eps=EPS, want_sum=True)
    for value, (exact, tol) in zip((got.residual, got.x, got.sum), want):
        ref.within(value, exact, tol, "out")
    assert torch.equal(got.residual[5], res[5])


def test_large_and_small_rows():
    """Rows of 1e4 and 1e-4: the norms bring both to the same size; an all-zero row stays zero."""
    T, h, k = 1300, 640, 2
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    Y, gate = randn(gen, T * k, h), randn(gen, T, k).softmax(-1)
    Y[: T // 3] *= 1e4
    Y[T // 3: T] *= 1e-4
    Y[-4:] = 0
    Y = Y.bfloat16()
    w = weights(gen, h)
    got = binding.combine(Y, gate, None, *w, eps=EPS)
    (r, tr), (x, tx), _ = forward_bounds(Y, gate, None, *w, T, k, h, torch.bfloat16)
    ref.within(got.residual, r, tr, "residual")
    ref.within(got.x, x, tx, "x")
    assert not got.x[-2:].any()


def backward_bounds(dres, dx, y, r, w_post, scale, w_pre, dtype):
    g, dy, dwp, dsc, dwn = ref.combine_backward(dres, dx, y, r, w_post, scale, w_pre, EPS)
    tg = torch.zeros_like(g)
    if dres is not None:
        tg = tg + 2.0 ** -22 * dres.double().abs()
    twn = None
    T = g.shape[0]
    if dx is not None:
        m = ref.rms(r.double(), EPS)
        hat, v = (r.double() / m).abs(), (dx.double() * w_pre.double()).abs()
        tg = tg + R * (v + hat * (hat * v).mean(-1, keepdim=True)) / m * 2
        twn = (R + T * 2.0 ** -23) * (dx.double().abs() * hat).sum(0) + 1e-30
    w = (scale.double().abs() if scale is not None else 1) * (w_post.double().abs() if w_post is not None else 1)
    tu, u = w * tg, w * g.abs()
    tdy, tS = tu + 2.0 ** -22 * u, None
    if y is not None:
        my = ref.rms(y.double(), EPS) if w_post is not None else torch.ones_like(g[:, :1])
        hy = y.double().abs() / my
        S = (tg * hy + R * g.abs() * hy).sum(0) + T * 2.0 ** -23 * (g.abs() * hy).sum(0)
        tS = (S * (scale.double().abs() if scale is not None else 1) + 1e-30, S * (w_post.double().abs() if w_post is not None else 1) + 1e-30)
        if w_post is not None:
            tdy = (tu + 2 * R * u + hy * (hy * (tu + 2 * R * u)).mean(-1, keepdim=True) + 2 * R * hy * (hy * u).mean(-1, keepdim=True)) / my
    return ((g, tg + half_step(g.abs() + tg, dtype) + 1e-30), (dy, tdy + half_step(dy.abs() + tdy, torch.bfloat16) + 1e-30),
            (dwp, tS and tS[0]), (dsc, tS and tS[1]), (dwn, twn))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,h,k", SHAPES)
def test_backward(T, h, k, dtype):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T + h + 1)
    y, r = (randn(gen, T, h) * k ** -0.5).bfloat16(), (2 * randn(gen, T, h)).to(DT[dtype])
    dres, dx = (0.02 * randn(gen, T, h)).to(DT[dtype]), (0.02 * randn(gen, T, h)).bfloat16()
    w = weights(gen, h)
    got = binding.combine_backward(dres, dx, y, r, *w, eps=EPS)
    want = backward_bounds(dres, dx, y, r, *w, DT[dtype])
    for name, (exact, tol) in zip(("dresidual", "dsum", "dw_post", "dscale", "dw_pre"), want):
        ref.within(getattr(got, name), exact, tol, name)


@pytest.mark.parametrize("have", ["dres", "dx", "w_post", "scale", "plain"])
@pytest.mark.parametrize("T,h", [(9, 256), (1400, 256), (1400, 1200)])
def test_backward_without(T, h, have):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    a = dict(dres=randn(gen, T, h).bfloat16(), dx=randn(gen, T, h).bfloat16(), y=randn(gen, T, h).bfloat16(), r=randn(gen, T, h).bfloat16())
    a["w_post"], a["scale"], a["w_pre"] = weights(gen, h)
    if have in a:
        a[have] = None
    if have == "plain":                                      # rows that were added as they are, no norm behind
        a.update(dx=None, y=None, w_post=None, scale=None, w_pre=None, r=None)
    if have == "dx":
        a.update(w_pre=None, r=None)
    names = ("dres", "dx", "y", "r", "w_post", "scale", "w_pre")
    got = binding.combine_backward(*[a[n] for n in names], eps=EPS)
    want = backward_bounds(*[a[n] for n in names], torch.bfloat16)
    asked = dict(dw_post=a["w_post"], dscale=a["scale"], dw_pre=a["dx"])
    for name, (exact, tol) in zip(("dresidual", "dsum", "dw_post", "dscale", "dw_pre"), want):
        value = getattr(got, name)
        if name in asked and asked[name] is None:
            assert value is None
        else:
            ref.within(value, exact, tol, name)


def test_reference_gradients_agree_with_differences():
    T, h, k = 4, 24, 3
    gen = torch.Generator(device="cuda")
    gen.manual_seed(11)
    Y, gate, res, dres, dx = (randn(gen, *n).double() for n in ((T * k, h), (T, k), (T, h), (T, h), (T, h)))
    w = [v.double() for v in weights(gen, h)]

    def loss(Y, res, *w):
        r, x, _ = ref.combine(Y, gate, res, *w, EPS, T, k, h)
        return float((r * dres).sum() + (x * dx).sum())

    r, _, y = ref.combine(Y, gate, res, *w, EPS, T, k, h)
    dr, dy, dwp, dsc, dwn = ref.combine_backward(dres, dx, y, r, *w, EPS)
    for which, grad in enumerate(((dy[:, None] * gate[..., None]).reshape(T * k, h), dr, dwp, dsc, dwn)):
        args = [Y, res, *w]
        direction = torch.randn_like(grad)
        args[which] = args[which] + 1e-5 * direction
        up = loss(*args)
        args[which] = args[which] - 2e-5 * direction
        slope = (up - loss(*args)) / 2e-5
        assert abs(slope - float((grad * direction).sum())) <= 1e-7 * max(1.0, abs(slope))


@pytest.mark.parametrize("T", [50, 1400])
def test_in_place_and_guards(T):
    """The residual stream updated in place; nothing around outputs or behind the workspace is written; the same bits again."""
    h, k = 264, 3
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    Y, gate, res = randn(gen, T * k, h).bfloat16(), randn(gen, T, k).softmax(-1), randn(gen, T, h).bfloat16()
    w = weights(gen, h)
    apart = binding.combine(Y, gate, res, *w, eps=EPS, want_sum=True)
    whole = torch.full((T + 64, h), 3.0, device="cuda").bfloat16()
    stream = whole[32:-32]
    stream.copy_(res)
    x = torch.empty((T, h), device="cuda").bfloat16()
    binding.more_combine(Y, gate, stream, *w, EPS, out_residual=stream, out_x=x)
    assert torch.equal(stream, apart.residual) and torch.equal(x, apart.x)
    assert (whole[:32] == 3).all() and (whole[-32:] == 3).all()
    dres, dx = randn(gen, T, h).bfloat16(), randn(gen, T, h).bfloat16()
    first = binding.combine_backward(dres, dx, apart.sum, apart.residual, *w, eps=EPS)
    need = binding.combine_workspace(T, h)
    ws = torch.full((need + 4096,), 0x5A, device="cuda", dtype=torch.uint8)
    stream.copy_(dres)
    dsum = torch.empty_like(dx)
    grads = [torch.empty(h, device="cuda") for _ in range(3)]
    binding.more_combine_backward(stream, dx, apart.sum, apart.residual, *w, EPS, stream, dsum, *grads, workspace=ws[:need])
    assert torch.equal(stream, first.dresidual) and torch.equal(dsum, first.dsum)
    assert all(torch.equal(a, b) for a, b in zip(grads, (first.dw_post, first.dscale, first.dw_pre)))
    assert (whole[:32] == 3).all() and (whole[-32:] == 3).all() and (ws[need:] == 0x5A).all()


@pytest.mark.parametrize("T", [5, 1400])
def test_no_gradient_of_the_next_norm_and_no_epsilon(T):
    """Where dx is left out nothing of the next norm is worked out, so that an epsilon of zero does no harm."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T)
    dres, y = randn(gen, T, 264).bfloat16(), randn(gen, T, 264).bfloat16()
    got = binding.combine_backward(dres, None, y, None, *weights(gen, 264)[:2], None, eps=0.0)
    again = binding.combine_backward(dres, None, y, None, *weights(gen, 264)[:2], None, eps=1e-12)
    assert torch.equal(got.dresidual, dres) and torch.isfinite(got.dsum).all() and torch.isfinite(got.dscale).all()
    assert torch.equal(again.dresidual, dres)


def test_no_tokens():
    e = torch.empty((0, 64), device="cuda").bfloat16()
    w = [torch.ones(64, device="cuda") for _ in range(3)]
    got = binding.combine(e, torch.empty((0, 2), device="cuda"), e, *w, want_sum=True)
    assert got.residual.shape == got.x.shape == got.sum.shape == (0, 64)
    g = binding.combine_backward(e, e, e, e, *w)
    assert g.dresidual.shape == (0, 64) and not g.dw_post.any() and not g.dscale.any() and not g.dw_pre.any()


def test_rows_beyond_32_bit_offsets():
    T, h, k = 16400, 8192, 17
    Y = torch.zeros((T * k, h), device="cuda", dtype=torch.bfloat16)
    Y[-k:] = 1
    gate = torch.full((T, k), 1 / 16, device="cuda")
    got = binding.combine(Y, gate, None)
    assert (got.residual[-1].float() == torch.tensor(17 / 16).bfloat16().float().item()).all() and not got.residual[:-1].any()


def test_captured_and_on_another_stream():
    T, h, k = 1300, 512, 4
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    Y, gate, res = randn(gen, T * k, h).bfloat16(), randn(gen, T, k).softmax(-1), randn(gen, T, h).bfloat16()
    dres, dx, w = randn(gen, T, h).bfloat16(), randn(gen, T, h).bfloat16(), weights(gen, h)
    direct = binding.combine(Y, gate, res, *w, want_sum=True)
    back = binding.combine_backward(dres, dx, direct.sum, direct.residual, *w)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = binding.combine(Y, gate, res, *w, want_sum=True, stream=stream)
    other_back = binding.combine_backward(dres, dx, other.sum, other.residual, *w, stream=stream)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        caught = binding.combine(Y, gate, res, *w, want_sum=True)
        caught_back = binding.combine_backward(dres, dx, caught.sum, caught.residual, *w)
    graph.replay()
    torch.cuda.synchronize()
    for a in (other, caught):
        assert torch.equal(a.x, direct.x) and torch.equal(a.residual, direct.residual) and torch.equal(a.sum, direct.sum)
    for b in (other_back, caught_back):
        for n in ("dresidual", "dsum", "dw_post", "dscale", "dw_pre"):
            assert torch.equal(getattr(b, n), getattr(back, n))


def test_refusals():
    T, h, k = 6, 64, 2
    Y, gate, res = torch.zeros((T * k, h), device="cuda").bfloat16(), torch.zeros((T, k), device="cuda"), torch.zeros((T, h), device="cuda").bfloat16()
    w = torch.ones(h, device="cuda")
    for bad in (dict(Y=Y.float()), dict(Y=Y[:-1]), dict(gate=gate.bfloat16()), dict(residual=res.half()), dict(residual=res.cpu()), dict(w_post=w[:-8]),
                dict(scale=w.bfloat16()), dict(Y=None, residual=None, gate=None), dict(residual=torch.zeros((T, 2 * h), device="cuda").bfloat16()[:, ::2])):
        with pytest.raises((TypeError, ValueError)):
            binding.combine(**{**dict(Y=Y, gate=gate, residual=res, w_post=w, scale=w, w_pre=w), **bad})
    with pytest.raises(binding.MoreRouteError):
        binding.combine(Y, gate, res, eps=-1.0)
    with pytest.raises(binding.MoreRouteError):
        binding.combine(Y, gate, res, eps=float("nan"))
    with pytest.raises(binding.MoreRouteError):                       # x without its weights
        binding.more_combine(Y, gate, res, None, None, None, EPS, out_x=res.clone())
    with pytest.raises(binding.MoreRouteError):                       # h not a multiple of 8
        binding.combine(Y[:, :60].contiguous(), gate, res[:, :60].contiguous())
    with pytest.raises(binding.MoreRouteError):                       # the norm in front needs the residual that it normed
        binding.combine_backward(res, res, res, None, w, w, w)
    with pytest.raises(binding.MoreRouteError):                       # the norm behind needs the sum
        binding.combine_backward(res, None, None, None, w, None, None)
    with pytest.raises(binding.MoreRouteError):
        binding.combine_backward(res, res, res, res, w, w, w, workspace=torch.empty(16, device="cuda", dtype=torch.uint8))
