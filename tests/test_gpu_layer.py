"""A layer run through the public calls, forward and backward, as a program uses them: norm -> route -> dispatch -> experts -> combine,
and the way back; every stage is held to its plain form on what the stage before it left."""
import numpy as np
import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

binding = pytest.importorskip("paper_2609_36301_b200.binding")

EPS = 1e-6


def close(got, want, rel):
    """2-norm: what rounding rows of the stages between leaves."""
    d = (got.double() - want).norm() / want.norm()
    assert d <= rel, f"{float(d):.3e}"


@pytest.mark.parametrize("T,h,r,M,k,s", [(1000, 512, 32, 256, 4, 64), (300, 264, 16, 1024, 6, 40), (5, 256, 16, 128, 2, 64)])
def test_training_layer(T, h, r, M, k, s):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T)
    rn = lambda *n: torch.randn(n, generator=gen, device="cuda")  # noqa: E731
    R1, R2 = (rn(h, r) * h ** -0.5).bfloat16(), (rn(r, M) * r ** -0.5).bfloat16()
    W1, W2 = (rn(M, h, 2 * s) * h ** -0.5).bfloat16(), (rn(M, s, h) * 1.7 * s ** -0.5).bfloat16()
    w_in, w_post, scale, w_next = (1 + 0.1 * rn(h) for _ in range(4))
    stream = rn(T, h)                                                # the residual stream in fp32
    X = binding.combine(None, None, stream, w_pre=w_in, eps=EPS).x
    routed = binding.route(X, R1, R2, k)
    offsets = torch.empty(M + 1, device="cuda", dtype=torch.int32)
    pairs = torch.empty(T * k, device="cuda", dtype=torch.int32)
    binding.more_dispatch(routed.idx, routed.counts, offsets, pairs)
    mlp = binding.experts(X, W1, W2, routed.idx, offsets, pairs, want_hidden=True)
    out = binding.combine(mlp.y, routed.gate, stream, w_post, scale, w_next, eps=EPS, want_sum=True)

    y, y_tol, _, _ = ref.experts(X, W1, W2, offsets, pairs, k)
    ref.within(mlp.y, y, y_tol, "y")
    want = ref.combine(y, routed.gate, stream, w_post, scale, w_next, EPS, T, k, h)
    # a rounded activation and a rounded row, each half a step of 2^-8 at the most, in the terms of a sum; then the output's own
    close(out.residual, want[0], 2 * ref.U)
    close(out.x, want[1], 3 * ref.U)

    dres, dx = 0.1 * rn(T, h), (0.1 * rn(T, h)).bfloat16()
    back = binding.combine_backward(dres, dx, out.sum, out.residual, w_post, scale, w_next, eps=EPS)
    grads = binding.experts_backward(X, W1, W2, routed.idx, offsets, pairs, routed.gate, mlp.hidden, back.dsum)
    inner = binding.combine_backward(back.dresidual, grads.dx, None, stream, None, None, w_in, eps=EPS)
    for name, (value, tol) in zip(("dx", "dgate", "dw1", "dw2"),
                                  ref.experts_backward(X, W1, W2, offsets, pairs, routed.gate, mlp.hidden, back.dsum)):
        ref.within(getattr(grads, name), value, tol, name)

    # end to end, in 64 bits, with the expert ids and gates that the router chose
    leaves = [t.double().requires_grad_() for t in (stream, W1, W2, w_post, scale, w_next, w_in, routed.gate)]
    st, a, b, wp, sc, wn, wi, gt = leaves
    x = st / ref.rms(st, EPS) * wi
    e = routed.idx.long().reshape(-1)
    u = torch.bmm(x.repeat_interleave(k, 0)[:, None], a[e])
    act = torch.nn.functional.silu(u[..., :s]) * u[..., s:]
    rows = torch.bmm(act, b[e]).view(T, k, h)
    yy = (rows * gt[..., None]).sum(1)
    rr = st + sc * wp * yy / ref.rms(yy, EPS)
    xx = rr / ref.rms(rr, EPS) * wn
    ((rr * dres.double()).sum() + (xx * dx.double()).sum()).backward()
    # X, hidden, du and the rows are rounded on the way (half a step each, in sums); 2-norms stay within a few of them
    for got, leaf in ((inner.dresidual, st), (grads.dw1, a), (grads.dw2, b), (back.dw_post, wp), (back.dscale, sc), (back.dw_pre, wn),
                      (inner.dw_pre, wi), (grads.dgate, gt)):
        close(got, leaf.grad, 4 * ref.U)


@pytest.mark.parametrize("T", [1, 7])
def test_decoding_layer(T):
    """A step of a few tokens, without dispatch, captured into a graph that is replayed on new tokens."""
    h, r, M, k, s = 512, 32, 4096, 8, 64
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T)
    rn = lambda *n: torch.randn(n, generator=gen, device="cuda")  # noqa: E731
    R1, R2 = (rn(h, r) * h ** -0.5).bfloat16(), (rn(r, M) * r ** -0.5).bfloat16()
    W1, W2 = (rn(M, h, 2 * s) * h ** -0.5).bfloat16(), (rn(M, s, h) * 1.7 * s ** -0.5).bfloat16()
    w_in, w_next = 1 + 0.1 * rn(h), 1 + 0.1 * rn(h)
    stream = rn(T, h).bfloat16()

    def step():
        X = binding.combine(None, None, stream, w_pre=w_in, eps=EPS).x
        routed = binding.route(X, R1, R2, k)
        y = binding.experts(X, W1, W2, routed.idx).y
        return X, routed, y, binding.combine(y, routed.gate, stream, w_pre=w_next, eps=EPS)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        X, routed, y, out = step()
    for _ in range(3):
        stream.copy_(rn(T, h))
        graph.replay()
        torch.cuda.synchronize()
        offsets, pairs = ref.lists(routed.idx, M)
        want, tol, _, _ = ref.experts(X, W1, W2, offsets, pairs, k, rounded=False)
        ref.within(y, want, tol, "y")
        close(out.x, ref.combine(y, routed.gate, stream, None, None, w_next, EPS, T, k, h)[1], ref.U)
        assert np.array_equal(np.bincount(routed.idx.cpu().numpy().ravel(), minlength=M), routed.counts.cpu().numpy())
