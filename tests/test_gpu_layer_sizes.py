"""The operators behind the router at the ends of their ranges: the widest rows and experts, very many experts, buffers whose offsets
pass 32 bits in each direction, and slots without a gate on every way through the joining norm."""
import pytest
import torch

import layer_reference as ref
from test_gpu_combine import EPS, backward_bounds, forward_bounds, randn, weights
from test_gpu_experts import make

pytestmark = pytest.mark.gpu

binding = pytest.importorskip("paper_2609_36301_b200.binding")


def check_backward(X, W1, W2, idx, offsets, pairs, gate, hidden, dout):
    got = binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate, hidden, dout)
    for name, (value, tol) in zip(("dx", "dgate", "dw1", "dw2"), ref.experts_backward(X, W1, W2, offsets, pairs, gate, hidden, dout)):
        ref.within(getattr(got, name), value, tol, name)


@pytest.mark.parametrize("T,h,s,M,k", [(200, 8192, 8192, 2, 1), (150, 8192, 8, 3, 2), (150, 8, 8192, 3, 2), (130, 8184, 1000, 2, 2)])
def test_widest_rows_and_experts(T, h, s, M, k):
    X, W1, W2, idx, offsets, pairs, gate, dout = make(T, h, s, M, k)
    res = binding.experts(X, W1, W2, idx, offsets, pairs, want_hidden=True, path=binding.EXPERTS_TILES)
    y, y_tol, hid, hid_tol = ref.experts(X, W1, W2, offsets, pairs, k)
    ref.within(res.hidden, hid, hid_tol, "hidden")
    ref.within(res.y, y, y_tol, "y")
    check_backward(X, W1, W2, idx, offsets, pairs, gate, res.hidden, dout)
    assert binding.more_route_status() == 0


@pytest.mark.parametrize("path", [binding.EXPERTS_TILES, binding.EXPERTS_PAIRS])
def test_a_million_experts(path):
    T, h, s, M, k = 300, 16, 8, 1 << 20, 4
    X, W1, W2, _, _, _, gate, dout = make(T, h, s, M, k)
    idx = torch.randint(0, M, (T, k), device="cuda", dtype=torch.int32)
    idx[0, 0], idx[1, 0] = 0, M - 1
    offsets, pairs = ref.lists(idx, M)
    hit = torch.unique(idx).long()
    local = torch.searchsorted(hit, idx.long()).int()
    few, few_pairs = ref.lists(local, len(hit))
    assert torch.equal(pairs, few_pairs)
    tiles = path == binding.EXPERTS_TILES
    y, y_tol, hid, hid_tol = ref.experts(X, W1[hit], W2[hit], few, pairs, k, rounded=tiles)
    res = binding.experts(X, W1, W2, idx, offsets, pairs, want_hidden=tiles, path=path)
    ref.within(res.y, y, y_tol, "y")
    if not tiles:
        return
    got = binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate, res.hidden, dout)
    dx, dgate, dw1, dw2 = ref.experts_backward(X, W1[hit], W2[hit], few, pairs, gate, res.hidden, dout)
    ref.within(got.dx, *dx, "dx")
    ref.within(got.dgate, *dgate, "dgate")
    ref.within(got.dw1[hit], *dw1, "dw1")
    ref.within(got.dw2[hit], *dw2, "dw2")
    for grad in (got.dw1, got.dw2):
        assert set(grad.view(M, -1).ne(0).any(1).nonzero().flatten().tolist()) <= set(hit.tolist())


def test_kept_projections_beyond_32_bit_offsets():
    """2.2e9 values of the kept projections and of their gradients; the last tokens, and the first and the last expert."""
    T, h, s, M = 1 << 20, 8, 1032, 64
    X, W1, W2, idx, offsets, pairs, gate, dout = make(T, h, s, M, 1, seed=7)
    res = binding.experts(X, W1, W2, idx, offsets, pairs, want_hidden=True)
    got = binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate, res.hidden, dout)
    b = offsets.tolist()
    for e in (0, M - 1):
        p = pairs[b[e]:b[e + 1]].long()
        n = len(p)
        one = torch.tensor([0, n], device="cuda", dtype=torch.int32)
        order = torch.arange(n, device="cuda", dtype=torch.int32)
        y, y_tol, hid, hid_tol = ref.experts(X[p], W1[e:e + 1], W2[e:e + 1], one, order, 1)
        ref.within(res.y[p], y, y_tol, "y")
        ref.within(res.hidden[b[e]:b[e + 1]], hid, hid_tol, "hidden")
        dx, dgate, dw1, dw2 = ref.experts_backward(X[p], W1[e:e + 1], W2[e:e + 1], one, order, gate[p], res.hidden[b[e]:b[e + 1]], dout[p])
        ref.within(got.dx[p], *dx, "dx")
        ref.within(got.dgate[p], *dgate, "dgate")
        ref.within(got.dw1[e:e + 1], *dw1, "dw1")
        ref.within(got.dw2[e:e + 1], *dw2, "dw2")


def test_gradients_of_rows_beyond_32_bit_offsets():
    """2.2e9 values of the slots' rows on the way to dX; the last tokens."""
    T, h, s, M, k = 65536, 2056, 8, 16, 16
    X, W1, W2, idx, offsets, pairs, gate, dout = make(T, h, s, M, k, seed=8)
    hidden = torch.randn((T * k, 2 * s), generator=torch.Generator("cuda").manual_seed(9), device="cuda").bfloat16()
    got = binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate, hidden, dout, want_dw=False)
    n = 40
    tail = torch.arange((T - n) * k, T * k, device="cuda")
    place = torch.empty(T * k, device="cuda", dtype=torch.int64)
    place[pairs.long()] = torch.arange(T * k, device="cuda")
    o, p = ref.lists(idx[-n:], M)
    dx, dgate, _, _ = ref.experts_backward(X[-n:], W1, W2, o, p, gate[-n:], hidden[place[tail[p.long()]]], dout[-n:])
    ref.within(got.dx[-n:], *dx, "dx")
    ref.within(got.dgate[-n:], *dgate, "dgate")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_joined_rows_beyond_32_bit_offsets(dtype):
    """2.2e9 values through the ring, forward and backward; the first and the last tokens."""
    T, h, k = 270000, 8192, 1
    gen = torch.Generator(device="cuda")
    gen.manual_seed(10)
    some = torch.cat((torch.arange(20, device="cuda"), torch.arange(T - 20, T, device="cuda")))
    Y = torch.zeros((T * k, h), device="cuda", dtype=torch.bfloat16)
    res = torch.zeros((T, h), device="cuda", dtype=dtype)
    Y[some], res[some] = randn(gen, 40, h).bfloat16(), (2 * randn(gen, 40, h)).to(dtype)
    gate, w = torch.rand((T, k), generator=gen, device="cuda"), weights(gen, h)
    got = binding.combine(Y, gate, res, *w, eps=EPS, want_sum=True)
    for name, value, (exact, tol) in zip(("residual", "x", "sum"), (got.residual, got.x, got.sum),
                                         forward_bounds(Y[some], gate[some], res[some], *w, 40, k, h, dtype)):
        ref.within(value[some], exact, tol, name)
    del Y, res
    dres, dx = torch.zeros((T, h), device="cuda", dtype=dtype), torch.zeros((T, h), device="cuda", dtype=torch.bfloat16)
    dres[some], dx[some] = (0.02 * randn(gen, 40, h)).to(dtype), (0.02 * randn(gen, 40, h)).bfloat16()
    back = binding.combine_backward(dres, dx, got.sum, got.residual, *w, eps=EPS)
    # (the other tokens' gradients are zeros and add nothing to those of the weights)
    want = backward_bounds(dres[some], dx[some], got.sum[some], got.residual[some], *w, dtype)
    for name, (exact, tol) in zip(("dresidual", "dsum", "dw_post", "dscale", "dw_pre"), want):
        value = getattr(back, name)
        ref.within(value[some] if value.dim() == 2 else value, exact, tol, name)


@pytest.mark.parametrize("T,h,k", [(1300, 64, 3), (1300, 512, 4), (1300, 1000, 4), (1300, 2048, 8), (1300, 8192, 2), (1300, 4096, 16), (1100, 8192, 3)])
def test_slots_with_a_gate_of_zero_add_nothing_on_any_path(T, h, k):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T + h)
    Y, gate, res = randn(gen, T * k, h).bfloat16(), randn(gen, T, k).softmax(-1), randn(gen, T, h).bfloat16()
    gate[::3, 1] = 0
    gate[5] = 0
    gate[-1] = -0.0
    w = weights(gen, h)
    want = forward_bounds(Y, gate, res, *w, T, k, h, torch.bfloat16)
    Y[(gate == 0).reshape(-1)] = float("nan")
    got = binding.combine(Y, gate, res, *w, eps=EPS, want_sum=True)
    for name, value, (exact, tol) in zip(("residual", "x", "sum"), (got.residual, got.x, got.sum), want):
        ref.within(value, exact, tol, name)
    assert torch.equal(got.residual[5], res[5]) and torch.equal(got.residual[-1], res[-1])
