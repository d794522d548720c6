"""Shapes whose stages change from many short ones to few long ones inside a CTA: where units of dW2 follow those of dW1, where long
runs follow short ones, and the other way round."""
import pytest
import torch

import layer_reference as ref
from test_gpu_experts import make

pytestmark = pytest.mark.gpu

binding = pytest.importorskip("paper_2609_36301_b200.binding")


def with_runs(lengths, h, s, seed):
    """Arguments with one slot per token and runs of those lengths."""
    M, T = len(lengths), int(lengths.sum())
    X, W1, W2, _, _, _, gate, dout = make(T, h, s, M, 1, seed=seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    idx = torch.repeat_interleave(torch.arange(M, device="cuda"), lengths)[torch.randperm(T, generator=gen, device="cuda")].int()[:, None].contiguous()
    offsets, pairs = ref.lists(idx, M)
    return X, W1, W2, idx, offsets, pairs, gate, dout


def check(X, W1, W2, idx, offsets, pairs, gate, dout):
    k = idx.shape[1]
    fwd = binding.experts(X, W1, W2, idx, offsets, pairs, want_hidden=True, path=binding.EXPERTS_TILES)
    y, y_tol, hid, hid_tol = ref.experts(X, W1, W2, offsets, pairs, k)
    ref.within(fwd.hidden, hid, hid_tol, "hidden")
    ref.within(fwd.y, y, y_tol, "y")
    args = (X, W1, W2, idx, offsets, pairs, gate, fwd.hidden, dout)
    got = binding.experts_backward(*args)
    for name, (value, tol) in zip(("dx", "dgate", "dw1", "dw2"), ref.experts_backward(X, W1, W2, offsets, pairs, gate, fwd.hidden, dout)):
        ref.within(getattr(got, name), value, tol, name)
    for _ in range(20):
        again, once_more = binding.experts_backward(*args), binding.experts(X, W1, W2, idx, offsets, pairs, want_hidden=True, path=binding.EXPERTS_TILES)
        for name in ("dx", "dgate", "dw1", "dw2"):
            assert torch.equal(getattr(again, name), getattr(got, name)), name
        assert torch.equal(once_more.y, fwd.y) and torch.equal(once_more.hidden, fwd.hidden)
    assert binding.more_route_status() == 0


@pytest.mark.parametrize("T,h,s,M,k", [(8000, 432, 24, 3000, 3), (12000, 432, 24, 3000, 6), (6000, 200, 24, 2500, 4), (5000, 1024, 16, 2000, 3), (6000, 256, 32, 1500, 8),
                                       (4000, 64, 128, 2000, 4), (3000, 64, 200, 1500, 4), (4000, 48, 64, 3000, 3)])
def test_units_of_both_gradients(T, h, s, M, k):
    check(*make(T, h, s, M, k, seed=T + h))


@pytest.mark.parametrize("h,s", [(432, 24), (64, 64), (64, 128), (56, 40), (512, 64), (264, 136)])
@pytest.mark.parametrize("order", ["short first", "long first", "by turns"])
def test_runs_of_unlike_lengths(h, s, order):
    """A CTA takes every 148th tile: hundreds of runs of one to eight pairs, and then of 100 to 300."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(h + s)
    times = 4 if (h, s) == (432, 24) else 2
    few, many = torch.randint(1, 9, (500 * times,), generator=gen, device="cuda"), torch.randint(100, 300, (150 * times,), generator=gen, device="cuda")
    lengths = torch.cat((few, many))
    if order == "long first":
        lengths = lengths.flip(0)
    if order == "by turns":
        lengths = torch.cat([torch.cat(x) for x in zip(few.chunk(5), many.chunk(5))])
    check(*with_runs(lengths, h, s, h))


def test_a_training_step_of_many_narrow_experts():
    """62478 x 6 pairs of 16083 experts: some experts' gradients against their plain form, the same bits every time."""
    T, h, s, M, k = 62478, 432, 24, 16083, 6
    X, W1, W2, idx, offsets, pairs, gate, dout = make(T, h, s, M, k, seed=5)
    hidden = torch.randn((T * k, 2 * s), generator=torch.Generator("cuda").manual_seed(6), device="cuda").bfloat16()
    args = (X, W1, W2, idx, offsets, pairs, gate, hidden, dout)
    got = binding.experts_backward(*args)
    assert binding.more_route_status() == 0
    b = offsets.tolist()
    for e in list(range(0, M, 53)) + [M - 1]:
        p = pairs[b[e]:b[e + 1]].long()
        one, order = torch.tensor([0, len(p)], device="cuda", dtype=torch.int32), torch.arange(len(p), device="cuda", dtype=torch.int32)
        t = p // k
        _, _, dw1, dw2 = ref.experts_backward(X[t], W1[e:e + 1], W2[e:e + 1], one, order, gate.reshape(-1, 1)[p], hidden[b[e]:b[e + 1]], dout[t])
        ref.within(got.dw1[e:e + 1], *dw1, "dw1")
        ref.within(got.dw2[e:e + 1], *dw2, "dw2")
    for _ in range(10):
        again = binding.experts_backward(*args)
        for name in ("dx", "dgate", "dw1", "dw2"):
            assert torch.equal(getattr(again, name), getattr(got, name)), name
    assert binding.more_route_status() == 0
