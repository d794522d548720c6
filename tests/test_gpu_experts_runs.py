"""Gradients of the experts' weights over long runs of pairs, which are summed in pieces."""
import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

binding = pytest.importorskip("paper_2609_36301_b200.binding")


@pytest.mark.parametrize("h,s", [(8, 8), (64, 64), (264, 72), (512, 40), (136, 264)])
def test_runs_around_the_length_of_a_piece(h, s):
    """Values with which everything on the way is exact (a gate projection of 64, whose sigmoid is 1 in 32 bits; signs and zeros; powers
    of two), so that the gradients are whole numbers of 1/64 below 2^24 of them and what comes out is their rounding to bf16."""
    runs = [16385, 0, 1, 8192, 63, 8193, 0, 24576, 8191, 20000, 64]
    M, T = len(runs), sum(runs)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(h + s)
    signs = lambda *n: torch.randint(-1, 2, n, generator=gen, device="cuda").bfloat16()  # noqa: E731
    X, dout = signs(T, h), signs(T, h)
    of = torch.repeat_interleave(torch.arange(M, device="cuda"), torch.tensor(runs, device="cuda"))
    idx = of[torch.randperm(T, generator=gen, device="cuda")].int()[:, None].contiguous()
    offsets, pairs = ref.lists(idx, M)
    hidden = torch.cat((torch.full((T, s), 64.0, device="cuda").bfloat16(), signs(T, s) / 64), 1).contiguous()
    W1 = torch.zeros((M, h, 2 * s), device="cuda").bfloat16()
    W2 = torch.zeros((M, s, h), device="cuda").bfloat16()
    column = torch.arange(s, device="cuda") % h
    W2[:, torch.arange(s, device="cuda"), column] = 1 / 64
    got = binding.experts_backward(X, W1, W2, idx, offsets, pairs, torch.ones((T, 1), device="cuda"), hidden, dout, want_dx=False)
    for e, a, b, p in ref.runs(offsets, pairs):
        x, d, up = X[p].double(), dout[p].double(), hidden[a:b, s:].double()
        c = d[:, column] / 64
        dw1 = x.T @ torch.cat((c * up, c * 64), 1)
        dw2 = (up * 64).T @ d
        assert torch.equal(got.dw1[e], dw1.float().bfloat16()), (e, b - a)
        assert torch.equal(got.dw2[e], dw2.float().bfloat16()), (e, b - a)
    for e in (1, 6):
        assert not got.dw1[e].any() and not got.dw2[e].any()
    assert binding.more_route_status() == 0


@pytest.mark.parametrize("T", [8192, 65536, 524288])
def test_long_runs_lose_nothing_to_truncation(T):
    """A dense block (one expert).  Sums in the tensor memory are truncated at every 16 pairs: a run of n in one piece comes out n / 16 x
    2/3 x 2^-24 too small (each truncation loses half of 2^-23 of what the sum has come to, in the mean, and the root of how far it has
    come is 2/3 of the end's), 1.3e-3 for 524288.  In pieces of 8192, joined by rounding additions, 2.0e-5 at any length.  That bias is the
    projection of the error on the gradient.  The roundings to bf16 (of du or gate a, and of the gradient: 2^-9 / sqrt(3) = 1.1e-3 each,
    of either sign) leave at most 1.1e-3 sqrt(3 / N) of N = 32768 values there, twice: 1.5e-5 in the root mean square; five times that."""
    h, s = 512, 64
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T)
    rn = lambda *n: torch.randn(n, generator=gen, device="cuda").bfloat16()  # noqa: E731
    X, dout, hidden = rn(T, h), rn(T, h), rn(T, 2 * s)
    W1, W2 = (rn(1, h, 2 * s) * h ** -0.5).bfloat16(), (rn(1, s, h) * s ** -0.5).bfloat16()
    gate = torch.rand((T, 1), generator=gen, device="cuda")
    idx = torch.zeros((T, 1), device="cuda", dtype=torch.int32)
    offsets, pairs = ref.lists(idx, 1)
    got = binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate, hidden, dout, want_dx=False)
    again = binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate, hidden, dout, want_dx=False)
    assert torch.equal(got.dw1, again.dw1) and torch.equal(got.dw2, again.dw2)
    dw1 = torch.zeros((h, 2 * s), device="cuda", dtype=torch.float64)
    dw2 = torch.zeros((s, h), device="cuda", dtype=torch.float64)
    for a in range(0, T, 65536):
        at = slice(a, a + 65536)
        x, d, u, gt = X[at].double(), dout[at].double(), hidden[at].double(), gate[at].double()
        g, up = u[:, :s], u[:, s:]
        sg = torch.sigmoid(g)
        c = gt * (d @ W2[0].double().T)
        dw1 += x.T @ torch.cat((c * up * sg * (1 + g * (1 - sg)), c * g * sg), 1)
        dw2 += (gt * g * sg * up).T @ d
    for name, value, want in (("dw1", got.dw1[0], dw1), ("dw2", got.dw2[0], dw2)):
        bias = float(((value.double() - want) * want).sum() / want.square().sum())
        print(name, T, bias)
        assert abs(bias) <= 2.0e-5 + 5 * 1.5e-5, (name, bias)
    assert binding.more_route_status() == 0
