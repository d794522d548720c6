"""Ways through the operators behind the router that their sizes choose, each reached by the shapes here: what the decoding kernel keeps in
flight, rows too long for the ring, turns of what a CTA knows of its tiles in advance, offsets of gradients past 32 bits."""
import pytest
import torch

import layer_reference as ref
from test_gpu_combine import EPS, backward_bounds, forward_bounds, randn, weights
from test_gpu_experts import make

pytestmark = pytest.mark.gpu

binding = pytest.importorskip("paper_2609_36301_b200.binding")

SMS = 148


def ranks_of(P, h):
    """CTAs of a pair's cluster (launch_experts_pairs)."""
    r = 1
    while r < 8 and P * r * 2 <= 2 * SMS and h // (r * 2) >= 32:
        r *= 2
    return r


# T, h, s, M, k, ranks: few pairs of wide experts, two batches of weights in flight all the time
WIDE = [(16, 4096, 128, 64, 8, 2), (2, 4096, 512, 8, 4, 8), (37, 1000, 520, 9, 8, 1), (9, 2056, 520, 11, 3, 8), (1, 4096, 1032, 2, 1, 8),
        (50, 1544, 1000, 5, 2, 2), (148, 8192, 136, 6, 2, 1), (3, 8192, 8192, 2, 1, 8)]


@pytest.mark.parametrize("ids", ["spread", "holes"])
@pytest.mark.parametrize("T,h,s,M,k,ranks", WIDE)
def test_few_pairs_of_wide_experts(T, h, s, M, k, ranks, ids):
    assert T * k <= 2 * SMS and ranks_of(T * k, h) == ranks and h // ranks * (s // 4) // 256 >= 128
    X, W1, W2, idx, offsets, pairs, _, _ = make(T, h, s, M, k, seed=1, ids=ids)
    y, y_tol, _, _ = ref.experts(X, W1, W2, offsets, pairs, k, rounded=False)
    used = idx.reshape(-1) >= 0
    got = binding.experts(X, W1, W2, idx, path=binding.EXPERTS_PAIRS).y
    ref.within(got[used], y[used], y_tol[used], "y")


@pytest.mark.parametrize("T,h,s,M,k", [(400, 512, 256, 9, 2), (300, 1032, 128, 7, 3), (150, 2048, 1000, 4, 2)])
def test_many_pairs_of_wide_experts(T, h, s, M, k):
    assert T * k > 2 * SMS and h * (s // 4) // 256 >= 32
    X, W1, W2, idx, offsets, pairs, _, _ = make(T, h, s, M, k, seed=2)
    y, y_tol, _, _ = ref.experts(X, W1, W2, offsets, pairs, k, rounded=False)
    ref.within(binding.experts(X, W1, W2, idx, path=binding.EXPERTS_PAIRS).y, y, y_tol, "y")


@pytest.mark.parametrize("T,h,s,M,k", [(7000, 64, 16, 9000, 2), (5600, 264, 72, 6400, 2)])
def test_more_than_32_tiles_per_cta(T, h, s, M, k):
    """Forward and backward: a warp's lanes know 32 units in advance, and begin anew."""
    X, W1, W2, idx, offsets, pairs, gate, dout = make(T, h, s, M, k, seed=3)
    tiles = int((offsets[1:] > offsets[:-1]).sum())
    assert tiles > 32 * SMS
    res = binding.experts(X, W1, W2, idx, offsets, pairs, want_hidden=True, path=binding.EXPERTS_TILES)
    y, y_tol, hid, hid_tol = ref.experts(X, W1, W2, offsets, pairs, k)
    ref.within(res.hidden, hid, hid_tol, "hidden")
    ref.within(res.y, y, y_tol, "y")
    got = binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate, res.hidden, dout)
    for name, (value, tol) in zip(("dx", "dgate", "dw1", "dw2"), ref.experts_backward(X, W1, W2, offsets, pairs, gate, res.hidden, dout)):
        ref.within(getattr(got, name), value, tol, name)
    assert binding.more_route_status() == 0


def test_gradients_beyond_32_bit_offsets():
    """4.3e9 values of dW1, 2.1e9 of dW2: experts with pairs at the start, in the middle and at the end, zeros everywhere else."""
    M, h, s, k, T = 16384, 2048, 64, 2, 70
    some = torch.tensor([0, 1, M // 2 - 1, M // 2, M - 2, M - 1], device="cuda")
    X, a, b, local, _, _, gate, dout = make(T, h, s, len(some), k)
    W1 = torch.zeros((M, h, 2 * s), device="cuda", dtype=torch.bfloat16)
    W2 = torch.zeros((M, s, h), device="cuda", dtype=torch.bfloat16)
    W1[some], W2[some] = a, b
    idx = some[local.long()].int()
    offsets, pairs = ref.lists(idx, M)
    few, few_pairs = ref.lists(local, len(some))
    assert torch.equal(pairs, few_pairs)                     # (the same order of runs)
    hidden = torch.randn((T * k, 2 * s), generator=torch.Generator("cuda").manual_seed(5), device="cuda").bfloat16()
    got = binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate, hidden, dout)
    dx, dgate, dw1, dw2 = ref.experts_backward(X, a, b, few, few_pairs, gate, hidden, dout)
    ref.within(got.dx, *dx, "dx")
    ref.within(got.dgate, *dgate, "dgate")
    ref.within(got.dw1[some], *dw1, "dw1")
    ref.within(got.dw2[some], *dw2, "dw2")
    for grad in (got.dw1, got.dw2):
        for part, at in zip(grad.split(1024), range(0, M, 1024)):
            there = part.view(part.shape[0], -1).ne(0).any(1).nonzero().flatten() + at
            assert set(there.tolist()) == {e for e in some.tolist() if at <= e < at + 1024}
    assert binding.more_route_status() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,h,k", [(1300, 4096, 16), (1201, 8192, 6), (1250, 2048, 32), (1190, 1024, 32)])
def test_rows_too_long_for_the_ring(T, h, k, dtype):
    """Many tokens whose rows do not fit the ring twice (the last one's do, barely): a CTA per token."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T)
    Y, gate, res = randn(gen, T * k, h).bfloat16(), randn(gen, T, k).softmax(-1), (2 * randn(gen, T, h)).to(dtype)
    w = weights(gen, h)
    got = binding.combine(Y, gate, res, *w, eps=EPS, want_sum=True)
    for name, value, (exact, tol) in zip(("residual", "x", "sum"), (got.residual, got.x, got.sum), forward_bounds(Y, gate, res, *w, T, k, h, dtype)):
        ref.within(value, exact, tol, name)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("have", ["scale", "w_post", "neither", "scale and no dx", "w_post and no dresidual"])
@pytest.mark.parametrize("T,h", [(1200, 8192), (700, 4104), (9, 4104)])
def test_backward_of_long_rows_without(T, h, have, dtype):
    """Two vectors per thread, and some of the weights or one of the gradients left out."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T + h)
    a = dict(dres=(0.02 * randn(gen, T, h)).to(dtype), dx=(0.02 * randn(gen, T, h)).bfloat16(), y=randn(gen, T, h).bfloat16(), r=(2 * randn(gen, T, h)).to(dtype))
    a["w_post"], a["scale"], a["w_pre"] = weights(gen, h)
    if "w_post" not in have:
        a["w_post"] = None
    if "scale" not in have:
        a["scale"] = None
    if "no dx" in have:
        a.update(dx=None, r=None, w_pre=None)
    if "no dresidual" in have:
        a["dres"] = None
    names = ("dres", "dx", "y", "r", "w_post", "scale", "w_pre")
    got = binding.combine_backward(*[a[n] for n in names], eps=EPS)
    asked = dict(dw_post=a["w_post"], dscale=a["scale"], dw_pre=a["dx"])
    for name, (exact, tol) in zip(("dresidual", "dsum", "dw_post", "dscale", "dw_pre"), backward_bounds(*[a[n] for n in names], dtype)):
        value = getattr(got, name)
        if name in asked and asked[name] is None:
            assert value is None
        else:
            ref.within(value, exact, tol, name)
