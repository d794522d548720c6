"""The activation's accuracy far from zero, where the gate gradients, which leave in 32 bits, show it."""
import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

binding = pytest.importorskip("paper_2609_36301_b200.binding")


def test_gate_gradients_of_far_gates_keep_32_bits():
    """One hidden column with a weight of 1 to one output column: a gate gradient is d silu(g), one term.  e^-g in 32 bits is good to two
    units of 2^-23, the sum with 1 to half of one, the quotient to two, the three products to half of one each: six in all, 7.2e-7 relative,
    at every g.  (An exponential of 2 + 1.2 |g| units, as hardware's alone is, is 10^-5 off at g = -80.)"""
    T, h, s = 4096, 8, 8
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    g = torch.linspace(-80, 20, T, device="cuda").bfloat16()
    dout = torch.randn((T, h), generator=gen, device="cuda").bfloat16()
    hidden = torch.zeros((T, 2 * s), device="cuda").bfloat16()
    hidden[:, 0], hidden[:, s] = g, 1
    X, W1, W2 = torch.zeros((T, h), device="cuda").bfloat16(), torch.zeros((1, h, 2 * s), device="cuda").bfloat16(), torch.zeros((1, s, h), device="cuda").bfloat16()
    W2[0, 0, 0] = 1
    idx = torch.zeros((T, 1), device="cuda", dtype=torch.int32)
    offsets, pairs = ref.lists(idx, 1)
    got = binding.experts_backward(X, W1, W2, idx, offsets, pairs, torch.ones((T, 1), device="cuda"), hidden, dout, want_dx=False, want_dw=False).dgate
    want = dout[:, :1].double() * (g.double() * torch.sigmoid(g.double()))[:, None]
    ref.within(got, want, 6 * 2.0 ** -23 * want.abs(), "dgate")
