"""Host threads that call the operators behind the router with different sizes: what one of them needs of shared memory must not
be what the other's launch is held to.  Each thread alternates a small and a large call on a stream of its own; every result is compared
with that of the same call made alone."""
import threading

import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

binding = pytest.importorskip("paper_2609_36301_b200.binding")

THREADS, CALLS, ROUNDS = 4, 200, 40         # calls of a thread in a row, how often


def randn(gen, *n):
    return torch.randn(n, generator=gen, device="cuda")


def combine_call(T, h, k, gen):
    """More than eight tokens per SM, so that rows come through the ring, whose stages take up what the row lengths say."""
    Y, gate, res = randn(gen, T * k, h).bfloat16(), randn(gen, T, k).softmax(-1), randn(gen, T, h).bfloat16()
    w = [1 + 0.1 * randn(gen, h) for _ in range(3)]

    def make():
        out = [torch.empty_like(res) for _ in range(3)]
        return out, lambda stream: binding.more_combine(Y, gate, res, *w, 1e-6, *out, stream=stream)
    return make


def combine_backward_call(T, h, gen):
    dres, dx, y, r = (randn(gen, T, h).bfloat16() for _ in range(4))
    w = [1 + 0.1 * randn(gen, h) for _ in range(3)]

    def make():
        out = [torch.empty_like(dx) for _ in range(2)] + [torch.empty_like(w[0]) for _ in range(3)]
        ws = torch.empty(binding.combine_workspace(T, h), device="cuda", dtype=torch.uint8)
        return out, lambda stream: binding.more_combine_backward(dres, dx, y, r, *w, 1e-6, *out, workspace=ws, stream=stream)
    return make


def pairs_call(T, h, s, M, k, gen):
    X, W1, W2 = randn(gen, T, h).bfloat16(), (randn(gen, M, h, 2 * s) * h ** -0.5).bfloat16(), (randn(gen, M, s, h) * s ** -0.5).bfloat16()
    idx = torch.arange(T * k, device="cuda", dtype=torch.int32).remainder(M).view(T, k)

    def make():
        out = [torch.empty((T * k, h), device="cuda", dtype=torch.bfloat16)]
        return out, lambda stream: binding.more_experts(X, W1, W2, idx, None, None, *out, path=binding.EXPERTS_PAIRS, stream=stream)
    return make


def tiles_call(T, h, s, M, k, gen):
    """Forward and backward, each with a workspace of its own."""
    X, W1, W2 = randn(gen, T, h).bfloat16(), (randn(gen, M, h, 2 * s) * h ** -0.5).bfloat16(), (randn(gen, M, s, h) * s ** -0.5).bfloat16()
    idx = torch.arange(T * k, device="cuda", dtype=torch.int32).remainder(M).view(T, k)
    offsets, pairs = ref.lists(idx, M)
    gate, dout = randn(gen, T, k), randn(gen, T, h).bfloat16()

    def make():
        out = [torch.empty((T * k, h), device="cuda", dtype=torch.bfloat16), torch.empty((T * k, 2 * s), device="cuda", dtype=torch.bfloat16),
               torch.empty_like(X), torch.empty_like(gate), torch.empty_like(W1), torch.empty_like(W2)]
        ws = [torch.empty(binding.experts_workspace(T, h, s, M, k, b), device="cuda", dtype=torch.uint8) for b in (False, True)]

        def call(stream):
            binding.more_experts(X, W1, W2, idx, offsets, pairs, *out[:2], path=binding.EXPERTS_TILES, workspace=ws[0], stream=stream)
            binding.more_experts_backward(X, W1, W2, idx, offsets, pairs, gate, out[1], dout, *out[2:], workspace=ws[1], stream=stream)
        return out, call
    return make


@pytest.mark.parametrize("op", ["combine", "combine_backward", "pairs", "tiles"])
def test_threads_with_different_sizes(op):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    if op == "combine":                      # rings of 32 and of 100 KB
        kinds = [combine_call(1200, 1024, 1, gen), combine_call(1200, 2048, 4, gen)]
    elif op == "combine_backward":           # 64 and 96 KB
        kinds = [combine_backward_call(64, 1032, gen), combine_backward_call(64, 2048, gen)]
    elif op == "tiles":
        kinds = [tiles_call(100, 64, 24, 5, 2, gen), tiles_call(300, 264, 136, 7, 3, gen)]
    else:                                    # 8 and 33 KB
        kinds = [pairs_call(2, 64, 8, 4, 2, gen), pairs_call(2, 64, 2048, 4, 2, gen)]
    alone = []
    for make in kinds:
        out, call = make()
        call(None)
        alone.append(out)
    torch.cuda.synchronize()
    errors = []
    together = threading.Barrier(THREADS)

    def worker(first):
        try:
            stream = torch.cuda.Stream()
            mine = [make() for make in kinds]
            torch.cuda.synchronize()
            for _ in range(ROUNDS):
                for out, _ in mine:
                    for o in out:
                        o.zero_()
                torch.cuda.synchronize()
                together.wait()
                for i in range(CALLS):
                    mine[(first + i) & 1][1](stream)
                stream.synchronize()
                for (got, _), want in zip(mine, alone):
                    for g, w in zip(got, want):
                        assert torch.equal(g, w)
        except Exception as e:               # noqa: BLE001 - reported to the main thread
            errors.append(repr(e))
            together.abort()

    threads = [threading.Thread(target=worker, args=(i,)) for i in range(THREADS)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    assert binding.more_route_status() == 0
