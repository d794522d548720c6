"""The experts' feed-forward blocks and their gradients against their plain 64-bit forms, with bounds from the arithmetic
(layer_reference.py); where they can go wrong: tiles that end inside a run, experts without pairs or with all of them, ids that
are none, sizes off the tile sizes, buffers behind the ends, captured and overlapping calls."""
import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

binding = pytest.importorskip("paper_2609_36301_b200.binding")


def make(T, h, s, M, k, seed=0, ids="spread"):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rn = lambda *n: torch.randn(n, generator=gen, device="cuda")  # noqa: E731
    X, W1, W2 = rn(T, h).bfloat16(), (rn(M, h, 2 * s) * h ** -0.5).bfloat16(), (rn(M, s, h) * 1.7 * s ** -0.5).bfloat16()
    first = torch.randint(0, M, (T, 1), generator=gen, device="cuda")
    idx = ((first + torch.arange(k, device="cuda")) % M).int()
    if ids == "one":                       # the same experts for every token: long runs, and many empty experts
        idx = ((M - 1 - torch.arange(k, device="cuda")) % M).int().expand(T, k).contiguous()
    if ids == "holes":                     # a third of the slots unused, as the merge of an expert-sharded router leaves them
        idx[torch.rand((T, k), generator=gen, device="cuda") < 0.33] = -1
        idx[-1] = -1
    offsets, pairs = ref.lists(idx, M)
    gate = rn(T, k).softmax(-1)
    return X, W1, W2, idx, offsets, pairs, gate, (rn(T, h) * 0.02).bfloat16()


SHAPES = [
    # T, h, s, M, k, ids
    (1, 64, 64, 4, 2, "spread"), (1, 8, 8, 1, 1, "spread"), (5, 72, 24, 7, 3, "spread"), (129, 64, 64, 3, 1, "one"), (300, 264, 40, 5, 4, "spread"),
    (127, 136, 72, 9, 2, "holes"), (128, 512, 64, 16, 4, "spread"), (257, 320, 136, 2, 2, "one"), (64, 1000, 264, 6, 6, "spread"),
    (40, 256, 328, 12, 5, "holes"), (700, 128, 200, 33, 8, "spread"), (33, 2048, 16, 40, 32, "spread"), (1000, 192, 512, 1, 1, "spread"),
    (2000, 24, 8, 1500, 3, "spread"),
]


@pytest.mark.parametrize("T,h,s,M,k,ids", SHAPES)
def test_forward_tiles(T, h, s, M, k, ids):
    X, W1, W2, idx, offsets, pairs, _, _ = make(T, h, s, M, k, ids=ids)
    y, y_tol, hid, hid_tol = ref.experts(X, W1, W2, offsets, pairs, k)
    res = binding.experts(X, W1, W2, idx, offsets, pairs, want_hidden=True, path=binding.EXPERTS_TILES)
    used = idx.reshape(-1) >= 0
    ref.within(res.hidden[: int(offsets[-1])], hid[: int(offsets[-1])], hid_tol[: int(offsets[-1])], "hidden")
    ref.within(res.y[used], y[used], y_tol[used], "y")
    assert binding.more_route_status() == 0


@pytest.mark.parametrize("listed", [True, False])
@pytest.mark.parametrize("T,h,s,M,k,ids", SHAPES)
def test_forward_pairs(T, h, s, M, k, ids, listed):
    X, W1, W2, idx, offsets, pairs, _, _ = make(T, h, s, M, k, seed=1, ids=ids)
    y, y_tol, _, _ = ref.experts(X, W1, W2, offsets, pairs, k, rounded=False)
    if not listed:
        offsets = pairs = None
    res = binding.experts(X, W1, W2, idx, offsets, pairs, path=binding.EXPERTS_PAIRS)
    used = idx.reshape(-1) >= 0
    ref.within(res.y[used], y[used], y_tol[used], "y")


@pytest.mark.parametrize("T,h,s,M,k,ids", SHAPES)
def test_backward(T, h, s, M, k, ids):
    X, W1, W2, idx, offsets, pairs, gate, dout = make(T, h, s, M, k, seed=2, ids=ids)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    hidden = torch.randn((T * k, 2 * s), generator=gen, device="cuda").bfloat16()
    dx, dgate, dw1, dw2 = ref.experts_backward(X, W1, W2, offsets, pairs, gate, hidden, dout)
    got = binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate, hidden, dout)
    ref.within(got.dgate, *dgate, "dgate")
    ref.within(got.dx, *dx, "dx")
    ref.within(got.dw1, *dw1, "dw1")
    ref.within(got.dw2, *dw2, "dw2")
    assert binding.more_route_status() == 0


def test_reference_gradients_agree_with_differences():
    """The formulas that the kernels are held to, against central differences of the forward form (all in 64 bits)."""
    T, h, s, M, k = 3, 16, 8, 4, 2
    X, W1, W2, idx, offsets, pairs, gate, dout = (t.double() if t.is_floating_point() else t for t in make(T, h, s, M, k, seed=4))

    def loss(X, W1, W2, gate):
        y = ref.experts(X, W1, W2, offsets, pairs, k)[0]
        return float(((y.view(T, k, h) * gate[..., None]).sum(1) * dout).sum())

    hidden = ref.experts(X, W1, W2, offsets, pairs, k)[2]
    grads = ref.experts_backward(X, W1, W2, offsets, pairs, gate, hidden, dout)
    for which, (grad, _) in zip((0, 3, 1, 2), grads):
        args = [X, W1, W2, gate]
        direction = torch.randn_like(grad)
        step = 1e-5
        args[which] = args[which] + step * direction
        up = loss(*args)
        args[which] = args[which] - 2 * step * direction
        slope = (up - loss(*args)) / (2 * step)
        assert abs(slope - float((grad * direction).sum())) <= 1e-7 * max(1.0, abs(slope))


@pytest.mark.parametrize("h", [512, 520, 1024, 4096, 8192])
def test_gate_gradients_of_wide_tokens_keep_32_bits(h):
    """Relative to their 2-norm.  Sums in the tensor memory are truncated at every 16 columns, by at most 2^-23 of what they have come
    to and half of that in the mean, and are as large as the sum at the end times the root of how far they have come: 32 truncations
    (512 columns) lose 32 x 2/3 x 2^-24 = 1.3e-6 of a sum at most.  Pieces of 512 columns keep that bound at every width, and add up to
    16 roundings of 2^-24, of either sign: 2.4e-7 together.  In one piece h = 4096 lost 4.6e-6."""
    X, W1, W2, idx, offsets, pairs, gate, dout = make(256, h, 64, 8, 2, seed=3)
    hidden = torch.randn((512, 128), generator=torch.Generator("cuda").manual_seed(4), device="cuda").bfloat16()
    got = binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate, hidden, dout, want_dw=False).dgate.double()
    want = ref.experts_backward(X, W1, W2, offsets, pairs, gate, hidden, dout)[1][0]
    assert float((got - want).norm()) <= 1.6e-6 * float(want.norm())


def test_some_gradients_only():
    X, W1, W2, idx, offsets, pairs, gate, dout = make(200, 128, 64, 8, 2)
    hidden = torch.randn((400, 128), device="cuda").bfloat16()
    full = binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate, hidden, dout)
    a = binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate, hidden, dout, want_dw=False)
    b = binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate, hidden, dout, want_dx=False, want_dgate=False)
    assert a.dw1 is None and a.dw2 is None and b.dx is None and b.dgate is None
    assert torch.equal(a.dx, full.dx) and torch.equal(a.dgate, full.dgate)
    assert torch.equal(b.dw1, full.dw1) and torch.equal(b.dw2, full.dw2)


def test_same_lists_same_bits_and_order_of_a_run_does_not_matter_forward():
    X, W1, W2, idx, offsets, pairs, gate, dout = make(600, 256, 64, 5, 2)
    y1 = binding.experts(X, W1, W2, idx, offsets, pairs, path=binding.EXPERTS_TILES).y
    y2 = binding.experts(X, W1, W2, idx, offsets, pairs, path=binding.EXPERTS_TILES).y
    other = torch.cat([p[torch.randperm(len(p), device="cuda")] for p in (pairs[int(a):int(b)] for a, b in zip(offsets[:-1], offsets[1:]))])
    y3 = binding.experts(X, W1, W2, idx, offsets, other, path=binding.EXPERTS_TILES).y
    assert torch.equal(y1, y2) and torch.equal(y1, y3)
    hidden = torch.randn((1200, 128), device="cuda").bfloat16()
    g1 = binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate, hidden, dout)
    g2 = binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate, hidden, dout)
    for n in ("dx", "dgate", "dw1", "dw2"):
        assert torch.equal(getattr(g1, n), getattr(g2, n))


def test_no_tokens():
    _, W1, W2, _, _, _, _, _ = make(1, 64, 16, 4, 2)
    X = torch.empty((0, 64), device="cuda", dtype=torch.bfloat16)
    idx = torch.empty((0, 2), device="cuda", dtype=torch.int32)
    offsets, pairs = torch.zeros(5, device="cuda", dtype=torch.int32), torch.empty(0, device="cuda", dtype=torch.int32)
    assert binding.experts(X, W1, W2, idx, offsets, pairs).y.shape == (0, 64)
    g = binding.experts_backward(X, W1, W2, idx, offsets, pairs, torch.empty((0, 2), device="cuda"),
                                 torch.empty((0, 32), device="cuda", dtype=torch.bfloat16), X)
    assert g.dx.shape == (0, 64) and not g.dw1.any() and not g.dw2.any()


def test_nothing_routed():
    X, W1, W2, idx, _, pairs, gate, dout = make(50, 64, 16, 4, 2)
    idx.fill_(-1)
    offsets = torch.zeros(5, device="cuda", dtype=torch.int32)
    y = torch.full((100, 64), 7.0, device="cuda", dtype=torch.bfloat16)
    for path in (binding.EXPERTS_TILES, binding.EXPERTS_PAIRS):
        binding.more_experts(X, W1, W2, idx, offsets, pairs, y, path=path)
        assert (y == 7).all()
    g = binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate, torch.zeros((100, 32), device="cuda", dtype=torch.bfloat16), dout)
    assert not g.dx.any() and not g.dgate.any() and not g.dw1.any() and not g.dw2.any()


@pytest.mark.parametrize("path", [binding.EXPERTS_TILES, binding.EXPERTS_PAIRS])
def test_unused_slots_and_what_lies_behind_are_left(path):
    """Rows of unused slots, places behind the last, and guard rows around every output and behind the workspace stay as they were."""
    T, h, s, M, k = 131, 136, 40, 6, 3
    X, W1, W2, idx, offsets, pairs, gate, dout = make(T, h, s, M, k, ids="holes")
    n, used = int(offsets[-1]), idx.reshape(-1) >= 0

    def guarded(rows, cols, dtype=torch.bfloat16):
        whole = torch.full((rows + 64, cols), 3.0, device="cuda", dtype=dtype)
        return whole, whole[32:-32]

    whole_y, y = guarded(T * k, h)
    whole_h, hid = guarded(T * k, 2 * s)
    need = binding.experts_workspace(T, h, s, M, k)
    ws = torch.full((need + 4096,), 0x5A, device="cuda", dtype=torch.uint8)
    tiles = path == binding.EXPERTS_TILES
    binding.more_experts(X, W1, W2, idx, offsets, pairs, y, hid if tiles else None, path=path, workspace=ws[:need])
    torch.cuda.synchronize()
    assert (whole_y[:32] == 3).all() and (whole_y[-32:] == 3).all() and (y[~used] == 3).all() and not (y[used] == 3).all(1).any()
    assert (whole_h[:32] == 3).all() and (whole_h[-32:] == 3).all() and (hid[n:] == 3).all()
    assert (ws[need:] == 0x5A).all()
    if not tiles:
        return
    need = binding.experts_workspace(T, h, s, M, k, backward=True)
    ws = torch.full((need + 4096,), 0x5A, device="cuda", dtype=torch.uint8)
    whole_dx, dx = guarded(T, h)
    whole_dg, dg = guarded(T, k, torch.float32)
    whole_1, w1 = guarded(M * h, 2 * s)
    whole_2, w2 = guarded(M * s, h)
    binding.more_experts_backward(X, W1, W2, idx, offsets, pairs, gate, hid, dout, dx, dg, w1.view(M, h, 2 * s), w2.view(M, s, h), workspace=ws[:need])
    torch.cuda.synchronize()
    for whole in (whole_dx, whole_dg, whole_1, whole_2):
        assert (whole[:32] == 3).all() and (whole[-32:] == 3).all()
    assert (ws[need:] == 0x5A).all()


def test_garbage_in_masked_places_does_not_spread():
    """NaN in rows that no slot uses (a token without experts, hidden places behind the last) stays out of every sum."""
    T, h, s, M, k = 90, 128, 64, 4, 2
    X, W1, W2, idx, offsets, pairs, gate, dout = make(T, h, s, M, k, ids="holes")
    n = int(offsets[-1])
    hidden = torch.randn((T * k, 2 * s), device="cuda").bfloat16()
    hidden[n:] = float("nan")
    X[-1] = float("nan")                                   # the last token has no expert
    dout[-1] = float("inf")
    want = ref.experts_backward(X, W1, W2, offsets, pairs, gate, hidden, dout)
    got = binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate, hidden, dout)
    for name, (value, tol) in zip(("dx", "dgate", "dw1", "dw2"), want):
        ref.within(getattr(got, name), value, tol, name)


def test_a_row_that_is_not_finite_spoils_only_its_own_rows():
    T, h, s, M, k = 200, 128, 64, 3, 1
    X, W1, W2, idx, offsets, pairs, _, _ = make(T, h, s, M, k)
    clean = binding.experts(X, W1, W2, idx, offsets, pairs, path=binding.EXPERTS_TILES).y
    X[7] = float("nan")
    got = binding.experts(X, W1, W2, idx, offsets, pairs, path=binding.EXPERTS_TILES).y
    rest = torch.arange(T, device="cuda") != 7
    assert torch.equal(got[rest], clean[rest]) and got[7].isnan().all()


def test_extreme_projections():
    """Gates far into both tails of the sigmoid: 0 and the gate itself, without overflow on the way."""
    T, h, s, M, k = 64, 64, 32, 1, 1
    X = torch.zeros((T, h), device="cuda").bfloat16()
    X[:, 0] = torch.linspace(-3000, 3000, T, device="cuda").bfloat16()
    X[:, 1] = 1
    W1 = torch.zeros((1, h, 2 * s), device="cuda").bfloat16()
    W1[0, 0, :s] = 1
    W1[0, 1, s:] = 2
    W2 = torch.randn((1, s, h), device="cuda").bfloat16()
    idx = torch.zeros((T, 1), device="cuda", dtype=torch.int32)
    offsets, pairs = ref.lists(idx, 1)
    for path in (binding.EXPERTS_TILES, binding.EXPERTS_PAIRS):
        y, tol, _, _ = ref.experts(X, W1, W2, offsets, pairs, k)
        ref.within(binding.experts(X, W1, W2, idx, offsets, pairs, path=path).y, y, tol, "y")


@pytest.mark.parametrize("path", [binding.EXPERTS_TILES, binding.EXPERTS_PAIRS])
def test_weights_beyond_32_bit_offsets(path):
    """The last experts of 8.6 GB of weights."""
    M, h, s, k, T = 16384, 2048, 64, 2, 70
    W1 = torch.zeros((M, h, 2 * s), device="cuda", dtype=torch.bfloat16)
    W2 = torch.zeros((M, s, h), device="cuda", dtype=torch.bfloat16)
    X, a, b, _, _, _, gate, dout = make(T, h, s, 3, k)
    W1[-3:], W2[-3:] = a, b
    idx = torch.randint(M - 3, M, (T, k), device="cuda", dtype=torch.int32)
    offsets, pairs = ref.lists(idx, M)
    few = torch.cat((offsets[M - 3:], ))
    y, tol, _, _ = ref.experts(X, a, b, few, pairs, k)
    ref.within(binding.experts(X, W1, W2, idx, offsets, pairs, path=path).y, y, tol, "y")


def test_rows_beyond_32_bit_offsets():
    """More than 2^31 values in the rows of the slots."""
    T, h, s, M, k = 65536, 2056, 8, 16, 16
    X, W1, W2, idx, offsets, pairs, _, _ = make(T, h, s, M, k)
    y = binding.experts(X, W1, W2, idx, offsets, pairs).y
    tail = slice(T - 40, T)
    o, p = ref.lists(idx[tail], M)
    want, tol, _, _ = ref.experts(X[tail], W1, W2, o, p, k)
    ref.within(y[-40 * k:], want, tol, "y")


def test_other_stream_capture_and_replay():
    """A layer's calls on a stream of their own, captured once and replayed on other data, with lists that have other lengths."""
    T, h, s, M, k = 150, 256, 64, 12, 3
    args = make(T, h, s, M, k)
    X, W1, W2, idx, offsets, pairs, gate, dout = args
    y, hid = torch.empty((T * k, h), device="cuda").bfloat16(), torch.empty((T * k, 2 * s), device="cuda").bfloat16()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    binding.more_experts(X, W1, W2, idx, offsets, pairs, y, hid, stream=stream)
    stream.synchronize()
    direct = y.clone()
    ws = torch.empty(binding.experts_workspace(T, h, s, M, k), device="cuda", dtype=torch.uint8)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.more_experts(X, W1, W2, idx, offsets, pairs, y, hid, workspace=ws)
        grads = binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate, hid, dout)
    y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, direct)
    for seed, ids in ((5, "one"), (6, "holes")):
        new = make(T, h, s, M, k, seed=seed, ids=ids)
        for old, value in zip(args, new):
            old.copy_(value)
        graph.replay()
        torch.cuda.synchronize()
        used = idx.reshape(-1) >= 0
        want, tol, _, _ = ref.experts(X, W1, W2, offsets, pairs, k)
        ref.within(y[used], want[used], tol[used], "y")
        for name, (value, bound) in zip(("dx", "dgate", "dw1", "dw2"), ref.experts_backward(X, W1, W2, offsets, pairs, gate, hid, dout)):
            ref.within(getattr(grads, name), value, bound, name)


def test_overlapping_calls_with_workspaces_of_their_own():
    cases = [make(400, 512, 64, 24, 4, seed=i) for i in range(2)]
    alone = [binding.experts(*c[:6], want_hidden=True) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[] for _ in cases]
    for _ in range(10):
        for i, (c, st) in enumerate(zip(cases, streams)):
            got[i].append(binding.experts(*c[:6], want_hidden=True, stream=st))
    torch.cuda.synchronize()
    for one, many in zip(alone, got):
        for r in many:
            assert torch.equal(r.y, one.y) and torch.equal(r.hidden, one.hidden)


def test_refusals():
    X, W1, W2, idx, offsets, pairs, gate, dout = make(10, 64, 16, 4, 2)
    hid = torch.zeros((20, 32), device="cuda").bfloat16()
    ok = dict(X=X, W1=W1, W2=W2, idx=idx, offsets=offsets, pairs=pairs)
    for name, bad in (("X", X.float()), ("X", X.cpu()), ("X", X[:, ::2]), ("W1", W1[:, :, :16]), ("W2", W2.transpose(1, 2)), ("idx", idx.long()),
                      ("offsets", offsets[:-1]), ("pairs", pairs[:-1])):
        with pytest.raises((TypeError, ValueError)):
            binding.experts(**{**ok, name: bad})
    with pytest.raises(binding.MoreRouteError):                       # lists are needed
        binding.experts(X, W1, W2, idx, path=binding.EXPERTS_TILES)
    with pytest.raises(binding.MoreRouteError):
        binding.experts(X, W1, W2, idx, want_hidden=True)
    with pytest.raises(binding.MoreRouteError):                       # kept projections come from the tiles
        binding.experts(**ok, want_hidden=True, path=binding.EXPERTS_PAIRS)
    with pytest.raises(binding.MoreRouteError):
        binding.experts(**ok, path=7)
    with pytest.raises(binding.MoreRouteError):                       # too little workspace
        binding.experts(**ok, path=binding.EXPERTS_TILES, workspace=torch.empty(256, device="cuda", dtype=torch.uint8))
    with pytest.raises(binding.MoreRouteError):                       # h not a multiple of 8
        binding.experts(X[:, :60].contiguous(), W1[:, :60].contiguous(), W2[:, :, :60].contiguous(), idx, offsets, pairs)
    with pytest.raises((TypeError, ValueError)):
        binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate.bfloat16(), hid, dout)
    with pytest.raises((TypeError, ValueError)):
        binding.experts_backward(X, W1, W2, idx, offsets, pairs, gate, hid[:-1], dout)
