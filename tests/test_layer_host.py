"""Host-side behaviour of the operators behind the router: exported names, argument errors (found before anything needs a device), the
sizes of workspaces, which path serves a call."""
import os
import re

import pytest

from paper_2609_36301_b200 import binding, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE, ALIGN, MODE, TOO_LARGE = -1, -2, -3, -4, -8
A = 4096                                                       # an address that is never read: every call here is refused first


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def experts(lib, **over):
    a = dict(X=A, W1=A, W2=A, idx=A, offsets=A, pairs=A, T=4, h=64, s=16, M=8, k=2, y=A, hidden=None, path=2, ws=A, n=1 << 40)
    a.update(over)
    return lib.more_experts(a["X"], a["W1"], a["W2"], a["idx"], a["offsets"], a["pairs"], a["T"], a["h"], a["s"], a["M"], a["k"], a["y"],
                            a["hidden"], a["path"], a["ws"], a["n"], None)


def experts_backward(lib, **over):
    a = dict(X=A, W1=A, W2=A, idx=A, offsets=A, pairs=A, gate=A, hidden=A, dout=A, T=4, h=64, s=16, M=8, k=2, dx=A, dgate=A, dw1=A, dw2=A, ws=A,
             n=1 << 40)
    a.update(over)
    return lib.more_experts_backward(*[a[n] for n in ("X", "W1", "W2", "idx", "offsets", "pairs", "gate", "hidden", "dout", "T", "h", "s", "M",
                                                      "k", "dx", "dgate", "dw1", "dw2", "ws", "n")], None)


def combine(lib, **over):
    a = dict(Y=A, gate=A, residual=A, type=0, w_post=A, scale=A, w_pre=A, eps=1e-6, T=4, h=64, k=2, r=A, x=A, sum=A)
    a.update(over)
    return lib.more_combine(*[a[n] for n in ("Y", "gate", "residual", "type", "w_post", "scale", "w_pre", "eps", "T", "h", "k", "r", "x", "sum")],
                            None)


def combine_backward(lib, **over):
    a = dict(dr=A, dx=A, sum=A, ro=A, type=0, w_post=A, scale=A, w_pre=A, eps=1e-6, T=4, h=64, odr=A, ods=A, dwp=A, dsc=A, dwn=A, ws=A, n=1 << 40)
    a.update(over)
    return lib.more_combine_backward(*[a[n] for n in ("dr", "dx", "sum", "ro", "type", "w_post", "scale", "w_pre", "eps", "T", "h", "odr", "ods",
                                                      "dwp", "dsc", "dwn", "ws", "n")], None)


def test_every_declared_function_is_exported_and_bound(lib):
    header = open(os.path.join(ROOT, "include", "more_route.h")).read()
    names = set(re.findall(r"^(?:int|long long) (more_(?:experts|combine)\w*)\(", header, re.M))
    assert names == {"more_experts", "more_experts_workspace", "more_experts_path", "more_experts_backward", "more_combine",
                     "more_combine_workspace", "more_combine_backward"}
    for n in names:
        assert getattr(lib, n).argtypes


@pytest.mark.parametrize("over,code", [
    (dict(T=-1), SHAPE), (dict(h=60), SHAPE), (dict(h=0), SHAPE), (dict(h=8200), SHAPE), (dict(s=12), SHAPE), (dict(s=0), SHAPE), (dict(s=8200), SHAPE),
    (dict(M=0), SHAPE), (dict(M=1 << 30, k=1, T=(1 << 31) - 1, h=8), TOO_LARGE), (dict(k=0), SHAPE), (dict(k=9), SHAPE), (dict(M=64, k=33), SHAPE),
    (dict(T=1 << 27, M=64, k=32), TOO_LARGE), (dict(path=3), MODE), (dict(path=-1), MODE),
    (dict(X=None), NULL), (dict(W1=None), NULL), (dict(W2=None), NULL), (dict(idx=None), NULL), (dict(y=None), NULL), (dict(offsets=None), NULL),
    (dict(pairs=None), NULL), (dict(path=0, pairs=None, hidden=A), NULL), (dict(path=1, hidden=A), SHAPE), (dict(ws=None), NULL),
    (dict(n=0), TOO_LARGE), (dict(X=A + 8), ALIGN), (dict(W1=A + 2), ALIGN), (dict(W2=A + 8), ALIGN), (dict(idx=A + 2), ALIGN),
    (dict(offsets=A + 1), ALIGN), (dict(pairs=A + 2), ALIGN), (dict(y=A + 8), ALIGN), (dict(hidden=A + 8), ALIGN), (dict(ws=A + 16), ALIGN),
])
def test_experts_refuses(lib, over, code):
    if over.get("M") == 1 << 30:
        over = dict(over, T=1 << 30, k=2)                      # 2^31 pairs
    assert experts(lib, **over) == code


@pytest.mark.parametrize("over,code", [(dict(h=60), SHAPE), (dict(k=9), SHAPE), (dict(T=-3), SHAPE), (dict(n=100), TOO_LARGE)] +
                         [({n: None}, NULL) for n in ("X", "W1", "W2", "idx", "offsets", "pairs", "gate", "hidden", "dout", "ws")] +
                         [({n: A + 8}, ALIGN) for n in ("X", "W1", "W2", "hidden", "dout", "dx", "dw1", "dw2", "ws")] +
                         [({n: A + 2}, ALIGN) for n in ("idx", "offsets", "pairs", "gate", "dgate")])
def test_experts_backward_refuses(lib, over, code):
    assert experts_backward(lib, **over) == code


@pytest.mark.parametrize("over,code", [
    (dict(type=2), MODE), (dict(T=-1), SHAPE), (dict(h=4), SHAPE), (dict(h=68), SHAPE), (dict(h=8200), SHAPE), (dict(k=0), SHAPE), (dict(k=33), SHAPE),
    (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(Y=None, residual=None), NULL), (dict(r=None, x=None, sum=None), NULL),
    (dict(w_pre=None), NULL)] + [({n: A + 8}, ALIGN) for n in ("Y", "residual", "w_post", "scale", "w_pre", "r", "x", "sum")] +
    [(dict(gate=A + 2), ALIGN)])
def test_combine_refuses(lib, over, code):
    assert combine(lib, **over) == code


@pytest.mark.parametrize("over,code", [
    (dict(type=2), MODE), (dict(h=68), SHAPE), (dict(h=8200), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(dr=None, dx=None), NULL),
    (dict(w_pre=None), NULL), (dict(ro=None), NULL), (dict(sum=None), NULL), (dict(sum=None, ods=None), NULL), (dict(ws=None), NULL),
    (dict(w_post=None), NULL), (dict(scale=None), NULL), (dict(dx=None), NULL), (dict(n=8), TOO_LARGE)] +
    [({n: A + 8}, ALIGN) for n in ("dr", "dx", "sum", "ro", "w_post", "scale", "w_pre", "odr", "ods", "ws")] +
    [({n: A + 2}, ALIGN) for n in ("dwp", "dsc", "dwn")])
def test_combine_backward_refuses(lib, over, code):
    assert combine_backward(lib, **over) == code


def test_workspaces(lib):
    assert binding.experts_workspace(0, 64, 16, 8, 2) > 0
    for T, h, s, M, k in ((1, 8, 8, 1, 1), (3001, 1000, 40, 504, 6), (65536, 2048, 64, 8192, 8)):
        P = T * k
        tiles = 16 * (1 + min(P, M) + P // 128)
        fwd, bwd = binding.experts_workspace(T, h, s, M, k), binding.experts_workspace(T, h, s, M, k, True)
        assert tiles + 2 * P * s <= fwd <= tiles + 2 * P * s + 1024
        assert bwd >= tiles + P * (4 * s + 2 * s + 2 * h)
    for bad in ((-1, 64, 16, 8, 2), (4, 60, 16, 8, 2), (4, 64, 16, 1, 2)):
        with pytest.raises(binding.MoreRouteError):
            binding.experts_workspace(*bad)
    assert binding.combine_workspace(0, 64) == 0
    assert binding.combine_workspace(65536, 2048) % (2 * 2048 * 4) == 0
    with pytest.raises(binding.MoreRouteError):
        binding.combine_workspace(4, 68)


def test_path_by_sizes(lib):
    """Few pairs: every pair reads its expert; many pairs, or few experts to share: tiles."""
    assert binding.experts_path(1, 2048, 64, 4096, 8) == binding.EXPERTS_PAIRS
    assert binding.experts_path(64, 2048, 64, 8192, 8) == binding.EXPERTS_PAIRS
    assert binding.experts_path(16384, 512, 64, 4096, 8) == binding.EXPERTS_TILES
    assert binding.experts_path(512, 512, 256, 8, 2) == binding.EXPERTS_TILES
    with pytest.raises(binding.MoreRouteError):
        binding.experts_path(4, 60, 16, 8, 2)
