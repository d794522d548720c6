"""The work of the operators behind the router, as cases that can be timed and compared.

A case is a dict of plain values.  ``op`` says which public entry point it goes through:

  experts      ``binding.experts``: the gated feed-forward blocks of M experts over the (token, slot) pairs of a routing.
  experts_bwd  ``binding.experts_backward``: gradients of the tokens, the gates and both weights of every expert.
  combine      ``binding.combine``: the gates join a token's expert rows; norm, residual scale, residual sum, norm.
  combine_bwd  ``binding.combine_backward``.

With ``own`` false, ``run`` computes the same in elementary torch operations: 32-bit products of the experts' tokens, padded to
the busiest expert (of single tokens where there are no more pairs than experts), and elementwise arithmetic.

Layouts: ``X [T,h]``, ``W1 [M,h,2s]`` (gate columns, then the other projection's), ``W2 [M,s,h]``, ``Y [T*k,h]`` in bf16; ``idx``,
``offsets``, ``pairs`` as the router and its dispatch leave them; ``hidden [T*k,2s]`` in the order of ``pairs``.
"""
import math

import torch

own = False

# Ranges that the cases stand for: tokens; hidden size, width of an expert and experts; slots per token.
T_MAX, H_MIN, H_MAX, S_MIN, S_MAX, M_MAX, K_MAX = 65536, 64, 4096, 8, 512, 16384, 16
ROWS_MAX = 65536 * 8 * 2048             # largest T * k * h of a forward pass
WEIGHTS_MAX = 8192 * 2048 * 64          # largest M * h * s of a forward pass
PRODUCT_MAX = 65536 * 8 * 2048 * 64     # largest T * k * h * s of a forward pass
EPS = 1e-6


def _experts(name, T, h, s, M, k, hidden=False):
    return dict(name=name, op="experts", T=T, h=h, s=s, M=M, k=k, hidden=hidden)


def _backward(name, T, h, s, M, k):
    return dict(name=name, op="experts_bwd", T=T, h=h, s=s, M=M, k=k)


def listed():
    return [
        # decode, one sequence: eight experts' weights are read for one token
        _experts("experts_decode_1", 1, 2048, 64, 4096, 8),
        # decode, 64 sequences: nearly every pair has an expert of its own
        _experts("experts_decode_64", 64, 2048, 64, 8192, 8),
        # chunked prefill or a training step on a small model, nothing round about it; keeps what the backward pass reads
        _experts("experts_ragged", 3001, 1000, 40, 504, 6, hidden=True),
        # prefill of a small model with narrow experts: bound by the weights
        _experts("experts_prefill_small", 16384, 512, 64, 4096, 8),
        # prefill with few, wide experts: a thousand tokens each, bound by the products
        _experts("experts_prefill_few", 32768, 512, 256, 256, 8),
        # prefill of a mid-sized model, tens of tokens per expert
        _experts("experts_prefill_mid", 65536, 2048, 64, 8192, 8),
        # backward of a small step with ragged sizes
        _backward("backward_ragged", 2000, 264, 24, 96, 3),
        # backward of a training step: the router's training shape
        _backward("backward_train", 65536, 512, 64, 8192, 4),
        # decode: a few rows, latency
        dict(name="combine_decode", op="combine", T=64, h=4096, k=16, residual="bf16", sum=False),
        # prefill of a mid-sized model
        dict(name="combine_prefill", op="combine", T=65536, h=2048, k=8, residual="bf16", sum=False),
        # training step on a residual stream kept in 32 bits
        dict(name="combine_bwd_ragged", op="combine_bwd", T=3001, h=1000, k=6, residual="fp32"),
        # training step, the router's training shape at the width of a mid-sized model
        dict(name="combine_bwd_train", op="combine_bwd", T=65536, h=2048, k=4, residual="bf16"),
    ]


def _log_int(rng, lo, hi, step=1):
    """An integer spread over the logarithm of [lo, hi], a multiple of ``step``."""
    v = math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))
    return max(lo, min(max(lo, hi), int(round(v / step)) * step))


def draw(rng):
    op = rng.choices(("experts", "experts_bwd", "combine", "combine_bwd"), (6, 4, 2, 2))[0]
    k = _log_int(rng, 1, K_MAX)
    h = _log_int(rng, H_MIN, H_MAX, 8)
    less = 4 if op == "experts_bwd" else 1
    if op in ("combine", "combine_bwd"):
        T = _log_int(rng, 1, min(T_MAX, ROWS_MAX // (k * h)))
        c = dict(op=op, T=T, h=h, k=k, residual=rng.choice(("bf16", "fp32")))
        return dict(c, sum=rng.random() < 0.5) if op == "combine" else c
    s = _log_int(rng, S_MIN, S_MAX, 8)
    M = _log_int(rng, k, min(M_MAX, WEIGHTS_MAX // (less * h * s)))
    T = _log_int(rng, 1, min(T_MAX, ROWS_MAX // (less * k * h), PRODUCT_MAX // (less * k * h * s)))
    c = dict(op=op, T=T, h=h, s=s, M=M, k=k)
    return dict(c, hidden=rng.random() < 0.3) if op == "experts" else c


def _routing(T, M, k, gen):
    """Expert ids of every token, distinct within a row; an eighth of the tokens share a sixteenth of the experts, as clustered
    tokens do.  With them the pairs in expert order and where each expert's run of them starts."""
    def integers(lo, hi, shape):
        return torch.randint(lo, hi, shape, generator=gen, device="cuda")
    first, step = integers(0, M, (T, 1)), integers(1, max(2, M // k), (T, 1))
    hot = M // 16
    idx = (first + step * torch.arange(k, device="cuda")) % M
    if hot >= k:
        near = (first + integers(1, max(2, hot // k), (T, 1)) * torch.arange(k, device="cuda")) % hot
        idx = torch.where(integers(0, 8, (T, 1)) == 0, near, idx)
    flat = idx.reshape(-1)
    counts = torch.bincount(flat, minlength=M)
    offsets = torch.zeros(M + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = counts.cumsum(0)
    pairs = flat.sort(stable=True).indices.to(torch.int32)
    return idx.to(torch.int32), offsets, pairs, int(counts.max())


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))

    def randn(shape, sd=1.0, mean=0.0, dtype=torch.bfloat16):
        v = torch.randn(shape, generator=gen, device="cuda", dtype=dtype)
        return v.mul_(sd).add_(mean) if mean else v.mul_(sd)

    T, h, k = c["T"], c["h"], c["k"]
    gates = torch.randn((T, k), generator=gen, device="cuda").softmax(-1)
    if c["op"] in ("experts", "experts_bwd"):
        s, M = c["s"], c["M"]
        c["idx"], c["offsets"], c["pairs"], c["busiest"] = _routing(T, M, k, gen)
        c["X"] = randn((T, h))
        # weights that keep both projections and the output of a unit-variance token at about unit variance
        c["W1"] = randn((M, h, 2 * s), h ** -0.5)
        c["W2"] = randn((M, s, h), 1.7 * s ** -0.5)
        if c["op"] == "experts_bwd":
            c["hidden"] = randn((T * k, 2 * s))
            c["gate"] = gates
            c["dout"] = randn((T, h), 0.02)
        return c
    rdt = torch.float32 if c["residual"] == "fp32" else torch.bfloat16
    c["w_post"], c["scale"], c["w_pre"] = (randn((h,), sd, m, torch.float32) for sd, m in ((0.1, 1.0), (0.05, 0.3), (0.1, 1.0)))
    c["res"] = randn((T, h), 2.0, dtype=rdt)
    if c["op"] == "combine":
        c["Y"] = randn((T * k, h))
        c["gate"] = gates
    else:
        # the residual sum that the forward pass left, the joined rows that it kept, and both outputs' gradients
        c["joined"] = randn((T, h), k ** -0.5)
        c["dres"] = randn((T, h), 0.02, dtype=rdt)
        c["dx"] = randn((T, h), 0.02)
    return c


def _places(s):
    """For every expert, the pairs in its run padded to the busiest expert's; which of them are pairs; their places in the list."""
    off = s["offsets"].long()
    at = off[:-1, None] + torch.arange(s["busiest"], device="cuda")
    live = at < off[1:, None]
    at = at.clamp_max(s["T"] * s["k"] - 1)
    return s["pairs"].long()[at], live, at


def _plain_experts(s):
    T, h, w, k = s["T"], s["h"], s["s"], s["k"]
    if T * k <= s["M"] and not s["hidden"]:                  # few pairs: each with its own expert's weights
        e = s["idx"].reshape(-1).long()
        u = torch.bmm(s["X"].float().repeat_interleave(k, 0)[:, None], s["W1"][e].float())
        y = torch.bmm(torch.nn.functional.silu(u[..., :w]) * u[..., w:], s["W2"][e].float())
        return dict(y=y[:, 0].bfloat16())
    pair, live, at = _places(s)
    u = torch.bmm(s["X"].float()[pair // k], s["W1"].float())
    y = torch.bmm(torch.nn.functional.silu(u[..., :w]) * u[..., w:], s["W2"].float())
    out = dict(y=torch.empty((T * k, h), dtype=torch.bfloat16, device="cuda"))
    out["y"][pair[live]] = y[live].bfloat16()
    if s["hidden"]:
        out["hidden"] = torch.empty((T * k, 2 * w), dtype=torch.bfloat16, device="cuda")
        out["hidden"][at[live]] = u[live].bfloat16()
    return out


def _plain_experts_backward(s):
    T, h, w, k = s["T"], s["h"], s["s"], s["k"]
    pair, live, at = _places(s)
    there = live[..., None].float()
    x, d = s["X"].float()[pair // k] * there, s["dout"].float()[pair // k] * there
    u = s["hidden"].float()[at]
    g, up, gate = u[..., :w], u[..., w:], s["gate"].reshape(-1)[pair][..., None]
    sig = torch.sigmoid(g)
    act = g * sig * up
    c = torch.bmm(d, s["W2"].float().mT)
    da = gate * c
    du = torch.cat((da * up * sig * (1 + g * (1 - sig)), da * g * sig), -1)
    per_pair = torch.empty((T * k, h), device="cuda")
    per_pair[pair[live]] = torch.bmm(du, s["W1"].float().mT)[live]
    dgate = torch.empty(T * k, device="cuda")
    dgate[pair[live]] = (c * act).sum(-1)[live]
    return dict(dx=per_pair.view(T, k, h).sum(1).bfloat16(), dgate=dgate.view(T, k),
                dw1=torch.bmm(x.mT, du).bfloat16(), dw2=torch.bmm((gate * act).mT, d).bfloat16())


def _inverse_rms(v):
    return torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS)


def _plain_combine(s):
    y = (s["Y"].float().view(s["T"], s["k"], s["h"]) * s["gate"][..., None]).sum(1)
    res = s["res"].float() + s["scale"] * (s["w_post"] * (y * _inverse_rms(y)))
    out = dict(residual=res.to(s["res"].dtype), x=(s["w_pre"] * (res * _inverse_rms(res))).bfloat16())
    return dict(out, sum=y.bfloat16()) if s["sum"] else out


def _plain_combine_backward(s):
    dx, y, res = s["dx"].float(), s["joined"].float(), s["res"].float()
    inv = _inverse_rms(res)
    hat, v = res * inv, dx * s["w_pre"]
    g = s["dres"].float() + inv * (v - hat * (hat * v).mean(-1, keepdim=True))
    inv_y = _inverse_rms(y)
    hat_y, u = y * inv_y, g * s["scale"] * s["w_post"]
    dy = inv_y * (u - hat_y * (hat_y * u).mean(-1, keepdim=True))
    columns = (g * hat_y).sum(0, dtype=torch.float64)
    return dict(dresidual=g.to(s["res"].dtype), dsum=dy.bfloat16(), dw_post=(columns * s["scale"]).float(),
                dscale=(columns * s["w_post"]).float(), dw_pre=(dx * hat).sum(0, dtype=torch.float64).float())


def run(s):
    if own:
        from paper_2609_36301_b200 import binding as mr
        if s["op"] == "experts":
            res = mr.experts(s["X"], s["W1"], s["W2"], s["idx"], s["offsets"], s["pairs"], want_hidden=s["hidden"])
            return dict(y=res.y, hidden=res.hidden) if s["hidden"] else dict(y=res.y)
        if s["op"] == "experts_bwd":
            res = mr.experts_backward(s["X"], s["W1"], s["W2"], s["idx"], s["offsets"], s["pairs"], s["gate"], s["hidden"], s["dout"])
            return dict(dx=res.dx, dgate=res.dgate, dw1=res.dw1, dw2=res.dw2)
        if s["op"] == "combine":
            res = mr.combine(s["Y"], s["gate"], s["res"], s["w_post"], s["scale"], s["w_pre"], eps=EPS, want_sum=s["sum"])
            return dict(residual=res.residual, x=res.x, sum=res.sum) if s["sum"] else dict(residual=res.residual, x=res.x)
        res = mr.combine_backward(s["dres"], s["dx"], s["joined"], s["res"], s["w_post"], s["scale"], s["w_pre"], eps=EPS)
        return dict(dresidual=res.dresidual, dsum=res.dsum, dw_post=res.dw_post, dscale=res.dscale, dw_pre=res.dw_pre)
    if s["op"] == "experts":
        return _plain_experts(s)
    if s["op"] == "experts_bwd":
        return _plain_experts_backward(s)
    return _plain_combine(s) if s["op"] == "combine" else _plain_combine_backward(s)


def work(case):
    T, h, k = case["T"], case["h"], case["k"]
    rows = 2 * T * h
    res = T * h * (4 if case.get("residual") == "fp32" else 2)
    if case["op"] == "combine":
        return dict(bytes=k * rows + 4 * T * k + 2 * res + rows + (rows if case["sum"] else 0) + 12 * h, flops=(2 * k + 9) * T * h)
    if case["op"] == "combine_bwd":
        return dict(bytes=3 * res + 3 * rows + 24 * h, flops=22 * T * h)
    s, M, P = case["s"], case["M"], T * k
    hit = M * (1 - (1 - 1 / M) ** P) if M > 1 else 1         # experts that some pair has, of evenly spread ids
    index = 8 * P + 4 * M
    if case["op"] == "experts":
        return dict(bytes=int(6 * hit * h * s) + rows + k * rows + index + (4 * P * s if case["hidden"] else 0), flops=6 * P * h * s)
    return dict(bytes=int(6 * hit * h * s) + 6 * M * h * s + 3 * rows + 4 * P * s + 8 * P + index, flops=12 * P * h * s)


def exact(case, seed):
    c = prepare(case, seed)
    T, h, k = c["T"], c["h"], c["k"]
    f64 = torch.float64

    def rms(v):
        return (v.pow(2).sum(-1, keepdim=True) / h + EPS).sqrt()

    if c["op"] == "combine":
        y = torch.zeros((T, h), dtype=f64, device="cuda")
        rows = c["Y"].view(T, k, h)
        for j in range(k):
            y += c["gate"][:, j:j + 1].to(f64) * rows[:, j].to(f64)
        r = c["res"].to(f64) + c["scale"].to(f64) * c["w_post"].to(f64) * y / rms(y)
        out = dict(residual=r, x=c["w_pre"].to(f64) * r / rms(r))
        return dict(out, sum=y) if c["sum"] else out
    if c["op"] == "combine_bwd":
        # the chain rule of v -> w v / rms(v), whose Jacobian is (I - v v^T / (h rms^2)) / rms behind the weights
        def through_norm(v, cotangent):
            m = rms(v)
            return cotangent / m - v * (v * cotangent).sum(-1, keepdim=True) / (h * m.pow(3))

        r, y, dx = c["res"].to(f64), c["joined"].to(f64), c["dx"].to(f64)
        g = c["dres"].to(f64) + through_norm(r, dx * c["w_pre"].to(f64))
        both = torch.einsum("th,th->h", g, y / rms(y))
        return dict(dresidual=g, dsum=through_norm(y, g * (c["scale"].to(f64) * c["w_post"].to(f64))),
                    dw_post=both * c["scale"].to(f64), dscale=both * c["w_post"].to(f64),
                    dw_pre=torch.einsum("th,th->h", dx, r / rms(r)))
    s, M = c["s"], c["M"]
    bounds, pairs = c["offsets"].tolist(), c["pairs"].long()
    runs = [(e, a, b) for e, (a, b) in enumerate(zip(bounds, bounds[1:])) if b > a]
    if c["op"] == "experts":
        out = dict(y=torch.zeros((T * k, h), dtype=f64, device="cuda"))
        if c["hidden"]:
            out["hidden"] = torch.zeros((T * k, 2 * s), dtype=f64, device="cuda")
        for e, a, b in runs:
            p = pairs[a:b]
            u = c["X"][p // k].to(f64) @ c["W1"][e].to(f64)
            g = u[:, :s]
            out["y"][p] = (g / (1 + torch.exp(-g)) * u[:, s:]) @ c["W2"][e].to(f64)
            if c["hidden"]:
                out["hidden"][a:b] = u
        return out
    out = dict(dx=torch.zeros((T, h), dtype=f64, device="cuda"), dgate=torch.zeros((T * k,), dtype=f64, device="cuda"),
               dw1=torch.zeros((M, h, 2 * s), dtype=f64, device="cuda"), dw2=torch.zeros((M, s, h), dtype=f64, device="cuda"))
    gates = c["gate"].reshape(-1).to(f64)
    for e, a, b in runs:
        p = pairs[a:b]
        t = p // k
        x, d, u = c["X"][t].to(f64), c["dout"][t].to(f64), c["hidden"][a:b].to(f64)
        g, up = u[:, :s], u[:, s:]
        q = 1 / (1 + torch.exp(-g))
        rows = (g * q * up) @ c["W2"][e].to(f64)
        out["dgate"][p] = (d * rows).sum(-1)
        scaled = gates[p, None] * d
        back = scaled @ c["W2"][e].to(f64).T
        du = torch.cat((back * up * (q + g * q * (1 - q)), back * g * q), -1)
        out["dx"][t] += du @ c["W1"][e].to(f64).T            # an expert has a token once
        out["dw1"][e] = x.T @ du
        out["dw2"][e] = (g * q * up).T @ scaled
    out["dgate"] = out["dgate"].view(T, k)
    return out
