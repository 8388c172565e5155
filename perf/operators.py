"""What the operators of a mixture of BitLinear experts are timed and checked on.

Kinds of case:
  route      expert ids of M tokens -> slots sorted by expert, the way back, and where each expert's slots begin
  product    the experts' 1-bit x 8-bit products over the sorted slots; `gather`: codes of tokens, read through the order
             (the projection into the experts), or codes of the slots themselves (the projection out of them)
  backward   the straight-through backward of such a product: gradient of the normalised input and of every latent weight
  combine    slots back to tokens with the router's weights; `train`: and the gradient
  nonlinear  what stands between the two projections: a non-linear function, LayerNorm, the 8-bit quantiser; `train`: with
             an 8-bit checkpoint of the function's input, and the backward pass from that checkpoint

`run` takes the plain form of each in elementary torch operations, or with `own` the library's entry points.
Widths of 2048, 4096 and 8192, 16384 are the hidden and feed-forward widths of the benchmark's layers.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
BLOCK = 128  # elements of a row that share a scale of the checkpoint


def listed():
    return [
        # a decoding step of a serving loop: the router's answer for a few users, nothing but latency
        dict(name="route_m16", kind="route", M=16, top_k=2, E=8, unrouted=0.0),
        # a long prompt over many small experts, a twentieth of it padding
        dict(name="route_m8191", kind="route", M=8191, top_k=8, E=64, unrouted=0.05),
        # one user's token through its two experts: the packed weights of two of eight experts
        dict(name="product_m1", kind="product", M=1, top_k=2, E=8, K=2048, N=8192, gather=True, per_tensor=False),
        # a few dozen users: every expert has a handful of rows, all weights are read
        dict(name="product_m48", kind="product", M=48, top_k=2, E=16, K=4096, N=4096, gather=True, per_tensor=False),
        # a ragged batch on its way out of the experts
        dict(name="product_m700", kind="product", M=700, top_k=2, E=8, K=8192, N=2048, gather=False, per_tensor=False),
        # a long prompt into the experts
        dict(name="product_m4096", kind="product", M=4096, top_k=2, E=8, K=4096, N=16384, gather=True, per_tensor=False),
        # a small training step, some 160 rows an expert
        dict(name="backward_m333", kind="backward", M=333, top_k=2, E=4, K=1024, N=4096, gather=True),
        # a training step at size
        dict(name="backward_m4096", kind="backward", M=4096, top_k=2, E=8, K=2048, N=8192, gather=True),
        # the end of a decoding step
        dict(name="combine_m16", kind="combine", M=16, top_k=2, N=2048, train=False),
        # the end of a training step's layer, forward and backward
        dict(name="combine_m8192", kind="combine", M=8192, top_k=2, N=2048, train=True),
        # between the projections of a decoding step
        dict(name="nonlinear_r32", kind="nonlinear", R=32, K=8192, fn="gelu", per_tensor=False, train=False),
        # between the projections of a training step: the paper's granularity for training, one gamma a tensor
        dict(name="nonlinear_r16384", kind="nonlinear", R=16384, K=8192, fn="gelu", per_tensor=True, train=True),
    ]


def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


# no drawn case costs more than the largest listed one of its kind
_MOST = {"product": 1.1e12, "backward": 5.5e11}


def draw(rng):
    kind = rng.choice(["route", "product", "product", "product", "backward", "backward", "combine", "nonlinear", "nonlinear"])
    M, top_k = _log_int(rng, 1, 8192), rng.choice([1, 2, 2, 3, 4, 8])
    if kind == "route":
        return dict(kind=kind, M=M, top_k=top_k, E=_log_int(rng, max(2, top_k), 128), unrouted=rng.choice([0.0, 0.1, 0.9]))
    if kind == "combine":
        N = _log_int(rng, 64, 8192)
        return dict(kind=kind, M=min(M, max(1, (1 << 25) // (N * top_k))), top_k=top_k, N=N, train=rng.random() < 0.6)
    if kind == "nonlinear":
        K = _log_int(rng, 256, 28672, 32)
        R = min(_log_int(rng, 1, 16384), (1 << 27) // K)
        return dict(kind=kind, R=R, K=K, fn=rng.choice(["relu", "relu2", "gelu", "silu"]),
                    per_tensor=rng.random() < 0.5, train=rng.random() < 0.6)
    c = dict(kind=kind, M=M, top_k=top_k, E=_log_int(rng, max(2, top_k), 32), K=_log_int(rng, 256, 8192, 32),
             N=_log_int(rng, 256, 8192), gather=rng.random() < 0.6)
    if kind == "product":
        c["per_tensor"] = rng.random() < 0.3
    while c["E"] * c["N"] * c["K"] > 1 << 29 and c["E"] > top_k:
        c["E"] -= 1
    while c["E"] * c["N"] * c["K"] > 1 << (29 if kind == "product" else 27) or work(c)["flops"] > _MOST[kind]:
        if work(c)["flops"] > _MOST[kind]:
            c["M"] = max(1, int(c["M"] * 0.7))
        else:
            c["N"] = max(256, int(c["N"] * 0.8))
            c["K"] = max(256, int(c["K"] * 0.9) // 32 * 32)
    return c


def work(case):
    kind = case["kind"]
    if kind == "nonlinear":
        RK = case["R"] * case["K"]
        if not case["train"]:
            return {"bytes": 5 * RK + 8 * case["R"], "flops": 20 * RK}
        # forward: u in, codes out; backward: the gradient in, the gradient out (the checkpoint is neither)
        return {"bytes": 5 * RK + 6 * RK + 8 * case["R"], "flops": 60 * RK}
    M, T = case["M"], case["M"] * case["top_k"]
    if kind == "route":
        return {"bytes": 12 * T + 4 * (case["E"] + 1), "flops": 0}
    if kind == "combine":
        fwd = 4 * T * case["N"] + 8 * T + 4 * M * case["N"]
        return {"bytes": fwd + (6 * T * case["N"] + 4 * M * case["N"] + 4 * T) * case["train"],
                "flops": 2 * T * case["N"] * (3 if case["train"] else 1)}
    E, K, N = case["E"], case["K"], case["N"]
    rows = M if case["gather"] else T
    if kind == "product":
        return {"bytes": rows * K + min(E, T) * N * K // 8 + 4 * T * N, "flops": 2 * T * N * K}
    return {"bytes": 2 * T * N + rows * K + E * N * K // 8 + 4 * T * K + 4 * E * N * K, "flops": 4 * T * N * K}


# ---- inputs ------------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _choices(case, E, g):
    """Expert ids [M, top_k], every token's experts distinct, some experts more popular than others."""
    M, k = case["M"], case["top_k"]
    score = torch.randn(M, E, device="cuda", generator=g) + 0.7 * torch.randn(1, E, device="cuda", generator=g)
    return score.topk(k, dim=1).indices.to(torch.int32)


def _sorted_slots(ids, E):
    """order, position [M, top_k], offsets [E + 1], as the router's step leaves them (every id is an expert's)."""
    order = torch.sort(ids.reshape(-1), stable=True).indices
    position = torch.empty_like(order)
    position[order] = torch.arange(order.numel(), device="cuda")
    counts = (ids.reshape(-1, 1) == torch.arange(E, device="cuda")).sum(0)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    return order.to(torch.int32), position.to(torch.int32).view(ids.shape), offsets.to(torch.int32)


def _codes(rows, K, per_tensor, g):
    x = torch.randn(rows, K, device="cuda", generator=g)
    gamma = x.abs().amax().reshape(1) if per_tensor else x.abs().amax(1)
    codes = (x * (128.0 / gamma).reshape(-1, 1)).round().clamp(-128, 127).to(torch.int8)
    return codes, gamma, codes.sum(1, dtype=torch.int32)


def prepare(case, seed):
    g, kind, st = _gen(seed), case["kind"], dict(case)
    if kind == "nonlinear":
        R, K = case["R"], case["K"]
        # rows of different sizes, as the outputs of a projection have
        st["u"] = torch.randn(R, K, device="cuda", generator=g) * torch.exp(0.5 * torch.randn(R, 1, device="cuda", generator=g))
        if case["train"]:
            st["d_xhat"] = torch.randn(R, K, device="cuda", generator=g) * 1e-3
        return st
    M, k = case["M"], case["top_k"]
    if kind == "route":
        ids = _choices(case, case["E"], g)
        pad = torch.rand(M, 1, device="cuda", generator=g) < case["unrouted"]
        st["ids"] = torch.where(pad, -1, ids).contiguous()
        return st
    if kind == "combine":
        N, T = case["N"], M * k
        _, st["position"], _ = _sorted_slots(_choices(case, max(8, k), g), max(8, k))
        st["y_slots"] = torch.randn(T, N, device="cuda", generator=g)
        st["weights"] = torch.softmax(torch.randn(M, k, device="cuda", generator=g), 1)
        if case["train"]:
            st["d_y"] = torch.randn(M, N, device="cuda", generator=g) * 1e-3
        return st
    E, K, N, T = case["E"], case["K"], case["N"], M * k
    st["order"], _, st["offsets"] = _sorted_slots(_choices(case, E, g), E)
    per_tensor = case.get("per_tensor", True)
    st["codes"], st["gamma"], st["rowsum"] = _codes(M if case["gather"] else T, K, per_tensor, g)
    W = torch.randn(E, N, K, device="cuda", generator=g).mul_(0.02)
    st["beta"] = W.abs().mean(dim=(1, 2), dtype=torch.float64).float()
    # the weights as each side's program keeps them: packed once, or as a matrix of signs
    if own:
        import paper_2310_11453_amd as bl

        st["packed"], _, _ = bl.bitlinear_pack_weights_experts(W)
    else:
        mean = W.mean(dim=(1, 2), dtype=torch.float64).float().view(E, 1, 1)
        st["signs"] = torch.where(W > mean, 1.0, -1.0)
    if kind == "backward":
        st["d_y"] = (torch.randn(T, N, device="cuda", generator=g) * 1e-3).to(torch.bfloat16)
    return st


# ---- the framework's calls ----------------------------------------------------------------------------
def _run_own(st):
    import paper_2310_11453_amd as bl

    kind = st["kind"]
    if kind == "route":
        order, position, offsets = bl.bitlinear_route(st["ids"], st["E"])
        return {"order": order, "position": position, "offsets": offsets}
    if kind == "combine":
        out = {"y": bl.bitlinear_combine(st["y_slots"], st["position"], st["weights"])}
        if st["train"]:
            out["d_y_slots"], out["d_weights"] = bl.bitlinear_combine_backward(
                st["d_y"], st["y_slots"], st["position"], st["weights"])
        return out
    if kind == "nonlinear":
        codes, gamma, _, check, scales = bl.bitlinear_quant_nonlinear(
            st["u"], st["fn"], ln_eps=EPS, per_tensor=st["per_tensor"], checkpoint=st["train"])
        out = {"codes": codes.to(torch.bfloat16), "gamma": gamma}
        if st["train"]:
            out["d_u"] = bl.bitlinear_nonlinear_backward(st["d_xhat"], check, scales, st["fn"], ln_eps=EPS)
        return out
    order, top_k = (st["order"], st["top_k"]) if st["gather"] else (None, 1)
    if kind == "product":
        return {"y": bl.bitlinear_matmul_experts(st["codes"], st["gamma"], st["rowsum"], st["packed"], st["N"], st["beta"],
                                                 st["offsets"], order=order, top_k=top_k, per_tensor=st["per_tensor"])}
    d_x, d_w = bl.bitlinear_backward_ste_experts(st["d_y"], st["codes"], st["gamma"], st["packed"], st["beta"],
                                                 st["offsets"], order=order, top_k=top_k, per_tensor=True)
    return {"d_x": d_x, "d_w": d_w}


# ---- the plain forms ----------------------------------------------------------------------------------
def _f(u, fn):
    """The non-linear function."""
    if fn == "relu":
        return torch.where(u > 0, u, 0)
    if fn == "relu2":
        return torch.where(u > 0, u * u, 0)
    if fn == "gelu":
        return 0.5 * u * (1 + torch.erf(u * math.sqrt(0.5)))
    return u / (1 + torch.exp(-u))


def _df(u, fn):
    """Its derivative (at 0: from the left)."""
    if fn == "relu":
        return (u > 0).to(u.dtype)
    if fn == "relu2":
        return torch.where(u > 0, 2 * u, 0)
    if fn == "gelu":
        return 0.5 * (1 + torch.erf(u * math.sqrt(0.5))) + u * torch.exp(-0.5 * u * u) / math.sqrt(2 * math.pi)
    s = 1 / (1 + torch.exp(-u))
    return s + u * s * (1 - s)


def _plain_nonlinear(st):
    # the normalisation in 64 bits: a code is decided next to a border, as in the library's quantiser
    u, fn = st["u"], st["fn"]
    R, K = u.shape
    h = _f(u, fn).double()
    mean = h.mean(1, keepdim=True)
    xhat = ((h - mean) / torch.sqrt((h - mean).square().mean(1, keepdim=True) + EPS)).float()
    gamma = (xhat.abs().amax().reshape(1) if st["per_tensor"] else xhat.abs().amax(1)).clamp_min(1e-5)
    codes = torch.round(xhat * (128.0 / gamma).reshape(-1, 1)).clamp(-128, 127)
    out = {"codes": codes.to(torch.bfloat16), "gamma": gamma}
    if st["train"]:
        pad = -K % BLOCK
        blocks = torch.cat([u, u.new_zeros(R, pad)], 1).view(R, -1, BLOCK)
        amax = blocks.abs().amax(2, keepdim=True)
        check = torch.round(blocks * torch.where(amax > 0, 127.0 / amax, 0))
        v = (check * (amax / 127.0)).view(R, -1)[:, :K].double()
        h = _f(v, fn)
        mean = h.mean(1, keepdim=True)
        rstd = 1 / torch.sqrt((h - mean).square().mean(1, keepdim=True) + EPS)
        xn, d = (h - mean) * rstd, st["d_xhat"].double()
        d_h = rstd * (d - d.mean(1, keepdim=True) - xn * (d * xn).mean(1, keepdim=True))
        out["d_u"] = (d_h * _df(v, fn)).to(torch.bfloat16)
    return out


def run(st):
    if own:
        return _run_own(st)
    kind = st["kind"]
    if kind == "route":
        ids, E = st["ids"].reshape(-1), st["E"]
        valid = (ids >= 0) & (ids < E)
        key = torch.where(valid, ids, E)
        order = torch.sort(key, stable=True).indices
        slot = torch.arange(order.numel(), device="cuda")
        position = torch.empty_like(order)
        position[order] = slot
        counts = (key.view(-1, 1) == torch.arange(E, device="cuda")).sum(0)
        offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
        order = torch.where(slot < offsets[E], order, -1)
        position = torch.where(valid, position, -1)
        return {"order": order.to(torch.int32), "position": position.to(torch.int32).view(st["ids"].shape),
                "offsets": offsets.to(torch.int32)}
    if kind == "combine":
        pos = st["position"].long()
        out = {"y": (st["weights"].unsqueeze(2) * st["y_slots"][pos]).sum(1)}
        if st["train"]:
            d = torch.empty(st["y_slots"].shape, dtype=torch.bfloat16, device="cuda")
            d[pos.view(-1)] = (st["weights"].unsqueeze(2) * st["d_y"].unsqueeze(1)).to(torch.bfloat16).view(-1, st["N"])
            out["d_y_slots"] = d
            out["d_weights"] = (st["d_y"].unsqueeze(1) * st["y_slots"][pos]).sum(2)
        return out
    if kind == "nonlinear":
        return _plain_nonlinear(st)
    rows = st["order"].long() // st["top_k"] if st["gather"] else slice(None)
    q, cut = st["codes"].float()[rows], st["offsets"].tolist()
    parts = list(zip(cut[:-1], cut[1:], range(st["E"])))
    if kind == "product":
        gamma = st["gamma"] if st["per_tensor"] else st["gamma"][rows].unsqueeze(1)
        y = torch.cat([(q[a:b] @ st["signs"][e].T) * st["beta"][e] for a, b, e in parts])
        return {"y": y * (gamma / 128.0)}
    d = st["d_y"].float()
    d_x = torch.cat([(d[a:b] @ st["signs"][e]) * st["beta"][e] for a, b, e in parts])
    d_w = torch.stack([d[a:b].T @ q[a:b] for a, b, e in parts])
    return {"d_x": d_x, "d_w": d_w.mul_(st["gamma"] / 128.0)}


# ---- the definitions in 64 bits ------------------------------------------------------------------------
def _exact_f(u, fn):
    """(f(u), f'(u))."""
    if fn == "relu":
        return u.clamp_min(0), torch.heaviside(u, torch.zeros_like(u))
    if fn == "relu2":
        return u.clamp_min(0) ** 2, 2 * u.clamp_min(0)
    if fn == "gelu":
        cdf = torch.special.ndtr(u)
        return u * cdf, cdf + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(u)
    return u * s, s * (1 + u * (1 - s))


def exact(case, seed):
    kind = case["kind"]
    if kind == "route":
        return None
    st = prepare(case, seed)
    f64 = torch.float64
    if kind == "nonlinear":
        u = st["u"].to(f64)
        h, _ = _exact_f(u, case["fn"])
        var, mean = torch.var_mean(h, dim=1, correction=0, keepdim=True)
        xhat = (h - mean) / (var + EPS).sqrt()
        gamma = (xhat.abs().max().view(1) if case["per_tensor"] else xhat.abs().max(dim=1).values).clamp_min(1e-5)
        out = {"codes": (xhat * 128 / gamma.view(-1, 1)).round().clamp(-128, 127), "gamma": gamma}
        if case["train"]:
            # each block by its own scale; a last short block is the same, a block of zeros stays one
            whole = torch.nn.functional.pad(u, (0, -case["K"] % BLOCK))
            step = whole.unflatten(1, (-1, BLOCK)).abs().max(dim=2).values.repeat_interleave(BLOCK, 1)[:, : case["K"]] / 127
            v = torch.where(step > 0, (u / step).round() * step, 0)
            h, slope = _exact_f(v, case["fn"])
            var, mean = torch.var_mean(h, dim=1, correction=0, keepdim=True)
            d, n = st["d_xhat"].to(f64), (h - mean) / (var + EPS).sqrt()
            along = d.mean(1, keepdim=True) + n * (n * d).mean(1, keepdim=True)
            out["d_u"] = (d - along) / (var + EPS).sqrt() * slope
        return out
    if kind == "combine":
        p, w, y = st["position"].flatten().long(), st["weights"].to(f64), st["y_slots"].to(f64)
        mine = y.index_select(0, p).view(case["M"], case["top_k"], case["N"])
        out = {"y": torch.matmul(w.unsqueeze(1), mine).squeeze(1)}
        if case["train"]:
            dy = st["d_y"].to(f64)
            out["d_weights"] = torch.matmul(mine, dy.unsqueeze(2)).squeeze(2)
            out["d_y_slots"] = torch.zeros_like(y).index_copy_(0, p, (w.unsqueeze(2) * dy.unsqueeze(1)).flatten(0, 1))
        return out
    signs = st.get("signs")
    if signs is None:
        return None
    token = torch.div(st["order"], case["top_k"], rounding_mode="floor") if case["gather"] else torch.arange(
        st["order"].numel(), device="cuda")
    x = (st["codes"].to(f64) * (st["gamma"].to(f64) / 128).view(-1, 1)).index_select(0, token.int())
    at = st["offsets"].tolist()
    if kind == "product":
        y = torch.empty(x.shape[0], case["N"], dtype=f64, device="cuda")
        for e in range(case["E"]):
            y[at[e]:at[e + 1]] = torch.mm(x[at[e]:at[e + 1]], signs[e].to(f64).t()) * st["beta"][e].to(f64)
        return {"y": y}
    dy = st["d_y"].to(f64)
    dx = torch.empty_like(x)
    dw = torch.empty(signs.shape, dtype=f64, device="cuda")
    for e in range(case["E"]):
        mine = slice(at[e], at[e + 1])
        dx[mine] = torch.mm(dy[mine], signs[e].to(f64)) * st["beta"][e].to(f64)
        dw[e] = torch.mm(dy[mine].t(), x[mine])
    return {"d_x": dx, "d_w": dw}
