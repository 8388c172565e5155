"""What the operators around an 8-bit linear layer are timed and checked on.

Beside the 1-bit projections a model keeps layers whose weights have 8 bits (the paper holds its input and output
embeddings so): the same 8-bit activations, int8 weights with a scale for each output channel.  Kinds of case:
  norm      the residual's addition, root-mean-square norm and the 8-bit quantiser in one pass: the updated residual, codes,
            gamma (a scale for each token, or one for the tensor) and the codes' sums
  norm_backward  from the gradient of the normalised input to that of the residual stream (its own gradient added) and
            of the gain
  pack      the weights' quantiser: int8 codes and a scale for each channel, and back to the values they stand for
  product   int8 codes x int8 weights, scaled by token and channel
  backward  the straight-through backward of that product: gradients of the normalised input and of the latent weight

`run` takes the plain form of each in elementary torch operations, or with `own` the library's entry points.
Widths of 2048, 4096, 7168 and 8192, 16384, 28672 are the hidden and feed-forward widths of the benchmark's layers.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one user's decoding step: nothing but latency
        dict(name="norm_m1", kind="norm", M=1, K=2048, x="bf16", h="bf16", residual=True, gain=True, per_tensor=False),
        # a training step: one gamma a tensor, everything in fp32
        dict(name="norm_m8192", kind="norm", M=8192, K=4096, x="fp32", h="fp32", residual=True, gain=True, per_tensor=True),
        # a short sequence, the residual stream and its gradient in bf16
        dict(name="norm_backward_m333", kind="norm_backward", M=333, K=2048, g="bf16", h="bf16", d="bf16", residual=True,
             gain=True),
        # a training step at size, the residual stream in fp32
        dict(name="norm_backward_m8192", kind="norm_backward", M=8192, K=4096, g="bf16", h="fp32", d="fp32", residual=True,
             gain=True),
        # a model's weights in bf16, laid out once for serving
        dict(name="pack_2048", kind="pack", N=2048, K=8192, w="bf16"),
        # the latent weights of a training step, quantised in every step
        dict(name="pack_16384", kind="pack", N=16384, K=4096, w="fp32"),
        # one user's token through a small layer
        dict(name="product_m1", kind="product", M=1, K=2048, N=8192, y="bf16", per_tensor=False),
        # a batch of users through the largest layer: 206 MB of weights
        dict(name="product_m64", kind="product", M=64, K=7168, N=28672, y="bf16", per_tensor=False),
        # a short prompt of odd length, an odd number of channels, a reduction that is no whole tile
        dict(name="product_m333", kind="product", M=333, K=8160, N=2045, y="fp32", per_tensor=False),
        # a long prompt
        dict(name="product_m4096", kind="product", M=4096, K=4096, N=16384, y="bf16", per_tensor=False),
        # a small training step
        dict(name="backward_m333", kind="backward", M=333, K=2048, N=2048),
        # a training step at size
        dict(name="backward_m8192", kind="backward", M=8192, K=4096, N=16384),
    ]


def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


# no drawn case costs more than the largest listed one of its kind: elements, or operations
_MOST = {"norm": 1 << 25, "norm_backward": 1 << 25, "pack": 1 << 26, "product": 5.4e11, "backward": 2.1e12}


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm_backward", "norm_backward", "pack", "product", "product", "product", "backward"])
    some = lambda: rng.choice(["fp32", "bf16"])  # noqa: E731
    if kind in ("norm", "norm_backward"):
        K = _log_int(rng, 256, 28672, 32)
        c = dict(kind=kind, M=min(_log_int(rng, 1, 16384), _MOST[kind] // K), K=K, h=some(), residual=rng.random() < 0.8,
                 gain=rng.random() < 0.7)
        if kind == "norm":
            return dict(c, x=some(), per_tensor=rng.random() < 0.4)
        return dict(c, g=some(), d=some())
    K = _log_int(rng, 256, 16384, 32)
    if kind == "pack":
        return dict(kind=kind, N=min(_log_int(rng, 64, 32768), _MOST[kind] // K), K=K, w=some())
    c = dict(kind=kind, M=_log_int(rng, 1 if kind == "product" else 16, 8192), K=K, N=_log_int(rng, 256, 28672))
    if kind == "product":
        c.update(y=some(), per_tensor=rng.random() < 0.3)
    while c["N"] * c["K"] > (200 if kind == "product" else 64) << 20 or work(c)["flops"] > _MOST[kind]:
        if c["N"] * c["K"] > 64 << 20:
            c["N"] = max(256, int(c["N"] * 0.8))
        else:
            c["M"] = max(1, int(c["M"] * 0.7))
    return c


def _size(name):
    return TYPES[name].itemsize


def work(case):
    kind, K = case["kind"], case["K"]
    if kind == "pack":
        # the weights in, codes and scales out, and the values they stand for
        NK = case["N"] * K
        return {"bytes": (_size(case["w"]) + 1 + 2) * NK + 4 * case["N"], "flops": 4 * NK}
    M = case["M"]
    if kind == "norm":
        h = _size(case["h"]) if case["residual"] else 0
        return {"bytes": (_size(case["x"]) + 2 * h + 1) * M * K + 8 * M + 4 * K * case["gain"], "flops": 8 * M * K}
    if kind == "norm_backward":
        d = _size(case["d"])
        return {"bytes": (_size(case["g"]) + _size(case["h"]) + d * (2 if case["residual"] else 1)) * M * K +
                8 * K * case["gain"], "flops": 10 * M * K}
    N = case["N"]
    if kind == "product":
        return {"bytes": M * K + N * K + _size(case["y"]) * M * N + 4 * (M + N), "flops": 2 * M * N * K}
    return {"bytes": 2 * M * N + M * K + N * K + 2 * M * K + 4 * N * K, "flops": 4 * M * N * K}


# ---- inputs ------------------------------------------------------------------------------------------
def _randn(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _weights(case, g):
    """int8 codes [N, K] and a scale for each channel, channels of different sizes."""
    N, K = case["N"], case["K"]
    W = _randn(g, N, K).mul_(0.02 * torch.exp(0.3 * _randn(g, N, 1)))
    most = W.abs().amax(1)
    return torch.round(W * (127.0 / most).unsqueeze(1)).to(torch.int8), most / 127.0


def _codes(M, K, per_tensor, g):
    x = _randn(g, M, K)
    gamma = x.abs().amax().reshape(1) if per_tensor else x.abs().amax(1)
    return (x * (128.0 / gamma).reshape(-1, 1)).round().clamp(-128, 127).to(torch.int8), gamma


def prepare(case, seed):
    g, kind, st = torch.Generator(device="cuda").manual_seed(seed), case["kind"], dict(case)
    K = case["K"]
    if kind == "pack":
        st["W"] = (_randn(g, case["N"], K) * (0.02 * torch.exp(0.3 * _randn(g, case["N"], 1)))).to(TYPES[case["w"]])
        return st
    M = case["M"]
    if kind in ("norm", "norm_backward"):
        # a residual stream: rows of different sizes, a few channels much larger than the others
        size = torch.exp(0.5 * _randn(g, M, 1)) * torch.where(torch.rand(1, K, device="cuda", generator=g) < 0.005, 12.0, 1.0)
        st["gain_"] = 1.0 + 0.2 * _randn(g, K) if case["gain"] else None
        stream = (_randn(g, M, K) * size).to(TYPES[case["h"]])
        if kind == "norm":
            st["x_"] = _randn(g, M, K).to(TYPES[case["x"]]) if case["residual"] else stream.to(TYPES[case["x"]])
            st["residual_"] = stream if case["residual"] else None
            return st
        st["h_"] = stream
        st["g_"] = (_randn(g, M, K) * 1e-3).to(TYPES[case["g"]])
        st["d_"] = (_randn(g, M, K) * 1e-3).to(TYPES[case["d"]]) if case["residual"] else None
        return st
    st["codes"], st["gamma"] = _codes(M, K, case.get("per_tensor", True), g)
    w, st["scale"] = _weights(case, g)
    # the weights as each side's program keeps them: laid out once, or as a matrix of codes
    if own:
        import paper_2310_11453_amd as bl

        st["packed"], _ = bl.bitlinear_pack_weights_i8(w)
    else:
        st["w_codes"] = w
    if kind == "backward":
        st["d_y"] = (_randn(g, M, case["N"]) * 1e-3).to(torch.bfloat16)
    return st


# ---- the framework's calls ----------------------------------------------------------------------------
def _run_own(st):
    import paper_2310_11453_amd as bl

    kind = st["kind"]
    if kind == "norm":
        codes, gamma, rowsum, h, _ = bl.bitlinear_quant_rmsnorm(st["x_"], st["residual_"], gain=st["gain_"], eps=EPS,
                                                                per_tensor=st["per_tensor"])
        out = {"codes": codes.to(torch.bfloat16), "gamma": gamma, "rowsum": rowsum}
        if st["residual"]:
            out["h"] = h
        return out
    if kind == "norm_backward":
        got = bl.bitlinear_rmsnorm_backward(st["g_"], st["h_"], gain=st["gain_"], eps=EPS, dresidual=st["d_"],
                                            want_dgain=st["gain"], dtype=TYPES[st["d"]])
        return {"d_h": got[0], "d_gain": got[1]} if st["gain"] else {"d_h": got}
    if kind == "pack":
        packed, scale = bl.bitlinear_pack_weights_i8(st["W"])
        return {"values": bl.bitlinear_unpack_weights_i8(packed, scale, st["N"], st["K"], dtype=torch.bfloat16),
                "scale": scale}
    if kind == "product":
        return {"y": bl.bitlinear_matmul_i8(st["codes"], st["gamma"], st["packed"], st["N"], st["scale"],
                                            per_tensor=st["per_tensor"], dtype=TYPES[st["y"]])}
    d_x, d_w = bl.bitlinear_backward_ste_i8(st["d_y"], st["codes"], st["gamma"], st["packed"], st["scale"],
                                            per_tensor=True, dtype=torch.bfloat16)
    return {"d_x": d_x, "d_w": d_w}


# ---- the plain forms ----------------------------------------------------------------------------------
def run(st):
    if own:
        return _run_own(st)
    kind = st["kind"]
    if kind == "norm":
        x, gain = st["x_"].float(), st["gain_"]
        h = x if st["residual_"] is None else (x + st["residual_"].float()).to(TYPES[st["h"]])
        # the normalisation in 64 bits: a code is decided next to a border
        hd = h.double()
        xhat = (hd / torch.sqrt((hd * hd).mean(1, keepdim=True) + EPS)).float()
        if gain is not None:
            xhat = xhat * gain
        gamma = (xhat.abs().amax().reshape(1) if st["per_tensor"] else xhat.abs().amax(1)).clamp_min(1e-5)
        codes = torch.round(xhat * (128.0 / gamma).reshape(-1, 1)).clamp(-128, 127)
        out = {"codes": codes.to(torch.bfloat16), "gamma": gamma, "rowsum": codes.sum(1, dtype=torch.float64).to(torch.int32)}
        if st["residual"]:
            out["h"] = h
        return out
    if kind == "norm_backward":
        hd, g = st["h_"].double(), st["g_"].double()
        rstd = 1 / torch.sqrt((hd * hd).mean(1, keepdim=True) + EPS)
        n = hd * rstd
        gn = g if st["gain_"] is None else g * st["gain_"]
        d = rstd * (gn - n * (gn * n).mean(1, keepdim=True))
        if st["d_"] is not None:
            d = d + st["d_"]
        out = {"d_h": d.to(TYPES[st["d"]])}
        if st["gain"]:
            out["d_gain"] = (g * n).sum(0).float()
        return out
    if kind == "pack":
        W = st["W"].float()
        most = W.abs().amax(1, keepdim=True)
        scale = most / 127.0
        codes = torch.round(W * (127.0 / most))
        return {"values": (codes * scale).to(torch.bfloat16), "scale": scale.reshape(-1)}
    q, w = st["codes"].float(), st["w_codes"].float()
    if kind == "product":
        y = (q @ w.T) * ((st["gamma"] / 128.0).reshape(-1, 1) * st["scale"])
        return {"y": y.to(TYPES[st["y"]])}
    d = st["d_y"].float()
    return {"d_x": ((d * st["scale"]) @ w).to(torch.bfloat16), "d_w": (d.T @ q) * (st["gamma"] / 128.0)}


# ---- the definitions in 64 bits ------------------------------------------------------------------------
def exact(case, seed):
    st, kind, f64 = prepare(case, seed), case["kind"], torch.float64
    if kind in ("norm", "norm_backward"):
        gain = torch.ones(case["K"], dtype=f64, device="cuda") if st["gain_"] is None else st["gain_"].to(f64)
    if kind == "norm":
        h = st["x_"].to(f64)
        if case["residual"]:
            h = torch.add(h, st["residual_"].to(f64)).to(TYPES[case["h"]]).to(f64)
        rms = (h.square().sum(1, keepdim=True) / case["K"] + EPS).sqrt()
        xhat = h / rms * gain
        gamma = torch.linalg.vector_norm(xhat, math.inf, dim=None if case["per_tensor"] else 1).view(-1).clamp_min(1e-5)
        out = {"codes": (xhat * 128 / gamma.view(-1, 1)).round().clamp(-128, 127), "gamma": gamma, "rowsum": None}
        if case["residual"]:
            out["h"] = h
        return out
    if kind == "norm_backward":
        h, g = st["h_"].to(f64), st["g_"].to(f64)
        rms = (h.square().sum(1, keepdim=True) / case["K"] + EPS).sqrt()
        t = g * gain
        along = (t * h).sum(1, keepdim=True) / (case["K"] * rms.square())
        d = (t - h * along) / rms
        out = {"d_h": d if st["d_"] is None else d + st["d_"].to(f64)}
        if case["gain"]:
            out["d_gain"] = torch.einsum("mk,mk->k", g, h / rms)
        return out
    if kind == "pack":
        W = st["W"].to(f64)
        step = torch.linalg.vector_norm(W, math.inf, dim=1) / 127
        return {"values": (W / step.view(-1, 1)).round() * step.view(-1, 1), "scale": step}
    w = st.get("w_codes")
    if w is None:
        return None
    values = w.to(f64) * st["scale"].to(f64).view(-1, 1)
    x = st["codes"].to(f64) * (st["gamma"].to(f64) / 128).view(-1, 1)
    if kind == "product":
        return {"y": torch.mm(x, values.t())}
    dy = st["d_y"].to(f64)
    return {"d_x": torch.mm(dy, values), "d_w": torch.mm(dy.t(), x)}
