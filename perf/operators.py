"""The 8-bit operators around the expanded projection, as cases that can be timed: the root-mean-square norm with the
residual's addition and e4m3 codes, the quantizers of activations and of weights, the product of codes with a scale for
each block of 128, and the gated product that feeds a down projection.

Activations have the structure of language-model activations that workloads.py uses (Gaussian rows with a few outlier
channels), weights are Gaussian; the hidden sizes are those of workloads.py.
"""
from __future__ import annotations

import torch

own = False

GROUP, TOP, LEAST = 128, 448.0, 2.0 ** -126
EPS = 1e-5
FP8 = torch.float8_e4m3fn
MOST_FLOPS = 2 * 4096 * 14336 * 4096
MOST_VALUES = 4096 * 14336


def _norm(T, d, x="bf16", residual=True):
    return {"do": "norm", "T": T, "d": d, "x": x, "residual": residual}


def _quant(T, d, x="bf16"):
    return {"do": "quant", "T": T, "d": d, "x": x}


def _weights(N, d, x="bf16"):
    return {"do": "weights", "N": N, "d": d, "x": x}


def _gemm(T, K, N):
    return {"do": "gemm", "T": T, "K": K, "N": N}


def _gated(T, K, N):
    return {"do": "gated", "T": T, "K": K, "N": N}


def listed():
    return [
        # one user's next token: the smallest call, all launch
        dict(_norm(1, 2048), name="norm 1 token"),
        # fp32 residual stream of a short prompt whose width is no whole number of groups, first norm of a model: nothing to add
        dict(_norm(333, 2000, "f32", False), name="norm 333 fp32 ragged"),
        # prefill of the 8B-shaped model
        dict(_norm(4096, 4096), name="norm 4096"),
        # eight decoding sequences, the input of a projection that follows no norm
        dict(_quant(8, 8192), name="quantize 8 tokens"),
        # the widest activations of a prefill, in the base precision
        dict(_quant(4096, 14336, "f32"), name="quantize 4096 fp32"),
        # loading a model: one small and one large weight matrix
        dict(_weights(2048, 2048), name="weights 2048"),
        dict(_weights(14336, 4096), name="weights 14336"),
        # the next token through a projection: bound by reading the weights
        dict(_gemm(1, 8192, 2048), name="product 1 token"),
        # a chunk of a chunked prefill, a ragged number of tokens
        dict(_gemm(333, 4096, 4096), name="product 333"),
        # prefill, the largest product of workloads.py
        dict(_gemm(4096, 14336, 4096), name="product 4096"),
        # eight decoding sequences through both projections of the 1B-shaped feed-forward block
        dict(_gated(8, 2048, 8192), name="gated 8 tokens"),
        # an odd number of prompt tokens through those of the 8B-shaped one
        dict(_gated(1999, 4096, 14336), name="gated 1999"),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _width(rng):
    d = _log(rng, 256, 16384)
    return d // 128 * 128 if rng.random() < 0.7 else d


def draw(rng):
    do = rng.choice(("norm", "quant", "weights", "gemm", "gemm", "gated", "gated"))
    if do in ("gemm", "gated"):
        K = max(2, _log(rng, 512, 14336) // 128) * 128
        N = _log(rng, 256, 14336)
        N = max(64, N // 64 * 64) if rng.random() < 0.75 else N
        T = _log(rng, 1, 64) if rng.random() < 0.4 else _log(rng, 65, 4096)
        T = max(1, min(T, MOST_FLOPS // (2 * K * N * (2 if do == "gated" else 1))))
        return _gemm(T, K, N) if do == "gemm" else _gated(T, K, N)
    x = "f32" if rng.random() < 0.3 else "bf16"
    d = _width(rng)
    rows = min(_log(rng, 256, 14336) if do == "weights" else _log(rng, 1, 4096), MOST_VALUES // d)
    if do == "norm":
        return _norm(rows, d, x, rng.random() < 0.7)
    return _quant(rows, d, x) if do == "quant" else _weights(rows, d, x)


_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def _up(n):
    return -(-n // GROUP)


def _activations(T, d, gen):
    x = torch.randn((T, d), device="cuda", generator=gen)
    x[:, torch.randperm(d, device="cuda", generator=gen)[: max(1, d // 100)]] *= 50.0
    return x


def _codes(v, amax):
    """Codes and scales of values whose blocks' largest magnitudes are `amax`, broadcast over the blocks."""
    s = torch.where(amax == 0, torch.ones_like(amax), (amax / TOP).clamp_min(LEAST))
    return (v / s).clamp_(-TOP, TOP).to(FP8), s


def _quant_rows(v):
    """v [T, d] fp32 -> codes [T, whole groups], scales [T, groups]."""
    T, d = v.shape
    G = _up(d)
    v = torch.nn.functional.pad(v, (0, G * GROUP - d)).view(T, G, GROUP)
    q, s = _codes(v, v.abs().amax(2, keepdim=True))
    return q.view(T, G * GROUP), s.view(T, G)


def _quant_blocks(v):
    """v [N, d] fp32 -> codes [N, whole groups], scales [blocks of 128 rows, groups]."""
    N, d = v.shape
    B, G = _up(N), _up(d)
    v = torch.nn.functional.pad(v, (0, G * GROUP - d, 0, B * GROUP - N)).view(B, GROUP, G, GROUP)
    q, s = _codes(v, v.abs().amax((1, 3), keepdim=True))
    return q.view(B * GROUP, G * GROUP)[:N].contiguous(), s.view(B, G)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    state = {"case": case}
    if case["do"] in ("gemm", "gated"):
        T, K, N = case["T"], case["K"], case["N"]
        state["qx"], state["sx"] = _quant_rows(_activations(T, K, gen))
        for name in ("w",) if case["do"] == "gemm" else ("g", "u"):
            state["q" + name], state["s" + name] = _quant_blocks(torch.randn((N, K), device="cuda", generator=gen) / K ** 0.5)
        state["y"] = torch.empty((T, N), dtype=torch.bfloat16, device="cuda")
        return state
    if case["do"] == "weights":
        rows, d, srows = case["N"], case["d"], _up(case["N"])
        state["x"] = (torch.randn((rows, d), device="cuda", generator=gen) / d ** 0.5).to(_DTYPE[case["x"]])
    else:
        rows, d, srows = case["T"], case["d"], case["T"]
        state["x"] = _activations(rows, d, gen).to(_DTYPE[case["x"]])
    if case["do"] == "norm":
        state["weight"] = (1.0 + 0.2 * torch.randn((d,), device="cuda", generator=gen)).to(_DTYPE[case["x"]])
        if case["residual"]:
            state["residual"] = (3.0 * torch.randn((rows, d), device="cuda", generator=gen)).to(_DTYPE[case["x"]])
            state["h"] = torch.empty_like(state["x"])
    state["q"] = torch.empty((rows, _up(d) * GROUP), dtype=FP8, device="cuda")
    state["s"] = torch.empty((srows, _up(d)), dtype=torch.float32, device="cuda")
    return state


def _rows32(q, s):
    return q.float().view(q.shape[0], -1, GROUP) * s[:, :, None]


def _blocks32(q, s):
    return _rows32(q, s.repeat_interleave(GROUP, 0)[: q.shape[0]])


def _product(qx, sx, qw, sw):
    return _rows32(qx, sx).flatten(1) @ _blocks32(qw, sw).flatten(1).t()


def run(state):
    s, case = state, state["case"]
    do = case["do"]
    if own:
        import paper_2503_17513_amd as pme
        if do == "norm":
            return pme.rmsnorm_quant_fp8(s["x"], s["weight"], EPS, s.get("residual"), s.get("h"), s["q"], s["s"])
        if do == "quant":
            return pme.quant_fp8(s["x"], s["q"], s["s"])
        if do == "weights":
            return pme.quantize_weights_fp8(s["x"], s["q"], s["s"])
        if do == "gemm":
            return pme.fp8_gemm(s["qx"], s["sx"], s["qw"], s["sw"], s["y"])
        return pme.fp8_gated_gemm(s["qx"], s["sx"], s["qg"], s["sg"], s["qu"], s["su"], s["y"])
    if do == "norm":
        h = s["x"].float()
        if case["residual"]:
            h = (h + s["residual"].float()).to(s["x"].dtype)          # the sum is kept in the stream's type, and that is what is normalized
        v = h.float()
        v = v * torch.rsqrt(v.square().mean(1, keepdim=True) + EPS) * s["weight"].float()
        return (*_quant_rows(v), h) if case["residual"] else _quant_rows(v)
    if do == "quant":
        return _quant_rows(s["x"].float())
    if do == "weights":
        return _quant_blocks(s["x"].float())
    if do == "gemm":
        return _product(s["qx"], s["sx"], s["qw"], s["sw"]).to(torch.bfloat16)
    g = _product(s["qx"], s["sx"], s["qg"], s["sg"])
    return (g * torch.sigmoid(g) * _product(s["qx"], s["sx"], s["qu"], s["su"])).to(torch.bfloat16)


def work(case):
    """Inputs and weights read once, outputs written once; two operations for each multiply-add of a product, and for each
    value of a norm or quantizer a few."""
    if case["do"] in ("gemm", "gated"):
        T, K, N = case["T"], case["K"], case["N"]
        mats = 2 if case["do"] == "gated" else 1
        weights = N * K + 4 * _up(N) * (K // GROUP)
        return {"bytes": T * K + 4 * T * (K // GROUP) + mats * weights + 2 * T * N, "flops": 2 * mats * T * K * N}
    rows = case["N"] if case["do"] == "weights" else case["T"]
    d, size, G = case["d"], 4 if case["x"] == "f32" else 2, _up(case["d"])
    scales = _up(rows) * G if case["do"] == "weights" else rows * G
    bytes_ = rows * d * size + rows * G * GROUP + 4 * scales
    if case["do"] == "norm":
        bytes_ += d * size + (2 * rows * d * size if case["residual"] else 0)
    return {"bytes": bytes_, "flops": rows * d * (6 if case["do"] == "norm" else 3)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["do"] in ("gemm", "gated"):
        K = case["K"]
        at = torch.arange(K, device="cuda") // 128
        x = s["qx"].double() * s["sx"].double()[:, at]
        y = []
        for name in ("w",) if case["do"] == "gemm" else ("g", "u"):
            rows = torch.arange(case["N"], device="cuda") // 128
            y.append(torch.mm(x, (s["q" + name].double() * s["s" + name].double()[rows][:, at]).t()))
        return y[0] if case["do"] == "gemm" else y[0] / (1 + torch.exp(-y[0])) * y[1]
    v = s["x"].double()
    h = None
    if case["do"] == "norm":
        if case["residual"]:
            h = v + s["residual"].double()
            v = h.to(s["x"].dtype).double()
        v = v / ((v * v).sum(1, keepdim=True) / case["d"] + EPS).sqrt() * s["weight"].double()
    # the codes are the quotients themselves, before their one rounding to 8 bits
    rows, d = v.shape
    whole = torch.zeros((rows, _up(d) * 128), dtype=torch.float64, device="cuda")
    whole[:, :d] = v
    amax = whole.abs().reshape(rows, -1, 128).max(2).values
    if case["do"] == "weights":
        of = torch.arange(rows, device="cuda") // 128
        block = torch.zeros((_up(rows), amax.shape[1]), dtype=torch.float64, device="cuda")
        block.scatter_reduce_(0, of[:, None].expand_as(amax), amax, "amax")
        scale = block / 448
        each = scale[of]
    else:
        each = scale = amax / 448
    q = whole / each.repeat_interleave(128, 1)
    return (q, scale) if h is None else (q, scale, h)
