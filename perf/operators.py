"""Workloads of the 8-bit integer linear, the expert router and the MoE layer over 8-bit integer experts, as a
program that uses them calls them, beside the same operators in plain torch.

`run` makes one pass: api.w8a8_gemm on a packed weight, api.moe_route on a router's weight, or one forward of an
api.W8MoELayer (where `own` is false: the same from products, sums, exp, comparisons and indexing).  Quantization
everywhere: the scale of a row (a token's activations, an output channel's weights, a routed row's SwiGLU output) is
its largest magnitude over 127 in binary32, its codes are the values over the scale, rounded half to even.  Sizes are
those of workloads.py (expert matrices of Mixtral-8x7B: hidden 4096, ffn 14336; a DeepSeek-MoE-style layer: hidden
2048, 64 + 2 experts of ffn 1408) and generic ones.
"""
import math

import torch

own = False

STD = 0.02                  # of the weights (activations: 1)
FEW_PAIRS = 16              # routed rows up to which the plain layer gathers a copy of an expert's weights per row


def _linear(M, N, K, dtype):
    return dict(kind="linear", M=M, N=N, K=K, dtype=dtype)


def _route(T, H, E, topk, shared, renormalize, dtype):
    return dict(kind="route", T=T, H=H, E=E, topk=topk, shared=shared, renormalize=renormalize, dtype=dtype)


def _moe(T, H, F, E, topk, shared, skew, dtype):
    return dict(kind="moe", T=T, H=H, F=F, E=E, topk=topk, shared=shared, skew=skew, dtype=dtype)


def listed():
    cases = [
        # One sequence's decode step through a dense up projection: the weight's bytes, once.
        ("linear_decode_1", _linear(1, 14336, 4096, "fp16")),
        # A small batch of sequences through a down projection (long K).
        ("linear_decode_16_bf16", _linear(16, 4096, 14336, "bf16")),
        # A chunk of ragged sizes: a vocabulary-like or pruned layer whose sides are no multiples of anything.
        ("linear_ragged_333", _linear(333, 5003, 2731, "fp16")),
        # A long prompt through an up projection, bound by the matrix cores.
        ("linear_prefill_4096_bf16", _linear(4096, 14336, 4096, "bf16")),
        # Routing of one token over eight experts: all latency.
        ("route_1", _route(1, 4096, 8, 2, 0, True, "fp16")),
        # Routing of a decode batch over many experts, with two always-on ones as extra columns.
        ("route_16_bf16", _route(16, 2048, 64, 6, 2, False, "bf16")),
        # Routing of a long prompt over many experts.
        ("route_4096", _route(4096, 2048, 64, 6, 2, False, "fp16")),
        # One token through a layer of many small experts: latency and 69 MB of weights.
        ("moe_deepseek_1_bf16", _moe(1, 2048, 1408, 64, 6, 2, 1.2, "bf16")),
        # Seven tokens (a ragged decode batch) through a layer of a few large experts: most of 1.4 GB of weights.
        ("moe_mixtral_7", _moe(7, 4096, 14336, 8, 2, 0, 0.0, "fp16")),
        # A mixed batch (a few decoding sequences and a short chunk) through a layer whose sides are no multiples.
        ("moe_ragged_45", _moe(45, 1000, 2730, 16, 4, 1, 0.0, "fp16")),
        # A prompt of 512 tokens through the layer of large experts.
        ("moe_mixtral_512_bf16", _moe(512, 4096, 14336, 8, 2, 0, 0.0, "bf16")),
        # A long prompt through the layer of many experts, whose popularity is skewed.
        ("moe_deepseek_4096", _moe(4096, 2048, 1408, 64, 6, 2, 1.2, "fp16")),
    ]
    return [dict(c, name=n) for n, c in cases]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(["fp16", "bf16"])
    kind = rng.choice(["linear", "linear", "route", "moe", "moe"])
    if kind == "linear":
        N, K = _log(rng, 256, 14336), _log(rng, 256, 14336)
        if rng.random() < 0.5:                                  # half of them as layers have them
            N, K = max(64, N // 64 * 64), max(64, K // 64 * 64)
        return _linear(_log(rng, 1, min(4096, 4096 * 14336 * 4096 // (N * K))), N, K, dtype)
    if kind == "route":
        E = _log(rng, 4, 128)
        return _route(_log(rng, 1, 4096), _log(rng, 256, 4096), E, rng.randint(1, min(8, E)), rng.choice([0, 0, 1, 2]),
                      rng.random() < 0.5, dtype)
    H, F, E = _log(rng, 256, 4096), _log(rng, 256, 14336), _log(rng, 4, 64)
    if rng.random() < 0.5:
        H, F = H // 64 * 64, F // 64 * 64
    while E * H * F > 8 * 4096 * 14336:
        E //= 2
    topk, shared = rng.randint(1, min(6, E)), rng.choice([0, 0, 1, 2])
    most = 4096 * 8 * 2048 * 1408 // ((topk + shared) * H * F)
    return _moe(_log(rng, 1, max(1, min(4096, most))), H, F, E, topk, shared, rng.choice([0.0, 1.2]), dtype)


def _type(case):
    return torch.float16 if case["dtype"] == "fp16" else torch.bfloat16


def _generator(seed, part):
    return torch.Generator(device="cuda").manual_seed(seed * 1000 + part)


def _normal(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _activations(case, seed, rows, width):
    """N(0, 1) with a few larger channels, as hidden states have them."""
    g = _generator(seed, 1)
    x = torch.randn((rows, width), generator=g, device="cuda")
    gain = torch.where(torch.rand(width, generator=g, device="cuda") < 0.01, 6.0, 1.0)
    return (x * gain).to(_type(case))


def _expert_matrix(case, seed, e, which):
    """Weight 0 (gate), 1 (up) [F, H] or 2 (down) [H, F] of expert e, fp16."""
    shape = (case["H"], case["F"]) if which == 2 else (case["F"], case["H"])
    return _normal(_generator(seed, 10 + 3 * e + which), shape, STD, torch.float16)


def _routing(case, seed):
    """Ids and gates of a softmax router with random logits; `skew`: expert e's logit falls with the log of its rank."""
    g = _generator(seed, 2)
    T, E, k, ns = case["T"], case["E"], case["topk"], case["shared"]
    logits = torch.randn((T, E), generator=g, device="cuda")
    order = torch.randperm(E, generator=g, device="cuda")
    logits = logits - case["skew"] * torch.log(order.float() + 1.0)
    gates, ids = torch.softmax(logits, dim=1).topk(k, dim=1)
    shared = torch.arange(E, E + ns, device="cuda").expand(T, ns)
    return (torch.cat([ids, shared], dim=1).to(torch.int32).contiguous(),
            torch.cat([gates, torch.ones((T, ns), device="cuda")], dim=1).contiguous())


# ---- the plain form -------------------------------------------------------------------------------------------

def _quantize(x):
    """Codes (whole numbers in fp32) and scales of the rows of x.  The quotient next to a border between two codes
    decides which one it is, so it is taken in 64 bits."""
    top = x.float().abs().amax(dim=-1, keepdim=True)
    scale = top / torch.full_like(top, 127.0)
    codes = torch.round(x.double() / scale.double()).float()
    return torch.where(scale >= 2.0 ** -126, codes, torch.zeros_like(codes)), scale


def _plain_linear(x, codes, scales):
    """One linear in fp32: x quantized by rows, weight codes [N, K] int8 and scales [N]."""
    xq, xs = _quantize(x)
    return (xq @ codes.float().t()) * xs * scales


def _plain_route(x, wg, topk, renormalize, shared):
    """Which experts are chosen hangs on the last bits of the logits, so these are 64-bit sums."""
    logits = x.double() @ wg.double().t()
    top, ids = torch.sort(logits, dim=1, descending=True, stable=True)
    weight = torch.exp(top - top[:, :1])
    total = weight[:, :topk].sum(1, keepdim=True) if renormalize else weight.sum(1, keepdim=True)
    T, E = logits.shape
    extra = torch.arange(E, E + shared, device=x.device).expand(T, shared)
    return (torch.cat([ids[:, :topk], extra], dim=1).to(torch.int32),
            torch.cat([(weight[:, :topk] / total).float(), torch.ones((T, shared), device=x.device)], dim=1))


def _silu_times(a, b):
    return a / (1.0 + torch.exp(-a)) * b


def _plain_moe(x, codes, scales, ids, gates):
    """codes: three int8 arrays [E, F, H], [E, F, H], [E, H, F]; scales: three of [E, rows]."""
    T, k = ids.shape
    if T * k <= FEW_PAIRS:
        e = ids.flatten().long()
        xq, xs = _quantize(x.repeat_interleave(k, dim=0))
        a, b = ((codes[i][e].float() @ xq[:, :, None])[:, :, 0] * xs * scales[i][e] for i in (0, 1))
        hq, hs = _quantize(_silu_times(a, b))
        y = (codes[2][e].float() @ hq[:, :, None])[:, :, 0] * hs * scales[2][e]
        return (y * gates.flatten()[:, None]).view(T, k, -1).sum(1).to(x.dtype)
    # Every expert on its own tokens: a batched product over all of them would multiply E / topk times as much.
    out = torch.zeros(x.shape, dtype=torch.float32, device=x.device)
    for e in range(codes[0].shape[0]):
        token, slot = torch.where(ids == e)
        rows = x[token]
        h = _silu_times(_plain_linear(rows, codes[0][e], scales[0][e]), _plain_linear(rows, codes[1][e], scales[1][e]))
        out[token] += _plain_linear(h, codes[2][e], scales[2][e]) * gates[token, slot][:, None]
    return out.to(x.dtype)


# ---- what the tools call --------------------------------------------------------------------------------------

def prepare(case, seed):
    """The inputs, and the weights as the program keeps them: packed once for the library, int8 codes and scales for
    the plain form."""
    if own:
        from paper_2504_02658_amd import api
    if case["kind"] == "linear":
        w = _normal(_generator(seed, 3), (case["N"], case["K"]), STD, torch.float16)
        state = {"case": case, "x": _activations(case, seed, case["M"], case["K"])}
        if own:
            state["w"] = api.pack_w8(w)
        else:
            codes, scales = _quantize(w)
            state |= {"codes": codes.to(torch.int8), "scales": scales[:, 0].contiguous()}
        return state
    if case["kind"] == "route":
        return {"case": case, "x": _activations(case, seed, case["T"], case["H"]),
                "wg": _normal(_generator(seed, 3), (case["E"], case["H"]), STD, _type(case))}
    ids, gates = _routing(case, seed)
    state = {"case": case, "x": _activations(case, seed, case["T"], case["H"]), "ids": ids, "gates": gates}
    E = case["E"] + case["shared"]
    if own:
        experts = [tuple(api.pack_w8(_expert_matrix(case, seed, e, i)) for i in range(3)) for e in range(E)]
        state["layer"] = api.W8MoELayer(experts, case["H"], case["F"])
    else:
        codes, scales = [], []
        for i in range(3):
            parts = [_quantize(_expert_matrix(case, seed, e, i)) for e in range(E)]
            codes.append(torch.stack([c.to(torch.int8) for c, _ in parts]))
            scales.append(torch.stack([s[:, 0] for _, s in parts]))
        state |= {"codes": codes, "scales": scales}
    return state


def run(state):
    """One pass; returns the linear's or the layer's output, or the router's ids and gates."""
    case, x = state["case"], state["x"]
    if own:
        from paper_2504_02658_amd import api
        if case["kind"] == "linear":
            return api.w8a8_gemm(x, state["w"])
        if case["kind"] == "route":
            return api.moe_route(x, state["wg"], case["topk"], renormalize=case["renormalize"], n_shared=case["shared"])
        return state["layer"].forward(x, state["ids"], state["gates"])
    if case["kind"] == "linear":
        return _plain_linear(x, state["codes"], state["scales"]).to(x.dtype)
    if case["kind"] == "route":
        return _plain_route(x, state["wg"], case["topk"], case["renormalize"], case["shared"])
    return _plain_moe(x, state["codes"], state["scales"], state["ids"], state["gates"])


def work(case):
    if case["kind"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": 2 * M * K + N * K + 4 * N + 2 * M * N, "flops": 2 * M * N * K}
    T, H, E, k = case["T"], case["H"], case["E"], case["topk"] + case["shared"]
    if case["kind"] == "route":
        return {"bytes": 2 * T * H + 2 * E * H + 8 * T * k, "flops": 2 * T * H * E}
    F = case["F"]
    met = E * (1.0 - (1.0 - case["topk"] / E) ** T) + case["shared"]        # experts that some token goes to, of equal popularity
    return {"bytes": int(met * (3 * F * H + 8 * F + 4 * H)) + 4 * T * H + 8 * T * k, "flops": 6 * T * k * H * F}


# ---- in 64 bits, from the definitions -------------------------------------------------------------------------

def _rows64(v):
    """Quantized rows of v as the 64-bit values that they stand for."""
    v = v.to(torch.float64)
    step = (v.abs().max(dim=1).values / 127.0).to(torch.float32).to(torch.float64).unsqueeze(1)
    return step * (v / step).round().clamp(-127, 127)


def exact(case, seed):
    if case["kind"] == "linear":
        w = _normal(_generator(seed, 3), (case["N"], case["K"]), STD, torch.float16)
        return torch.mm(_rows64(_activations(case, seed, case["M"], case["K"])), _rows64(w).t())
    x = _activations(case, seed, case["T"], case["H"])
    if case["kind"] == "route":
        wg = _normal(_generator(seed, 3), (case["E"], case["H"]), STD, _type(case))
        p = torch.softmax(torch.mm(x.to(torch.float64), wg.to(torch.float64).t()), dim=1)
        chosen = torch.argsort(-p, dim=1, stable=True)[:, :case["topk"]]
        gate = torch.gather(p, 1, chosen)
        if case["renormalize"]:
            gate = gate / gate.sum(dim=1, keepdim=True)
        T, E, ns = case["T"], case["E"], case["shared"]
        extra = torch.arange(E, E + ns, device="cuda").repeat(T, 1)
        return (torch.cat([chosen, extra], 1).to(torch.int32),
                torch.cat([gate, torch.ones((T, ns), dtype=torch.float64, device="cuda")], 1))
    ids, gates = _routing(case, seed)
    xq = _rows64(x)
    y = torch.zeros_like(xq)
    for e in torch.unique(ids).tolist():
        rows, cols = (ids == e).nonzero(as_tuple=True)
        w1, w3, w2 = (_rows64(_expert_matrix(case, seed, e, i)) for i in range(3))
        gate_in = torch.mm(xq[rows], w1.t())
        h = torch.sigmoid(gate_in) * gate_in * torch.mm(xq[rows], w3.t())
        y.index_add_(0, rows, torch.mm(_rows64(h), w2.t()) * gates[rows, cols].to(torch.float64).unsqueeze(1))
    return y
