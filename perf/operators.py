"""Performance cases of the operators around the sparse products of a Transformer layer.

Activations are feature-major as everywhere in this library: [batch, features, tokens], tokens contiguous, rows `pad`
elements further apart than there are tokens where they are a column slice of wider activations.

  norm        h = x + residual, kept for the next block; RMS norm over the features of every token; the result in the
              activations' type, or in int8 with one scale per token: the operand of an int8 product
  dequantize  the int32 result of an int8 product times its row (weight) and column (token) scales
  adapters    low-rank adapters beside a shared projection: every token adds alpha_a U_a (V_a x) of its request's adapter
              to the projection's result; with int8 activations the result is the int32 one, scaled on the way

A case holds: op, dtype (of the activations: f32, f16 or, adapters only, i8), out (norm: f32, f16, i8; the others: the
type of the result), the sizes, batch (problems per call), pad, and for adapters rank, count (adapters loaded) and mix
("tokens": every token is a request of its own; "requests": runs of tokens of ragged lengths).  One token in eight (one
run in eight) has no adapter.
"""
import math

import torch

own = False   # False: elementary torch operations in 32 bits; True: the library's entry points

_TORCH = {"f32": torch.float32, "f16": torch.float16, "i8": torch.int8}
_SIZE = {"f32": 4, "f16": 2, "i8": 1}
_EPS = 1e-6

# Bounds of what draw() may give, taken from the largest listed cases.
_MAX_BYTES = 1.3e8
_MAX_FLOPS = 2.1e9


def _norm(name, dtype, out, K, N, batch=1, pad=0):
    return {"name": name, "op": "norm", "dtype": dtype, "out": out, "K": K, "N": N, "batch": batch, "pad": pad}


def _dequantize(name, out, M, N, batch=1, pad=0):
    return {"name": name, "op": "dequantize", "out": out, "M": M, "N": N, "batch": batch, "pad": pad}


def _adapters(name, dtype, out, M, K, N, rank, count, mix, batch=1, pad=0):
    return {"name": name, "op": "adapters", "dtype": dtype, "out": out, "M": M, "K": K, "N": N, "rank": rank, "count": count,
            "mix": mix, "batch": batch, "pad": pad}


def listed():
    return [
        # one sequence being generated: a single token through the norm before a projection; launch and latency
        _norm("norm_f16_one_token", "f16", "f16", 1024, 1),
        # a batch of sequences being generated, in front of an int8 product
        _norm("norm_i8_decode", "f16", "i8", 4096, 16),
        # the norm in front of the up projection of a feed-forward layer, 8 x 128 tokens, quantised
        _norm("norm_i8_fc_up", "f16", "i8", 768, 1024),
        # odd sizes, a column slice of wider activations, single precision
        _norm("norm_f32_odd_slice", "f32", "f32", 1027, 771, pad=13),
        # prompts through a wide layer
        _norm("norm_f16_large", "f16", "f16", 4096, 4096),
        # the int8 down projection's result, 8 x 128 tokens
        _dequantize("dequantize_f16_fc_down", "f16", 768, 1024),
        # a wide layer's result for prompts, odd number of tokens, rows on odd addresses
        _dequantize("dequantize_f32_large_odd", "f32", 4096, 4093, pad=4),
        # one token, a small adapter: launch and latency
        _adapters("adapters_f16_one_token", "f16", "f16", 1024, 1024, 1, 8, 4, "tokens"),
        # a batch of sequences being generated, every one with an adapter of its own: bound by reading adapters
        _adapters("adapters_f16_decode", "f16", "f16", 4096, 4096, 48, 16, 32, "tokens"),
        # eight prompts of 128 tokens on average through an up projection
        _adapters("adapters_f16_prompts", "f16", "f16", 4096, 1024, 1024, 16, 8, "requests"),
        # odd sizes and rank, a column slice of wider activations, single precision
        _adapters("adapters_f32_odd_slice", "f32", "f32", 1021, 1027, 771, 12, 5, "requests", pad=13),
        # many tokens through an int8 projection with wide adapters
        _adapters("adapters_i8_prompts", "i8", "f16", 4096, 4096, 2048, 64, 16, "requests"),
    ]


def _log_int(rng, lo, hi, steps=(1, 8, 64)):
    """Log-uniform integer; most are rounded to a multiple of 8 or 64, as layer widths are."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    step = rng.choice(steps)
    return int(min(hi, max(lo, round(v / step) * step)))


def draw(rng):
    while True:
        op = rng.choice(["norm", "norm", "dequantize", "adapters", "adapters"])
        N, batch = _log_int(rng, 1, 4096, (1, 1, 8)), rng.choice([1, 1, 1, 1, 3])
        pad = rng.choice([0, 0, 0, 8, rng.randint(1, 64)])
        if op == "norm":
            dtype = rng.choice(["f32", "f16", "f16"])
            case = _norm("", dtype, rng.choice([dtype, "i8"]), _log_int(rng, 64, 8192), N, batch, pad)
        elif op == "dequantize":
            case = _dequantize("", rng.choice(["f32", "f16"]), _log_int(rng, 64, 4096), N, batch, pad)
        else:
            dtype = rng.choice(["f32", "f16", "f16", "i8"])
            out = rng.choice(["f32", "f16"]) if dtype == "i8" else dtype
            case = _adapters("", dtype, out, _log_int(rng, 64, 4096), _log_int(rng, 64, 4096), N,
                             rng.choice([4, 8, 8, 16, 16, 32, 64, rng.randint(1, 64)]), _log_int(rng, 1, 64, (1,)),
                             rng.choice(["tokens", "requests"]), batch, pad)
        del case["name"]
        w = work(case)
        if w["bytes"] <= _MAX_BYTES and w["flops"] <= _MAX_FLOPS:
            return case


def _used(case):
    """Adapters that a call reads, at most."""
    runs = case["N"] * case["batch"] if case["mix"] == "tokens" else _runs(case)
    return min(case["count"], runs)


def _runs(case):
    return max(1, case["N"] * case["batch"] // 128)


def work(case):
    n = case["N"] * case["batch"]
    if case["op"] == "norm":
        e, o = _SIZE[case["dtype"]], _SIZE[case["out"]]
        return {"bytes": case["K"] * n * (3 * e + o) + case["K"] * 4 + (n * 4 if case["out"] == "i8" else 0), "flops": 5 * case["K"] * n}
    if case["op"] == "dequantize":
        return {"bytes": case["M"] * n * (4 + _SIZE[case["out"]]) + (case["M"] + n) * 4, "flops": 2 * case["M"] * n}
    e, o, c = _SIZE[case["dtype"]], _SIZE[case["out"]], 4 if case["dtype"] == "i8" else _SIZE[case["out"]]
    weights = _used(case) * (case["M"] + case["K"]) * case["rank"] * o
    return {"bytes": case["K"] * n * e + case["M"] * n * (c + o) + weights + n * 4, "flops": 2 * case["rank"] * (case["M"] + case["K"]) * n}


def _wide(gen, case, rows, scale=1.0):
    """[batch, rows, N + pad] of N(0, scale^2): the N columns of it are the operand."""
    return torch.randn(case["batch"], rows, case["N"] + case["pad"], generator=gen, device="cuda") * scale


def _index(gen, case):
    """The adapter of every token, -1 for none."""
    n = case["N"] * case["batch"]
    runs = n if case["mix"] == "tokens" else _runs(case)
    adapter = torch.randint(0, case["count"], (runs,), generator=gen, device="cuda", dtype=torch.int32)
    adapter[torch.rand(runs, generator=gen, device="cuda") < 0.125] = -1
    if case["mix"] == "requests":
        cuts = torch.sort(torch.randint(0, n, (runs - 1,), generator=gen, device="cuda")).values
        adapter = adapter[torch.bucketize(torch.arange(n, device="cuda"), cuts, right=True)]
    return adapter.reshape(case["batch"], case["N"])


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    N, b = case["N"], case["batch"]
    uniform = lambda lo, hi, *shape: torch.rand(*shape, generator=gen, device="cuda") * (hi - lo) + lo  # noqa: E731
    if case["op"] == "norm":
        t, K = _TORCH[case["dtype"]], case["K"]
        loud = torch.where(torch.rand(K, 1, generator=gen, device="cuda") < 0.01, 8.0, 1.0)   # a few features are large in every token
        return {"x": _wide(gen, case, K).to(t), "residual": (_wide(gen, case, K, 2.0) * loud).to(t), "gamma": uniform(0.5, 1.5, K)}
    acc = lambda M: torch.round(_wide(gen, case, M, 15000.0)).to(torch.int32)  # noqa: E731
    if case["op"] == "dequantize":
        return {"c": acc(case["M"]), "row": uniform(1e-4, 1e-3, case["M"]), "col": uniform(0.01, 0.1, b, N)}
    M, K, r, A, t = case["M"], case["K"], case["rank"], case["count"], _TORCH[case["out"]]
    s = {"down": (torch.randn(A, r, K, generator=gen, device="cuda") / math.sqrt(K)).to(t),
         "up": (torch.randn(A, M, r, generator=gen, device="cuda") / math.sqrt(r)).to(t),
         "alpha": uniform(0.25, 2.0, A), "index": _index(gen, case)}
    if case["dtype"] == "i8":
        s["x"] = torch.clamp(torch.round(_wide(gen, case, K, 32.0)), -127, 127).to(torch.int8)
        s["c"], s["row"], s["col"] = acc(M), uniform(1e-4, 1e-3, M), uniform(0.01, 0.1, b, N)
    else:
        s["x"], s["c"] = _wide(gen, case, K).to(t), _wide(gen, case, M).to(t)
    return s


def prepare(case, seed):
    """The activations, weights, result buffers and, for the library's calls, the descriptor of the call."""
    s = {"case": case, **_inputs(case, seed)}
    b, N, pad = case["batch"], case["N"], case["pad"]
    rows = case["K"] if case["op"] == "norm" else case["M"]
    s["y"] = torch.empty(b, rows, N + pad, dtype=_TORCH[case["out"]], device="cuda")
    if case["op"] == "norm":
        s["h"] = torch.empty_like(s["x"])
        s["scale"] = torch.empty(b, N, dtype=torch.float32, device="cuda")
        s["values"] = torch.empty(b, rows, N, dtype=torch.float16, device="cuda") if case["out"] == "i8" else None
    if own:
        from paper_2008_11849_amd import sparsert as sp
        kind = {"f32": sp.F32, "f16": sp.F16, "i8": sp.I8}
        ld = N + pad
        s["sp"], s["stream"] = sp, torch.cuda.current_stream().cuda_stream
        if case["op"] == "norm":
            s["call"] = sp.RmsNorm(case["K"], N, dtype=kind[case["dtype"]], out_dtype=kind[case["out"]], eps=_EPS, batch=b, ldx=ld, ldh=ld, ldy=ld)
            s["workspace"] = torch.empty(s["call"].workspace_bytes(), dtype=torch.uint8, device="cuda")
        elif case["op"] == "dequantize":
            s["call"] = sp.Dequantize(case["M"], N, dtype=kind[case["out"]], batch=b, ldc=ld, ldy=ld)
        else:
            s["call"] = sp.Adapters(case["M"], case["K"], N, case["rank"], case["count"], dtype=kind[case["out"]], x_dtype=kind[case["dtype"]],
                                    batch=b, ldx=ld, ldc=ld, ldy=ld)
            s["workspace"] = torch.empty(s["call"].workspace_bytes(), dtype=torch.uint8, device="cuda")
        s["at"] = {k: v.data_ptr() for k, v in s.items() if isinstance(v, torch.Tensor)}
    return s


def _own_norm(s):
    at, N = s["at"], s["case"]["N"]
    s["sp"].rms_norm(s["call"], at["x"], at["residual"], at["gamma"], at["h"], at["y"], at["scale"] if s["values"] is not None else 0,
                     at["workspace"], s["workspace"].numel(), s["stream"])
    if s["values"] is None:
        return {"sum": s["h"][..., :N], "out": s["y"][..., :N]}
    torch.mul(s["y"][..., :N], s["scale"][:, None, :], out=s["values"])   # what the int8 result stands for
    return {"sum": s["h"][..., :N], "out": s["values"], "scale": s["scale"]}


def _own_dequantize(s):
    at = s["at"]
    s["sp"].dequantize(s["call"], at["c"], at["row"], at["col"], at["y"], s["stream"])
    return {"out": s["y"][..., :s["case"]["N"]]}


def _own_adapters(s):
    at = s["at"]
    s["sp"].adapters(s["call"], at["x"], at["down"], at["up"], at["index"], at["alpha"], at["c"], at.get("row", 0), at.get("col", 0), at["y"],
                     at["workspace"], s["workspace"].numel(), s["stream"])
    return {"out": s["y"][..., :s["case"]["N"]]}


def _plain_norm(s):
    N = s["case"]["N"]
    h = s["x"][..., :N].float() + s["residual"][..., :N].float()
    inv = torch.rsqrt((h * h).mean(dim=1) + _EPS)
    v = h * s["gamma"][:, None]
    total = h.to(s["x"].dtype)
    if s["case"]["out"] != "i8":
        return {"sum": total, "out": (v * inv[:, None, :]).to(s["y"].dtype)}
    top = v.abs().amax(dim=1)
    q = torch.round(v * (127.0 / top)[:, None, :])
    scale = top * inv / 127.0
    return {"sum": total, "out": (q * scale[:, None, :]).half(), "scale": scale}


def _plain_dequantize(s):
    return {"out": (s["c"][..., :s["case"]["N"]].float() * s["col"][:, None, :] * s["row"][:, None]).to(s["y"].dtype)}


def _plain_adapters(s):
    """Every adapter against every token as one product; what is not a token's own is masked in between."""
    case, N = s["case"], s["case"]["N"]
    A, r = case["count"], case["rank"]
    x, c = s["x"][..., :N].float(), s["c"][..., :N].float()
    if case["dtype"] == "i8":
        x, c = x * s["col"][:, None, :], c * s["col"][:, None, :] * s["row"][:, None]
    x = x.permute(1, 0, 2).reshape(case["K"], -1)
    t = (s["down"].float().reshape(A * r, -1) @ x).reshape(A, r, -1) * s["alpha"][:, None, None]
    mine = s["index"].reshape(1, 1, -1) == torch.arange(A, device="cuda")[:, None, None]
    t = torch.where(mine, t, torch.zeros_like(t)).reshape(A * r, -1)
    up = s["up"].float().permute(1, 0, 2).reshape(case["M"], A * r)
    y = (up @ t).reshape(case["M"], case["batch"], N).permute(1, 0, 2)
    return {"out": (c + y).to(s["y"].dtype)}


def run(state):
    op = state["case"]["op"]
    if own:
        return _own_norm(state) if op == "norm" else _own_dequantize(state) if op == "dequantize" else _own_adapters(state)
    return _plain_norm(state) if op == "norm" else _plain_dequantize(state) if op == "dequantize" else _plain_adapters(state)


def exact(case, seed):
    s, N = _inputs(case, seed), case["N"]
    if case["op"] == "norm":
        h = s["x"].double()[..., :N] + s["residual"].double()[..., :N]
        rms = torch.sqrt(h.square().sum(dim=1, keepdim=True) / case["K"] + _EPS)
        v = h * s["gamma"].double().reshape(1, -1, 1)
        if case["out"] != "i8":
            return {"sum": h, "out": v / rms}
        step = v.abs().amax(dim=1, keepdim=True) / 127
        return {"sum": h, "out": torch.round(v / step) * (step / rms), "scale": (step / rms)[:, 0]}
    if case["op"] == "dequantize":
        return {"out": s["c"].double()[..., :N] * (s["row"].double().reshape(1, -1, 1) * s["col"].double().reshape(case["batch"], 1, N))}
    x, y = s["x"].double()[..., :N], s["c"].double()[..., :N]
    if case["dtype"] == "i8":
        col = s["col"].double().reshape(case["batch"], 1, N)
        x, y = x * col, y * (s["row"].double().reshape(1, -1, 1) * col)
    y = y.clone()
    for b in range(case["batch"]):
        for a in range(case["count"]):   # one adapter after the other, on its own tokens
            at = torch.nonzero(s["index"][b] == a).reshape(-1)
            if at.numel():
                y[b][:, at] += s["alpha"][a].double() * (s["up"][a].double() @ (s["down"][a].double() @ x[b][:, at].contiguous()))
    return {"out": y}
