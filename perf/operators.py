"""The operators around a factored layer in 8 bits, as cases to time: the norm before a block, the norm after it with its
gate and residual, the quantiser (with the SiLU gate or without) and the matrix product of 8-bit operands with a scale for
each block of 128.

8-bit values are e4m3 codes with scales.  Activations [R, C] have a scale per row and 128 columns, laid out
[ceil(C / 128), R]: the block's largest magnitude over 448, at least 2^-100, rounded to bf16.  Weights [N, K] have an fp32
scale per 128 x 128, laid out [ceil(N / 128), ceil(K / 128)].

A case is one call with what a program holds before it: activations, weights, norm parameters and, as a serving loop keeps
them, the buffers that the results go to.  With ``own`` false the operators are computed from elementary torch operations in
32 bits; with it, by the library.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK, LARGEST, SMALLEST_SCALE, EPS = 128, 448.0, 2.0 ** -100, 1e-6


def _norm_in(M, d, type="bf16", out="f8", add=True, kind="rms"):
    return dict(op="norm_in", M=M, d=d, type=type, out=out, add=add, kind=kind)


def _norm_out(M, d, type="bf16", res="bf16", gate="none", gate_rows=1, norm=True, branch=False, out="none", kind="rms"):
    return dict(op="norm_out", M=M, d=d, type=type, res=res, gate=gate, gate_rows=gate_rows, norm=norm, branch=branch,
                out=out, kind=kind)


def _quantize(M, d, type="bf16", gated=True):
    return dict(op="quantize", M=M, d=d, type=type, gated=gated)


def _matmul(M, K, N, out="bf16"):
    return dict(op="matmul", M=M, K=K, N=N, out=out)


def listed():
    named = dict(
        # one token of one sequence: the branch before joins the residual, and the norm hands 8-bit codes to the first product
        norm_in_m1=_norm_in(1, 4096),
        # a prefill of the benchmark's headline layer, the same chain
        norm_in_m4096=_norm_in(4096, 4096),
        # off every tile and vector: odd rows, odd row length, fp32, mean and bias (a model checked before it goes to 8 bits)
        norm_in_f32_ragged=_norm_in(1777, 2687, "f32", "f32", False, "layer"),
        # a decode batch: norm after the block, residual, and the next block's norm to 8 bits in the same pass
        norm_out_m16=_norm_out(16, 4096, out="f8"),
        # the widest layer, fp32 residual stream, a gate per sequence of 512 tokens and a scale per channel
        norm_out_wide=_norm_out(8192, 5120, res="f32", gate="tanh", gate_rows=512, branch=True, out="bf16"),
        # the gated activation of a decode batch on its way to the down projection
        quantize_gated_m16=_quantize(16, 14336),
        # ... and of a prefill
        quantize_gated_m4096=_quantize(4096, 14336),
        # one token through a wide layer: the weights are read once, nothing else counts
        matmul_m1=_matmul(1, 4096, 14336),
        # a decode batch into the rank of the down projection: a long contraction for few outputs, which leave in 8 bits
        matmul_m16_rank=_matmul(16, 14336, 512, "f8"),
        # a larger decode batch on the small layer of the benchmark
        matmul_m128=_matmul(128, 2048, 8192),
        # a prompt off every tile: rows, columns and contraction odd
        matmul_m1777_ragged=_matmul(1777, 2687, 7301),
        # the shape of the paper's kernel evaluation as one dense product
        matmul_m4096=_matmul(4096, 8192, 16384),
    )
    return [dict(name=k, **c) for k, c in named.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A row length: mostly a multiple of 128 as model configurations have them, sometimes any number."""
    n = _log(rng, lo, hi)
    return max(128, n // 128 * 128) if rng.random() < 0.65 else n


def draw(rng):
    """One more case: the operator first, then sizes spread over its range."""
    op = rng.choice(["norm_in", "norm_out", "quantize", "matmul", "matmul"])
    while True:
        M = _log(rng, 1, 8192)
        if op == "matmul":
            c = _matmul(M, _width(rng, 100, 16384), _width(rng, 100, 16384), rng.choice(["bf16", "bf16", "f8"]))
            if c["M"] * c["K"] * c["N"] <= 4096 * 8192 * 16384 and c["K"] * c["N"] <= 8192 * 16384:
                return c
            continue
        if op == "quantize":
            return _quantize(M, _width(rng, 200, 14336), rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.6)
        d, type, kind = _width(rng, 100, 8192), rng.choice(["bf16", "bf16", "f32"]), rng.choice(["rms", "rms", "layer"])
        if M * d > 8192 * 5120:
            continue
        if op == "norm_in":
            return _norm_in(M, d, type, rng.choice(["f8", type]), rng.random() < 0.6, kind)
        return _norm_out(M, d, type, rng.choice(["f32", type]), rng.choice(["none", "plain", "sigmoid", "tanh"]),
                         rng.choice([1, 1, 7, 512]), rng.random() < 0.7, rng.random() < 0.5, rng.choice(["none", "f8", type]), kind)


def _expand(scales, width):
    """[blocks of 128 columns, rows] -> [rows, width]"""
    return scales.t().repeat_interleave(BLOCK, 1)[:, :width]


def _coded(v):
    """Codes and scales, per row and 128 columns, of fp32 v."""
    R, C = v.shape
    nb = -(-C // BLOCK)
    amax = torch.nn.functional.pad(v, (0, nb * BLOCK - C)).view(R, nb, BLOCK).abs().amax(2)
    s = torch.clamp(amax / LARGEST, min=SMALLEST_SCALE).t().contiguous().to(torch.bfloat16)
    # a scale that was rounded down leaves at most 449.75, which rounds to 448
    return (v / _expand(s.float(), C)).to(torch.float8_e4m3fn), s


def _empty(out, M, d):
    """The buffer of a result: rows of codes are padded to 16 bytes."""
    if out == "f8":
        return (torch.empty(M, -(-d // 16) * 16, device="cuda", dtype=torch.float8_e4m3fn)[:, :d],
                torch.empty(-(-d // BLOCK), M, device="cuda", dtype=torch.bfloat16))
    return None if out == "none" else torch.empty(M, d, device="cuda", dtype=_DTYPES[out])


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(*shape, generator=g, device="cuda").mul_(std).add_(mean)

    def activation(M, d, type):
        """Rows of different sizes, and one channel in 50 ten times larger, as residual streams have them."""
        size = torch.where(torch.rand(d, generator=g, device="cuda") < 0.02, 10.0, 1.0) * torch.exp(normal(M, 1, std=0.5))
        return (normal(M, d) * size).to(_DTYPES[type])

    s, M = dict(case=case), case["M"]
    if case["op"] == "matmul":
        K, N = case["K"], case["N"]
        pad = -(-K // 16) * 16       # rows of codes are 16-byte aligned
        for name, v in (("a", activation(M, K, "f32")), ("w", normal(N, K, std=K ** -0.5))):
            if name == "w":          # a scale per 128 x 128
                nb, kb = -(-N // BLOCK), -(-K // BLOCK)
                full = torch.nn.functional.pad(v, (0, kb * BLOCK - K, 0, nb * BLOCK - N)).view(nb, BLOCK, kb, BLOCK)
                scale = (full.abs().amax((1, 3)) / LARGEST).contiguous()
                v = (full / scale[:, None, :, None]).view(nb * BLOCK, kb * BLOCK)[:N, :K].to(torch.float8_e4m3fn)
            else:
                v, scale = _coded(v)
            codes = torch.zeros(v.shape[0], pad, device="cuda", dtype=torch.float8_e4m3fn)
            codes[:, :K] = v
            s[name], s[name + "_scale"] = codes[:, :K], scale
        s["out"] = _empty(case["out"], M, N)
        return s
    d = case["d"]
    if case["op"] == "quantize":
        s.update(x=activation(M, d, case["type"]), u=activation(M, d, case["type"]) if case["gated"] else None,
                 out=_empty("f8", M, d))
        return s
    t = _DTYPES[case["type"]]
    s["weight"] = normal(d, std=0.1, mean=1.0).to(t)
    s["bias"] = normal(d, std=0.1).to(t) if case["kind"] == "layer" else None
    if case["op"] == "norm_in":
        s.update(x=activation(M, d, case["type"]), add=normal(M, d).to(t) if case["add"] else None,
                 h=_empty(case["type"], M, d) if case["add"] else None, out=_empty(case["out"], M, d))
        return s
    s.update(y=activation(M, d, case["type"]), residual=activation(M, d, case["res"]),
             gate=normal(-(-M // case["gate_rows"]), d).to(t) if case["gate"] != "none" else None,
             branch=normal(d, std=0.1, mean=0.5).to(t) if case["branch"] else None,
             next_weight=normal(d, std=0.1, mean=1.0).to(t), h=_empty(case["res"], M, d), out=_empty(case["out"], M, d))
    return s


def _normed(v, kind, weight, bias, wide):
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    n = v / torch.sqrt((v * v).mean(1, keepdim=True) + EPS) * weight.to(wide)
    return n if bias is None else n + bias.to(wide)


def _activated(g, gate):
    return torch.sigmoid(g) if gate == "sigmoid" else torch.tanh(g) if gate == "tanh" else g


def _by_definition(s, wide):
    """The operator in `wide` precision: its outputs before they are rounded to their types."""
    c = s["case"]
    if c["op"] == "matmul":
        a = s["a"].to(wide) * _expand(s["a_scale"].to(wide), c["K"])
        w = s["w"].to(wide) * s["w_scale"].to(wide).repeat_interleave(BLOCK, 0)[:c["N"]].repeat_interleave(BLOCK, 1)[:, :c["K"]]
        return [(a @ w.t(), c["out"])]
    if c["op"] == "quantize":
        x = s["x"].to(wide)
        return [(x / (1 + torch.exp(-x)) * s["u"].to(wide) if c["gated"] else x, "f8")]
    if c["op"] == "norm_in":
        h = s["x"].to(wide)
        outs = []
        if c["add"]:
            h = h + s["add"].to(wide)
            outs = [(h, c["type"])]
        return outs + [(_normed(h, c["kind"], s["weight"], s["bias"], wide), c["out"])]
    b = s["y"].to(wide)
    if c["norm"]:
        b = _normed(b, c["kind"], s["weight"], s["bias"], wide)
    if c["branch"]:
        b = b * s["branch"].to(wide)
    if c["gate"] != "none":
        b = b * _activated(s["gate"].to(wide), c["gate"]).repeat_interleave(c["gate_rows"], 0)[:c["M"]]
    h = s["residual"].to(wide) + b
    outs = [(h, c["res"])]
    if c["out"] != "none":
        outs.append((_normed(h, "rms", s["next_weight"], None, wide), c["out"]))
    return outs


def run(state):
    if not own:
        got = []
        for v, out in _by_definition(state, torch.float32):
            got.append(_coded(v) if out == "f8" else v.to(_DTYPES[out]))
        return got
    from paper_2510_25977_amd import binding as B

    s, c = state, state["case"]
    if c["op"] == "matmul":
        return [B.scaled_matmul((s["a"], s["a_scale"]), (s["w"], s["w_scale"]), out=s["out"])]
    if c["op"] == "quantize":
        return [B.quantize(s["x"], gate_with=s["u"], out=s["out"])]
    norm = dict(rms=B.NORM_RMS, layer=B.NORM_LAYER)
    if c["op"] == "norm_in":
        n = B.norm_in(s["x"], s["weight"], bias=s["bias"], add=s["add"], kind=norm[c["kind"]], eps=EPS, h=s["h"], out=s["out"])
        return [s["h"], n] if c["add"] else [n]
    kind = norm[c["kind"]] if c["norm"] else B.NORM_NONE
    gate = dict(none=B.GATE_PLAIN, plain=B.GATE_PLAIN, sigmoid=B.GATE_SIGMOID, tanh=B.GATE_TANH)[c["gate"]]
    h, n = B.norm_out(s["y"], s["residual"], s["weight"] if c["norm"] else None, bias=s["bias"] if c["norm"] else None,
                      kind=kind, eps=EPS, branch_scale=s["branch"], gate=s["gate"], gate_rows=c["gate_rows"], gate_act=gate,
                      next_weight=s["next_weight"] if c["out"] != "none" else None, h=s["h"], out=s["out"])
    return [h] if c["out"] == "none" else [h, n]


def exact(case, seed):
    """The same in 64 bits, from the operators' definitions, before any result is rounded to its type: codes come as the values
    that they round, v / scale, and scales before they go to bf16."""
    s = prepare(case, seed)
    got = []
    for v, out in _in_64_bits(s, case):
        if out != "f8":
            got.append(v)
            continue
        scales, ratios = [], []
        for at in range(0, v.shape[1], BLOCK):       # a column block at a time
            part = v[:, at:at + BLOCK]
            scale = torch.clamp(torch.max(torch.abs(part), 1)[0] / LARGEST, min=SMALLEST_SCALE)
            scales.append(scale)
            ratios.append(part / scale[:, None])
        got.append((torch.cat(ratios, 1), torch.stack(scales)))
    return got


def _in_64_bits(s, c):
    def f(name):
        return s[name].double()

    def standard(v, kind):
        d = v.shape[1]
        centred = v - v.sum(1, keepdim=True) / d if kind == "layer" else v
        return centred * torch.rsqrt((centred ** 2).sum(1, keepdim=True) / d + EPS)

    if c["op"] == "matmul":
        total = torch.zeros(c["M"], c["N"], dtype=torch.float64, device="cuda")
        step = 16 * BLOCK
        for at in range(0, c["K"], step):            # 16 blocks of the contraction at a time
            end = min(at + step, c["K"])
            blocks = torch.arange(at, end, device="cuda") // BLOCK
            a = f("a")[:, at:end] * f("a_scale")[blocks].t()
            rows = torch.arange(c["N"], device="cuda") // BLOCK
            w = f("w")[:, at:end] * f("w_scale")[rows][:, blocks]
            total += torch.mm(a, w.t().contiguous())
        return [(total, c["out"])]
    if c["op"] == "quantize":
        return [(f("x") * torch.sigmoid(f("x")) * f("u") if c["gated"] else f("x"), "f8")]
    affine = (lambda v: v * f("weight") + f("bias")) if s["bias"] is not None else (lambda v: v * f("weight"))
    if c["op"] == "norm_in":
        h = f("x") + f("add") if c["add"] else f("x")
        n = (affine(standard(h, c["kind"])), c["out"])
        return [(h, c["type"]), n] if c["add"] else [n]
    b = affine(standard(f("y"), c["kind"])) if c["norm"] else f("y")
    if c["branch"]:
        b = b * f("branch")
    if c["gate"] != "none":
        rows = torch.arange(c["M"], device="cuda") // c["gate_rows"]
        gate = f("gate")
        gate = dict(plain=lambda: gate, sigmoid=lambda: 1 / (1 + torch.exp(-gate)), tanh=lambda: 2 / (1 + torch.exp(-2 * gate)) - 1)[c["gate"]]()
        b = b * gate[rows]
    h = f("residual") + b
    return [(h, c["res"])] + ([] if c["out"] == "none" else [(standard(h, "rms") * f("next_weight"), c["out"])])


def work(case):
    """Inputs in once, results out once; two operations a multiply-add."""
    size = dict(bf16=2, f32=4, none=0)
    M, op = case["M"], case["op"]

    def result(out, C):
        return M * C + 2 * M * -(-C // BLOCK) if out == "f8" else M * C * size[out]

    if op == "matmul":
        K, N = case["K"], case["N"]
        kb = -(-K // BLOCK)
        return {"bytes": float(M * K + N * K + 2 * M * kb + 4 * -(-N // BLOCK) * kb + result(case["out"], N)), "flops": 2.0 * M * N * K}
    d, t = case["d"], size[case["type"]]
    if op == "quantize":
        return {"bytes": float(M * d * t * (2 if case["gated"] else 1) + result("f8", d)), "flops": (8.0 if case["gated"] else 3.0) * M * d}
    if op == "norm_in":
        return {"bytes": float(M * d * t * (3 if case["add"] else 1) + d * t + result(case["out"], d)), "flops": 6.0 * M * d}
    moved = M * d * (t + 2 * size[case["res"]]) + d * t * (1 + case["branch"]) + result(case["out"], d)
    if case["gate"] != "none":
        moved += -(-M // case["gate_rows"]) * d * t
    return {"bytes": float(moved), "flops": 12.0 * M * d}
