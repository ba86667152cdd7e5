"""The 8-bit integer operators of a decoder layer, as cases that a program can time.

A case names one operator and its sizes:

* ``norm``:   the residual's addition and RMSNorm, with an output in 8 bits and one scale per row;
* ``rows``:   rows (the attention's output) in 8 bits with one scale per row;
* ``swiglu``: SiLU(gate) * up with an output in 8 bits and one scale per row;
* ``linear``: the matrix product of such rows with weights in 8 bits that have one scale per output channel.

A row t in 8 bits: scale = max|t| / 127, code = the integer nearest to t / scale, ties to even.  Where ``own`` is false a pass is
made of elementary torch operations in 32 bits.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _norm(rows, d, dtype, delta):
    return dict(op="norm", rows=rows, d=d, dtype=dtype, delta=delta)


def _rows(rows, d, dtype):
    return dict(op="rows", rows=rows, d=d, dtype=dtype)


def _swiglu(rows, ffn, dtype):
    return dict(op="swiglu", rows=rows, ffn=ffn, dtype=dtype)


def _linear(rows, n, k, out):
    return dict(op="linear", rows=rows, n=n, k=k, out=out)


def listed():
    named = lambda name, case: dict(case, name=name)  # noqa: E731
    return [
        # one row of the 7B-class width: autoregressive decoding of one sequence, where latency is all
        named("norm_1x4096", _norm(1, 4096, "bf16", "fp32")),
        # the residual stream of one 64-node tree, between two products
        named("norm_64x4096", _norm(64, 4096, "bf16", "fp32")),
        # sixteen such trees of the wider shape, whose products leave 16-bit rows
        named("norm_1024x5120", _norm(1024, 5120, "fp16", "fp16")),
        # the attention's output of six 15-node trees: 90 rows, a size that is a multiple of nothing
        named("rows_90x4096", _rows(90, 4096, "fp16")),
        # a long batch of rows of an odd width, whose rows start at odd addresses
        named("rows_4000x1387", _rows(4000, 1387, "bf16")),
        # one tree's feed-forward activations
        named("swiglu_64x11008", _swiglu(64, 11008, "bf16")),
        # a batch's, at the width of the grouped-head model
        named("swiglu_1024x12800", _swiglu(1024, 12800, "fp16")),
        # decoding one sequence: the QKV product, a stream of weights
        named("linear_1x12288x4096", _linear(1, 12288, 4096, "fp32")),
        # one tree's gate and up products, the largest matrix of a layer
        named("linear_64x22016x4096", _linear(64, 22016, 4096, "bf16")),
        # one tree's down product: few columns, a long sum
        named("linear_64x4096x11008", _linear(64, 4096, 11008, "fp32")),
        # a few ragged sequences on the grouped-head model's QKV product
        named("linear_200x6144x4096", _linear(200, 6144, 4096, "fp32")),
        # sixteen trees' gate and up products: bound by the matrix cores
        named("linear_1024x22016x4096", _linear(1024, 22016, 4096, "bf16")),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width as models have it (a multiple of 32), or any."""
    v = _log_int(rng, lo, hi)
    return v if rng.random() < 0.3 else max(32, v // 32 * 32)


def draw(rng):
    op = rng.choice(["norm", "norm", "rows", "swiglu", "linear", "linear", "linear"])
    dtype = rng.choice(["bf16", "fp16"])
    if op == "norm":
        return _norm(_log_int(rng, 1, 4096), _width(rng, 200, 8192), dtype, rng.choice(["none", "fp32", dtype]))
    if op == "rows":
        return _rows(_log_int(rng, 1, 4096), _width(rng, 200, 8192), dtype)
    if op == "swiglu":
        return _swiglu(_log_int(rng, 1, 2048), _width(rng, 500, 14000), dtype)
    n, k = _width(rng, 200, 28000), _width(rng, 200, 14000)
    return _linear(min(_log_int(rng, 1, 2048), 1024 * 22016 * 4096 // (n * k)), n, k, rng.choice(["fp32", "bf16", "fp16"]))


def _inputs(case, seed):
    """The data of a case, from the seed alone."""
    gen = torch.Generator(DEV).manual_seed(seed)

    def normal(*shape, dtype=torch.float32, std=1.0):
        return torch.empty(*shape, device=DEV, dtype=dtype).normal_(0.0, std, generator=gen)

    def uniform(*shape):
        return torch.empty(*shape, device=DEV).uniform_(generator=gen)

    op, rows = case["op"], case["rows"]
    if op == "norm":  # a residual stream whose rows differ in size, an update that is smaller, gains around 1
        d, delta = case["d"], case["delta"]
        return dict(x=normal(rows, d) * (0.5 + 4 * uniform(rows, 1)), gain=(1 + normal(d, std=0.3)).to(TYPES[case["dtype"]]),
                    delta=None if delta == "none" else normal(rows, d, dtype=TYPES[delta], std=0.2))
    if op == "rows":  # averages of value rows
        return dict(src=normal(rows, case["d"], dtype=TYPES[case["dtype"]], std=0.3))
    if op == "swiglu":
        return dict(gate_up=normal(rows, 2 * case["ffn"], dtype=TYPES[case["dtype"]], std=1.3))
    # codes as rows of bell-shaped numbers have them: the largest near 127 and four standard deviations out
    n, k = case["n"], case["k"]
    codes = lambda *shape: normal(*shape).mul_(32).round_().clamp_(-127, 127).to(torch.int8)  # noqa: E731
    return dict(codes=codes(rows, k), scales=(0.5 + uniform(rows)) / 32, w_codes=codes(n, k), w_scales=(0.5 + uniform(n)) * 6e-4)


EPS = 1e-5


def prepare(case, seed):
    st = dict(case=case, **_inputs(case, seed))
    if own:
        import paper_2603_03383_amd as P

        rows, i8 = case["rows"], dict(device=DEV, dtype=torch.int8)
        if case["op"] == "linear":  # the packed weights and the workspace that a user's program keeps
            n, k = case["n"], case["k"]
            st["packed"] = torch.empty(P.medusa_packed_i8_bytes(n, k), device=DEV, dtype=torch.uint8)
            P.medusa_pack_codes_i8(st["w_codes"], st["w_scales"], st["packed"], n)
            st["ws"] = torch.empty(P.medusa_linear_i8_workspace_bytes(rows, n, k), device=DEV, dtype=torch.uint8)
            st["y"] = torch.empty(rows, n, device=DEV, dtype=TYPES[case["out"]])
        else:
            d = case["ffn"] if case["op"] == "swiglu" else case["d"]
            st["out_codes"], st["out_scales"] = torch.empty(rows, d, **i8), torch.empty(rows, device=DEV)
            st["values"] = torch.empty(rows, d, device=DEV, dtype=TYPES[case["dtype"]])
            if case["op"] == "norm":
                st["x_out"] = None if st["delta"] is None else torch.empty_like(st["x"])
        st["P"] = P
    return st


def _in_8_bits(t):
    """Codes (as numbers) and scales of the rows of t."""
    scale = t.abs().amax(1, keepdim=True) / 127
    scale = torch.where(scale > 0, scale, torch.ones_like(scale))
    return (t / scale).round().clamp(-127, 127), scale


def run(st):
    case = st["case"]
    op = case["op"]
    if own:
        P = st["P"]
        if op == "linear":
            P.medusa_linear_i8(st["codes"], st["scales"], st["packed"], st["y"], st["ws"])
            return dict(y=st["y"])
        if op == "norm":
            P.medusa_residual_rmsnorm_i8(st["x"], st["delta"], st["gain"], EPS, st["x_out"], st["out_codes"], st["out_scales"], st["values"])
            out = dict(scales=st["out_scales"], values=st["values"])
            return out if st["delta"] is None else dict(out, x=st["x_out"])
        if op == "rows":
            P.medusa_quantize_rows_i8(st["src"], st["out_codes"], st["out_scales"], st["values"])
        else:
            P.medusa_swiglu_i8(st["gate_up"], st["out_codes"], st["out_scales"], st["values"])
        return dict(scales=st["out_scales"], values=st["values"])
    if op == "linear":
        y = (st["codes"].float() @ st["w_codes"].float().t()) * st["scales"][:, None] * st["w_scales"]
        return dict(y=y.to(TYPES[case["out"]]))
    td = TYPES[case["dtype"]]
    if op == "norm":
        x = st["x"] if st["delta"] is None else st["x"] + st["delta"].float()
        codes, scale = _in_8_bits(x * st["gain"].float())
        scale = scale * torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)
        out = dict(scales=scale[:, 0], values=(codes * scale).to(td))
        return out if st["delta"] is None else dict(out, x=x)
    if op == "rows":
        codes, scale = _in_8_bits(st["src"].float())
    else:
        gate, up = st["gate_up"].float().split(case["ffn"], dim=1)
        codes, scale = _in_8_bits(gate / (1 + torch.exp(-gate)) * up)
    return dict(scales=scale[:, 0], values=(codes * scale).to(td))


def work(case):
    op, rows = case["op"], case["rows"]
    size = lambda name: 0 if name == "none" else 4 if name == "fp32" else 2  # noqa: E731
    if op == "linear":
        n, k = case["n"], case["k"]
        return {"bytes": rows * k + n * k + rows * n * size(case["out"]) + 4 * (rows + n), "flops": 2 * rows * n * k}
    d, es = case["ffn"] if op == "swiglu" else case["d"], size(case["dtype"])
    out = rows * d * (1 + es) + 4 * rows  # codes, the values they stand for, scales
    if op == "norm":
        stream = 4 if case["delta"] == "none" else 4 + 4 + size(case["delta"])
        return {"bytes": out + rows * d * stream + d * es, "flops": 8 * rows * d}
    if op == "rows":
        return {"bytes": out + rows * d * es, "flops": 4 * rows * d}
    return {"bytes": out + 2 * rows * d * es, "flops": 9 * rows * d}


def exact(case, seed):
    """From the definitions, in 64 bits."""
    t = {k: v.double() for k, v in _inputs(case, seed).items() if v is not None}
    op = case["op"]
    if op == "linear":
        return dict(y=torch.mm(t["codes"] * t["scales"].unsqueeze(1), (t["w_codes"] * t["w_scales"].unsqueeze(1)).t().contiguous()))
    more = {}
    if op == "norm":
        x = t["x"] + t.get("delta", 0.0)
        v = t["gain"] * x / torch.sqrt((x * x).sum(1, keepdim=True) / case["d"] + EPS)
        more = {} if case["delta"] == "none" else dict(x=x)
    elif op == "rows":
        v = t["src"]
    else:
        g, u = t["gate_up"][:, :case["ffn"]], t["gate_up"][:, case["ffn"]:]
        v = g * torch.sigmoid(g) * u
    step = v.abs().max(dim=1).values / 127
    return dict(more, scales=step, values=torch.round(v / step[:, None]) * step[:, None])
