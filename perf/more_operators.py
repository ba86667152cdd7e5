"""Operators of a sampled decoding step whose weights are in 4 bits, as cases that a program can time.

A case names one operator and its sizes:

* ``linear``: rows times a matrix in 4 bits with a scale per group of input features, with or without zero points;
* ``swiglu``: SiLU(rows x gate) * (rows x up) of two such matrices;
* ``sample``: one token per row of logits, from a given random number, with a temperature, top-k, top-p and min-p.

A matrix in 4 bits: codes q of 0 .. 15; a group of `group` consecutive features of a row has one scale s and one zero point z (8 where there
are no zero points), and its elements stand for (q - z) * s.

Sampling: tokens in the order of their logits, descending, ties to the lowest index; a token's mass is exp((logit - largest) / temperature).
top-k keeps the first k; top-p of those the tokens before which less than p of their mass lies; min-p those whose mass is at least
min_p times the largest's.  Drawn is the first kept token up to and with which more than u of the kept mass lies.

Where ``own`` is false a pass is made of elementary torch operations: in 32 bits, and in 64 for sampling, where a token stands or falls with
the last bits of a long sum.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _linear(rows, n, k, group, zeros, dtype, out):
    return dict(op="linear", rows=rows, n=n, k=k, group=group, zeros=zeros, dtype=dtype, out=out)


def _swiglu(rows, n, k, group, zeros, dtype):
    return dict(op="swiglu", rows=rows, n=n, k=k, group=group, zeros=zeros, dtype=dtype, out=dtype)


def _sample(rows, vocab, dtype, per, temperature, top_k, top_p, min_p):
    return dict(op="sample", rows=rows, vocab=vocab, dtype=dtype, per=per, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)


def listed():
    named = lambda name, case: dict(case, name=name)  # noqa: E731
    return [
        # decoding one sequence: the QKV product, a stream of weights
        named("linear_1x12288x4096", _linear(1, 12288, 4096, 128, False, "bf16", "fp32")),
        # the down product of eight sequences decoded together: a long sum, zero points
        named("linear_8x4096x11008", _linear(8, 4096, 11008, 64, True, "fp16", "fp16")),
        # one 64-node tree's output projection: few columns
        named("linear_64x4096x4096", _linear(64, 4096, 4096, 128, False, "bf16", "fp32")),
        # six 15-node trees on a matrix of odd height, whose output rows start at odd addresses, in small groups
        named("linear_90x1387x4000", _linear(90, 1387, 4000, 32, True, "fp16", "fp32")),
        # one tree's logits: the vocabulary's matrix, the longest stream of all
        named("linear_64x128000x4096", _linear(64, 128000, 4096, 128, False, "bf16", "fp32")),
        # decoding one sequence: the gated half of the feed-forward block
        named("swiglu_1x11008x4096", _swiglu(1, 11008, 4096, 128, False, "bf16")),
        # the same of one tree
        named("swiglu_64x11008x4096", _swiglu(64, 11008, 4096, 128, False, "bf16")),
        # a few ragged sequences, at the feed-forward width of the grouped-head model
        named("swiglu_200x12800x4096", _swiglu(200, 12800, 4096, 64, True, "fp16")),
        # sixteen trees: bound by the matrix cores
        named("swiglu_1024x11008x4096", _swiglu(1024, 11008, 4096, 128, False, "bf16")),
        # the next token of one sequence, where latency is all
        named("sample_1x128000", _sample(1, 128000, "fp32", 1, 0.8, 40, 0.95, 0.0)),
        # every node of one tree, with one sequence's settings
        named("sample_64x128000", _sample(64, 128000, "fp32", 64, 1.0, 0, 0.9, 0.02)),
        # a batch of 15-node trees on 16-bit logits (many ties) of an odd vocabulary
        named("sample_240x32003", _sample(240, 32003, "bf16", 15, 0.7, 200, 0.8, 0.0)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width as models have it (a multiple of 32), or any."""
    v = _log_int(rng, lo, hi)
    return v if rng.random() < 0.3 else max(32, v // 32 * 32)


def draw(rng):
    op = rng.choice(["linear", "linear", "linear", "swiglu", "swiglu", "sample", "sample"])
    if op == "sample":
        vocab = _width(rng, 1000, 160000)
        rows = min(_log_int(rng, 1, 256), max(1, 64 * 128000 // vocab))
        return _sample(rows, vocab, rng.choice(["fp32", "fp32", "bf16", "fp16"]), rng.choice([1, 15, 64]), round(rng.uniform(0.4, 1.4), 2),
                       rng.choice([0, 0, 1, _log_int(rng, 2, 1000)]), rng.choice([1.0, round(rng.uniform(0.3, 0.99), 3)]),
                       rng.choice([0.0, 0.0, round(rng.uniform(0.01, 0.2), 3)]))
    dtype, group, zeros = rng.choice(["bf16", "fp16"]), rng.choice([32, 64, 128]), rng.random() < 0.4
    n, k = _width(rng, 200, 22000 if op == "linear" else 12800), _width(rng, 200, 11008)
    rows = min(_log_int(rng, 1, 1024), 1024 * 11008 * 4096 // (n * k))
    if op == "swiglu":
        return _swiglu(rows, n, k, group, zeros, dtype)
    return _linear(rows, n, k, group, zeros, dtype, rng.choice(["fp32", dtype]))


def _gen(seed):
    return torch.Generator(DEV).manual_seed(seed)


def _matrix(gen, case):
    """Codes as bell-shaped weights have them, one scale per group, zero points around the middle."""
    n, k, groups = case["n"], case["k"], -(-case["k"] // case["group"])
    codes = torch.empty(n, k, device=DEV, dtype=torch.float16).normal_(7.8, 2.7, generator=gen).round_().clamp_(0, 15).to(torch.uint8)
    scales = torch.empty(n, groups, device=DEV).uniform_(0.5, 1.5, generator=gen).mul_(0.35 / math.sqrt(k)).to(TYPES[case["dtype"]])
    zeros = torch.randint(5, 12, (n, groups), device=DEV, dtype=torch.uint8, generator=gen) if case["zeros"] else None
    return codes, scales, zeros


def _logits(gen, case):
    """A bell of unlikely tokens and a few likely ones, in rows that are more and less sure."""
    rows, vocab = case["rows"], case["vocab"]
    bulk = torch.empty(rows, vocab, device=DEV).normal_(0.0, 2.0, generator=gen)
    likely = torch.empty(rows, vocab, device=DEV).uniform_(generator=gen) < 30.0 / vocab
    lift = torch.empty(rows, vocab, device=DEV).uniform_(2.0, 14.0, generator=gen)
    sure = torch.empty(rows, 1, device=DEV).uniform_(0.5, 1.2, generator=gen)
    return ((bulk + likely * lift) * sure).to(TYPES[case["dtype"]])


def _inputs(case, seed):
    """The data of a case, from the seed alone."""
    gen = _gen(seed)
    if case["op"] == "sample":
        rows = case["rows"]
        sequences = -(-rows // case["per"])
        many = lambda v, dtype: torch.full((sequences,), v, device=DEV, dtype=dtype)  # noqa: E731
        return dict(logits=_logits(gen, case), u=torch.empty(rows, device=DEV).uniform_(generator=gen),
                    temperature=many(case["temperature"], torch.float32), top_k=many(case["top_k"], torch.int32),
                    top_p=many(case["top_p"], torch.float32), min_p=many(case["min_p"], torch.float32))
    # rows as a norm leaves them, a few features larger than the others
    size = 1 + 6 * (torch.empty(case["k"], device=DEV).uniform_(generator=gen) < 0.01)
    x = (torch.empty(case["rows"], case["k"], device=DEV).normal_(generator=gen) * size).to(TYPES[case["dtype"]])
    return dict(x=x, matrices=[_matrix(gen, case) for _ in range(2 if case["op"] == "swiglu" else 1)])


def prepare(case, seed):
    st = dict(case=case, **_inputs(case, seed))
    if not own:
        return st
    import paper_2603_03383_amd as P

    st["P"] = P
    rows = case["rows"]
    if case["op"] == "sample":
        st["ws"] = torch.empty(P.medusa_sample_workspace_bytes(rows, case["vocab"]), device=DEV, dtype=torch.uint8)
        st["token"], st["prob"] = torch.empty(rows, device=DEV, dtype=torch.int32), torch.empty(rows, device=DEV)
        return st
    # the packed weights and the workspace that a user's program keeps
    n, k, group, zeros = case["n"], case["k"], case["group"], case["zeros"]
    st["packed"] = []
    for codes, scales, zero_points in st["matrices"]:
        packed = torch.empty(P.medusa_packed_i4_bytes(n, k, group, zeros), device=DEV, dtype=torch.uint8)
        P.medusa_pack_codes_i4(codes, scales, zero_points, group, packed, n)
        st["packed"].append(packed)
    need = P.medusa_swiglu_i4_workspace_bytes if case["op"] == "swiglu" else P.medusa_linear_i4_workspace_bytes
    st["ws"] = torch.empty(need(rows, n, k), device=DEV, dtype=torch.uint8)
    st["y"] = torch.empty(rows, n, device=DEV, dtype=TYPES[case["out"]])
    return st


def _weights(matrix, case):
    codes, scales, zeros = matrix
    spread = lambda t: t.float().repeat_interleave(case["group"], dim=1)[:, :case["k"]]  # noqa: E731
    q = codes.float() - (8.0 if zeros is None else spread(zeros))
    return q.mul_(spread(scales))


def _drawn(st):
    """Token and probability of each row, in 64 bits."""
    case = st["case"]
    row = lambda t: t.double().repeat_interleave(case["per"])[:case["rows"], None]  # noqa: E731
    l, order = torch.sort(st["logits"], dim=1, descending=True, stable=True)
    w = torch.exp((l.double() - l[:, :1].double()) / row(st["temperature"]))
    top_k, place = row(st["top_k"]), torch.arange(case["vocab"], device=DEV)
    w = torch.where((top_k <= 0) | (place < top_k), w, torch.zeros_like(w))
    up_to = torch.cumsum(w, dim=1)
    top_p = row(st["top_p"])
    kept = ((top_p >= 1) | (up_to - w < top_p * up_to[:, -1:])) & (w >= row(st["min_p"]))
    kept[:, 0] = True
    w = torch.where(kept, w, torch.zeros_like(w))
    up_to = torch.cumsum(w, dim=1)
    at = (up_to <= st["u"].double()[:, None] * up_to[:, -1:]).sum(dim=1, keepdim=True)
    at = torch.minimum(at, (w > 0).sum(dim=1, keepdim=True) - 1)
    return order.gather(1, at)[:, 0].to(torch.int32), (w.gather(1, at) / up_to[:, -1:])[:, 0].float()


def run(st):
    case = st["case"]
    op = case["op"]
    if own:
        P = st["P"]
        if op == "sample":
            P.medusa_sample(st["logits"], st["u"], st["token"], st["prob"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"],
                            min_p=st["min_p"], rows_per_setting=case["per"], ws=st["ws"])
            return dict(token=st["token"], prob=st["prob"])
        if op == "swiglu":
            P.medusa_swiglu_i4(st["x"], st["packed"][0], st["packed"][1], case["group"], case["zeros"], st["y"], st["ws"])
        else:
            P.medusa_linear_i4(st["x"], st["packed"][0], case["group"], case["zeros"], st["y"], st["ws"])
        return dict(y=st["y"])
    if op == "sample":
        token, prob = _drawn(st)
        return dict(token=token, prob=prob)
    x = st["x"].float()
    y = x @ _weights(st["matrices"][0], case).t()
    if op == "swiglu":
        y = y / (1 + torch.exp(-y)) * (x @ _weights(st["matrices"][1], case).t())
    return dict(y=y.to(TYPES[case["out"]]))


def work(case):
    rows = case["rows"]
    size = lambda name: 4 if name == "fp32" else 2  # noqa: E731
    if case["op"] == "sample":
        # each logit once: a difference, a factor, an exponential, a sum
        return {"bytes": rows * case["vocab"] * size(case["dtype"]) + 12 * rows + 16 * -(-rows // case["per"]), "flops": 4 * rows * case["vocab"]}
    n, k, matrices = case["n"], case["k"], 2 if case["op"] == "swiglu" else 1
    groups = n * -(-k // case["group"])
    matrix = (n * k + 1) // 2 + 2 * groups + ((groups + 1) // 2 if case["zeros"] else 0)  # codes, scales, zero points
    return {"bytes": rows * k * 2 + matrices * matrix + rows * n * size(case["out"]), "flops": 2 * rows * n * k * matrices}


def exact(case, seed):
    """From the definitions, in 64 bits."""
    t = _inputs(case, seed)
    if case["op"] == "sample":
        token, prob = [], []
        for r in range(case["rows"]):
            s = r // case["per"]
            l = t["logits"][r].double()
            mass = ((l - l.max()) / t["temperature"][s].double()).exp()
            order = torch.sort(l, descending=True, stable=True).indices
            if case["top_k"] > 0:
                order = order[:case["top_k"]]
            if case["top_p"] < 1:
                before = torch.cat([mass.new_zeros(1), mass[order].cumsum(0)[:-1]])
                order = order[before < t["top_p"][s].double() * mass[order].sum()]
            order = order[mass[order] >= min(t["min_p"][s].double().item(), 1.0)]
            share = mass[order] / mass[order].sum()
            at = min(int(torch.searchsorted(share.cumsum(0), t["u"][r].double(), right=True)), len(order) - 1)
            token.append(order[at])
            prob.append(share[at])
        return dict(token=torch.stack(token).to(torch.int32), prob=torch.stack(prob))
    x = t["x"].double()

    def product(matrix):
        codes, scales, zeros = matrix
        y = torch.zeros(case["rows"], case["n"], device=DEV, dtype=torch.float64)
        for g in range(scales.shape[1]):  # a group's sum, then its scale
            at = slice(g * case["group"], (g + 1) * case["group"])
            q = codes[:, at].double() - (8 if zeros is None else zeros[:, g:g + 1].double())
            y += torch.mm(x[:, at], q.t().contiguous()) * scales[:, g].double()
        return y

    y = product(t["matrices"][0])
    return dict(y=y * torch.sigmoid(y) * product(t["matrices"][1]) if case["op"] == "swiglu" else y)
