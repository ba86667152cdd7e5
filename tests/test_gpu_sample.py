"""Sampling on the GPU against its definition (oracle/sampling.py), at the sizes, values and settings where it can go wrong."""
import numpy as np
import pytest
import torch

import paper_2603_03383_amd as P
from oracle import sampling

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TD = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
GUARD = 3
# A token's mass is rounded to 2^-45 of the largest at up to 131072 tokens (2^-44 at 262144), its exponential to 7e-15 of itself and 2^-52 a few times:
# running sums are off by at most 2^18 * 2^-45 + 1e-14 = 8e-9 of the largest, which is kept, and two of them decide.
BORDER = 2e-8


def _rows(seed, rows, vocab, dtype="fp32", kind="bell"):
    g = torch.Generator(DEV).manual_seed(seed)
    l = torch.empty(rows, vocab, device=DEV).normal_(0.0, 2.5, generator=g)
    if kind == "flat":
        l = torch.full((rows, vocab), 1.25, device=DEV)
    elif kind == "near":   # thousands of different logits in one bin
        l = l * 1e-4
    elif kind == "steps":  # thousands of tokens at each of a few logits
        l = (l / 2).round()
    elif kind == "sure":
        l[:, vocab // 2] += 40
    return l.to(TD[dtype])


def call(logits, u, fill=0xA5, rows_per_setting=1, **settings):
    rows, vocab = logits.shape
    n = -(-rows // rows_per_setting)
    dev = {k: None if v is None else torch.as_tensor(v, dtype=torch.int32 if k == "top_k" else torch.float32).expand(n).contiguous().to(DEV) for k, v in settings.items()}
    token = torch.full((rows + GUARD,), 77, dtype=torch.int32, device=DEV)
    prob = torch.full((rows + GUARD,), 7.5, device=DEV)
    need = P.medusa_sample_workspace_bytes(rows, vocab)
    ws = torch.full((need + 64,), fill, dtype=torch.uint8, device=DEV)
    P.medusa_sample(logits, u, token[:rows], prob[:rows], rows_per_setting=rows_per_setting, ws=ws[:need], **dev)
    assert bool((token[rows:] == 77).all()) and bool((prob[rows:] == 7.5).all()) and bool((ws[need:] == fill).all())
    return token[:rows].cpu().numpy(), prob[:rows].double().cpu().numpy()


def check(logits, u, token, prob, per=1, **settings):
    l, us = logits.double().cpu().numpy(), u.double().cpu().numpy()
    close = 0
    for r in range(l.shape[0]):
        mine = {k: float(np.float32(v[r // per] if np.ndim(v) else v)) if k != "top_k" else int(v[r // per] if np.ndim(v) else v) for k, v in settings.items() if v is not None}
        want, p, border = sampling.draw(l[r], us[r], **mine)
        if border < BORDER:
            close += 1
            continue
        assert token[r] == want, (r, token[r], want, border, mine)
        # rounded once to fp32 from a quotient of sums that are off as above
        assert abs(prob[r] - p) <= p * 2.0 ** -24 + BORDER + 2.0 ** -149, (r, prob[r], p)
    assert close <= max(1, l.shape[0] // 20)


SETTINGS = [
    dict(),
    dict(temperature=0.7),
    dict(top_k=1),
    dict(temperature=0.8, top_k=40),
    dict(top_p=0.9),
    dict(temperature=1.3, top_p=0.35),
    dict(min_p=0.05),
    dict(temperature=0.6, top_k=50, top_p=0.95, min_p=0.02),
    dict(top_k=3000, top_p=0.5),
    dict(temperature=2.5, min_p=0.5, top_p=0.999),
]
SIZES = [(1, 1), (3, 2), (5, 65), (4, 1024), (3, 8192), (2, 8193), (5, 32003), (1, 128000), (9, 128001), (300, 500)]


@pytest.mark.parametrize("rows,vocab", SIZES)
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_sizes_and_settings(dtype, rows, vocab):
    logits = _rows(rows * vocab, rows, vocab, dtype)
    for i, s in enumerate(SETTINGS):
        u = torch.rand(rows, generator=torch.Generator().manual_seed(i)).to(DEV)
        check(logits, u, *call(logits, u, **s), **s)


@pytest.mark.parametrize("kind", ["flat", "near", "steps", "sure"])
@pytest.mark.parametrize("rows,vocab", [(4, 5000), (4, 40000), (300, 9000)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_ties_and_flat_rows(dtype, rows, vocab, kind):
    logits = _rows(11, rows, vocab, dtype, kind)
    u = torch.rand(rows, generator=torch.Generator().manual_seed(5)).to(DEV)
    for s in SETTINGS + [dict(top_k=2500), dict(top_k=4999, top_p=0.77), dict(min_p=1.0)]:
        check(logits, u, *call(logits, u, **s), **s)


@pytest.mark.parametrize("vocab", [3000, 20000])
def test_flat_rows_are_counted(vocab):
    """Equal logits: the token is the u-th share of the kept ones, by index."""
    n = 64
    logits = torch.zeros(n, vocab, device=DEV)
    logits[:, 7] = -0.0  # ties with zero
    u = (torch.arange(n, device=DEV).float() + 0.5) / n
    for k in (1, 5, 2048, 2049, 2999):
        token, prob = call(logits, u, top_k=k)
        assert np.array_equal(token, np.floor(u.double().cpu().numpy() * k).astype(np.int32))
        assert np.array_equal(prob, np.full(n, float(np.float32(1 / k))))


def test_every_share_of_a_small_row():
    logits = torch.tensor([0.5, -1.0, 2.0, 2.0, -3.0, 0.0, 1.0, 2.0], device=DEV)
    n = 4096
    rows, u = logits.expand(n, -1).contiguous(), torch.arange(n, device=DEV).float() / n
    token, prob = call(rows, u)
    order, mass = sampling.kept_tokens(logits.cpu().numpy())
    share = mass / mass.sum()
    for t, s in zip(order, share):
        assert abs((token == t).sum() - s * n) <= 1  # the numbers between two borders, each end off by less than one
        assert np.allclose(prob[token == t], s, rtol=2.0 ** -23, atol=0)
    assert order[:3].tolist() == [2, 3, 7] and token[0] == 2 and token[-1] == 4


@pytest.mark.parametrize("vocab", [50, 30000])
def test_logits_that_cannot_be_drawn(vocab):
    inf, nan = float("inf"), float("nan")
    base = _rows(3, 12, vocab)
    base[0, ::2] = -inf
    base[1, 1::3] = nan
    base[2] = -inf
    base[3] = nan
    base[4, 17] = inf
    base[5, [4, 40]] = inf
    base[6] = -inf
    base[6, 31] = -5.0
    base[7, 0] = 3e38
    base[8] = -3e38
    base[9, 5] = nan
    base[9, 6] = inf
    base[10, 0::2], base[10, 1::2] = nan, -inf
    u = torch.rand(12, generator=torch.Generator().manual_seed(8)).to(DEV)
    for s in SETTINGS:
        token, prob = call(base, u, **s)
        check(base, u, token, prob, **s)
        assert token[2] == token[3] == token[10] == -1 and prob[2] == prob[3] == prob[10] == 0
        assert token[4] == 17 and token[5] in (4, 40) and token[6] == 31 and token[9] == 6
    assert call(base, torch.full((12,), 0.6, device=DEV))[0][5] == 40 and call(base, torch.full((12,), 0.4, device=DEV))[0][5] == 4


@pytest.mark.parametrize("vocab", [77, 12345])
def test_settings_at_their_ends(vocab):
    logits = _rows(4, 6, vocab)
    u = torch.tensor([0.0, 0.3, 0.5, 0.999, 1 - 2.0 ** -24, 0.7], device=DEV)
    first = logits.argmax(1).cpu().numpy()
    for t in (0.0, -1.0, float("nan"), 1e-30, 1e-42):
        token, prob = call(logits, u, temperature=t)
        assert np.array_equal(token, first) and (prob == 1).all()
    for s in (dict(temperature=float("inf")), dict(temperature=1e30), dict(top_k=-3), dict(top_k=vocab), dict(top_k=2 ** 31 - 1), dict(top_p=1.0), dict(top_p=7.0),
              dict(min_p=-0.5), dict(temperature=float("inf"), top_p=0.5, min_p=0.3)):
        check(logits, u, *call(logits, u, **s), **s)
    for s in (dict(top_p=0.0), dict(top_p=-1.0), dict(min_p=1.0), dict(min_p=5.0), dict(top_k=1)):
        token, prob = call(logits, u, **s)
        assert np.array_equal(token, first) and (prob == 1).all()
    # u outside [0, 1): its nearer end
    last = call(logits, torch.full((6,), 1.0, device=DEV), top_k=9)[0]
    for v in (1.0, 2.0, float("inf")):
        assert np.array_equal(call(logits, torch.full((6,), v, device=DEV), top_k=9)[0], last)
    assert np.array_equal(last, np.argsort(-logits.cpu().numpy(), axis=1, kind="stable")[:, 8])
    for v in (-1.0, float("nan"), float("-inf")):
        assert np.array_equal(call(logits, torch.full((6,), v, device=DEV))[0], first)


def test_settings_of_sequences():
    """Seven nodes of each of five trees, every tree with settings of its own."""
    rows, per, vocab = 35, 7, 9000
    logits = _rows(6, rows, vocab)
    u = torch.rand(rows, generator=torch.Generator().manual_seed(2)).to(DEV)
    s = dict(temperature=[0.0, 0.5, 1.0, 1.5, 0.9], top_k=[0, 10, 0, 300, 1], top_p=[1.0, 0.9, 0.5, 1.0, 0.1], min_p=[0.0, 0.0, 0.1, 0.01, 0.0])
    check(logits, u, *call(logits, u, rows_per_setting=per, **s), per=per, **s)
    # the last tree's nodes may be fewer
    check(logits[:31], u[:31].contiguous(), *call(logits[:31], u[:31].contiguous(), rows_per_setting=per, **s), per=per, **s)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [501, 10001])
def test_rows_that_lie_apart_or_start_on_any_element(dtype, vocab):
    room = _rows(9, 6, vocab + 37, dtype)
    u = torch.rand(6, generator=torch.Generator().manual_seed(1)).to(DEV)
    for at in (0, 1, 3):
        part = room[:, at:at + vocab]
        assert not part.is_contiguous()
        want = call(part.contiguous(), u, temperature=0.9, top_p=0.9)
        got = call(part, u, temperature=0.9, top_p=0.9)
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


def test_a_row_does_not_depend_on_its_neighbours():
    """Alone, among few and among many rows (other kernels): the same token and the same probability, bit for bit."""
    vocab = 9001
    logits = _rows(13, 300, vocab)
    u = torch.rand(300, generator=torch.Generator().manual_seed(3)).to(DEV)
    s = dict(temperature=0.8, top_k=400, top_p=0.9)
    many = call(logits, u, **s)
    few = call(logits[:20], u[:20].contiguous(), **s)
    assert np.array_equal(few[0], many[0][:20]) and np.array_equal(few[1], many[1][:20])
    for r in range(5):
        one = call(logits[r:r + 1], u[r:r + 1].contiguous(), **s)
        assert one[0][0] == many[0][r] and one[1][0] == many[1][r]
    for fill in (0, 0xFF):  # nothing in the workspace has to be set
        again = call(logits[:20], u[:20].contiguous(), fill=fill, **s)
        assert np.array_equal(again[0], few[0]) and np.array_equal(again[1], few[1])


def test_no_rows():
    e = torch.empty(0, device=DEV)
    P.medusa_sample(torch.empty(0, 100, device=DEV), e, torch.empty(0, dtype=torch.int32, device=DEV), e)


def test_on_another_stream_and_in_a_graph():
    rows, vocab = 30, 20000
    logits = _rows(21, rows, vocab)
    u, token, prob = torch.rand(rows, device=DEV), torch.zeros(rows, dtype=torch.int32, device=DEV), torch.zeros(rows, device=DEV)
    top_p = torch.full((rows,), 0.9, device=DEV)
    ws = torch.empty(P.medusa_sample_workspace_bytes(rows, vocab), dtype=torch.uint8, device=DEV)

    def draw():
        P.medusa_sample(logits, u, token, prob, top_p=top_p, ws=ws)
    draw()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        draw()
    for i in range(3):
        u.copy_(torch.rand(rows, generator=torch.Generator().manual_seed(i)))
        draw()
        want, wp = token.clone(), prob.clone()
        token.fill_(-9), prob.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(token, want) and torch.equal(prob, wp)
    token.fill_(-9)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        draw()
    side.synchronize()
    assert torch.equal(token, want)
