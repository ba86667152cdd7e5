"""Refusals of the products with 4-bit weights and of sampling, each by the check that it names (no GPU work: pointers are never followed)."""
import os

import pytest
import torch

import paper_2603_03383_amd as P
from paper_2603_03383_amd import binding

EINVAL, ESHAPE, EUNSUPPORTED, EWORKSPACE = -1, -2, -3, -4


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(P.LIB_PATH):
        import __graft_entry__ as g
        g.build()


def _bf(*s):
    return torch.zeros(*s, dtype=torch.bfloat16)


def _f(*s):
    return torch.zeros(*s)


def _u8(*s):
    return torch.zeros(*s, dtype=torch.uint8)


def _i32(*s):
    return torch.zeros(*s, dtype=torch.int32)


def _packed(n=32, k=64, group=32, zeros=False):
    return _u8(P.medusa_packed_i4_bytes(n, k, group, zeros))


# ---- the C entries: (status, what the message names, call) --------------------------------------
A = 4096  # an address that is aligned to everything here
BIG = 1 << 60


def _linear(dtype=P.MDZ_BF16, x=A, packed=A, M=4, N=32, K=64, group=32, zeros=0, out=P.MDZ_BF16, y=A, ws=A, ws_bytes=BIG):
    return P.lib().medusa_linear_i4(dtype, x, packed, M, N, K, group, zeros, out, y, ws, ws_bytes, None)


def _swiglu(dtype=P.MDZ_BF16, x=A, gate=A, up=A, M=4, N=32, K=64, group=32, zeros=0, y=A, ws=A, ws_bytes=BIG):
    return P.lib().medusa_swiglu_i4(dtype, x, gate, up, M, N, K, group, zeros, y, ws, ws_bytes, None)


def _pack(dtype=P.MDZ_BF16, src=A, n=32, k=64, group=32, zeros=0, dst=A, rows=32, tile=0):
    return P.lib().medusa_pack_weight_i4(dtype, src, n, k, group, zeros, dst, rows, tile, None)


def _codes(dtype=P.MDZ_BF16, codes=A, scales=A, zeros=None, n=32, k=64, group=32, dst=A, rows=32, tile=0):
    return P.lib().medusa_pack_codes_i4(dtype, codes, scales, zeros, n, k, group, dst, rows, tile, None)


def _sample(dtype=P.MDZ_FP32, logits=A, ld=20000, rows=4, vocab=20000, t=None, k=None, p=None, m=None, per=1, u=A, token=A, prob=A, ws=A, ws_bytes=BIG):
    return P.lib().medusa_sample(dtype, logits, ld, rows, vocab, t, k, p, m, per, u, token, prob, ws, ws_bytes, None)


ENTRIES = {
    "linear: rows of fp32": (EUNSUPPORTED, "bf16 or fp16", lambda: _linear(dtype=P.MDZ_FP32)),
    "linear: no type": (EINVAL, "bf16 or fp16", lambda: _linear(dtype=9)),
    "linear: outputs of no type": (EINVAL, "dtype", lambda: _linear(out=9)),
    "linear: groups of 16": (EINVAL, "groups", lambda: _linear(group=16)),
    "linear: groups of 96": (EINVAL, "groups", lambda: _linear(group=96)),
    "linear: zeros 2": (EINVAL, "zeros", lambda: _linear(zeros=2)),
    "linear: rows below zero": (EINVAL, "[-1,64]", lambda: _linear(M=-1)),
    "linear: no columns": (EINVAL, "[0,64]", lambda: _linear(N=0)),
    "linear: no features": (EINVAL, "[32,0]", lambda: _linear(K=0)),
    "linear: too many features": (EUNSUPPORTED, "input features", lambda: _linear(K=(1 << 24) + 1)),
    "linear: too many outputs": (EUNSUPPORTED, "outputs", lambda: _linear(M=1 << 20, N=1 << 20)),
    "linear: x NULL": (EINVAL, "NULL", lambda: _linear(x=None)),
    "linear: packed NULL": (EINVAL, "NULL", lambda: _linear(packed=None)),
    "linear: y NULL": (EINVAL, "NULL", lambda: _linear(y=None)),
    "linear: packed off 16 bytes": (EINVAL, "16 bytes", lambda: _linear(packed=A + 8)),
    "linear: x off its elements": (EINVAL, "aligned", lambda: _linear(x=A + 1)),
    "linear: y off its elements": (EINVAL, "aligned", lambda: _linear(y=A + 2, out=P.MDZ_FP32)),
    "linear: no workspace": (EWORKSPACE, "workspace", lambda: _linear(M=17, ws=None)),
    "linear: a byte too few": (EWORKSPACE, "workspace", lambda: _linear(M=17, ws_bytes=17 * 256 - 1)),
    "linear: ws off 16 bytes": (EINVAL, "workspace", lambda: _linear(M=17, ws=A + 8)),
    "linear: more than a launch": (EUNSUPPORTED, "more than one launch", lambda: _linear(M=2, N=1 << 30)),
    "linear: more than a launch, many rows": (EUNSUPPORTED, "more than one launch", lambda: _linear(x=A, M=1000, N=1 << 30, K=64)),
    "swiglu: gate NULL": (EINVAL, "NULL", lambda: _swiglu(gate=None)),
    "swiglu: up NULL": (EINVAL, "NULL", lambda: _swiglu(up=None)),
    "swiglu: up off 16 bytes": (EINVAL, "16 bytes", lambda: _swiglu(up=A + 4)),
    "swiglu: rows of fp32": (EUNSUPPORTED, "bf16 or fp16", lambda: _swiglu(dtype=P.MDZ_FP32)),
    "swiglu: a byte too few": (EWORKSPACE, "workspace", lambda: _swiglu(M=17, ws_bytes=17 * 256 - 1)),
    "pack: fp32": (EUNSUPPORTED, "bf16 or fp16", lambda: _pack(dtype=P.MDZ_FP32)),
    "pack: no rows": (EINVAL, "sizes", lambda: _pack(n=0)),
    "pack: dst off 16 bytes": (EINVAL, "16 bytes", lambda: _pack(dst=A + 4)),
    "pack: src off its elements": (EINVAL, "aligned", lambda: _pack(src=A + 1)),
    "pack: src NULL": (EINVAL, "NULL", lambda: _pack(src=None)),
    "pack: behind the last row": (ESHAPE, "exceed", lambda: _pack(tile=1)),
    "pack: before the first row": (EINVAL, "sizes", lambda: _pack(tile=-1)),
    "pack: a part of a tile amid others": (ESHAPE, "tile height", lambda: _pack(n=17, rows=64)),
    "pack: groups of 256": (EINVAL, "groups", lambda: _pack(group=256)),
    "pack codes: scales NULL": (EINVAL, "NULL", lambda: _codes(scales=None)),
    "pack codes: behind the last row": (ESHAPE, "exceed", lambda: _codes(tile=1)),
    "sample: no type": (EINVAL, "dtype", lambda: _sample(dtype=9)),
    "sample: rows below zero": (EINVAL, "rows", lambda: _sample(rows=-1)),
    "sample: no vocabulary": (EINVAL, "logits", lambda: _sample(vocab=0)),
    "sample: too large a vocabulary": (EUNSUPPORTED, "2^24", lambda: _sample(vocab=(1 << 24) + 1, ld=1 << 25)),
    "sample: too many rows": (EUNSUPPORTED, "2^21", lambda: _sample(rows=(1 << 21) + 1)),
    "sample: no rows per setting": (EINVAL, "per setting", lambda: _sample(per=0)),
    "sample: rows that overlap": (ESHAPE, "apart", lambda: _sample(ld=19999)),
    "sample: logits NULL": (EINVAL, "NULL", lambda: _sample(logits=None)),
    "sample: u NULL": (EINVAL, "NULL", lambda: _sample(u=None)),
    "sample: token NULL": (EINVAL, "NULL", lambda: _sample(token=None)),
    "sample: logits off their elements": (EINVAL, "aligned", lambda: _sample(logits=A + 2)),
    "sample: a setting off its elements": (EINVAL, "aligned", lambda: _sample(p=A + 2)),
    "sample: no workspace": (EWORKSPACE, "workspace", lambda: _sample(ws=None)),
    "sample: a byte too few": (EWORKSPACE, "workspace", lambda: _sample(ws_bytes=P.medusa_sample_workspace_bytes(4, 20000) - 1)),
    "sample: ws off 16 bytes": (EINVAL, "workspace", lambda: _sample(ws=A + 8)),
}


@pytest.mark.parametrize("what", ENTRIES)
def test_an_entry_refuses(what):
    status, names, call = ENTRIES[what]
    assert call() == status
    assert names in P.lib().medusa_last_error().decode()


def test_no_rows_is_no_work():
    """Nothing is enqueued (there is no GPU to enqueue it on) and no buffer is looked at."""
    assert _linear(M=0, x=None, y=None, ws=None, ws_bytes=0) == 0
    assert _swiglu(M=0, x=None, y=None, ws=None, ws_bytes=0) == 0
    assert _sample(rows=0, logits=None, u=None, token=None, ws=None, ws_bytes=0) == 0


def test_sizes_of_packed_matrices():
    for n, k, group, zeros in [(1, 1, 32, 0), (16, 128, 128, 1), (17, 129, 64, 1), (4096, 11008, 32, 0)]:
        blocks = -(-n // 16) * -(-k // 128)
        per = 128 // group
        assert P.medusa_packed_i4_bytes(n, k, group, zeros) == blocks * (1024 + 32 * per + zeros * 16 * per)
    for n, k, group, zeros, status in [(0, 1, 32, 0, EINVAL), (1, 0, 32, 0, EINVAL), (1, 1, 48, 0, EINVAL), (1, 1, 32, 3, EINVAL), (1, (1 << 24) + 1, 32, 0, EUNSUPPORTED),
                                       (1 << 31, 1, 32, 0, EUNSUPPORTED)]:
        assert P.lib().medusa_packed_i4_bytes(n, k, group, zeros) == status


# ---- the binding ---------------------------------------------------------------------------------
def _call_linear(x, packed, y, group=32, zeros=False, ws=None):
    return P.medusa_linear_i4(x, packed, group, zeros, y, ws, stream=0)


def _call_sample(logits, u, token, prob=None, **kw):
    return P.medusa_sample(logits, u, token, prob, stream=0, **kw)


# Calls whose operands are right but for one; they lie in host memory, which is refused last and with another status, so a check that is missing shows.
WRONG = {
    "product: another number of rows": lambda: _call_linear(_bf(2, 64), _packed(), _f(3, 32)),
    "product: more columns": lambda: _call_linear(_bf(2, 64), _packed(), _f(2, 33)),
    "product: more features": lambda: _call_linear(_bf(2, 129), _packed(), _f(2, 32)),
    "product: packed in other groups": lambda: _call_linear(_bf(2, 64), _packed(group=64), _f(2, 32)),
    "product: packed with zero points": lambda: _call_linear(_bf(2, 64), _packed(zeros=True), _f(2, 32)),
    "product: packed without zero points": lambda: _call_linear(_bf(2, 64), _packed(), _f(2, 32), zeros=True),
    "product: x of integers": lambda: _call_linear(_u8(2, 64), _packed(), _f(2, 32)),
    "product: x in one axis": lambda: _call_linear(_bf(64), _packed(), _f(1, 32)),
    "product: x transposed": lambda: _call_linear(_bf(64, 2).t(), _packed(), _f(2, 32)),
    "product: y transposed": lambda: _call_linear(_bf(2, 64), _packed(), _f(32, 2).t()),
    "product: every other byte of ws": lambda: _call_linear(_bf(2, 64), _packed(), _f(2, 32), ws=_u8(64)[::2]),
    "swiglu: y of another type": lambda: P.medusa_swiglu_i4(_bf(2, 64), _packed(), _packed(), 32, False, _f(2, 32), stream=0),
    "swiglu: gate of another height": lambda: P.medusa_swiglu_i4(_bf(2, 64), _packed(64), _packed(), 32, False, _bf(2, 32), stream=0),
    "swiglu: up of another height": lambda: P.medusa_swiglu_i4(_bf(2, 64), _packed(), _packed(64), 32, False, _bf(2, 32), stream=0),
    "swiglu: x transposed": lambda: P.medusa_swiglu_i4(_bf(64, 2).t(), _packed(), _packed(), 32, False, _bf(2, 32), stream=0),
    "pack: transposed": lambda: P.medusa_pack_weight_i4(_bf(64, 32).t(), 32, _packed(), 32, stream=0),
    "pack: integers": lambda: P.medusa_pack_weight_i4(_u8(32, 64), 32, _packed(), 32, stream=0),
    "pack: a matrix of other sizes": lambda: P.medusa_pack_weight_i4(_bf(32, 64), 32, _packed(64), 32, stream=0),
    "pack codes: a scale too few": lambda: P.medusa_pack_codes_i4(_u8(32, 64), _bf(32, 1), None, 32, _packed(), 32, stream=0),
    "pack codes: scales of fp32": lambda: P.medusa_pack_codes_i4(_u8(32, 64), torch.zeros(32, 2, dtype=torch.float64), None, 32, _packed(), 32, stream=0),
    "pack codes: signed codes": lambda: P.medusa_pack_codes_i4(_u8(32, 64).view(torch.int8), _bf(32, 2), None, 32, _packed(), 32, stream=0),
    "pack codes: zero points of bf16": lambda: P.medusa_pack_codes_i4(_u8(32, 64), _bf(32, 2), _bf(32, 2), 32, _packed(zeros=True), 32, stream=0),
    "pack codes: a zero point too few": lambda: P.medusa_pack_codes_i4(_u8(32, 64), _bf(32, 2), _u8(32, 1), 32, _packed(zeros=True), 32, stream=0),
    "pack codes: one axis": lambda: P.medusa_pack_codes_i4(_u8(64), _bf(1, 2), None, 32, _packed(1), 1, stream=0),
    "sample: logits of integers": lambda: _call_sample(_i32(2, 9), _f(2), _i32(2)),
    "sample: one row without its axis": lambda: _call_sample(_f(9), _f(1), _i32(1)),
    "sample: logits transposed": lambda: _call_sample(_f(9, 2).t(), _f(2), _i32(2)),
    "sample: every other logit": lambda: _call_sample(_f(2, 18)[:, ::2], _f(2), _i32(2)),
    "sample: one row for all": lambda: _call_sample(_f(1, 9).expand(2, 9), _f(2), _i32(2)),
    "sample: u too short": lambda: _call_sample(_f(2, 9), _f(1), _i32(2)),
    "sample: u of 64 bits": lambda: _call_sample(_f(2, 9), _f(2).double(), _i32(2)),
    "sample: tokens of 64 bits": lambda: _call_sample(_f(2, 9), _f(2), _i32(2).long()),
    "sample: prob of bf16": lambda: _call_sample(_f(2, 9), _f(2), _i32(2), _bf(2)),
    "sample: a temperature too many": lambda: _call_sample(_f(2, 9), _f(2), _i32(2), temperature=_f(3)),
    "sample: settings for rows that share theirs": lambda: _call_sample(_f(4, 9), _f(4), _i32(4), top_p=_f(4), rows_per_setting=2),
    "sample: top_k of floats": lambda: _call_sample(_f(2, 9), _f(2), _i32(2), top_k=_f(2)),
    "sample: min_p of integers": lambda: _call_sample(_f(2, 9), _f(2), _i32(2), min_p=_i32(2)),
    "sample: every other byte of ws": lambda: _call_sample(_f(2, 9), _f(2), _i32(2), ws=_u8(64)[::2]),
}


@pytest.mark.parametrize("what", WRONG)
def test_a_wrong_operand_is_refused_for_itself(what):
    with pytest.raises(P.MedusaError) as e:
        WRONG[what]()
    assert e.value.status == ESHAPE


def test_operands_in_host_memory_are_refused():
    calls = [lambda: _call_linear(_bf(2, 64), _packed(), _f(2, 32), ws=_u8(64)),
             lambda: P.medusa_swiglu_i4(_bf(2, 64), _packed(), _packed(), 32, False, _bf(2, 32), stream=0),
             lambda: P.medusa_pack_weight_i4(_bf(32, 64), 32, _packed(), 32, stream=0),
             lambda: P.medusa_pack_codes_i4(_u8(32, 64), _bf(32, 2), _u8(32, 2), 32, _packed(zeros=True), 32, stream=0),
             lambda: _call_sample(_f(4, 9), _f(4), _i32(4), _f(4), temperature=_f(2), top_k=_i32(2), top_p=_f(2), min_p=_f(2), rows_per_setting=2, ws=_u8(64))]
    for call in calls:
        with pytest.raises(P.MedusaError) as e:
            call()
        assert e.value.status == EINVAL and "GPU" in str(e.value)


def test_sizes_beyond_32_bits_are_refused():
    """The library takes these sizes as 32-bit integers; 2^32 + 16 handed on as they are would arrive as 16."""
    big = 2 ** 32 + 16
    calls = [lambda s=s, q=q: q(*s) for s in [(big, 16, 16), (1, big, 16), (1, 16, big)] for q in (P.medusa_linear_i4_workspace_bytes, P.medusa_swiglu_i4_workspace_bytes)]
    calls += [lambda: P.medusa_sample_workspace_bytes(big, 16), lambda: P.medusa_sample_workspace_bytes(16, big),
              lambda: _call_linear(_bf(0, big), _u8(16), _f(0, 16)), lambda: _call_linear(_bf(0, 16), _u8(16), _f(0, big)),
              lambda: _call_sample(_f(0, big), _f(0), _i32(0))]
    for k, call in enumerate(calls):
        with pytest.raises(P.MedusaError) as e:
            call()
        assert e.value.status == EUNSUPPORTED, (k, e.value)
    for per in (0, -1, big):
        with pytest.raises(P.MedusaError) as e:
            _call_sample(_f(2, 9), _f(2), _i32(2), rows_per_setting=per)
        assert e.value.status == EINVAL


def test_sampling_belongs_to_steps_with_logits():
    """run_step refuses before the draw: nothing that argmax gave is taken for a drawn token."""
    import types

    from paper_2603_03383_amd import runtime

    calls = []
    fake = types.SimpleNamespace(MedusaError=P.MedusaError, tree_verify_step=lambda *a: calls.append("verify"), accept_longest_prefix=lambda *a: calls.append("accept"))
    keep, runtime.B = runtime.B, fake
    try:
        buf = types.SimpleNamespace(batch=1, max_prefix=0, tree_tokens=None, node_argmax=None, hidden=None, logits=None, ws=None)
        model = types.SimpleNamespace(desc=None, weights=None)
        with pytest.raises(P.MedusaError) as e:
            runtime.run_step(model, types.SimpleNamespace(desc=None), buf, None, None, None, None, with_heads=False, sampling=object())
        assert e.value.status == EINVAL and "accept" not in calls
    finally:
        runtime.B = keep


def test_without_the_check_of_operands_these_calls_would_pass(monkeypatch):
    """What the test of wrong operands relies on: with a check that looks at nothing (and no GPU to ask for), most of them end as right ones do here."""
    monkeypatch.setattr(binding, "_operand", lambda name, t, *rest: 4096)
    monkeypatch.setattr(binding, "_packed_i4", lambda *a: 4096)
    passed = set()
    for what, call in WRONG.items():
        with pytest.raises(P.MedusaError) as e:
            call()
        if e.value.status == EINVAL:
            passed.add(what)
    kept = {"product: x of integers", "product: x in one axis", "pack: integers", "pack codes: scales of fp32", "pack codes: one axis", "sample: logits of integers",
            "sample: one row without its axis", "sample: logits transposed", "sample: every other logit", "sample: one row for all"}  # refused before their operands are looked at one by one
    assert passed == set(WRONG) - kept
