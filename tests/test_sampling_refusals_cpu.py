"""Sampling put into a step: what cannot be drawn is refused before anything of the step is enqueued, and drawn tokens reach the buffer that was given."""
import types

import pytest
import torch

import paper_2603_03383_amd as P
from paper_2603_03383_amd import runtime

EINVAL, ESHAPE = -1, -2
BATCH, T, VOCAB = 2, 3, 7


@pytest.fixture
def calls(monkeypatch):
    """The library's calls by name; sampling writes the tokens 0, 1, 2, .. into what it gets."""
    seen = []

    def record(name):
        return lambda *a, **k: seen.append(name)

    def sample(logits, u, token, prob, **k):
        assert logits.shape == (BATCH * T, VOCAB) and u.shape == token.shape == prob.shape == (BATCH * T,)
        token.copy_(torch.arange(BATCH * T, dtype=torch.int32))
        seen.append("sample")

    names = ("medusa_heads", "tree_verify_step", "accept_longest_prefix", "kv_compact")
    monkeypatch.setattr(runtime, "B", types.SimpleNamespace(MedusaError=P.MedusaError, medusa_sample=sample, medusa_sample_workspace_bytes=lambda *a: 0,
                                                            **{n: record(n) for n in names}))
    return seen


def _model():
    return types.SimpleNamespace(desc=types.SimpleNamespace(vocab=VOCAB), weights=None, tree=None, tree_info=dict(T=T), device="cpu")


def _buffers(logits=True):
    names = ("cand_flat", "tree_tokens", "head_logits", "ws", "hidden", "accept_len", "best_path", "acc_nodes", "acc_tokens", "next_root", "last_node", "kv_src_slots")
    return types.SimpleNamespace(batch=BATCH, max_prefix=0, logits=torch.zeros(BATCH, T, VOCAB) if logits else None,
                                 node_argmax=torch.full((BATCH, T), -7, dtype=torch.int32), **dict.fromkeys(names))


def _step(buf, sampling):
    hidden = torch.zeros(BATCH, T, 4)
    runtime.run_step(_model(), types.SimpleNamespace(desc=None), buf, hidden, None, None, None, sampling=sampling)


def test_a_step_draws_into_its_buffer(calls):
    buf = _buffers()
    _step(buf, runtime.Sampling(_model(), BATCH, temperature=0.5))
    assert calls == ["medusa_heads", "tree_verify_step", "sample", "accept_longest_prefix", "kv_compact"]
    assert buf.node_argmax.tolist() == [[0, 1, 2], [3, 4, 5]]


def test_a_step_without_logits_is_refused_whole(calls):
    with pytest.raises(P.MedusaError) as e:
        _step(_buffers(logits=False), runtime.Sampling(_model(), BATCH))
    assert e.value.status == EINVAL and calls == []


@pytest.mark.parametrize("batch", [1, 3])
def test_sampling_of_another_batch_is_refused_whole(calls, batch):
    with pytest.raises(P.MedusaError) as e:
        _step(_buffers(), runtime.Sampling(_model(), batch))
    assert e.value.status == ESHAPE and calls == []


def test_tokens_that_do_not_lie_side_by_side_are_refused(calls):
    """A flattened copy of them would be drawn into, and lost."""
    sampling = runtime.Sampling(_model(), BATCH)
    with pytest.raises(P.MedusaError) as e:
        sampling.draw(torch.zeros(BATCH, T, VOCAB), torch.zeros(BATCH, T + 1, dtype=torch.int32)[:, :T])
    assert e.value.status == ESHAPE and calls == []
