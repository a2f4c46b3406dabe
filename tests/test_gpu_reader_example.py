"""The example that runs index, prompt attention, cache and pages together:
its last logits against the same model without a cache.

Bound: an int8 code is off by at most half a step, 1/254 of its block's
largest; for normal values that is a relative error (2-norm) of about
3.5/127/sqrt(12) = 0.8% of keys and of values, e4m3 about 2.7%; two layers of it stay under 4 times that."""
import importlib.util
import os

import pytest
import torch

import paper_2607_16973_amd as tq
from tests.reader import starts_of

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("kind,bound", [("int8", 0.032), ("fp8", 0.108)])
def test_answers_from_passages(kind, bound):
    spec = importlib.util.spec_from_file_location("answers", os.path.join(ROOT, "examples", "answers_from_passages.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    told, logits, whole, reader, live = m.answer(kind=kind)
    assert len(told) == 12 and all(len(row) == 12 for row in told)
    # answers of one question differ in their first token
    assert all(len({told[4 * q + i][0] for i in range(4)}) == 4 for q in range(3))
    counts = [len(row) for row in whole]
    starts = starts_of(counts)
    plain = reader.run(torch.tensor(sum(whole, []), device="cuda"),
                       lambda layer, q, k, v: tq.attention(q, k, v, starts))[starts[1:].long() - 1].double()
    got = logits.double()
    assert torch.linalg.norm(got - plain) <= bound * torch.linalg.norm(plain)
    # the answers that stay: whole pages of a prompt once, a page or two of their own
    kept = [i for i in range(12) if i % 2]
    shared = sum(min((counts[i] - 12) // 64 for i in kept if i // 4 == q) for q in range(3))
    own = sum(-(-counts[i] // 64) - (counts[i] - 12) // 64 for i in kept)
    assert live == shared + own
