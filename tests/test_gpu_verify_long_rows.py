"""Judging of drafted tokens whose rows have more logits than 256 spans of 1024, against oracle/branch.py: a span has several rounds, which the other tests do not reach.

Answers are whole numbers and have to be equal.  Both sides compute in 64 bits, with roundings of 1e-15 or so a border: a draw has a chance of V * 1e-15, 7e-8 or less, to fall
next to one, and fewer than 300 are made."""
import numpy as np
import pytest
import torch

from oracle import branch as ob
from tests.test_gpu_verify import call, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [262143, 262144, 262145, 263169, 300007, 524289])
@pytest.mark.parametrize("dtype, drawn, tree", [("bf16", True, True), ("f32", True, False), ("bf16", False, True)])
def test_rows_of_several_rounds(vocab, dtype, drawn, tree):
    s = make(vocab, [1, 4, 0, 9, 3], vocab, dtype, drawn, tree, spread=1.0)
    check(s, call(s))
    s["temperature"][1], s["temperature"][3] = 0.0, 40.0
    s["accept"][2::3] = 0.9999
    s["sample"][:] = [0.0, 1 - 2.0 ** -24, 0.5, 0.999, 0.7]
    check(s, call(s))


def test_chains_of_many_logits():
    s = make(5, [9, 20, 4], 270001, "bf16", True, False)           # 33 rows: more than 2^23 logits, whose first sums have 32 bits
    check(s, call(s))


def test_a_batch_that_samples():
    """One token a request, more requests than there are workgroups for spans of their own."""
    s = make(6, [1] * 150, 265000, "bf16", False, False)
    check(s, call(s))


@pytest.mark.parametrize("vocab, drawn", [(5000011, True), (1 << 26, False)])
def test_the_longest_rows(vocab, drawn):
    rng = np.random.default_rng(7)
    T = 3 if drawn else 1
    target = torch.from_numpy(rng.standard_normal((T, vocab), np.float32)).bfloat16()
    draft = torch.from_numpy(rng.standard_normal((T, vocab), np.float32)).bfloat16() if drawn else None
    s = dict(target=target, draft=draft, vocab=vocab, tokens=np.array([0, 77, vocab - 1], np.int32)[:T], q_start=np.array([0, T], np.int32), sizes=[T], mask=None,
             temperature=np.ones(1, np.float32), accept=np.full(T, 0.3, np.float32), sample=np.array([0.77], np.float32), max_q=T)
    check(s, call(s))
    s["target"][0, vocab - 1] = s["target"][0].max() * 2
    s["temperature"][:] = 0
    check(s, call(s))
    assert drawn or call(s)[2][0] == ob.first_largest(s["target"][0].float().numpy()) == vocab - 1
