"""The oracle's results do not depend on how many threads share a call."""
import os

import numpy as np
import pytest

import attention_ref
from ckks_inputs import make_params
from oracle import ref


def _calls(shape, B, nl):
    p = make_params(*shape)
    c = ref.RefContext(p)
    s = attention_ref.Shape(p, c, 2, 2, 4)
    a, b, key = s.cts((B,), nl), s.cts((B,), nl), s.mult_key
    d = c.tensor_acc(a, b)
    w, pt = s.draw(p.q[:nl] + p.p, (1, 2)), s.draw(p.q[:nl] + p.p, (2, 2))
    ids = list(range(nl))
    return [d, c.tensor_acc(a, b, d), c.hrot(a, s.baby[0], key), c.hmult_relin(a, b, key), c.relin(d, key), c.rescale(a),
            c.hrot_sum(a, s.baby, s.baby_keys), c.rope(a, w, s.baby, s.baby_keys), c.relin_rotated(d, key, a[None], s.giant, s.giant_keys),
            c.switch_sum(d, key, a, s.baby, s.baby_keys, more=True), c.keyswitch(np.ascontiguousarray(a[:, 0]), key),
            c.pcmm_bsgs_double_hoisted(a, pt, 2, 2, 4, s.baby_keys, s.giant_keys), c.ntt(a, ids), c.intt(a, ids),
            c.pointwise(a, b, ids, "mul"), c.automorph(a, ids, s.baby[0], True)]


@pytest.mark.parametrize("shape,B,nl", [((10, 5, 50, 2, 60, 3), 3, 5), ((13, 4, 60, 2, 60, 2), 1, 3), ((12, 10, 45, 10, 60, 1), 2, 10)])
def test_any_number_of_threads(shape, B, nl):
    try:
        ref.set_team(1)
        want = _calls(shape, B, nl)
        for threads, team in ((1, 5), (4, 1), (2, 16)):
            ref.set_threads(threads)
            ref.set_team(team)
            for i, (x, y) in enumerate(zip(_calls(shape, B, nl), want)):
                assert (x == y).all(), (threads, team, i)
    finally:
        ref.set_threads(1)
        ref.set_team(min(16, os.cpu_count() or 1))
