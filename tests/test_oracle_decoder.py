"""The formulas of tests/decoder_ref.py, which the GPU is held to, through the oracle's keys and decryption: division by a main prime
with the special ones, attention with a window and sinks, the norm with its plan. CPU only."""
import math

import numpy as np
import pytest

import attention_ref
import decoder_ref
from ckks_inputs import make_params, uniform_residues
from harness import Keys, encode_plain_eval
from oracle import ref
from paper_2604_03425_amd.binding import attn_pairs
from paper_2604_03425_amd.norm import _step, rmsnorm_plan


def _lanes(p, keys, ctx, n1, n2):
    lanes = p.N // 2 // (n1 * n2)
    s = attention_ref.Shape(p, ctx, n1, n2, lanes)
    s.mult_key = keys.relin_key()
    s.baby_keys, s.giant_keys = ([keys.rotation_key(g) for g in e] for e in (s.baby, s.giant))
    return s, lanes


@pytest.mark.parametrize("shape", [(10, 5, 40, 2, 50, 3), (10, 4, 60, 1, 60, 4), (10, 3, 45, 3, 60, 1)])
def test_the_division_by_a_main_prime_too(shape):
    """With X the accumulators: ModDown is x = X / P + e, |e| <= K / 2 + 1, the division by q P is y = X / (P q) + f, |f| <= (K + 1) / 2 + 1,
    so q y - x is at most q ((K + 1) / 2 + 1) + K / 2 + 1 modulo the primes."""
    p = make_params(*shape)
    c, N = ref.RefContext(p), p.N
    nl, K = len(p.q), len(p.p)
    d = uniform_residues(3, p.q, (1, 3), N)
    key = uniform_residues(4, p.moduli, (p.dnum, 2), N)
    both, plain = c.switch_sum(d, key, more=True), c.switch_sum(d, key)
    last, Q = p.q[nl - 1], math.prod(p.q[:nl - 1])
    for comp in (0, 1):
        x = ref.crt_centred(c.intt(plain[:, comp], list(range(nl)))[0], p.q)
        y = ref.crt_centred(c.intt(both[:, comp], list(range(nl - 1)))[0], p.q[:nl - 1])
        for a, b in list(zip(x, y))[:200]:
            e = (last * int(b) - int(a) + last * Q // 2) % (last * Q) - last * Q // 2
            assert abs(e) <= last * ((K + 1) // 2 + 1) + K


def test_slot_sums_and_scores_decrypt():
    """(x + bias)^2 of scores x, at scale 2^40 on 50-bit primes: each input carries at most 2^-26 of its unit (test_oracle_attention.py), a
    score is a sum of d products; the primes are 2^50 give or take 2^-30."""
    n1, n2, d = 4, 2, 8
    p = make_params(10, 6, 50, 2, 60, 3)
    c = ref.RefContext(p)
    keys = Keys(p, c, 5)
    s, lanes = _lanes(p, keys, c, n1, n2)
    rng = np.random.default_rng(1)
    q, k = rng.uniform(-.5, .5, (2, d, lanes))
    scale = 2.0 ** 45
    cq, ck = (keys.encrypt_slots(x.reshape(-1), scale, 6)[None] for x in (q, k))
    after = scale ** 2 / p.q[5]
    for squarings in (0, 1, 2):
        u = decoder_ref.score(s, cq, ck, round(after), squarings)
        sc = after
        for i in range(squarings):
            sc = sc * sc / p.q[4 - i]
        assert u.shape[-2] == 5 - squarings
        x = (q * k).sum(axis=0) + 1.0
        want = np.tile(x ** (1 << squarings), d)
        err = np.abs(keys.decrypt_slots(u[0], sc).real - want).max()
        # noise 2^20 at the scale of the last step, times the derivative of the squarings, x at most 3
        assert err < (1 << squarings) * 3.0 ** (1 << squarings) * 2.0 ** 20 / min(after, sc), (squarings, err)


def test_attention_decrypts_to_itself():
    n1, n2, d = 2, 2, 4
    p = make_params(10, 6, 50, 2, 60, 3)
    c = ref.RefContext(p)
    keys = Keys(p, c, 7)
    s, lanes = _lanes(p, keys, c, n1, n2)
    rng = np.random.default_rng(2)
    T, new, scale = 6, 2, 2.0 ** 45
    q, k, v = rng.uniform(-.5, .5, (3, T, d, lanes))
    enc = lambda x: np.stack([keys.encrypt_slots(t.reshape(-1), scale, 6) for t in x])   # noqa: E731
    ck, cv, cq = enc(k), enc(v), enc(q[T - new:])
    after = scale ** 2 / p.q[5]
    for window, sinks in ((0, 0), (2, 0), (2, 1), (1, 4)):
        o = decoder_ref.attention(s, cq, [ck], [cv], [new], window, sinks, round(after), 1)
        for r, t in enumerate(range(T - new, T)):
            see = [u for u in range(t + 1) if not window or t - u < window or u < sinks]
            assert decoder_ref.visible(t, window, sinks) == see
            w = [((q[t] * k[u]).sum(axis=0) + 1.0) ** 2 for u in see]
            want = sum(x * v[u] for x, u in zip(w, see))
            got = keys.decrypt_slots(o[r], after ** 2 / p.q[4] * scale).real.reshape(d, lanes)
            assert np.abs(got - want).max() < len(see) * 2 * 9 * 2.0 ** 20 / (after ** 2 / p.q[4])
        assert attn_pairs([new], [T], window, sinks) == sum(len(decoder_ref.visible(t, window, sinks)) for t in range(T - new, T))


@pytest.mark.parametrize("lo,hi,iterations", [(.5, 2, 0), (.5, 2, 1), (.1, 2, 2), (.05, 4, 3), (.5, .5, 1), (1e-3, 10, 4), (.9, 1.1, 2)])
@pytest.mark.parametrize("scale", [2.0 ** 30, 2.0 ** 40, 2.0 ** 45])
def test_the_plan_in_plain_numbers(lo, hi, iterations, scale):
    """The call's formula on real numbers with the plan's integers: what it says about the error, in units of the last place of doubles
    times what the roundings of the integers (2^-28 at the smallest scales) make of it."""
    from ckks_inputs import find_ntt_primes
    q, nl, d = find_ntt_primes(50, 12, 12), 11, 16
    plan = rmsnorm_plan(q, nl, scale, d, lo, hi, iterations)
    assert len(plan["factors"]) == iterations
    mean = np.geomspace(lo, hi, 1001)
    m = plan["square"] * d * scale ** 2 * mean / q[nl - 1]
    y = plan["start"] - m
    a = nl - 1
    for f in plan["factors"]:
        u, w = m * y / q[a - 1], y * y / q[a - 1]
        y = (f * y - u * w) / q[a - 2]
        a -= 2
        assert np.abs(y).max() < 2.0 ** 62
    rel = y / plan["scale"] * np.sqrt(mean) - 1.0
    assert np.abs(rel).max() <= plan["error"] * (1 + 1e-6) + 2.0 ** -28
    assert np.abs(rel).max() >= plan["error"] * (1 - 1e-2) - 2.0 ** -28       # and it is not a loose bound
    if iterations:
        worse = 1.0 - _step(_step(.5))
        assert plan["error"] < 1.0 and (lo < .2 or iterations < 2 or plan["error"] < worse)


@pytest.mark.parametrize("bad", [dict(lo=0.0), dict(lo=2.0, hi=1.0), dict(iterations=5), dict(iterations=-1), dict(nlimbs=13),
                                 dict(scale=2.0 ** 52), dict(nlimbs=1)])
def test_the_plan_refuses(bad):
    from ckks_inputs import find_ntt_primes
    q = find_ntt_primes(50, 12, 12)
    with pytest.raises(ValueError):
        rmsnorm_plan(**dict(dict(q=q, nlimbs=11, scale=2.0 ** 40, components=16, lo=.1, hi=1.0, iterations=2), **bad))


def test_the_norm_decrypts_to_itself():
    n1, n2, d = 4, 2, 8
    p = make_params(10, 9, 50, 3, 60, 3)
    c = ref.RefContext(p)
    keys = Keys(p, c, 9)
    s, lanes = _lanes(p, keys, c, n1, n2)
    rng = np.random.default_rng(3)
    scale, its, nl = 2.0 ** 45, 2, 9
    x, r = rng.uniform(-1, 1, (2, d, lanes))
    gain = rng.uniform(.5, 2, d)
    h = x + r
    mean = (h * h).mean(axis=0) + .01
    plan = rmsnorm_plan(p.q, nl, scale, d, mean.min(), mean.max(), its, eps=.01)
    L = nl - 1 - 2 * its
    cx, cr = (keys.encrypt_slots(t.reshape(-1), scale, nl)[None] for t in (x, r))
    pt = encode_plain_eval(c, np.repeat(gain, lanes), float(p.q[L]), L + 1)
    for w in (None, pt):
        out, hh = decoder_ref.rmsnorm(s, cx, cr, w, plan["square"], plan["eps"], plan["start"], plan["factors"])
        assert out.shape == (1, 2, L, p.N)
        want = h / np.sqrt(mean) * (1.0 if w is None else gain[:, None])
        got = keys.decrypt_slots(out[0], scale * plan["scale"]).real.reshape(d, lanes)
        # the start's distance, as the plan says, and noise: 2^20 at the input's scale, grown by the steps' derivatives (below 2^4 each)
        assert np.abs(got - want).max() < plan["error"] * np.abs(want).max() + 2.0 ** 20 * 2.0 ** 8 / scale * 8
        assert np.abs(keys.decrypt_slots(hh[0], scale).real.reshape(d, lanes) - h).max() < 2.0 ** 15 / scale
