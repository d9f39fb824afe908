"""Rotary tables against the rotation of pairs by complex numbers, and the attention formulas of tests/attention_ref.py, which the
GPU is held to, against linear attention on plain numbers through the oracle's keys and decryption. CPU only."""
import numpy as np
import pytest

import attention_ref as ra
from ckks_inputs import galois_element, make_params
from harness import Keys, encode_plain_eval_ext
from oracle import ref
from paper_2604_03425_amd.rope import rope_frequencies, rope_tables


@pytest.mark.parametrize("packing", ["components", "tokens"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("head,rot", [(2, 2), (8, 8), (8, 4), (6, 2), (16, 16)])
@pytest.mark.parametrize("scaling", [None, dict(kind="linear", factor=3.0), dict(kind="base", factor=4.0),
                                     dict(kind="by_parts", factor=8.0, original=64)])
def test_tables_turn_pairs(packing, layout, head, rot, scaling):
    lanes = 16
    slots = lanes * head
    rng = np.random.default_rng(head * 31 + rot)
    pos = rng.integers(0, 100000, (2, lanes)).astype(float)
    factors = rng.uniform(.5, 2, (2, lanes))
    x = rng.normal(size=(lanes, head))
    steps, w = rope_tables(slots, head, pos, rot, layout, packing, scaling=scaling, factors=factors)
    assert w.shape == (2, len(steps) + 1, slots) and len(steps) <= 2
    freq, grow = rope_frequencies(rot, scaling=scaling)
    flat = (x.T if packing == "components" else x).reshape(-1)
    for s in range(2):
        got = w[s, 0] * flat + sum(w[s, r + 1] * np.roll(flat, -st) for r, st in enumerate(steps))
        got = got.reshape(head, lanes).T if packing == "components" else got.reshape(lanes, head)
        lo, hi = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
        z = (x[:, lo] + 1j * x[:, hi]) * np.exp(1j * pos[s][:, None] * freq) * grow
        want = x.copy()
        want[:, lo], want[:, hi] = z.real, z.imag
        # angles up to 1e5 are off by half a step of 1e5 at most, 2^-37; products and sums of a few doubles of magnitude below 10
        assert np.abs(got - want * factors[s][:, None]).max() < 1e5 * 2.0 ** -50 * 10


def test_frequencies():
    f = rope_frequencies(64)[0]
    assert f[0] == 1.0 and abs(f[-1] - 10000.0 ** (-62 / 64)) < 1e-18 and (np.diff(f) < 0).all()
    assert np.allclose(rope_frequencies(64, scaling=dict(kind="linear", factor=8))[0] * 8, f, rtol=1e-15)
    g = rope_frequencies(64, scaling=dict(kind="base", factor=8))[0]
    assert g[0] == 1.0 and abs(g[-1] * 8 / f[-1] - 1) < 1e-12
    h, grow = rope_frequencies(64, scaling=dict(kind="by_parts", factor=8, original=2048))
    assert h[0] == f[0] and abs(h[-1] * 8 / f[-1] - 1) < 1e-12 and abs(grow - (0.1 * np.log(8) + 1)) < 1e-15


@pytest.mark.parametrize("bad", [dict(head_dim=5), dict(rot_dim=3), dict(rot_dim=16), dict(rot_dim=0), dict(layout="pairs"),
                                 dict(packing="rows"), dict(positions=np.zeros((1, 7))), dict(positions=np.zeros(8)),
                                 dict(scaling=dict(kind="linear", factor=.5)), dict(scaling=dict(kind="none", factor=2))])
def test_tables_refuse(bad):
    with pytest.raises(ValueError):
        rope_tables(**dict(dict(slots=64, head_dim=8, positions=np.zeros((1, 8))), **bad))


def test_linear_attention_decrypts_to_itself():
    """A chunk of 3 tokens, its decay, then a step: rotary positions with the decays folded in, per-lane decays. Errors: an input at
    scale 2^40 on a ring of 2^10 carries at most 2^14 of encryption, rounding and key-switch noise, 2^-26 of its unit; an output is a
    sum of T d products of three such numbers and factors of at most decay^-3 = 3."""
    d, n1, n2, lanes_bits = 8, 4, 2, 6
    p = make_params(10, 7, 50, 3, 60, 3)
    c, S, lanes = ref.RefContext(p), p.N // 2, 1 << lanes_bits
    assert lanes * d == S
    keys = Keys(p, c, 3)
    s = ra.Shape(p, c, n1, n2, lanes)
    s.mult_key = keys.relin_key()
    s.baby_keys, s.giant_keys, s.value_keys = ([keys.rotation_key(g) for g in e] for e in (s.baby, s.giant, s.value))
    assert s.value == s.giant[::-1]      # the lanes' rotations are cyclic: a value's key is a giant step's
    rng = np.random.default_rng(2)
    T, scale = 4, 2.0 ** 40
    q, k, v = (rng.uniform(-1, 1, (T, lanes, d)) for _ in range(3))
    decay, pos = rng.uniform(.7, 1, lanes), rng.integers(0, 500, lanes).astype(float)
    enc = lambda x: np.stack([keys.encrypt_slots(t.T.reshape(-1), scale, 7) for t in x])[:, None]   # noqa: E731
    cq, ck, cv = enc(q), enc(k), enc(v)
    rope_key = {}

    def rotary(ct, t, sign, in_call, nl):
        steps, w = rope_tables(S, d, (pos + t)[None], factors=decay[None] ** (sign * (in_call + 1)))
        pt = np.stack([encode_plain_eval_ext(c, row, float(p.q[nl - 1]), nl) for row in w[0]])[None]
        gs = [galois_element(x % S, p.logN) for x in steps]
        for g in gs:
            rope_key.setdefault(g, keys.rotation_key(g))
        return c.rescale(c.rope(np.ascontiguousarray(ct[:, :, :nl]), pt, gs, [rope_key[g] for g in gs]))

    turned = lambda ct, ts, sign, nl: np.stack([rotary(ct[t], t, sign, t - ts[0], nl) for t in ts])   # noqa: E731
    fade = ref.encode(np.repeat(decay[None] ** 3, d, axis=0).reshape(-1), p.N, float(p.q[5]))
    pt_fade = c.ntt(c.signed_to_rns(fade, list(range(6)))[None], list(range(6)))[0]
    o, st = ra.chunk(s, turned(cq, [0, 1, 2], 1, 7), turned(ck, [0, 1, 2], -1, 7), np.ascontiguousarray(cv[:3, :, :, :6]), None, pt_fade)
    st = c.rescale(st.reshape(-1, 2, 6, p.N)).reshape(n2, n1, 1, 2, 5, p.N)
    o3, st3 = ra.step(s, turned(cq, [3], 1, 6)[0], turned(ck, [3], -1, 6)[0], np.ascontiguousarray(cv[3, :, :, :5]), st, None)
    freq = rope_frequencies(d)[0]
    turn = lambda x, t: np.concatenate((x[:, :4] * np.cos((pos + t)[:, None] * freq) - x[:, 4:] * np.sin((pos + t)[:, None] * freq),   # noqa: E731
                                        x[:, 4:] * np.cos((pos + t)[:, None] * freq) + x[:, :4] * np.sin((pos + t)[:, None] * freq)), 1)
    state = np.zeros((lanes, d, d))
    for t in range(T):
        state = decay[:, None, None] * state + np.einsum("li,lj->lij", turn(k[t], t), v[t])
        want = np.einsum("li,lij->lj", turn(q[t], t), state)
        got = keys.decrypt_slots((o[t] if t < 3 else o3)[0], scale ** 3).real.reshape(d, lanes).T
        assert np.abs(got - want).max() < T * d * 3 * 3 * 2.0 ** -26, t
    # the new state's diagonals, before the last token's decay: decay^-1 times the state
    for g in range(n2):
        for b in range(n1):
            got = keys.decrypt_slots(st3[g, b, 0], scale ** 2).real.reshape(d, lanes).T
            i = np.arange(d)
            want = state[:, (i + b) % d, (i - g * n1) % d] / decay[:, None]
            assert np.abs(got - want).max() < T * 3 * 3 * 2.0 ** -26
