"""The attention example of the README, run as it stands on the oracle's calls in the library's place: it decrypts to linear attention
on the plain numbers. CPU only."""
import os
import re
from types import SimpleNamespace

import numpy as np

import attention_ref as ra
from ckks_inputs import galois_element, make_params
from harness import Keys, encode_plain_eval, encode_plain_eval_ext
from oracle import ref
from paper_2604_03425_amd.rope import rope_frequencies, rope_tables

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def _block():
    blocks = re.findall(r"```python\n(.*?)```", open(README).read(), flags=re.S)
    block, = [b for b in blocks if "ckks_linattn_chunk" in b]
    return block


def _library(c, shape):
    """The calls of the example, by the oracle."""
    def rope(ctx, out, x, B, nl, weights, npt, elements, keys, ws):
        assert weights.shape[0] == npt and x.shape[-2] == nl
        out[:] = c.rope(x.reshape(B, 2, nl, -1), weights, elements, keys).reshape(out.shape)

    def rescale(ctx, out, x, B, nl, ws):
        assert x.shape[-2] == nl
        out[:] = c.rescale(x.reshape(B, 2, nl, -1)).reshape(out.shape)

    def attention(f, o, state_out, q, k, v, state_in, decay, B, nl, n1, n2, stride, keys, lead):
        assert (n1, n2, stride) == (shape.n1, shape.n2, c.N // 2 // (n1 * n2))
        assert all(x.shape == lead + (B, 2, nl, c.N) for x in (o, q, k, v)) and state_out.shape == (n2, n1, B, 2, nl, c.N)
        assert (state_in is None or state_in.shape == state_out.shape) and decay.shape == (nl, c.N)
        shape.mult_key, shape.baby_keys, shape.giant_keys, shape.value_keys = keys
        if f is ra.step:
            q, k, v = q[0], k[0], v[0]
        got = f(shape, q, k, v, state_in, decay)
        o[:], state_out[:] = got[0].reshape(o.shape), got[1]

    def step(ctx, o, out, q, k, v, S, decay, B, nl, n1, n2, stride, mult, baby, giant, value, ws):
        attention(ra.step, o, out, q, k, v, S, decay, B, nl, n1, n2, stride, (mult, baby, giant, value), (1,))

    def chunk(ctx, o, out, q, k, v, S, decay, tokens, B, nl, n1, n2, stride, mult, baby, giant, value, ws):
        attention(ra.chunk, o, out, q, k, v, S, decay, B, nl, n1, n2, stride, (mult, baby, giant, value), (tokens,))

    return SimpleNamespace(rope_tables=rope_tables, ckks_rope=rope, ckks_rescale=rescale, ckks_linattn_step=step,
                           ckks_linattn_chunk=chunk, OP_ROPE=8, OP_RESCALE=5, OP_LINATTN_STEP=9, OP_LINATTN_CHUNK=10)


def test_the_attention_example_decrypts_to_attention():
    """The shape and with it the errors of test_linear_attention_decrypts_to_itself: sums of T d products of three numbers that are
    2^-26 of their unit off, and factors of at most decay^-3 = 3."""
    head, n1, n2, tokens, nl = 8, 4, 2, 3, 6
    p = make_params(10, 7, 50, 3, 60, 3)
    c, N, lanes = ref.RefContext(p), p.N, p.N // 2 // head
    keys = Keys(p, c, 4)
    shape = ra.Shape(p, c, n1, n2, lanes)
    rng = np.random.default_rng(6)
    T, scale = tokens + 1, 2.0 ** 40
    plain = {x: rng.uniform(-1, 1, (T, lanes, head)) for x in "qkv"}
    decay, positions = rng.uniform(.7, 1, lanes), rng.integers(0, 500, lanes).astype(float)
    cts = {x: np.stack([keys.encrypt_slots(t.T.reshape(-1), scale, 7) for t in plain[x]])[:, None] for x in "qkv"}
    rope_step, = rope_tables(N // 2, head, positions[None])[0]
    made = [keys.rotation_key(g) for g in shape.baby], [keys.rotation_key(g) for g in shape.giant]
    names = dict(
        np=np, ck=_library(c, shape), ctx=SimpleNamespace(workspace=lambda *a: None, linattn_workspace=lambda *a: None), p=p, N=N,
        galois_element=galois_element, head=head, lanes=lanes, n1=n1, n2=n2, tokens=tokens, nl=nl, decay=decay, positions=positions,
        new=lambda *s: np.zeros(s, dtype=np.uint64), cut=lambda x, limbs: np.ascontiguousarray(x[..., :limbs, :]),
        encode=lambda slots, scale, nl: encode_plain_eval(c, slots, float(scale), nl),
        encode_ext=lambda slots, scale, nl: np.stack([[encode_plain_eval_ext(c, w, float(scale), nl) for w in s] for s in slots]),
        rope_keys=[keys.rotation_key(galois_element(rope_step, p.logN))], evk_mult=keys.relin_key(), evk_baby=made[0],
        evk_giant=made[1], evk_value=made[1][::-1], **cts)
    exec(_block(), names)
    outs = [*names["o"][:, 0], *names["o1"][:, 0]]
    assert len(outs) == T and names["state"].shape[-2] == nl - 2
    freq, h = rope_frequencies(head)[0], head // 2

    def turn(x, t):
        a = (positions + t)[:, None] * freq
        return np.concatenate((x[:, :h] * np.cos(a) - x[:, h:] * np.sin(a), x[:, h:] * np.cos(a) + x[:, :h] * np.sin(a)), 1)

    state = np.zeros((lanes, head, head))
    for t in range(T):
        state = decay[:, None, None] * state + np.einsum("li,lj->lij", turn(plain["k"][t], t), plain["v"][t])
        want = np.einsum("li,lij->lj", turn(plain["q"][t], t), state)
        got = keys.decrypt_slots(outs[t], scale ** 3).real.reshape(head, lanes).T
        assert np.abs(got - want).max() < T * head * 3 * 3 * 2.0 ** -26, t
