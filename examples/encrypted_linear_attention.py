"""Linear attention with rotary positions and a decay for each head, on ciphertexts: a prompt of a few tokens as one chunk, then
new tokens one by one, each lane (one head of one sequence) with its own positions and decay.

The client (keys, encryption, decryption) is played by the CPU oracle; everything between runs on the GPU. Prints how far the
decrypted outputs are from the same attention on the plain numbers.

    python examples/encrypted_linear_attention.py [--logN 12] [--head 8] [--tokens 3] [--new 2]
"""
import argparse
import os
import sys

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path[:0] = [ROOT, os.path.join(ROOT, "tests")]


def plain_attention(q, k, v, decay, frequencies, first):
    """o [T][lanes][d] of o_t = q_t S_t, S_t = decay S_{t-1} + k_t v_t^T, with q and k turned to their positions ("half" layout)."""
    T, lanes, d = q.shape
    h = d // 2

    def turn(x, t):
        a = (first + t)[:, None] * frequencies
        lo, hi = x[:, :h], x[:, h:]
        return np.concatenate((lo * np.cos(a) - hi * np.sin(a), hi * np.cos(a) + lo * np.sin(a)), axis=1)

    S, out = np.zeros((lanes, d, d)), []
    for t in range(T):
        S = decay[:, None, None] * S + np.einsum("li,lj->lij", turn(k[t], t), v[t])
        out.append(np.einsum("li,lij->lj", turn(q[t], t), S))
    return np.stack(out)


def main(logN=12, head=8, tokens=3, new=2, seed=7, quiet=False):
    import torch
    import paper_2604_03425_amd as ck
    from ckks_inputs import galois_element, make_params
    from gpu_util import to_dev, to_host
    from harness import Keys, encode_plain_eval, encode_plain_eval_ext
    from oracle import ref

    n1 = 1 << ((head.bit_length()) // 2)
    n2 = head // n1
    nq = 5 + new + 1                      # one level for the positions, one for the state's decay after the chunk and after each token
    p = make_params(logN, nq, 50, 3, 60, -(-nq // 3))
    rc, ctx = ref.RefContext(p), ck.Context(p, 0)
    keys, N, S = Keys(p, rc, seed), p.N, p.N // 2
    lanes, scale = S // head, 2.0 ** 40

    # the client's data: T tokens of every lane, [-1, 1]
    rng = np.random.default_rng(seed)
    T = tokens + new
    q, k, v = (rng.uniform(-1, 1, (T, lanes, head)) for _ in range(3))
    decay, first = rng.uniform(.7, 1, lanes), rng.integers(0, 1000, lanes).astype(float)
    pack = lambda x: x.T.reshape(-1)      # component i of lane l in slot i * lanes + l   # noqa: E731
    encrypt = lambda x: to_dev(np.stack([keys.encrypt_slots(pack(t), scale, nq) for t in x])[:, None])   # noqa: E731
    ct = {name: encrypt(x) for name, x in (("q", q), ("k", k), ("v", v))}

    # keys of the rotations: components by b and by g * n1, all lanes at once; values turn the other way, which is n2 - g forward
    element = lambda step: galois_element(step % S, logN)   # noqa: E731
    rot_key = lambda step: to_dev(keys.rotation_key(element(step)))   # noqa: E731
    evk_mult = to_dev(keys.relin_key())
    baby = [rot_key(b * lanes) for b in range(1, n1)]
    giant = [rot_key(g * n1 * lanes) for g in range(1, n2)]
    value = giant[::-1]

    # positions, and the decays that a call's queries and keys carry: decay^(t+1) and decay^(-t-1) at its token t
    def rotary(x, t0, n, sign, nl):
        in_call = np.arange(n)[:, None] + 1
        steps, w = ck.rope_tables(S, head, first[None] + t0 + np.arange(n)[:, None], factors=decay[None] ** (sign * in_call))
        pt = to_dev(np.stack([[encode_plain_eval_ext(rc, row, float(p.q[nl - 1]), nl) for row in one] for one in w]))
        out, low = torch.empty_like(x), torch.empty((n, 1, 2, nl - 1, N), dtype=x.dtype, device=x.device)
        if not rope_keys:
            rope_keys.extend(rot_key(s) for s in steps)
        ck.ckks_rope(ctx, out, x, n, nl, pt, n, [element(s) for s in steps], rope_keys, ctx.workspace(ck.OP_ROPE, n, nl))
        ck.ckks_rescale(ctx, low, out, n, nl, ctx.workspace(ck.OP_RESCALE, n, nl))     # the weights' scale is the dropped prime
        return low

    rope_keys = []

    def call(t0, n, nl, state):
        """One call on n tokens at nl limbs: outputs, and the state times decay^n, a level down."""
        cut = lambda x, m: x[t0:t0 + n, :, :, :m].contiguous()   # noqa: E731
        Q, K, V = rotary(cut(ct["q"], nl + 1), t0, n, 1, nl + 1), rotary(cut(ct["k"], nl + 1), t0, n, -1, nl + 1), cut(ct["v"], nl)
        fade = to_dev(encode_plain_eval(rc, pack(np.repeat(decay[:, None] ** n, head, axis=1)), float(p.q[nl - 1]), nl))
        o = torch.empty((n, 1, 2, nl, N), dtype=Q.dtype, device=Q.device)
        full = torch.empty((n2, n1, 1, 2, nl, N), dtype=Q.dtype, device=Q.device)
        low = torch.empty((n2, n1, 1, 2, nl - 1, N), dtype=Q.dtype, device=Q.device)
        tail = (1, nl, n1, n2, lanes, evk_mult, baby, giant, value)
        if n > 1:
            ck.ckks_linattn_chunk(ctx, o, full, Q, K, V, state, fade, n, *tail, ctx.linattn_workspace(ck.OP_LINATTN_CHUNK, n, 1, nl, n1, n2))
        else:
            ck.ckks_linattn_step(ctx, o, full, Q, K, V, state, fade, *tail, ctx.linattn_workspace(ck.OP_LINATTN_STEP, 1, 1, nl, n1, n2))
        ck.ckks_rescale(ctx, low, full, head, nl, ctx.workspace(ck.OP_RESCALE, head, nl))
        return o, low

    got, state, nl = [], None, nq - 1
    t0 = 0
    for n in [tokens] + [1] * new:
        o, state = call(t0, n, nl, state)
        got += [keys.decrypt_slots(x[0], scale ** 3).real.reshape(head, lanes).T for x in to_host(o)]
        t0, nl = t0 + n, nl - 1
    want = plain_attention(q, k, v, decay, ck.rope_frequencies(head)[0], first)
    errors = [float(np.abs(g - w).max()) for g, w in zip(got, want)]
    if not quiet:
        for t, e in enumerate(errors):
            print("token %d (%s): largest error %.2e, largest output %.2f" % (t, "chunk" if t < tokens else "step", e, np.abs(want[t]).max()))
    return errors


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in (("logN", 12), ("head", 8), ("tokens", 3), ("new", 2)):
        ap.add_argument("--" + name, type=int, default=default)
    main(**vars(ap.parse_args()))
