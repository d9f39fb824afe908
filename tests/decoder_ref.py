"""Attention over a paged cache and the root-mean-square norm from the oracle's calls (numpy arrays), by the formulas of the public
header. Keys come from attention_ref.Shape."""
import numpy as np


def _number(s, value, nl):
    """A number in every slot, as residues [1][1][nl][N]."""
    return np.stack([np.full(s.p.N, value % m, dtype=np.uint64) for m in s.p.q[:nl]])[None]


def _pointwise(s, a, b, op):
    nl, N = a.shape[-2:]
    b = np.broadcast_to(b, a.shape)
    return s.c.pointwise(np.ascontiguousarray(a.reshape(-1, nl, N)), np.ascontiguousarray(b.reshape(-1, nl, N)), list(range(nl)),
                         op).reshape(a.shape)


def plus(s, ct, value):
    """ct [B][2][nl][N] plus a number in every slot."""
    out = ct.copy()
    out[:, 0] = _pointwise(s, ct[:, 0], _number(s, value, ct.shape[-2]), "add")
    return out


def times(s, x, value):
    return _pointwise(s, x, _number(s, value, x.shape[-2]), "mul")


def cut(ct, nl):
    return np.ascontiguousarray(ct[..., :nl, :])


def slot_sum(s, d):
    steps = [(e, k) for e, k in ((s.baby, s.baby_keys), (s.giant, s.giant_keys)) if e]
    p = s.c.switch_sum(d, s.mult_key, more=not steps)
    for i, (elements, keys) in enumerate(steps):
        p = s.c.switch_sum(p, y=p, galois_elts=elements, evks=keys, more=i + 1 == len(steps))
    return p


def score(s, q, k, bias, squarings):
    """q, k [B][2][nl][N]: the weights u."""
    u = plus(s, slot_sum(s, s.c.tensor_acc(q, k)), bias)
    for _ in range(squarings):
        u = s.c.switch_sum(s.c.tensor_acc(u, u), s.mult_key, more=True)
    return u


def visible(t, window, sinks):
    return [u for u in range(t + 1) if window == 0 or t - u < window or u < sinks]


def attention(s, q, keys, values, new_lens, window, sinks, bias, squarings):
    """q [rows][2][nl][N]; keys, values: every sequence's cached ciphertexts [len][2][limbs][N]."""
    nl = q.shape[-2]
    L = nl - 1 - squarings
    out, row = [], 0
    for k, v, m in zip(keys, values, new_lens):
        for t in range(len(k) - m, len(k)):
            see = visible(t, window, sinks)
            u = score(s, np.repeat(q[row:row + 1], len(see), axis=0), cut(k[see], nl), bias, squarings)
            d = None
            for i, x in enumerate(see):
                d = s.c.tensor_acc(u[i:i + 1], cut(v[x:x + 1], L), d)
            out.append(s.c.relin(d, s.mult_key)[0])
            row += 1
    return np.stack(out)


def rmsnorm(s, x, res, gain, square, eps, start, factors):
    h = x if res is None else _pointwise(s, x, res, "add")
    m = plus(s, slot_sum(s, times(s, s.c.tensor_acc(h, h), square)), eps)
    y = plus(s, times(s, m, -1), start)
    for f in factors:
        nl = y.shape[-2]
        u, w = (s.c.switch_sum(s.c.tensor_acc(z, y), s.mult_key, more=True) for z in (cut(m, nl), y))
        d = times(s, s.c.tensor_acc(u, w), -1)
        d[:, :2] = _pointwise(s, d[:, :2], times(s, cut(y, nl - 1), f), "add")
        y = s.c.switch_sum(d, s.mult_key, more=True)
    L = y.shape[-2]
    g = cut(h, L) if gain is None else s.c.rescale(s.c.pmult(cut(h, L + 1), gain))
    return s.c.relin(s.c.tensor_acc(g, y), s.mult_key), h
