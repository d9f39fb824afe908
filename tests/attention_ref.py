"""Linear attention on ciphertexts from the oracle's calls (numpy arrays), by the formulas of the public header."""
import numpy as np

from ckks_inputs import galois_element, uniform_residues


class Shape:
    """A parameter set's keys and inputs for heads of n1 * n2 components: uniform residues, which is what keys and ciphertexts are."""

    def __init__(self, params, ref_ctx, n1, n2, stride, seed=1):
        self.p, self.c, self.n1, self.n2, self.seed = params, ref_ctx, n1, n2, seed
        L = params.logN
        self.baby = [galois_element(b * stride % (params.N // 2), L) for b in range(1, n1)]
        self.giant = [galois_element(g * n1 * stride % (params.N // 2), L) for g in range(1, n2)]
        self.value = [galois_element(-g * n1 * stride % (params.N // 2), L) for g in range(1, n2)]
        self.mult_key = self.key()
        self.baby_keys = [self.key() for _ in self.baby]
        self.giant_keys = [self.key() for _ in self.giant]
        self.value_keys = [self.key() for _ in self.value]

    def draw(self, moduli, lead):
        self.seed += 1
        return uniform_residues(self.seed * 7919, moduli, lead, self.p.N)

    def key(self):
        return self.draw(self.p.moduli, (self.p.dnum, 2))

    def cts(self, lead, nl):
        return self.draw(self.p.q[:nl], tuple(lead) + (2,))


def _rotations(s, ct, elements, keys):
    return [ct] + [s.c.hrot(ct, g, k) for g, k in zip(elements, keys)]


def _add(s, a, b):
    return s.c.pointwise(a, b, list(range(a.shape[-2])), "add")


def _products(s, pairs, acc=None):
    for a, b in pairs:
        acc = s.c.tensor_acc(np.ascontiguousarray(a), np.ascontiguousarray(b), acc)
    return acc


def read(s, q, state, extra):
    """q [B][2][nl][N], state [n2][n1][B][2][nl][N] or None, extra [B][3][nl][N] or None."""
    if state is None:
        return s.c.relin(extra, s.mult_key)
    Q = _rotations(s, q, s.baby, s.baby_keys)
    d = _products(s, zip(Q, state[0]), extra)
    y = [s.c.relin(_products(s, zip(Q, state[g])), s.mult_key) for g in range(1, s.n2)]
    return s.c.relin_rotated(d, s.mult_key, np.stack(y) if y else None, s.giant, s.giant_keys)


def update(s, k, v, state):
    """k, v [C][B][2][nl][N]."""
    K = [_rotations(s, x, s.baby, s.baby_keys) for x in k]
    V = [_rotations(s, x, s.value, s.value_keys) for x in v]
    out = []
    for g in range(s.n2):
        row = []
        for b in range(s.n1):
            m = s.c.relin(_products(s, [(K[c][b], V[c][g]) for c in range(len(k))]), s.mult_key)
            row.append(m if state is None else _add(s, m, np.ascontiguousarray(state[g][b])))
        out.append(np.stack(row))
    return np.stack(out)


def decayed(s, state, decay):
    if decay is None:
        return state
    n2, n1, B, two, nl, N = state.shape
    return s.c.pmult(state.reshape(-1, two, nl, N), decay).reshape(state.shape)


def step(s, q, k, v, state, decay):
    m = update(s, k[None], v[None], state)
    return read(s, q, m, None), decayed(s, m, decay)


def score(s, q, k):
    p = s.c.relin(s.c.tensor_acc(q, k), s.mult_key)
    p = s.c.hrot_sum(p, s.baby, s.baby_keys) if s.baby else p
    return s.c.hrot_sum(p, s.giant, s.giant_keys) if s.giant else p


def chunk(s, q, k, v, state, decay):
    outs = [read(s, q[t], state, _products(s, [(score(s, q[t], k[u]), v[u]) for u in range(t + 1)])) for t in range(len(q))]
    return np.stack(outs), decayed(s, update(s, k, v, state), decay)
