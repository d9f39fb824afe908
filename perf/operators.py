"""Softmax-free attention on encrypted data: rotary positions, and linear attention with a decay for each head.

Everything here works on RNS-CKKS ciphertexts, (c0, c1) modulo the main primes q_0..q_{nl-1}, evaluation domain, and is exact
integer work, so the two forms of an operator agree in every residue. P is the product of the special primes p_0..p_{K-1};
sigma_g is the Galois map X -> X^g; A(d; key) stands for the two accumulators of a hybrid key switch of the polynomial d before
ModDown (extended basis: the main primes, then the special ones); Rot_r is the rotation of the slots to the left by r,
g = 5^r mod 2N; Relin(d0, d1, d2) = (d0, d1) + ModDown(A(d2; mult key)); ModDown divides by P.

`rope`, rotary positions. A slot vector x becomes w_0 x + sum_r w_r Rot_r(x): w_0 holds the cosines, w_r the sines of the pairs
whose partner is r slots away. Ciphertext b of B takes the weights of set b // (B / npt):
    out = ModDown( w_0 (P c0, P c1) + sum_r w_r (A(sigma_r(c1); key_r) + (P sigma_r(c0), 0)) ).

Linear attention keeps, for a head of d = n1 * n2 components, the matrix S = sum_s decay^(t-s) k_s v_s^T as d ciphertexts, its
diagonals: state[g][b][lane, i] = S[i + b][i - g n1], component i of lane l in slot i * stride + l, where a lane is one head of
one sequence. Decays inside a call come with the weights of the rotary call (q_t scaled by decay^(t+1), k_s by decay^(-s-1));
`decay` is decay^C for every lane as a plaintext.
    K[b] = Rot_{b stride}(k),  Q[b] = Rot_{b stride}(q),  V[g] = Rot_{-g n1 stride}(v)
    read(q, S, e) = ModDown( A(d2; mult key) + (P d0, P d1) + sum_{g>=1} (A(sigma_g(y_g.c1); giant key g) + (P sigma_g(y_g.c0), 0)) )
        with d = e + sum_b Q[b] * S[0][b] (three components), y_g = Relin(sum_b Q[b] * S[g][b]), sigma_g of Rot_{g n1 stride}
`step`, one token:     M = S + Relin(K[b] * V[g]),  o = read(q, M, 0),  new state = decay M
`chunk`, C tokens:     o_t = read(q_t, S, sum_{s<=t} p_ts * v_s),  p_ts = sum2(sum1(Relin(q_t * k_s))),
                       new state = decay (S + Relin(sum_s K_s[b] * V_s[g]))
        sum1(x) = ModDown(P x + sum_{b>=1} (A(sigma_b(c1); baby key b) + (P sigma_b(c0), 0))), sum2 the same over giant steps.
A state that is not given is zero, a decay that is not given is one.
"""
import math
from collections import OrderedDict
from types import SimpleNamespace

import numpy as np
import torch

own = False
DEVICE = "cuda:0"


def _shape(logN, nq, q_bits, np, p_bits, dnum):
    """A parameter set: ring degree, main primes, special primes (number and bits of each) and digits."""
    return dict(logN=logN, nq=nq, q_bits=q_bits, np=np, p_bits=p_bits, dnum=dnum)


MICRO = _shape(16, 24, 50, 8, 60, 3)        # the key-switch micro-benchmark's and the FFN layer's parameters
ATTENTION = _shape(16, 20, 50, 5, 60, 4)    # the attention layer's parameters


def listed():
    return [
        # one new token for eight small groups of lanes on the smallest ring: launches and latency
        dict(name="rope_token_small", op="rope", layout="half", head=16, rot=16, lanes="inner", scaling=1.0, npt=1, nlimbs=4,
             batch=8, **_shape(12, 4, 40, 1, 50, 2)),
        # one new token, one ciphertext, at the benchmark's parameters: a serving loop of one group of lanes
        dict(name="rope_token", op="rope", layout="half", head=64, rot=64, lanes="inner", scaling=1.0, npt=1, nlimbs=24, batch=1,
             **MICRO),
        # a prompt of 16 ciphertexts, token-major as the attention units pack it: 4 position ranges shared by 4 heads each
        dict(name="rope_prompt", op="rope", layout="interleaved", head=64, rot=32, lanes="outer", scaling=8.0, npt=4, nlimbs=20,
             batch=16, **ATTENTION),
        # main primes as large as the special ones, two limbs below the top, a short last digit, a set of weights per ciphertext
        dict(name="rope_60bit_primes", op="rope", layout="half", head=32, rot=8, lanes="outer", scaling=2.5, npt=5, nlimbs=11,
             batch=5, **_shape(15, 13, 60, 3, 60, 5)),
        # the first token of a sequence on a small ring: no state yet
        dict(name="step_first_token", op="step", n1=2, n2=2, state=False, decay=False, nlimbs=5, batch=1,
             **_shape(12, 5, 45, 2, 60, 3)),
        # a token of three groups of lanes with their decays
        dict(name="step_head_16", op="step", n1=4, n2=4, state=True, decay=True, nlimbs=7, batch=3, **_shape(14, 8, 50, 3, 60, 3)),
        # a token of 512 lanes of 64 components each
        dict(name="step_head_64", op="step", n1=8, n2=8, state=True, decay=True, nlimbs=9, batch=1, **_shape(16, 9, 50, 3, 60, 3)),
        # the first chunk of a prompt, uneven splits of the head
        dict(name="chunk_first", op="chunk", tokens=5, n1=4, n2=2, state=False, decay=False, nlimbs=6, batch=2,
             **_shape(13, 6, 50, 2, 60, 3)),
        # a later chunk, two groups of lanes
        dict(name="chunk_ring_15", op="chunk", tokens=3, n1=4, n2=4, state=True, decay=False, nlimbs=9, batch=2,
             **_shape(15, 10, 50, 4, 60, 3)),
        # a later chunk at the attention layer's ring
        dict(name="chunk_head_32", op="chunk", tokens=4, n1=8, n2=4, state=True, decay=True, nlimbs=8, batch=1,
             **_shape(16, 8, 50, 4, 60, 2)),
    ]


def _log_int(rng, lo, hi):
    """An integer in [lo, hi], spread evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


# main primes that a ring degree is used with (its security level bounds the total size of the modulus)
_LIMBS = {12: (2, 5), 13: (2, 6), 14: (3, 9), 15: (5, 18), 16: (4, 24)}


def _draw_shape(rng, logN, most_limbs):
    lo, hi = _LIMBS[logN]
    nq = rng.randint(lo, min(hi, most_limbs))
    dnum = rng.choice([d for d in (1, 2, 3, 4, 6) if d <= nq])
    alpha = -(-nq // dnum)
    return _shape(logN, nq, rng.choice([50, 50, 50, 45, 40, 55, 60]), rng.choice([alpha, alpha, alpha + 1]), 60, dnum)


def draw(rng):
    op = rng.choice(["rope", "rope", "step", "chunk"])
    logN = rng.choice([12, 13, 14, 15, 16])
    if op == "rope":
        s = _draw_shape(rng, logN, 24)
        head = rng.choice([8, 16, 32, 64, 128])
        npt = rng.choice([1, 1, 2, 3])
        return dict(op=op, layout=rng.choice(["half", "interleaved"]), head=head, rot=rng.choice([head, head, head // 2]),
                    lanes=rng.choice(["inner", "outer"]), scaling=rng.choice([1.0, 1.0, 4.0, 7.5]), npt=npt,
                    nlimbs=rng.randint((s["nq"] + 1) // 2, s["nq"]),
                    batch=npt * _log_int(rng, 1, max(1, (1 << 20) // (s["nq"] << logN) if logN < 16 else 2)), **s)
    s = _draw_shape(rng, logN, 10)
    most = {12: 16, 13: 16, 14: 16, 15: 8, 16: 4}[logN]
    n1 = rng.choice([1, 2, 3, 4, 5, 8])
    n2 = rng.randint(1, max(1, most // n1))
    c = dict(op=op, n1=n1, n2=n2, state=rng.random() < .7, decay=rng.random() < .5, nlimbs=rng.randint((s["nq"] + 1) // 2, s["nq"]),
             batch=rng.randint(1, 3 if logN < 15 else 1), **s)
    if op == "chunk":
        c["tokens"] = rng.randint(1, 5 if logN < 15 else 3)
    return c


# ---- parameters: primes = 1 mod 2N downwards from 2^bits, and a primitive 2N-th root of unity for each ----
def _is_prime(n):
    d, r = n - 1, 0
    while d % 2 == 0:
        d, r = d // 2, r + 1
    for b in (2, 3, 5, 7, 11, 13, 17, 19, 23, 29, 31, 37):
        if n % b == 0:
            return n == b
        x = pow(b, d, n)
        if x in (1, n - 1):
            continue
        for _ in range(r - 1):
            x = x * x % n
            if x == n - 1:
                break
        else:
            return False
    return True


def _primes(bits, count, two_n, taken=()):
    out, q = [], ((1 << bits) - 1) // two_n * two_n + 1
    while len(out) < count:
        if q not in taken and _is_prime(q):
            out.append(q)
        q -= two_n
    return out


def _root(q, two_n):
    g = 2
    while pow(g, (q - 1) // 2, q) != q - 1:
        g += 1
    return pow(g, (q - 1) // two_n, q)


_SHAPE = ("logN", "nq", "q_bits", "np", "p_bits", "dnum")
_params = {}


def _parameters(case):
    key = tuple(case[k] for k in _SHAPE)
    if key not in _params:
        logN, nq, q_bits, np_, p_bits, dnum = key
        two_n = 2 << logN
        q = _primes(q_bits, nq, two_n)
        p = _primes(p_bits, np_, two_n, q)
        _params[key] = SimpleNamespace(logN=logN, q=q, p=p, moduli=q + p, dnum=dnum, psi=[_root(m, two_n) for m in q + p])
    return _params[key]


def _bitrev(bits):
    r = np.zeros(1 << bits, dtype=np.int64)
    for k in range(bits):
        r[1 << k:2 << k] = r[:1 << k] + (1 << (bits - 1 - k))
    return r


def _element(step, logN):
    return pow(5, step % (1 << (logN - 1)), 2 << logN)


# ---- residues in torch: products modulo primes below 2^60 in 64-bit words ----
class _Moduli:
    """Moduli along the last dimension but one of a residue tensor (the last but two with `wide`: butterflies split the last)."""

    def __init__(self, moduli, wide=False):
        self.list = list(moduli)
        self.narrow = max(moduli) < 1 << 50
        self.v = torch.tensor(moduli, dtype=torch.int64, device=DEVICE).reshape((-1, 1, 1) if wide else (-1, 1))
        self.d = self.v.double()

    def const(self, values):
        return torch.tensor(values, dtype=torch.int64, device=DEVICE)[:, None]


def _product(a, b, m):
    """a * b mod m for a < m < 2^60 and b <= 2^30, or for a, b < m < 2^50: the quotient is below 2^50 and its estimate in doubles
    at most 1 off, so the difference of the two wrapped products is the remainder give or take m."""
    r = a * b - (a.double() * (b.double() / m.d)).long() * m.v
    r = torch.where(r < 0, r + m.v, r)
    return torch.where(r >= m.v, r - m.v, r)


def _mulmod(a, b, m):
    if m.narrow:
        return _product(a, b, m)
    high = _product(a, b >> 30, m)
    high = _product(high, torch.full_like(high, 1 << 30), m)
    return _addmod(high, _product(a, b & ((1 << 30) - 1), m), m)


def _addmod(a, b, m):
    r = a + b
    return torch.where(r >= m.v, r - m.v, r)


def _submod(a, b, m):
    r = a - b
    return torch.where(r < 0, r + m.v, r)


class _Basis:
    """A group of primes with its transforms. Evaluation order: index k holds the value at psi^(2 bitrev(k) + 1)."""

    def __init__(self, moduli, psi, logN):
        self.logN, N = logN, 1 << logN
        self.m, self.wide = _Moduli(moduli), _Moduli(moduli, wide=True)
        order = torch.from_numpy(_bitrev(logN)).to(DEVICE)
        self.fwd, self.inv = [self._powers(r, N)[:, order] for r in (psi, [pow(w, -1, q) for w, q in zip(psi, moduli)])]
        self.n_inv = self.m.const([pow(N, -1, q) for q in moduli])

    def _powers(self, roots, N):
        x = torch.ones((len(roots), 1), dtype=torch.int64, device=DEVICE)
        while x.shape[1] < N:
            w = self.m.const([pow(r, x.shape[1], q) for r, q in zip(roots, self.m.list)])
            x = torch.cat((x, _mulmod(x, w, self.m)), dim=1)
        return x

    def ntt(self, x):
        shape, m = x.shape, self.wide
        for s in range(self.logN):
            h = 1 << s
            x = x.reshape(*shape[:-1], h, 2, -1)
            u, v = x[..., 0, :], _mulmod(x[..., 1, :], self.fwd[:, h:2 * h, None], m)
            x = torch.stack((_addmod(u, v, m), _submod(u, v, m)), dim=-2)
        return x.reshape(shape)

    def intt(self, x):
        shape, m = x.shape, self.wide
        for s in reversed(range(self.logN)):
            h = 1 << s
            x = x.reshape(*shape[:-1], h, 2, -1)
            u, v = x[..., 0, :], x[..., 1, :]
            x = torch.stack((_addmod(u, v, m), _mulmod(_submod(u, v, m), self.inv[:, h:2 * h, None], m)), dim=-2)
        return _mulmod(x.reshape(shape), self.n_inv, self.m)


class _Plain:
    """Tables of one parameter set for the plain forms."""

    def __init__(self, p):
        self.p, self.N, self.K, self.nq = p, 1 << p.logN, len(p.p), len(p.q)
        self.alpha = -(-self.nq // p.dnum)
        self.main = _Basis(p.q, p.psi[:self.nq], p.logN)
        self.special = _Basis(p.p, p.psi[self.nq:], p.logN)
        self._parts, self._maps = {}, {}

    def part(self, ids):
        """The basis of some of the main primes."""
        if ids not in self._parts:
            b = _Basis.__new__(_Basis)
            moduli, i = [self.p.q[k] for k in ids], list(ids)
            b.logN, b.m, b.wide = self.p.logN, _Moduli(moduli), _Moduli(moduli, wide=True)
            b.fwd, b.inv, b.n_inv = self.main.fwd[i], self.main.inv[i], self.main.n_inv[i]
            self._parts[ids] = b
        return self._parts[ids]

    def limbs(self, n):
        return self.part(tuple(range(n)))

    def sigma(self, x, g):
        """The Galois map X -> X^g, evaluation domain: value k of the result is the value of x at psi^(g (2 bitrev(k) + 1))."""
        if g == 1:
            return x
        if g not in self._maps:
            br = _bitrev(self.p.logN)
            self._maps[g] = torch.from_numpy(br[(g * (2 * br + 1) % (2 * self.N) - 1) // 2]).to(DEVICE)
        return x[..., self._maps[g]]


def _convert(x, src, dst):
    """sum_i y_i (C / c_i) mod every target, y_i = [x_i (C / c_i)^-1] centred; x is in coefficient form."""
    C = math.prod(src.list)
    y = _mulmod(x, src.const([pow(C // c, -1, c) for c in src.list]), src)
    y = torch.where(y > src.v // 2, y - src.v, y)
    out = None
    for i, c in enumerate(src.list):
        t = _mulmod(torch.remainder(y[..., i:i + 1, :], dst.v), dst.const([C // c % t for t in dst.list]), dst)
        out = t if out is None else _addmod(out, t, dst)
    return out


def _digits(R, d):
    """The digits of d [.., nl, N] in the extended basis: (first digit limb, values on the main primes, on the special ones)."""
    nl = d.shape[-2]
    every = R.limbs(nl)
    coef = every.intt(d)
    out = []
    for lo in range(0, nl, R.alpha):
        own_ids = tuple(range(lo, min(nl, lo + R.alpha)))
        others = tuple(i for i in range(nl) if i not in own_ids)
        src, x = R.part(own_ids).m, coef[..., list(own_ids), :]
        main = d.clone()
        if others:
            main[..., list(others), :] = R.part(others).ntt(_convert(x, src, R.part(others).m))
        out.append((main, R.special.ntt(_convert(x, src, R.special.m))))
    return out


def _accumulate(R, digits, key, g=1, total=None):
    """A(sigma_g(d); key) from the digits of d (the map commutes with the centred conversion), added to `total` if given: a pair
    of tensors [.., 2, nl, N] and [.., 2, K, N]."""
    nl = digits[0][0].shape[-2]
    m, k = R.limbs(nl).m, R.special.m
    for j, (main, special) in enumerate(digits):
        a = _mulmod(R.sigma(main, g)[..., None, :, :], key[j, :, :nl], m)
        b = _mulmod(R.sigma(special, g)[..., None, :, :], key[j, :, R.nq:], k)
        total = (a, b) if total is None else (_addmod(total[0], a, m), _addmod(total[1], b, k))
    return total


def _times_P(R, x):
    m = R.limbs(x.shape[-2]).m
    P = math.prod(R.p.p)
    return _mulmod(x, m.const([P % q for q in m.list]), m)


def _add_main(R, acc, x, component=None):
    """acc plus P x on the main primes, of both components or of one."""
    a, m = acc[0], R.limbs(x.shape[-2]).m
    if component is None:
        return _addmod(a, _times_P(R, x), m), acc[1]
    a = a.clone()
    a[..., component, :, :] = _addmod(a[..., component, :, :], _times_P(R, x), m)
    return a, acc[1]


def _mod_down(R, acc):
    main, special = acc
    b = R.limbs(main.shape[-2])
    t = b.ntt(_convert(R.special.intt(special), R.special.m, b.m))
    P = math.prod(R.p.p)
    return _mulmod(_submod(main, t, b.m), b.m.const([pow(P, -1, q) for q in b.m.list]), b.m)


def _rotated(R, ct, digits, g, key):
    """The extended-basis form of the rotation of ct."""
    return _add_main(R, _accumulate(R, digits, key, g), R.sigma(ct[..., 0, :, :], g), 0)


def _stack(accs):
    return tuple(torch.stack(x) for x in zip(*accs))


def _add_acc(R, x, y):
    return _addmod(x[0], y[0], R.limbs(x[0].shape[-2]).m), _addmod(x[1], y[1], R.special.m)


def _rotations(R, ct, elements, keys):
    """ct and its rotations, [len(elements) + 1][..]."""
    if not elements:
        return ct[None]
    digits = _digits(R, ct[..., 1, :, :])
    return torch.cat((ct[None], _mod_down(R, _stack([_rotated(R, ct, digits, g, k) for g, k in zip(elements, keys)]))))


def _sum_of_rotations(R, ct, elements, keys):
    if not elements:
        return ct
    digits, total = _digits(R, ct[..., 1, :, :]), None
    for g, key in zip(elements, keys):
        x = _rotated(R, ct, digits, g, key)
        total = x if total is None else _add_acc(R, total, x)
    return _mod_down(R, _add_main(R, total, ct))


def _tensor(R, a, b):
    """The product of ciphertexts in three components."""
    m = R.limbs(a.shape[-2]).m
    a0, a1, b0, b1 = a[..., 0, :, :], a[..., 1, :, :], b[..., 0, :, :], b[..., 1, :, :]
    mid = _addmod(_mulmod(a0, b1, m), _mulmod(a1, b0, m), m)
    return torch.stack((_mulmod(a0, b0, m), mid, _mulmod(a1, b1, m)), dim=-3)


def _sum_tensor(R, pairs, acc=None):
    for a, b in pairs:
        t = _tensor(R, a, b)
        acc = t if acc is None else _addmod(acc, t, R.limbs(a.shape[-2]).m)
    return acc


def _relin_accumulators(R, d, key):
    return _add_main(R, _accumulate(R, _digits(R, d[..., 2, :, :]), key), d[..., :2, :, :])


def _relin(R, d, key):
    return _mod_down(R, _relin_accumulators(R, d, key))


def _read(R, s, q, state, extra):
    """read(q, state, extra) of the module's text for every token: q [C][B][2][nl][N], state [n2][n1][B][2][nl][N] or None."""
    if state is None:
        return _relin(R, extra, s["mult_key"])
    Q = _rotations(R, q, s["baby"], s["baby_keys"])
    total = _relin_accumulators(R, _sum_tensor(R, zip(Q, state[0]), extra), s["mult_key"])
    for g in range(1, s["n2"]):
        y = _relin(R, _sum_tensor(R, zip(Q, state[g])), s["mult_key"])
        x = _rotated(R, y, _digits(R, y[..., 1, :, :]), s["giant"][g - 1], s["giant_keys"][g - 1])
        total = _add_acc(R, total, x)
    return _mod_down(R, total)


def _updated(R, s, k, v, state):
    """state + Relin(sum_s K_s[b] * V_s[g]); k, v [C][B][2][nl][N]."""
    K = _rotations(R, k, s["baby"], s["baby_keys"])
    V = _rotations(R, v, s["value"], s["value_keys"])
    d = torch.stack([torch.stack([_sum_tensor(R, zip(K[b], V[g])) for b in range(s["n1"])]) for g in range(s["n2"])])
    rows = torch.stack([_relin(R, row, s["mult_key"]) for row in d]) if d.numel() > 1 << 25 else _relin(R, d, s["mult_key"])
    return rows if state is None else _addmod(rows, state, R.limbs(k.shape[-2]).m)


def _decayed(R, state, decay):
    return state if decay is None else _mulmod(state, decay, R.limbs(state.shape[-2]).m)


def _plain_run(s):
    R, op = s["plain"], s["op"]
    if op == "rope":
        ct, w, nl = s["ct"], s["weights"], s["nl"]
        m, k = R.limbs(nl).m, R.special.m
        w = w.repeat_interleave(ct.shape[0] // w.shape[0], dim=0)[:, :, None]    # [B][R + 1][1][nl + K][N]
        digits, total = _digits(R, ct[:, 1]), None
        for r, (g, key) in enumerate(zip(s["elements"], s["keys"])):
            x, y = _rotated(R, ct, digits, g, key)
            x = _mulmod(x, w[:, r + 1, :, :nl], m), _mulmod(y, w[:, r + 1, :, nl:], k)
            total = x if total is None else _add_acc(R, total, x)
        return _mod_down(R, _add_main(R, total, _mulmod(ct, w[:, 0, :, :nl], m)))
    q, k, v = s["q"], s["k"], s["v"]
    if op == "step":
        M = _updated(R, s, k, v, s["state"])
        return dict(o=_read(R, s, q, M, None)[0], state=_decayed(R, M, s["decay"]))
    pairs = [(t, u) for t in range(q.shape[0]) for u in range(t + 1)]
    p = _relin(R, _tensor(R, q[[t for t, _ in pairs]], k[[u for _, u in pairs]]), s["mult_key"])
    p = _sum_of_rotations(R, _sum_of_rotations(R, p, s["baby"], s["baby_keys"]), s["giant"], s["giant_keys"])
    scored = torch.stack([_sum_tensor(R, [(p[i], v[u]) for i, (t, u) in enumerate(pairs) if t == tok])
                          for tok in range(q.shape[0])])
    return dict(o=_read(R, s, q, s["state"], scored), state=_decayed(R, _updated(R, s, k, v, s["state"]), s["decay"]))


# ---- the framework's calls ----
def _own_run(s):
    import paper_2604_03425_amd as ck
    ctx, op, nl = s["ctx"], s["op"], s["nl"]
    if op == "rope":
        ck.ckks_rope(ctx, s["out"], s["ct"], s["ct"].shape[0], nl, s["weights"], s["weights"].shape[0], s["elements"], s["keys"],
                     s["ws"])
        return s["out"]
    keys = (s["n1"], s["n2"], s["stride"], s["mult_key"], s["baby_keys"], s["giant_keys"], s["value_keys"], s["ws"])
    if op == "step":
        ck.ckks_linattn_step(ctx, s["out"], s["state_out"], s["q"], s["k"], s["v"], s["state"], s["decay"], s["B"], nl, *keys)
        return dict(o=s["out"][0], state=s["state_out"])
    ck.ckks_linattn_chunk(ctx, s["out"], s["state_out"], s["q"], s["k"], s["v"], s["state"], s["decay"], s["q"].shape[0], s["B"],
                          nl, *keys)
    return dict(o=s["out"], state=s["state_out"])


def run(state):
    return _own_run(state) if own else _plain_run(state)


# ---- what a program has in hand before the call ----
_plans = OrderedDict()   # contexts or plain tables of the most recent parameter sets, as a program keeps its context


def _plan(case, kind, make):
    key = (kind,) + tuple(case[k] for k in _SHAPE)
    if key not in _plans:
        while len(_plans) >= 4:
            _plans.popitem(last=False)
        _plans[key] = make(_parameters(case))
    _plans.move_to_end(key)
    return _plans[key]


def _rotary_slots(case, first):
    """(steps, weights [npt][steps + 1][N / 2]) of a rotary embedding. The head's first `rot` components turn in pairs by the
    angle position / scaling * 10000^(-2 i / rot): component i with i + rot/2 ("half") or 2i with 2i + 1 ("interleaved").
    lanes "inner": slot component * (slots / head) + lane, a position for every lane (one new token of many sequences); "outer":
    slot token * head + component (a prompt). `first` is the position of the first lane or token of each set."""
    S, head, rot = 1 << (case["logN"] - 1), case["head"], case["rot"]
    T = S // head
    lane = np.arange(T)
    h = rot // 2
    freq = 10000.0 ** (-2.0 * np.arange(h) / rot)
    half = case["layout"] == "half"
    low, high = (np.arange(h), np.arange(h) + h) if half else (2 * np.arange(h), 2 * np.arange(h) + 1)
    width = T if case["lanes"] == "inner" else 1                 # slots between two components of a token
    step = (h if half else 1) * width
    cyclic = half and rot == head and width > 1                  # the partner lies half of all slots away, both ways
    steps = [step] if cyclic else [step, -step]
    w = np.zeros((len(first), len(steps) + 1, T, head))
    for i, f in enumerate(first):
        pos = f + (lane * 37 % 1024 if case["lanes"] == "inner" else lane)
        angle = pos[:, None] / case["scaling"] * freq
        w[i, 0, :, rot:] = 1.0
        w[i, 0][:, low] = w[i, 0][:, high] = np.cos(angle)
        w[i, 1][:, low] = -np.sin(angle)                         # the partner of a low component lies `step` to the right
        w[i, 1 if cyclic else 2][:, high] = np.sin(angle)
    if case["lanes"] == "inner":
        w = w.transpose(0, 1, 3, 2)
    return steps, w.reshape(len(first), len(steps) + 1, S)


def _encode(slots, logN, bits=40):
    """Coefficients (rounded, int64) of the real polynomials whose values at zeta^(5^i) are the slots times 2^bits."""
    N = 1 << logN
    e = np.empty(N // 2, dtype=np.int64)
    x = 1
    for i in range(N // 2):
        e[i], x = x, x * 5 % (2 * N)
    v = torch.zeros((slots.shape[0], N), dtype=torch.complex128, device=DEVICE)
    z = torch.from_numpy(slots).to(DEVICE).to(torch.complex128)
    v[:, torch.from_numpy((e - 1) // 2).to(DEVICE)] = z
    v[:, torch.from_numpy((2 * N - e - 1) // 2).to(DEVICE)] = z
    j = torch.arange(N, dtype=torch.float64, device=DEVICE) * (-math.pi / N)
    c = torch.fft.fft(v) / N * torch.polar(torch.ones_like(j), j)
    return torch.round(c.real * 2.0 ** bits).long()


class _Inputs:
    """Seeded uniform residues on the GPU: ciphertexts, keys and encoded plaintexts are uniform modulo every prime."""

    def __init__(self, seed):
        self.gen = torch.Generator(device=DEVICE).manual_seed(int(seed))

    def residues(self, lead, moduli, N):
        x = torch.empty(tuple(lead) + (len(moduli), N), dtype=torch.int64, device=DEVICE)
        for i, m in enumerate(moduli):
            x[..., i, :].random_(0, m, generator=self.gen)
        return x


def prepare(case, seed):
    p, op, B, nl = _parameters(case), case["op"], case["batch"], case["nlimbs"]
    N, rnd = 1 << p.logN, _Inputs(seed)
    s = dict(op=op, nl=nl, B=B)

    def keys(count):
        return [rnd.residues((p.dnum, 2), p.moduli, N) for _ in range(count)]

    if op == "rope":
        plain = _plan(case, "plain", _Plain)                     # its transforms encode the weights
        position = np.random.default_rng(seed).integers(0, 4096, size=case["npt"])
        steps, slots = _rotary_slots(case, position.tolist())
        coef = _encode(slots.reshape(-1, N // 2), p.logN)[:, None]
        w = torch.cat([b.ntt(torch.remainder(coef, b.m.v)) for b in (plain.limbs(nl), plain.special)], dim=-2)
        s.update(ct=rnd.residues((B, 2), p.q[:nl], N), weights=w.reshape(case["npt"], len(steps) + 1, nl + len(p.p), N).contiguous(),
                 elements=[_element(r, p.logN) for r in steps], keys=keys(len(steps)))
    else:
        n1, n2, C = case["n1"], case["n2"], case.get("tokens", 1)
        stride = max(1, (N // 2) // (n1 * n2))
        for name in ("q", "k", "v"):
            s[name] = rnd.residues((C, B, 2), p.q[:nl], N)
        s.update(n1=n1, n2=n2, stride=stride, mult_key=keys(1)[0],
                 baby=[_element(b * stride, p.logN) for b in range(1, n1)], baby_keys=keys(n1 - 1),
                 giant=[_element(g * n1 * stride, p.logN) for g in range(1, n2)], giant_keys=keys(n2 - 1),
                 value=[_element(-g * n1 * stride, p.logN) for g in range(1, n2)], value_keys=keys(n2 - 1),
                 state=rnd.residues((n2, n1, B, 2), p.q[:nl], N) if case["state"] else None,
                 decay=rnd.residues((), p.q[:nl], N) if case["decay"] else None)
    if not own:
        s["plain"] = _plan(case, "plain", _Plain)
        return s
    import paper_2604_03425_amd as ck
    ctx = s["ctx"] = _plan(case, "own", lambda params: ck.Context(params, 0))
    if op == "rope":
        s.update(out=torch.empty_like(s["ct"]), ws=ctx.workspace(ck.OP_ROPE, B, nl))
    else:
        C = s["q"].shape[0]
        s.update(out=torch.empty_like(s["q"]), state_out=torch.empty((n2, n1, B, 2, nl, N), dtype=torch.int64, device=DEVICE),
                 ws=ctx.linattn_workspace(ck.OP_LINATTN_STEP if op == "step" else ck.OP_LINATTN_CHUNK, C, B, nl, n1, n2))
    return s


# ---- what a pass cannot do without ----
def work(case):
    """bytes: every input read once, every output written once. flops: 2 for each modular product and its addition, in the
    transforms (a product a butterfly), the base conversions, the products with keys and weights, and the tensor products."""
    N, nl, K, B, op = 1 << case["logN"], case["nlimbs"], case["np"], case["batch"], case["op"]
    alpha = -(-case["nq"] // case["dnum"])
    beta, ext = -(-nl // alpha), nl + K
    poly = 8 * N
    ntt = case["logN"] / 2 + 1
    front = nl * ntt + sum(min(alpha, nl - j * alpha) * (ext - min(alpha, nl - j * alpha)) for j in range(beta)) \
        + (beta * ext - nl) * ntt                                # digits of one polynomial, per coefficient
    inner = 2 * beta * ext                                       # their products with a key
    down = 2 * (K * ntt + K * nl + nl * ntt + nl)                # ModDown of both accumulators
    key = 2 * beta * ext
    ct = 2 * nl
    if op == "rope":
        R = 1 if case["layout"] == "half" and case["rot"] == case["head"] and case["lanes"] == "inner" else 2
        moved = 2 * B * ct + case["npt"] * (nl + R * ext) + R * key
        done = B * (front + R * (inner + 2 * ext) + ct + down)
    else:
        n1, n2, C = case["n1"], case["n2"], case.get("tokens", 1)
        d = n1 * n2
        state = case["state"]
        read = op == "step" or state
        moved = B * ct * (4 * C + d * (2 if state else 1)) + key * (1 + n1 - 1 + 2 * (n2 - 1)) + (nl if case["decay"] else 0)
        rotations = (front if n1 > 1 else 0) + (n1 - 1) * (inner + down)
        values = (front if n2 > 1 else 0) + (n2 - 1) * (inner + down)
        update = C * (rotations + values + 4 * d * nl) + d * (front + inner + down)
        reading = C * (rotations + 4 * d * nl + n2 * (front + inner) + (n2 - 1) * (down + front + inner) + down) if read else \
            C * (front + inner + down)
        score = 4 * nl + front + inner + down + sum(front + (n - 1) * inner + down for n in (n1, n2) if n > 1) + 4 * nl
        pairs = C * (C + 1) // 2 if op == "chunk" else 0
        done = B * (update + reading + pairs * score + (d * ct if case["decay"] else 0))
    return {"bytes": int(poly * moved), "flops": int(2 * N * done)}


# ---- the definitions once more, in Python's integers, for the smallest rings ----
def exact(case, seed):
    """The rotary operator on rings up to 2^12 by the definitions: coefficients by evaluating at the roots of unity, one big
    integer for each conversion. None for the rest, whose outputs are whole numbers that have to be equal anyway."""
    if case["op"] != "rope" or case["logN"] > 12 or case["batch"] * (case["nlimbs"] + case["np"]) > 40:
        return None
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    p, nl, N = _parameters(case), case["nlimbs"], 1 << case["logN"]
    host = {k: s[k].cpu().numpy().astype(object) for k in ("ct", "weights")}
    keys = [k.cpu().numpy().astype(object) for k in s["keys"]]
    mods, K, P = p.q[:nl] + p.p, len(p.p), math.prod(p.p)
    alpha, br = -(-len(p.q) // p.dnum), _bitrev(p.logN)
    roots = p.psi[:nl] + p.psi[len(p.q):]

    def cyclic(a, w, q):
        """sum_j a_j w^(jk) for every k."""
        n = len(a)
        if n == 1:
            return a
        even, odd = cyclic(a[::2], w * w % q, q), cyclic(a[1::2], w * w % q, q)
        tw = np.array([1] * (n // 2), dtype=object)
        for k in range(1, n // 2):
            tw[k] = tw[k - 1] * w % q
        odd = odd * tw % q
        return np.concatenate(((even + odd) % q, (even - odd) % q))

    def powers(w, q):
        out = [1] * N
        for k in range(1, N):
            out[k] = out[k - 1] * w % q
        return np.array(out, dtype=object)

    def values(a, t):
        q, w = mods[t], roots[t]
        return cyclic(a % q * powers(w, q) % q, w * w % q, q)[br]

    def coefficients(x, t):
        q, w = mods[t], roots[t]
        y = np.empty_like(x)
        y[br] = x
        a = cyclic(y, pow(w, -2, q), q) * pow(N, -1, q) % q
        return a * powers(pow(w, -1, q), q) % q

    def centred(parts, ids):
        """The integer sum_i y_i (C / c_i) of every coefficient."""
        C = math.prod(mods[i] for i in ids)
        total = 0
        for x, i in zip(parts, ids):
            c = mods[i]
            y = x * pow(C // c, -1, c) % c
            total = total + np.where(y > c // 2, y - c, y) * (C // c)
        return total

    e = np.array([(2 * int(b) + 1) for b in br], dtype=object)
    out = np.empty(host["ct"].shape, dtype=np.int64)
    for b in range(case["batch"]):
        c0, c1 = host["ct"][b]
        w = host["weights"][b // (case["batch"] // case["npt"])]
        T = [[c[t] * P % mods[t] * w[0][t] % mods[t] if t < nl else 0 * c[0] for t in range(nl + K)] for c in (c0, c1)]
        for r, g in enumerate(s["elements"]):
            at = br[np.array((e * g % (2 * N) - 1) // 2, dtype=np.int64)]
            turned = [c1[t][at] for t in range(nl)]
            coef = [coefficients(turned[t], t) for t in range(nl)]
            for j, lo in enumerate(range(0, nl, alpha)):
                ids = list(range(lo, min(nl, lo + alpha)))
                whole = centred([coef[i] for i in ids], ids)
                for t in range(nl + K):
                    x = turned[t] if t in ids else values(whole, t)
                    row = t if t < nl else len(p.q) + t - nl
                    for c in (0, 1):
                        T[c][t] = (T[c][t] + x * keys[r][j][c][row] % mods[t] * w[r + 1][t]) % mods[t]
            for t in range(nl):
                T[0][t] = (T[0][t] + c0[t][at] * P % mods[t] * w[r + 1][t]) % mods[t]
        for c in (0, 1):
            ids = list(range(nl, nl + K))
            low = centred([coefficients(T[c][t], t) for t in ids], ids)
            for t in range(nl):
                q = mods[t]
                out[b, c, t] = np.array((T[c][t] - values(low, t)) * pow(P, -1, q) % q, dtype=np.int64)
    return out
