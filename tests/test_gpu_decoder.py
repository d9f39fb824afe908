"""Attention over a paged cache and the root-mean-square norm on the GPU against the oracle, residue for residue: every ring and
arithmetic kind, ragged sequences, pages that end inside windows and chunks, windows and sinks, levels below the top."""
import numpy as np
import pytest
import torch

import attention_ref
import decoder_ref
from ckks_inputs import CkksParams, find_ntt_primes, find_psi, make_params
from gpu_util import assert_same, to_dev, to_host
from oracle import ref

pytestmark = pytest.mark.gpu


def _mixed(logN):
    """Main primes of all three kinds (below 2^50, below 2^52, 60 bits) and special primes of two."""
    q = find_ntt_primes(49, 2, logN) + find_ntt_primes(51, 2, logN) + find_ntt_primes(60, 1, logN)
    p = find_ntt_primes(59, 2, logN) + find_ntt_primes(45, 1, logN)
    return CkksParams(logN=logN, q=q, p=p, dnum=2, psi=[find_psi(m, logN) for m in q + p])


PARAMS = {
    "ring10": lambda: make_params(10, 6, 50, 2, 60, 3),
    "ring11": lambda: make_params(11, 4, 60, 1, 60, 4),
    "ring12": lambda: make_params(12, 5, 45, 2, 60, 3),
    "ring12_wide": lambda: make_params(12, 12, 50, 12, 60, 1),
    "ring13": lambda: make_params(13, 5, 50, 2, 60, 3),
    "ring13_int": lambda: make_params(13, 5, 60, 2, 60, 3),
    "ring13_mixed": lambda: _mixed(13),
    "ring13_fp": lambda: make_params(13, 5, 45, 2, 48, 3),        # special primes in double precision too
    "ring14": lambda: make_params(14, 7, 50, 3, 60, 3),
    "ring14_wide": lambda: make_params(14, 10, 50, 10, 60, 1),    # conversions of more than 8 sources
    "ring14_eight": lambda: make_params(14, 8, 50, 8, 60, 1),     # 8 special primes and a main one: 9 sources
    "ring15": lambda: make_params(15, 5, 55, 3, 60, 2),
    "ring16": lambda: make_params(16, 5, 50, 2, 60, 3),
    "ring17": lambda: make_params(17, 4, 50, 1, 60, 4),
}
_contexts = {}


def contexts(name):
    import paper_2604_03425_amd as ck
    if name not in _contexts:
        p = PARAMS[name]()
        ref.set_threads(8)
        _contexts[name] = (p, ref.RefContext(p), ck.Context(p, 0))
    return _contexts[name]


def device_keys(s):
    return to_dev(s.mult_key), [to_dev(x) for x in s.baby_keys], [to_dev(x) for x in s.giant_keys]


class Cache:
    """Pages of a cache that holds the tokens before the new ones; everything else in them is -1."""

    def __init__(self, lens, new, page, k_limbs, v_limbs, N, keys, values):
        counts = [-(-n // page) for n in lens]
        self.k = torch.full((sum(counts), page, 2, k_limbs, N), -1, dtype=torch.int64, device="cuda")
        self.v = torch.full((sum(counts), page, 2, v_limbs, N), -1, dtype=torch.int64, device="cuda")
        order = np.random.default_rng(sum(lens)).permutation(sum(counts)).tolist()
        self.table = [[order.pop() for _ in range(c)] for c in counts]
        self.page = page
        for b, (n, m) in enumerate(zip(lens, new)):
            for t in range(n - m):
                self.put(b, t, keys[b][t], values[b][t])
        flat = [x for row in self.table for x in row]
        self.args = ([self.k[i] for i in flat], [self.v[i] for i in flat], page, k_limbs, v_limbs)

    def put(self, b, t, k, v):
        at = self.table[b][t // self.page], t % self.page
        self.k[at], self.v[at] = to_dev(k[:, :self.k.shape[-2]]), to_dev(v[:, :self.v.shape[-2]])


def run_attention(name, nl, lens, new, page, window, sinks, squarings, n1, n2, k_extra=0, v_extra=0, bias=12345678901234567):
    import paper_2604_03425_amd as ck
    p, rc, ctx = contexts(name)
    stride = max(1, (p.N // 2) // (n1 * n2))
    s = attention_ref.Shape(p, rc, n1, n2, stride, seed=sum(lens) + 7 * nl)
    L = nl - 1 - squarings
    kl, vl = nl + k_extra, L + v_extra
    both, rows = max(kl, vl), sum(new)
    keys, values = ([s.cts((n,), both) for n in lens] for _ in range(2))
    q = s.cts((rows,), nl)
    want = decoder_ref.attention(s, q, keys, values, new, window, sinks, bias, squarings)
    cache = Cache(lens, new, page, kl, vl, p.N, keys, values)
    full = Cache(lens, [0] * len(lens), page, kl, vl, p.N, keys, values)
    fresh = [to_dev(np.concatenate([x[n - m:n] for x, n, m in zip(xs, lens, new)])) for xs in (keys, values)]
    ck.ckks_kv_append(ctx, *fresh, both, new, lens, *cache.args)
    assert torch.equal(cache.k, full.k) and torch.equal(cache.v, full.v)      # and nothing else was written
    ws = ctx.attn_workspace(rows, ck.attn_pairs(new, lens, window, sinks), nl, n1, n2, squarings).random_()
    out = torch.full((rows + 1, 2, L, p.N), -1, dtype=torch.int64, device="cuda")
    ck.ckks_attn_paged(ctx, out, to_dev(q), nl, new, lens, *cache.args, window, sinks, bias, squarings, n1, n2, stride, *device_keys(s), ws)
    assert_same(to_host(out[:rows]), want, "attention %s" % name)
    assert (out[rows] == -1).all()
    assert torch.equal(cache.k, full.k) and torch.equal(cache.v, full.v)


@pytest.mark.parametrize("name,nl,lens,new,page,window,sinks,squarings,n1,n2,k_extra,v_extra", [
    ("ring10", 6, (1,), (1,), 1, 0, 0, 0, 1, 1, 0, 0),            # one token that sees itself, one component
    ("ring10", 2, (3, 1), (3, 1), 2, 0, 0, 0, 2, 1, 3, 4),        # one limb left
    ("ring10", 5, (9, 0, 4), (2, 0, 0), 4, 3, 2, 3, 1, 3, 1, 0),  # an empty sequence, one with nothing new; three squarings
    ("ring10", 4, (7,), (3,), 3, 1, 0, 1, 2, 2, 0, 1),            # a window of the token itself
    ("ring10", 4, (7,), (2,), 3, 2, 9, 0, 2, 2, 0, 0),            # more sinks than tokens
    ("ring11", 4, (5, 2), (1, 1), 2, 0, 0, 1, 2, 2, 0, 0),
    ("ring12", 5, (4, 6), (1, 2), 3, 2, 1, 1, 2, 2, 0, 0),
    ("ring12_wide", 11, (3,), (2,), 8, 0, 0, 1, 2, 1, 1, 0),
    ("ring13", 5, (6,), (2,), 5, 0, 0, 0, 3, 2, 0, 1),
    ("ring13", 4, (5, 3), (1, 2), 2, 2, 1, 2, 2, 2, 1, 0),
    ("ring13_int", 5, (4,), (2,), 3, 0, 0, 1, 2, 2, 0, 0),
    ("ring13_int", 3, (3,), (1,), 3, 0, 0, 0, 1, 2, 2, 1),
    ("ring13_mixed", 5, (4, 2), (1, 1), 2, 0, 0, 2, 2, 2, 0, 0),
    ("ring13_mixed", 3, (4,), (2,), 4, 2, 0, 0, 2, 1, 1, 0),
    ("ring13_fp", 5, (4,), (2,), 2, 0, 0, 1, 2, 2, 0, 0),
    ("ring14", 7, (5,), (2,), 2, 0, 0, 2, 2, 2, 0, 0),
    ("ring14", 4, (6, 3), (1, 1), 4, 2, 1, 1, 1, 4, 2, 1),
    ("ring14_wide", 10, (3,), (1,), 2, 0, 0, 1, 2, 2, 0, 0),
    ("ring14_eight", 7, (3,), (2,), 2, 0, 0, 1, 2, 1, 0, 0),
    ("ring15", 5, (3,), (1,), 2, 0, 0, 1, 2, 2, 0, 0),
    ("ring16", 5, (3,), (2,), 2, 0, 0, 1, 2, 2, 0, 0),
    ("ring17", 4, (2,), (1,), 2, 0, 0, 1, 2, 1, 0, 0),
])
def test_attention_matches_the_oracle(name, nl, lens, new, page, window, sinks, squarings, n1, n2, k_extra, v_extra):
    run_attention(name, nl, lens, new, page, window, sinks, squarings, n1, n2, k_extra, v_extra)


@pytest.mark.parametrize("bias", [0, 1, -1, (1 << 62), -(1 << 62), -(1 << 63), (1 << 63) - 1])
def test_any_bias(bias):
    run_attention("ring10", 4, (2,), (1,), 2, 0, 0, 1, 1, 2, bias=bias)
    run_attention("ring11", 3, (2,), (1,), 2, 0, 0, 0, 1, 2, bias=bias)


def run_norm(name, nl, B, n1, n2, iterations, res, gain, numbers=None, in_place=False, check=None):
    import paper_2604_03425_amd as ck
    p, rc, ctx = contexts(name)
    stride = max(1, (p.N // 2) // (n1 * n2))
    s = attention_ref.Shape(p, rc, n1, n2, stride, seed=nl + 31 * B)
    L = nl - 1 - 2 * iterations
    rng = np.random.default_rng(nl)
    square, eps, start, *factors = numbers or [int(x) for x in rng.integers(-(1 << 62), 1 << 62, 3 + iterations)]
    x = s.cts((B,), nl)
    r = s.cts((B,), nl) if res else None
    w = s.draw(p.q[:L + 1], ()) if gain else None
    at = slice(None) if check is None else check
    want, h = decoder_ref.rmsnorm(s, x[at], None if r is None else r[at], w, square, eps, start, factors)
    dx, dr = to_dev(x), to_dev(r) if res else None
    h_out = None if not res else dx if in_place else torch.full((B, 2, nl, p.N), -1, dtype=torch.int64, device="cuda")
    out = torch.full((B, 2, L, p.N), -1, dtype=torch.int64, device="cuda")
    ws = ctx.rmsnorm_workspace(B, nl, n1, n2, iterations).random_()
    args = (dx, dr, to_dev(w) if gain else None, square, eps, start, factors, B, nl, n1, n2, stride, *device_keys(s), ws)
    if res and not in_place:
        ck.ckks_rmsnorm(ctx, out, None, *args)        # the sum may stay inside
        assert_same(to_host(out)[at], want, "norm %s" % name)
        out.fill_(-1), ws.random_()
    ck.ckks_rmsnorm(ctx, out, h_out, *args)
    assert_same(to_host(out)[at], want, "norm %s" % name)
    if res:
        assert_same(to_host(h_out)[at], h, "residual sum %s" % name)
    if not in_place:
        assert_same(to_host(dx), x, "input")


@pytest.mark.parametrize("name,nl,B,n1,n2,iterations,res,gain", [
    ("ring10", 6, 1, 2, 2, 1, True, True), ("ring10", 6, 3, 1, 1, 2, False, False), ("ring10", 2, 2, 2, 1, 0, True, True),
    ("ring11", 4, 2, 1, 2, 1, True, True), ("ring12", 5, 3, 2, 2, 1, True, True), ("ring12_wide", 12, 2, 2, 1, 2, True, False),
    ("ring13", 5, 2, 2, 2, 1, True, True), ("ring13", 4, 1, 3, 2, 1, False, True), ("ring13_int", 5, 3, 2, 2, 1, True, True),
    ("ring13_mixed", 5, 2, 2, 2, 1, True, True), ("ring13_mixed", 4, 2, 2, 2, 1, False, False), ("ring13_fp", 5, 2, 2, 2, 1, True, True),
    ("ring14", 7, 2, 2, 2, 2, True, True), ("ring14", 5, 3, 4, 1, 1, False, True), ("ring14_wide", 10, 2, 2, 2, 3, True, True),
    ("ring14_eight", 8, 1, 2, 2, 2, True, True), ("ring15", 5, 2, 2, 2, 1, True, True), ("ring16", 5, 2, 2, 2, 1, True, True),
    ("ring17", 4, 1, 2, 1, 1, True, True)])
def test_norm_matches_the_oracle(name, nl, B, n1, n2, iterations, res, gain):
    run_norm(name, nl, B, n1, n2, iterations, res, gain)


@pytest.mark.parametrize("numbers", [(0, 0, 0, 0), (1, 0, 0, 1), (-(1 << 63), (1 << 63) - 1, -(1 << 63), -(1 << 63)), (1, 1, 1, -1)])
def test_norm_with_numbers_at_the_ends_of_their_range(numbers):
    run_norm("ring10", 5, 1, 2, 1, 1, True, False, numbers=numbers)
    run_norm("ring13_mixed", 4, 1, 1, 2, 1, True, True, numbers=numbers)


def test_the_residual_sum_in_place():
    run_norm("ring10", 4, 2, 2, 1, 1, True, True, in_place=True)
    run_norm("ring13", 4, 2, 2, 1, 1, True, True, in_place=True)
