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


def test_more_pairs_than_a_key_switch_takes():
    """Slices that end inside a row: the slice of 2^16 is 128 pairs, rows of 50 and 51 tokens, launches of 128 pairs; and a row that begins in
    one slice, fills the next and ends in a third (1024 pairs on 2^10)."""
    run_attention("ring16", 2, (51,), (3,), 7, 0, 0, 0, 1, 1)
    run_attention("ring10", 2, (2100, 3), (1, 1), 100, 0, 0, 0, 1, 2)
    run_attention("ring10", 3, (1030,), (2,), 64, 1025, 2, 1, 1, 1)


def test_the_norm_of_more_than_a_key_switch_takes():
    run_norm("ring16", 4, 65, 2, 1, 1, True, True, check=[0, 63, 64])
    run_norm("ring10", 4, 520, 1, 2, 1, True, False, check=[0, 511, 512, 519])


def test_ring_12_in_both_forms():
    """By whole limbs, and from some 20 ciphertexts of 12 limbs on one kernel per step."""
    PARAMS.setdefault("ring12_steps", lambda: make_params(12, 12, 50, 4, 60, 3))
    run_attention("ring12_steps", 12, (66,), (1,), 9, 0, 0, 1, 2, 2)
    run_attention("ring12_steps", 12, (3,), (1,), 9, 0, 0, 2, 2, 2)
    run_norm("ring12_steps", 12, 66, 2, 1, 1, True, True, check=[0, 65])
    run_norm("ring12_steps", 11, 2, 2, 2, 2, True, True)


@pytest.mark.parametrize("name", ["ring10", "ring13_mixed", "ring14"])
@pytest.mark.parametrize("n1,n2,stride", [(33, 1, 1), (40, 2, 2), (34, 1, 8), (2, 35, 4), (3, 5, 7), (4, 4, 16), (64, 4, 2), (8, 8, 64)])
def test_sums_of_rotations_near_and_far(name, n1, n2, stride):
    """Rotations that stay in blocks of 256 positions and that do not, more of them than a launch takes, digits in several tiles."""
    import paper_2604_03425_amd as ck
    p, rc, ctx = contexts(name)
    nl, rows = 3, 5
    s = attention_ref.Shape(p, rc, 1, 1, 1, seed=n1)
    elements = [pow(5, i * stride, 2 * p.N) for i in range(1, n1)], [pow(5, i * n1 * stride % (p.N // 2), 2 * p.N) for i in range(1, n2)]
    few = [s.key() for _ in range(3)]
    s.baby, s.giant = elements
    s.baby_keys, s.giant_keys = ([few[i % 3] for i in range(len(e))] for e in elements)
    dev = [to_dev(k) for k in few]
    keys = to_dev(s.mult_key), [dev[i % 3] for i in range(n1 - 1)], [dev[i % 3] for i in range(n2 - 1)]
    q, k, v = s.cts((rows,), nl), [s.cts((1,), nl) for _ in range(rows)], [s.cts((1,), nl) for _ in range(rows)]
    want = decoder_ref.attention(s, q, k, v, [1] * rows, 0, 0, 3, 0)
    out = torch.empty((rows, 2, nl - 1, p.N), dtype=torch.int64, device="cuda")
    ck.ckks_attn_paged(ctx, out, to_dev(q), nl, [1] * rows, [1] * rows, [to_dev(x) for x in k], [to_dev(x) for x in v], 1, nl, nl, 0, 0, 3, 0,
                       n1, n2, stride, *keys, ctx.attn_workspace(rows, rows, nl, n1, n2, 0))
    assert_same(to_host(out), want, "sums")


def test_residues_at_the_ends_of_their_range():
    """Every input at its largest value, or that and zero in turn: what the lazy ranges of the kernels are argued from."""
    import paper_2604_03425_amd as ck
    for name in ("ring10", "ring12", "ring13", "ring13_int", "ring13_mixed", "ring13_fp", "ring16"):
        p, rc, ctx = contexts(name)
        n1 = n2 = 2
        nl, rows = 4, 3
        s = attention_ref.Shape(p, rc, n1, n2, p.N // 8)
        top = np.array(p.moduli, dtype=np.uint64)[:, None] - np.uint64(1)
        for step in (1, 2):
            full = np.zeros((len(p.moduli), p.N), dtype=np.uint64)
            full[:, ::step] = top
            key = np.broadcast_to(full, (p.dnum, 2) + full.shape).copy()
            s.mult_key, s.baby_keys, s.giant_keys = key, [key], [key]
            ct = np.broadcast_to(full[:nl], (rows, 2, nl, p.N)).copy()
            dk = to_dev(key), [to_dev(key)], [to_dev(key)]
            want = decoder_ref.attention(s, ct, [ct], [ct], [1], 0, 0, -1, 1)
            out = torch.empty((1, 2, nl - 2, p.N), dtype=torch.int64, device="cuda")
            pages = [to_dev(ct)]
            ck.ckks_attn_paged(ctx, out, to_dev(ct), nl, [1], [rows], pages, pages, rows, nl, nl, 0, 0, -1, 1, n1, n2, p.N // 8, *dk,
                               ctx.attn_workspace(1, 3, nl, n1, n2, 1))
            assert_same(to_host(out), want, "attention " + name)
            want, _ = decoder_ref.rmsnorm(s, ct, ct, full[:2], -1, -1, -1, [-1])
            out = torch.empty((rows, 2, 1, p.N), dtype=torch.int64, device="cuda")
            ck.ckks_rmsnorm(ctx, out, None, to_dev(ct), to_dev(ct), to_dev(full[:2]), -1, -1, -1, [-1], rows, nl, n1, n2, p.N // 8, *dk,
                            ctx.rmsnorm_workspace(rows, nl, n1, n2, 1))
            assert_same(to_host(out), want, "norm " + name)


def test_a_prompt_then_tokens_then_the_norm():
    """As a model runs them: chunks and single tokens on the same cache, pages handed out as it grows and given back as the window leaves
    them, a shared prefix, the norm of the result with the stream of residuals. A chunk and its tokens one by one agree."""
    import paper_2604_03425_amd as ck
    p, rc, ctx = contexts("ring13")
    n1, n2, nl, page, window, sinks, T = 2, 2, 5, 2, 3, 1, 9
    L = nl - 2
    s = attention_ref.Shape(p, rc, n1, n2, p.N // 8, seed=77)
    q, k, v = (s.cts((T,), nl) for _ in range(3))
    keys = device_keys(s)
    dq, dk, dv = (to_dev(x) for x in (q, k, v))
    want = decoder_ref.attention(s, q, [k], [v], [T], window, sinks, 9, 1)

    def run(chunks, seqs):
        pages = {}
        outs, done = [], 0
        for n in chunks:
            lens, new = [done + n] * seqs, [n] + [0] * (seqs - 1)
            for i in range(done // page, -(-(done + n) // page)):
                pages.setdefault(i, (torch.full((page, 2, nl, p.N), -1, dtype=torch.int64, device="cuda"),
                                     torch.full((page, 2, L, p.N), -1, dtype=torch.int64, device="cuda")))
            table = [pages.get(i, (None, None)) for i in range(-(-(done + n) // page))] * seqs    # the other sequences share all of it
            kp, vp = [x for x, _ in table], [x for _, x in table]
            ck.ckks_kv_append(ctx, dk[done:done + n], dv[done:done + n], nl, new, lens, kp, vp, page, nl, L)
            o = torch.empty((n, 2, L, p.N), dtype=torch.int64, device="cuda")
            ck.ckks_attn_paged(ctx, o, dq[done:done + n], nl, new, lens, kp, vp, page, nl, L, window, sinks, 9, 1, n1, n2, p.N // 8, *keys,
                               ctx.attn_workspace(n, ck.attn_pairs(new, lens, window, sinks), nl, n1, n2, 1))
            outs.append(o)
            done += n
            for i in list(pages):
                if i * page >= sinks and (i + 1) * page <= done - window + 1:      # no later token sees it
                    del pages[i]
        assert len(pages) < -(-T // page)
        return torch.cat(outs)

    for chunks, seqs in (([T], 1), ([1] * T, 1), ([4, 1, 1, 3], 2), ([2, 5, 2], 1)):
        if chunks == [T]:
            assert_same(to_host(run([5, 4], 1)), want, "chunks")
        else:
            assert_same(to_host(run(chunks, seqs)), want, "tokens")
    o = run([6, 3], 1)
    x = s.cts((T,), L)
    w = s.draw(p.q[:L], ())
    # a norm that takes the attention's limbs, without steps: L - 1 limbs, the gain at L
    ref_out, ref_h = decoder_ref.rmsnorm(s, x, want, w, 3, 4, 5, [])
    out, h = torch.empty((T, 2, L - 1, p.N), dtype=torch.int64, device="cuda"), torch.empty_like(o)
    ck.ckks_rmsnorm(ctx, out, h, to_dev(x), o, to_dev(w), 3, 4, 5, [], T, L, n1, n2, p.N // 8, *keys, ctx.rmsnorm_workspace(T, L, n1, n2, 0))
    assert_same(to_host(out), ref_out, "norm")
    assert_same(to_host(h), ref_h, "sum")


def test_on_another_stream_and_in_graphs():
    """The calls enqueue on the current stream alone and allocate nothing; two captured graphs that share a workspace, replayed in turn on new
    inputs with eager work between them, give what eager calls give."""
    import paper_2604_03425_amd as ck
    for name in ("ring12", "ring13", "ring10"):
        p, rc, ctx = contexts(name)
        n1 = n2 = 2
        nl, page, lens, new = 4, 2, [3, 2], [1, 1]
        s = attention_ref.Shape(p, rc, n1, n2, p.N // 8, seed=9)
        keys = device_keys(s)
        table = [torch.empty((page, 2, nl, p.N), dtype=torch.int64, device="cuda") for _ in range(6)]
        kp, vp = table[:3], table[3:]
        need = max(ck.ckks_attn_workspace_bytes(ctx, 2, 5, nl, n1, n2, 1), ck.ckks_rmsnorm_workspace_bytes(ctx, 2, nl, n1, n2, 1))
        ws = torch.empty(need // 8, dtype=torch.int64, device="cuda")
        q, k, v, x = (torch.empty((2, 2, nl, p.N), dtype=torch.int64, device="cuda") for _ in range(4))
        o, out, h = (torch.empty((2, 2, n, p.N), dtype=torch.int64, device="cuda") for n in (nl - 2, 1, nl))

        def attend():
            ck.ckks_kv_append(ctx, k, v, nl, new, lens, kp, vp, page, nl, nl)
            ck.ckks_attn_paged(ctx, o, q, nl, new, lens, kp, vp, page, nl, nl, 0, 0, 7, 1, n1, n2, p.N // 8, *keys, ws)

        def norm():
            ck.ckks_rmsnorm(ctx, out, h, x, q, None, 3, 4, 5, [6], 2, nl, n1, n2, p.N // 8, *keys, ws)

        def fill(seed):
            s.seed = 1000 * seed
            for t in (q, k, v, x):
                t.copy_(to_dev(s.cts((2,), nl)))
            for t in table:
                t.copy_(to_dev(s.cts((page,), nl)))
            for t in (o, out, h):
                t.fill_(-1)
            ws.random_()
            torch.cuda.synchronize()

        def expected(seed):
            fill(seed)
            attend(), norm()
            torch.cuda.synchronize()
            return [t.clone() for t in (o, out, h, *table)]

        def check(want, what):
            torch.cuda.synchronize()
            for a, b in zip((o, out, h, *table), want):
                assert torch.equal(a, b), (name, what)

        want = expected(1)
        fill(1)
        side = torch.cuda.Stream()
        before = torch.cuda.memory_allocated()
        with torch.cuda.stream(side):
            attend(), norm()
        check(want, "side stream")
        assert torch.cuda.memory_allocated() == before
        graphs = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[0]):
            attend()
        with torch.cuda.graph(graphs[1]):
            norm()
        for trial in range(2, 5):
            want = expected(trial)          # eager calls between the replays
            fill(trial)
            graphs[trial % 2].replay()
            graphs[1 - trial % 2].replay()
            check(want, trial)


@pytest.mark.parametrize("knob,value", [(0, 0), (1, 1), (2, 1), (2, 2), (3, 1), (4, 0), (5, 1)])
@pytest.mark.parametrize("name", ["ring12", "ring13_mixed", "ring16"])
def test_tuning_knobs_change_no_result(name, knob, value):
    import paper_2604_03425_amd as ck
    p, rc, ctx = contexts(name)
    default = {0: -1, 1: 0, 2: 0, 3: 2, 4: 1, 5: 0}[knob]
    ck.ckks_tune_set(ctx, knob, value)
    try:
        run_attention(name, 4, (3,), (1,), 2, 0, 0, 1, 2, 2)
        run_norm(name, 4, 2, 2, 2, 1, True, True)
    finally:
        ck.ckks_tune_set(ctx, knob, default)


def test_small_primes_as_integers():
    """Main primes below 2^36, which knob 1 gives integer bodies: the divisions' conversion leaves the fused kernel then."""
    import paper_2604_03425_amd as ck
    PARAMS.setdefault("ring13_small", lambda: make_params(13, 4, 34, 2, 40, 2))
    p, rc, ctx = contexts("ring13_small")
    for value in (0, 1, 0):
        ck.ckks_tune_set(ctx, 1, value)
        run_attention("ring13_small", 4, (3,), (1,), 2, 0, 0, 1, 2, 2, bias=1 << 60)
        run_norm("ring13_small", 4, 2, 2, 2, 1, True, True)


def test_a_cache_beyond_2_to_32_words():
    """One allocation of 40 GB for all pages: tokens at its end alone give the same as in a small cache."""
    import paper_2604_03425_amd as ck
    p, rc, ctx = contexts("ring16")
    nl, page, N = 5, 64, p.N
    pages = 120
    k = torch.empty((pages, page, 2, nl, N), dtype=torch.int64, device="cuda")
    assert k.numel() > 1 << 32
    gen = torch.Generator(device="cuda").manual_seed(3)

    def residues(lead, moduli):
        x = torch.empty(tuple(lead) + (len(moduli), N), dtype=torch.int64, device="cuda")
        for i, m in enumerate(moduli):
            x[..., i, :].random_(0, m, generator=gen)
        return x

    key = residues((p.dnum, 2), p.moduli)
    last = residues((2, 2), p.q)
    first = residues((1, 2), p.q)
    v = residues((3, 2), p.q)
    q = residues((1, 2), p.q)
    # a sequence as long as the cache; sinks on its first page, the window on its last
    n = pages * page
    vt = torch.empty((page, 2, nl, N), dtype=torch.int64, device="cuda")
    ve = torch.empty_like(vt)
    kp, vp = [None] * pages, [None] * pages
    kp[0], kp[-1], vp[0], vp[-1] = k[0], k[-1], vt, ve
    k[0, 0], vt[0], k[-1, -2], ve[-2] = first[0], v[0], last[0], v[1]
    ck.ckks_kv_append(ctx, last[1:], v[2:], nl, [1], [n], kp, vp, page, nl, nl)
    assert torch.equal(k[-1, -1], last[1]) and torch.equal(ve[-1], v[2])
    args = (9, 1, 1, 1, 1, key, [], [], ctx.attn_workspace(1, 3, nl, 1, 1, 1))
    o, small = (torch.empty((1, 2, nl - 2, N), dtype=torch.int64, device="cuda") for _ in range(2))
    ck.ckks_attn_paged(ctx, o, q, nl, [1], [n], kp, vp, page, nl, nl, 2, 1, *args)
    few = torch.cat([first, last]).contiguous()
    ck.ckks_attn_paged(ctx, small, q, nl, [1], [3], [few], [v], 3, nl, nl, 2, 1, *args)
    torch.cuda.synchronize()
    assert torch.equal(o, small)
    # and as one flat page, whose last tokens lie beyond 2^32 words
    flat = k.view(1, n, 2, nl, N)[0]
    ck.ckks_attn_paged(ctx, small, q, nl, [1], [n], [flat], [flat], n, nl, nl, 2, 1, *args)
    tail = torch.cat([flat[:1], flat[-2:]]).contiguous()
    ck.ckks_attn_paged(ctx, o, q, nl, [1], [3], [tail], [tail], 3, nl, nl, 2, 1, *args)
    torch.cuda.synchronize()
    assert torch.equal(o, small)
    del k, kp, flat
    torch.cuda.empty_cache()


def test_the_binding_refuses():
    import paper_2604_03425_amd as ck
    p, rc, ctx = contexts("ring10")
    N, nl = p.N, 4
    new = lambda *shape: torch.zeros(shape, dtype=torch.int64, device="cuda")   # noqa: E731
    key = new(p.dnum, 2, len(p.moduli), N)
    page, ct = new(2, 2, nl, N), new(1, 2, nl, N)
    ws = ctx.attn_workspace(1, 3, nl, 1, 2, 1)
    good = dict(o_out=new(1, 2, 2, N), q=ct, nlimbs=nl, new_lens=[1], lens=[3], k_pages=[page, page], v_pages=[page, page], page_tokens=2,
                k_limbs=nl, v_limbs=nl, window=0, sinks=0, bias=1, squarings=1, n1=1, n2=2, stride=N // 4, evk_mult=key, evk_baby=[],
                evk_giant=[key], ws=ws)
    ck.ckks_attn_paged(ctx, **good)
    for error, change in ((ValueError, dict(k_pages=[page])), (ValueError, dict(evk_baby=[key])), (ValueError, dict(new_lens=[1, 0])),
                          (ValueError, dict(k_pages=[page, page[:1]])), (ValueError, dict(o_out=new(1, 2, 1, N))), (ValueError, dict(lens=[-1])),
                          (ValueError, dict(q=ct[:, :1].contiguous())), (TypeError, dict(q=ct.cpu())), (TypeError, dict(v_pages=[page, page.float()])),
                          (TypeError, dict(k_pages=[page, page.transpose(0, 1)])), (ValueError, dict(evk_mult=key[:1])), (ValueError, dict(page_tokens=0)),
                          (ValueError, dict(bias=1 << 63)), (ValueError, dict(bias=-(1 << 63) - 1)), (ValueError, dict(window=-1)), (ValueError, dict(sinks=-1)),
                          (ValueError, dict(squarings=-1)),
                          (ck.CkksError, dict(k_pages=[None, page])), (ck.CkksError, dict(squarings=3, o_out=new(1, 2, 2, N)))):
        with pytest.raises(error):
            ck.ckks_attn_paged(ctx, **dict(good, **change))
    with pytest.raises(ck.CkksError):
        ctx.attn_workspace(1, 0, nl, 1, 2, 1)
    with pytest.raises(ck.CkksError):
        ctx.rmsnorm_workspace(1, 3, 1, 2, 1)
    app = dict(k=ct, v=ct, in_limbs=nl, new_lens=[1], lens=[3], k_pages=[None, page], v_pages=[None, new(2, 2, nl, N)], page_tokens=2, k_limbs=nl, v_limbs=nl)
    ck.ckks_kv_append(ctx, **app)
    for error, change in ((ValueError, dict(k=ct[:, :1].contiguous())), (ck.CkksError, dict(v_pages=[None, page])), (ck.CkksError, dict(k=page)),
                          (TypeError, dict(v=None))):
        with pytest.raises(error):
            ck.ckks_kv_append(ctx, **dict(app, **change))
    norm = dict(ct_out=new(1, 2, 1, N), h_out=new(1, 2, nl, N), ct_x=ct, ct_res=new(1, 2, nl, N), gain=new(2, N), square=1, eps=0, start=5, factors=[3],
                B=1, nlimbs=nl, n1=1, n2=2, stride=N // 4, evk_mult=key, evk_baby=[], evk_giant=[key], ws=ctx.rmsnorm_workspace(1, nl, 1, 2, 1))
    ck.ckks_rmsnorm(ctx, **norm)
    for error, change in ((ValueError, dict(ct_out=new(1, 2, 1, N // 2))), (ValueError, dict(gain=new(1, N))), (ValueError, dict(evk_giant=[])),
                          (ck.CkksError, dict(factors=[3, 3])), (ValueError, dict(factors=[1 << 63])), (ValueError, dict(start=1 << 64)),
                          (TypeError, dict(ct_res=ct.cpu())), (ck.CkksError, dict(ct_out=norm["h_out"]))):
        with pytest.raises(error):
            ck.ckks_rmsnorm(ctx, **dict(norm, **change))


def test_calls_in_flight_on_two_streams():
    """Two calls at once: the same context, keys and cache, a stream and a workspace each."""
    import paper_2604_03425_amd as ck
    for name in ("ring12", "ring13"):
        p, rc, ctx = contexts(name)
        nl, n, page = 4, 5, 2
        s = attention_ref.Shape(p, rc, 2, 2, p.N // 8, seed=31)
        keys = device_keys(s)
        k, v, q, x = (s.cts((m,), nl) for m in (n, n, 2, 3))
        cache = Cache([n], [0], page, nl, nl, p.N, [k], [v])
        want = [decoder_ref.attention(s, q[i:i + 1], [k], [v], [1], 0, 0, 5 + i, 1) for i in range(2)]
        want += decoder_ref.rmsnorm(s, x, None, None, 2, 3, 4, [5])[:1]
        q, x = to_dev(q), to_dev(x)
        outs = [torch.empty((m, 2, limbs, p.N), dtype=torch.int64, device="cuda") for m, limbs in ((1, nl - 2), (1, nl - 2), (3, 1))]
        spaces = [ctx.attn_workspace(1, n, nl, 2, 2, 1) for _ in range(2)] + [ctx.rmsnorm_workspace(3, nl, 2, 2, 1)]
        streams = [torch.cuda.Stream() for _ in range(3)]
        for trial in range(3):
            for t in outs + spaces:
                t.fill_(-1)
            torch.cuda.synchronize()
            for i in range(2):
                with torch.cuda.stream(streams[i]):
                    ck.ckks_attn_paged(ctx, outs[i], q[i:i + 1], nl, [1], [n], *cache.args, 0, 0, 5 + i, 1, 2, 2, p.N // 8, *keys, spaces[i])
            with torch.cuda.stream(streams[2]):
                ck.ckks_rmsnorm(ctx, outs[2], None, x, None, None, 2, 3, 4, [5], 3, nl, 2, 2, p.N // 8, *keys, spaces[2])
            torch.cuda.synchronize()
            for got, ref in zip(outs, want):
                assert_same(to_host(got), ref, "%s, trial %d" % (name, trial))


def test_tensors_that_begin_on_an_odd_word():
    """Rows, pages and a gain 8 bytes behind an aligned place."""
    import paper_2604_03425_amd as ck

    def odd(x):
        t = torch.empty(x.size + 1, dtype=torch.int64, device="cuda")[1:].view(x.shape)
        return t.copy_(to_dev(x))

    for name in ("ring10", "ring12", "ring13"):
        p, rc, ctx = contexts(name)
        nl, n = 4, 3
        s = attention_ref.Shape(p, rc, 2, 1, p.N // 4, seed=41)
        keys = device_keys(s)
        k, v, q, x, r = (s.cts((m,), nl) for m in (n, n, 1, 2, 2))
        gain = s.draw(p.q[:2], ())
        want = decoder_ref.attention(s, q, [k], [v], [1], 0, 0, 5, 1)
        kp, vp = ([odd(np.zeros((n, 2, nl, p.N), dtype=np.uint64))] for _ in range(2))
        assert kp[0].data_ptr() % 16 == 8
        o = odd(np.zeros((1, 2, nl - 2, p.N), dtype=np.uint64))
        ck.ckks_kv_append(ctx, odd(k), odd(v), nl, [n], [n], kp, vp, n, nl, nl)
        ck.ckks_attn_paged(ctx, o, odd(q), nl, [1], [n], kp, vp, n, nl, nl, 0, 0, 5, 1, 2, 1, p.N // 4, *keys, ctx.attn_workspace(1, n, nl, 2, 1, 1))
        assert_same(to_host(o), want, "attention " + name)
        want, want_h = decoder_ref.rmsnorm(s, x, r, gain, 2, 3, 4, [5])
        out, h = odd(np.zeros((2, 2, 1, p.N), dtype=np.uint64)), odd(np.zeros((2, 2, nl, p.N), dtype=np.uint64))
        ck.ckks_rmsnorm(ctx, out, h, odd(x), odd(r), odd(gain), 2, 3, 4, [5], 2, nl, 2, 1, p.N // 4, *keys, ctx.rmsnorm_workspace(2, nl, 2, 1, 1))
        assert_same(to_host(out), want, "norm " + name)
        assert_same(to_host(h), want_h, "sum " + name)


@pytest.mark.parametrize("name,nl,n1,n2,squarings", [
    ("ring13", 5, 2, 2, 1), ("ring13_int", 5, 1, 1, 1), ("ring13_mixed", 5, 2, 1, 2), ("ring13_fp", 5, 1, 2, 1), ("ring14", 7, 2, 2, 1),
    ("ring14_wide", 10, 1, 2, 1), ("ring14_eight", 7, 1, 1, 1)])
def test_relinearisations_of_many_ciphertexts(name, nl, n1, n2, squarings):
    """34 pairs, and 17 ciphertexts of a norm: the fused kernels of a key switch, where most shapes above are few enough for those of sums."""
    run_attention(name, nl, (34,), (1,), 7, 0, 0, squarings, n1, n2)
    run_norm(name, nl, 17, n1, n2, 1, True, True)


@pytest.mark.parametrize("name,knobs", [("ring13", {2: 2, 4: 0}), ("ring13", {2: 1, 4: 0}), ("ring13_two_kinds", {4: 0}), ("ring13_nine", {4: 0})])
def test_the_second_stream_changes_no_result(name, knobs):
    """Shapes whose relinearisations by a main prime too run part of a key switch on the context's second stream: 13 pairs and ciphertexts at 2^13
    are above those that go as sums."""
    import paper_2604_03425_amd as ck

    def two_kinds():
        q, p = find_ntt_primes(60, 1, 13) + find_ntt_primes(50, 3, 13), find_ntt_primes(60, 3, 13)[1:]
        return CkksParams(logN=13, q=q, p=p, dnum=2, psi=[find_psi(m, 13) for m in q + p])

    PARAMS.setdefault("ring13_two_kinds", two_kinds)
    PARAMS.setdefault("ring13_nine", lambda: make_params(13, 9, 50, 9, 60, 1))
    p, rc, ctx = contexts(name)
    nl = min(len(p.q), 5) if name != "ring13_nine" else 9
    try:
        for knob, value in knobs.items():
            ck.ckks_tune_set(ctx, knob, value)
        for _ in range(3):
            run_attention(name, nl, (13,), (1,), 5, 0, 0, 1, 1, 1)
        run_norm(name, nl, 13, 1, 1, 1, False, False)
    finally:
        for knob, value in {2: 0, 4: 1}.items():
            ck.ckks_tune_set(ctx, knob, value)


@pytest.mark.parametrize("name,nl,rows,n1,n2,stride", [("ring14", 7, 28, 34, 2, 32), ("ring14", 7, 28, 34, 1, 32), ("ring13_mixed", 5, 66, 2, 36, 16),
                                                       ("ring13_int", 5, 74, 40, 1, 16)])
def test_more_rotations_than_a_launch_takes_with_finished_limbs(name, nl, rows, n1, n2, stride):
    """Enough ciphertexts for the main limbs' sums to be finished in the kernel that forms them, over two launches of rotations of which the
    second one adds to the first one's sums."""
    import paper_2604_03425_amd as ck
    p, rc, ctx = contexts(name)
    assert -(-rows // 4) * (p.N // 256) * (nl + len(p.p)) > 4096
    s = attention_ref.Shape(p, rc, 1, 1, 1, seed=n1 + n2)
    elements = [pow(5, i * stride, 2 * p.N) for i in range(1, n1)], [pow(5, i * n1 * stride % (p.N // 2), 2 * p.N) for i in range(1, n2)]
    assert all(g % (p.N // 128) == 1 for e in elements for g in e)       # near rotations
    few = [s.key() for _ in range(3)]
    s.baby, s.giant = elements
    s.baby_keys, s.giant_keys = ([few[i % 3] for i in range(len(e))] for e in elements)
    dev = [to_dev(k) for k in few]
    keys = to_dev(s.mult_key), [dev[i % 3] for i in range(n1 - 1)], [dev[i % 3] for i in range(n2 - 1)]
    q, k, v = s.cts((rows,), nl), s.cts((rows,), nl), s.cts((rows,), nl)
    at = [0, 1, rows // 2, rows - 1]
    want = decoder_ref.attention(s, q[at], [k[i:i + 1] for i in at], [v[i:i + 1] for i in at], [1] * len(at), 0, 0, 3, 0)
    out = torch.empty((rows, 2, nl - 1, p.N), dtype=torch.int64, device="cuda")
    ws = ctx.attn_workspace(rows, rows, nl, n1, n2, 0).random_()
    dk, dv = to_dev(k), to_dev(v)
    ck.ckks_attn_paged(ctx, out, to_dev(q), nl, [1] * rows, [1] * rows, [x[None] for x in dk], [x[None] for x in dv], 1, nl, nl, 0, 0, 3, 0, n1, n2,
                       stride, *keys, ws)
    assert_same(to_host(out)[at], want, "sums")


@pytest.mark.parametrize("name,nl", [("ring12", 4), ("ring13", 4), ("ring14", 5)])
def test_the_norm_of_1024_components(name, nl):
    """A hidden vector of 1024 (768 filled up with zeros): near giant steps, baby steps that leave their blocks."""
    run_norm(name, nl, 2, 32, 32, 1, True, True)


@pytest.mark.parametrize("nl", [6, 3, 2])
def test_digits_of_one_limb(nl):
    """Every digit a limb: the last one's own limb is the one that is divided away."""
    PARAMS.setdefault("ring13_one", lambda: make_params(13, 6, 50, 1, 60, 6))
    run_attention("ring13_one", nl, (13,), (1,), 5, 0, 0, min(1, nl - 2), 1, 1)
    run_attention("ring13_one", nl, (3,), (2,), 2, 0, 0, min(1, nl - 2), 2, 2)
    run_norm("ring13_one", nl, 13, 1, 2, (nl - 2) // 2, True, True)


@pytest.mark.parametrize("knob,value", [(0, 0), (1, 1), (2, 1), (2, 2), (3, 1), (4, 0), (5, 1)])
@pytest.mark.parametrize("name", ["ring13_mixed", "ring13"])
def test_tuning_knobs_on_many_ciphertexts(name, knob, value):
    """13 of them: more than the relinearisations that go as sums of one rotation."""
    import paper_2604_03425_amd as ck
    p, rc, ctx = contexts(name)
    default = {0: -1, 1: 0, 2: 0, 3: 2, 4: 1, 5: 0}[knob]
    ck.ckks_tune_set(ctx, knob, value)
    try:
        run_attention(name, 4, (13,), (1,), 5, 0, 0, 1, 1, 2)
        run_norm(name, 4, 13, 1, 1, 1, True, True)
    finally:
        ck.ckks_tune_set(ctx, knob, default)
