"""What the host side of the attention calls asks for and refuses, and the launches it books, on a stand-in for the HIP runtime: no
GPU, no kernel runs."""
import json
import os
import random
import re
import subprocess
import sys

import numpy as np
import pytest

from launch_trace import ROOT, _runtime

CALLS = r"""
import ctypes as C, json, sys
from ckks_inputs.params import find_ntt_primes, find_psi
logN, q_bits, nq, p_bits, np, dnum, jobs = json.loads(sys.argv[2])
q = find_ntt_primes(q_bits, nq, logN)
p = find_ntt_primes(p_bits, np, logN, exclude=set(q))
lib = C.CDLL(sys.argv[1])
lib.ckks_linattn_workspace_bytes.restype = lib.ckks_workspace_bytes.restype = C.c_size_t
lib.ckks_last_error.restype = lib.ckks_prof_kind_name.restype = C.c_char_p
array = lambda v: (C.c_uint64 * len(v))(*v)
ctx = C.c_void_p()
assert lib.ckks_ctx_create(C.byref(ctx), logN, array(q), nq, array(p), np, dnum, array([find_psi(m, logN) for m in q + p]), 0) == 0
at = lambda k: C.c_void_p(k << 44)      # device addresses, which nothing reads here
STEP, CHUNK = 9, 10
def run(job):
    what, C_, B, nl, n1, n2 = job[:6]
    op = STEP if what == "step" else CHUNK
    if what == "rope":
        n = lib.ckks_workspace_bytes(ctx, 8, B, nl, 0)
        return lib.ckks_rope(ctx, at(1), at(2), B, nl, at(3), 1, (C.c_uint32 * 1)(5), (C.c_void_p * 1)(4 << 44), 1, at(5), C.c_size_t(n), at(6))
    n = lib.ckks_linattn_workspace_bytes(ctx, op, C_, B, nl, n1, n2)
    if what == "bytes" or not n:
        return n
    keys = lambda k, count: (C.c_void_p * max(1, count))(*[(k << 44) + (i << 36) for i in range(count)])
    sizes = ([] if op == STEP else [C_]) + [B, nl, n1, n2, max(1, (1 << (logN - 1)) // (n1 * n2))]
    call = lib.ckks_linattn_step if op == STEP else lib.ckks_linattn_chunk
    lib.ckks_prof_enable(ctx, 1)
    rc = call(ctx, *[at(k) for k in range(1, 6)], None, None, *sizes, at(7), keys(8, n1 - 1), keys(9, n2 - 1), keys(10, n2 - 1),
              at(11), C.c_size_t(n), at(12))
    if rc: sys.exit(lib.ckks_last_error().decode())
    lib.ckks_prof_collect(ctx)
    out = {}
    for kind in range(lib.ckks_prof_num_kinds()):
        ms, count = C.c_double(), C.c_uint64()
        lib.ckks_prof_read(ctx, kind, C.byref(ms), C.byref(count))
        if count.value: out[lib.ckks_prof_kind_name(kind).decode()] = count.value
    lib.ckks_prof_reset(ctx)
    return out
print(json.dumps([run(job) for job in jobs]), file=sys.stderr)   # stdout has the launches
"""


def answers(shape, jobs):
    """shape: logN, bits and number of the main primes, of the special primes, digits. Jobs (what, tokens, batch, limbs, n1, n2): "bytes"
    is the workspace of a chunk, "step" and "chunk" the launches that the library's profile counts, by name (0: the shape is refused),
    "rope" the code that one rotation returns. Also the launched kernels' names."""
    import paper_2604_03425_amd as pkg
    env = dict(os.environ, LD_LIBRARY_PATH=_runtime(), PYTHONPATH=ROOT)
    res = subprocess.run([sys.executable, "-c", CALLS, pkg.library_path(), json.dumps(list(shape) + [jobs])], env=env,
                         stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
    assert res.returncode == 0, res.stderr
    launches = [line.split() for line in res.stdout.splitlines()]
    return json.loads(res.stderr.splitlines()[-1]), [words[2] for words in launches if words[0] == "launch"]


@pytest.mark.parametrize("shape,nl", [((12, 45, 5, 60, 2, 3), 5), ((13, 50, 4, 60, 2, 2), 4), ((16, 50, 24, 60, 8, 3), 24)])
@pytest.mark.parametrize("tokens,batch,n1,n2", [(1, 1, 2, 2), (1, 2, 2, 2), (2, 1, 2, 2), (1, 1, 4, 4), (1, 1, 1, 1)])
def test_a_small_call_takes_a_small_workspace(shape, nl, tokens, batch, n1, n2):
    """A call has max(n1 n2, (3 n1 + n2) tokens, tokens (tokens + 1) / 2) * batch ciphertexts at most to switch at a time. For each one
    there are, in polynomials of one limb: digits beta * next, accumulators twice 2 * next, a product 3 nl, inputs, results and two
    kinds of scores 4 * 2 nl, ModDown's 2 nl and a coefficient form nl; rotations that a call keeps are among those. Twice that is room
    for the pieces' own rounding and for the terms from inside a chunk."""
    (got,), _ = answers(shape, [("bytes", tokens, batch, nl, n1, n2)])
    logN, _, nq, _, K, dnum = shape
    alpha = -(-nq // dnum)
    beta, ext = -(-nl // alpha), nl + K
    cts = max(n1 * n2, (3 * n1 + n2) * tokens, tokens * (tokens + 1) // 2) * batch
    assert 0 < got <= 2 * cts * (beta * ext + 4 * ext + 14 * nl) * (8 << logN)


@pytest.mark.parametrize("shape", [(10, 50, 4, 60, 2, 2), (13, 50, 4, 60, 2, 2)])
@pytest.mark.parametrize("what,tokens", [("step", 1), ("chunk", 2)])
def test_the_profile_names_the_kernels_that_ran(shape, what, tokens):
    (counts,), launched = answers(shape, [(what, tokens, 2, 4, 2, 2)])
    for name in ("gather_kernel", "rot_sum_kernel", "prod_sum_kernel"):
        assert counts.get(name, 0) == sum(name in k for k in launched), name
    assert counts["gather_kernel"] == 1
    # (a relinearisation in steps starts from a copy of its first two components, which the profile counts among the additions)
    assert counts.get("addto_kernel", 0) == sum("addto_kernel" in k or "first_two_components_kernel" in k for k in launched)


def _limits(call):
    """The limits that the header states for a call, as Python expressions."""
    text = open(os.path.join(ROOT, "include", "ckks_mi355.h")).read()
    text = text[re.search(r"\* %s[:,] " % call, text).start():]
    text = re.sub(r"\n \* *", " ", text[text.index("Limits: "):text.index("*/")])
    return re.search(r"Limits: ([^.]*)\.", text).group(1).split("; ")


def _within(limits, **names):
    for limit in limits:
        lefts, right = limit.split(" <= ")
        for left in re.split(r", (?![^(]*\))", lefts):
            if eval(left, dict(names, max=max)) > int(right):
                return False
    return True


@pytest.mark.parametrize("dnum", [1, 3, 5])
def test_the_header_states_the_limits_of_linear_attention(dnum):
    """Shapes on both sides of every limit: a workspace is asked for where the header allows the call, nowhere else."""
    limits, rng = _limits("ckks_linattn_step"), random.Random(dnum)
    shapes = [(1, b, 5, n1, n2) for n1 in (1, 2) for n2 in (1, 2) for b in (65535 // max(2, dnum), 65535 // max(2, dnum) + 1, 32767, 32768)]
    shapes += [(1, 511, 5, 64, 64), (1, 512, 5, 64, 64), (4096, 1, 5, 1, 1), (4097, 1, 5, 1, 1), (1, 1, 5, 4096, 1), (1, 1, 5, 4097, 1),
               (1, 1, 5, 1, 4096), (1, 1, 5, 1, 4097), (4095, 8, 5, 2, 2), (4096, 8, 5, 2, 2), (3, 4369, 5, 1, 5), (3, 4370, 5, 1, 5)]
    for _ in range(200):
        at = lambda most: min(most, int(2 ** rng.uniform(0, most.bit_length())))   # noqa: E731
        shapes.append((max(1, at(8192)), max(1, at(40000)), 5, max(1, at(5000)), max(1, at(5000))))
    got, _ = answers((10, 50, 5, 60, 5, dnum), [("bytes",) + s for s in shapes])
    want = [_within(limits, tokens=t, B=b, n1=n1, n2=n2, dnum=dnum) for t, b, _, n1, n2 in shapes]
    assert [bool(n) for n in got] == want and 20 < sum(want) < len(want) - 20


@pytest.mark.parametrize("dnum", [1, 3, 5])
def test_the_header_states_the_limits_of_rotary_positions(dnum):
    limits, nl = _limits("ckks_rope"), 5
    digits = -(-nl // -(-5 // dnum))
    batches = [1, 65535 // max(2, digits), 65535 // max(2, digits) + 1, 32767, 32768]
    got, _ = answers((10, 50, 5, 60, 5, dnum), [("rope", 1, b, nl, 1, 1) for b in batches])
    assert [rc == 0 for rc in got] == [_within(limits, B=b, digits=digits) for b in batches]
    assert set(got) == {0, -2}


@pytest.mark.parametrize("n1,n2,stride,valid", [(2, 4, 8, True), (4, 2, 8, True), (1, 8, 8, True), (2, 4, 2, True), (4, 4, 1, True),
                                                (3, 2, 8, False), (2, 2, 24, False), (5, 1, 12, False)])
def test_the_slot_formulas_are_attention_where_the_header_says_so(n1, n2, stride, valid):
    """One lane set of S = 64 slots, rotations as they are: K[b] V[g] are diagonals of k v^T, the read's sum is q^T S, and sum1 and sum2 give
    a lane's score in all of its slots, where n1 n2 stride divides S and the vectors repeat."""
    S, d = 64, n1 * n2
    rng = np.random.default_rng(d)
    assert valid == (S % (d * stride) == 0)
    q, k, v = rng.integers(-9, 10, (3, d, stride))
    spread = lambda x: np.resize(x.reshape(-1), S)       # component i of lane l in slot i * stride + l, again and again   # noqa: E731
    rot = lambda x, r: np.roll(x, -r)                    # noqa: E731
    Q, K = ([rot(spread(x), b * stride) for b in range(n1)] for x in (q, k))
    V = [rot(spread(v), -g * n1 * stride) for g in range(n2)]
    state = [[K[b] * V[g] for b in range(n1)] for g in range(n2)]
    o = sum(rot(sum(Q[b] * state[g][b] for b in range(n1)), g * n1 * stride) for g in range(n2))
    want = spread((q * k).sum(axis=0) * v)
    assert (o == want).all() == valid
    p = spread(q) * spread(k)
    p = sum(rot(p, b * stride) for b in range(n1))
    p = sum(rot(p, g * n1 * stride) for g in range(n2))
    if valid:
        assert (p * spread(v) == want).all()
