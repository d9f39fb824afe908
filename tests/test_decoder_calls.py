"""What the host side of attention over a paged cache and of the norm asks for, refuses and launches, on a stand-in for the HIP runtime:
no GPU, no kernel runs."""
import json
import os
import re
import subprocess
import sys

import pytest

from launch_trace import ROOT, _runtime

CALLS = r"""
import ctypes as C, json, sys
from ckks_inputs.params import find_ntt_primes, find_psi
logN, q_bits, nq, p_bits, np, dnum, jobs = json.loads(sys.argv[2])
q = find_ntt_primes(q_bits, nq, logN)
p = find_ntt_primes(p_bits, np, logN, exclude=set(q)) if np else []
lib = C.CDLL(sys.argv[1])
lib.ckks_attn_workspace_bytes.restype = lib.ckks_rmsnorm_workspace_bytes.restype = lib.ckks_workspace_bytes.restype = C.c_size_t
lib.ckks_last_error.restype = lib.ckks_prof_kind_name.restype = C.c_char_p
array = lambda v: (C.c_uint64 * max(1, len(v)))(*v)
u32s = lambda v: None if v is None else (C.c_uint32 * max(1, len(v)))(*v)
ptrs = lambda v: None if v is None else (C.c_void_p * max(1, len(v)))(*v)
i64s = lambda v: None if v is None else (C.c_int64 * max(1, len(v)))(*v)
at = lambda v: None if v is None else C.c_void_p(v)
ctx = C.c_void_p()
assert lib.ckks_ctx_create(C.byref(ctx), logN, array(q), nq, array(p), np, dnum, array([find_psi(m, logN) for m in q + p]), 0) == 0
out = []
flush = C.CDLL(None).fflush            # the launches are written by C's own buffer
for j in jobs:
    flush(None)
    print("job", flush=True)
    kind = j.pop("call")
    if kind == "attn_bytes":
        out.append(lib.ckks_attn_workspace_bytes(ctx, j["rows"], C.c_uint64(j["pairs"]), j["nl"], j["n1"], j["n2"], j["sq"]))
        continue
    if kind == "norm_bytes":
        out.append(lib.ckks_rmsnorm_workspace_bytes(ctx, j["B"], j["nl"], j["n1"], j["n2"], j["its"]))
        continue
    if j.get("profile"):
        lib.ckks_prof_enable(ctx, 1)
    if kind == "append":
        rc = lib.ckks_kv_append(ctx if j["ctx"] else None, at(j["k"]), at(j["v"]), j["inl"], len(j["lens"] or []), u32s(j["new"]), u32s(j["lens"]),
                                ptrs(j["kp"]), ptrs(j["vp"]), j["page"], j["kl"], j["vl"], at(1 << 50))
    elif kind == "attn":
        n = lib.ckks_attn_workspace_bytes(ctx, max(1, sum(j["new"] or [])), C.c_uint64(j.get("pairs", 1000)), max(1, j["nl"]), j["n1"], j["n2"], j["sq"]) + j["ws_less"]
        rc = lib.ckks_attn_paged(ctx if j["ctx"] else None, at(j["o"]), at(j["q"]), j["nl"], len(j["lens"] or []), u32s(j["new"]), u32s(j["lens"]), ptrs(j["kp"]),
                                 ptrs(j["vp"]), j["page"], j["kl"], j["vl"], j["window"], j["sinks"], C.c_int64(j["bias"]), j["sq"], j["n1"],
                                 j["n2"], j["stride"], at(j["mult"]), ptrs(j["baby"]), ptrs(j["giant"]), at(j["ws"]), C.c_size_t(n), at(1 << 50))
    else:
        n = lib.ckks_rmsnorm_workspace_bytes(ctx, max(1, j["B"]), max(1, j["nl"]), j["n1"], j["n2"], j["its"]) + j["ws_less"]
        rc = lib.ckks_rmsnorm(ctx if j["ctx"] else None, at(j["out"]), at(j["h"]), at(j["x"]), at(j["res"]), at(j["gain"]), C.c_int64(3), C.c_int64(-1),
                              C.c_int64(1 << 50), i64s(j["factors"]), j["its"], j["B"], j["nl"], j["n1"], j["n2"], j["stride"],
                              at(j["mult"]), ptrs(j["baby"]), ptrs(j["giant"]), at(j["ws"]), C.c_size_t(n), at(1 << 50))
    out.append([rc, lib.ckks_last_error().decode() if rc else ""])
    if j.get("profile"):
        lib.ckks_prof_collect(ctx)
        lib.ckks_prof_enable(ctx, 0)
        out[-1].append({})
        for i in range(lib.ckks_prof_num_kinds()):
            ms, count = C.c_double(), C.c_uint64()
            lib.ckks_prof_read(ctx, i, C.byref(ms), C.byref(count))
            out[-1][-1][lib.ckks_prof_kind_name(i).decode()] = count.value
        lib.ckks_prof_reset(ctx)
flush(None)
print(json.dumps(out), file=sys.stderr)
"""


def answers(shape, jobs):
    """(results, launched kernels of each job)"""
    import paper_2604_03425_amd as pkg
    env = dict(os.environ, LD_LIBRARY_PATH=_runtime(), PYTHONPATH=ROOT)
    res = subprocess.run([sys.executable, "-c", CALLS, pkg.library_path(), json.dumps(list(shape) + [jobs])], env=env,
                         stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
    assert res.returncode == 0, res.stderr
    launches = []
    for line in res.stdout.splitlines():
        if line == "job":
            launches.append([])
        elif line.startswith("launch"):
            launches[-1].append(line.split()[2])
    return json.loads(res.stderr.splitlines()[-1]), launches


SHAPE = (10, 50, 5, 60, 2, 3)
CT = 2 * 1024 * 8                      # bytes of a ciphertext's limb
PAGES = [(20 << 40) + (i << 30) for i in range(4)], [(30 << 40) + (i << 30) for i in range(4)]
CACHE = dict(lens=[5, 3], new=[2, 1], kp=PAGES[0], vp=PAGES[1], page=3, kl=4, vl=3, ctx=True)
KEYS = dict(n1=2, n2=2, stride=256, mult=4 << 40, baby=[5 << 40], giant=[6 << 40], ws=7 << 40, ws_less=0)
ATTN = dict(call="attn", o=1 << 40, q=2 << 40, nl=4, window=0, sinks=0, bias=5, sq=1, **CACHE, **KEYS)
APPEND = dict(call="append", k=1 << 40, v=2 << 40, inl=4, **CACHE)
NORM = dict(call="norm", out=1 << 40, h=8 << 40, x=2 << 40, res=3 << 40, gain=9 << 40, factors=[1 << 51], its=1, B=2, nl=5, ctx=True, **KEYS)

REFUSALS = [(APPEND, code, change) for code, change in [
    (-1, dict(ctx=False)), (-1, dict(k=None)), (-1, dict(v=None)), (-1, dict(new=None)), (-1, dict(lens=None)), (-1, dict(kp=None)),
    (-1, dict(vp=None)), (-1, dict(kp=[PAGES[0][0], None, PAGES[0][2], PAGES[0][3]])), (-1, dict(vp=PAGES[1][:2] + [None])),
    (-1, dict(kp=PAGES[0][:2] + [PAGES[0][1] - 7 * CT])),         # the second sequence's third token begins inside the first one's fourth
    (-1, dict(kp=PAGES[0][:2] + [PAGES[0][1] - 4 * CT])),         # it has the place of the first one's fifth
    (-1, dict(vp=[PAGES[1][0], PAGES[0][1], PAGES[1][2]])),       # a value in the place of a key
    (-1, dict(kp=[PAGES[0][0], 1 << 40, PAGES[0][2]])), (-1, dict(vp=[PAGES[1][0], (2 << 40) - 3 * CT, PAGES[1][2]])),   # over k, over v
    (-2, dict(inl=0)), (-2, dict(inl=6)), (-2, dict(inl=3)), (-2, dict(kl=0)), (-2, dict(vl=0)), (-2, dict(kl=6, inl=5)), (-2, dict(vl=5)),
    (-2, dict(page=0)), (-2, dict(new=[6, 1])), (-2, dict(lens=[5, 1 << 31])), (-2, dict(lens=[40000, 3], new=[32767, 1], page=40000)),
]] + [(ATTN, code, change) for code, change in [
    (-1, dict(ctx=False)), (-1, dict(o=None)), (-1, dict(q=None)), (-1, dict(new=None)), (-1, dict(lens=None)), (-1, dict(kp=None)), (-1, dict(vp=None)),
    (-1, dict(mult=None)), (-1, dict(baby=None)), (-1, dict(giant=None)), (-1, dict(baby=[None])), (-1, dict(giant=[None])),
    (-1, dict(kp=[None] + PAGES[0][1:])), (-1, dict(vp=PAGES[1][:2] + [None])),
    (-1, dict(kp=[None] + PAGES[0][1:], window=2, sinks=1)),      # a sink is on it
    (-1, dict(kp=[None] + PAGES[0][1:], window=3)),               # the first new token's window begins on it
    (-1, dict(o=2 << 40)), (-1, dict(o=(2 << 40) + 3 * 4 * CT - 8)), (-1, dict(o=PAGES[0][1])), (-1, dict(o=PAGES[1][2] + 9 * CT - 8)),
    (-2, dict(nl=0)), (-2, dict(nl=6)), (-2, dict(nl=1, sq=0)), (-2, dict(sq=3)), (-2, dict(kl=3)), (-2, dict(vl=1)), (-2, dict(page=0)),
    (-2, dict(stride=0)), (-2, dict(n1=0)), (-2, dict(n2=0)), (-2, dict(n1=4097)), (-2, dict(new=[6, 0])),
    (-3, dict(ws=None)), (-3, dict(ws=(7 << 40) + 8)), (-3, dict(ws_less=-256, pairs=12)),
]] + [(NORM, code, change) for code, change in [
    (-1, dict(ctx=False)), (-1, dict(out=None)), (-1, dict(x=None)), (-1, dict(factors=None)), (-1, dict(mult=None)), (-1, dict(baby=[None])), (-1, dict(giant=None)),
    (-1, dict(res=None)),                                          # h without a residual
    (-1, dict(out=2 << 40)), (-1, dict(out=(3 << 40) + 2 * 5 * CT - 8)), (-1, dict(out=9 << 40)), (-1, dict(h=1 << 40)), (-1, dict(h=9 << 40)),
    (-1, dict(h=(2 << 40) + 8)), (-1, dict(h=(3 << 40) - 8)),
    (-2, dict(B=0)), (-2, dict(nl=0)), (-2, dict(nl=6)), (-2, dict(nl=3)), (-2, dict(its=2)), (-2, dict(stride=0)), (-2, dict(n1=0)),
    (-2, dict(B=32768)), (-3, dict(ws=None)), (-3, dict(ws=(7 << 40) + 128)), (-3, dict(ws_less=-256)),
]]


def test_refusals():
    """The code, a message, and nothing enqueued; the calls that the changes start from go through."""
    jobs = [dict(base, **change) for base, _, change in REFUSALS] + [dict(b) for b in (APPEND, ATTN, NORM)]
    got, launched = answers(SHAPE, jobs)
    for (base, code, change), (rc, text), kernels in zip(REFUSALS, got, launched):
        assert rc == code and text and not kernels, (base["call"], change, rc, text)
    assert [g[0] for g in got[-3:]] == [0, 0, 0] and all(launched[-3:])


def test_calls_that_look_odd_and_are_allowed():
    none = dict(ATTN, new=[0, 0], o=None, q=None, kp=[None] * 3, vp=[None] * 3, ws=None)
    jobs = [none, dict(APPEND, new=[0, 0], k=None, v=None, kp=[None] * 3, vp=[None] * 3), dict(ATTN, lens=[], new=[], kp=[], vp=[]),
            dict(ATTN, kp=[None] + PAGES[0][1:], vp=[None] + PAGES[1][1:], window=1),     # pages behind every window
            dict(ATTN, lens=[9, 0, 3], new=[1, 0, 0], kp=[PAGES[0][0], None, PAGES[0][2], None], vp=[PAGES[1][0], None, PAGES[1][2], None],
                 window=2, sinks=3),                                                      # between sinks and window
            dict(APPEND, kp=[None, PAGES[0][1], PAGES[0][2]], vp=[None, PAGES[1][1], PAGES[1][2]]),
            dict(ATTN, kp=[PAGES[0][0], PAGES[0][1], PAGES[0][0]], vp=[PAGES[1][0], PAGES[1][1], PAGES[1][0]]),   # a shared prefix
            dict(NORM, h=2 << 40), dict(NORM, h=3 << 40), dict(NORM, h=None), dict(NORM, h=None, res=None), dict(NORM, gain=None),
            dict(NORM, its=0, factors=None, nl=2), dict(NORM, res=2 << 40, h=2 << 40)]
    got, launched = answers(SHAPE, jobs)
    assert [g[0] for g in got] == [0] * len(jobs), got
    assert [bool(x) for x in launched] == [False] * 3 + [True] * 11


def test_a_context_without_special_primes_is_refused():
    got, launched = answers((10, 50, 5, 60, 0, 5), [dict(ATTN), dict(NORM)])
    assert [g[0] for g in got] == [-2, -2] and not any(launched)


def test_workspaces():
    """Nothing on a bad argument; growth with the pairs up to what fills the chip."""
    a = dict(call="attn_bytes", rows=2, pairs=8, nl=5, n1=2, n2=2, sq=1)
    n = dict(call="norm_bytes", B=2, nl=5, n1=2, n2=2, its=1)
    bad = [dict(a, **x) for x in (dict(rows=0), dict(rows=32768, pairs=40000), dict(pairs=1), dict(nl=1), dict(nl=6), dict(sq=4), dict(n1=0), dict(n2=4097))]
    bad += [dict(n, **x) for x in (dict(B=0), dict(B=32768), dict(nl=1), dict(its=2), dict(its=1 << 31), dict(n1=0))]
    good = [dict(a, pairs=x) for x in (2, 8, 1024, 1025, 1 << 40)] + [dict(n, B=x) for x in (1, 512, 513, 32767)]
    got, _ = answers(SHAPE, bad + good)
    assert got[:len(bad)] == [0] * len(bad)
    p = got[len(bad):]
    assert 0 < p[0] < p[1] < p[2] == p[3] == p[4] and 0 < p[5] < p[6] == p[7] == p[8]


def test_a_token_takes_a_workspace_of_its_size():
    """For each pair, in polynomials of one limb: digits beta * next, accumulators 2 * next, a product 3 nl, two ciphertexts 2 * 2 nl, ModDown's
    2 nl, a coefficient form nl; for each row a product. A half more is room for the pieces' rounding."""
    for logN, nl, K, beta in ((10, 5, 2, 3), (16, 5, 2, 3)):
        (got,), _ = answers((logN, 50, 5, 60, K, 3), [dict(call="attn_bytes", rows=1, pairs=7, nl=nl, n1=8, n2=8, sq=0)])
        per = beta * (nl + K) + 2 * (nl + K) + 10 * nl
        assert 0 < got <= 1.5 * (7 * per + 3 * nl) * (8 << logN)


def test_the_header_documents_every_argument():
    text = open(os.path.join(ROOT, "include", "ckks_mi355.h")).read()
    doc = text[text.index("Attention over a paged cache of ciphertexts"):text.index("int ckks_kv_append(")]
    for name in ("new_lens", "lens", "k_pages", "v_pages", "page_tokens", "k_limbs", "v_limbs", "in_limbs", "window", "sinks", "bias",
                 "squarings", "square", "eps", "start", "factors", "iterations", "gain", "ct_res", "h_out", "ct_out", "o_out"):
        assert re.search(r"\b%s\b" % name, doc), name


@pytest.mark.parametrize("shape,most", [((12, 45, 5, 60, 2, 3), (21, 32)), ((13, 50, 5, 60, 2, 3), (28, 44)), ((16, 50, 5, 60, 2, 3), (28, 44))])
def test_launches_of_one_token(shape, most):
    """A key switch, a sum of rotations and a division take no more launches than they do now."""
    logN = shape[0]
    stride = (1 << (logN - 1)) // 4
    got, launched = answers(shape, [dict(APPEND, new=[1, 1]), dict(ATTN, new=[1, 1], sq=0, stride=stride), dict(NORM, gain=None, stride=stride)])
    assert [g[0] for g in got] == [0, 0, 0]
    assert len(launched[0]) == 1
    assert len(launched[1]) <= most[0] and len(launched[2]) <= most[1], [len(x) for x in launched]


@pytest.mark.parametrize("shape", [(10, 50, 5, 60, 2, 3), (12, 45, 5, 60, 2, 3), (13, 50, 5, 60, 2, 3)])
@pytest.mark.parametrize("stride", [1, 64])
def test_the_profile_names_the_kernels_that_ran(shape, stride):
    """A rotation by 1 leaves its block of 256 positions, those by multiples of 64 stay in them: 5^64 = 1 mod 2N / 256."""
    change = dict(stride=stride, profile=True)
    got, launched = answers(shape, [dict(APPEND, profile=True), dict(ATTN, **change), dict(NORM, **change)])
    for (code, _, counts), names in zip(got, launched):
        assert code == 0
        for name in ("pair_products_kernel", "weighted_values_kernel", "ct_products_kernel", "kv_append_kernel", "rot_sum_kernel",
                     "block_sum_kernel"):
            assert counts[name] == sum(name in k for k in names), name
        assert sum(counts.values()) == len(names)
    assert any(("block_sum_kernel" if stride == 64 else "rot_sum_kernel") in k for k in launched[2])


def test_the_profile_names_the_product_with_a_gain():
    got, launched = answers((13, 50, 5, 60, 2, 3), [dict(NORM, stride=64, profile=True), dict(NORM, stride=64, gain=None, profile=True)])
    for (code, _, counts), names, gains in zip(got, launched, (1, 0)):
        assert code == 0 and sum("cut_pmult_kernel" in k for k in names) == gains
        for name in ("cut_pmult_kernel", "tensor_kernel"):
            assert counts[name] == sum(name in k for k in names), name
        assert sum(counts.values()) == len(names)
