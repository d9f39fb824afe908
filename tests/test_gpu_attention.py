"""Rotary positions and linear attention on the GPU against the oracle, residue for residue: every ring and arithmetic kind, states
absent, separate and in place, decays, levels below the top, batches and splits of the head of every parity, work in slices."""
import numpy as np
import pytest
import torch

import attention_ref as ref_attention
from ckks_inputs import CkksParams, find_ntt_primes, find_psi, galois_element, make_params, uniform_residues
from gpu_util import assert_same, to_dev, to_host
from oracle import ref

pytestmark = pytest.mark.gpu


def _mixed(logN):
    """Main primes of all three kinds (below 2^50, below 2^52, 60 bits) and special primes of two."""
    q = find_ntt_primes(49, 2, logN) + find_ntt_primes(51, 2, logN) + find_ntt_primes(60, 1, logN)
    p = find_ntt_primes(59, 2, logN) + find_ntt_primes(45, 1, logN)
    return CkksParams(logN=logN, q=q, p=p, dnum=2, psi=[find_psi(m, logN) for m in q + p])


PARAMS = {
    "ring10": lambda: make_params(10, 4, 50, 2, 60, 2),
    "ring11": lambda: make_params(11, 3, 60, 1, 60, 3),
    "ring12": lambda: make_params(12, 5, 45, 2, 60, 3),
    "ring12_steps": lambda: make_params(12, 12, 50, 4, 60, 3),   # large batches of it leave the whole-limb kernels
    "ring13": lambda: make_params(13, 4, 50, 2, 60, 2),
    "ring13_int": lambda: make_params(13, 5, 60, 2, 60, 3),
    "ring13_mixed": lambda: _mixed(13),
    "ring13_fp": lambda: make_params(13, 4, 45, 2, 48, 2),       # special primes in double precision too
    "ring14": lambda: make_params(14, 7, 50, 3, 60, 3),
    "ring14_wide": lambda: make_params(14, 10, 50, 10, 60, 1),   # conversions of more than 8 sources
    "ring15": lambda: make_params(15, 5, 55, 3, 60, 2),
    "ring16": lambda: make_params(16, 4, 50, 2, 60, 2),
    "ring17": lambda: make_params(17, 2, 50, 1, 60, 2),
}
_contexts = {}


def contexts(name):
    import paper_2604_03425_amd as ck
    if name not in _contexts:
        p = PARAMS[name]()
        ref.set_threads(8)
        _contexts[name] = (p, ref.RefContext(p), ck.Context(p, 0))
    return _contexts[name]


ONE_ROTATION = [("ring13", 3, 4, 2, 1), ("ring13_int", 4, 3, 1, 1), ("ring13_mixed", 5, 4, 4, 1), ("ring13_mixed", 4, 3, 1, 1),
                ("ring13_fp", 3, 4, 2, 1), ("ring14_wide", 10, 3, 3, 1), ("ring15", 4, 2, 1, 1), ("ring16", 1, 6, 2, 1)]


@pytest.mark.parametrize("name,nl,B,npt,R", ONE_ROTATION + [
    ("ring10", 4, 1, 1, 1), ("ring10", 1, 3, 1, 2), ("ring10", 3, 2, 2, 33), ("ring10", 2, 2, 1, 65), ("ring11", 2, 4, 2, 2),
    ("ring12", 5, 8, 1, 1), ("ring12", 3, 3, 3, 2), ("ring13", 4, 5, 1, 2), ("ring13", 2, 1, 1, 0), ("ring13_int", 5, 2, 1, 2),
    ("ring13_int", 3, 6, 3, 1), ("ring13_mixed", 5, 3, 3, 2), ("ring13_mixed", 3, 1, 1, 34), ("ring13_fp", 4, 4, 2, 2),
    ("ring14", 7, 2, 1, 2), ("ring14", 4, 7, 1, 1), ("ring14_wide", 10, 2, 2, 2), ("ring14_wide", 9, 1, 1, 1),
    ("ring15", 5, 3, 1, 2), ("ring16", 4, 1, 1, 1), ("ring16", 3, 9, 3, 2), ("ring17", 2, 1, 1, 2)])
def test_rope_matches_the_oracle(name, nl, B, npt, R):
    import paper_2604_03425_amd as ck
    p, rc, ctx = contexts(name)
    ext = p.q[:nl] + p.p
    ct = uniform_residues(11, p.q[:nl], (B, 2), p.N)
    w = uniform_residues(12, ext, (npt, R + 1), p.N)
    steps = [(3 * r + 1) * (-1) ** r for r in range(R)]
    gs = [galois_element(s % (p.N // 2), p.logN) for s in steps]
    evks = [uniform_residues(20 + r % 3, p.moduli, (p.dnum, 2), p.N) for r in range(R)]
    want = rc.rope(ct, w, gs, evks)
    dev = [to_dev(e) for e in evks]
    ws = ctx.workspace(ck.OP_ROPE, B, nl).random_()
    out = torch.full((B, 2, nl, p.N), -1, dtype=torch.int64, device="cuda")
    ck.ckks_rope(ctx, out, to_dev(ct), B, nl, to_dev(w), npt, gs, dev, ws)
    assert_same(to_host(out), want, "rope %s" % name)


def _run(op, name, nl, B, C, n1, n2, state, decay, in_place=False, check=None):
    import paper_2604_03425_amd as ck
    p, rc, ctx = contexts(name)
    stride = max(1, (p.N // 2) // (n1 * n2))
    s = ref_attention.Shape(p, rc, n1, n2, stride, seed=100 + C)
    q, k, v = (s.cts((C, B), nl) for _ in range(3))
    S = s.cts((n2, n1, B), nl) if state else None
    dec = s.draw(p.q[:nl], ()) if decay else None
    dev = lambda x: None if x is None else to_dev(x)   # noqa: E731
    keys = (to_dev(s.mult_key), [to_dev(x) for x in s.baby_keys], [to_dev(x) for x in s.giant_keys],
            [to_dev(x) for x in s.value_keys])
    dS = dev(S)
    o = torch.full((C, B, 2, nl, p.N), -1, dtype=torch.int64, device="cuda")
    out = dS if in_place else torch.full((n2, n1, B, 2, nl, p.N), -1, dtype=torch.int64, device="cuda")
    dq, dk, dv, dd = dev(q), dev(k), dev(v), dev(dec)
    ws = ctx.linattn_workspace(ck.OP_LINATTN_STEP if op == "step" else ck.OP_LINATTN_CHUNK, C, B, nl, n1, n2).random_()
    if op == "step":
        ck.ckks_linattn_step(ctx, o, out, dq, dk, dv, dS, dd, B, nl, n1, n2, stride, *keys, ws)
    else:
        ck.ckks_linattn_chunk(ctx, o, out, dq, dk, dv, dS, dd, C, B, nl, n1, n2, stride, *keys, ws)
    got_o, got_s = to_host(o), to_host(out)
    check = list(range(B)) if check is None else check    # the lanes' ciphertexts are independent of each other
    pick = lambda x, at: None if x is None else np.ascontiguousarray(np.take(x, check, axis=at))   # noqa: E731
    q, k, v, S = pick(q, 1), pick(k, 1), pick(v, 1), pick(S, 2)
    if op == "step":
        want_o, want_s = ref_attention.step(s, q[0], k[0], v[0], S, dec)
        want_o = want_o[None]
    else:
        want_o, want_s = ref_attention.chunk(s, q, k, v, S, dec)
    assert_same(got_o[:, check], want_o, "%s o %s" % (op, name))
    assert_same(got_s[:, :, check], want_s, "%s state %s" % (op, name))
    if not in_place and S is not None:
        assert_same(to_host(dS)[:, :, check], S, "state_in is left alone")


CASES = [("ring10", 4, 1, 2, 2, True, True), ("ring10", 3, 3, 3, 2, True, False), ("ring10", 2, 2, 1, 3, False, True),
         ("ring10", 1, 1, 4, 1, True, False), ("ring10", 4, 1, 1, 1, True, True), ("ring11", 3, 2, 2, 2, False, False),
         ("ring12", 5, 2, 2, 3, True, True), ("ring13", 4, 1, 2, 2, True, True), ("ring13_int", 4, 2, 2, 2, True, False),
         ("ring13_mixed", 5, 1, 3, 2, True, True), ("ring13_fp", 3, 2, 2, 2, False, True), ("ring14", 6, 1, 2, 2, True, False),
         ("ring14_wide", 10, 1, 2, 1, True, True), ("ring15", 3, 1, 1, 2, True, False)]


@pytest.mark.parametrize("name,nl,B,n1,n2,state,decay", CASES)
def test_step_matches_the_oracle(name, nl, B, n1, n2, state, decay):
    _run("step", name, nl, B, 1, n1, n2, state, decay)


@pytest.mark.parametrize("C,case", [(1, CASES[0]), (3, CASES[0]), (2, CASES[1]), (4, CASES[2]), (2, CASES[3]), (3, CASES[4]),
                                    (2, CASES[5]), (3, CASES[6]), (2, CASES[7]), (2, CASES[8]), (2, CASES[9]), (3, CASES[10]),
                                    (2, CASES[11]), (1, CASES[12]), (2, CASES[13])])
def test_chunk_matches_the_oracle(C, case):
    name, nl, B, n1, n2, state, decay = case
    _run("chunk", name, nl, B, C, n1, n2, state, decay)


@pytest.mark.parametrize("op,C", [("step", 1), ("chunk", 2)])
@pytest.mark.parametrize("name", ["ring10", "ring13"])
def test_state_in_place(op, C, name):
    _run(op, name, 3, 2, C, 2, 2, True, True, in_place=True)


def test_work_in_slices():
    """More ciphertexts than one key switch takes at a time: products of the state, tokens of the read, pairs of the scores."""
    _run("step", "ring16", 2, 24, 1, 3, 2, True, True, check=[0, 23])
    _run("chunk", "ring16", 2, 40, 3, 2, 1, True, False, check=[0, 39])


def test_ring_12_in_both_forms():
    """By whole limbs and, from 64 ciphertexts of 12 limbs on, one kernel per step."""
    test_rope_matches_the_oracle("ring12_steps", 12, 3, 3, 2)
    test_rope_matches_the_oracle("ring12_steps", 12, 66, 2, 2)
    _run("step", "ring12_steps", 12, 66, 1, 2, 1, True, True, check=[0, 65])
    _run("chunk", "ring12_steps", 12, 33, 2, 1, 2, True, False, check=[0, 32])
    _run("chunk", "ring12_steps", 11, 1, 2, 2, 2, True, False)


def test_work_in_more_slices():
    """Several slices at each place: rows of the state that make one and a half, pieces of a row, tokens one slice after another."""
    _run("step", "ring16", 2, 24, 1, 3, 3, True, True, check=[0, 23])
    _run("step", "ring16", 1, 100, 1, 2, 1, True, False, check=[0, 99])
    _run("chunk", "ring16", 1, 50, 3, 2, 1, True, True, check=[0, 49])


def test_a_chunk_of_one_token_and_a_longer_one_agree():
    """Outputs depend on no later token."""
    import paper_2604_03425_amd as ck
    p, rc, ctx = contexts("ring10")
    s = ref_attention.Shape(p, rc, 2, 2, p.N // 8, seed=5)
    C, B, nl = 70, 1, 2
    q, k, v = (to_dev(s.cts((C, B), nl)) for _ in range(3))
    keys = (to_dev(s.mult_key), [to_dev(x) for x in s.baby_keys], [to_dev(x) for x in s.giant_keys],
            [to_dev(x) for x in s.value_keys])
    outs = []
    for n in (1, 9, C):
        o = torch.empty((n, B, 2, nl, p.N), dtype=torch.int64, device="cuda")
        st = torch.empty((2, 2, B, 2, nl, p.N), dtype=torch.int64, device="cuda")
        ck.ckks_linattn_chunk(ctx, o, st, q[:n], k[:n], v[:n], None, None, n, B, nl, 2, 2, p.N // 8, *keys,
                              ctx.linattn_workspace(ck.OP_LINATTN_CHUNK, n, B, nl, 2, 2))
        outs.append(to_host(o))
    assert (outs[0][0] == outs[2][0]).all() and (outs[1] == outs[2][:9]).all()
    # the last token from its definition
    h = lambda x: x.cpu().numpy().view(np.uint64)   # noqa: E731
    d = ref_attention._products(s, [(ref_attention.score(s, h(q[C - 1]), h(k[u])), h(v[u])) for u in range(C)])
    assert_same(outs[2][C - 1], s.c.relin(d, s.mult_key), "token 69")


def test_refusals():
    import paper_2604_03425_amd as ck
    p, rc, ctx = contexts("ring10")
    nl, B, n1, n2, N = 2, 2, 2, 2, p.N
    new = lambda *shape: torch.zeros(shape, dtype=torch.int64, device="cuda")   # noqa: E731
    key = new(p.dnum, 2, len(p.moduli), N)
    ct, w = new(B, 2, nl, N), new(2, 2, nl + len(p.p), N)
    ws = ctx.workspace(ck.OP_ROPE, B, nl)

    def rope(code, out=None, ct_in=ct, B=B, nl=nl, w=w, npt=1, gs=(5,), keys=(key,), ws=ws):
        with pytest.raises(ck.CkksError) as e:
            ck.ckks_rope(ctx, new(4, 2, 4, N) if out is None else out, ct_in, B, nl, w, npt, list(gs), list(keys), ws)
        assert e.value.code == code, e.value

    rope(-1, out=ct)                       # overlaps the input
    rope(-1, gs=(4,))
    rope(-1, gs=(2 * N + 1,))
    rope(-2, npt=0)
    rope(-2, npt=3, w=new(3, 2, 4, N), ct_in=new(4, 2, nl, N), B=4)
    rope(-2, nl=5, ct_in=new(2, 2, 5, N), out=new(2, 2, 5, N), w=new(2, 2, 7, N))
    rope(-2, B=0)
    rope(-3, ws=ws[:-64])
    rope(-3, ws=ws[1:])
    with pytest.raises(ValueError):
        ck.ckks_rope(ctx, new(B, 2, nl, N), ct, B, nl, w, 1, [5, 25], [key], ws)
    with pytest.raises(ValueError):
        ck.ckks_rope(ctx, new(B, 2, nl, N), ct, B, nl, w[:1], 2, [5], [key], ws)

    q, state = new(1, B, 2, nl, N), new(n2, n1, B, 2, nl, N)
    lws = ctx.linattn_workspace(ck.OP_LINATTN_CHUNK, 1, B, nl, n1, n2)
    good = dict(o=new(1, B, 2, nl, N), out=new(n2, n1, B, 2, nl, N), q=q, k=q, v=q, state=state, decay=None, C=1, B=B, nl=nl, n1=n1,
                n2=n2, stride=N // 8, ws=lws, baby=[key], giant=[key], value=[key])

    def linattn(code, op, **change):
        a = dict(good, **change)
        tail = (a["B"], a["nl"], a["n1"], a["n2"], a["stride"], key, a["baby"], a["giant"], a["value"], a["ws"])
        head = (ctx, a["o"], a["out"], a["q"], a["k"], a["v"], a["state"], a["decay"])
        with pytest.raises(ck.CkksError) as e:
            if op == "step":
                ck.ckks_linattn_step(*head, *tail)
            else:
                ck.ckks_linattn_chunk(*head, a["C"], *tail)
        assert e.value.code == code, e.value

    for op in ("step", "chunk"):
        linattn(-1, op, o=q)
        linattn(-1, op, out=state.view(-1)[N:], state=state.view(-1), B=1)       # overlaps state_in without being it
        linattn(-1, op, o=good["out"])
        linattn(-1, op, decay=good["o"])
        linattn(-2, op, stride=0)
        linattn(-2, op, B=0)
        linattn(-3, op, ws=lws[:64])
        linattn(-3, op, ws=lws[1:])
    linattn(-2, "chunk", C=0)
    assert ck.ckks_linattn_workspace_bytes(ctx, ck.OP_LINATTN_STEP, 2, B, nl, n1, n2) == 0
    assert ck.ckks_linattn_workspace_bytes(ctx, ck.OP_HROT, 1, B, nl, n1, n2) == 0
    assert ck.ckks_linattn_workspace_bytes(ctx, ck.OP_LINATTN_CHUNK, 0, B, nl, n1, n2) == 0
    assert ck.ckks_linattn_workspace_bytes(ctx, ck.OP_LINATTN_CHUNK, 5000, B, nl, n1, n2) == 0
    assert ck.ckks_linattn_workspace_bytes(ctx, ck.OP_LINATTN_CHUNK, 4000, 20, nl, n1, n2) == 0
    with pytest.raises(ValueError):
        ck.ckks_linattn_step(ctx, good["o"], good["out"], q, q, q, None, None, B, nl, n1, n2, 1, key, [], [key], [key], lws)
    with pytest.raises(TypeError):
        ck.ckks_linattn_step(ctx, good["o"], good["out"], q.cpu(), q, q, None, None, B, nl, n1, n2, 1, key, [key], [key], [key], lws)


def test_calls_on_another_stream_and_in_a_graph():
    """The calls enqueue on the current stream alone and allocate nothing, so they can be captured; replays give the same result."""
    import paper_2604_03425_amd as ck
    p, rc, ctx = contexts("ring13")
    n1 = n2 = 2
    nl, B, C = 3, 2, 2
    s = ref_attention.Shape(p, rc, n1, n2, p.N // 8, seed=9)
    q, k, v = (to_dev(s.cts((C, B), nl)) for _ in range(3))
    S = to_dev(s.cts((n2, n1, B), nl))
    keys = (to_dev(s.mult_key), [to_dev(x) for x in s.baby_keys], [to_dev(x) for x in s.giant_keys],
            [to_dev(x) for x in s.value_keys])
    ws = ctx.linattn_workspace(ck.OP_LINATTN_CHUNK, C, B, nl, n1, n2)
    o, out = torch.empty_like(q), torch.empty_like(S)

    def call():
        ck.ckks_linattn_chunk(ctx, o, out, q, k, v, S, None, C, B, nl, n1, n2, p.N // 8, *keys, ws)

    call()
    want = to_host(o).copy(), to_host(out).copy()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o.fill_(-1)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    assert (to_host(o) == want[0]).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        o.fill_(-1), out.fill_(-1), ws.random_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert (to_host(o) == want[0]).all() and (to_host(out) == want[1]).all()


def test_the_example_decrypts_to_plain_attention():
    """Errors as in test_oracle_attention.py: 2^-26 an input, on a ring of 2^12 twice that; T d products of three inputs, decay^-3 at most."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "encrypted_linear_attention.py")
    spec = importlib.util.spec_from_file_location("encrypted_linear_attention", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    errors = mod.main(logN=12, head=8, tokens=3, new=2, quiet=True)
    assert len(errors) == 5 and max(errors) < 5 * 8 * 3 * 3 * 2.0 ** -25, errors


@pytest.mark.parametrize("knob,value", [(0, 0), (1, 1), (2, 1), (2, 2), (3, 1), (4, 0), (5, 1)])
@pytest.mark.parametrize("name", ["ring13_mixed", "ring16"])
def test_tuning_knobs_change_no_result(name, knob, value):
    import paper_2604_03425_amd as ck
    p, rc, ctx = contexts(name)
    default = {0: -1, 1: 0, 2: 0, 3: 2, 4: 1, 5: 0}[knob]
    nl = min(3, len(p.q))
    ck.ckks_tune_set(ctx, knob, value)
    try:
        test_rope_matches_the_oracle(name, nl, 2, 1, 1)
        test_rope_matches_the_oracle(name, nl, 2, 2, 2)
        _run("step", name, nl, 1, 1, 2, 1, True, True)
        _run("chunk", name, nl, 1, 2, 1, 2, True, False)
    finally:
        ck.ckks_tune_set(ctx, knob, default)


def test_a_state_beyond_2_to_32_words():
    """64 components of 24 lanes' ciphertexts at the benchmark's ring, 38 GB of state: the last ciphertext alone gives the same."""
    import paper_2604_03425_amd as ck
    from ckks_inputs import config_params
    p = config_params("keyswitch_micro")
    ctx = ck.Context(p, 0)
    n1 = n2 = 8
    nl, B, N = 24, 24, p.N
    gen = torch.Generator(device="cuda").manual_seed(3)

    def residues(lead, moduli):
        x = torch.empty(tuple(lead) + (len(moduli), N), dtype=torch.int64, device="cuda")
        for i, m in enumerate(moduli):
            x[..., i, :].random_(0, m, generator=gen)
        return x

    key = lambda: residues((p.dnum, 2), p.moduli)   # noqa: E731
    keys = (key(), [key()] * (n1 - 1), [key()] * (n2 - 1), [key()] * (n2 - 1))
    q, k, v = (residues((1, B, 2), p.q) for _ in range(3))
    decay = residues((), p.q)
    state = residues((n2, n1, B, 2), p.q)
    assert state.numel() > 1 << 32
    last = state[:, :, -1:].contiguous()
    o = torch.empty_like(q)
    ck.ckks_linattn_step(ctx, o, state, q, k, v, state, decay, B, nl, n1, n2, N // 128, *keys,
                         ctx.linattn_workspace(ck.OP_LINATTN_STEP, 1, B, nl, n1, n2))
    one, ql, kl, vl = torch.empty_like(o[:, :1]), *(x[:, -1:].contiguous() for x in (q, k, v))
    ck.ckks_linattn_step(ctx, one, last, ql, kl, vl, last, decay, 1, nl, n1, n2, N // 128, *keys,
                         ctx.linattn_workspace(ck.OP_LINATTN_STEP, 1, 1, nl, n1, n2))
    torch.cuda.synchronize()
    assert torch.equal(o[:, -1:], one) and torch.equal(state[:, :, -1:], last)
    del state, last, ctx
    torch.cuda.empty_cache()
