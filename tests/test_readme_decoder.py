"""The cached-attention example of the README, run as it stands on the oracle's calls in the library's place: it decrypts to a layer on the
plain numbers. CPU only."""
import os
import re
from types import SimpleNamespace

import numpy as np

import attention_ref
import decoder_ref
from ckks_inputs import make_params
from harness import Keys, encode_plain_eval
from oracle import ref
from paper_2604_03425_amd.binding import attn_pairs
from paper_2604_03425_amd.norm import rmsnorm_plan

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def _library(c, s):
    def append(ctx, k, v, limbs, new, lens, k_pages, v_pages, page, k_limbs, v_limbs):
        row = at = 0
        for n, m in zip(lens, new):
            for t in range(n - m, n):
                k_pages[at + t // page][t % page], v_pages[at + t // page][t % page] = k[row][:, :k_limbs], v[row][:, :v_limbs]
                row += 1
            at += -(-n // page)

    def attn(ctx, o, q, nl, new, lens, k_pages, v_pages, page, k_limbs, v_limbs, window, sinks, bias, squarings, n1, n2, stride, mult, baby,
             giant, ws):
        assert ws == ("attn", len(q), attn_pairs(new, lens, window, sinks), nl, n1, n2, squarings)
        counts = np.cumsum([0] + [-(-n // page) for n in lens])
        assert all(x.shape == (page, 2, k_limbs, c.N) for x in k_pages) and q.shape[-2] == nl and len(k_pages) == counts[-1]
        keys, values = ([np.concatenate(p[a:b])[:n] for a, b, n in zip(counts, counts[1:], lens)] for p in (k_pages, v_pages))
        assert (n1, n2, stride) == (s.n1, s.n2, c.N // 2 // (n1 * n2))
        s.mult_key, s.baby_keys, s.giant_keys = mult, baby, giant
        o[:] = decoder_ref.attention(s, q, keys, values, new, window, sinks, bias, squarings)

    def rescale(ctx, out, x, B, nl, ws):
        assert x.shape == (B, 2, nl, c.N)
        out[:] = c.rescale(x)

    def norm(ctx, out, h, x, res, gain, square, eps, start, factors, B, nl, n1, n2, stride, mult, baby, giant, ws):
        assert ws == ("norm", B, nl, n1, n2, len(factors)) and x.shape == res.shape == h.shape == (B, 2, nl, c.N)
        assert gain.shape == (nl - 2 * len(factors), c.N)
        out[:], h[:] = decoder_ref.rmsnorm(s, x, res, gain, square, eps, start, factors)

    return SimpleNamespace(ckks_kv_append=append, ckks_attn_paged=attn, ckks_rescale=rescale, ckks_rmsnorm=norm, attn_pairs=attn_pairs,
                           rmsnorm_plan=rmsnorm_plan, OP_RESCALE=5)


def test_the_layer_decrypts_to_itself():
    """Two sequences, one new token each, a window and a sink. Errors: encryption and key switches at 2^-25 of their unit or less (scale 2^45), a
    norm's start as the plan says."""
    n1, n2, d, nl, page = 2, 2, 4, 9, 2
    p = make_params(10, 9, 50, 3, 60, 3)
    c, N = ref.RefContext(p), p.N
    lanes = N // 2 // d
    keys = Keys(p, c, 11)
    s = attention_ref.Shape(p, c, n1, n2, lanes)
    rng = np.random.default_rng(5)
    lens, new, scale, window, sinks, bias, eps = [4, 2], [1, 1], 2.0 ** 45, 2, 1, 1.0, .05
    L = nl - 2
    q = rng.uniform(-.5, .5, (2, d, lanes))
    k, v = ([rng.uniform(-.5, .5, (n, d, lanes)) for n in lens] for _ in range(2))
    enc = lambda x, sc, limbs: keys.encrypt_slots(x.reshape(-1), sc, limbs)   # noqa: E731
    k_pages, v_pages = ([np.zeros((page, 2, limbs, N), dtype=np.uint64) for n in lens for _ in range(-(-n // page))] for limbs in (nl, L))
    first = 0
    for b, n in enumerate(lens):
        for t in range(n - 1):
            k_pages[first + t // page][t % page], v_pages[first + t // page][t % page] = enc(k[b][t], scale, nl), enc(v[b][t], scale, L)
        first += -(-n // page)
    o = []
    for b, n in enumerate(lens):
        see = decoder_ref.visible(n - 1, window, sinks)
        o.append(sum(((q[b] * k[b][u]).sum(axis=0) + bias) ** 2 * v[b][u] for u in see))
    residual, gain = rng.uniform(-1, 1, (2, d, lanes)), rng.uniform(.5, 2, d)
    h = np.stack(o) + residual
    mean = (h * h).mean(axis=1) + eps
    at = (scale ** 2 / p.q[nl - 1]) ** 2 / p.q[nl - 2] * scale / p.q[L - 1]
    block, = [b for b in re.findall(r"```python\n(.*?)```", open(README).read(), flags=re.S) if "ckks_attn_paged" in b]
    names = dict(ck=_library(c, s), p=p, N=N, n1=n1, n2=n2, lanes=lanes, page_tokens=page, window=window, sinks=sinks, score_bias=bias, eps=eps,
                 ctx=SimpleNamespace(workspace=lambda *a: None, attn_workspace=lambda *a: ("attn",) + a, rmsnorm_workspace=lambda *a: ("norm",) + a),
                 empty=lambda *shape: np.empty(shape, dtype=np.uint64), evk_mult=keys.relin_key(),
                 evk_baby=[keys.rotation_key(g) for g in s.baby], evk_giant=[keys.rotation_key(g) for g in s.giant])
    exec(block, names)
    pt = encode_plain_eval(c, np.repeat(gain, lanes), float(p.q[L - 4]), L - 3)
    last = lambda x: np.stack([enc(x[b][-1], scale, nl) for b in range(2)])   # noqa: E731
    out, stream, out_scale, stream_scale = names["decoder_layer"](
        np.stack([enc(x, scale, nl) for x in q]), last(k), last(v), new, lens, k_pages, v_pages, np.stack([enc(x, at, L - 1) for x in residual]),
        pt, mean.min(), mean.max(), nl, scale)
    assert abs(stream_scale / at - 1) < 1e-12
    for b in range(2):
        got = keys.decrypt_slots(stream[b], stream_scale).real.reshape(d, lanes)
        noise = 2.0 ** 20 / at
        assert np.abs(got - h[b]).max() < 64 * noise
        plan = rmsnorm_plan(p.q, L - 1, at, d, mean.min(), mean.max(), 1, eps)
        want = h[b] / np.sqrt(mean[b]) * gain[:, None]
        got = keys.decrypt_slots(out[b], out_scale).real.reshape(d, lanes)
        assert np.abs(got - want).max() < plan["error"] * np.abs(want).max() + 2.0 ** 14 * noise, (np.abs(got - want).max(), plan["error"])
