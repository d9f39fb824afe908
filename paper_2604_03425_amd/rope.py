"""Weights of ckks_rope: rotary position tables as slot vectors, in double precision on the host. Encoding them into plaintexts over
the extended basis is the caller's step, as for every pre-encoded plaintext.

A head has `head_dim` components, the first `rot_dim` of which turn in pairs: component i with i + rot_dim/2 (layout "half") or 2i
with 2i + 1 ("interleaved"). At position t the pair i turns by t * frequency[i]:
    low' = low cos - high sin,   high' = high cos + low sin,
which on slot vectors is w_0 x + sum_r w_r Rot_r(x): Rot_r brings a pair's other component into the slot.

Packing "components": component i of lane l in slot i * lanes + l (lanes = slots / head_dim). A whole head in the "half" layout then
needs one rotation, because the other component lies half of all slots away in either direction. Packing "tokens": component i of
token l in slot l * head_dim + i.
"""
import numpy as np


def rope_frequencies(rot_dim, base=10000.0, scaling=None):
    """(frequencies of the rot_dim / 2 pairs, factor of the turned components). scaling: None, or a dict of
        kind "linear":   positions divided by `factor` (position interpolation, arXiv 2306.15595);
        kind "base":     the base raised so that the slowest pair turns `factor` times slower and the fastest stays as it is (arXiv
                         2309.00071, Sec. 3);
        kind "by_parts": pairs that turn more than `fast` times over `original` positions stay, those that turn less than `slow` times
                         are slowed by `factor`, the ones between are mixed linearly in the number of turns' index; the turned
                         components grow by 0.1 ln(factor) + 1 (the same paper's rule by parts)."""
    if rot_dim < 2 or rot_dim % 2:
        raise ValueError("rot_dim must be even and positive")
    i = np.arange(rot_dim // 2)
    if scaling is None:
        return base ** (-2.0 * i / rot_dim), 1.0
    kind, factor = scaling["kind"], float(scaling["factor"])
    if factor < 1.0:
        raise ValueError("a scaling factor is at least 1")
    if kind == "linear":
        return base ** (-2.0 * i / rot_dim) / factor, 1.0
    if kind == "base":
        if rot_dim == 2:   # one pair, the fastest
            return np.ones(1), 1.0
        return (base * factor ** (rot_dim / (rot_dim - 2.0))) ** (-2.0 * i / rot_dim), 1.0
    if kind == "by_parts":
        f = base ** (-2.0 * i / rot_dim)

        def pair(turns):   # the (fractional) pair that turns so many times over the original positions
            return rot_dim * np.log(scaling["original"] / (turns * 2.0 * np.pi)) / (2.0 * np.log(base))

        lo = max(0.0, np.floor(pair(scaling.get("fast", 32.0))))
        hi = min(rot_dim - 1.0, np.ceil(pair(scaling.get("slow", 1.0))))
        mix = np.clip((i - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
        return f * (1.0 - mix) + f / factor * mix, 0.1 * np.log(factor) + 1.0
    raise ValueError("unknown scaling kind %r" % kind)


def rope_tables(slots, head_dim, positions, rot_dim=None, layout="half", packing="components", base=10000.0, scaling=None,
                factors=None):
    """(rotation steps, weights [sets][steps + 1][slots]) for ckks_rope.
    positions: [sets][lanes], the position of every lane (or token) of each set; factors: None or [sets][lanes], a factor for all
    components of a lane (the decays that linear attention wants folded into its queries and keys)."""
    rot_dim = head_dim if rot_dim is None else rot_dim
    if head_dim < 1 or slots % head_dim:
        raise ValueError("head_dim must divide the number of slots")
    if rot_dim > head_dim:
        raise ValueError("rot_dim must be at most head_dim")
    if layout not in ("half", "interleaved") or packing not in ("components", "tokens"):
        raise ValueError("layout is 'half' or 'interleaved', packing 'components' or 'tokens'")
    lanes, h = slots // head_dim, rot_dim // 2
    pos = np.asarray(positions, dtype=np.float64)
    if pos.ndim != 2 or pos.shape[1] != lanes:
        raise ValueError("positions must be [sets][%d]" % lanes)
    freq, grow = rope_frequencies(rot_dim, base, scaling)
    low, high = (np.arange(h), np.arange(h) + h) if layout == "half" else (2 * np.arange(h), 2 * np.arange(h) + 1)
    step = (h if layout == "half" else 1) * (lanes if packing == "components" else 1)
    steps = [step] if 2 * step == slots else [step, -step]
    angle = pos[..., None] * freq
    w = np.zeros((pos.shape[0], len(steps) + 1, lanes, head_dim))
    w[:, 0, :, rot_dim:] = 1.0
    w[:, 0][..., low] = w[:, 0][..., high] = grow * np.cos(angle)
    w[:, 1][..., low] = -grow * np.sin(angle)
    w[:, -1][..., high] = grow * np.sin(angle)
    if factors is not None:
        w *= np.asarray(factors, dtype=np.float64)[:, None, :, None]
    if packing == "components":
        w = w.transpose(0, 1, 3, 2)
    return steps, w.reshape(pos.shape[0], len(steps) + 1, slots)
