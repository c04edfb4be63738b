"""Oracle, part 6: the 4-bit cache and the forms of rotary embedding in fp64.  TEST INFRASTRUCTURE — not a product path.

`Kv4Store` is a `KVStore` whose contents are what a 4-bit pool holds: for every 32 neighbouring elements of a token's K or V of
one kv head, whole numbers -7 .. 7 times the smallest number of five significant bits that is at least a seventh of the largest
magnitude, within 2^-110 .. 31 * 2^106.
"""
from __future__ import annotations

import math

import numpy as np

from .attention import KVStore, _to_f32

GROUP, TOP = 32, 7
SCALE_MIN, SCALE_MAX = 2.0 ** -110, 31 * 2.0 ** 106


def scales(x: np.ndarray) -> np.ndarray:
    """x [..., dim] fp64 -> [..., dim / 32]."""
    amax = np.abs(x.reshape(x.shape[:-1] + (x.shape[-1] // GROUP, GROUP))).max(-1)
    m, e = np.frexp(amax / TOP)                            # amax is an fp32 number: 53 bits tell a seventh of it from its neighbours
    return np.clip(np.ldexp(np.ceil(m * 32) / 32, e), SCALE_MIN, SCALE_MAX)


def held(x: np.ndarray) -> np.ndarray:
    """What a 4-bit pool holds of x [..., dim] (fp64, finite)."""
    s = np.repeat(scales(x), GROUP, axis=-1)
    return np.clip(np.round(x / s), -TOP, TOP) * s


class Kv4Store(KVStore):
    def __init__(self, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int):
        super().__init__(n_pages, page_size, n_kv_heads, head_dim)
        self.k = self.k.astype(np.float64)
        self.v = self.v.astype(np.float64)
        self.nonfinite = 0

    def write(self, slots, k_new, v_new) -> None:
        new = [_to_f32(k_new).astype(np.float64), _to_f32(v_new).astype(np.float64)]
        for which, store in ((0, self.k), (1, self.v)):
            bad = ~np.isfinite(new[which])
            self.nonfinite += int(bad.sum())
            x = held(np.where(bad, 0.0, new[which]))
            for i, (page, off) in enumerate(slots):
                store[page, off] = x[i]


USUAL = {"layout": "half", "rotary_dim": 0, "scaling": "none", "factor": 1.0, "original_length": 0.0, "low": 1.0, "high": 4.0,
         "magnitude": 0.0}


def frequencies(dim: int, theta: float, form: dict):
    """(f_i of every rotated pair, magnitude) of a form, written out case by case."""
    form = {**USUAL, **form}
    R = form["rotary_dim"] or dim
    factor, length, low, high = form["factor"], form["original_length"], form["low"], form["high"]
    if form["scaling"] == "base":
        theta = theta * factor ** (R / (R - 2))
    f = theta ** (-2.0 * np.arange(R // 2) / R)
    turns = length * f / (2 * math.pi)
    if form["scaling"] == "linear":
        f = f / factor
    elif form["scaling"] == "wavelength":
        between = (turns - low) / (high - low)
        f = np.where(turns > high, f, np.where(turns < low, f / factor, f * (between + (1 - between) / factor)))
    elif form["scaling"] == "ramp":
        p = lambda t: R * math.log(length / (2 * math.pi * t)) / (2 * math.log(theta))
        first, last = max(0, math.floor(p(high))), min(R - 1, math.ceil(p(low)))
        if last <= first:
            last = first + 0.001
        stretched = np.clip((np.arange(R // 2) - first) / (last - first), 0, 1)
        f = f * (1 - stretched) + f / factor * stretched
    size = form["magnitude"] or (0.1 * math.log(factor) + 1 if form["scaling"] == "ramp" else 1.0)
    return f, size


def rotate_form(x, positions, theta: float, form: dict) -> np.ndarray:
    """x [n, heads, dim] turned by its tokens' positions, in fp64."""
    x = _to_f32(x).astype(np.float64)
    f, size = frequencies(x.shape[-1], theta, form)
    R = 2 * len(f)
    z = size * np.exp(1j * np.asarray(positions, dtype=np.float64)[:, None, None] * f)
    out = x.copy()
    pairs = (slice(0, R // 2), slice(R // 2, R)) if {**USUAL, **form}["layout"] == "half" else (slice(0, R, 2), slice(1, R, 2))
    turned = (x[..., pairs[0]] + 1j * x[..., pairs[1]]) * z
    out[..., pairs[0]], out[..., pairs[1]] = turned.real, turned.imag
    return out
