"""Oracle, part 5: the 8-bit cache and capped scores in fp64.  TEST INFRASTRUCTURE — not a product path.

`Kv8Store` is a `KVStore` whose contents are what an 8-bit pool holds: e4m3 codes times a power-of-two scale per (page, kv
head) for K and for V.  The tokens of one `write` that fall into one page are taken together; their scale is the smallest
power of two that brings the largest magnitude to at most 448, within 2^-64 .. 2^63, and never less than that of the tokens
already in the page, which are rounded again when it grows.
"""
from __future__ import annotations

import numpy as np

from .attention import KVStore, _to_f32

E_MIN, E_MAX = -64, 63


def e4m3_round(y: np.ndarray) -> np.ndarray:
    """Nearest e4m3 value (ties to even, saturating at 448): four significant bits, steps of 2^-9 below 2^-6."""
    y = np.clip(np.asarray(y, dtype=np.float64), -448.0, 448.0)
    _, p = np.frexp(y)                                    # 2^(p-1) <= |y| < 2^p
    step = np.ldexp(1.0, np.maximum(p, -5) - 4)
    return np.round(y / step) * step


def scale_exponent(amax: float) -> int:
    if amax == 0:
        return E_MIN
    e = int(np.frexp(amax)[1]) - 9                        # 2^(e+8) <= amax < 2^(e+9)
    if amax > 448.0 * 2.0 ** e:
        e += 1
    return min(max(e, E_MIN), E_MAX)


class Kv8Store(KVStore):
    def __init__(self, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int):
        super().__init__(n_pages, page_size, n_kv_heads, head_dim)
        self.k = self.k.astype(np.float64)
        self.v = self.v.astype(np.float64)
        self.exp = np.zeros((2, n_pages, n_kv_heads), dtype=np.int64)
        self.nonfinite = 0

    def write(self, slots, k_new, v_new) -> None:
        new = [_to_f32(k_new).astype(np.float64), _to_f32(v_new).astype(np.float64)]
        at = 0
        while at < len(slots):
            page, off = slots[at]
            n = 1
            while at + n < len(slots) and slots[at + n] == (page, off + n):
                n += 1
            for which, store in ((0, self.k), (1, self.v)):
                x = new[which][at:at + n]
                bad = ~np.isfinite(x)
                self.nonfinite += int(bad.sum())
                x = np.where(bad, 0.0, x)
                for g in range(x.shape[1]):
                    e = scale_exponent(float(np.abs(x[:, g]).max()))
                    if off > 0:
                        old = int(self.exp[which, page, g])
                        e = max(e, old)
                        if e > old:
                            held = store[page, :off, g]
                            store[page, :off, g] = e4m3_round(held * 2.0 ** -e) * 2.0 ** e
                    self.exp[which, page, g] = e
                    store[page, off:off + n, g] = e4m3_round(x[:, g] * 2.0 ** -e) * 2.0 ** e
            at += n


def rotate(k: np.ndarray, positions, theta: float) -> np.ndarray:
    """Rotate-half embedding of k [n, heads, d] in fp64, rounded once to fp32."""
    k = _to_f32(k).astype(np.float64)
    d = k.shape[-1]
    ang = np.asarray(positions, dtype=np.float64)[:, None] * theta ** (-2.0 * np.arange(d // 2) / d)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    lo, hi = k[..., :d // 2], k[..., d // 2:]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], axis=-1).astype(np.float32)


def decode_attention_capped(model, store, queries, q, scale=None, cap=0.0, spread=None):
    """`attention.decode_attention` with scores capped by cap * tanh(s / cap) (cap = 0: as they are).  A list given as
    `spread` receives, per query, (visible tokens) x (largest softmax weight of any head)."""
    q = _to_f32(q).astype(np.float64)
    out = np.zeros(q.shape)
    lse = np.zeros(q.shape[:2])
    group = q.shape[1] // store.k.shape[2]
    scale = 1.0 / np.sqrt(q.shape[2]) if scale is None else scale
    for i, query in enumerate(queries):
        k, v = store.gather(model.visible_slots(*query))
        top = 0.0
        for h in range(q.shape[1]):
            s = (k[:, h // group] @ q[i, h]) * scale
            if cap:
                s = cap * np.tanh(s / cap)
            m = s.max()
            w = np.exp(s - m)
            out[i, h] = w @ v[:, h // group] / w.sum()
            lse[i, h] = m + np.log(w.sum())
            top = max(top, 1.0 / w.sum())
        if spread is not None:
            spread.append(top * len(k))
    return out, lse
