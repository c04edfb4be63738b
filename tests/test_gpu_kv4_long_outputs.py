"""4-bit pools: attention over long contexts, element by element.  The mean of n values of either sign is some n^-1/2 of one, so the bound goes
by the values' own weighted magnitudes (tests/test_gpu_kv4_large_scores.py): outputs that are off by a hundredth of themselves fail.  For
independent roundings the error is far smaller than that, which the root mean square of all of a step's outputs is held to: a weight is
off by at most 2^-8 of itself, evenly spread (root mean square at most 2^-8 / 3^1/2), so out is off by that times (sum w^2 v^2)^1/2, and by
that times (sum w^2)^1/2 |out| for the sum of the rounded weights; 2 ds and 2^-16 of sum w |v| are for scores and sums."""
import numpy as np
import pytest

from test_gpu_kv4 import _randn, forked, lib  # noqa: F401  (fixture + helpers)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prefix,threads", [(500, 1), (2047, 1), (700, 9), (900, 17), (8191, 1), (2500, 12), (1200, 40), (33000, 1)])
@pytest.mark.parametrize("hq,hkv,d,flags", [(8, 2, 128, 0), (8, 8, 64, 0), (8, 1, 64, 0), (8, 2, 128, 2)])
def test_every_element(lib, hq, hkv, d, flags, prefix, threads):
    import torch
    pool, model, store = forked(lib, threads, hq, hkv, d, prefix=prefix, flags=flags)
    q = _randn((1, threads, hq, d), 9)
    pool.step_begin([0] * threads, list(range(threads)), [0] * threads)
    out, lse = torch.full((1, threads, hq, d), 7.0, device="cuda"), torch.empty((1, threads, hq), device="cuda")
    pool.decode_attn(q.cuda(), out, lse)
    got, qf = out[0].double().cpu().numpy(), q[0].double().numpy()
    square, expected = 0.0, 0.0
    for t in sorted({0, 1, threads // 2, threads - 1} & set(range(threads))):
        k, v = store.gather(model.visible_slots(0, t))
        for h in range(hq):
            K, V = k[:, h * hkv // hq], v[:, h * hkv // hq]
            s = K @ qf[t, h] / np.sqrt(d)
            w = np.exp(s - s.max())
            total = w.sum()
            w /= total
            ds = (d + 8) * 2.0 ** -23 * (np.abs(K) @ np.abs(qf[t, h])).max() / np.sqrt(d) + 2.0 ** -21
            want, size = w @ V, w @ np.abs(V)
            err = np.abs(got[t, h] - want)
            assert (err <= (2.0 ** -8 + 2 * ds + 2.0 ** -16) * (size + np.abs(want))).all(), (t, h)
            assert abs(float(lse[0, t, h]) - (s.max() + np.log(total))) <= 2.0 ** -8 + ds
            spread = 2.0 ** -8 / np.sqrt(3)
            square += (err ** 2).sum()
            expected += ((spread * (np.sqrt((w ** 2) @ V ** 2) + np.sqrt((w ** 2).sum()) * np.abs(want)) + (2 * ds + 2.0 ** -16) * size) ** 2).sum()
    assert square <= expected, (square / expected) ** 0.5
    assert pool.status() == 0
    pool.close()
