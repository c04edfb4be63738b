"""4-bit pools: decode attention without workspace for steps whose own plan has more partial rows than that call holds.
Bound as in tests/test_gpu_kv4_layer_by_layer.py."""
import numpy as np
import pytest

from test_gpu_kv4 import _randn, lib  # noqa: F401  (fixture + helpers)
from test_gpu_kv4_large_scores import exact
from test_gpu_kv4_layer_by_layer import filled

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layers", [1, 8])
@pytest.mark.parametrize("lengths,forks,d", [([12000], 16, 128), ([7000, 60, 5000], 18, 128), ([9000, 11000], 15, 64)])
def test_steps_that_have_to_be_cut_less(lib, lengths, forks, d, layers):
    import torch
    hq, hkv, T, n = 32, 8, forks + 1, sum(lengths)
    k, v = _randn((1, n, hkv, d), 1), _randn((1, n, hkv, d), 2)
    pool = filled(lib, lengths, forks, k.expand(layers, n, hkv, d), v.expand(layers, n, hkv, d), layers, hq, hkv, d)
    words = pool.plan_words()
    assert words[31] > 0                                              # an assignment of its own
    q = _randn((len(lengths) * T, hq, d), 3).cuda()
    out, lse, again = torch.full((len(lengths) * T, hq, d), 7.0, device="cuda"), torch.empty((len(lengths) * T, hq), device="cuda"), None
    for l in (0, layers - 1):
        pool.decode_attn_noalloc(q, out, lse, layer=l)
        assert again is None or torch.equal(out, again)
        again = out.clone()
    full = torch.empty((1,) + out.shape, device="cuda")
    pool.decode_attn(q[None], full, layer_begin=0, layer_count=1)
    pool.decode_attn_noalloc(q, out, lse)                             # between launches of the other assignment
    assert torch.equal(out, again)
    for r in range(len(lengths)):
        hk, hv = (x.double().cpu().numpy() for x in pool.kv_read(0, r, 0, 0, lengths[r]))
        for h in (0, 13, hq - 1):
            rows = q[r * T:(r + 1) * T, h].double().cpu().numpy()
            want, want_lse, mean_abs, ds = exact(rows, hk[:, h // 4], hv[:, h // 4], d ** -0.5)
            tol = (2.0 ** -8 + 2 * ds[:, None] + 2.0 ** -16) * (mean_abs + np.abs(want))
            for got in (out, full[0]):
                assert (np.abs(got[r * T:(r + 1) * T, h].double().cpu().numpy() - want) <= tol).all()
            assert (np.abs(lse[r * T:(r + 1) * T, h].double().cpu().numpy() - want_lse) <= 2.0 ** -8 + ds).all()
    assert pool.status() == 0
    pool.close()
