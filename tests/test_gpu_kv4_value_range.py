"""4-bit pools: values of any size that the cache holds, under weights of any size.

An element is off by (2^-8 + 2 ds + 2^-16) (sum w |v| + |out|) (tests/test_gpu_kv4_large_scores.py) and, where products of weights and
values leave the range of fp32 at its lower end, by 2^-36 of its row's largest for every token."""
import numpy as np
import pytest

from test_gpu_kv4 import _randn, lib  # noqa: F401  (fixture + helpers)
from test_gpu_kv4_large_scores import exact, one_request

pytestmark = pytest.mark.gpu


def check(pool, q, hk, hv, d, cap=0.0):
    import torch
    threads = q.shape[0]
    out = torch.full((1, threads, 4, d), 7.0, device="cuda"); lse = torch.full((1, threads, 4), 7.0, device="cuda")
    for _ in range(2):
        pool.decode_attn(q[None].cuda(), out, lse)
    want, want_lse, mean_abs, ds = exact(q.double().numpy().reshape(-1, d), hk, hv, d ** -0.5, cap)
    got = out[0].double().cpu().numpy().reshape(-1, d)
    tol = (2.0 ** -8 + 2 * ds[:, None] + 2.0 ** -16) * (mean_abs + np.abs(want)) + len(hk) * 2.0 ** -36 * np.abs(want).max(1, keepdims=True)
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()
    assert (np.abs(lse[0].double().cpu().numpy().reshape(-1) - want_lse) <= 2.0 ** -8 + ds + 2.0 ** -21 * np.abs(want_lse)).all()
    assert pool.status() == 0
    pool.close()


@pytest.mark.parametrize("exponent", [112, 100, 20, -40, -80, -100])
@pytest.mark.parametrize("levels", [(6.5, 0, -5, -12), (-20, -30, -39, -41), (-43, -100, 40, 6)])
@pytest.mark.parametrize("threads,n", [(1, 1), (1, 100), (2, 300), (17, 3000), (3, 40000)])
@pytest.mark.parametrize("d,flags", [(128, 0), (64, 0), (128, 2)])
def test_values_of_any_size(lib, d, flags, threads, n, levels, exponent):
    """Rows whose scores lie around the levels (natural units) over values around 2^exponent."""
    import torch
    if flags and exponent > 100 and n > 1 << 14:
        pytest.skip("the warp-shuffle kernel adds up weighted values before it divides by the weights: 2^14 of the largest fit")
    k = (torch.ones((1, n, 1, d)) * (8 / d ** 0.5) * (1 + 0.02 * _randn((1, n, 1, 1), 4).float())).to(torch.bfloat16)
    v = (_randn((1, n, 1, d), 2).float() * 2.0 ** exponent).to(torch.bfloat16)
    if exponent > 100:
        v = v.abs()                                                   # (nothing cancels)
    pool, hk, hv = one_request(lib, d, threads, k, v, flags)
    q = torch.tensor(levels, dtype=torch.float32)[None, :, None] * torch.ones(threads, 4, d) / 8
    q *= 1 + torch.arange(threads)[:, None, None] / (16 * threads)
    check(pool, q.to(torch.bfloat16), hk, hv, d)


@pytest.mark.parametrize("cap", [5.0, 30.0])
@pytest.mark.parametrize("exponent", [112, -100])
@pytest.mark.parametrize("d", [128, 64])
def test_under_capped_scores(lib, d, exponent, cap):
    import torch
    n = 2000
    k = (torch.ones((1, n, 1, d)) * (8 / d ** 0.5) * (1 + 0.1 * _randn((1, n, 1, 1), 4).float())).to(torch.bfloat16)
    v = (_randn((1, n, 1, d), 2).float() * 2.0 ** exponent).to(torch.bfloat16)
    if exponent > 100:
        v = v.abs()
    pool, hk, hv = one_request(lib, d, 6, k, v, cap=cap)
    q = torch.tensor([40.0, 6.0, -7.0, -60.0])[None, :, None] * torch.ones(6, 4, d) / 8 * (1 + torch.arange(6)[:, None, None] / 100)
    check(pool, q.to(torch.bfloat16), hk, hv, d, cap)
