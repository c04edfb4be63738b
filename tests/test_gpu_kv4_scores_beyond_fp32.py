"""4-bit pools: tokens whose score with a query leaves the range of fp32.  Below it they weigh nothing, above it the row is not a number;
under a cap they count as the cap, of either sign.  Tolerances as in tests/test_gpu_kv4_large_scores.py."""
import numpy as np
import pytest

from test_gpu_kv4 import _randn, lib  # noqa: F401  (fixture + helpers)
from test_gpu_kv4_large_scores import exact, one_request

pytestmark = pytest.mark.gpu
HUGE = 2.0 ** 100


def places(n, which):
    at = {"first page": range(0, 16), "second tile": range(128, 256), "one in three": range(0, n, 3), "all but the last": range(n - 1)}[which]
    return [t for t in at if t < n]


@pytest.mark.parametrize("which", ["first page", "second tile", "one in three", "all but the last"])
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("threads,n", [(1, 40), (2, 300), (17, 3000)])
@pytest.mark.parametrize("d,flags", [(128, 0), (64, 0), (128, 2), (64, 2)])
def test_below(lib, d, flags, threads, n, cap, which):
    """Rows of 2^40 times an ordinary query over 2^-40 times ordinary keys, and some tokens' keys at -2^100 of the query's signs."""
    import torch
    sign = (1.0 - 2.0 * (torch.arange(d) % 2))[None, None, None, :]
    k = _randn((1, n, 1, d), 1).float() * 2.0 ** -40
    k[0, places(n, which)] = -HUGE * sign[0]
    pool, hk, hv = one_request(lib, d, threads, k.to(torch.bfloat16), _randn((1, n, 1, d), 2), flags, cap)
    q = (_randn((threads, 4, d), 3).float().abs() * 2.0 ** 40 * sign[0]).to(torch.bfloat16)
    q[0, 2] = 0                                                       # sees every token alike
    out = torch.full((1, threads, 4, d), 7.0, device="cuda"); lse = torch.full((1, threads, 4), 7.0, device="cuda")
    pool.decode_attn(q[None].cuda(), out, lse)
    rows = q.double().numpy().reshape(-1, d)
    want, want_lse, mean_abs, _ = exact(rows, hk, hv, d ** -0.5, cap)
    near = np.abs(hk).max(1) < 1
    ds = ((d + 8) * 2.0 ** -23 * (np.abs(rows) @ np.abs(hk[near]).T).max(1) * d ** -0.5 + 2.0 ** -21 * (1 + cap))[:, None]
    got = out[0].double().cpu().numpy().reshape(-1, d)
    assert (np.abs(got - want) <= (2.0 ** -8 + 2 * ds + 2.0 ** -16) * (mean_abs + np.abs(want))).all(), np.nanmax(np.abs(got - want))
    assert (np.abs(lse[0].double().cpu().numpy().reshape(-1) - want_lse) <= 2.0 ** -8 + ds[:, 0] + 2.0 ** -21 * np.abs(want_lse)).all()
    assert pool.status() == 0
    pool.close()


@pytest.mark.parametrize("threads,n", [(1, 20), (3, 700)])
@pytest.mark.parametrize("d,flags", [(128, 0), (64, 0), (128, 2), (64, 2)])
def test_nothing_left(lib, d, flags, threads, n):
    """Every score of a row below the range: it has nothing to attend to, as zeros and a log of zero; the others are as ever."""
    import torch
    k = -torch.ones((1, n, 1, d), dtype=torch.bfloat16) * HUGE
    pool, hk, hv = one_request(lib, d, threads, k, _randn((1, n, 1, d), 2), flags)
    q = torch.zeros((threads, 4, d))
    q[:, 1] = 2.0 ** 40
    out = torch.full((1, threads, 4, d), 7.0, device="cuda"); lse = torch.full((1, threads, 4), 7.0, device="cuda")
    pool.decode_attn(q.to(torch.bfloat16)[None].cuda(), out, lse)
    assert bool((out[0, :, 1] == 0).all()) and bool((lse[0, :, 1] == float("-inf")).all())
    mean = torch.from_numpy(hv.mean(0)).cuda()
    assert (out[0][:, [0, 2, 3]].double() - mean).abs().max() <= 2.0 ** -16 * np.abs(hv).max()
    assert (lse[0][:, [0, 2, 3]].double() - np.log(n)).abs().max() <= 2.0 ** -8
    assert pool.status() == 0
    pool.close()


@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("threads,n", [(1, 40), (2, 300), (17, 3000)])
@pytest.mark.parametrize("d,flags", [(128, 0), (64, 0), (128, 2), (64, 2)])
def test_above(lib, d, flags, threads, n, cap):
    """One token's score above the range: NaN without a cap, the cap with one; rows that do not turn to it are as ever."""
    import torch
    k = _randn((1, n, 1, d), 1).float()
    k[0, n // 2] = HUGE
    pool, hk, hv = one_request(lib, d, threads, k.to(torch.bfloat16), _randn((1, n, 1, d), 2), flags, cap)
    q = torch.zeros((threads, 4, d))
    q[threads - 1, 1] = 2.0 ** 40
    q[threads - 1, 2] = -2.0 ** 40                                    # that token's score is below the range, the others' are large
    out = torch.full((1, threads, 4, d), 7.0, device="cuda"); lse = torch.full((1, threads, 4), 7.0, device="cuda")
    pool.decode_attn(q.to(torch.bfloat16)[None].cuda(), out, lse)
    keep = np.ones((threads, 4), dtype=bool)
    keep[threads - 1, 1:3] = False
    got, got_lse = out[0].double().cpu().numpy(), lse[0].double().cpu().numpy()
    assert np.abs(got[keep] - hv.mean(0)).max() <= 2.0 ** -16 * np.abs(hv).max() and np.abs(got_lse[keep] - np.log(n)).max() <= 2.0 ** -8
    if cap:
        # Scores here are the cap or minus the cap, but for keys that cancel: a sum of d products of 2^40 has d roundings of 2^-23 of their
        # magnitudes, which is far above the cap, so such a token may come out anywhere between the two.  Its weight is then between
        # nothing and 1 of the n_top tokens at the cap, which moves out by up to 2 max |v| / n_top and lse by 1 / n_top.
        rows = q[threads - 1, 1:3].double().numpy()
        want, want_lse, mean_abs, ds = exact(rows, hk, hv, d ** -0.5, cap)
        s = rows @ hk.T * d ** -0.5
        own = (d + 8) * 2.0 ** -23 * (np.abs(rows) @ np.abs(hk).T) * d ** -0.5
        open_ones = ((np.abs(s) <= own + 10 * cap).sum(1) / np.maximum(1, (s > own + 10 * cap).sum(1)))[:, None]
        tol = (2.0 ** -8 + 2.0 ** -14) * (mean_abs + np.abs(want)) + 2 * open_ones * np.abs(hv).max()
        assert (np.abs(got[threads - 1, 1:3] - want) <= tol).all()
        assert (np.abs(got_lse[threads - 1, 1:3] - want_lse) <= 2.0 ** -8 + 2.0 ** -14 + open_ones[:, 0]).all()
    else:
        assert np.isnan(got[threads - 1, 1]).all() and not np.isfinite(got_lse[threads - 1, 1])
        s = hk @ np.full(d, -2.0 ** 40)
        assert np.abs(got[threads - 1, 2] - hv[s.argmax()]).max() <= 2.0 ** -16 * np.abs(hv).max()
    assert pool.status() == 0
    pool.close()
