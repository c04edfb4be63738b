"""8-bit pools: scores far beyond what a softmax tells apart.  A row whose best token is ahead by more than the scores'
errors is that token's V to within the rounding of one weight, 2^-8."""
import numpy as np
import pytest

from test_gpu_kv8 import _pool, _randn, lib  # noqa: F401  (fixture + helpers)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("exponent", [15, 18, 20, 22, 24, 25, 26, 28, 32, 48, 80, 115])
@pytest.mark.parametrize("threads", [1, 9, 17])
@pytest.mark.parametrize("d,flags", [(128, 0), (64, 0), (128, 2)])
def test_the_best_token_takes_all(lib, d, flags, threads, exponent):
    import torch
    hq, hkv, n = 4, 1, 1000
    pool = _pool(lib, n // 16 + threads + 2, threads=threads, hq=hq, hkv=hkv, d=d, flags=flags, max_step_queries=threads)
    pool.request_begin()
    pool.kv_append_run(0, 0, n, _randn((1, n, hkv, d), 1).cuda(), _randn((1, n, hkv, d), 2).cuda())
    for _ in range(threads - 1):
        pool.thread_spawn(0)
    pool.step_begin([0] * threads, list(range(threads)), [0] + [1] * (threads - 1))
    if threads > 1:
        small = torch.full((1, threads - 1, hkv, d), 2.0 ** -10, dtype=torch.bfloat16, device="cuda")
        pool.kv_append(small, small)                                    # never the best token
    plain = _randn((1, threads, hq, d), 3)
    q = (plain.float() * 2.0 ** exponent).to(torch.bfloat16)
    q[0, 0, 1] = plain[0, 0, 1]                                         # an ordinary row among them
    q[0, threads - 1, 2] *= -1
    out = torch.full((1, threads, hq, d), float("nan"), device="cuda"); lse = torch.full((1, threads, hq), float("nan"), device="cuda")
    pool.decode_attn(q.cuda(), out, lse)
    k, v = [x.double().cpu().numpy()[:, 0] for x in pool.kv_read(0, 0, 0, 0, n)]
    rows = q[0].double().numpy().reshape(-1, d)
    s = rows @ k.T / np.sqrt(d)
    # a score's error: the sums' rounding and the split of q, on sums of at most d |q| |k|
    bound = ((d + 8) * 2.0 ** -23 + 2.0 ** -17) * d * np.abs(rows).max(1) * np.abs(k).max() / np.sqrt(d)
    best = s.argmax(1)
    second = np.partition(s, -2, axis=1)[:, -2]
    sharp = (s.max(1) - second > 2 * bound + 25) & (np.arange(len(rows)) != 1)        # n e^-25: below 2^-25
    assert sharp.sum() >= len(rows) // 2
    got, got_lse = out[0].double().cpu().numpy().reshape(-1, d), lse[0].double().cpu().numpy().reshape(-1)
    assert np.all(np.isfinite(got)) and np.all(np.isfinite(got_lse))
    assert np.all(np.abs(got[sharp] - v[best[sharp]]) <= 2.0 ** -8 * np.abs(v[best[sharp]]) + 2.0 ** -20)
    # a row that is not sharp is some mixture of V
    assert np.abs(got).max() <= (1 + 2.0 ** -7) * np.abs(v).max()
    assert np.all(np.abs(got_lse - s.max(1))[sharp] <= bound[sharp])
    w = np.exp(s[1] - s[1].max())
    assert np.abs(got[1] - w @ v / w.sum()).max() <= (2.0 ** -8 + 2 * bound[1]) * np.abs(v).max()
    assert pool.status() == 0


@pytest.mark.parametrize("d,flags", [(128, 0), (64, 0), (128, 2), (64, 2)])
def test_scores_that_leave_fp32_are_never_wrong_numbers(lib, d, flags):
    """The largest queries there are: a row is NaN, or its best token's V."""
    import torch
    hq, n = 8, 600
    pool = _pool(lib, 60, hq=hq, hkv=2, d=d, flags=flags)
    pool.request_begin()
    pool.kv_append_run(0, 0, n, (3 * _randn((1, n, 2, d), 1)).cuda(), _randn((1, n, 2, d), 2).cuda())
    pool.step_begin([0], [0], [0])
    sizes = torch.tensor([2.0 ** e for e in (112, 116, 118, 120, 122, 124, 126, 127)]).reshape(1, 1, hq, 1)
    q = (torch.sign(_randn((1, 1, hq, d), 3).float()) * sizes).to(torch.bfloat16)
    out = torch.full((1, 1, hq, d), 7.0, device="cuda"); lse = torch.full((1, 1, hq), 7.0, device="cuda")
    pool.decode_attn(q.cuda(), out, lse)
    k, v = [x.double().cpu().numpy() for x in pool.kv_read(0, 0, 0, 0, n)]
    got = out[0, 0].double().cpu().numpy()
    for h in range(hq):
        s = k[:, h // 4] @ q[0, 0, h].double().numpy()
        best = v[s.argmax(), h // 4]
        if np.isfinite(got[h]).any():
            assert np.all(np.abs(got[h] - best) <= 2.0 ** -8 * np.abs(best) + 2.0 ** -20), h
        else:
            assert np.isnan(got[h]).all() and h > 0 and not np.isfinite(lse[0, 0, h].item()), h
    assert pool.status() == 0
