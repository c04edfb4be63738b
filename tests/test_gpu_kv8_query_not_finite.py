"""8-bit pools: a query row with a number that is not finite comes out as NaN on every kernel, and spoils no other row."""
import pytest

from test_gpu_kv8 import _pool, _randn, lib  # noqa: F401  (fixture + helpers)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("threads,n", [(1, 1), (1, 300), (2, 3000), (9, 700), (17, 5), (17, 3000), (33, 300)])
@pytest.mark.parametrize("d,flags", [(128, 0), (64, 0), (128, 2), (64, 2), (128, 4)])
def test_rows_that_are_not_finite(lib, d, flags, threads, n, cap):
    import torch
    hq, hkv = 8, 2
    pool = _pool(lib, n // 16 + threads + 2, threads=threads, hq=hq, hkv=hkv, d=d, flags=flags, max_step_queries=threads)
    pool.request_begin()
    pool.kv_append_run(0, 0, n, _randn((1, n, hkv, d), 1).cuda(), _randn((1, n, hkv, d), 2).cuda())
    for _ in range(threads - 1):
        pool.thread_spawn(0)
    pool.step_begin([0] * threads, list(range(threads)), [0] + [1] * (threads - 1))
    if threads > 1:
        pool.kv_append(_randn((1, threads - 1, hkv, d), 3).cuda(), _randn((1, threads - 1, hkv, d), 4).cuda())
    pool.set_softcap(cap)
    q = _randn((1, threads, hq, d), 5)
    spoilt = torch.zeros((threads, hq), dtype=torch.bool)
    bad = q.clone()
    for i, x in enumerate([float("inf"), float("nan"), float("-inf")]):
        t, h = (5 * i) % threads, (3 * i + 1) % hq
        bad[0, t, h, (37 * i + d - 1) % d] = x
        spoilt[t, h] = True
    bad[0, threads - 1, 0] = float("inf")                               # and a whole row of them
    spoilt[threads - 1, 0] = True
    kind = torch.bfloat16 if flags & 4 else torch.float32
    outs = []
    for x in (q, bad):
        out = torch.full((1, threads, hq, d), 7.0, dtype=kind, device="cuda"); lse = torch.full((1, threads, hq), 7.0, device="cuda")
        pool.decode_attn(x.cuda(), out, lse)
        outs.append((out[0].cpu(), lse[0].cpu()))
    (clean, clean_lse), (out, lse) = outs
    assert torch.equal(out[~spoilt], clean[~spoilt]) and torch.equal(lse[~spoilt], clean_lse[~spoilt])
    assert bool(torch.isfinite(clean).all())
    assert bool(torch.isnan(out[spoilt]).all()) and not bool(torch.isfinite(lse[spoilt]).any())
    if not flags & 4:
        one = torch.full((threads, hq, d), 7.0, device="cuda")
        pool.decode_attn_noalloc(bad[0].cuda(), one)
        assert bool(torch.isnan(one.cpu()[spoilt]).all()) and torch.equal(one.cpu()[~spoilt], clean[~spoilt])
    assert pool.status() == 0
