"""Capped scores: a row's result is its own, whatever its neighbours, the pages' unused tails and the size of its query are."""
import numpy as np
import pytest

from oracle import KVStore, PoolModel
from oracle.kv8 import Kv8Store, decode_attention_capped
from test_gpu_kv8 import _randn, lib  # noqa: F401  (fixture + helper)

pytestmark = pytest.mark.gpu

KINDS = [(128, 8), (64, 8), (128, 8 | 2), (128, 0), (64, 0)]             # head_dim, flags: 8 = 8-bit pool, 2 = warp-shuffle kernel


def _attend(lib, pool, q):
    import torch
    out = torch.full(q.shape, float("nan"), device="cuda"); lse = torch.empty(q.shape[:3], device="cuda")
    pool.decode_attn(q, out, lse)
    return out, lse


@pytest.mark.parametrize("cap", [1e-3, 0.05, 0.5, 50.0])
@pytest.mark.parametrize("d,flags", KINDS)
def test_scores_of_zero_stay_zero(lib, d, flags, cap):
    """Keys of zeros in a page with a huge one: their scores stay 0 under a cap whatever is in q, the huge key's is at most cap.
    Weights are off by at most 2^-8 (2^-7 where they are divided by the sum of the rounded ones), capped scores by 2^-20 of the
    cap or 2^-15 of themselves (tanh does not stretch the 2^-17 or so that the products carry)."""
    import torch
    hq, n = 8, 50
    pool = lib.Pool(1, hq, 2, d, 8, 1, 2, 6, flags=flags)
    model = PoolModel(8, 16)
    store = (Kv8Store if flags & 8 else KVStore)(8, 16, 2, d)
    signs = 1.0 - 2.0 * (torch.arange(d) % 2)
    k, v = torch.zeros((1, n, 2, d), dtype=torch.bfloat16), _randn((1, n, 2, d), 2)
    k[0, 20] = (signs * 2.0 ** 60).to(torch.bfloat16)
    pool.request_begin(); model.request_begin()
    pool.kv_append_run(0, 0, n, k.cuda(), v.cuda())
    store.write(model.append_run(0, 0, n), k[0], v[0])
    sizes = torch.tensor([0.0, 2.0 ** -133, 2.0 ** -126, 2.0 ** -60, 1.0, 2.0 ** 60, 2.0 ** 120, 3.3e38]).reshape(1, 1, hq, 1)
    q = (signs * sizes).to(torch.bfloat16)
    pool.step_begin([0], [0], [0])
    pool.set_softcap(cap)
    out, lse = _attend(lib, pool, q.cuda())
    want, want_lse = decode_attention_capped(model, store, [(0, 0)], q[0], cap=cap)
    ds = 2.0 ** -15 * cap
    weights = 2.0 ** -8 if flags & 8 else 2.0 ** -7
    assert np.abs(out[0].double().cpu().numpy() - want).max() <= (weights + 2 * ds + 2.0 ** -20) * np.abs(store.v).max()
    assert np.abs(lse[0].double().cpu().numpy() - want_lse).max() <= ds + (2.0 ** -18 if flags & 8 else 2.0 ** -8)
    assert pool.status() == 0


@pytest.mark.parametrize("threads", [2, 9, 17])
@pytest.mark.parametrize("d,flags", KINDS)
def test_a_row_beyond_the_cap_leaves_the_others_as_they_are(lib, d, flags, threads):
    import torch
    hq, n = 8, 900
    pool = lib.Pool(1, hq, 2, d, 80, 1, threads, 2 * threads + 2, flags=flags, max_step_queries=threads)
    pool.request_begin()
    pool.kv_append_run(0, 0, n, _randn((1, n, 2, d), 1).cuda(), _randn((1, n, 2, d), 2).cuda())
    for _ in range(threads - 1):
        pool.thread_spawn(0)
    pool.step_begin([0] * threads, list(range(threads)), [0] + [1] * (threads - 1))
    pool.kv_append(_randn((1, threads - 1, 2, d), 3).cuda(), _randn((1, threads - 1, 2, d), 4).cuda())
    pool.set_softcap(20.0)
    q = _randn((1, threads, hq, d), 5).cuda()
    out, lse = _attend(lib, pool, q)
    big = q.clone()
    big[0, 1, 2] *= 1000.0                                              # scores far beyond the cap in one row of each ...
    big[0, 1, 6] *= 1000.0                                              # ... kv head's
    out2, lse2 = _attend(lib, pool, big)
    rest = torch.ones((threads, hq), dtype=torch.bool)
    rest[1, 2] = rest[1, 6] = False
    assert torch.equal(out[0][rest], out2[0][rest]) and torch.equal(lse[0][rest], lse2[0][rest])
    assert not torch.equal(out, out2)
    assert pool.status() == 0


@pytest.mark.parametrize("d,flags", KINDS)
def test_what_a_page_held_before_leaves_no_trace(lib, d, flags):
    """The unused tail of a page holds another response's keys, far beyond the cap: the same bits as over a fresh page."""
    import torch
    hq, results = 8, []
    for dirty in (False, True):
        pool = lib.Pool(1, hq, 2, d, 8, 2, 1, 4, flags=flags)
        if dirty:
            k = (300.0 * _randn((1, 128, 2, d), 9)).cuda()
            assert pool.request_begin() == 0
            pool.kv_append_run(0, 0, 128, k, k)                          # every page of the pool
            pool.request_end(0)
        req = pool.request_begin()
        pool.kv_append_run(req, 0, 101, _randn((1, 101, 2, d), 1).cuda(), _randn((1, 101, 2, d), 2).cuda())
        pool.step_begin([req], [0], [0])
        pool.set_softcap(20.0)
        results.append(_attend(lib, pool, _randn((1, 1, hq, d), 5).cuda()))
        assert pool.status() == 0
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])
