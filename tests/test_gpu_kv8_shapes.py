"""8-bit pools: the row counts at which the kernels change their form, requests of several forms in one step, scales other than
the default, and pools larger than 32-bit offsets reach."""
import numpy as np
import pytest

from oracle import PoolModel
from oracle.kv8 import Kv8Store, decode_attention_capped
from test_gpu_kv8 import _pool, _randn, compare, lib  # noqa: F401  (fixture + helpers)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 2, 128), (8, 1, 64)])
@pytest.mark.parametrize("threads", [[4], [8], [8, 1], [9, 8], [16], [16, 2, 5], [17, 16, 8, 1], [32, 4], [33, 8], [3, 64]])
def test_row_classes(lib, threads, hq, hkv, d):
    import torch
    n_pages = sum(30 + 3 * t for t in threads)
    R, most = len(threads), max(threads)
    pool = _pool(lib, n_pages, requests=R, threads=most, hq=hq, hkv=hkv, d=d, max_step_queries=sum(threads))
    model = PoolModel(n_pages, 16, None, R, most, 2 * most + 2)
    store = Kv8Store(n_pages, 16, hkv, d)
    entries = []
    for r, count in enumerate(threads):
        pool.request_begin(); model.request_begin()
        for t in range(count):
            m = 150 + 70 * r if t == 0 else 1 + (11 * t + 5 * r) % 37
            if t:
                pool.thread_spawn(r); model.thread_spawn(r)
            k, v = _randn((1, m, hkv, d), 100 * r + t), _randn((1, m, hkv, d), 5000 + 100 * r + t)
            pool.kv_append_run(r, t, m, k.cuda(), v.cuda()); store.write(model.append_run(r, t, m), k[0], v[0])
            entries.append((r, t))
    q = _randn((1, len(entries), hq, d), 9)
    pool.step_begin([e[0] for e in entries], [e[1] for e in entries], [0] * len(entries))
    for scale in (0.0, 0.3, 1e-3):
        out = torch.full((1, len(entries), hq, d), float("nan"), device="cuda"); lse = torch.empty((1, len(entries), hq), device="cuda")
        pool.decode_attn(q.cuda(), out, lse, scale=scale)
        spread = []
        want, want_lse = decode_attention_capped(model, store, entries, q[0], scale=scale or None, spread=spread)
        compare(out[0], lse[0], want, want_lse, q[0].float().numpy(), store, spread, scale=scale or None)
    assert pool.status() == 0


@pytest.mark.parametrize("hq,hkv,d,n_pages", [(8, 8, 128, 140_000), (16, 16, 64, 140_000)])
def test_pages_beyond_4_gib(lib, hq, hkv, d, n_pages):
    """The last pages of a pool of two layers of 4.6 GB each hold, give and attend to the same as the first ones of a small pool."""
    import torch
    L, n, T = 2, 777, 3
    results = []
    for pages, order in ((60, None), (n_pages, np.arange(n_pages - 1, -1, -1))):
        pool = _pool(lib, pages, threads=T, hq=hq, hkv=hkv, d=d, layers=L, max_step_queries=T, free_order=order)
        pool.request_begin()
        pool.kv_append_run_rope(0, 0, n, _randn((L, n, hkv, d), 1).cuda(), _randn((L, n, hkv, d), 2).cuda(), 10000.0)
        for _ in range(T - 1):
            pool.thread_spawn(0)
        pool.step_begin([0] * T, list(range(T)), [1] * T)
        pool.kv_append(_randn((L, T, hkv, d), 3).cuda(), _randn((L, T, hkv, d), 4).cuda())
        if order is not None:
            assert pool.step_slots()[:, 0].min() > n_pages - 60
        out = torch.empty((L, T, hq, d), device="cuda")
        pool.decode_attn(_randn((L, T, hq, d), 5).cuda(), out)
        k, v = pool.kv_read_layers(0, 0, 0, n + 1)
        results.append((out, k, v))
        assert pool.status() == 0
        pool.close()
        pool.kv = pool._kv_raw = pool.workspace = None
    assert all(torch.equal(a, b) for a, b in zip(*results))
