"""GPU parity of capped attention scores, s -> cap tanh(s / cap), on both caches and every kernel that computes scores.

Tolerance.  bf16 pools: the tensor-core kernel rounds weights to bf16 (at most 2^-8 each) and divides by the sum of the
rounded ones, so an output is a convex combination of the values with weights off by at most 2^-8 each:
|out - exact| <= 2^-8 max |v - out| <= 2^-7 max |v|, plus twice a score's error; lse is off by at most 2^-8 + that error.  The
warp-shuffle kernel rounds nothing.  8-bit pools: see test_gpu_kv8."""
import numpy as np
import pytest

from oracle import KVStore, PoolModel
from oracle.kv8 import Kv8Store, decode_attention_capped
from pasta_workloads import Geometry, random_script, run_tensors, step_tensors
from test_gpu_kv8 import _randn, compare, run, score_bound

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2502_11517_b200 import binding, build
    build()
    return binding


@pytest.mark.parametrize("geo", [Geometry(2, 8, 2, 128, 16), Geometry(1, 8, 4, 64, 16)])
@pytest.mark.parametrize("cap", [2.0, 50.0])
def test_8bit_pools(lib, geo, cap):
    run(lib, random_script(330, n_ops=60, geo=geo), cap=cap)


@pytest.mark.parametrize("geo", [Geometry(1, 8, 2, 128, 16), Geometry(1, 4, 4, 64, 16)])
def test_8bit_pools_on_the_warp_path(lib, geo):
    run(lib, random_script(331, n_ops=50, geo=geo), cap=5.0, flags=lib.FLAG_NO_TENSOR_PATH)


def _filled(lib, lengths, hq, hkv, d, gain_q, flags=0, layers=1):
    """Requests with two forks each (chunks of 1 and 21 tokens), K and V N(0,1), on the library and the oracle."""
    import torch
    n_pages = sum(m // 16 + 5 for m in lengths)
    eight = flags & lib.FLAG_KV_FP8
    pool = lib.Pool(layers, hq, hkv, d, n_pages, len(lengths), 3, 8, flags=flags, max_step_queries=3 * len(lengths))
    model = PoolModel(n_pages, 16, None, len(lengths), 3, 8)
    store = (Kv8Store if eight else KVStore)(n_pages, 16, hkv, d)
    entries = []
    for r, m in enumerate(lengths):
        pool.request_begin(); model.request_begin()
        for t, n in ((0, m), (1, 1), (2, 21)):
            if t:
                pool.thread_spawn(r); model.thread_spawn(r)
            k, v = _randn((layers, n, hkv, d), 7 * r + t), _randn((layers, n, hkv, d), 900 + 7 * r + t)
            pool.kv_append_run(r, t, n, k.cuda(), v.cuda()); store.write(model.append_run(r, t, n), k[0], v[0])
            entries.append((r, t))
    q = _randn((layers, len(entries), hq, d), 77, gain_q)
    pool.step_begin([e[0] for e in entries], [e[1] for e in entries], [0] * len(entries))
    return pool, model, store, entries, q


@pytest.mark.parametrize("hq,hkv,d,flags", [(8, 2, 128, 0), (8, 1, 128, 0), (8, 2, 128, 2), (4, 4, 64, 0), (8, 2, 64, 8),
                                            (8, 2, 128, 8), (16, 2, 128, 8 | 2)])
@pytest.mark.parametrize("cap,gain", [(1.0, 1.0), (20.0, 4.0), (50.0, 30.0)])
def test_caps_and_gains(lib, hq, hkv, d, flags, cap, gain):
    """Scores far below, around and far above the cap; prefixes from one token to several tiles."""
    import torch
    pool, model, store, entries, q = _filled(lib, [1, 17, 130, 700], hq, hkv, d, gain, flags)
    out = torch.full((1, len(entries), hq, d), float("nan"), device="cuda"); lse = torch.empty((1, len(entries), hq), device="cuda")
    pool.decode_attn(q.cuda(), out, lse)
    plain = out.clone()
    pool.set_softcap(cap)
    pool.decode_attn(q.cuda(), out, lse)
    spread = []
    want, want_lse = decode_attention_capped(model, store, entries, q[0], cap=cap, spread=spread)
    qf = q[0].float().numpy()
    if flags & lib.FLAG_KV_FP8:
        compare(out[0], lse[0], want, want_lse, qf, store, spread, cap=cap)
    else:
        ds = score_bound(qf, store.k, 1 / np.sqrt(d), cap)
        got = out[0].double().cpu().numpy()
        assert np.abs(got - want).max() <= (2.0 ** -7 + 2 * ds) * np.abs(store.v).max()
        assert np.abs(lse[0].double().cpu().numpy() - want_lse).max() <= 2.0 ** -8 + ds + 2.0 ** -21 * np.abs(want_lse).max()
    assert not torch.equal(out, plain)
    pool.set_softcap(0.0)                                              # off again: the plain results, bit for bit
    pool.decode_attn(q.cuda(), out, lse)
    assert torch.equal(out, plain)
    assert pool.status() == 0


@pytest.mark.parametrize("hq,hkv,d,flags", [(8, 2, 128, 0), (8, 2, 128, 2), (4, 4, 64, 0), (8, 2, 64, 8), (8, 2, 128, 8), (16, 2, 128, 8 | 2)])
def test_a_cap_far_above_the_scores(lib, hq, hkv, d, flags):
    """The largest cap there is leaves ordinary scores as they are: no error that grows with the cap."""
    import torch
    pool, model, store, entries, q = _filled(lib, [1, 17, 130, 700], hq, hkv, d, 4.0, flags)
    out = torch.full((1, len(entries), hq, d), float("nan"), device="cuda"); lse = torch.empty((1, len(entries), hq), device="cuda")
    pool.set_softcap(1e6)
    pool.decode_attn(q.cuda(), out, lse)
    spread = []
    want, want_lse = decode_attention_capped(model, store, entries, q[0], cap=1e6, spread=spread)
    qf = q[0].float().numpy()
    # the capped score is good to 2^-22 of itself: less than the sums' own rounding, which the bound without a cap holds
    if flags & lib.FLAG_KV_FP8:
        compare(out[0], lse[0], want, want_lse, qf, store, spread)
    else:
        ds = score_bound(qf, store.k, 1 / np.sqrt(d))
        assert np.abs(out[0].double().cpu().numpy() - want).max() <= (2.0 ** -7 + 2 * ds) * np.abs(store.v).max()
        assert np.abs(lse[0].double().cpu().numpy() - want_lse).max() <= 2.0 ** -8 + ds + 2.0 ** -21 * np.abs(want_lse).max()
    assert pool.status() == 0


def test_cap_reaches_every_entry_point(lib):
    import torch
    hq, hkv, d = 8, 2, 128
    pool, model, store, entries, q = _filled(lib, [40, 300], hq, hkv, d, 4.0)
    pool.set_softcap(10.0)
    qc = q.cuda()
    ref = torch.empty((1, len(entries), hq, d), device="cuda")
    pool.decode_attn(qc, ref)
    one = torch.empty((len(entries), hq, d), device="cuda")
    pool.decode_attn_noalloc(qc[0], one)
    assert torch.equal(one, ref[0])
    out = torch.empty_like(ref)
    r, t = [e[0] for e in entries], [e[1] for e in entries]
    nothing = torch.empty((1, 0, hkv, d), dtype=torch.bfloat16, device="cuda")
    pool.step_device(r, t, [0] * len(entries), nothing, nothing, qc, out)
    assert torch.equal(out, ref)
    staging = torch.empty(pool.step_host_bytes(len(entries)), dtype=torch.uint8, device="cuda")
    host = torch.empty(ref.shape).pin_memory()
    pool.step_host(r, t, [0] * len(entries), nothing.cpu(), nothing.cpu(), q.pin_memory(), host, staging)
    assert torch.equal(host, ref.cpu())


def test_graph_keeps_its_cap(lib):
    import torch
    pool, _, _, entries, q = _filled(lib, [200], 8, 2, 128, 4.0)
    qc = q.cuda()
    out, capped = (torch.empty((1, len(entries), 8, 128), device="cuda") for _ in range(2))
    pool.set_softcap(5.0)
    pool.decode_attn(qc, capped)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pool.decode_attn(qc, out)
    pool.set_softcap(0.0)
    out.zero_()
    graph.replay()
    assert torch.equal(out, capped)
