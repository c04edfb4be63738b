"""GPU parity of 8-bit pools: what the cache holds is bit-exact against the fp64 oracle (codes, scales, their growth, the
rotation), attention over it is compared on the numbers held.

Tolerance of the outputs.  With weights w (sum 1) over the values held, out = sum w v.  What each kernel does to a weight
before it meets its value:
  head_dim 64, matrix kernel   fp16 once: off by at most 2^-11 of it, or 2^-25 of the row's reference;
  head_dim 128, tensor cores   two e4m3 terms: off by at most 2^-8 of it (two halves of 4 significant bits), or by half a step
                               of 2^-9 where the largest contribution of the row, weight times V's scale, is at least 2^4
                               (the reference is set 2^4 below it): 2^-14 of the largest, for each of the n visible tokens.  The
                               codes of a page reach at least 224 of 448, so a contribution of the largest size is at most
                               twice max |v| times the largest weight: n * 2^-14 * 2 * w_max * max |v| in all;
  warp-shuffle kernel          nothing.
The sum of the weights is unrounded.  A score carries the fp32 sums' rounding, D + 8 additions of at most 2^-23 of
sum |q k| (and on the tensor cores the split of q into two e4m3 terms, at most 2^-17 of the row's largest element each: D
terms of 2^-17 max |q| max |k|), and exp2 its own 2^-22; ds bounds it.  So |out - exact| <= (rounding + 2 ds) max |v| and
|lse - exact| <= ds + 2^-21 |lse|."""
import numpy as np
import pytest

from oracle import OracleReplay, PoolModel
from oracle.kv8 import Kv8Store, decode_attention_capped, rotate
from pasta_workloads import Geometry, cfg2_single_request, cfg4_long_prefix, random_script, run_tensors, step_tensors

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2502_11517_b200 import binding, build
    build()
    return binding


def score_bound(q, k, scale, cap=0.0):
    d = q.shape[-1]
    total = np.abs(q).max() * np.abs(k).max() * d * scale
    return ((d + 8) * 2.0 ** -23 + 2.0 ** -17) * total + 2.0 ** -21 * (cap if cap else 1.0) + 2.0 ** -21


def compare(got, got_lse, want, want_lse, q, store, spread, scale=None, cap=0.0, what=""):
    """spread: per query, visible tokens times the largest weight (see decode_attention_capped)."""
    got = got.double().cpu().numpy()
    assert np.all(np.isfinite(got)), what
    scale = 1.0 / np.sqrt(q.shape[-1]) if scale is None else scale
    ds = score_bound(q, store.k, scale, cap)
    weights = 2.0 ** -11 if q.shape[-1] == 64 else 2.0 ** -8 + 2.0 ** -13 * max(spread)
    tol = (weights + 2 * ds) * np.abs(store.v).max()
    assert np.abs(got - want).max() <= tol, (what, np.abs(got - want).max(), tol)
    if got_lse is not None:
        err = np.abs(got_lse.double().cpu().numpy() - want_lse)
        assert (err - 2.0 ** -21 * np.abs(want_lse)).max() <= ds, (what, err.max(), ds)


def held_equals(pool, model, stores, layers):
    """Every stream's contents, bit for bit."""
    for req, r in pool.dump()["requests"].items():
        for sid, s in r["streams"].items():
            if s["len"] == 0:
                continue
            slots = [(s["pages"][t // 16], t % 16) for t in range(s["len"])]
            k_all, v_all = pool.kv_read_layers(req, sid, 0, s["len"])
            for i, l in enumerate(layers):
                wk, wv = stores[l].gather(slots)
                k, v = pool.kv_read(i, req, sid, 0, s["len"])
                assert np.array_equal(k.double().cpu().numpy(), wk), (req, sid, l)
                assert np.array_equal(v.double().cpu().numpy(), wv), (req, sid, l)
                assert np.array_equal(k_all[i].double().cpu().numpy(), wk) and np.array_equal(v_all[i].double().cpu().numpy(), wv)


def run(lib, script, flags=0, cap=0.0, theta=None, check=None, tensors=None, **kw):
    """Replays a script on an 8-bit pool and on the oracle."""
    import torch
    from lib_replay import LibReplay, make_pool
    geo = script.geometry
    pool = make_pool(script, flags=flags | lib.FLAG_KV_FP8, **kw)
    if cap:
        pool.set_softcap(cap)
    rep = LibReplay(script, pool, rope_theta=theta)
    layers = list(range(geo.n_layers))
    model = PoolModel(script.n_pages, 16, script.free_order, script.max_requests, script.max_threads_per_request,
                      script.max_segments_per_thread)
    stores = {l: Kv8Store(script.n_pages, 16, geo.n_kv_heads, geo.head_dim) for l in layers}
    checked = 0
    for i, op in enumerate(script.ops):
        kind = op[0]
        got = rep.apply(i, attend=check is None or i in check)
        if kind == "begin":
            model.request_begin()
        elif kind == "end":
            model.request_end(op[1])
        elif kind == "spawn":
            model.thread_spawn(op[1], op[3] if len(op) > 3 else 0, op[4] if len(op) > 4 else 0)
        elif kind == "finish":
            model.thread_finish(op[1], op[2])
        elif kind == "merge":
            model.sync_merge(op[1], None if op[2] is None else list(op[2]))
        elif kind == "run":
            pos0 = model.requests[op[1]].pos_next[op[2]]
            slots = model.append_run(op[1], op[2], op[3])
            for l in layers:
                k, v = run_tensors(script, i, l)
                stores[l].write(slots, rotate(k, np.arange(pos0, pos0 + op[3]), theta) if theta else k, v)
        elif kind == "step":
            slots = [s for s in model.reserve(op[1]) if s is not None]
            queries = model.queries_of(op[1])
            pos = pool.step_positions()
            app = [p for p, q3 in zip(pos, _appending(op[1])) if q3]
            for l in layers:
                k, v, q = step_tensors(script, i, l)
                stores[l].write(slots, rotate(k, app, theta) if theta else k, v)
                if got is None:
                    continue
                if theta:
                    q = torch.from_numpy(rotate(q, pos, theta)).to(torch.bfloat16)
                qf = q.float().numpy()
                spread = []
                want, want_lse = decode_attention_capped(model, stores[l], queries, qf, cap=cap, spread=spread)
                if theta:          # the queries' own rotation is rounded to bf16: one ulp may differ, so allow its effect
                    assert np.abs(got[0][l].double().cpu().numpy() - want).max() <= 1e-2
                else:
                    compare(got[0][l], got[1][l], want, want_lse, qf, stores[l], spread, cap=cap, what=(i, l))
                checked += 1
    assert checked and pool.dump() == model.dump()
    held_equals(pool, model, stores, layers)
    assert pool.status() == 0
    pool.close()


def _appending(entries):
    return [n_new > 0 for _, _, n_new in entries for _ in range(max(1, n_new))]


@pytest.mark.parametrize("geo", [Geometry(2, 4, 2, 64, 16), Geometry(2, 8, 2, 128, 16), Geometry(1, 4, 4, 128, 16),
                                 Geometry(1, 8, 1, 64, 16), Geometry(1, 4, 2, 128, 16)])
@pytest.mark.parametrize("seed", range(2))
def test_random_scripts(lib, geo, seed):
    run(lib, random_script(300 + seed, n_ops=70, geo=geo, multi_token=bool(seed)))


@pytest.mark.parametrize("geo", [Geometry(1, 4, 2, 64, 16), Geometry(1, 8, 2, 128, 16), Geometry(1, 8, 8, 64, 16),
                                 Geometry(1, 8, 1, 128, 16)])
def test_random_scripts_on_the_warp_path(lib, geo):
    run(lib, random_script(310, n_ops=60, geo=geo, multi_token=True), flags=lib.FLAG_NO_TENSOR_PATH)


@pytest.mark.parametrize("geo", [Geometry(2, 8, 2, 128, 16), Geometry(2, 4, 2, 64, 16)])
def test_rotated_appends(lib, geo):
    run(lib, random_script(320, n_ops=70, geo=geo, predictions=True), theta=10000.0)


@pytest.mark.parametrize("maker", [lambda: cfg2_single_request("a"), lambda: cfg2_single_request("b"),
                                   lambda: cfg4_long_prefix(1, 2500, 16)])
def test_configurations(lib, maker):
    run(lib, maker())


def _pool(lib, n_pages, requests=1, threads=1, hq=8, hkv=2, d=128, layers=1, flags=0, **kw):
    return lib.Pool(layers, hq, hkv, d, n_pages, requests, threads, 2 * threads + 2, flags=flags | lib.FLAG_KV_FP8, **kw)


def _randn(shape, seed, gain=1.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    return (gain * torch.randn(shape, generator=g)).to(torch.bfloat16)


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 33, 63, 64, 65, 127, 129, 500, 2047])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (8, 8, 64), (8, 1, 64)])
def test_lengths(lib, length, hq, hkv, d):
    import torch
    pool = _pool(lib, length // 16 + 1, hq=hq, hkv=hkv, d=d)
    model = PoolModel(length // 16 + 1, 16)
    store = Kv8Store(length // 16 + 1, 16, hkv, d)
    k, v, q = _randn((1, length, hkv, d), length), _randn((1, length, hkv, d), length + 1), _randn((1, 1, hq, d), 5)
    pool.request_begin(); model.request_begin()
    pool.kv_append_run(0, 0, length, k.cuda(), v.cuda())
    store.write(model.append_run(0, 0, length), k[0], v[0])
    pool.step_begin([0], [0], [0])
    out = torch.empty((1, 1, hq, d), device="cuda"); lse = torch.empty((1, 1, hq), device="cuda")
    pool.decode_attn(q.cuda(), out, lse)
    spread = []
    want, want_lse = decode_attention_capped(model, store, [(0, 0)], q[0], spread=spread)
    compare(out[0], lse[0], want, want_lse, q[0].float().numpy(), store, spread)
    held_equals(pool, model, {0: store}, [0])
    assert pool.status() == 0


@pytest.mark.parametrize("threads", [2, 4, 5, 9, 17, 31, 33, 40])
def test_numbers_of_threads(lib, threads):
    """8 to 128 stacked rows on the matrix path in blocks of 32, more on the warp path; ragged private chunks."""
    import torch
    hq, hkv, d = 8, 2, 128
    n_pages = 200 + threads * 4
    pool = _pool(lib, n_pages, threads=threads, hq=hq, hkv=hkv, d=d, max_step_queries=threads)
    model = PoolModel(n_pages, 16, None, 1, threads, 2 * threads + 2)
    store = Kv8Store(n_pages, 16, hkv, d)
    pool.request_begin(); model.request_begin()
    for t in range(threads):
        m = 40 + 3 * t
        k, v = _randn((1, m, hkv, d), 10 + t), _randn((1, m, hkv, d), 500 + t)
        pool.kv_append_run(0, 0, m, k.cuda(), v.cuda()); store.write(model.append_run(0, 0, m), k[0], v[0])
        if t:
            assert pool.thread_spawn(0) == t == model.thread_spawn(0)
    for t in range(1, threads):
        m = 1 + (7 * t) % 45
        k, v = _randn((1, m, hkv, d), 1000 + t), _randn((1, m, hkv, d), 1500 + t)
        pool.kv_append_run(0, t, m, k.cuda(), v.cuda()); store.write(model.append_run(0, t, m), k[0], v[0])
    q = _randn((1, threads, hq, d), 9)
    pool.step_begin([0] * threads, list(range(threads)), [0] * threads)
    out = torch.full((1, threads, hq, d), float("nan"), device="cuda"); lse = torch.empty((1, threads, hq), device="cuda")
    pool.decode_attn(q.cuda(), out, lse)
    spread = []
    want, want_lse = decode_attention_capped(model, store, [(0, t) for t in range(threads)], q[0], spread=spread)
    compare(out[0], lse[0], want, want_lse, q[0].float().numpy(), store, spread)
    assert pool.status() == 0


@pytest.mark.parametrize("d", [64, 128])
def test_pages_of_very_different_scale(lib, d):
    """V pages scaled by 2^-20 .. 2^20 and K pages by 2^-3 .. 2^1: the weights carry V's exponents."""
    import torch
    n = 40
    hq, hkv = 4, 1
    pool = _pool(lib, n, hq=hq, hkv=hkv, d=d)
    model, store = PoolModel(n, 16), Kv8Store(n, 16, hkv, d)
    pool.request_begin(); model.request_begin()
    rng = np.random.default_rng(8)
    gain_v = torch.from_numpy(2.0 ** rng.integers(-20, 21, n)).float().repeat_interleave(16)[None, :, None, None]
    gain_k = torch.from_numpy(2.0 ** rng.integers(-3, 2, n)).float().repeat_interleave(16)[None, :, None, None]
    k = (_randn((1, 16 * n, hkv, d), 1).float() * gain_k).to(torch.bfloat16)
    v = (_randn((1, 16 * n, hkv, d), 2).float() * gain_v).to(torch.bfloat16)
    pool.kv_append_run(0, 0, 16 * n, k.cuda(), v.cuda()); store.write(model.append_run(0, 0, 16 * n), k[0], v[0])
    q = _randn((1, 1, hq, d), 3, 2.0)
    pool.step_begin([0], [0], [0])
    out = torch.empty((1, 1, hq, d), device="cuda"); lse = torch.empty((1, 1, hq), device="cuda")
    pool.decode_attn(q.cuda(), out, lse)
    want, want_lse = decode_attention_capped(model, store, [(0, 0)], q[0])
    # the bound, element by element: rounding of each weight times its value, and the steps of the smallest weights, which
    # are relative to the row's largest contribution, weight times V's scale, and meet codes of up to 448
    qf = q[0].float().numpy()
    ds = score_bound(qf, store.k, 1 / np.sqrt(d))
    kk, vv = store.gather(model.visible_slots(0, 0))
    s = np.einsum("hd,nd->hn", qf[0].astype(np.float64), kk[:, 0]) / np.sqrt(d)
    w = np.exp(s - s.max(1, keepdims=True)); w /= w.sum(1, keepdims=True)
    mag = w @ np.abs(vv[:, 0])
    scales = np.repeat(2.0 ** store.exp[1][[p for p, _ in model.visible_slots(0, 0)[::16]], 0], 16)
    largest = (w * scales).max(1)[:, None]
    relative, step = (2.0 ** -11, 2.0 ** -25) if d == 64 else (2.0 ** -8, 2.0 ** -14)
    tol = (relative + 2 * ds) * mag + 16 * n * step * largest * 448
    assert np.all(np.abs(out[0, 0].double().cpu().numpy() - want[0]) <= tol)
    assert np.abs(lse[0].double().cpu().numpy() - want_lse).max() <= ds + 2.0 ** -21 * np.abs(want_lse).max()
    held_equals(pool, model, {0: store}, [0])


def test_a_growing_page_in_steps(lib):
    """Tokens of growing and shrinking magnitude, one and several per step, into the same pages; every layer its own scale."""
    import torch
    hq, hkv, d, L = 4, 2, 128, 3
    pool = _pool(lib, 8, hq=hq, hkv=hkv, d=d, layers=L, max_step_queries=8)
    model = PoolModel(8, 16)
    stores = {l: Kv8Store(8, 16, hkv, d) for l in range(L)}
    pool.request_begin(); model.request_begin()
    rng = np.random.default_rng(5)
    for step, n in enumerate([1, 1, 3, 1, 5, 1, 1, 7, 1, 1, 2, 6, 1, 1, 1, 4]):
        gain = torch.from_numpy(2.0 ** rng.integers(-12, 13, (L, n, hkv, 1))).float()
        k = (_randn((L, n, hkv, d), 20 + step).float() * gain).to(torch.bfloat16)
        v = (_randn((L, n, hkv, d), 60 + step).float() / gain).to(torch.bfloat16)
        pool.step_begin([0], [0], [n])
        slots = model.reserve([(0, 0, n)])
        if step % 2:
            pool.kv_append(k.cuda(), v.cuda())
        else:
            for l in range(L):                                       # layer by layer, as a model runs
                pool.kv_append(k[l:l + 1].cuda(), v[l:l + 1].cuda(), layer_begin=l, layer_count=1)
        for l in range(L):
            stores[l].write(slots, k[l], v[l])
    held_equals(pool, model, stores, list(range(L)))
    assert pool.status() == 0


def test_values_that_are_not_finite_are_stored_as_zero_and_reported(lib):
    import torch
    pool = _pool(lib, 4)
    model, store = PoolModel(4, 16), Kv8Store(4, 16, 2, 128)
    pool.request_begin(); model.request_begin()
    k, v = _randn((1, 40, 2, 128), 1), _randn((1, 40, 2, 128), 2)
    k[0, 3, 0, 5] = float("nan"); k[0, 20, 1, 64] = float("inf"); v[0, 39, 1, 127] = float("-inf"); v[0, 17, 0, 0] = float("nan")
    v[0, 5, 0, 0] = 3e38                                              # finite, beyond the range: saturates
    pool.kv_append_run(0, 0, 40, k.cuda(), v.cuda()); store.write(model.append_run(0, 0, 40), k[0], v[0])
    assert store.nonfinite == 4
    held_equals(pool, model, {0: store}, [0])
    assert pool.status() == lib.DEVICE_CHECK and pool.status() == 0
    pool.step_begin([0], [0], [1])                                    # a rotated pair with an infinity in it: both zero
    k1, v1 = _randn((1, 1, 2, 128), 3), _randn((1, 1, 2, 128), 4)
    k1[0, 0, 1, 70] = float("inf")
    pool.kv_append_rope(k1.cuda(), v1.cuda(), 10000.0)
    got, _ = pool.kv_read(0, 0, 0, 40, 1)
    assert got[0, 1, 70] == 0 and got[0, 1, 6] == 0 and torch.isfinite(got).all() and (got != 0).sum() > 200
    assert pool.status() == lib.DEVICE_CHECK


@pytest.mark.parametrize("d,theta,runs", [(64, 10000.0, [5, 2048 * 16 + 200]), (64, 0.0, [11, 65 * 16, 2048 * 16]),
                                          (128, 500000.0, [1, 63 * 16, 16, 64 * 16 + 15])])
def test_runs_of_more_pages_than_a_launch_carries(lib, d, theta, runs):
    """Runs around and beyond the two sizes of page list, starting inside a page."""
    n = sum(runs)
    pool = _pool(lib, n // 16 + 1, hq=1, hkv=1, d=d)
    model, store = PoolModel(n // 16 + 1, 16), Kv8Store(n // 16 + 1, 16, 1, d)
    pool.request_begin(); model.request_begin()
    at = 0
    for i, m in enumerate(runs):
        k, v = _randn((1, m, 1, d), 30 + i, gain=2.0 ** i), _randn((1, m, 1, d), 40 + i)
        slots = model.append_run(0, 0, m)
        if theta:
            pool.kv_append_run_rope(0, 0, m, k.cuda(), v.cuda(), theta)
            store.write(slots, rotate(k[0], np.arange(at, at + m), theta), v[0])
        else:
            pool.kv_append_run(0, 0, m, k.cuda(), v.cuda())
            store.write(slots, k[0], v[0])
        at += m
    held_equals(pool, model, {0: store}, [0])
    k, v = pool.kv_read_layers(0, 0, 7, n - 9)                        # a part, neither end on a page
    slots = [(p, o) for p, o in model.visible_slots(0, 0)][7:n - 2]
    wk, wv = store.gather(slots)
    assert np.array_equal(k[0].double().cpu().numpy(), wk) and np.array_equal(v[0].double().cpu().numpy(), wv)
    assert pool.status() == 0


@pytest.mark.parametrize("theta", [0.0, 10000.0])
def test_numbers_at_the_ends_of_the_range(lib, theta):
    """Zeros, subnormal, smallest and largest bf16 numbers, alone in a page and side by side; a rotation that leaves fp32."""
    import torch
    sizes = [0.0, 2.0 ** -133, 2.0 ** -127, 2.0 ** -126, 2.0 ** -70, 1.0, 2.0 ** 60, 2.0 ** 72, 2.0 ** 100, 3.3e38]
    n = 16 * (len(sizes) + 1)
    pool = _pool(lib, n // 16)
    model, store = PoolModel(n // 16, 16), Kv8Store(n // 16, 16, 2, 128)
    pool.request_begin(); model.request_begin()
    g = torch.Generator().manual_seed(3)
    unit = 1.0 - 2.0 * torch.randint(0, 2, (1, n, 2, 128), generator=g)
    gain = torch.tensor(sizes + [1.0]).repeat_interleave(16).reshape(1, n, 1, 1).repeat(1, 1, 2, 1)
    gain[0, -16:, 0, 0] = torch.tensor((sizes * 2)[:16])               # the last page mixes them
    k, v = (unit * gain).to(torch.bfloat16), (unit.flip(1) * gain).to(torch.bfloat16)
    slots = model.append_run(0, 0, n)
    if theta:
        pool.kv_append_run_rope(0, 0, n, k.cuda(), v.cuda(), theta)
        with np.errstate(over="ignore"):
            store.write(slots, rotate(k[0], np.arange(n), theta), v[0])
    else:
        pool.kv_append_run(0, 0, n, k.cuda(), v.cuda())
        store.write(slots, k[0], v[0])
    held_equals(pool, model, {0: store}, [0])
    assert (pool.status() == lib.DEVICE_CHECK) == (store.nonfinite > 0)


@pytest.mark.parametrize("d,flags", [(64, 0), (128, 0), (128, 2)])
def test_query_rows_of_any_size(lib, d, flags):
    """Rows of zeros, subnormal and huge numbers.  Over K = 0 every score is 0, so each row is the mean of V, whatever is in q."""
    import torch
    hq, n = 8, 50
    pool = _pool(lib, 8, threads=2, hq=hq, hkv=2, d=d, flags=flags)
    k, v = torch.zeros((1, n, 2, d), dtype=torch.bfloat16), _randn((1, n, 2, d), 2)
    pool.request_begin()
    pool.kv_append_run(0, 0, n, k.cuda(), v.cuda())
    sizes = torch.tensor([0.0, 2.0 ** -133, 2.0 ** -126, 2.0 ** -60, 1.0, 2.0 ** 60, 2.0 ** 120, 3.3e38]).reshape(1, 1, hq, 1)
    q = ((1.0 - 2.0 * (torch.arange(d) % 2)) * sizes).to(torch.bfloat16)
    pool.step_begin([0], [0], [0])
    out = torch.empty((1, 1, hq, d), device="cuda"); lse = torch.empty((1, 1, hq), device="cuda")
    pool.decode_attn(q.cuda(), out, lse)
    _, held = pool.kv_read(0, 0, 0, 0, n)
    mean = held.double().mean(0).repeat_interleave(4, 0)
    # equal weights 1 / n: each rounded as above, by at most 2^-8 of itself
    assert (out[0, 0].double() - mean).abs().max() <= (2.0 ** -8 + 2.0 ** -20) * held.double().abs().max()
    assert (lse[0, 0].double() - np.log(n)).abs().max() <= 2.0 ** -18
    assert pool.status() == 0


@pytest.mark.parametrize("d", [64, 128])
def test_two_pools_at_once_on_two_streams(lib, d):
    """Steps of two pools enqueued in turn on two streams, and one of them captured and replayed beside the other's calls."""
    import torch
    T, L, n = 9, 2, 700
    tensors, pools, refs = [], [], []
    for i in range(2):
        pool = _pool(lib, 80, threads=T, hq=8, hkv=2, d=d, layers=L, max_step_queries=T)
        pool.request_begin()
        pool.kv_append_run(0, 0, n + 50 * i, _randn((L, n + 50 * i, 2, d), i).cuda(), _randn((L, n + 50 * i, 2, d), 10 + i).cuda())
        for _ in range(T - 1):
            pool.thread_spawn(0)
        kn, vn, q = (_randn((L, T, h, d), s + i).cuda() for h, s in ((2, 20), (2, 30), (8, 40)))
        pool.step_begin([0] * T, list(range(T)))
        pool.kv_append(kn, vn)
        out = torch.empty((L, T, 8, d), device="cuda")
        pool.decode_attn(q, out)
        torch.cuda.synchronize()
        pools.append(pool); tensors.append(q); refs.append(out)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.full_like(refs[i], 7.0) for _ in range(12)] for i in range(2)]
    for j in range(12):
        for i in range(2):
            pools[i].decode_attn(tensors[i], outs[i][j], stream=streams[i])
    torch.cuda.synchronize()
    assert all(torch.equal(o, refs[i]) for i in range(2) for o in outs[i])
    graph, captured = torch.cuda.CUDAGraph(), torch.zeros_like(refs[0])
    with torch.cuda.graph(graph):
        pools[0].decode_attn(tensors[0], captured)
    other = torch.zeros_like(refs[1])
    for _ in range(5):
        with torch.cuda.stream(streams[0]):
            graph.replay()
        pools[1].decode_attn(tensors[1], other, stream=streams[1])
    torch.cuda.synchronize()
    assert torch.equal(captured, refs[0]) and torch.equal(other, refs[1])
    assert pools[0].status() == 0 and pools[1].status() == 0


def test_every_way_to_run_a_step_gives_the_same(lib):
    """decode_attn on another stream, captured and replayed, per layer, without workspace, through step_device and step_host,
    with launches that do not overlap, and with bf16 outputs."""
    import torch
    hq, hkv, d, L, T = 8, 2, 128, 3, 5
    outs = {}
    k0, v0 = _randn((L, 300, hkv, d), 1).cuda(), _randn((L, 300, hkv, d), 2).cuda()
    kn, vn, q = _randn((L, T, hkv, d), 3).cuda(), _randn((L, T, hkv, d), 4).cuda(), _randn((L, T, hq, d), 6).cuda()
    reqs, thr = [0] * T, list(range(T))

    def filled(flags=0):
        pool = _pool(lib, 60, threads=T, hq=hq, hkv=hkv, d=d, layers=L, flags=flags, max_step_queries=T)
        pool.request_begin()
        pool.kv_append_run(0, 0, 300, k0, v0)
        for _ in range(T - 1):
            pool.thread_spawn(0)
        return pool

    pool = filled()
    pool.step_begin(reqs, thr)
    pool.kv_append(kn, vn)
    ref = torch.empty((L, T, hq, d), device="cuda"); ref_lse = torch.empty((L, T, hq), device="cuda")
    pool.decode_attn(q, ref, ref_lse)
    out = torch.empty_like(ref); lse = torch.empty_like(ref_lse)
    for l in range(L):
        pool.decode_attn(q[l:l + 1], out[l:l + 1], lse[l:l + 1], layer_begin=l, layer_count=1)
    assert torch.equal(out, ref) and torch.equal(lse, ref_lse)
    out.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    pool.decode_attn(q, out, None, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, ref)
    out.zero_()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        pool.decode_attn(q, out, lse)
    out.zero_()
    graph.replay(); graph.replay()
    assert torch.equal(out, ref) and torch.equal(lse, ref_lse)
    out.zero_()
    pool.debug_set_launch_overlap(False)
    try:
        pool.decode_attn(q, out)
    finally:
        pool.debug_set_launch_overlap(True)
    assert torch.equal(out, ref)
    one = torch.empty((T, hq, d), device="cuda")
    pool.decode_attn_noalloc(q[2], one, layer=2)
    assert torch.equal(one, ref[2])
    pool.close()

    pool = filled()
    out.zero_()
    pool.step_device(reqs, thr, None, kn, vn, q, out, lse)
    assert torch.equal(out, ref) and torch.equal(lse, ref_lse)
    pool.close()

    pool = filled()
    host = [x.cpu().pin_memory() for x in (kn, vn, q)]
    oh = torch.empty((L, T, hq, d)).pin_memory()
    staging = torch.empty(pool.step_host_bytes(T), dtype=torch.uint8, device="cuda")
    pool.step_host(reqs, thr, None, *host, oh, staging)
    assert torch.equal(oh, ref.cpu())
    pool.close()

    pool = filled(lib.FLAG_OUT_BF16)
    ob = torch.empty((L, T, hq, d), dtype=torch.bfloat16, device="cuda")
    pool.step_device(reqs, thr, None, kn, vn, q, ob)
    assert torch.equal(ob, ref.to(torch.bfloat16))
    assert pool.status() == 0


def test_refusals(lib):
    pool = _pool(lib, 4, layers=2)
    L = lib.lib()
    req = pool.request_begin()
    k = _randn((2, 20, 2, 128), 1).cuda()
    pool.kv_append_run(req, 0, 20, k, k)
    p = k.data_ptr()
    bad = lambda *a: L.pasta_kv_read_layers(pool._h, *a[:6], lib._dev(a[6]), lib._dev(a[6]), None)
    assert bad(0, 2, 0, 0, 0, 20, k) == lib.OK
    assert bad(0, 3, 0, 0, 0, 20, k) == lib.INVALID_ARG and bad(-1, 1, 0, 0, 0, 20, k) == lib.INVALID_ARG
    assert bad(2, 1, 0, 0, 0, 20, k) == lib.INVALID_ARG and bad(0, 1, 1, 0, 0, 20, k) == lib.INVALID_ARG
    assert bad(0, 1, 0, 1, 0, 20, k) == lib.INVALID_ARG and bad(0, 1, 0, 0, 1, 20, k) == lib.INVALID_ARG
    assert bad(0, 1, 0, 0, -1, 2, k) == lib.INVALID_ARG and bad(0, 1, 0, 0, 0, 20, None) == lib.INVALID_ARG
    assert bad(0, 0, 0, 0, 0, 20, None) == lib.OK and bad(0, 1, 0, 0, 20, 0, None) == lib.OK
    for cap in (-1.0, float("nan"), float("inf"), 1e-4, 1e7):
        with pytest.raises(lib.PastaError):
            pool.set_softcap(cap)
    pool.set_softcap(30.0); pool.set_softcap(0.0)
    assert pool.status() == 0 and p


def test_tensors_that_are_not_aligned_are_refused(lib):
    """Rows are read and written 16 bytes at a time; nothing is launched, and a refused append takes no slot."""
    import torch
    pool = _pool(lib, 4)
    flat = torch.zeros(20 * 2 * 128 + 8, dtype=torch.bfloat16, device="cuda")
    good, odd = flat[:20 * 2 * 128].view(1, 20, 2, 128), flat[1:1 + 20 * 2 * 128].view(1, 20, 2, 128)
    pool.request_begin()
    for k, v in ((odd, good), (good, odd)):
        with pytest.raises(lib.PastaError):
            pool.kv_append_run(0, 0, 20, k, v)
        with pytest.raises(lib.PastaError):
            pool.kv_append_run_rope(0, 0, 20, k, v)
    pool.kv_append_run(0, 0, 20, good, good)
    assert pool.dump()["requests"][0]["streams"][0]["len"] == 20
    pool.step_begin([0], [0], [1])
    one = flat[:256].view(1, 1, 2, 128)
    q, out = flat[:1024].view(1, 1, 8, 128), torch.empty(1030, device="cuda")
    for k, v in ((flat[4:260].view(1, 1, 2, 128), one), (one, flat[4:260].view(1, 1, 2, 128))):
        with pytest.raises(lib.PastaError):
            pool.kv_append(k, v)
        with pytest.raises(lib.PastaError):
            pool.kv_append_rope(k, v, 10000.0)
    pool.kv_append(one, one)
    for a, b in ((flat[1:1025].view(1, 1, 8, 128), out[:1024]), (q, out[1:1025])):
        with pytest.raises(lib.PastaError):
            pool.decode_attn(a, b)
        with pytest.raises(lib.PastaError):
            pool.decode_attn_noalloc(a, b)
    assert lib.lib().pasta_kv_read_layers(pool._h, 0, 1, 0, 0, 0, 20, lib._dev(odd), lib._dev(good), None) == lib.INVALID_ARG
    pool.decode_attn(q, out[:1024])
    assert pool.status() == 0
