"""GPU parity of 4-bit pools: what the cache holds is bit-exact against the fp64 oracle, attention over it is compared on the
numbers held.

Tolerance of the outputs.  Queries, keys and values enter as they are.  A score is a sum of head_dim exact products in fp32 (or in
the tensor cores' accumulators), at most head_dim + 8 roundings of 2^-23 of sum |q k|, and its exponential is good to 2^-21; ds
bounds it.  A weight is rounded to bf16 once on the tensor cores (half a step is at most 2^-8 of it) and the sum of the weights is that of
the rounded ones, so out = sum w (1 + e) v / sum w (1 + e) with |e| <= 2^-8 + 2 ds is within 2 (2^-8 + 2 ds) max |v| of the exact
row, to first order, and lse within 2^-8 + ds; the fp32 sums add 2^-16 of max |v|.  The warp-shuffle kernel rounds no weight; the
same bound holds."""
import numpy as np
import pytest

from oracle import PoolModel
from oracle.kv4 import Kv4Store, rotate_form
from oracle.kv8 import decode_attention_capped
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
    return (d + 8) * 2.0 ** -23 * total + 2.0 ** -21 * (cap if cap else 1.0) + 2.0 ** -21


def compare(got, got_lse, want, want_lse, q, store, scale=None, cap=0.0, what=""):
    got = got.double().cpu().numpy()
    assert np.all(np.isfinite(got)), what
    scale = 1.0 / np.sqrt(q.shape[-1]) if scale is None else scale
    ds = score_bound(q, store.k, scale, cap)
    tol = (2.0 ** -7 + 4 * ds + 2.0 ** -16) * np.abs(store.v).max()
    assert np.abs(got - want).max() <= tol, (what, np.abs(got - want).max(), tol)
    if got_lse is not None:
        err = np.abs(got_lse.double().cpu().numpy() - want_lse)
        assert (err - 2.0 ** -21 * np.abs(want_lse)).max() <= ds + 2.0 ** -8, (what, err.max(), ds)


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


def turned(x, positions, theta, form):
    return rotate_form(x, positions, theta, form).astype(np.float32)


def run(lib, script, flags=0, cap=0.0, theta=None, form=None, **kw):
    """Replays a script on a 4-bit pool and on the oracle."""
    import torch
    from lib_replay import LibReplay, make_pool
    geo = script.geometry
    pool = make_pool(script, flags=flags | lib.FLAG_KV_INT4, **kw)
    if cap:
        pool.set_softcap(cap)
    if form:
        pool.set_rope(**form)
    form = form or {}
    rep = LibReplay(script, pool, rope_theta=theta)
    layers = list(range(geo.n_layers))
    model = PoolModel(script.n_pages, 16, script.free_order, script.max_requests, script.max_threads_per_request,
                      script.max_segments_per_thread)
    stores = {l: Kv4Store(script.n_pages, 16, geo.n_kv_heads, geo.head_dim) for l in layers}
    checked = 0
    for i, op in enumerate(script.ops):
        kind = op[0]
        got = rep.apply(i)
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
                stores[l].write(slots, turned(k, np.arange(pos0, pos0 + op[3]), theta, form) if theta else k, v)
        elif kind == "step":
            slots = [s for s in model.reserve(op[1]) if s is not None]
            queries = model.queries_of(op[1])
            pos = pool.step_positions()
            appending = [n_new > 0 for _, _, n_new in op[1] for _ in range(max(1, n_new))]
            app = [p for p, a in zip(pos, appending) if a]
            for l in layers:
                k, v, q = step_tensors(script, i, l)
                stores[l].write(slots, turned(k, app, theta, form) if theta else k, v)
                if got is None:
                    continue
                if theta:
                    q = torch.from_numpy(turned(q, pos, theta, form)).to(torch.bfloat16)
                qf = q.float().numpy()
                want, want_lse = decode_attention_capped(model, stores[l], queries, qf, cap=cap)
                if theta:          # the queries' own rotation is rounded to bf16: one ulp may differ, so allow its effect
                    assert np.abs(got[0][l].double().cpu().numpy() - want).max() <= 1e-2
                else:
                    compare(got[0][l], got[1][l], want, want_lse, qf, stores[l], cap=cap, what=(i, l))
                checked += 1
    assert checked and pool.dump() == model.dump()
    held_equals(pool, model, stores, layers)
    assert pool.status() == 0
    pool.close()


@pytest.mark.parametrize("geo", [Geometry(2, 4, 2, 64, 16), Geometry(2, 8, 2, 128, 16), Geometry(1, 4, 4, 128, 16),
                                 Geometry(1, 8, 1, 64, 16), Geometry(1, 4, 2, 128, 16)])
@pytest.mark.parametrize("seed", range(2))
def test_random_scripts(lib, geo, seed):
    run(lib, random_script(300 + seed, n_ops=70, geo=geo, multi_token=bool(seed)))


@pytest.mark.parametrize("geo", [Geometry(1, 4, 2, 64, 16), Geometry(1, 8, 2, 128, 16), Geometry(1, 8, 8, 64, 16),
                                 Geometry(1, 8, 1, 128, 16)])
def test_random_scripts_on_the_warp_path(lib, geo):
    run(lib, random_script(310, n_ops=60, geo=geo, multi_token=True), flags=lib.FLAG_NO_TENSOR_PATH)


@pytest.mark.parametrize("form", [{}, {"layout": "interleaved", "rotary_dim": 32, "scaling": "ramp", "factor": 4.0,
                                       "original_length": 64.0, "high": 32.0}])
@pytest.mark.parametrize("geo", [Geometry(2, 8, 2, 128, 16), Geometry(2, 4, 2, 64, 16)])
def test_rotated_appends(lib, geo, form):
    run(lib, random_script(320, n_ops=70, geo=geo, predictions=True), theta=10000.0, form=form)


@pytest.mark.parametrize("maker", [lambda: cfg2_single_request("a"), lambda: cfg2_single_request("b"),
                                   lambda: cfg4_long_prefix(1, 2500, 16)])
def test_configurations(lib, maker):
    run(lib, maker())


@pytest.mark.parametrize("cap", [2.0, 50.0])
@pytest.mark.parametrize("geo,flags", [(Geometry(1, 8, 2, 128, 16), 0), (Geometry(1, 4, 2, 64, 16), 0), (Geometry(1, 8, 2, 128, 16), 2)])
def test_capped_scores(lib, geo, flags, cap):
    run(lib, random_script(330, n_ops=50, geo=geo, multi_token=True), flags=flags, cap=cap)


def _pool(lib, n_pages, requests=1, threads=1, hq=8, hkv=2, d=128, layers=1, flags=0, **kw):
    return lib.Pool(layers, hq, hkv, d, n_pages, requests, threads, 2 * threads + 2, flags=flags | lib.FLAG_KV_INT4, **kw)


def _randn(shape, seed, gain=1.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    return (gain * torch.randn(shape, generator=g)).to(torch.bfloat16)


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 33, 63, 64, 65, 127, 128, 129, 500, 2047])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (8, 8, 64), (8, 1, 64), (8, 8, 128)])
def test_lengths(lib, length, hq, hkv, d):
    import torch
    pool = _pool(lib, length // 16 + 1, hq=hq, hkv=hkv, d=d)
    model = PoolModel(length // 16 + 1, 16)
    store = Kv4Store(length // 16 + 1, 16, hkv, d)
    k, v, q = _randn((1, length, hkv, d), length), _randn((1, length, hkv, d), length + 1), _randn((1, 1, hq, d), 5)
    pool.request_begin(); model.request_begin()
    pool.kv_append_run(0, 0, length, k.cuda(), v.cuda())
    store.write(model.append_run(0, 0, length), k[0], v[0])
    pool.step_begin([0], [0], [0])
    out = torch.empty((1, 1, hq, d), device="cuda"); lse = torch.empty((1, 1, hq), device="cuda")
    pool.decode_attn(q.cuda(), out, lse)
    want, want_lse = decode_attention_capped(model, store, [(0, 0)], q[0])
    compare(out[0], lse[0], want, want_lse, q[0].float().numpy(), store)
    held_equals(pool, model, {0: store}, [0])
    assert pool.status() == 0


def forked(lib, threads, hq, hkv, d, prefix=40, layers=1, flags=0, gain_k=1.0, **kw):
    """A response whose threads split off along the prompt, with private chunks of ragged length, and its oracle."""
    n_pages = (prefix + 3 * threads) * threads // 16 + threads * 5 + 8
    pool = _pool(lib, n_pages, threads=threads, hq=hq, hkv=hkv, d=d, layers=layers, flags=flags, max_step_queries=threads, **kw)
    model = PoolModel(n_pages, 16, None, 1, threads, 2 * threads + 2)
    store = Kv4Store(n_pages, 16, hkv, d)
    pool.request_begin(); model.request_begin()

    def append(t, m, seed):
        k, v = _randn((layers, m, hkv, d), seed, gain_k), _randn((layers, m, hkv, d), seed + 500)
        pool.kv_append_run(0, t, m, k.cuda(), v.cuda())
        store.write(model.append_run(0, t, m), k[0], v[0])

    for t in range(threads):
        append(0, prefix + 3 * t if t < 20 else 3, 10 + t)
        if t:
            assert pool.thread_spawn(0) == t == model.thread_spawn(0)
    for t in range(1, threads):
        append(t, 1 + (7 * t) % 45, 2000 + t)
    return pool, model, store


@pytest.mark.parametrize("threads", [2, 4, 5, 9, 16, 17, 20, 24, 25, 31, 32, 33, 40])
@pytest.mark.parametrize("d", [128, 64])
def test_numbers_of_threads(lib, threads, d):
    """8 to 128 stacked rows on the tensor cores in every class of sizes, more on the warp path; ragged private chunks."""
    import torch
    hq, hkv = 8, 2
    pool, model, store = forked(lib, threads, hq, hkv, d)
    q = _randn((1, threads, hq, d), 9)
    pool.step_begin([0] * threads, list(range(threads)), [0] * threads)
    out = torch.full((1, threads, hq, d), float("nan"), device="cuda"); lse = torch.empty((1, threads, hq), device="cuda")
    pool.decode_attn(q.cuda(), out, lse)
    want, want_lse = decode_attention_capped(model, store, [(0, t) for t in range(threads)], q[0])
    compare(out[0], lse[0], want, want_lse, q[0].float().numpy(), store)
    assert pool.status() == 0


@pytest.mark.parametrize("threads,hq,hkv", [(1, 1, 1), (3, 1, 1), (13, 2, 1), (70, 1, 1), (128, 1, 1), (16, 8, 1), (9, 16, 2), (2, 2, 2)])
@pytest.mark.parametrize("d", [128, 64])
def test_group_sizes(lib, threads, hq, hkv, d):
    import torch
    pool, model, store = forked(lib, threads, hq, hkv, d, prefix=70)
    q = _randn((1, threads, hq, d), 9)
    pool.step_begin([0] * threads, list(range(threads)), [0] * threads)
    out = torch.full((1, threads, hq, d), float("nan"), device="cuda"); lse = torch.empty((1, threads, hq), device="cuda")
    pool.decode_attn(q.cuda(), out, lse)
    want, want_lse = decode_attention_capped(model, store, [(0, t) for t in range(threads)], q[0])
    compare(out[0], lse[0], want, want_lse, q[0].float().numpy(), store)
    assert pool.status() == 0


@pytest.mark.parametrize("gain_q,gain_k,scale", [(4.0, 4.0, None), (1.0, 1.0, 1.0), (30.0, 30.0, None), (0.01, 1.0, 0.02), (1e4, 1.0, None)])
@pytest.mark.parametrize("d,flags", [(128, 0), (64, 0), (128, 2)])
def test_peaked_and_flat_scores(lib, d, flags, gain_q, gain_k, scale):
    """Scores up to many thousands: the reference of a row is raised again and again, and rows are decided by single tokens."""
    import torch
    hq, hkv, threads = 8, 2, 7
    pool, model, store = forked(lib, threads, hq, hkv, d, prefix=150, flags=flags, gain_k=gain_k)
    q = _randn((1, threads, hq, d), 9, gain_q)
    pool.step_begin([0] * threads, list(range(threads)), [0] * threads)
    out = torch.empty((1, threads, hq, d), device="cuda"); lse = torch.empty((1, threads, hq), device="cuda")
    pool.decode_attn(q.cuda(), out, lse, scale=scale or 0.0)
    want, want_lse = decode_attention_capped(model, store, [(0, t) for t in range(threads)], q[0], scale=scale)
    qf = q[0].float().numpy()
    ds = score_bound(qf, store.k, scale or d ** -0.5)
    if ds < 0.05:                      # the bound's first order
        compare(out[0], lse[0], want, want_lse, qf, store, scale=scale)
    else:                              # scores themselves are only known to ds: compare where one token decides for certain
        assert bool(torch.isfinite(out).all())
        assert np.abs(lse[0].double().cpu().numpy() - want_lse).max() <= ds + 2.0 ** -8 + 2.0 ** -21 * np.abs(want_lse).max()
    assert pool.status() == 0


@pytest.mark.parametrize("d", [64, 128])
def test_growing_scores_along_a_run(lib, d):
    """Keys planted at growing multiples of a row's own query, each above the reference by more than the kernel tolerates, with
    whole tiles that some rows do not see before them."""
    import torch
    n, hq, hkv = 1200, 4, 1
    pool = _pool(lib, n // 16 + 4, threads=2, hq=hq, hkv=hkv, d=d)
    model, store = PoolModel(n // 16 + 4, 16, None, 1, 2, 8), Kv4Store(n // 16 + 4, 16, hkv, d)
    k, v, q = _randn((1, n, hkv, d), 1), _randn((1, n, hkv, d), 2), _randn((1, 2, hq, d), 3)
    for i, at in enumerate([5, 130, 135, 300, 511, 640, 897, 1100, 1199]):
        k[0, at, 0] = (0.3 * (i + 1) * q[0, i % 2, i % hq].float()).to(torch.bfloat16)
    pool.request_begin(); model.request_begin()
    pool.kv_append_run(0, 0, 600, k[:, :600].cuda(), v[:, :600].cuda()); store.write(model.append_run(0, 0, 600), k[0, :600], v[0, :600])
    assert pool.thread_spawn(0) == model.thread_spawn(0) == 1
    pool.kv_append_run(0, 1, 600, k[:, 600:].contiguous().cuda(), v[:, 600:].contiguous().cuda()); store.write(model.append_run(0, 1, 600), k[0, 600:], v[0, 600:])
    pool.step_begin([0, 0], [0, 1], [0, 0])
    out = torch.empty((1, 2, hq, d), device="cuda"); lse = torch.empty((1, 2, hq), device="cuda")
    pool.decode_attn(q.cuda(), out, lse)
    want, want_lse = decode_attention_capped(model, store, [(0, 0), (0, 1)], q[0])
    compare(out[0], lse[0], want, want_lse, q[0].float().numpy(), store)


def test_scores_far_below_zero(lib):
    """Every score of a row is about -2000, and a thread whose first tiles are all invisible to the other."""
    import torch
    for d in (64, 128):
        q = torch.ones((1, 2, 4, d), dtype=torch.bfloat16) * 8
        k = -torch.ones((1, 300, 1, d), dtype=torch.bfloat16) * (2000 / (8 * d ** 0.5))
        k = (k.float() * (1 + 0.01 * _randn((1, 300, 1, 1), 4).float())).to(torch.bfloat16)
        v = _randn((1, 300, 1, d), 2)
        pool = _pool(lib, 60, threads=2, hq=4, hkv=1, d=d)
        model, store = PoolModel(60, 16, None, 1, 2, 8), Kv4Store(60, 16, 1, d)
        pool.request_begin(); model.request_begin()
        pool.kv_append_run(0, 0, 10, k[:, :10].cuda(), v[:, :10].cuda()); store.write(model.append_run(0, 0, 10), k[0, :10], v[0, :10])
        pool.thread_spawn(0); model.thread_spawn(0)
        pool.kv_append_run(0, 0, 280, k[:, 10:290].contiguous().cuda(), v[:, 10:290].contiguous().cuda()); store.write(model.append_run(0, 0, 280), k[0, 10:290], v[0, 10:290])
        pool.kv_append_run(0, 1, 10, k[:, 290:].contiguous().cuda(), v[:, 290:].contiguous().cuda()); store.write(model.append_run(0, 1, 10), k[0, 290:], v[0, 290:])
        pool.step_begin([0, 0], [0, 1], [0, 0])
        out = torch.empty((1, 2, 4, d), device="cuda"); lse = torch.empty((1, 2, 4), device="cuda")
        pool.decode_attn(q.cuda(), out, lse)
        want, want_lse = decode_attention_capped(model, store, [(0, 0), (0, 1)], q[0])
        compare(out[0], lse[0], want, want_lse, q[0].float().numpy(), store)


@pytest.mark.parametrize("d", [64, 128])
def test_pages_and_elements_of_very_different_scale(lib, d):
    """V tokens scaled by 2^-20 .. 2^20 and K's groups of 32 by 2^-6 .. 2^2."""
    import torch
    n, hq, hkv = 640, 4, 1
    pool = _pool(lib, n // 16, hq=hq, hkv=hkv, d=d)
    model, store = PoolModel(n // 16, 16), Kv4Store(n // 16, 16, hkv, d)
    pool.request_begin(); model.request_begin()
    rng = np.random.default_rng(8)
    gain_v = torch.from_numpy(2.0 ** rng.integers(-20, 21, n)).float()[None, :, None, None]
    gain_k = torch.from_numpy(2.0 ** rng.integers(-6, 3, d // 32)).float().repeat_interleave(32)[None, None, None, :]
    k = (_randn((1, n, hkv, d), 1).float() * gain_k).to(torch.bfloat16)
    v = (_randn((1, n, hkv, d), 2).float() * gain_v).to(torch.bfloat16)
    pool.kv_append_run(0, 0, n, k.cuda(), v.cuda()); store.write(model.append_run(0, 0, n), k[0], v[0])
    q = _randn((1, 1, hq, d), 3, 2.0)
    pool.step_begin([0], [0], [0])
    out = torch.empty((1, 1, hq, d), device="cuda"); lse = torch.empty((1, 1, hq), device="cuda")
    pool.decode_attn(q.cuda(), out, lse)
    want, want_lse = decode_attention_capped(model, store, [(0, 0)], q[0])
    qf = q[0].float().numpy()
    ds = score_bound(qf, store.k, d ** -0.5)
    kk, vv = store.gather(model.visible_slots(0, 0))
    s = np.einsum("hd,nd->hn", qf[0].astype(np.float64), kk[:, 0]) / np.sqrt(d)
    w = np.exp(s - s.max(1, keepdims=True)); w /= w.sum(1, keepdims=True)
    tol = (2.0 ** -8 + 2 * ds + 2.0 ** -16) * (w @ np.abs(vv[:, 0]) + np.abs(want[0]))          # element by element
    assert np.all(np.abs(out[0, 0].double().cpu().numpy() - want[0]) <= tol)
    held_equals(pool, model, {0: store}, [0])


def test_tokens_one_and_several_at_a_time(lib):
    """Tokens of growing and shrinking magnitude into the same pages, layer by layer and all layers at once."""
    import torch
    for d in (128, 64):
        hq, hkv, L = 4, 2, 3
        pool = _pool(lib, 8, hq=hq, hkv=hkv, d=d, layers=L, max_step_queries=17)
        model = PoolModel(8, 16)
        stores = {l: Kv4Store(8, 16, hkv, d) for l in range(L)}
        pool.request_begin(); model.request_begin()
        rng = np.random.default_rng(5)
        for step, n in enumerate([1, 1, 3, 1, 5, 1, 1, 7, 1, 17, 2, 6, 1, 1, 1, 4]):
            gain = torch.from_numpy(2.0 ** rng.integers(-12, 13, (L, n, hkv, 1))).float()
            k = (_randn((L, n, hkv, d), 20 + step).float() * gain).to(torch.bfloat16)
            v = (_randn((L, n, hkv, d), 60 + step).float() / gain).to(torch.bfloat16)
            pool.step_begin([0], [0], [n])
            slots = model.reserve([(0, 0, n)])
            if step % 2:
                pool.kv_append(k.cuda(), v.cuda())
            else:
                for l in range(L):
                    pool.kv_append(k[l:l + 1].cuda(), v[l:l + 1].cuda(), layer_begin=l, layer_count=1)
            for l in range(L):
                stores[l].write(slots, k[l], v[l])
        held_equals(pool, model, stores, list(range(L)))
        assert pool.status() == 0


def test_pages_used_before_by_others(lib):
    """A request's pages go to the next one: what stood in them before is neither seen nor does it spoil anything."""
    import torch
    for d in (64, 128):
        pool = _pool(lib, 20, hq=8, hkv=2, d=d)
        model, store = PoolModel(20, 16), Kv4Store(20, 16, 2, d)
        for round_, (n, gain) in enumerate([(300, 1e30), (37, 1.0), (161, 1e-3), (5, 1.0)]):
            assert pool.request_begin() == model.request_begin()
            k, v = _randn((1, n, 2, d), 70 + round_), _randn((1, n, 2, d), 80 + round_, gain)
            pool.kv_append_run(0, 0, n, k.cuda(), v.cuda()); store.write(model.append_run(0, 0, n), k[0], v[0])
            q = _randn((1, 1, 8, d), 90 + round_)
            pool.step_begin([0], [0], [0])
            out = torch.empty((1, 1, 8, d), device="cuda"); lse = torch.empty((1, 1, 8), device="cuda")
            pool.decode_attn(q.cuda(), out, lse)
            want, want_lse = decode_attention_capped(model, store, [(0, 0)], q[0])
            fresh = Kv4Store(1, 16, 2, d)
            fresh.k, fresh.v = store.gather(model.visible_slots(0, 0))
            compare(out[0], lse[0], want, want_lse, q[0].float().numpy(), fresh)
            pool.request_end(0); model.request_end(0)


@pytest.mark.parametrize("d", [128, 64])
def test_values_that_are_not_finite_are_stored_as_zero_and_reported(lib, d):
    import torch
    pool = _pool(lib, 4, d=d)
    model, store = PoolModel(4, 16), Kv4Store(4, 16, 2, d)
    pool.request_begin(); model.request_begin()
    k, v = _randn((1, 40, 2, d), 1), _randn((1, 40, 2, d), 2)
    k[0, 3, 0, 5] = float("nan"); k[0, 20, 1, d // 2] = float("inf"); v[0, 39, 1, d - 1] = float("-inf"); v[0, 17, 0, 0] = float("nan")
    v[0, 5, 0, 0] = 3e38; k[0, 6, 0, 0] = -3e38                        # finite, beyond the range: saturate
    pool.kv_append_run(0, 0, 40, k.cuda(), v.cuda()); store.write(model.append_run(0, 0, 40), k[0], v[0])
    assert store.nonfinite == 4
    held_equals(pool, model, {0: store}, [0])
    assert pool.status() == lib.DEVICE_CHECK and pool.status() == 0
    pool.set_rope(rotary_dim=32)
    pool.step_begin([0], [0], [1])                                    # a rotated pair with an infinity in it: both zero; beyond: one
    k1, v1 = _randn((1, 1, 2, d), 3), _randn((1, 1, 2, d), 4)
    k1[0, 0, 1, 20] = float("inf"); k1[0, 0, 0, 40] = float("nan")
    pool.kv_append_rope(k1.cuda(), v1.cuda(), 10000.0)
    got, _ = pool.kv_read(0, 0, 0, 40, 1)
    clean = k1[0].float().numpy()
    clean[0, 1, 20] = clean[0, 1, 4] = clean[0, 0, 40] = 0
    store.write([(0, 0)], turned(clean, [40], 1e4, {"rotary_dim": 32}), v1[0])
    assert np.array_equal(got.double().cpu().numpy()[0], store.k[0, 0])
    assert pool.status() == lib.DEVICE_CHECK


@pytest.mark.parametrize("d,theta,runs", [(64, 10000.0, [5, 2048 * 16 + 200]), (64, 0.0, [11, 65 * 16, 2048 * 16]),
                                          (128, 500000.0, [1, 63 * 16, 16, 64 * 16 + 15])])
def test_runs_of_more_pages_than_a_launch_carries(lib, d, theta, runs):
    """Runs around and beyond the two sizes of page list, starting inside a page; read back, appended again, and read again."""
    import torch
    n = sum(runs)
    pool = _pool(lib, 2 * (n // 16 + 1), requests=2, hq=1, hkv=1, d=d)
    model, store = PoolModel(2 * (n // 16 + 1), 16, None, 2), Kv4Store(2 * (n // 16 + 1), 16, 1, d)
    pool.request_begin(); model.request_begin()
    at = 0
    for i, m in enumerate(runs):
        k, v = _randn((1, m, 1, d), 30 + i, gain=2.0 ** i), _randn((1, m, 1, d), 40 + i)
        slots = model.append_run(0, 0, m)
        if theta:
            pool.kv_append_run_rope(0, 0, m, k.cuda(), v.cuda(), theta)
            store.write(slots, turned(k[0], np.arange(at, at + m), theta, {}), v[0])
        else:
            pool.kv_append_run(0, 0, m, k.cuda(), v.cuda())
            store.write(slots, k[0], v[0])
        at += m
    held_equals(pool, model, {0: store}, [0])
    k, v = pool.kv_read_layers(0, 0, 7, n - 9)                        # a part, neither end on a page
    slots = [(p, o) for p, o in model.visible_slots(0, 0)][7:n - 2]
    wk, wv = store.gather(slots)
    assert np.array_equal(k[0].double().cpu().numpy(), wk) and np.array_equal(v[0].double().cpu().numpy(), wv)
    r = pool.request_begin()
    pool.kv_append_run(r, 0, n - 9, k, v)
    k2, v2 = pool.kv_read_layers(r, 0, 0, n - 9)
    assert torch.equal(k, k2) and torch.equal(v, v2)
    assert pool.status() == 0


@pytest.mark.parametrize("theta", [0.0, 10000.0])
def test_numbers_at_the_ends_of_the_range(lib, theta):
    import torch
    sizes = [0.0, 2.0 ** -133, 2.0 ** -127, 2.0 ** -126, 2.0 ** -110, 2.0 ** -108, 2.0 ** -70, 1.0, 2.0 ** 60, 2.0 ** 111, 2.0 ** 114, 3.3e38]
    n = 16 * (len(sizes) + 1)
    pool = _pool(lib, n // 16)
    model, store = PoolModel(n // 16, 16), Kv4Store(n // 16, 16, 2, 128)
    pool.request_begin(); model.request_begin()
    g = torch.Generator().manual_seed(3)
    unit = (1.0 - 2.0 * torch.randint(0, 2, (1, n, 2, 128), generator=g)) * (1 + torch.randint(0, 8, (1, n, 2, 128), generator=g) / 8.1)
    gain = torch.tensor(sizes + [1.0]).repeat_interleave(16).reshape(1, n, 1, 1).repeat(1, 1, 2, 1) / 2
    gain[0, -16:, 0, 0] = torch.tensor((sizes * 2)[:16]) / 2            # the last page mixes them
    k, v = (unit * gain).to(torch.bfloat16), (unit.flip(1) * gain).to(torch.bfloat16)
    slots = model.append_run(0, 0, n)
    if theta:
        pool.kv_append_run_rope(0, 0, n, k.cuda(), v.cuda(), theta)
        with np.errstate(over="ignore"):
            store.write(slots, turned(k[0], np.arange(n), theta, {}), v[0])
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
    # equal weights are rounded alike and their sum with them
    assert (out[0, 0].double() - mean).abs().max() <= 2.0 ** -16 * held.double().abs().max()
    assert (lse[0, 0].double() - np.log(n)).abs().max() <= 2.0 ** -8
    assert pool.status() == 0


@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("threads,n", [(1, 1), (1, 300), (2, 3000), (9, 700), (17, 5), (17, 3000), (31, 400), (33, 300)])
@pytest.mark.parametrize("d,flags", [(128, 0), (64, 0), (128, 2), (64, 2), (128, 4)])
def test_query_rows_that_are_not_finite(lib, d, flags, threads, n, cap):
    """They come out as NaN on every kernel, and spoil no other row."""
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


@pytest.mark.parametrize("d", [128, 64])
def test_every_way_to_run_a_step_gives_the_same(lib, d):
    """decode_attn on another stream, captured and replayed, per layer, without workspace, through step_device and step_host,
    with launches that do not overlap, and with bf16 outputs."""
    import torch
    hq, hkv, L, T = 8, 2, 3, 5
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
        pool.kv_append(kn, vn)
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


def test_pages_beyond_four_gigabytes(lib):
    """Pages at the far end of a pool of more than 4 GiB hold and give what pages at the near end do."""
    import torch
    n_pages, hkv = 240_000, 8
    order = list(range(n_pages - 30, n_pages)) + list(range(n_pages - 30))
    outs = []
    for free_order in (None, order):
        pool = lib.Pool(1, 32, hkv, 128, n_pages, 1, 3, 8, flags=lib.FLAG_KV_INT4, free_order=free_order)
        assert pool.kv.numel() > 1 << 32
        pool.request_begin()
        k, v = _randn((1, 333, hkv, 128), 1).cuda(), _randn((1, 333, hkv, 128), 2).cuda()
        pool.kv_append_run_rope(0, 0, 333, k, v)
        pool.thread_spawn(0)
        pool.step_begin([0, 0], [0, 1])
        pool.kv_append(k[:, :2].contiguous(), v[:, :2].contiguous())
        out = torch.empty((1, 2, 32, 128), device="cuda")
        pool.decode_attn(_randn((1, 2, 32, 128), 3).cuda(), out)
        outs.append((out,) + pool.kv_read(0, 0, 0, 0, 334) + pool.kv_read(0, 0, 1, 0, 1))
        assert pool.status() == 0
        pool.close()
        del pool
        torch.cuda.empty_cache()
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_many_requests_and_layers(lib):
    """Several units per CTA, units handed out at run time, more layers than a launch takes; sampled queries against the oracle."""
    import torch
    hq, hkv, d, L, R = 32, 8, 128, 3, 40
    lengths = [150 + 53 * i for i in range(R)]
    pages = sum(n // 16 + 4 for n in lengths)
    pool = _pool(lib, pages, requests=R, threads=3, hq=hq, hkv=hkv, d=d, layers=L, max_step_queries=3 * R, max_layers_per_launch=2)
    model = PoolModel(pages, 16, None, R, 3, 8)
    stores = {l: Kv4Store(pages, 16, hkv, d) for l in (0, 2)}
    for r, n in enumerate(lengths):
        pool.request_begin(); model.request_begin()
        k, v = _randn((L, n, hkv, d), r), _randn((L, n, hkv, d), 100 + r)
        pool.kv_append_run(r, 0, n, k.cuda(), v.cuda())
        slots = model.append_run(r, 0, n)
        for l in stores:
            stores[l].write(slots, k[l], v[l])
        for _ in range(r % 3):
            pool.thread_spawn(r); model.thread_spawn(r)
    entries = [(r, t, int(t > 0)) for r in range(R) for t in range(1 + r % 3)]
    n_app = sum(e[2] for e in entries)
    k, v, q = _randn((L, n_app, hkv, d), 7), _randn((L, n_app, hkv, d), 8), _randn((L, len(entries), hq, d), 9)
    pool.step_begin([e[0] for e in entries], [e[1] for e in entries], [e[2] for e in entries])
    slots = [s for s in model.reserve(entries) if s is not None]
    pool.kv_append(k.cuda(), v.cuda())
    out = torch.empty((L, len(entries), hq, d), device="cuda"); lse = torch.empty((L, len(entries), hq), device="cuda")
    pool.decode_attn(q.cuda(), out, lse)
    for l in stores:
        stores[l].write(slots, k[l], v[l])
        for i in range(l, len(entries), 13):
            want, want_lse = decode_attention_capped(model, stores[l], [model.queries_of(entries)[i]], q[l, i:i + 1])
            compare(out[l, i:i + 1], lse[l, i:i + 1], want, want_lse, q[l, i:i + 1].float().numpy(), stores[l], what=(l, i))
    again = torch.empty_like(out)
    pool.decode_attn(q.cuda(), again)
    assert torch.equal(again, out) and pool.status() == 0


def test_naive_rows_copy_what_is_held(lib):
    """The comparison layout duplicates a row by reading and appending it: the same codes, hence the same results."""
    import torch
    from paper_2502_11517_b200.naive_rows import NaiveRows
    pool = lib.Pool(2, 8, 2, 128, 40, 3, 1, 4, flags=lib.FLAG_KV_INT4)
    rows = NaiveRows(pool)
    rows.begin(0)
    rows.run(0, 0, 100, _randn((2, 100, 2, 128), 1).cuda(), _randn((2, 100, 2, 128), 2).cuda())
    rows.spawn(0, 1)
    q = _randn((2, 1, 8, 128), 3).cuda().repeat(1, 2, 1, 1)
    out = torch.empty((2, 2, 8, 128), device="cuda")
    nothing = torch.empty((2, 0, 2, 128), dtype=torch.bfloat16, device="cuda")
    rows.step([(0, 0, 0), (0, 1, 0)], nothing, nothing, q, out)
    assert torch.equal(out[:, 0], out[:, 1]) and pool.status() == 0


def test_refusals(lib):
    """Tensors that are not aligned are refused; nothing is launched, and a refused append takes no slot."""
    import torch
    with pytest.raises(lib.PastaError) as e:
        lib.Pool(1, 8, 2, 128, 4, 1, 1, 4, flags=lib.FLAG_KV_INT4 | lib.FLAG_KV_FP8)
    assert e.value.code == lib.INVALID_ARG
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
    launches = pool.launch_count()
    pool.step_begin([0], [0], [1])
    one = flat[:256].view(1, 1, 2, 128)
    q, out = flat[:1024].view(1, 1, 8, 128), torch.empty(1030, device="cuda")
    for k, v in ((flat[4:260].view(1, 1, 2, 128), one), (one, flat[4:260].view(1, 1, 2, 128))):
        with pytest.raises(lib.PastaError):
            pool.kv_append(k, v)
        with pytest.raises(lib.PastaError):
            pool.kv_append_rope(k, v, 10000.0)
    assert pool.launch_count() == launches
    pool.kv_append(one, one)
    for a, b in ((flat[1:1025].view(1, 1, 8, 128), out[:1024]), (q, out[1:1025])):
        with pytest.raises(lib.PastaError):
            pool.decode_attn(a, b)
        with pytest.raises(lib.PastaError):
            pool.decode_attn_noalloc(a, b)
        with pytest.raises(lib.PastaError):
            pool.step_device([0], [0], [1], one, one, a, b)
    assert pool.dump()["requests"][0]["streams"][0]["len"] == 21
    assert lib.lib().pasta_kv_read_layers(pool._h, 0, 1, 0, 0, 0, 20, lib._dev(odd), lib._dev(good), None) == lib.INVALID_ARG
    pool.decode_attn(q, out[:1024])
    assert pool.status() == 0


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("length", [100, 3000])
@pytest.mark.parametrize("levels", [(-5, -30, -39, -41), (-43, -60, -86, -88), (-95, -104, -140, 3), (20, 88, 300, -700)])
def test_rows_at_levels_from_faint_to_large(lib, d, length, levels):
    """Four rows of one unit whose scores all lie around the given numbers (natural units): some are within the range of a weight
    whose reference is zero, some below it, some above."""
    import torch
    q = torch.tensor(levels, dtype=torch.float32)[:, None] * torch.ones(4, d) / 8
    q = q.to(torch.bfloat16)[None, None]                                  # [1, 1, 4, d]
    k = torch.ones((1, length, 1, d)) * (8 / d ** 0.5) * (1 + 0.02 * _randn((1, length, 1, 1), 4).float())
    k, v = k.to(torch.bfloat16), _randn((1, length, 1, d), 2)
    pool = _pool(lib, length // 16 + 2, hq=4, hkv=1, d=d)
    model, store = PoolModel(length // 16 + 2, 16, None, 1, 1, 4), Kv4Store(length // 16 + 2, 16, 1, d)
    pool.request_begin(); model.request_begin()
    pool.kv_append_run(0, 0, length, k.cuda(), v.cuda()); store.write(model.append_run(0, 0, length), k[0], v[0])
    pool.step_begin([0], [0], [0])
    out = torch.empty((1, 1, 4, d), device="cuda"); lse = torch.empty((1, 1, 4), device="cuda")
    for _ in range(2):
        pool.decode_attn(q.cuda(), out, lse)
        want, want_lse = decode_attention_capped(model, store, [(0, 0)], q[0])
        compare(out[0], lse[0], want, want_lse, q[0].float().numpy(), store)
    assert pool.status() == lib.OK
