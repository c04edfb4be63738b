"""Plans of 4-bit pools, executed on the CPU: whole runs handed out at run time (the longest first), runs cut into shares in advance,
and both in one step."""
import numpy as np
import pytest

import plan_interpreter
from paper_2502_11517_b200 import binding, build
from pasta_workloads import Geometry, cfg1_tiny, cfg3_batched, cfg4_long_prefix, random_script
from test_plan import check_script


@pytest.fixture(scope="module", autouse=True)
def _built():
    build()


@pytest.mark.parametrize("seed", range(40, 46))
@pytest.mark.parametrize("geo", [Geometry(1, 4, 2, 64, 16), Geometry(1, 8, 2, 128, 16), Geometry(1, 4, 4, 128, 16)])
@pytest.mark.parametrize("tail", [None, (0, 16)])
def test_random_scripts(seed, geo, tail):
    stats = check_script(random_script(seed, n_ops=70, geo=geo), flags=binding.FLAG_KV_INT4, tail=tail)
    assert (stats["tunits"] > 0) == (tail is not None)          # short runs: all handed out at run time, or none


def _shares(script, steps=None, **kw):
    """Units assigned in advance, units handed out at run time, and plans without partial rows."""
    before = plan_interpreter.STATS.get("dunits", 0), plan_interpreter.STATS.get("no_merge_plans", 0)
    stats = check_script(script, flags=binding.FLAG_KV_INT4, steps=steps, **kw)
    return (stats["tunits"], plan_interpreter.STATS["dunits"] - before[0],
            plan_interpreter.STATS.get("no_merge_plans", 0) - before[1], stats["steps"])


@pytest.mark.parametrize("maker,layers,whole", [(lambda: cfg1_tiny(), 1, True), (lambda: cfg3_batched(24, 1, prefix_range=(20, 900)), 8, True),
                                                (lambda: cfg3_batched(24, 1, prefix_range=(20, 900)), 1, False),
                                                (lambda: cfg4_long_prefix(2, 3000, 3), 1, False)])
def test_runs_stay_whole_unless_they_take_longer_than_a_launch(maker, layers, whole):
    """Launches of several layers have other units to fill the time that the longest run takes; one layer's have not."""
    assigned, shared, final, steps = _shares(maker(), layers=layers)
    if whole:
        assert assigned == 0 and shared > 0 and final == steps
    else:
        assert assigned > 0 and final < steps


def test_a_step_of_both():
    """Two long texts among short ones: the long ones are cut over the CTAs, short ones are handed out whole."""
    lengths = [90000] + [40 + 90 * i for i in range(12)] + [70000]
    geo = Geometry(1, 4, 2, 128, 16)
    pool = binding.Pool(8, geo.n_q_heads, geo.n_kv_heads, geo.head_dim, sum(n // 16 + 2 for n in lengths), len(lengths), 1, 2,
                        flags=binding.FLAG_KV_INT4 | binding.FLAG_HOST_ONLY)
    for r, n in enumerate(lengths):
        assert pool.request_begin() == r
        pool.kv_append_run(r, 0, n)
    pool.step_begin(list(range(len(lengths))), [0] * len(lengths), [0] * len(lengths))
    w = np.array(pool.plan_words())
    assert w[4] > 4 and 0 < w[23] <= 2 * 12
    # (every CTA takes part in handing out; those with nothing assigned come last, and are not what the interpreter looks at)
    cta = w[w[14]: w[14] + 2 * w[8]].reshape(-1, 2)
    w[8] = int((cta[:, 1] > cta[:, 0]).sum())
    rng = np.random.default_rng(1)
    K, V = rng.standard_normal((2, sum(n // 16 + 2 for n in lengths), 16, 2, 128))
    q = rng.standard_normal((len(lengths), 4, 128))
    got, _ = plan_interpreter.run_plan(w, K, V, q, 2)
    for r, n in enumerate(lengths):
        pages = pool.dump()["requests"][r]["streams"][0]["pages"]
        k, v = K[pages].reshape(-1, 2, 128)[:n], V[pages].reshape(-1, 2, 128)[:n]
        for h in range(4):
            s = k[:, h // 2] @ q[r, h] / np.sqrt(128)
            p = np.exp(s - s.max())
            np.testing.assert_allclose(got[r, h], p @ v[:, h // 2] / p.sum(), rtol=0, atol=1e-11)
    pool.close()


def test_without_room_for_more_rows():
    """With room for one row set per run, runs are not cut into more pieces than fit, or the step is refused."""
    script = cfg4_long_prefix(2, 3000, 3)
    with pytest.raises(binding.PastaError):
        check_script(script, flags=binding.FLAG_KV_INT4, max_partial_rows=8)


@pytest.mark.parametrize("threads,parts", [(20, 1), (21, 2), (40, 2), (41, 3), (160, 8), (161, 0)])
def test_requests_of_many_threads_are_split(threads, parts):
    """80 rows to a part, 8 parts at most, more rows take the warp path; every query is in one part."""
    pool = binding.Pool(1, 8, 2, 128, 40 + 2 * threads, 1, threads, 2 * threads + 2,
                        flags=binding.FLAG_KV_INT4 | binding.FLAG_HOST_ONLY, max_step_queries=threads)
    pool.request_begin()
    pool.kv_append_run(0, 0, 200)
    for t in range(1, threads):
        assert pool.thread_spawn(0) == t
        pool.kv_append_run(0, t, 1 + t % 20)
    pool.step_begin([0] * threads, list(range(threads)), [0] * threads)
    w = np.array(pool.plan_words())
    assert w[3] == parts and w[4] + w[23] >= 2 * parts and (w[5] > 0) == (parts == 0)
    rng = np.random.default_rng(2)
    K, V = rng.standard_normal((2, 40 + 2 * threads, 16, 2, 128))
    q = rng.standard_normal((threads, 8, 128))
    got, _ = plan_interpreter.run_plan(w, K, V, q, 2)
    streams = pool.dump()["requests"][0]["streams"]
    for t in range(threads):
        k, v = (np.concatenate([X[streams[i]["pages"]].reshape(-1, 2, 128)[:streams[i]["len"]] for i in ([0, t] if t else [0])]) for X in (K, V))
        for h in range(8):
            s = k[:, h // 4] @ q[t, h] / np.sqrt(128)
            p = np.exp(s - s.max())
            np.testing.assert_allclose(got[t, h], p @ v[:, h // 4] / p.sum(), rtol=0, atol=1e-11)
    pool.close()
