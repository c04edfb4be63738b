"""Plans of 4-bit pools that have room for few partial rows: runs are cut into fewer pieces, or not at all, before a step is refused."""
import numpy as np
import pytest

import plan_interpreter
from paper_2502_11517_b200 import binding, build


@pytest.fixture(scope="module", autouse=True)
def _built():
    build()


def long_prompts(lengths, forks, hq=8, hkv=2, d=128, layers=1, flags=0, **kw):
    """A step of prompts with forks that have one token each; host only."""
    T = forks + 1
    pool = binding.Pool(layers, hq, hkv, d, sum(n // 16 + 1 + forks for n in lengths), len(lengths), T, 2 * T + 2,
                        flags=flags | binding.FLAG_KV_INT4 | binding.FLAG_HOST_ONLY, max_step_queries=len(lengths) * T, **kw)
    for r, n in enumerate(lengths):
        pool.request_begin()
        pool.kv_append_run(r, 0, n)
        for _ in range(forks):
            pool.thread_spawn(r)
    R = len(lengths)
    try:
        pool.step_begin([r for r in range(R) for _ in range(T)], list(range(T)) * R, ([0] + [1] * forks) * R)
    except binding.PastaError:
        pool.close()
        raise
    return pool


def run(pool, w, hq=8, hkv=2, d=128):
    """The plan executed, against attention over what each thread sees."""
    w = w.copy()
    cta = w[w[14]: w[14] + 2 * w[8]].reshape(-1, 2)
    w[8] = int((cta[:, 1] > cta[:, 0]).sum())                          # (CTAs that only take part in handing out come last)
    dump = pool.dump()
    n_pages = sum(len(s["pages"]) for r in dump["requests"].values() for s in r["streams"].values()) + len(dump["free"])
    rng = np.random.default_rng(3)
    K, V = rng.standard_normal((2, n_pages, 16, hkv, d))
    threads = [(r, t) for r, q in sorted(dump["requests"].items()) for t in sorted(q["threads"])]
    q = rng.standard_normal((len(threads), hq, d))
    got, _ = plan_interpreter.run_plan(w, K, V, q, hkv)
    for i, (r, t) in enumerate(threads):
        streams = dump["requests"][r]["streams"]
        k, v = (np.concatenate([X[streams[j]["pages"]].reshape(-1, hkv, d)[:streams[j]["len"]] for j in ([0, t] if t else [0])]) for X in (K, V))
        for h in range(hq):
            s = k[:, h * hkv // hq] @ q[i, h] / np.sqrt(d)
            p = np.exp(s - s.max())
            np.testing.assert_allclose(got[i, h], p @ v[:, h * hkv // hq] / p.sum(), rtol=0, atol=1e-11)


@pytest.mark.parametrize("flags", [0, binding.FLAG_NO_TENSOR_PATH])
@pytest.mark.parametrize("lengths,forks", [([4000, 3000], 3), ([6000], 8), ([4000, 40, 300, 3000, 200], 2), ([2000], 25)])
def test_fewer_cuts_before_a_refusal(lengths, forks, flags):
    pool = long_prompts(lengths, forks, flags=flags)
    free = np.array(pool.plan_words())
    pool.close()
    whole = len(lengths) * (forks + 1) * 8                            # partial rows of runs that are not cut, one set per query and head
    if not flags:
        assert free[7] > 2 * whole                                    # with room for them the runs are cut
    least = whole if not flags else len(lengths) * (2 * forks + 1) * 8     # (on the warp path: every stream apart)
    seen = set()
    for rows in sorted({least, (least + int(free[7])) // 2, int(free[7]) - 1}):
        pool = long_prompts(lengths, forks, flags=flags, max_partial_rows=rows)
        w = np.array(pool.plan_words())
        assert w[7] <= rows
        run(pool, w)
        seen.add(int(w[4]) + int(w[23]) + int(w[5]))
        pool.close()
    assert len(seen) >= 2                                             # as many cuts as there is room for
    with pytest.raises(binding.PastaError) as e:
        long_prompts(lengths, forks, flags=flags, max_partial_rows=least - 1)
    assert e.value.code == binding.CAPACITY
