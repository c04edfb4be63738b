"""Plans of 4-bit pools of many layers: a launch of one layer goes by the assignment that a pool of one layer would get."""
import numpy as np
import pytest

from paper_2502_11517_b200 import binding, build
from test_plan_kv4_rows import long_prompts, run

N_TUNITS, T_GRID, OFF_TRANGE, OFF_TUNIT, OFF_TCTA, N_DUNITS, OFF_DUNIT, OFF_DRANGE, FEWEST, OFF_FEW = 4, 8, 12, 13, 14, 23, 24, 25, 29, 30


@pytest.fixture(scope="module", autouse=True)
def _built():
    build()


def words(lengths, forks, layers, hq=32, hkv=8, **kw):
    pool = long_prompts(lengths, forks, hq=hq, hkv=hkv, layers=layers, **kw)
    w = np.array(pool.plan_words())
    pool.close()
    return w


def by_header(w, at):
    """The plan as the header at that word gives it."""
    w = w.copy()
    w[:32] = w[at:at + 32]
    return w


def tables(w):
    """Units, ranges of CTAs and ranges of runs."""
    return [w[w[off]:w[off] + n].tolist() for off, n in ((OFF_TUNIT, 12 * w[N_TUNITS]), (OFF_DUNIT, 12 * w[N_DUNITS]), (OFF_TCTA, 2 * w[T_GRID]))]


STEPS = [([256 + 119 * i for i in range(16)], 4), ([4096, 5500, 7000, 8192], 0), ([2000 + 850 * i for i in range(8)], 0), ([32768] * 8, 16),
         ([90000] + [40 + 90 * i for i in range(12)] + [70000], 1)]


@pytest.mark.parametrize("lengths,forks", STEPS)
@pytest.mark.parametrize("layers", [2, 8, 32])
def test_one_layer_of_many(lengths, forks, layers):
    alone, main = words(lengths, forks, 1), words(lengths, forks, layers)
    assert alone[FEWEST] == 0
    one = by_header(main, main[OFF_FEW]) if main[FEWEST] > 1 else main
    assert tables(one) == tables(alone)


@pytest.mark.parametrize("lengths,forks", STEPS[:3])
def test_each_number_of_layers(lengths, forks):
    """Whole from as many layers on as the header says, and what a pool with launches of that many would do."""
    main = words(lengths, forks, 8)
    fewest = int(main[FEWEST])                                       # (0: one assignment for all)
    assert fewest <= 8 and (fewest > 1 or len(lengths) != 16)
    for n in range(1, 9):
        assert (tables(words(lengths, forks, 32, max_layers_per_launch=n)) == tables(main)) == (n >= fewest)


@pytest.mark.parametrize("hq,hkv,lengths,forks", [(8, 2, [4000, 3000, 300], 2), (4, 1, [2500], 12), (8, 2, [3000], 25)])
def test_executed(hq, hkv, lengths, forks):
    pool = long_prompts(lengths, forks, hq=hq, hkv=hkv, layers=8, max_layers_per_launch=8)
    w = np.array(pool.plan_words())
    run(pool, w, hq, hkv)
    if w[FEWEST] > 1:
        assert w[OFF_FEW] % 4 == 0
        run(pool, by_header(w, w[OFF_FEW]), hq, hkv)
    pool.close()


def test_steps_of_short_runs_have_one_assignment():
    assert words([300] * 4, 2, 32)[FEWEST] == 0
