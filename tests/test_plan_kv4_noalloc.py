"""Plans of 4-bit pools for the call that has a fixed number of partial rows: where the step's own need more, there is an assignment that fits."""
import numpy as np
import pytest

from paper_2502_11517_b200 import binding, build
from test_plan_kv4_layers import by_header, tables, words
from test_plan_kv4_rows import long_prompts, run

ROWS, FEWEST, OFF_FEW, OFF_NOALLOC, MOST = 7, 29, 30, 31, 16384


@pytest.fixture(scope="module", autouse=True)
def _built():
    build()


@pytest.mark.parametrize("layers", [1, 8, 32])
@pytest.mark.parametrize("lengths,forks", [([32768] * 8, 16), ([12000], 16), ([60000, 200, 3000], 18), ([20000] * 4, 19)])
def test_there_is_one_that_fits(lengths, forks, layers):
    w = words(lengths, forks, layers)
    one = by_header(w, w[OFF_FEW]) if w[FEWEST] > 1 else w
    assert one[ROWS] > MOST and w[OFF_NOALLOC] > 0
    tight = by_header(w, w[OFF_NOALLOC])
    assert MOST // 2 < tight[ROWS] <= MOST and tight[FEWEST] == tight[OFF_FEW] == tight[OFF_NOALLOC] == 0
    assert tables(tight) != tables(one)


@pytest.mark.parametrize("lengths,forks,flags", [([300] * 6, 2, 0), ([9000], 3, 0), ([12000], 16, binding.FLAG_OUT_BF16),
                                                 ([40] * 32, 16, 0)])
def test_there_is_none_where_none_is_needed_or_possible(lengths, forks, flags):
    w = words(lengths, forks, 8, flags=flags)
    assert w[OFF_NOALLOC] == 0 and (w[ROWS] <= MOST or flags or len(lengths) * (forks + 1) * 32 > MOST)


def test_executed():
    pool = long_prompts([7000], 16, hq=32, hkv=8)
    w = np.array(pool.plan_words())
    assert w[ROWS] > MOST
    run(pool, by_header(w, w[OFF_NOALLOC]), 32, 8)
    pool.close()
