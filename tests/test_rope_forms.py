"""Forms of the rotary embedding on the host: the oracle's properties, the library's frequencies, refusals.

Frequencies agree with the oracle's to 2^-46 relative: a power, a logarithm or a few products on either side, each good to a few
times 2^-53, with exponents of at most 30 in front of them."""
import ctypes as C

import numpy as np
import pytest

from oracle import rope
from oracle.kv4 import frequencies, rotate_form

FORMS = [{}, {"layout": "interleaved"}, {"rotary_dim": 16}, {"rotary_dim": 48, "layout": "interleaved"}, {"scaling": "linear", "factor": 2.5},
         {"scaling": "base", "factor": 4.0, "rotary_dim": 32}, {"scaling": "base", "factor": 8.0},
         {"scaling": "wavelength", "factor": 8.0, "original_length": 8192.0},
         {"scaling": "wavelength", "factor": 32.0, "original_length": 500.0, "low": 0.5, "high": 9.0, "layout": "interleaved"},
         {"scaling": "ramp", "factor": 4.0, "original_length": 4096.0, "high": 32.0},
         {"scaling": "ramp", "factor": 16.0, "original_length": 6.0, "high": 32.0},
         {"scaling": "ramp", "factor": 2.0, "original_length": 2048.0, "low": 2.0, "high": 3.0, "magnitude": 1.25, "rotary_dim": 64},
         {"magnitude": 0.5, "rotary_dim": 32}]


def _pool(d=128):
    from paper_2502_11517_b200 import binding, build
    build()
    return binding, binding.Pool(1, 8, 2, d, 4, 1, 1, 2, flags=binding.FLAG_HOST_ONLY)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("d,theta", [(128, 10000.0), (64, 500000.0)])
def test_frequencies(form, d, theta):
    b, pool = _pool(d)
    for _ in range(2):
        pool.set_rope(**form)
        f, size = pool.rope_frequencies(theta)
        want, want_size = frequencies(d, theta, form)
        assert len(f) == len(want) and np.abs(f / want - 1).max() <= 2.0 ** -46 and abs(size / want_size - 1) <= 2.0 ** -50
        pool.set_rope()
        f, size = pool.rope_frequencies(theta)
        assert len(f) == d // 2 and size == 1.0 and np.abs(f * theta ** (2.0 * np.arange(d // 2) / d) - 1).max() <= 2.0 ** -46


def test_the_usual_form_is_the_oracles():
    x = np.random.default_rng(0).standard_normal((9, 2, 64)).astype(np.float32)
    pos = np.array([0, 1, 2, 5, 100, 4096, 70001, 131072, 1000000])
    assert np.abs(rotate_form(x, pos, 10000.0, {}) - rope(x, pos)).max() <= 1e-9


@pytest.mark.parametrize("form", FORMS)
def test_properties(form):
    """Scores depend on distances only; rotated elements keep their size but for the magnitude; the rest stays as it is."""
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 1, 128)).astype(np.float32)
    R = form.get("rotary_dim") or 128
    size = frequencies(128, 1e4, form)[1]
    dots = [np.vdot(rotate_form(q, [a + 77], 1e4, form)[..., :R], rotate_form(k, [a], 1e4, form)[..., :R]) for a in (0, 5, 9000)]
    assert np.ptp(dots) <= 1e-9
    y = rotate_form(q, [12345], 1e4, form)
    assert abs(np.linalg.norm(y[..., :R]) - size * np.linalg.norm(q[..., :R].astype(np.float64))) <= 1e-9
    assert np.array_equal(y[..., R:], q[..., R:])


def test_interleaved_is_half_with_the_elements_in_another_order():
    x = np.random.default_rng(2).standard_normal((4, 1, 64)).astype(np.float32)
    order = np.concatenate([np.arange(0, 64, 2), np.arange(1, 64, 2)])
    a = rotate_form(x, [3, 50, 700, 9000], 1e4, {"layout": "interleaved"})[..., order]
    assert np.array_equal(a, rotate_form(x[..., order], [3, 50, 700, 9000], 1e4, {}))


def test_what_the_scalings_do_at_their_ends():
    one = {s: frequencies(128, 1e4, {"scaling": s, "factor": 1.0, "original_length": 4096.0, "high": 32.0})
           for s in ("none", "linear", "base", "wavelength", "ramp")}
    for f, size in one.values():
        assert np.abs(f / one["none"][0] - 1).max() <= 2.0 ** -50 and size == 1.0
    for s in ("wavelength", "ramp"):
        f, _ = frequencies(128, 1e4, {"scaling": s, "factor": 8.0, "original_length": 4096.0, "high": 32.0})
        assert f[0] == 1.0 and abs(f[-1] * 8 / one["none"][0][-1] - 1) <= 2.0 ** -50 and np.all(np.diff(f) < 0)
    f, _ = frequencies(128, 1e4, {"scaling": "base", "factor": 8.0})
    assert f[0] == 1.0 and abs(f[-1] * 8 / one["none"][0][-1] - 1) <= 2.0 ** -48           # the longest wave is stretched by the factor


def test_refusals():
    b, pool = _pool(64)
    good = {"layout": "interleaved", "rotary_dim": 32, "scaling": "ramp", "factor": 4.0, "original_length": 4096.0, "low": 1.0, "high": 32.0}
    pool.set_rope(**good)
    before = pool.rope_frequencies(1e4)
    nan, inf = float("nan"), float("inf")
    for change in ({"layout": "other"}, {"scaling": "other"}, {"rotary_dim": 8}, {"rotary_dim": -16}, {"rotary_dim": 80}, {"rotary_dim": 33},
                   {"factor": 0.5}, {"factor": nan}, {"factor": inf}, {"original_length": 0.0}, {"original_length": nan},
                   {"low": 0.0}, {"low": -1.0}, {"low": nan}, {"high": 1.0}, {"high": 0.5}, {"high": nan}, {"high": inf},
                   {"magnitude": -1.0}, {"magnitude": nan}, {"magnitude": 1e-9}, {"magnitude": inf}):
        with pytest.raises(b.PastaError) as e:
            pool.set_rope(**{**good, **change})
        assert e.value.code == b.INVALID_ARG
        after = pool.rope_frequencies(1e4)
        assert np.array_equal(after[0], before[0]) and after[1] == before[1]
    L, n = b.lib(), C.c_int32()
    form = b.RopeForm(0, 0, 0, 1, 1.0, 0.0, 0.0, 0.0, 0.0)
    assert L.pasta_set_rope(pool._h, C.byref(form)) == b.INVALID_ARG and L.pasta_set_rope(None, None) == b.INVALID_ARG
    ask = lambda theta, f, cap, count: L.pasta_rope_frequencies(pool._h, C.c_float(theta), f, cap, count, None)
    buf = (C.c_double * 64)()
    assert ask(1e4, None, 0, C.byref(n)) == b.OK and n.value == 16
    assert ask(1e4, buf, 15, C.byref(n)) == b.CAPACITY and ask(1e4, buf, 16, C.byref(n)) == b.OK
    assert ask(1e4, None, 16, C.byref(n)) == b.INVALID_ARG and ask(1e4, buf, -1, C.byref(n)) == b.INVALID_ARG
    assert ask(1e4, buf, 16, None) == b.INVALID_ARG
    for theta in (1.0, 0.0, -5.0, nan, inf):
        assert ask(theta, buf, 16, C.byref(n)) == b.INVALID_ARG
    assert L.pasta_set_rope(pool._h, None) == b.OK
    assert ask(1e4, None, 0, C.byref(n)) == b.OK and n.value == 32
    # what a scaling does not use is not looked at
    pool.set_rope(scaling="none", factor=nan, original_length=nan, low=nan, high=nan)
    pool.set_rope(scaling="linear", factor=2.0, original_length=nan, low=nan, high=nan)
    with pytest.raises(b.PastaError) as e:
        pool.rope_queries(None, 1e4, out=None, stream=0)                   # host-only pool
    assert e.value.code == b.BAD_STATE
    assert L.pasta_rope_queries_to(pool._h, 1, None, None, C.c_float(1e4), None) == b.BAD_STATE
