"""Pins for the oracle of 4-bit pools (closed forms and properties) and host checks of the pools' configuration."""
import ctypes as C

import numpy as np
import pytest

from oracle.kv4 import GROUP, SCALE_MAX, SCALE_MIN, Kv4Store, held, scales


def _lib():
    from paper_2502_11517_b200 import binding, build
    build()
    return binding


def _brute(amax):
    """Smallest m * 2^e, m = 16 .. 31, with amax <= 7 m 2^e."""
    return min(m * 2.0 ** e for e in range(-120, 110) for m in range(16, 32) if amax <= 7 * m * 2.0 ** e)


def test_scales_are_the_smallest_that_hold_the_largest():
    rng = np.random.default_rng(1)
    for amax in [7.0, 7.0001, 6.9999, 16 * 7 / 8, 17 * 7.0, 31 * 7.0, np.float32(31 * 7) * (1 + 2.0 ** -23), 1.0, 3.0] + list(
            np.exp(rng.uniform(-60, 60, 40)).astype(np.float32)):
        x = np.zeros(GROUP)
        x[5] = -float(amax)
        assert scales(x)[0] == _brute(float(amax)), amax


def test_ties_go_to_the_even_number():
    x = np.zeros(GROUP)
    x[:9] = [7, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 6.5, -6.5]
    assert held(x)[:9].tolist() == [7, 0, 2, 2, 0, -2, -2, 6, -6]


def test_zeros_and_the_ends_of_the_range():
    x = np.zeros((3, GROUP))
    x[1, 0], x[2, 0], x[2, 1] = 2.0 ** -113, 3e38, -1e33
    assert scales(x)[:, 0].tolist() == [SCALE_MIN, SCALE_MIN, SCALE_MAX]
    assert held(x)[0].max() == 0 and held(x)[1].max() == 0
    assert held(x)[2, 0] == 7 * SCALE_MAX and held(x)[2, 1] == 0


def test_error_is_below_a_thirteenth_and_the_result_holds_itself():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((500, 4 * GROUP)).astype(np.float32).astype(np.float64) * np.exp(rng.uniform(-20, 20, (500, 1)))
    y = held(x)
    amax = np.abs(x.reshape(500, 4, GROUP)).max(-1)
    assert (np.abs(y - x).reshape(500, 4, GROUP).max(-1) < amax / 13).all()
    assert np.array_equal(held(y), y) and np.array_equal(scales(y), scales(x))
    bits = y.astype(np.float32).view(np.uint32)
    assert not (bits & 0xFFFF).any() and np.array_equal(y.astype(np.float32), y)          # bf16 numbers


def test_a_token_depends_on_itself_alone():
    rng = np.random.default_rng(3)
    k, v = rng.standard_normal((2, 20, 2, 64)).astype(np.float32)
    one, many = Kv4Store(2, 16, 2, 64), Kv4Store(2, 16, 2, 64)
    slots = [(i // 16, i % 16) for i in range(20)]
    one.write(slots, k, v)
    for i in reversed(range(20)):
        many.write([slots[i]], k[i:i + 1], v[i:i + 1])
    assert np.array_equal(one.k, many.k) and np.array_equal(one.v, many.v)


def test_sizes_and_flags():
    b = _lib()
    cfg = b.Config(n_layers=3, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, n_pages=5, max_requests=1,
                   max_threads_per_request=1, max_segments_per_thread=2, flags=b.FLAG_KV_INT4 | b.FLAG_HOST_ONLY)
    size = C.c_size_t()
    assert b.lib().pasta_kv_bytes(C.byref(cfg), C.byref(size)) == b.OK
    assert size.value == 3 * 5 * 2 * 18 * 128
    cfg.flags |= b.FLAG_KV_FP8
    assert b.lib().pasta_kv_bytes(C.byref(cfg), C.byref(size)) == b.INVALID_ARG
    assert b.lib().pasta_workspace_bytes(C.byref(cfg), C.byref(size)) == b.INVALID_ARG
    handle = C.c_void_p()
    assert b.lib().pasta_pool_create(C.byref(cfg), C.byref(handle)) == b.INVALID_ARG and not handle


@pytest.mark.parametrize("d", [64, 128])
def test_bookkeeping_is_that_of_any_pool(d):
    b = _lib()
    dumps = []
    for flags in (0, b.FLAG_KV_INT4):
        pool = b.Pool(1, 8, 2, d, 20, 2, 4, 12, flags=flags | b.FLAG_HOST_ONLY)
        r = pool.request_begin()
        pool.kv_append_run(r, 0, 37)
        t = pool.thread_spawn(r)
        pool.step_begin([r, r], [0, t], [1, 3])
        pool.thread_finish(r, t)
        pool.sync_merge(r)
        dumps.append(pool.dump())
    assert dumps[0] == dumps[1]
