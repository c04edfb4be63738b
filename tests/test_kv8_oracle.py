"""CPU tests of the 8-bit cache's and the capped scores' oracle, of the plans made for an 8-bit pool, and of refusals."""
import ctypes

import dataclasses

import numpy as np
import pytest

from oracle import OracleReplay, PoolModel
from oracle.kv8 import Kv8Store, decode_attention_capped, e4m3_round, rotate, scale_exponent
from paper_2502_11517_b200 import binding, build
from pasta_workloads import Geometry, cfg3_batched, cfg4_long_prefix, random_script
from test_plan import check_script


@pytest.fixture(scope="module", autouse=True)
def _built():
    build()


def test_e4m3_rounding_agrees_with_the_type():
    import torch
    values = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    values = np.sort(values[np.isfinite(values)])
    assert np.array_equal(e4m3_round(values), values)
    rng = np.random.default_rng(1)
    y = np.concatenate([rng.uniform(-448, 448, 4000), rng.uniform(-2.0 ** -5, 2.0 ** -5, 4000),
                        (values[1:] + values[:-1]) / 2])                     # ties
    want = torch.from_numpy(y.astype(np.float32)).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(e4m3_round(y.astype(np.float32)), want)
    # off by at most half a step of four significant bits, or of the subnormal step
    assert np.all(np.abs(e4m3_round(y) - y) <= np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10))


def test_scale_exponent_is_the_smallest_that_fits():
    for amax in [448.0, 448.5, 1.0, 1.75, 1.7500001, 3.5, 3.501, 1e-3, 5e18, 2.0 ** -40]:
        e = scale_exponent(amax)
        assert amax <= 448 * 2.0 ** e and amax > 448 * 2.0 ** (e - 1)
    assert scale_exponent(0.0) == -64 and scale_exponent(1e-30) == -64 and scale_exponent(1e38) == 63


def test_growing_a_page_token_by_token():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((16, 2, 64)) * 2.0 ** np.arange(16)[:, None, None] / 64
    one, many = Kv8Store(1, 16, 2, 64), Kv8Store(1, 16, 2, 64)
    many.write([(0, t) for t in range(16)], x, x)
    for t in range(16):
        one.write([(0, t)], x[t:t + 1], x[t:t + 1])
    assert np.array_equal(one.exp, many.exp)
    step = 2.0 ** (many.exp[0, 0].astype(float) - 10)[None, :, None]            # half a subnormal step of the final scale
    held = many.k[0]
    assert np.all(np.abs(held - x) <= np.maximum(2.0 ** -4 * np.abs(x), step))
    # token by token: once more rounded where the code has become subnormal, never elsewhere
    normal = np.abs(held) >= 2.0 ** -5 * 2.0 ** many.exp[0, 0].astype(float)[None, :, None]
    assert np.array_equal(one.k[0][normal], held[normal])
    assert np.all(np.abs(one.k[0] - held) <= 2 * step)


def test_capped_attention_limits():
    """A huge cap changes nothing; a tiny one makes every visible score +-cap or 0, so the weights become nearly equal."""
    rng = np.random.default_rng(3)
    m = PoolModel(4, 16, None, 1, 1, 4)
    m.request_begin()
    slots = m.append_run(0, 0, 40)
    st = Kv8Store(4, 16, 1, 64)
    st.write(slots, rng.standard_normal((40, 1, 64)), rng.standard_normal((40, 1, 64)))
    q = rng.standard_normal((1, 2, 64)).astype(np.float32)
    plain = decode_attention_capped(m, st, [(0, 0)], q)
    far = decode_attention_capped(m, st, [(0, 0)], q, cap=1e7)
    assert np.abs(plain[0] - far[0]).max() < 1e-9 and np.abs(plain[1] - far[1]).max() < 1e-9
    tiny = decode_attention_capped(m, st, [(0, 0)], q, cap=1e-6)
    assert np.abs(tiny[0] - st.gather(slots)[1].mean(axis=0)).max() < 1e-5
    assert np.abs(tiny[1] - np.log(40)).max() < 2e-6


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("head_dim", [64, 128])
def test_plan_of_an_8bit_pool_on_random_scripts(seed, head_dim):
    geo = Geometry(1, 8, 2, head_dim, 16)
    stats = check_script(random_script(200 + seed, n_ops=70, geo=geo, multi_token=bool(seed % 2)), flags=binding.FLAG_KV_FP8)
    assert stats["wunits"] == 0 and stats["tunits"] > 0


@pytest.mark.parametrize("maker", [lambda: cfg3_batched(8, 1), lambda: cfg4_long_prefix(2, 3000, 16)])
def test_plan_of_an_8bit_pool_cuts_evenly(maker):
    stats = check_script(maker(), flags=binding.FLAG_KV_FP8)
    assert stats["tunits"] > 0


def test_plan_of_an_8bit_pool_respects_the_partial_rows():
    """Few partial rows: the pieces get longer until they fit, whole runs at the least."""
    script = cfg4_long_prefix(1, 3000, 16)
    script = dataclasses.replace(script, geometry=dataclasses.replace(script.geometry, head_dim=64))
    rows = 17 * script.geometry.n_q_heads
    for factor in (1, 2, 3, 8):
        check_script(script, flags=binding.FLAG_KV_FP8, max_partial_rows=rows * factor)


def _config(**kw):
    cfg = binding.Config()
    base = dict(n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, n_pages=10, max_requests=1,
                max_threads_per_request=2, max_segments_per_thread=4)
    for k, v in {**base, **kw}.items():
        setattr(cfg, k, v)
    return cfg


@pytest.mark.parametrize("head_dim", [64, 128])
def test_bytes_of_an_8bit_pool(head_dim):
    out = ctypes.c_size_t()
    lib = binding.lib()
    assert lib.pasta_kv_bytes(ctypes.byref(_config(head_dim=head_dim, flags=binding.FLAG_KV_FP8)), ctypes.byref(out)) == 0
    assert out.value == 2 * (10 * 2 * 32 * head_dim + 1024)                     # 40 bytes of scales, rounded up to 1024
    assert lib.pasta_kv_bytes(ctypes.byref(_config(head_dim=head_dim)), ctypes.byref(out)) == 0
    assert out.value == 2 * 10 * 2 * 64 * head_dim


def test_compute_calls_are_refused_on_a_host_only_pool():
    pool = binding.Pool(1, 4, 2, 64, 4, 1, 2, 3, flags=binding.FLAG_HOST_ONLY | binding.FLAG_KV_FP8)
    lib = binding.lib()
    assert lib.pasta_set_softcap(pool._h, ctypes.c_float(30.0)) == binding.BAD_STATE
    assert lib.pasta_set_softcap(None, ctypes.c_float(30.0)) == binding.INVALID_ARG
    assert lib.pasta_kv_read_layers(pool._h, 0, 1, 0, 0, 0, 1, None, None, None) == binding.BAD_STATE
    assert lib.pasta_kv_read_layers(None, 0, 1, 0, 0, 0, 1, None, None, None) == binding.INVALID_ARG
    req = pool.request_begin()
    pool.kv_append_run(req, 0, 20)                                              # bookkeeping is what it always was
    assert pool.dump()["requests"][0]["streams"][0]["len"] == 20
    pool.close()


def test_rotation_keeps_lengths():
    rng = np.random.default_rng(4)
    k = rng.standard_normal((5, 2, 64)).astype(np.float32)
    r = rotate(k, [0, 1, 7, 1000, 40000], 10000.0)
    assert np.array_equal(r[0], k[0])
    assert np.abs(np.linalg.norm(r, axis=-1) - np.linalg.norm(k, axis=-1)).max() < 1e-5
