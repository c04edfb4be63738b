"""Bases of the rotary embedding that are refused, by every call that takes one (an infinite base has no first frequency: every pair's angle
would be 0 but that of pair 0, which infinity to the power 0 leaves undefined)."""
import pytest

from paper_2502_11517_b200 import binding, build

BAD = [float("inf"), float("nan"), 1.0, 0.0, -10.0]
KINDS = [0, binding.FLAG_KV_FP8, binding.FLAG_KV_INT4]


@pytest.fixture(scope="module", autouse=True)
def _built():
    build()


@pytest.mark.parametrize("theta", BAD)
@pytest.mark.parametrize("flags", KINDS)
def test_runs_without_layers(flags, theta):
    pool = binding.Pool(1, 4, 2, 64, 4, 1, 1, 4, flags=flags | binding.FLAG_HOST_ONLY)
    pool.request_begin()
    with pytest.raises(binding.PastaError) as e:
        pool.kv_append_run_rope(0, 0, 5, None, None, theta, layer_count=0, stream=0)
    assert e.value.code == binding.INVALID_ARG and pool.dump()["requests"][0]["streams"][0]["len"] == 0
    pool.kv_append_run_rope(0, 0, 5, None, None, 3e38, layer_count=0, stream=0)
    assert pool.dump()["requests"][0]["streams"][0]["len"] == 5
    pool.close()


@pytest.mark.gpu
@pytest.mark.parametrize("form", [{}, {"layout": "interleaved", "scaling": "base", "factor": 2.0}])
@pytest.mark.parametrize("flags", KINDS)
def test_every_call(flags, form):
    import torch
    pool = binding.Pool(1, 4, 2, 64, 8, 1, 1, 4, flags=flags)
    pool.set_rope(**form)
    pool.request_begin()
    k = torch.ones((1, 5, 2, 64), dtype=torch.bfloat16, device="cuda")
    q = torch.ones((1, 1, 4, 64), dtype=torch.bfloat16, device="cuda")
    pool.kv_append_run(0, 0, 5, k, k)
    pool.step_begin([0], [0], [1])
    launches = pool.launch_count()
    one = k[:, :1].contiguous()
    for theta in BAD:
        for call in (lambda: pool.kv_append_rope(one, one, theta), lambda: pool.rope_queries(q, theta),
                     lambda: pool.rope_queries(q, theta, out=torch.empty_like(q)), lambda: pool.kv_append_run_rope(0, 0, 5, k, k, theta),
                     lambda: pool.rope_frequencies(theta)):
            with pytest.raises(binding.PastaError) as e:
                call()
            assert e.value.code == binding.INVALID_ARG
    assert pool.launch_count() == launches and pool.dump()["requests"][0]["streams"][0]["len"] == 6
    pool.kv_append_rope(one, one, 3e38)
    pool.rope_queries(q, 3e38)
    _, v = pool.kv_read(0, 0, 0, 0, 6)
    assert bool(torch.isfinite(q).all()) and bool((v > 0.9).all())
    assert pool.status() == 0
    pool.close()
