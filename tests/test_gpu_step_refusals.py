"""A whole step that is refused for its arguments reserves nothing and launches nothing."""
import pytest

from test_gpu_kv8 import _randn, lib  # noqa: F401  (fixture + helper)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("flags", [0, 8], ids=["bf16", "8bit"])
def test_a_refused_step_leaves_the_pool_as_it_was(lib, flags):
    import torch
    pool = lib.Pool(1, 8, 2, 128, 8, 1, 2, 6, flags=flags)
    L = lib.lib()
    pool.request_begin()
    pool.kv_append_run(0, 0, 16, _randn((1, 16, 2, 128), 1).cuda(), _randn((1, 16, 2, 128), 2).cuda())
    pool.thread_spawn(0)
    flat = _randn((4096,), 3).cuda()
    kv, odd_kv = flat[:512].view(1, 2, 2, 128), flat[1:513].view(1, 2, 2, 128)
    q, odd_q = flat[:2048].view(1, 2, 8, 128), flat[1:2049].view(1, 2, 8, 128)
    room = torch.zeros(2056, device="cuda")
    out, odd_out = room[:2048], room[1:2049]
    nan = float("nan")
    calls = [(None, kv, q, out, 0.0), (kv, None, q, out, 0.0), (kv, kv, None, out, 0.0), (kv, kv, q, None, 0.0),
             (kv, kv, q, out, nan), (kv, kv, q, out, -1.0)]
    if flags:
        calls += [(odd_kv, kv, q, out, 0.0), (kv, odd_kv, q, out, 0.0), (kv, kv, odd_q, out, 0.0), (kv, kv, q, odd_out, 0.0)]
    before = pool.dump()
    held = pool.kv_read(0, 0, 0, 0, 16)
    launches = pool.launch_count()
    r, t = lib._i32([0, 0]), lib._i32([0, 1])
    ptr = lambda x: lib._dev(x) if x is not None else None

    def step(k, v, qq, o, scale):
        return L.pasta_step_device(pool._h, 2, lib._ptr(r), lib._ptr(t), None, ptr(k), ptr(v), ptr(qq), ptr(o), None, lib.C.c_float(scale), None)

    for i, call in enumerate(calls):
        assert step(*call) == lib.INVALID_ARG, i
        assert pool.dump() == before and pool.launch_count() == launches, i
    host = [x.cpu().pin_memory() for x in (kv, q)]
    oh = torch.empty(2048).pin_memory()
    staging = torch.empty(pool.step_host_bytes(2), dtype=torch.uint8, device="cuda")
    for scale in (nan, -1.0):
        with pytest.raises(lib.PastaError) as e:
            pool.step_host([0, 0], [0, 1], None, host[0], host[0], host[1], oh, staging, scale=scale)
        assert e.value.code == lib.INVALID_ARG and pool.dump() == before and pool.launch_count() == launches
    assert step(kv, kv, q, out, 0.0) == lib.OK                          # the same step with its arguments in order
    torch.cuda.synchronize()
    dump = pool.dump()["requests"][0]["streams"]
    assert dump[0]["len"] == 17 and dump[1]["len"] == 1
    assert all(torch.equal(a, b) for a, b in zip(held, pool.kv_read(0, 0, 0, 0, 16)))
    assert bool(torch.isfinite(out).all()) and pool.status() == 0


def test_a_step_without_new_tokens_needs_none(lib):
    import torch
    for flags in (0, 8):
        pool = lib.Pool(1, 8, 2, 128, 8, 1, 2, 6, flags=flags)
        pool.request_begin()
        pool.kv_append_run(0, 0, 16, _randn((1, 16, 2, 128), 1).cuda(), _randn((1, 16, 2, 128), 2).cuda())
        q, out = _randn((1, 1, 8, 128), 3).cuda(), torch.zeros((1, 1, 8, 128), device="cuda")
        nothing = torch.empty((1, 0, 2, 128), dtype=torch.bfloat16, device="cuda")
        pool.step_device([0], [0], [0], nothing, nothing, q, out)
        assert bool((out != 0).any()) and pool.status() == 0
