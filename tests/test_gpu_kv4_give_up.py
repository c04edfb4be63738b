"""4-bit pools: matrix products that never start make the attention kernel give up cleanly.

The test hook holds them back, every warp that waits for them runs into a short limit, the CTA waits for what is in flight, takes
its last number from the counter of units handed out at run time, and returns; the status says TIMEOUT; the same step then gives
the bits it gave before, so every unit was handed out again."""
import time

import pytest

from test_gpu_kv4 import _pool, _randn, lib  # noqa: F401  (fixture + helpers)

pytestmark = pytest.mark.gpu


def _filled(lib, lengths, threads, hq, hkv, d, layers):
    pages = sum(n // 16 + threads + 1 for n in lengths)
    R = len(lengths)
    pool = _pool(lib, pages, requests=R, threads=threads, hq=hq, hkv=hkv, d=d, layers=layers, max_step_queries=R * threads)
    for r, n in enumerate(lengths):
        pool.request_begin()
        pool.kv_append_run(r, 0, n, _randn((layers, n, hkv, d), r).cuda(), _randn((layers, n, hkv, d), 100 + r).cuda())
        for _ in range(threads - 1):
            pool.thread_spawn(r)
    n_q = R * threads
    pool.step_begin([r for r in range(R) for _ in range(threads)], list(range(threads)) * R, ([0] + [1] * (threads - 1)) * R)
    if threads > 1:
        pool.kv_append(_randn((layers, n_q - R, hkv, d), 7).cuda(), _randn((layers, n_q - R, hkv, d), 8).cuda())
    return pool, _randn((layers, n_q, hq, d), 9).cuda()


# (threads x group rows of every class; runs handed out at run time, cut in advance, and both)
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("threads", [2, 9, 17, 30])
@pytest.mark.parametrize("lengths", [[300], [120 + 37 * i for i in range(40)], [40000], [30000, 200, 300, 25000]],
                         ids=["one", "many", "long", "mixed"])
def test_held_products(lib, lengths, threads, d):
    import torch
    pool, q = _filled(lib, lengths, threads, 8, 2, d, 2)
    ref, out = (torch.zeros(q.shape, device="cuda") for _ in range(2))
    words = pool.plan_words()                          # units assigned in advance, units handed out at run time
    assert words[4] + words[23] > 0
    pool.decode_attn(q, ref)
    torch.cuda.synchronize()
    assert pool.status() == lib.OK
    for _ in range(2):
        pool.debug_set_wait_limit(400_000)             # about 0.2 ms
        pool.debug_hold_roles(2)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        pool.decode_attn(q, out)
        torch.cuda.synchronize()
        assert time.perf_counter() - t0 < 2.0
        assert pool.status() == lib.TIMEOUT and pool.status() == lib.OK
        pool.debug_hold_roles(0)
        pool.debug_set_wait_limit(0)
        pool.decode_attn(q, out)
        assert torch.equal(out, ref) and pool.status() == lib.OK
    pool.close()


@pytest.mark.parametrize("d", [128, 64])
def test_copies_and_the_warp_shuffle_kernel_have_nothing_to_hold(lib, d):
    import torch
    for flags, mask in ((0, 1), (lib.FLAG_NO_TENSOR_PATH, 31)):
        pool = _pool(lib, 60, flags=flags, d=d)
        pool.request_begin()
        pool.kv_append_run(0, 0, 500, _randn((1, 500, 2, d), 1).cuda(), _randn((1, 500, 2, d), 2).cuda())
        pool.step_begin([0], [0], [0])
        out = torch.zeros((1, 1, 8, d), device="cuda")
        pool.debug_hold_roles(mask)
        pool.decode_attn(_randn((1, 1, 8, d), 3).cuda(), out)
        assert pool.status() == lib.OK and bool((out != 0).any())
        pool.close()


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("threads", [2, 17])
@pytest.mark.parametrize("lengths", [[300], [120 + 37 * i for i in range(40)], [30000, 200, 300, 25000]], ids=["one", "many", "mixed"])
def test_giving_up_while_products_are_under_way(lib, lengths, threads, d):
    """A limit so short that a wait for a product that has just begun may give up: the CTA waits for it before it frees the tensor
    memory, and the launches behind it find everything as it was."""
    import torch
    pool, q = _filled(lib, lengths, threads, 8, 2, d, 2)
    ref, out = (torch.zeros(q.shape, device="cuda") for _ in range(2))
    pool.decode_attn(q, ref)
    assert pool.status() == lib.OK
    for _ in range(5):
        pool.debug_set_wait_limit(1)
        for _ in range(3):
            pool.decode_attn(q, out)
        status = pool.status()
        assert status == lib.TIMEOUT or (status == lib.OK and torch.equal(out, ref))
        pool.debug_set_wait_limit(0)
        pool.decode_attn(q, out)
        assert torch.equal(out, ref) and pool.status() == lib.OK
    pool.close()
