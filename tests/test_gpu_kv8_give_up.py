"""8-bit pools: a role of an attention kernel that never starts makes the kernel give up cleanly.

One role is held back by the test hook (a flag that nothing sets), those that wait for it run into a short limit, the CTA waits
for its copies and MMAs in flight and returns; the status says TIMEOUT; the same step then gives the bits it gave before."""
import time

import pytest

from test_gpu_kv8 import _pool, _randn, lib  # noqa: F401  (fixture + helpers)

pytestmark = pytest.mark.gpu


def _give_up(lib, pool, q, mask):
    import torch
    ref, out = (torch.zeros(q.shape, device="cuda") for _ in range(2))
    pool.decode_attn(q, ref)
    torch.cuda.synchronize()
    assert pool.status() == lib.OK
    pool.debug_set_wait_limit(400_000)                 # about 0.2 ms
    pool.debug_hold_roles(mask)
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


@pytest.mark.parametrize("threads", [2, 9, 17])
@pytest.mark.parametrize("mask", [1, 2, 4, 8, 16], ids=["producer", "mma_issue", "query_builder", "softmax_0", "softmax_1"])
def test_tensor_core_kernel(lib, mask, threads):
    """Every row class, several units per CTA, two layers."""
    pool, q = _filled(lib, [120 + 37 * i for i in range(40)], threads, 32, 8, 128, 2)
    words = pool.plan_words()                          # t-units, and units handed out at run time
    assert words[4] > 2 * 148 and (words[23] > 0) == (threads > 2)
    _give_up(lib, pool, q, mask)


@pytest.mark.parametrize("lengths", [[700, 900], [500 + 31 * i for i in range(60)]], ids=["six_warps", "two_warps"])
@pytest.mark.parametrize("threads,mask", [(1, 1), (8, 1), (8, 2)], ids=["copies", "copies_shared_ring", "consumers"])
def test_matrix_kernel_of_head_dim_64(lib, lengths, threads, mask):
    pool, q = _filled(lib, lengths, threads, 16, 4, 64, 2)
    _give_up(lib, pool, q, mask)


def test_warp_shuffle_kernel_is_not_held(lib):
    """The hook belongs to the matrix kernels: the warp-shuffle kernel has one role and nobody to wait for."""
    import torch
    pool = _pool(lib, 60, flags=lib.FLAG_NO_TENSOR_PATH)
    pool.request_begin()
    pool.kv_append_run(0, 0, 500, _randn((1, 500, 2, 128), 1).cuda(), _randn((1, 500, 2, 128), 2).cuda())
    pool.step_begin([0], [0], [0])
    out = torch.zeros((1, 1, 8, 128), device="cuda")
    pool.debug_hold_roles(31)
    pool.decode_attn(_randn((1, 1, 8, 128), 3).cuda(), out)
    assert pool.status() == lib.OK and bool((out != 0).any())
