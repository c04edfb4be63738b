"""4-bit pools: a page id outside the pool in the device's copy of the plan is reported, and its page is left out, on both attention kernels.

The plan lies in the workspace, which belongs to the caller; the test looks it up there and overwrites page ids before the launch.
Every kernel compares an id with the number of pages before it forms an address."""
import numpy as np
import pytest

from test_gpu_kv4 import _pool, _randn, lib  # noqa: F401  (fixture + helpers)

pytestmark = pytest.mark.gpu
OFF_PAGES = 16                                                        # header word (pasta_plan.h)


def plan_in(pool):
    """The step's plan as it stands in the workspace."""
    words = pool.plan_words()
    space = pool.workspace.view(dtype=__import__("torch").int32)
    host = space.cpu().numpy()
    at = [i for i in np.flatnonzero(host == words[0]) if np.array_equal(host[i:i + len(words)], words)]
    assert len(at) == 1
    return space[at[0]:at[0] + len(words)], words


@pytest.mark.parametrize("bad", [-1, -2, -2 ** 31, 2 ** 31 - 1, "the first behind the pool"])
@pytest.mark.parametrize("threads", [1, 12])
@pytest.mark.parametrize("d,flags", [(128, 0), (64, 0), (128, 2)])
def test_reported_and_left_out(lib, d, flags, threads, bad):
    import torch
    n, hq, hkv = 400, 8, 2
    n_pages = n // 16 + threads
    pool = _pool(lib, n_pages, threads=threads, hq=hq, hkv=hkv, d=d, flags=flags, max_step_queries=threads)
    pool.request_begin()
    k, v = _randn((1, n, hkv, d), 1), _randn((1, n, hkv, d), 2)
    pool.kv_append_run(0, 0, n, k.cuda(), v.cuda())
    for _ in range(threads - 1):
        pool.thread_spawn(0)
    pool.step_begin([0] * threads, list(range(threads)), [0] * threads)
    q = _randn((1, threads, hq, d), 3).cuda()
    ref, out = torch.empty((1, threads, hq, d), device="cuda"), torch.zeros((1, threads, hq, d), device="cuda")
    pool.decode_attn(q, ref)
    assert pool.status() == lib.OK
    plan, words = plan_in(pool)
    which = 10
    good = int(plan[words[OFF_PAGES] + which])
    assert 0 <= good < n_pages
    plan[words[OFF_PAGES] + which] = n_pages if isinstance(bad, str) else bad
    pool.decode_attn(q, out)
    assert pool.status() == lib.DEVICE_CHECK and pool.status() == lib.OK
    assert bool(torch.isfinite(out).all()) and not torch.equal(out, ref)
    if not flags:                                                     # left out: as if those 16 tokens were not there
        hk, hv = (x.double().cpu().numpy() for x in pool.kv_read(0, 0, 0, 0, n))
        keep = np.r_[0:16 * which, 16 * which + 16:n]
        rows = q[0].double().cpu().numpy()
        for h in range(hq):
            s = rows[:, h] @ hk[keep, h // 4].T / np.sqrt(d)
            w = np.exp(s - s.max(1, keepdims=True))
            w /= w.sum(1, keepdims=True)
            want = w @ hv[keep, h // 4]
            # a weight rounded to bf16 and the sum of the rounded ones; scores of this size are good to 2^-12
            tol = (2.0 ** -8 + 2.0 ** -11) * (w @ np.abs(hv[keep, h // 4]) + np.abs(want))
            assert (np.abs(out[0, :, h].double().cpu().numpy() - want) <= tol).all()
    plan[words[OFF_PAGES] + which] = good
    pool.decode_attn(q, out)
    assert torch.equal(out, ref) and pool.status() == lib.OK
    pool.close()
