"""4-bit pools: rows whose scores are finite but far from 0, where neighbouring fp32 numbers are many powers of e apart.

Keys are c_j times a row of ones, with c_0 the largest by a fifth at least and at least 1 (the smallest by that much in the other sign), so from
scores of 10^4 on one token has all the weight: a weight of 1 is exact, the others are zero, and out is that token's V as held; fp32
sums and the merge add 2^-16 of max |v| at most.  lse is its score: head_dim exact products summed in fp32, one product by the scale and
two conversions between bases, head_dim + 8 roundings of 2^-23.  Rows with ordinary scores beside them are held to their own bound:
the scores' error ds <= (head_dim + 8) 2^-23 sum |q k| scale + 2^-21, a weight rounded to bf16 (2^-8 of it, or half that at best)
and the sum rounded with it, so an element is off by (2^-8 + 2 ds + 2^-16) (sum w |v| + |out|)."""
import numpy as np
import pytest

from oracle import PoolModel
from oracle.kv4 import Kv4Store
from test_gpu_kv4 import _pool, _randn, lib  # noqa: F401  (fixture + helpers)

pytestmark = pytest.mark.gpu


def exact(q, k, v, scale, cap=0.0):
    """(out, lse, sum w |v|, bound of the scores) of rows q [n, d] over k, v [tokens, d], fp64."""
    s = (q @ k.T) * scale
    if cap:
        s = cap * np.tanh(s / cap)
    m = s.max(1, keepdims=True)
    w = np.exp(s - m)
    lse = m[:, 0] + np.log(w.sum(1))
    w /= w.sum(1, keepdims=True)
    ds = (q.shape[1] + 8) * 2.0 ** -23 * (np.abs(q) @ np.abs(k).T).max(1) * scale + 2.0 ** -21
    return w @ v, lse, w @ np.abs(v), ds


def one_request(lib, d, threads, k, v, flags=0, cap=0.0, **kw):
    """A response with this prompt and forks at its end that add nothing, and what the pool holds of it."""
    n = k.shape[1]
    pool = _pool(lib, n // 16 + 2, threads=threads, hq=4, hkv=1, d=d, flags=flags, max_step_queries=threads, **kw)
    model, store = PoolModel(n // 16 + 2, 16, None, 1, threads, 2 * threads + 2), Kv4Store(n // 16 + 2, 16, 1, d)
    pool.request_begin(); model.request_begin()
    pool.kv_append_run(0, 0, n, k.cuda(), v.cuda())
    store.write(model.append_run(0, 0, n), k[0], v[0])
    for _ in range(threads - 1):
        pool.thread_spawn(0)
    pool.step_begin([0] * threads, list(range(threads)), [0] * threads)
    pool.set_softcap(cap)
    held_k, held_v = store.gather(model.visible_slots(0, 0))
    return pool, held_k[:, 0], held_v[:, 0]


@pytest.mark.parametrize("size", [1e6, 3e8, 1e10, -1e10, 1e20, -1e20, 1e36, -1e36])
@pytest.mark.parametrize("threads,n", [(1, 1), (2, 90), (3, 700), (17, 300), (17, 5000)])
@pytest.mark.parametrize("d,flags", [(128, 0), (64, 0), (128, 2), (64, 2)])
def test_one_token_decides(lib, d, flags, threads, n, size):
    import torch
    c = torch.linspace(0.3, 0.75, n) if size > 0 else torch.linspace(1.5, 2.0, n)
    at = (n * 5) // 7
    c[at] = 1.0
    k = (c[None, :, None, None] * torch.ones((1, n, 1, d))).to(torch.bfloat16)
    v = _randn((1, n, 1, d), 2)
    pool, hk, hv = one_request(lib, d, threads, k, v, flags)
    q = torch.ones((threads, 4, d)) * abs(size) / d ** 0.5 * (1 if size > 0 else -1)
    q *= 1 + torch.arange(4 * threads).reshape(threads, 4, 1) / (8 * threads)
    q[:, 1] = _randn((threads, d), 5).float()                         # a row of ordinary scores in every thread
    q = q.to(torch.bfloat16)
    out = torch.full((1, threads, 4, d), 7.0, device="cuda"); lse = torch.full((1, threads, 4), 7.0, device="cuda")
    pool.decode_attn(q[None].cuda(), out, lse)
    rows = q.double().numpy().reshape(-1, d)
    want, want_lse, mean_abs, ds = exact(rows, hk, hv, d ** -0.5)
    got, got_lse = out[0].double().cpu().numpy().reshape(-1, d), lse[0].double().cpu().numpy().reshape(-1)
    far = np.arange(4 * threads) % 4 != 1
    top = np.abs(hv).max()
    assert np.abs(want[far] - hv[at]).max() <= 1e-9                  # as the first paragraph has it
    assert np.abs(got[far] - want[far]).max() <= 2.0 ** -16 * top, np.abs(got[far] - want[far]).max()
    assert (np.abs(got_lse[far] / want_lse[far] - 1)).max() <= (d + 8) * 2.0 ** -23
    tol = (2.0 ** -8 + 2 * ds[:, None] + 2.0 ** -16) * (mean_abs + np.abs(want))
    assert (np.abs(got - want)[~far] <= tol[~far]).all(), np.abs(got - want)[~far].max()
    assert (np.abs(got_lse - want_lse)[~far] <= 2.0 ** -8 + ds[~far]).all()
    assert pool.status() == 0
    pool.close()


@pytest.mark.parametrize("size", [1e10, -1e10, 1e30])
@pytest.mark.parametrize("d,flags", [(128, 0), (64, 0), (128, 2)])
def test_tokens_with_the_same_key_share_the_weight(lib, d, flags, size):
    """Equal keys far apart in the run have equal scores, however large: the row is the mean of their values."""
    import torch
    n, twins = 3000, [3, 130, 131, 1500, 2999]
    c = torch.linspace(0.3, 0.75, n) if size > 0 else torch.linspace(1.5, 2.0, n)
    c[twins] = 1.0
    k = (c[None, :, None, None] * torch.ones((1, n, 1, d))).to(torch.bfloat16)
    pool, hk, hv = one_request(lib, d, 5, k, _randn((1, n, 1, d), 2), flags)
    q = (torch.ones((1, 5, 4, d)) * size / d ** 0.5 * (1 + torch.arange(20).reshape(1, 5, 4, 1) / 32)).to(torch.bfloat16)
    out = torch.full((1, 5, 4, d), 7.0, device="cuda"); lse = torch.full((1, 5, 4), 7.0, device="cuda")
    pool.decode_attn(q.cuda(), out, lse)
    want = hv[twins].mean(0)                                         # five weights of 1 (exact); fp32 sums
    assert np.abs(out[0].double().cpu().numpy() - want).max() <= 2.0 ** -16 * np.abs(hv).max()
    assert pool.status() == 0
    pool.close()

