"""4-bit pools of many layers whose attention is called for one layer, some layers and all of them.

One layer at a time gives the bits of a pool of one layer.  Other launches cut runs elsewhere, and are held to the definition:
an element is off by (2^-8 + 2 ds + 2^-16) (sum w |v| + |out|), ds <= (head_dim + 8) 2^-23 sum |q k| scale + 2^-21."""
import numpy as np
import pytest

from test_gpu_kv4 import _randn, lib  # noqa: F401  (fixture + helpers)
from test_gpu_kv4_large_scores import exact

pytestmark = pytest.mark.gpu


def filled(lib, lengths, forks, k, v, layers, hq, hkv, d, cap=0.0, **kw):
    """A step of prompts whose forks see all of theirs, over the given layers' K and V."""
    T, R = forks + 1, len(lengths)
    pool = lib.Pool(layers, hq, hkv, d, sum(n // 16 + 1 for n in lengths) + R * T, R, T, 2 * T + 2, flags=lib.FLAG_KV_INT4,
                    max_step_queries=R * T, **kw)
    at = 0
    for r, n in enumerate(lengths):
        pool.request_begin()
        pool.kv_append_run(r, 0, n, k[:, at:at + n].contiguous().cuda(), v[:, at:at + n].contiguous().cuda())
        at += n
        for _ in range(forks):
            pool.thread_spawn(r)
    pool.set_softcap(cap)
    pool.step_begin([r for r in range(R) for _ in range(T)], list(range(T)) * R, [0] * (R * T))
    return pool


@pytest.mark.parametrize("lengths,forks,hq,hkv,d,cap", [([256 + 119 * i for i in range(16)], 4, 32, 8, 128, 0.0),
                                                        ([16000, 9000], 16, 8, 2, 128, 0.0), ([30000] + [40 + 90 * i for i in range(12)], 1, 4, 2, 128, 20.0),
                                                        ([150 + 90 * i for i in range(24)], 3, 16, 8, 64, 0.0), ([12000], 21, 8, 2, 64, 0.0)])
def test_any_number_of_layers(lib, lengths, forks, hq, hkv, d, cap):
    import torch
    L, T, n = 8, forks + 1, sum(lengths)
    k, v = _randn((L, n, hkv, d), 1), _randn((L, n, hkv, d), 2)
    q = _randn((L, len(lengths) * T, hq, d), 3).cuda()
    pool = filled(lib, lengths, forks, k, v, L, hq, hkv, d, cap)
    words = pool.plan_words()
    single, lse1, out, lse = (torch.full(q.shape[:3] + x, 7.0, device="cuda") for x in ((d,), (), (d,), ()))
    for l in range(L):
        pool.decode_attn(q[l:l + 1], single[l:l + 1], lse1[l:l + 1], layer_begin=l, layer_count=1)
    for l in (0, L - 1):
        alone = filled(lib, lengths, forks, k[l:l + 1], v[l:l + 1], 1, hq, hkv, d, cap)
        want, want_lse = torch.empty_like(out[:1]), torch.empty_like(lse[:1])
        alone.decode_attn(q[l:l + 1], want, want_lse)
        assert torch.equal(single[l:l + 1], want) and torch.equal(lse1[l:l + 1], want_lse)
        if words[7] <= 16384:
            one = torch.zeros_like(out[0])
            pool.decode_attn_noalloc(q[l], one, layer=l)
            assert torch.equal(one, want[0])
        alone.close()
    # by twos and threes, all at once, and captured one by one
    results = [single.clone()]
    for step in (2, 3, L):
        out.fill_(7.0)
        for l in range(0, L, step):
            c = min(step, L - l)
            pool.decode_attn(q[l:l + c], out[l:l + c], lse[l:l + c], layer_begin=l, layer_count=c)
        results.append(out.clone())
    out.fill_(7.0)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        for l in range(L):
            pool.decode_attn(q[l:l + 1], out[l:l + 1], layer_begin=l, layer_count=1)
    graph.replay(); graph.replay()
    assert torch.equal(out, single) and pool.status() == 0
    group, at = hq // hkv, 0
    starts = np.cumsum([0] + list(lengths))
    for l in (0, 5):
        for r in range(0, len(lengths), max(1, len(lengths) // 4)):
            hk, hv = (x.double().cpu().numpy() for x in pool.kv_read(l, r, 0, 0, lengths[r]))
            for h in (0, hq - 1):
                rows = q[l, r * T:(r + 1) * T, h].double().cpu().numpy()
                want, want_lse, mean_abs, ds = exact(rows, hk[:, h // group], hv[:, h // group], d ** -0.5, cap)
                tol = (2.0 ** -8 + 2 * ds[:, None] + 2.0 ** -16 + (2.0 ** -20 * cap)) * (mean_abs + np.abs(want))
                for got in results:
                    assert (np.abs(got[l, r * T:(r + 1) * T, h].double().cpu().numpy() - want) <= tol).all()
                assert (np.abs(lse1[l, r * T:(r + 1) * T, h].double().cpu().numpy() - want_lse) <= 2.0 ** -8 + ds + 2.0 ** -20 * cap).all()
    pool.close()
