"""8-bit pools: rows in which one token takes most of the weight and thousands of small weights make up the rest.

Tolerance, element by element.  With weights w (sum 1) and values v held in pages of scale 2^ev, a weight is off by at most
2^-8 of itself at head_dim 128 (three e5m2 terms) and 2^-11 at head_dim 64 (fp16), or, where that is more, by 2^-24 of the
row's largest contribution L = max w 2^ev, taken relative to its own page's scale: 2^-24 L 2^-ev.  The sum of the weights is
not rounded.  A score carries the fp32 sums' rounding and the split of q (see test_gpu_kv8), ds in all, which moves every
weight by at most 2 ds of itself against the sum.  The sums over n values are made in fp32, n / 16 additions of pages and
joins, each off by at most 2^-23 of what has been added up, sum w |v|:
|out - exact| <= sum over tokens of (max(relative w, 2^-24 L 2^-ev) + (2 ds + 2^-23 (n / 16 + 64)) w) |v|."""
import numpy as np
import pytest

from oracle import PoolModel
from oracle.kv8 import Kv8Store
from test_gpu_kv8 import _pool, lib, score_bound  # noqa: F401  (fixture + helpers)

pytestmark = pytest.mark.gpu


def _case(n, share, sink_at, d, rows, spike, seed=3):
    """One stream of n tokens seen by `rows` query rows; K, V, q on the host.  Every row has the same component along one
    direction, in which the sink's key points; the other scores are about N(0, 1).  V: a mean per channel, 0.05 at the sink."""
    import torch
    rng = np.random.default_rng(seed)
    u = rng.standard_normal(d); u /= np.linalg.norm(u)
    along = 8.0
    q = rng.standard_normal((rows, d))
    q += (along - q @ u)[:, None] * u
    k = rng.standard_normal((n, d))
    want = np.log(n) + 0.5 * (1 + along ** 2 / d) + np.log(share / (1 - share))      # the sink's score for that share
    k[sink_at] = u * want * np.sqrt(d) / along
    v = 0.3 * np.sign(rng.standard_normal(d)) * (1 + 0.1 * rng.standard_normal((n, d)))
    v[sink_at] = 0.05 * rng.standard_normal(d)
    v[sink_at, 5] = spike                       # a page whose scale is far above the others'
    bf = lambda x: torch.from_numpy(x).to(torch.bfloat16)
    return bf(q), bf(k), bf(v)


# head_dim, flags (2: warp-shuffle kernel), threads, tokens, share of the sink, where it is, its V's largest element, cap
CASES = [(128, 0, 1, 8192, 0.6, 0, 0.05, 0.0), (128, 0, 1, 8192, 0.9, 0, 0.05, 0.0), (128, 0, 1, 32768, 0.9, 0, 0.05, 0.0),
         (128, 0, 9, 8192, 0.9, 0, 0.05, 0.0), (128, 0, 9, 32768, 0.6, 0, 0.05, 0.0), (128, 0, 17, 8192, 0.9, 0, 0.05, 0.0),
         (128, 0, 17, 32768, 0.6, 0, 0.05, 0.0), (128, 0, 17, 32768, 0.9, 0, 0.05, 0.0), (128, 0, 1, 8191, 0.9, 5000, 0.05, 0.0),
         (128, 0, 17, 8191, 0.9, 8190, 0.05, 0.0), (128, 0, 1, 4096, 0.5, 0, 20.0, 0.0), (128, 0, 9, 4096, 0.5, 2000, 20.0, 0.0),
         (128, 0, 17, 4096, 0.5, 0, 20.0, 0.0), (128, 0, 1, 8192, 0.9, 0, 0.05, 50.0), (128, 0, 17, 8192, 0.9, 0, 0.05, 50.0),
         (64, 0, 1, 32768, 0.9, 0, 0.05, 0.0), (64, 0, 9, 8192, 0.6, 0, 0.05, 0.0), (64, 0, 17, 32768, 0.9, 8190, 0.05, 0.0),
         (64, 0, 17, 4096, 0.5, 0, 20.0, 0.0), (128, 2, 1, 8192, 0.9, 0, 0.05, 0.0), (64, 2, 2, 8192, 0.9, 0, 20.0, 50.0)]


@pytest.mark.parametrize("d,flags,threads,n,share,sink_at,spike,cap", CASES)
def test_one_token_with_most_of_the_weight(lib, d, flags, threads, n, share, sink_at, spike, cap):
    """37 requests of 4 kv heads, as many runs as an sm_100a GPU has SMs: on the tensor cores a CTA then walks a run as a whole.
    All requests and kv heads hold the same tokens; their queries differ from kv head to kv head."""
    import torch
    R, hkv, group = 37, 4, 4
    hq = hkv * group
    q, k, v = _case(n, share, sink_at, d, threads * hq, spike)
    q = q.reshape(threads, hq, d)
    per_request = -(-n // 16) + threads
    pool = _pool(lib, R * per_request, requests=R, threads=threads, hq=hq, hkv=hkv, d=d, flags=flags, max_step_queries=R * threads)
    model, store = PoolModel(per_request, 16, None, 1, threads, 2 * threads + 2), Kv8Store(per_request, 16, 1, d)
    model.request_begin()
    store.write(model.append_run(0, 0, n), k.reshape(n, 1, d), v.reshape(n, 1, d))
    wide = lambda x: x.reshape(1, -1, 1, d).repeat(1, 1, hkv, 1).cuda()
    kd, vd = wide(k), wide(v)
    for r in range(R):
        assert pool.request_begin() == r
        pool.kv_append_run(r, 0, n, kd, vd)
        for _ in range(threads - 1):            # forks without tokens yet: the step appends one to each
            pool.thread_spawn(r)
    for _ in range(threads - 1):
        model.thread_spawn(0)
    pool.set_softcap(cap)
    new = [0] + [1] * (threads - 1)
    pool.step_begin(np.repeat(np.arange(R), threads).tolist(), list(range(threads)) * R, new * R)
    slots = [s for s in model.reserve(list(zip([0] * threads, range(threads), new))) if s is not None]
    if threads > 1:
        kn = 0.1 * torch.ones((threads - 1, 1, d), dtype=torch.bfloat16)
        store.write(slots, kn, kn)
        pool.kv_append(wide(kn).repeat(1, R, 1, 1), wide(kn).repeat(1, R, 1, 1))
    out = torch.full((1, R * threads, hq, d), float("nan"), device="cuda"); lse = torch.empty((1, R * threads, hq), device="cuda")
    pool.decode_attn(q.repeat(R, 1, 1)[None].cuda(), out, lse)
    got, got_lse = out.reshape(R, threads, hq, d).double().cpu().numpy(), lse.reshape(R, threads, hq).double().cpu().numpy()
    qf = q.float().numpy().astype(np.float64)
    relative = 0.0 if flags else 2.0 ** -11 if d == 64 else 2.0 ** -8
    ds = score_bound(qf, store.k, 1 / np.sqrt(d), cap)
    for t in range(threads):
        visible = model.visible_slots(0, t)
        kk, vv = store.gather(visible)
        s = qf[t] @ kk[:, 0].T / np.sqrt(d)
        if cap:
            s = cap * np.tanh(s / cap)
        m = s.max(1, keepdims=True)
        w = np.exp(s - m)
        want_lse = m[:, 0] + np.log(w.sum(1))
        w /= w.sum(1, keepdims=True)
        assert cap or 0.35 < w.max(1).min() and w.max(1).max() < 0.95          # the case is what it is meant to be
        scales = 2.0 ** store.exp[1][np.array([p for p, _ in visible]), 0]
        floor = 0.0 if flags else 2.0 ** -24 * (w * scales).max(1, keepdims=True) / scales
        per_weight = np.maximum(relative * w, floor) + (2 * ds + 2.0 ** -23 * (len(visible) / 16 + 64)) * w
        want, tol = w @ vv[:, 0], per_weight @ np.abs(vv[:, 0])
        err = np.abs(got[:, t] - want)
        row_error = (np.linalg.norm(err, axis=2) / np.linalg.norm(want, axis=1)).max()
        assert np.all(err <= tol), (t, "error over tolerance", (err / tol).max(), "of the row", row_error)
        assert np.all(np.abs(got_lse[:, t] - want_lse) <= ds + 2.0 ** -20 * np.abs(want_lse)), t
    assert pool.status() == 0
    pool.close()
