"""GPU parity of the forms of rotary embedding, for queries and for keys on every kind of pool.

An element is the 64-bit rotation rounded to fp32 and then to bf16.  The library's 64-bit value and the oracle's differ by a few
times 2^-53 of the pair's size times the angle (whose product with the frequency is rounded, 2^-53 of it, and whose frequency is good to 2^-46):
for positions up to 2^21 less than 2^-23 of the pair.  So the result is off the oracle's by half a step of bf16 (8 significant bits:
steps of 2^-7 to 2^-8 of a number, half of one at most 2^-8 of it), 2^-24 of it for the first rounding, and 2^-22 of the pair's
size."""
import numpy as np
import pytest

from oracle.kv4 import Kv4Store, frequencies, rotate_form
from oracle.kv8 import Kv8Store
from test_gpu_kv4 import _randn, lib  # noqa: F401  (fixture + helper)
from test_rope_forms import FORMS

pytestmark = pytest.mark.gpu


def close(got, x, positions, theta, form):
    got = got.double().cpu().numpy()
    want = rotate_form(x, positions, theta, form)
    size = frequencies(x.shape[-1], theta, form)[1]
    pair = size * np.abs(x.float().numpy()).max(-1, keepdims=True) * 2 ** 0.5
    assert np.all(np.abs(got - want) <= (2.0 ** -8 + 2.0 ** -24) * np.abs(want) + 2.0 ** -22 * pair)
    R = form.get("rotary_dim") or x.shape[-1]
    assert np.array_equal(got[..., R:], x.float().numpy()[..., R:])


def _pool(lib, d, hq=8, hkv=2, layers=2, n_pages=80, requests=1, threads=6, flags=0, queries=64):
    return lib.Pool(layers, hq, hkv, d, n_pages, requests, threads, 2 * threads + 2, flags=flags, max_step_queries=queries)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("d,theta", [(128, 10000.0), (64, 500000.0)])
def test_queries(lib, form, d, theta):
    """In place and into another array; far positions; several threads and several tokens of one."""
    import torch
    pool = _pool(lib, d)
    pool.set_rope(**form)
    pool.request_begin()
    ahead = [0, 0, 5, 70_000, 130_000, 1_700_000]
    for a in ahead[1:]:
        pool.thread_spawn_predicted(0, a)
    pool.step_begin([0] * 6, [5, 4, 3, 2, 1, 0], [1, 1, 2, 1, 1, 19])
    pos = pool.step_positions()
    assert pos.max() > 1_900_000
    q = _randn((2, len(pos), 8, d), 3)
    given = q.cuda()
    out = torch.full_like(given, 7.0)
    pool.rope_queries(given, theta, out=out)
    assert torch.equal(given.cpu(), q)
    for l in range(2):
        close(out[l], q[l], pos, theta, form)
    pool.rope_queries(given, theta)
    if form:
        assert torch.equal(given, out)
    else:                              # the usual form in place has a kernel of its own
        for l in range(2):
            close(given[l], q[l], pos, theta, form)
    one = torch.full_like(out[:1], 7.0)
    pool.rope_queries(q[:1].cuda(), theta, layer_count=1, out=one)
    assert torch.equal(one, out[:1]) and pool.status() == 0


@pytest.mark.parametrize("n,hq", [(1, 1), (1, 32), (3, 8), (40, 4), (700, 2), (5000, 1)])
def test_numbers_of_queries(lib, n, hq):
    """One token per CTA up to sixteen."""
    import torch
    form = {"layout": "interleaved", "rotary_dim": 48, "scaling": "linear", "factor": 3.0}
    pool = _pool(lib, 128, hq=hq, hkv=max(1, hq // 8), layers=3, n_pages=n // 16 + 2, threads=1, queries=n)
    pool.set_rope(**form)
    pool.request_begin()
    pool.step_begin([0], [0], [n])
    q = _randn((3, n, hq, 128), 4)
    out = torch.empty_like(q, device="cuda")
    pool.rope_queries(q.cuda(), 1e4, out=out)
    for l in (0, 2):
        close(out[l], q[l], np.arange(n), 1e4, form)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("kind", ["bf16", "8bit", "4bit"])
@pytest.mark.parametrize("d", [128, 64])
def test_keys_of_every_pool(lib, form, kind, d):
    """A run and a step's tokens, read back: bf16 keys by the tolerance, codes bit for bit."""
    import torch
    flags = {"bf16": 0, "8bit": lib.FLAG_KV_FP8, "4bit": lib.FLAG_KV_INT4}[kind]
    pool = _pool(lib, d, flags=flags)
    pool.set_rope(**form)
    pool.request_begin()
    n = 83
    pool.thread_spawn_predicted(0, 9_000)
    k, v = _randn((2, n, 2, d), 1), _randn((2, n, 2, d), 2)
    pool.kv_append_run_rope(0, 0, n, k.cuda(), v.cuda(), 10000.0)
    pool.step_begin([0, 0], [1, 0], [2, 3])
    pos = pool.step_positions()
    k1, v1 = _randn((2, 5, 2, d), 5), _randn((2, 5, 2, d), 6)
    pool.kv_append_rope(k1.cuda(), v1.cuda(), 10000.0)
    where = np.concatenate([np.arange(9_000, 9_000 + n), pos[2:]])
    got_k, got_v = pool.kv_read_layers(0, 0, 0, n + 3)
    fork_k, fork_v = pool.kv_read_layers(0, 1, 0, 2)
    for l in range(2):
        x, y = torch.cat([k[l], k1[l, 2:]]), torch.cat([v[l], v1[l, 2:]])
        for got, values, positions, want_v, read_v in ((got_k[l], x, where, y, got_v[l]), (fork_k[l], k1[l, :2], pos[:2], v1[l, :2], fork_v[l])):
            if kind == "bf16":
                close(got, values, positions, 1e4, form)
                assert torch.equal(read_v.cpu(), want_v)
                continue
            turned = rotate_form(values, positions, 1e4, form).astype(np.float32)
            m = len(values)
            if kind == "4bit":
                store = Kv4Store(10, 16, 2, d)
                store.write([(i // 16, i % 16) for i in range(m)], turned, want_v)
            else:                      # a page's scale is that of the tokens that came together, and grows with later ones
                store = Kv8Store(10, 16, 2, d)
                split = n if m > 2 else m
                store.write([(i // 16, i % 16) for i in range(split)], turned[:split], want_v[:split])
                store.write([(i // 16, i % 16) for i in range(split, m)], turned[split:], want_v[split:])
            wk, wv = store.gather([(i // 16, i % 16) for i in range(m)])
            assert np.array_equal(got.double().cpu().numpy(), wk) and np.array_equal(read_v.double().cpu().numpy(), wv)
    assert pool.status() == 0


@pytest.mark.parametrize("d", [64, 128])
def test_long_runs_on_a_bf16_pool(lib, d):
    """More tokens than one launch takes, from inside a page on, several layers."""
    import torch
    form = {"scaling": "wavelength", "factor": 8.0, "original_length": 1024.0, "rotary_dim": 32}
    n = 8192 + 700
    pool = _pool(lib, d, hkv=1, hq=1, n_pages=n // 16 + 2, threads=1)
    pool.set_rope(**form)
    pool.request_begin()
    k, v = _randn((2, n, 1, d), 1), _randn((2, n, 1, d), 2)
    pool.kv_append_run_rope(0, 0, 5, k[:, :5].contiguous().cuda(), v[:, :5].contiguous().cuda(), 5e5)
    pool.kv_append_run_rope(0, 0, n - 5, k[:, 5:].contiguous().cuda(), v[:, 5:].contiguous().cuda(), 5e5)
    got_k, got_v = pool.kv_read_layers(0, 0, 0, n)
    for l in range(2):
        close(got_k[l], k[l], np.arange(n), 5e5, form)
    assert torch.equal(got_v.cpu(), v) and pool.status() == 0


@pytest.mark.parametrize("form", [{"layout": "interleaved"}, {"rotary_dim": 32}, {"rotary_dim": 64, "layout": "interleaved"}])
def test_numbers_that_are_not_finite(lib, form):
    """Queries, and keys of a bf16 pool: an infinity or a NaN spoils the pair it is in and nothing else."""
    import torch
    pool = _pool(lib, 128)
    pool.set_rope(**form)
    pool.request_begin()
    pool.kv_append_run(0, 0, 40)
    pool.step_begin([0], [0], [2])
    R = form.get("rotary_dim") or 128
    pair = (lambda i: i ^ 1) if form.get("layout") else (lambda i: i + R // 2 if i < R // 2 else i - R // 2)
    q = _randn((1, 2, 8, 128), 3)
    bad = q.clone()
    spoilt = torch.zeros(q.shape, dtype=torch.bool)
    for i, x in enumerate([float("inf"), float("nan"), float("-inf"), float("inf")]):
        e = [3, R - 1, R // 2, 127][i]
        bad[0, i % 2, i, e] = x
        for at in {e, pair(e) if e < R else e}:
            spoilt[0, i % 2, i, at] = True
    outs = [torch.empty_like(q, device="cuda") for _ in range(2)]
    pool.rope_queries(q.cuda(), out=outs[0])
    pool.rope_queries(bad.cuda(), out=outs[1])
    clean, out = (o.cpu() for o in outs)
    assert torch.equal(clean[~spoilt], out[~spoilt]) and not bool(torch.isfinite(out[spoilt]).any())
    pool.kv_append_rope(bad[:, :, :2].contiguous().cuda(), q[:, :, :2].contiguous().cuda(), layer_count=1)
    got, _ = pool.kv_read(0, 0, 0, 40, 2)
    want = out[0, :, :2]
    assert torch.equal(torch.nan_to_num(got.cpu()), torch.nan_to_num(want)) and torch.equal(got.cpu().isnan(), want.isnan())


def test_small_and_large_numbers(lib):
    """Subnormal and huge bf16 numbers turn as others do."""
    import torch
    pool = _pool(lib, 128)
    pool.set_rope(layout="interleaved", scaling="linear", factor=2.0)
    pool.request_begin()
    pool.kv_append_run(0, 0, 1000)
    pool.step_begin([0], [0], [1])
    sizes = torch.tensor([2.0 ** -133, 2.0 ** -128, 2.0 ** -126, 2.0 ** -60, 1.0, 2.0 ** 60, 2.0 ** 120, 2.0 ** 126]).reshape(1, 1, 8, 1)
    q = (_randn((1, 1, 8, 128), 3).float().clamp(-3, 3) * sizes * 0.25).to(torch.bfloat16)
    out = torch.empty_like(q, device="cuda")
    pool.rope_queries(q.cuda(), out=out)
    want = rotate_form(q[0], [1000], 1e4, {"layout": "interleaved", "scaling": "linear", "factor": 2.0})
    step = np.maximum(2.0 ** -8 * np.abs(want), 2.0 ** -134)               # half a step, of subnormal results too
    pair = 2.0 ** -22 * np.abs(q.float().numpy()[0]).max(-1, keepdims=True)
    assert np.all(np.abs(out[0].double().cpu().numpy() - want) <= step * (1 + 2.0 ** -10) + pair)


def test_a_form_stays_with_what_was_captured(lib):
    """A captured call keeps the form it was made with; later calls take the new one; other pools keep theirs."""
    import torch
    pool, other = _pool(lib, 128), _pool(lib, 128)
    for p in (pool, other):
        p.request_begin()
        p.kv_append_run(0, 0, 500)
        p.step_begin([0], [0], [1])
    q = _randn((2, 1, 8, 128), 3).cuda()
    out = torch.empty_like(q)
    pool.set_rope(layout="interleaved")
    pool.rope_queries(q, out=out)
    first = out.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pool.rope_queries(q, out=out)
    pool.set_rope(rotary_dim=32)
    later, usual = torch.empty_like(q), torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    pool.rope_queries(q, out=later, stream=side)
    other.rope_queries(q, out=usual)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, first) and not torch.equal(later, first)
    for l in range(2):
        close(later[l], q[l].cpu(), [500], 1e4, {"rotary_dim": 32})
        close(usual[l], q[l].cpu(), [500], 1e4, {})
    pool.set_rope()
    pool.rope_queries(q, out=later)
    assert torch.equal(later, usual)


def test_steps_that_attend_in_a_form(lib):
    """Rotated keys and queries of one form through a whole step on each kind of pool: scores depend on distances alone, so a context
    and a query moved on by 5000 positions give what they give at the start."""
    import torch
    for kind, flags in (("bf16", 0), ("8bit", lib.FLAG_KV_FP8), ("4bit", lib.FLAG_KV_INT4)):
        outs = []
        for start in (0, 5000):
            pool = _pool(lib, 128, layers=1, flags=flags)
            pool.set_rope(layout="interleaved", rotary_dim=64, scaling="base", factor=4.0)
            pool.request_begin()
            pool.thread_spawn_predicted(0, start)
            k, v, q = _randn((1, 200, 2, 128), 1).cuda(), _randn((1, 200, 2, 128), 2).cuda(), _randn((1, 1, 8, 128), 3).cuda()
            pool.kv_append_run_rope(0, 0, 199, k[:, :199].contiguous(), v[:, :199].contiguous())
            pool.step_begin([0], [0], [1])
            pool.kv_append_rope(k[:, 199:].contiguous(), v[:, 199:].contiguous())
            pool.rope_queries(q)
            out = torch.empty((1, 1, 8, 128), device="cuda")
            pool.decode_attn(q, out)
            outs.append(out)
            assert pool.status() == 0
        # rotated keys are rounded to bf16 or to codes of 4 or 8 bits, elsewhere for each start: shares of a key's size by which
        # its scores may move (of sqrt(128) elements each up to 1/13 of the largest for 4 bits, independent of one another)
        noise = {"bf16": 0.05, "8bit": 0.2, "4bit": 0.6}[kind]
        assert (outs[0] - outs[1]).abs().max() <= noise and (outs[0] - outs[1]).abs().max() < outs[0].abs().max()


def test_refusals(lib):
    import torch
    pool = _pool(lib, 128, layers=1)
    pool.request_begin()
    flat = torch.zeros(4096, dtype=torch.bfloat16, device="cuda")
    q, odd = flat[:1024].view(1, 1, 8, 128), flat[1:1025].view(1, 1, 8, 128)
    with pytest.raises(lib.PastaError) as e:
        pool.rope_queries(q, out=flat[1024:2048])
    assert e.value.code == lib.BAD_STATE                                  # no step
    pool.set_rope(layout="interleaved")
    k, odd_k = flat[:256].view(1, 1, 2, 128), flat[4:260].view(1, 1, 2, 128)
    for a, b in ((odd_k, k), (k, odd_k)):
        with pytest.raises(lib.PastaError):
            pool.kv_append_run_rope(0, 0, 1, a, b)
    assert pool.dump()["requests"][0]["streams"][0]["len"] == 0 and pool.launch_count() == 0
    pool.step_begin([0], [0], [1])
    for call in (lambda: pool.rope_queries(odd), lambda: pool.rope_queries(q, out=odd), lambda: pool.rope_queries(odd, out=q),
                 lambda: pool.rope_queries(q, 1.0), lambda: pool.rope_queries(q, float("nan")), lambda: pool.rope_queries(q, float("inf")),
                 lambda: pool.rope_queries(q, layer_count=2), lambda: pool.rope_queries(q, layer_count=-1),
                 lambda: pool.rope_queries(None, out=q), lambda: pool.kv_append_rope(odd_k, k), lambda: pool.kv_append_rope(k, odd_k)):
        with pytest.raises(lib.PastaError) as e:
            call()
        assert e.value.code == lib.INVALID_ARG
    assert pool.launch_count() == 0
    pool.rope_queries(q, layer_count=0, out=odd)
    pool.rope_queries(q)
    pool.kv_append_rope(k, k)
    assert pool.launch_count() == 2 and pool.status() == 0
