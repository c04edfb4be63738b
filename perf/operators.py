"""The operators around the 8-bit KV cache and capped attention scores, as cases that can be timed and compared.

Three operators of a decode step:

* ``store``   a prompt's keys (rotated by position) and values enter a cache that holds them in 8 bits (e4m3) with one
              power-of-two scale for the keys and one for the values of every page of 16 tokens and kv head; what the cache
              then holds is read back;
* ``attend``  decode attention of every thread of every response over that cache: each response has one prompt stream that
              its threads share up to their spawn point, and one private chunk per fork;
* ``attend`` with ``cap`` > 0: the same with scores capped by ``cap * tanh(score / cap)``, over a bf16 cache or the 8-bit one.

``own = False`` computes them with elementary torch operations; ``own = True`` makes the calls of the package.
"""
import math
import random

import torch

own = False

PAGE = 16            # tokens of one page, which share a scale
E4M3_MAX = 448.0
EXP_MIN, EXP_MAX = -64, 63      # range of a page's scale exponent

def _attend(name, cache, layers, heads, head_dim, requests, prefix, forks, chunk, cap=0.0, gain=1.0, lengths=1):
    return {"name": name, "op": "attend", "cache": cache, "layers": layers, "q_heads": heads[0], "kv_heads": heads[1],
            "head_dim": head_dim, "requests": requests, "prefix_lo": prefix[0], "prefix_hi": prefix[1],
            "forks_lo": forks[0], "forks_hi": forks[1], "chunk_lo": chunk[0], "chunk_hi": chunk[1],
            "cap": cap, "gain": gain, "lengths": lengths}


def _store(name, layers, kv_heads, head_dim, tokens, theta):
    return {"name": name, "op": "store", "cache": "8bit", "layers": layers, "kv_heads": kv_heads, "head_dim": head_dim,
            "tokens": tokens, "theta": theta}


def listed():
    return [
        # one response a little way into its text, two forks just spawned: what a single user waits for, latency only
        _attend("attend8 one response", "8bit", 1, (32, 8), 128, 1, (203, 203), (2, 2), (9, 40)),
        # many responses of mixed length on a small model's heads
        _attend("attend8 mixed d64", "8bit", 2, (16, 8), 64, 32, (61, 1500), (0, 4), (10, 300)),
        # the batched decode step: 64 responses, some without forks, some with eight
        _attend("attend8 batch", "8bit", 2, (32, 8), 128, 64, (256, 2048), (0, 8), (10, 300)),
        # eight long documents with sixteen forks each: the shared prefix is nearly everything that is read
        _attend("attend8 long prefix", "8bit", 1, (32, 8), 128, 8, (32768, 32768), (16, 16), (50, 400)),
        # capped scores for one response of the usual length, bf16 cache
        _attend("capped one response", "bf16", 1, (32, 8), 128, 1, (768, 768), (4, 4), (20, 200), cap=50.0, gain=4.0),
        # capped scores in the batched decode step, bf16 cache
        _attend("capped batch", "bf16", 1, (32, 8), 128, 64, (256, 2048), (0, 8), (10, 300), cap=30.0, gain=4.0),
        # capped scores over the 8-bit cache while many short responses run, eight query heads to a kv head
        _attend("capped8 short responses", "8bit", 4, (32, 4), 128, 64, (64, 1024), (2, 6), (1, 160), cap=50.0, gain=4.0),
        # capped scores with a kv head for every query head, head size 64, bf16 cache
        _attend("capped d64 no groups", "bf16", 1, (8, 8), 64, 16, (100, 3001), (0, 3), (10, 300), cap=20.0, gain=3.0),
        # a question of a few words enters the cache of one layer
        _store("store8 question", 1, 8, 128, 37, 10000.0),
        # a page of text enters the cache of eight layers
        _store("store8 page", 8, 8, 128, 1023, 10000.0),
        # keys that arrive rotated already, head size 64
        _store("store8 unrotated d64", 4, 4, 64, 4095, 0.0),
        # a long document enters the cache of one layer
        _store("store8 document", 1, 8, 128, 32768, 500000.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.499)))))))


def draw(rng):
    head_dim = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 8])
    if rng.random() < 0.3:
        layers = rng.choice([1, 1, 2, 4])
        tokens = min(_log_int(rng, 1, 32768), 32768 * 1024 // (layers * kv_heads * head_dim))
        case = _store("", layers, kv_heads, head_dim, tokens, rng.choice([0.0, 10000.0, 500000.0]))
    else:
        group = rng.choice([1, 2, 4, 4, 8])
        capped = rng.random() < 0.5
        cache = rng.choice(["8bit", "bf16"]) if capped else "8bit"
        layers = rng.choice([1, 1, 2])
        prefix_hi = _log_int(rng, 1, 32768)
        prefix_lo = rng.randint(max(1, prefix_hi // 8), prefix_hi)
        forks_hi = rng.choice([0, 1, 2, 4, 8, 16])
        forks_lo = rng.randint(0, forks_hi)
        chunk_hi = _log_int(rng, 1, 400)
        chunk_lo = rng.randint(1, chunk_hi)
        room = 150_000_000 // (layers * kv_heads * head_dim * (prefix_hi + forks_hi * chunk_hi + PAGE))
        room = min(room, 40_000_000 // (group * kv_heads * (1 + forks_hi) * (prefix_hi + forks_hi * chunk_hi + PAGE)))
        requests = min(_log_int(rng, 1, 64), max(1, room))
        cap, gain = (rng.choice([20.0, 30.0, 50.0]), rng.choice([1.0, 4.0])) if capped else (0.0, rng.choice([1.0, 2.0]))
        case = _attend("", cache, layers, (kv_heads * group, kv_heads), head_dim, requests, (prefix_lo, prefix_hi),
                       (forks_lo, forks_hi), (chunk_lo, chunk_hi), cap, gain, rng.randrange(1 << 30))
    del case["name"]
    return case


# ---------------------------------------------------------------------------------------------------------------------
# the responses of a case: lengths come from the case alone, values from the seed
# ---------------------------------------------------------------------------------------------------------------------
def _responses(case):
    """Per response: (prompt length, [(spawn point, chunk length) of every fork, in order of spawning])."""
    rng = random.Random(case["lengths"])
    out = []
    for _ in range(case["requests"]):
        prefix = rng.randint(case["prefix_lo"], case["prefix_hi"])
        n = rng.randint(case["forks_lo"], case["forks_hi"])
        points = sorted(rng.randint(max(1, prefix - 256), prefix) for _ in range(n))
        out.append((prefix, [(c, rng.randint(case["chunk_lo"], case["chunk_hi"])) for c in points]))
    return out


def _pages(tokens):
    return -(-tokens // PAGE)


class _Layout:
    """Where the tokens of a case lie in a paged cache: streams one after the other, a response's streams together."""

    def __init__(self, case):
        self.responses = _responses(case)
        self.streams = []                       # (response, stream, first page, length); stream 0 is the prompt
        self.first = []                         # first stream of every response
        page = 0
        for r, (prefix, forks) in enumerate(self.responses):
            self.first.append(len(self.streams))
            for s, length in enumerate([prefix] + [n for _, n in forks]):
                self.streams.append((r, s, page, length))
                page += _pages(length)
        self.n_pages = page
        self.n_threads = [1 + len(forks) for _, forks in self.responses]
        self.n_queries = sum(self.n_threads)

    def visible(self, r, thread):
        """(stream, visible tokens) of everything the thread attends to."""
        prefix, forks = self.responses[r]
        return [(0, prefix)] if thread == 0 else [(0, forks[thread - 1][0]), (thread, forks[thread - 1][1])]


def _inputs(case, seed):
    """Keys and values in page order, zero in slots that hold no token, and the queries: bf16, on the GPU."""
    lay = _Layout(case)
    L, H, Hq, D = case["layers"], case["kv_heads"], case["q_heads"], case["head_dim"]
    g = torch.Generator(device="cuda").manual_seed(seed)
    # a key channel has a size of its own, as the keys of trained models do
    channel = torch.exp(0.5 * torch.randn(H, D, generator=g, device="cuda"))
    shape = (L, lay.n_pages, PAGE, H, D)
    k = (torch.randn(shape, generator=g, device="cuda") * channel).bfloat16()
    v = torch.randn(shape, generator=g, device="cuda").bfloat16()
    q = (case["gain"] * torch.randn((L, lay.n_queries, Hq, D), generator=g, device="cuda")).bfloat16()
    held = torch.full((lay.n_pages,), PAGE, dtype=torch.int64)
    for _, _, page, length in lay.streams:
        if length % PAGE:
            held[page + length // PAGE] = length % PAGE
    empty = (torch.arange(PAGE)[None, :] >= held[:, None]).cuda()
    k[:, empty] = 0
    v[:, empty] = 0
    return lay, k, v, q


def _prompt(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    shape = (case["layers"], case["tokens"], case["kv_heads"], case["head_dim"])
    channel = torch.exp(0.5 * torch.randn(shape[2:], generator=g, device="cuda"))
    k = (torch.randn(shape, generator=g, device="cuda") * channel).bfloat16()
    v = torch.randn(shape, generator=g, device="cuda").bfloat16()
    return k, v


# ---------------------------------------------------------------------------------------------------------------------
# plain form
# ---------------------------------------------------------------------------------------------------------------------
def _power_of_two(e):
    """2^e as fp32 for integers -126 <= e <= 127, from its bits: a library's pow may be off in the last place."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantise(pages):
    """pages [..., PAGE, heads, dim] fp32 -> e4m3 codes of the same shape and exponents [..., heads] (value = code * 2^e)."""
    amax = pages.abs().amax(dim=(-3, -1))
    m, e = torch.frexp(amax)                               # amax = m * 2^e, 0.5 <= m < 1; 448 = 0.875 * 2^9
    e = (e - 9 + (m > 0.875).to(e.dtype)).clamp(EXP_MIN, EXP_MAX)
    e = torch.where(amax > 0, e, torch.full_like(e, EXP_MIN))
    scaled = (pages * _power_of_two(-e)[..., None, :, None]).clamp(-E4M3_MAX, E4M3_MAX)
    return scaled.to(torch.float8_e4m3fn), e


def _dequantise(codes, e):
    return codes.float() * _power_of_two(e)[..., None, :, None]


def _rotate(k, theta):
    """Rotate-half position embedding of [layers, tokens, heads, dim] by position = token index, angles in 64 bits."""
    L, T, H, D = k.shape
    i = torch.arange(D // 2, dtype=torch.float64, device=k.device)
    angle = torch.arange(T, dtype=torch.float64, device=k.device)[:, None, None] * theta ** (-2.0 * i / D)
    c, s = angle.cos(), angle.sin()
    lo, hi = k[..., : D // 2].double(), k[..., D // 2 :].double()
    return torch.cat([lo * c - hi * s, hi * c + lo * s], dim=-1).float()


def _plain_store(st):
    k, v, theta = st["k"], st["v"], st["theta"]
    L, T, H, D = k.shape
    both = torch.stack([_rotate(k, theta) if theta else k.float(), v.float()])
    both = torch.nn.functional.pad(both, (0, 0, 0, 0, 0, _pages(T) * PAGE - T))
    codes, e = _quantise(both.reshape(2, L, _pages(T), PAGE, H, D))
    held = _dequantise(codes, e).reshape(2, L, -1, H, D)[:, :, :T].bfloat16()
    return {"k": held[0], "v": held[1]}


def _plain_attend(st):
    case = st["case"]
    L, H, D = case["layers"], case["kv_heads"], case["head_dim"]
    G = case["q_heads"] // H
    table, seen, rows = st["table"], st["seen"], st["rows"]       # [R, P], [R, N, P], [R, N]
    R, P = table.shape
    N = seen.shape[1]
    if case["cache"] == "8bit":
        k = _dequantise(st["k"][:, table], st["k_exp"][:, table])
        v = _dequantise(st["v"][:, table], st["v_exp"][:, table])
    else:
        k, v = st["k"][:, table].float(), st["v"][:, table].float()
    k = k.reshape(L, R, P * PAGE, H, D).permute(0, 1, 3, 4, 2)                        # [L, R, H, D, T]
    v = v.reshape(L, R, P * PAGE, H, D).permute(0, 1, 3, 2, 4)                        # [L, R, H, T, D]
    q = st["q"].float()[:, rows].reshape(L, R, N, H, G, D).permute(0, 1, 3, 2, 4, 5).reshape(L, R, H, N * G, D)
    s = torch.matmul(q, k) * (1.0 / math.sqrt(D))
    if case["cap"]:
        s = case["cap"] * torch.tanh(s / case["cap"])
    mask = (torch.arange(PAGE, device=q.device) < seen[..., None]).reshape(R, 1, N, 1, P * PAGE)
    s = s.reshape(L, R, H, N, G, P * PAGE).masked_fill(~mask, float("-inf")).reshape(L, R, H, N * G, P * PAGE)
    top = s.amax(dim=-1, keepdim=True).clamp_min(-3.0e38)         # a padding row of this form sees nothing
    w = torch.exp(s - top)
    total = w.sum(dim=-1, keepdim=True).clamp_min(1e-30)
    out = torch.matmul(w, v) / total
    out = out.reshape(L, R, H, N, G, D).permute(0, 1, 3, 2, 4, 5).reshape(L, R * N, H * G, D)[:, st["where"]].bfloat16()
    return {"out": out}


def _plain_state(case, lay, k, v, q):
    """The paged cache, page tables and per-page visible lengths that a program of plain torch operations would keep."""
    R, N = len(lay.responses), max(lay.n_threads)
    pages_of = [[] for _ in range(R)]             # (stream, page index in the stream, page)
    for r, s, page, length in lay.streams:
        pages_of[r] += [(s, i, page + i) for i in range(_pages(length))]
    P = max(len(p) for p in pages_of)
    table = torch.zeros((R, P), dtype=torch.int64)
    seen = torch.zeros((R, N, P), dtype=torch.int64)
    rows = torch.zeros((R, N), dtype=torch.int64)
    where, at = [], 0
    for r in range(R):
        s, i, page = (torch.tensor(x) for x in zip(*pages_of[r]))
        table[r, : len(page)] = page
        for t in range(lay.n_threads[r]):
            for stream, n in lay.visible(r, t):
                seen[r, t, : len(page)] += torch.where(s == stream, (n - i * PAGE).clamp(0, PAGE), 0)
            rows[r, t] = at
            where.append(r * N + t)
            at += 1
    st = {"case": case, "q": q, "table": table.cuda(), "seen": seen.cuda(), "rows": rows.cuda(),
          "where": torch.tensor(where).cuda()}
    if case["cache"] == "8bit":
        st["k"], st["k_exp"] = _quantise(k.float())
        st["v"], st["v_exp"] = _quantise(v.float())
    else:
        st["k"], st["v"] = k, v
    return st


# ---------------------------------------------------------------------------------------------------------------------
# the package's calls
# ---------------------------------------------------------------------------------------------------------------------
def _own_pool(case, n_pages, requests, threads, segments, queries):
    from paper_2502_11517_b200 import binding
    flags = binding.FLAG_OUT_BF16 | (binding.FLAG_KV_FP8 if case["cache"] == "8bit" else 0)
    return binding.Pool(case["layers"], case.get("q_heads", case["kv_heads"]), case["kv_heads"], case["head_dim"], n_pages,
                        requests, threads, segments, max_step_queries=queries, flags=flags,
                        device=torch.cuda.current_device())


def _own_attend_state(case, lay, k, v, q):
    """The pool with every response's tokens in it, and the step in which all its threads attend."""
    n = max(lay.n_threads)
    pool = _own_pool(case, lay.n_pages, len(lay.responses), n, 2 * n + 2, lay.n_queries)
    L, _, _, H, D = k.shape

    def append(req, stream, page, lo, hi):
        if hi > lo:
            part = [x[:, page : page + _pages(hi)].reshape(L, -1, H, D)[:, lo:hi].contiguous() for x in (k, v)]
            pool.kv_append_run(req, stream, hi - lo, *part)

    reqs, threads = [], []
    for r, (prefix, forks) in enumerate(lay.responses):
        req = pool.request_begin()
        streams = lay.streams[lay.first[r] : lay.first[r] + lay.n_threads[r]]
        at = 0
        for cut, _ in forks:
            append(req, 0, streams[0][2], at, cut)
            at = cut
            pool.thread_spawn(req)
        append(req, 0, streams[0][2], at, prefix)
        for _, s, page, length in streams[1:]:
            append(req, s, page, 0, length)
        reqs += [req] * len(streams)
        threads += list(range(len(streams)))
    if case["cap"]:
        pool.set_softcap(case["cap"])
    pool.step_begin(reqs, threads, [0] * len(reqs))
    return {"case": case, "pool": pool, "q": q}


def _own_attend(st):
    case, pool, q = st["case"], st["pool"], st["q"]
    out = torch.empty_like(q)
    pool.decode_attn(q, out)
    return {"out": out}


def _own_store(st):
    pool, k, v, theta = st["pool"], st["k"], st["v"], st["theta"]
    L, T = k.shape[:2]
    req = pool.request_begin()
    if theta:
        pool.kv_append_run_rope(req, 0, T, k, v, theta)
    else:
        pool.kv_append_run(req, 0, T, k, v)
    k_held, v_held = pool.kv_read_layers(req, 0, 0, T)
    pool.request_end(req)
    return {"k": k_held, "v": v_held}


# ---------------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    if case["op"] == "store":
        k, v = _prompt(case, seed)
        st = {"case": case, "k": k, "v": v, "theta": case["theta"]}
        if own:
            st["pool"] = _own_pool(case, _pages(case["tokens"]), 1, 1, 2, 1)
        return st
    lay, k, v, q = _inputs(case, seed)
    return _own_attend_state(case, lay, k, v, q) if own else _plain_state(case, lay, k, v, q)


def run(state):
    if state["case"]["op"] == "store":
        return _own_store(state) if own else _plain_store(state)
    return _own_attend(state) if own else _plain_attend(state)


def work(case):
    L, H, D = case["layers"], case["kv_heads"], case["head_dim"]
    if case["op"] == "store":
        T = case["tokens"]
        values = 2.0 * L * T * H * D
        scales = 2.0 * L * _pages(T) * H
        # keys and values in (bf16), codes and scales into the cache, keys and values out (bf16)
        return {"bytes": values * (2 + 1 + 2) + scales, "flops": values * (3 if case["theta"] else 1)}
    lay = _Layout(case)
    tokens = sum(length for _, _, _, length in lay.streams)
    pairs = sum(n for r in range(len(lay.responses)) for t in range(lay.n_threads[r]) for _, n in lay.visible(r, t))
    eight = case["cache"] == "8bit"
    cache = 2.0 * L * tokens * H * D * (1 if eight else 2) + (2.0 * L * lay.n_pages * H if eight else 0)
    rows = L * lay.n_queries * case["q_heads"]
    return {"bytes": cache + rows * D * 4.0, "flops": 4.0 * L * pairs * case["q_heads"] * D}


# ---------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _held(x):
    """What the 8-bit cache holds of one page's numbers x [..., tokens, dim] (64 bits, one kv head): the scale is the
    smallest power of two that brings the page's largest magnitude to at most 448, the numbers are rounded to the nearest
    e4m3 value of that scale (four significant bits, step 2^-9 below 2^-6), ties to even."""
    two = lambda n: ((n.to(torch.int64) + 1023) << 52).view(torch.float64)
    amax = x.abs().amax(dim=(-2, -1), keepdim=True)
    e = torch.frexp(amax).exponent.long() - 8                               # amax < 256 * 2^e, one more than may be needed
    e = e - (amax <= E4M3_MAX * two(e - 1)).long()
    e = torch.where(amax > 0, e.clamp(EXP_MIN, EXP_MAX), torch.full_like(e, EXP_MIN))
    y = (x * two(-e)).clamp(-E4M3_MAX, E4M3_MAX)
    step = two(torch.frexp(y).exponent.long().clamp_min(-5) - 4)            # 2^(p - 1) <= |y| < 2^p has steps of 2^(p - 4)
    return torch.round(y / step) * step * two(e)


def _exact_store(case, seed):
    k, v = (x.double() for x in _prompt(case, seed))
    L, T, H, D = k.shape
    if case["theta"]:
        pos = torch.arange(T, device="cuda", dtype=torch.float64)
        out = torch.empty_like(k)
        for i in range(D // 2):
            turn = torch.exp(-(2.0 * i / D) * math.log(case["theta"]) * torch.ones((), dtype=torch.float64, device="cuda")) * pos
            turn = torch.polar(torch.ones_like(turn), turn)[None, :, None]
            z = torch.complex(k[..., i], k[..., i + D // 2]) * turn
            out[..., i], out[..., i + D // 2] = z.real, z.imag
        k = out.float().double()                           # a rotated key is a 32-bit number before it is quantised
    held = []
    for x in (k, v):
        pad = torch.zeros((L, _pages(T) * PAGE, H, D), dtype=torch.float64, device="cuda")
        pad[:, :T] = x
        pad = pad.reshape(L, _pages(T), PAGE, H, D).transpose(2, 3)
        held.append(_held(pad).transpose(2, 3).reshape(L, -1, H, D)[:, :T])
    return {"k": held[0], "v": held[1]}


def _exact_attend(case, seed):
    lay, k, v, q = _inputs(case, seed)
    L, H, D = case["layers"], case["kv_heads"], case["head_dim"]
    G = case["q_heads"] // H
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    for layer in range(L):
        row = 0
        for r in range(len(lay.responses)):
            streams = lay.streams[lay.first[r] : lay.first[r] + lay.n_threads[r]]
            for h in range(H):
                parts = []
                for _, _, page, length in streams:
                    pair = []
                    for x in (k, v):
                        y = x[layer, page : page + _pages(length), :, h].double()          # [pages, PAGE, D]
                        pair.append((_held(y) if case["cache"] == "8bit" else y).reshape(-1, D))
                    parts.append(pair)
                for t in range(lay.n_threads[r]):
                    kt = torch.cat([parts[s][0][:n] for s, n in lay.visible(r, t)])
                    vt = torch.cat([parts[s][1][:n] for s, n in lay.visible(r, t)])
                    s = q[layer, row + t, h * G : (h + 1) * G].double() @ kt.T / math.sqrt(D)
                    if case["cap"]:
                        s = case["cap"] * torch.tanh(s / case["cap"])
                    out[layer, row + t, h * G : (h + 1) * G] = torch.softmax(s, dim=1) @ vt
            row += lay.n_threads[r]
    return {"out": out}


def exact(case, seed):
    return _exact_store(case, seed) if case["op"] == "store" else _exact_attend(case, seed)
