"""The operators around a 4-bit KV cache and the forms of rotary position embedding, as cases that can be timed and compared.

Three operators of a decode step:

* ``store``   a prompt's keys (rotated by position, in one of the forms below) and values enter a cache; what the cache then
              holds is read back.  The cache holds numbers in 4 bits: 32 neighbouring elements of one token's key (or value) of
              one kv head share a scale s, the smallest number of five significant bits with |x| <= 7 s, and an element is held
              as a whole number -7 ... 7 times s.  One case writes rotated keys to a bf16 cache instead;
* ``attend``  decode attention of every thread of every response over the 4-bit cache: each response has one prompt stream that
              its threads share up to their spawn point, and one private chunk per fork; with ``cap`` > 0 the scores are capped
              by ``cap * tanh(score / cap)``;
* ``rotate``  the queries of a step are rotated by their positions.

Forms of the rotation: a pair of elements (i and i + R/2 of the first R elements of a head, "half", or 2 i and 2 i + 1,
"interleaved") turns by position * f_i, f_i = theta^(-2i/R); for long contexts the f_i are scaled:

* "linear"      f_i / factor;
* "base"        theta becomes theta * factor^(R / (R - 2));
* "wavelength"  waves longer than original / low are stretched by the factor, those shorter than original / high are kept, and
                in between f_i goes linearly in original / wave from one to the other;
* "ramp"        pairs that turn more than `high` times over the original length are kept, those that turn less than `low` times
                are stretched, with a linear ramp over the pairs in between; what is rotated is also multiplied by
                0.1 ln(factor) + 1, or by `magnitude` where that is given.

``own = False`` computes them with elementary torch operations; ``own = True`` makes the calls of the package.
"""
import math
import random

import torch

own = False

PAGE = 16               # tokens of one page
BLOCK = 32              # elements that share a scale
TOP = 7                 # largest code
SCALE_MIN, SCALE_MAX = 2.0 ** -110, 31 * 2.0 ** 106      # range of a block's scale

PLAIN = {"theta": 10000.0, "layout": "half", "rotary_dim": 0, "scaling": "none", "factor": 1.0, "original": 0, "low": 1.0,
         "high": 4.0, "magnitude": 0.0}


def _form(**changes):
    return {**PLAIN, **changes}


def _attend(name, layers, heads, head_dim, requests, prefix, forks, chunk, cap=0.0, gain=1.0, lengths=1):
    return {"name": name, "op": "attend", "layers": layers, "q_heads": heads[0], "kv_heads": heads[1],
            "head_dim": head_dim, "requests": requests, "prefix_lo": prefix[0], "prefix_hi": prefix[1],
            "forks_lo": forks[0], "forks_hi": forks[1], "chunk_lo": chunk[0], "chunk_hi": chunk[1],
            "cap": cap, "gain": gain, "lengths": lengths}


def _store(name, cache, layers, kv_heads, head_dim, tokens, form):
    return {"name": name, "op": "store", "cache": cache, "layers": layers, "kv_heads": kv_heads, "head_dim": head_dim,
            "tokens": tokens, **form}


def _rotate(name, layers, heads, head_dim, requests, tokens, start, form):
    return {"name": name, "op": "rotate", "layers": layers, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": head_dim,
            "requests": requests, "tokens": tokens, "start": start, **form}


def listed():
    return [
        # one response a little way into its text, two forks just spawned: what a single user waits for, latency only
        _attend("attend4 one response", 1, (32, 8), 128, 1, (203, 203), (2, 2), (9, 40)),
        # many responses of mixed length on a small model's heads
        _attend("attend4 mixed d64", 2, (16, 8), 64, 32, (61, 1500), (0, 4), (10, 300)),
        # the batched decode step: 64 responses, some without forks, some with eight
        _attend("attend4 batch", 2, (32, 8), 128, 64, (256, 2048), (0, 8), (10, 300)),
        # eight long documents with sixteen forks each: the shared prefix is nearly everything that is read
        _attend("attend4 long prefix", 1, (32, 8), 128, 8, (32768, 32768), (16, 16), (50, 400)),
        # capped scores while many short responses run, eight query heads to a kv head
        _attend("attend4 short capped", 4, (32, 4), 128, 64, (64, 1024), (2, 6), (1, 160), cap=50.0, gain=4.0),
        # a question of a few words enters the cache of one layer
        _store("store4 question", "4bit", 1, 8, 128, 37, _form()),
        # a page of text enters the cache of eight layers, neighbouring elements paired, half of each head rotated
        _store("store4 page", "4bit", 8, 8, 128, 1023, _form(layout="interleaved", rotary_dim=64)),
        # keys that arrive rotated already, head size 64
        _store("store4 unrotated d64", "4bit", 4, 4, 64, 4095, _form(theta=0.0)),
        # a long document enters the cache of one layer, positions stretched by wavelength
        _store("store4 document", "4bit", 1, 8, 128, 32768,
               _form(theta=500000.0, scaling="wavelength", factor=8.0, original=8192)),
        # the same kind of document in a bf16 cache, positions stretched along a ramp over the pairs
        _store("store16 document", "bf16", 1, 8, 128, 16384,
               _form(scaling="ramp", factor=4.0, original=4096, low=1.0, high=32.0)),
        # the queries of one response's decode step with a few threads, far into a long text
        _rotate("rotate step", 2, (32, 8), 128, 1, 5, 70001, _form(theta=500000.0, scaling="linear", factor=4.0)),
        # the queries of prompts that are fed in chunks
        _rotate("rotate chunks", 8, (32, 8), 128, 4, 256, 1000, _form(layout="interleaved", scaling="base", factor=2.0)),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.499)))))))


def _draw_form(rng, head_dim):
    original = rng.choice([2048, 4096, 8192])
    scaling = rng.choice(["none", "linear", "base", "wavelength", "ramp"])
    low, high = (1.0, 32.0) if scaling == "ramp" else (1.0, 4.0)
    return _form(theta=rng.choice([10000.0, 500000.0, 1000000.0]), layout=rng.choice(["half", "interleaved"]),
                 rotary_dim=rng.choice([0, 0, 16, 32, 48, 64, head_dim // 2, head_dim]), scaling=scaling,
                 factor=1.0 if scaling == "none" else rng.choice([2.0, 2.5, 4.0, 8.0, 32.0]), original=original, low=low, high=high,
                 magnitude=rng.choice([0.0, 0.0, 1.25]) if scaling == "ramp" else 0.0)


def draw(rng):
    head_dim = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 8])
    kind = rng.random()
    if kind < 0.35:
        layers = rng.choice([1, 1, 2, 4])
        cache = rng.choice(["4bit", "4bit", "4bit", "bf16"])
        tokens = min(_log_int(rng, 1, 32768), 32768 * 1024 // (layers * kv_heads * head_dim))
        form = _draw_form(rng, head_dim)
        if rng.random() < 0.2:
            form["theta"] = 0.0
        case = _store("", cache, layers, kv_heads, head_dim, tokens, form)
    elif kind < 0.55:
        group = rng.choice([1, 2, 4, 8])
        layers = rng.choice([1, 2, 4, 8])
        requests = rng.choice([1, 1, 3, 16])
        tokens = min(_log_int(rng, 1, 1024), max(1, 1024 // requests), 32768 * 1024 // (layers * kv_heads * group * head_dim * requests))
        case = _rotate("", layers, (kv_heads * group, kv_heads), head_dim, requests, max(1, tokens), _log_int(rng, 1, 200000),
                       _draw_form(rng, head_dim))
    else:
        group = rng.choice([1, 2, 4, 4, 8])
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
        cap, gain = (rng.choice([20.0, 30.0, 50.0]), rng.choice([1.0, 4.0])) if rng.random() < 0.3 else (0.0, rng.choice([1.0, 2.0]))
        case = _attend("", layers, (kv_heads * group, kv_heads), head_dim, requests, (prefix_lo, prefix_hi),
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


def _queries(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    shape = (case["layers"], case["requests"] * case["tokens"], case["q_heads"], case["head_dim"])
    return torch.randn(shape, generator=g, device="cuda").bfloat16()


def _step_positions(case):
    """Position of every query of a rotate case: request r starts where the one before it does, 17 further on."""
    at = torch.arange(case["tokens"], dtype=torch.float64)
    return torch.cat([at + case["start"] + 17 * r for r in range(case["requests"])])


# ---------------------------------------------------------------------------------------------------------------------
# plain form
# ---------------------------------------------------------------------------------------------------------------------
def _frequencies(case):
    """(f_i of every pair, what the rotated elements are multiplied by), in 64 bits."""
    R = case["rotary_dim"] or case["head_dim"]
    theta, scaling, factor, original = case["theta"], case["scaling"], case["factor"], case["original"]
    if scaling == "base":
        theta = theta * factor ** (R / (R - 2))
    f = [theta ** (-2.0 * i / R) for i in range(R // 2)]
    if scaling == "linear":
        f = [x / factor for x in f]
    elif scaling == "wavelength":
        out = []
        for x in f:
            wave = 2 * math.pi / x
            if wave < original / case["high"]:
                out.append(x)
            elif wave > original / case["low"]:
                out.append(x / factor)
            else:
                t = (original / wave - case["low"]) / (case["high"] - case["low"])
                out.append((1 - t) * x / factor + t * x)
        f = out
    elif scaling == "ramp":
        def pair(turns):                    # the pair that turns so often over the original length, as a real number
            return R * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(theta))
        lo, hi = max(0, math.floor(pair(case["high"]))), min(R - 1, math.ceil(pair(case["low"])))
        if hi <= lo:
            hi = lo + 0.001
        stretched = [min(1.0, max(0.0, (i - lo) / (hi - lo))) for i in range(R // 2)]
        f = [x / factor * s + x * (1 - s) for x, s in zip(f, stretched)]
    size = 1.0
    if scaling == "ramp":
        size = case["magnitude"] or (0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0)
    return torch.tensor(f, dtype=torch.float64), size


def _turned(x, positions, case):
    """x [layers, tokens, heads, dim] rotated by the tokens' positions; angles and products in 64 bits, the result fp32."""
    f, size = _frequencies(case)
    R = 2 * len(f)
    angle = (positions.to(x.device)[:, None] * f.to(x.device))[:, None, :]
    c, s = angle.cos() * size, angle.sin() * size
    head = x[..., :R].double()
    if case["layout"] == "half":
        a, b = head[..., : R // 2], head[..., R // 2 :]
        head = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    else:
        a, b = head[..., 0::2], head[..., 1::2]
        head = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    return torch.cat([head.float(), x[..., R:].float()], dim=-1)


def _power_of_two(e):
    """2^e in 64 bits for whole -1022 <= e <= 1023, from its bits: a library's pow and ldexp may be off in the last place."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _quantise(x):
    """x [..., dim] fp32 -> whole numbers -7 ... 7 of the same shape and scales [..., dim / 32].  Scales and quotients are
    worked out in 64 bits: a quotient next to a border decides a code."""
    y = x.reshape(*x.shape[:-1], -1, BLOCK).double()
    m, e = torch.frexp(y.abs().amax(dim=-1) / TOP)                       # amax / 7 = m * 2^e, 0.5 <= m < 1
    s = (torch.ceil(m * 32) / 32 * _power_of_two(e)).clamp(SCALE_MIN, SCALE_MAX)
    n = torch.round(y / s[..., None]).clamp(-TOP, TOP)
    return n.reshape(x.shape).to(torch.int8), s.float()


def _dequantise(n, s):
    return (n.reshape(*s.shape, BLOCK).float() * s[..., None]).reshape(n.shape)


def _plain_store(st):
    k, v, case = st["k"], st["v"], st["case"]
    if case["theta"]:
        k = _turned(k, torch.arange(k.shape[1], dtype=torch.float64), case)
    if case["cache"] == "bf16":
        return {"k": k.bfloat16(), "v": v.clone()}
    return {"k": _dequantise(*_quantise(k.float())).bfloat16(), "v": _dequantise(*_quantise(v.float())).bfloat16()}


def _plain_attend(st):
    case = st["case"]
    L, H, D = case["layers"], case["kv_heads"], case["head_dim"]
    G = case["q_heads"] // H
    table, seen, rows = st["table"], st["seen"], st["rows"]       # [R, P], [R, N, P], [R, N]
    R, P = table.shape
    N = seen.shape[1]
    k = _dequantise(st["k"][:, table], st["k_scale"][:, table])
    v = _dequantise(st["v"][:, table], st["v_scale"][:, table])
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
    st["k"], st["k_scale"] = _quantise(k.float())
    st["v"], st["v_scale"] = _quantise(v.float())
    return st


# ---------------------------------------------------------------------------------------------------------------------
# the package's calls
# ---------------------------------------------------------------------------------------------------------------------
def _own_pool(case, n_pages, requests, threads, segments, queries, four_bits=True):
    from paper_2502_11517_b200 import binding
    flags = binding.FLAG_OUT_BF16 | (binding.FLAG_KV_INT4 if four_bits else 0)
    return binding.Pool(case["layers"], case.get("q_heads", case["kv_heads"]), case["kv_heads"], case["head_dim"], n_pages,
                        requests, threads, segments, max_step_queries=queries, flags=flags,
                        device=torch.cuda.current_device())


def _own_form(pool, case):
    pool.set_rope(layout=case["layout"], rotary_dim=case["rotary_dim"], scaling=case["scaling"], factor=case["factor"],
                  original_length=case["original"], low=case["low"], high=case["high"], magnitude=case["magnitude"])


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
    pool, q = st["pool"], st["q"]
    out = torch.empty_like(q)
    pool.decode_attn(q, out)
    return {"out": out}


def _own_store(st):
    pool, k, v, theta = st["pool"], st["k"], st["v"], st["case"]["theta"]
    T = k.shape[1]
    req = pool.request_begin()
    if theta:
        pool.kv_append_run_rope(req, 0, T, k, v, theta)
    else:
        pool.kv_append_run(req, 0, T, k, v)
    k_held, v_held = pool.kv_read_layers(req, 0, 0, T)
    pool.request_end(req)
    return {"k": k_held, "v": v_held}


def _own_rotate_state(case, q):
    """A pool whose requests are as far into their texts as the case says, and the step that feeds the next tokens."""
    n, m = case["requests"], case["tokens"]
    pool = _own_pool(case, n * _pages(m), n, 2, 4, n * m, four_bits=False)
    _own_form(pool, case)
    for r in range(n):
        # a block of that predicted length moves the main thread's next position
        pool.thread_spawn_predicted(pool.request_begin(), case["start"] + 17 * r)
    pool.step_begin(list(range(n)), [0] * n, [m] * n)
    return {"case": case, "pool": pool, "q": q}


def _own_rotate(st):
    out = torch.empty_like(st["q"])
    st["pool"].rope_queries(st["q"], st["case"]["theta"], out=out)
    return {"q": out}


# ---------------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    if case["op"] == "store":
        k, v = _prompt(case, seed)
        st = {"case": case, "k": k, "v": v}
        if own:
            st["pool"] = _own_pool(case, _pages(case["tokens"]), 1, 1, 2, 1, case["cache"] == "4bit")
            _own_form(st["pool"], case)
        return st
    if case["op"] == "rotate":
        q = _queries(case, seed)
        return _own_rotate_state(case, q) if own else {"case": case, "q": q, "positions": _step_positions(case).cuda()}
    lay, k, v, q = _inputs(case, seed)
    return _own_attend_state(case, lay, k, v, q) if own else _plain_state(case, lay, k, v, q)


def run(state):
    op = state["case"]["op"]
    if op == "store":
        return _own_store(state) if own else _plain_store(state)
    if op == "rotate":
        return _own_rotate(state) if own else {"q": _turned(state["q"], state["positions"], state["case"]).bfloat16()}
    return _own_attend(state) if own else _plain_attend(state)


def work(case):
    L, H, D = case["layers"], case["kv_heads"], case["head_dim"]
    code = 0.5 + 2.0 / BLOCK                    # bytes of an element in the cache, its share of a scale included
    if case["op"] == "store":
        values = 2.0 * L * case["tokens"] * H * D
        # keys and values in (bf16), into the cache, and out again (bf16)
        return {"bytes": values * (2 + (code if case["cache"] == "4bit" else 2) + 2), "flops": values * (3 if case["theta"] else 1)}
    if case["op"] == "rotate":
        values = 1.0 * L * case["requests"] * case["tokens"] * case["q_heads"] * D
        return {"bytes": 4 * values, "flops": 3 * values}
    lay = _Layout(case)
    tokens = sum(length for _, _, _, length in lay.streams)
    pairs = sum(n for r in range(len(lay.responses)) for t in range(lay.n_threads[r]) for _, n in lay.visible(r, t))
    rows = L * lay.n_queries * case["q_heads"]
    return {"bytes": 2.0 * L * tokens * H * D * code + rows * D * 4.0, "flops": 4.0 * L * pairs * case["q_heads"] * D}


# ---------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _held(x):
    """What the 4-bit cache holds of x [..., dim] (64 bits): of the numbers 16 ... 31 times a power of two, a block's scale is
    the smallest that is at least a seventh of the block's largest magnitude; elements go to the nearest whole number of
    scales, ties to the even one, at most seven."""
    b = x.unflatten(-1, (-1, BLOCK))
    amax = b.abs().amax(dim=-1, keepdim=True)
    low = torch.frexp(torch.where(amax > 0, amax, torch.ones_like(amax))).exponent - 8      # 7 * 31 * 2^(low + 1) > amax
    two = lambda n: ((n.to(torch.int64) + 1023) << 52).view(torch.float64)
    scale = torch.full_like(amax, float("inf"))
    for up in range(3):
        for m in range(16, 32):
            s = m * two(low + up - 1)
            scale = torch.where((scale == float("inf")) & (amax <= TOP * s), s, scale)
    scale = torch.where(amax > 0, scale, torch.full_like(scale, SCALE_MIN)).clamp(SCALE_MIN, SCALE_MAX)
    y = (b / scale).clamp(-TOP, TOP)
    near = torch.floor(y)
    rest = y - near
    near = near + ((rest > 0.5) | ((rest == 0.5) & (near % 2 != 0))).double()
    return (near * scale).flatten(-2)


def _exact_turn(x, positions, case):
    """The rotation as a product of complex numbers, pair by pair."""
    D = case["head_dim"]
    R = case["rotary_dim"] or D
    out = x.clone()
    factor, original, size = case["factor"], float(case["original"]), 1.0
    log_theta = math.log(case["theta"])
    if case["scaling"] == "base":
        log_theta += math.log(factor) * R / (R - 2)
    if case["scaling"] == "ramp":
        size = case["magnitude"] if case["magnitude"] else 1.0 + 0.1 * math.log(factor)
        first = math.floor(R / 2 * math.log(original / (2 * math.pi * case["high"])) / log_theta)
        last = math.ceil(R / 2 * math.log(original / (2 * math.pi * case["low"])) / log_theta)
        first, last = max(first, 0), min(last, R - 1)
    for i in range(R // 2):
        f = math.exp(-2.0 * i / R * log_theta)
        keep = 1.0                                         # share of the unstretched frequency
        if case["scaling"] == "linear":
            keep = 0.0
        elif case["scaling"] == "wavelength":
            turns = original * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - case["low"]) / (case["high"] - case["low"])))
        elif case["scaling"] == "ramp":
            keep = 1.0 - min(1.0, max(0.0, (i - first) / max(last - first, 0.001)))
        f = f * (keep + (1.0 - keep) / factor)
        a, b = (i, i + R // 2) if case["layout"] == "half" else (2 * i, 2 * i + 1)
        angle = positions.to(x.device) * f
        z = torch.complex(x[..., a], x[..., b]) * torch.polar(torch.full_like(angle, size), angle)[None, :, None]
        out[..., a], out[..., b] = z.real, z.imag
    return out


def _exact_store(case, seed):
    k, v = (x.double() for x in _prompt(case, seed))
    if case["theta"]:
        k = _exact_turn(k, torch.arange(case["tokens"], dtype=torch.float64), case)
    if case["cache"] == "bf16":
        return {"k": k, "v": v}
    return {"k": _held(k.float().double()), "v": _held(v)}     # a rotated key is a 32-bit number before it is quantised


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
                parts = [[_held(x[layer, page : page + _pages(n), :, h].double()).reshape(-1, D) for x in (k, v)]
                         for _, _, page, n in streams]
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
    if case["op"] == "store":
        return _exact_store(case, seed)
    if case["op"] == "rotate":
        return {"q": _exact_turn(_queries(case, seed).double(), _step_positions(case), case)}
    return _exact_attend(case, seed)
