"""The operators of a long image-and-text session over an 8-bit paged KV cache: rotary positions with
several axes, append to and attention over the cache, and eviction by accumulated attention weight.

Each case names one operator and its sizes; ``run`` computes it in plain torch operations, or, where
``own`` is true, through the framework's entry points.

The cache: a pool of page records, each [K codes: Hkv x P x D bytes][V codes: same]
[K scales: Hkv x P/32 fp32][V scales: same].  A code is an e4m3 value; the scale of a block of 32 positions of
a KV head is a power of two 2^e, e the smallest exponent with (largest magnitude of the block) <= 448 * 2^e,
limited to [-40, 40].  A block that gets more rows keeps the larger of its scale and theirs, its earlier
codes rounded again under it.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 32          # positions that share a scale
E_MIN, E_MAX = -40, 40


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------
def listed():
    return [
        # rotary positions of one decode step of 32 requests (24 query heads, 4 KV heads): the launch's latency
        dict(name="rope_step_32", op="rope", tokens=32, hq=24, hkv=4, d=256, rot=64, axes=3, layout="interleaved",
             pairing="half", inverse=False, dtype="bf16"),
        # a prefill chunk of an image prompt, every channel rotated
        dict(name="rope_chunk_2048", op="rope", tokens=2048, hq=24, hkv=4, d=256, rot=256, axes=3, layout="sectioned",
             pairing="half", inverse=False, dtype="bf16"),
        # the gradient of a training batch's queries and keys, an odd count of tokens, adjacent pairs, fp16
        dict(name="rope_grad_16391", op="rope", tokens=16391, hq=16, hkv=4, d=128, rot=128, axes=3, layout="interleaved",
             pairing="adjacent", inverse=True, dtype="fp16"),
        # the append of one decode step of 32 requests, each somewhere inside a block
        dict(name="append_step_32", op="append", batch=32, lo=1025, hi=65535, rows=1, hkv=4, d=256, page=256),
        # the append of a 2,048-row prompt chunk that starts inside a block
        dict(name="append_chunk_2048", op="append", batch=1, lo=30725, hi=30725, rows=2048, hkv=4, d=256, page=256),
        # single-token attention: the smallest context of the benchmark, on its small head shape
        dict(name="decode_4096", op="decode", batch=1, lo=4096, hi=4096, empty=False, hq=8, hkv=2, d=128, page=256,
             weights=False),
        # one request at its full window
        dict(name="decode_256k", op="decode", batch=1, lo=262144, hi=262144, empty=False, hq=24, hkv=4, d=256, page=256,
             weights=False),
        # a mixed batch of 32 requests, one of them without a position yet, weights added up for eviction
        dict(name="decode_mixed_32_weights", op="decode", batch=32, lo=1025, hi=65535, empty=True, hq=24, hkv=4, d=256,
             page=64, weights=True),
        # a prompt's chunk of 2,048 queries after 30,720 positions
        dict(name="prefill_2048", op="prefill", q_start=30720, chunk=2048, hq=24, hkv=4, d=256, page=256),
        # a short last chunk after an odd prefix, small head shape
        dict(name="prefill_77", op="prefill", q_start=4001, chunk=77, hq=8, hkv=2, d=128, page=128),
        # a batch of mid-length requests cut to a budget, some of them below it
        dict(name="evict_8", op="evict", batch=8, lo=1500, hi=16383, budget=2048, sinks=4, recent=256, hkv=4, d=128,
             page=128),
        # one request at its full window cut to an eighth
        dict(name="evict_256k", op="evict", batch=1, lo=262144, hi=262144, budget=32768, sinks=4, recent=1024, hkv=4,
             d=256, page=256),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "decode", "decode", "prefill", "evict"])
    d = rng.choice([128, 256])
    if op == "rope":
        # the largest costs no more than the gradient case: tokens * heads * d
        hkv = rng.choice([1, 2, 4, 8])
        hq = hkv * rng.choice([1, 2, 4, 6])
        top = max(2, min(16391, 16391 * 20 * 128 // ((hq + hkv) * d)))
        return dict(op="rope", tokens=_log(rng, 1, top), hq=hq, hkv=hkv, d=d, rot=rng.choice([32, 64, 96, d]),
                    axes=rng.choice([1, 2, 3]), layout=rng.choice(["sectioned", "interleaved"]),
                    pairing=rng.choice(["half", "adjacent"]), inverse=rng.random() < 0.5,
                    dtype=rng.choice(["bf16", "fp16"]))
    hkv = rng.choice([1, 2, 4])
    hq = hkv * rng.choice([1, 2, 4, 6, 8])
    page = rng.choice([64, 128, 256])
    if op == "append":
        batch = _log(rng, 1, 64)
        return dict(op="append", batch=batch, lo=_log(rng, 1, 1000), hi=_log(rng, 1001, 32768),
                    rows=_log(rng, 1, max(1, 2048 // batch)), hkv=hkv, d=d, page=page)
    if op == "decode":
        batch = rng.choice([1, 1, 2, 5, 16, 33])
        hi = _log(rng, 64, 262144 if batch == 1 else 65535 * 4 // batch)
        return dict(op="decode", batch=batch, lo=max(1, hi // rng.choice([1, 3, 20])), hi=hi,
                    empty=batch > 1 and rng.random() < 0.5, hq=hq, hkv=hkv, d=d, page=page, weights=rng.random() < 0.5)
    if op == "prefill":
        return dict(op="prefill", q_start=rng.choice([0, _log(rng, 1, 30720)]), chunk=_log(rng, 1, 2000), hq=hq, hkv=hkv,
                    d=d, page=page)
    batch = rng.choice([1, 2, 7])
    hi = _log(rng, 600, 262144 // batch)
    budget = max(64, hi // rng.choice([2, 5, 9]))
    return dict(op="evict", batch=batch, lo=max(1, hi // rng.choice([1, 4, 12])), hi=hi, budget=budget,
                sinks=rng.choice([0, 4, 17]), recent=rng.choice([0, 1, budget // 3]), hkv=hkv, d=d, page=page)


def _lens(case):
    """Context lengths spread evenly over the logarithm of [lo, hi]."""
    n, lo, hi = case["batch"], case["lo"], case["hi"]
    lens = [int(round(lo * (hi / lo) ** (i / (n - 1)))) if n > 1 else hi for i in range(n)]
    if case.get("empty"):
        lens[1] = 0
    return lens


# ---------------------------------------------------------------------------------------------
# the 8-bit block format in plain operations
# ---------------------------------------------------------------------------------------------
def _exponent(amax):
    """Smallest e with amax <= 448 * 2^e, limited to [E_MIN, E_MAX]."""
    m, e = torch.frexp(amax)                       # amax = m * 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.where(amax > 0, e, torch.full_like(e, E_MIN)).clamp(E_MIN, E_MAX)


def _two(e):
    """2^e as fp32, exactly, for integers e of a normal number's range."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _round8(x, e):
    """x rounded to e4m3 under the exponents e (broadcast), as values."""
    return (x * _two(-e)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).float() * _two(e)


def _record(pool, c):
    """Views of a pool's page records: codes [pages, 2, Hkv, P, D] (uint8) and scales [pages, 2, Hkv, P / 32]."""
    n, at = pool.shape[0], 2 * c["hkv"] * c["page"] * c["d"]
    codes = pool[:, :at].view(n, 2, c["hkv"], c["page"], c["d"])
    scales = pool[:, at:].view(torch.float32).view(n, 2, c["hkv"], c["page"] // BLOCK)
    return codes, scales


def _values(pool, table, c):
    """K and V of the pages of `table` [B, pages] as fp32 values [B, Hkv, pages * P, D] each."""
    codes, scales = _record(pool, c)
    b, n = table.shape
    at = table.long().clamp(min=0).reshape(-1)
    x = codes[at].view(torch.float8_e4m3fn).float().view(b, n, 2, c["hkv"], c["page"] // BLOCK, BLOCK, c["d"])
    x = x * scales[at].view(b, n, 2, c["hkv"], c["page"] // BLOCK, 1, 1)
    x = x.permute(2, 0, 3, 1, 4, 5, 6).reshape(2, b, c["hkv"], n * c["page"], c["d"])
    return x[0], x[1]


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _kv(g, n, c):
    """n rows of K (four channels of each head 20 times the others) and V, bf16 [n, Hkv, D]."""
    k = torch.randn(n, c["hkv"], c["d"], generator=g, device="cuda")
    v = torch.randn(n, c["hkv"], c["d"], generator=g, device="cuda")
    big = torch.rand(c["hkv"], c["d"], generator=g, device="cuda").argsort(-1) < 4
    k = torch.where(big, k * 20, k)
    return k.bfloat16(), v.bfloat16()


def _tables(g, need, spare=0):
    """Page tables [B, max] of distinct pages in no order (-1 past a request's pages), and the pool's pages."""
    total = sum(need) + spare
    perm = torch.randperm(total, generator=g, device="cuda").int()
    table = torch.full((len(need), max(max(need), 1)), -1, dtype=torch.int32, device="cuda")
    off = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[off:off + n]
        off += n
    return table, total


def _pool(g, c, lens, table, pages):
    """A pool that holds lens[b] random positions of each request; slots that hold none keep stale bytes."""
    hkv, p, d = c["hkv"], c["page"], c["d"]
    size = 2 * hkv * (p * d + 4 * (p // BLOCK))
    pool = torch.randint(0, 256, (pages, size), dtype=torch.uint8, device="cuda", generator=g)
    codes, scales = _record(pool, c)
    for b, n in enumerate(lens):
        if n == 0:
            continue
        k, v = _kv(g, n, c)
        x = torch.stack([k, v]).float()                                            # [2, n, Hkv, D]
        full = -(-n // p)
        pad = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, full * p - n))
        blocks = pad.view(2, full, p // BLOCK, BLOCK, hkv, d)
        e = _exponent(blocks.abs().amax((3, 5)))                                   # [2, full, P / 32, Hkv]
        y = (blocks * _two(-e)[:, :, :, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        y = y.view(2, full, p, hkv, d).permute(1, 0, 3, 2, 4)                      # [full, 2, Hkv, P, D]
        at = table[b, :full].long()
        if n % p:
            y, r = y.contiguous(), n % p
            y[-1, :, :, r:] = codes[at[-1], :, :, r:]
        codes[at] = y
        sc = _two(e).permute(1, 0, 3, 2)
        if n % p:
            sc, r = sc.contiguous(), -(-(n % p) // BLOCK)
            sc[-1, :, :, r:] = scales[at[-1], :, :, r:]
        scales[at] = sc
    return pool


def _pairs(c):
    """The axis of each rotated pair and its frequency."""
    half = c["rot"] // 2
    if c["axes"] == 1:
        sections = [half]
    elif c["axes"] == 2:
        sections = [half - half // 2, half // 2]
    else:
        sections = [half - 2 * (3 * half // 8), 3 * half // 8, 3 * half // 8]
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    if c["layout"] == "interleaved":
        n = len(sections)
        axis = [i % n if i < n * sections[i % n] else 0 for i in range(half)]
    freq = (1e7 ** (-np.arange(half, dtype=np.float64) / half)).astype(np.float32)
    return sections, axis, freq


def prepare(case, seed):
    g, c = _gen(seed), dict(case)
    s = {"c": c, "own": {}}
    d = c["d"]
    if c["op"] == "rope":
        n, dt = c["tokens"], torch.bfloat16 if c["dtype"] == "bf16" else torch.float16
        s["sections"], axis, freq = _pairs(c)
        s["axis"] = torch.tensor(axis, device="cuda")
        s["freq"] = torch.from_numpy(freq).cuda()
        # text runs at one place on every axis, image patches spread over height and width
        t = torch.randint(0, 30000, (1, n), generator=g, device="cuda")
        hw = torch.randint(0, 96, (2, n), generator=g, device="cuda")
        image = torch.rand(n, generator=g, device="cuda") < 0.5
        s["pos"] = torch.cat([t, t + torch.where(image, hw, 0)])[:c["axes"]].int().contiguous()
        # queries and keys lie in one fused projection, as a model's layer leaves them
        qk = torch.randn(n, c["hq"] + c["hkv"], d, generator=g, device="cuda").to(dt)
        s["q"], s["k"] = qk[:, :c["hq"]], qk[:, c["hq"]:]
        s["q_out"] = torch.zeros(n, c["hq"], d, dtype=dt, device="cuda")
        s["k_out"] = torch.zeros(n, c["hkv"], d, dtype=dt, device="cuda")
        return s
    p, hkv = c["page"], c["hkv"]
    s["err"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if c["op"] == "append":
        start, r = _lens(c), c["rows"]
        s["table"], pages = _tables(g, [-(-(n + r) // p) for n in start])
        s["pool"] = _pool(g, c, start, s["table"], pages)
        s["k"], s["v"] = _kv(g, len(start) * r, c)
        # some rows larger than what their block holds
        grow = 1 + 7 * (torch.rand(len(start) * r, 1, 1, generator=g, device="cuda") < 0.2)
        s["k"], s["v"] = s["k"] * grow.bfloat16(), s["v"] * grow.bfloat16()
        first = [n // BLOCK * BLOCK for n in start]
        size = [n + r - f for n, f in zip(start, first)]
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        s["start"], s["rows"] = ints(start), ints([i * r for i in range(len(start) + 1)])
        s["first"], s["size"] = ints(first), ints(np.concatenate([[0], np.cumsum(size)]).tolist())
        # places of the touched blocks' positions: (request, position), and which of them are new rows
        req = np.repeat(np.arange(len(start)), size)
        pos = np.concatenate([np.arange(f, n + r) for f, n in zip(first, start)])
        row = np.where(pos >= np.array(start)[req], pos - np.array(start)[req] + req * r, -1)
        blocks = np.concatenate([[0], np.cumsum([-(-z // BLOCK) for z in size])])
        s["req"], s["pos"], s["row"] = (torch.from_numpy(x).cuda() for x in (req, pos, row))
        s["block"] = torch.from_numpy((pos - np.array(first)[req]) // BLOCK + blocks[req]).cuda()
        s["blocks"] = int(blocks[-1])
        s["k_out"] = torch.zeros(len(pos), hkv, d, dtype=torch.bfloat16, device="cuda")
        s["v_out"] = torch.zeros_like(s["k_out"])
        return s
    if c["op"] == "prefill":
        n = c["q_start"] + c["chunk"]
        s["table"], pages = _tables(g, [-(-n // p)])
        s["pool"] = _pool(g, c, [n], s["table"], pages)
        s["q"] = torch.randn(c["chunk"], c["hq"], d, generator=g, device="cuda").bfloat16()
        s["out"] = torch.zeros_like(s["q"])
        return s
    lens = _lens(c)
    s["ctx"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["top"] = max(lens)
    if c["op"] == "decode":
        s["table"], pages = _tables(g, [-(-n // p) for n in lens])
        s["pool"] = _pool(g, c, lens, s["table"], max(pages, 1))
        s["q"] = torch.randn(len(lens), c["hq"], d, generator=g, device="cuda").bfloat16()
        s["out"] = torch.zeros_like(s["q"])
        if c["weights"]:
            s["w"] = torch.rand(len(lens), hkv, s["top"], generator=g, device="cuda") / 64
            s["w_out"] = torch.zeros_like(s["w"])
        return s
    keep = [min(n, c["budget"]) for n in lens]
    need = [-(-n // p) for n in lens] + [-(-n // p) for n in keep]
    table, pages = _tables(g, need)
    s["table"], s["dst"] = table[:len(lens)].contiguous(), table[len(lens):, :-(-max(keep) // p)].contiguous()
    s["pool"] = _pool(g, c, lens, s["table"], pages)
    # weights as they add up over a session: most positions near nothing, some never seen at all
    w = torch.exp(2.0 * torch.randn(len(lens), hkv, s["top"], generator=g, device="cuda")) / 64
    s["w"] = torch.where(torch.rand(w.shape, generator=g, device="cuda") < 0.3, torch.zeros_like(w), w)
    s["w_out"] = torch.zeros(len(lens), hkv, c["budget"], device="cuda")
    s["kept"] = torch.zeros(len(lens), hkv, c["budget"], dtype=torch.int32, device="cuda")
    s["ctx_out"] = torch.zeros_like(s["ctx"])
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    s["first"], s["size"] = ints([0] * len(keep)), ints(np.concatenate([[0], np.cumsum(keep)]).tolist())
    s["flat"] = torch.from_numpy(np.concatenate([b * c["budget"] + np.arange(n) for b, n in enumerate(keep)])).cuda()
    s["k_out"] = torch.zeros(sum(keep), hkv, d, dtype=torch.bfloat16, device="cuda")
    s["v_out"] = torch.zeros_like(s["k_out"])
    return s


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def run(state):
    op = state["c"]["op"]
    if own:
        return {"rope": _own_rope, "append": _own_append, "decode": _own_decode, "prefill": _own_prefill,
                "evict": _own_evict}[op](state)
    return {"rope": _rope, "append": _append, "decode": _decode, "prefill": _prefill, "evict": _evict}[op](state)


def _rotate(x, cos, sin, c):
    rot = c["rot"]
    x = x.float()
    r, rest = x[..., :rot], x[..., rot:]
    if c["pairing"] == "half":
        a, b = r[..., :rot // 2], r[..., rot // 2:]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([y, rest], -1)


def _rope(s):
    c = s["c"]
    angle = s["pos"].float()[s["axis"]].t() * s["freq"]            # [tokens, rot / 2]
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    sin = -sin if c["inverse"] else sin
    return {"q": _rotate(s["q"], cos, sin, c).to(s["q"].dtype), "k": _rotate(s["k"], cos, sin, c).to(s["k"].dtype)}


def _append(s):
    c = s["c"]
    codes, scales = _record(s["pool"], c)
    page = s["table"][s["req"], s["pos"] // c["page"]].long()
    slot = s["pos"] % c["page"]
    old = codes[page, :, :, slot].view(torch.float8_e4m3fn).float()                 # [n, 2, Hkv, D]
    es = scales[page, :, :, slot // BLOCK]                                          # [n, 2, Hkv]
    new = torch.stack([s["k"], s["v"]], 1).float()[s["row"].clamp(min=0)]
    is_new = (s["row"] >= 0)[:, None, None]
    e_old = torch.frexp(es)[1] - 1
    old = old * es[..., None]
    x = torch.where(is_new[..., None], new, old)
    e = torch.where(is_new, _exponent(new.abs().amax(-1)), e_old)
    top = torch.full((s["blocks"], 2, c["hkv"]), E_MIN, dtype=e.dtype, device=e.device)
    top = top.scatter_reduce(0, s["block"][:, None, None].expand_as(e), e, "amax")
    y = _round8(x, top[s["block"]][..., None]).bfloat16()
    return {"k": y[:, 0], "v": y[:, 1]}


def _softmax(x):
    """Weights of the last axis, 0 where a row has nothing (-inf throughout)."""
    m = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    n = x.sum(-1, keepdim=True)
    return x / torch.where(n > 0, n, torch.ones_like(n))


def _decode(s):
    c = s["c"]
    k, v = _values(s["pool"], s["table"], c)
    seen = torch.arange(k.shape[2], device="cuda") < s["ctx"][:, None]              # [B, T]
    v = torch.where(seen[:, None, :, None], v, torch.zeros_like(v))
    q = s["q"].float().view(-1, c["hkv"], c["hq"] // c["hkv"], c["d"])
    x = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(c["d"])
    w = _softmax(torch.where(seen[:, None, None], x, torch.full_like(x, -math.inf)))
    out = torch.matmul(w, v).reshape(s["q"].shape).bfloat16()
    if not c["weights"]:
        return {"out": out}
    t = s["top"]
    return {"out": out, "weights": torch.where(seen[:, None, :t], s["w"] + w.sum(2)[..., :t], torch.zeros_like(s["w"]))}


def _prefill(s):
    c = s["c"]
    n, grp = c["q_start"] + c["chunk"], c["hq"] // c["hkv"]
    k, v = _values(s["pool"], s["table"], c)
    k, v = k[0, :, :n], v[0, :, :n]                                                 # [Hkv, T, D]
    q = s["q"].float().view(c["chunk"], c["hkv"], grp, c["d"]).permute(1, 2, 0, 3)  # [Hkv, G, C, D]
    x = torch.matmul(q, k[:, None].transpose(-1, -2)) / math.sqrt(c["d"])
    seen = torch.arange(n, device="cuda") <= c["q_start"] + torch.arange(c["chunk"], device="cuda")[:, None]
    w = _softmax(torch.where(seen, x, torch.full_like(x, -math.inf)))
    out = torch.matmul(w, v[:, None]).permute(2, 0, 1, 3).reshape(s["q"].shape)
    return {"out": out.bfloat16()}


def _evict(s):
    c = s["c"]
    n, budget = s["top"], c["budget"]
    t = torch.arange(n, device="cuda")
    ctx = s["ctx"][:, None, None]
    safe = (t < c["sinks"]) | (t >= ctx - c["recent"])
    key = torch.where(safe, torch.full_like(s["w"], math.inf), s["w"])
    key = torch.where(t < ctx, key, torch.full_like(key, -math.inf))
    first = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :budget]
    keep = torch.clamp(ctx, max=budget)
    j = torch.arange(budget, device="cuda")
    if first.shape[-1] < budget:
        first = torch.nn.functional.pad(first, (0, budget - first.shape[-1]))
    at = torch.where(j < keep, first, torch.full_like(first, n)).sort(-1).values
    live = at < n
    pos = torch.where(live, at, torch.zeros_like(at))                               # [B, Hkv, budget]
    codes, scales = _record(s["pool"], c)
    b = torch.arange(pos.shape[0], device="cuda")[:, None, None]
    h = torch.arange(c["hkv"], device="cuda")[None, :, None]
    page, slot = s["table"][b, pos // c["page"]].long(), pos % c["page"]
    page = torch.where(live, page, torch.zeros_like(page))
    x = codes[page, :, h, slot].view(torch.float8_e4m3fn).float() * scales[page, :, h, slot // BLOCK][..., None]
    x = torch.where(live[..., None, None], x, torch.zeros_like(x))                  # [B, Hkv, budget, 2, D]
    x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, -budget % BLOCK))
    blocks = x.view(*x.shape[:2], -1, BLOCK, 2, c["d"])
    e = _exponent(blocks.abs().amax((3, 5)))
    y = _round8(blocks, e[:, :, :, None, :, None]).view(x.shape)[:, :, :budget].bfloat16()
    y = y.permute(0, 2, 3, 1, 4).reshape(-1, 2, c["hkv"], c["d"])[s["flat"]]
    w = torch.where(live, torch.gather(s["w"], 2, pos), torch.zeros_like(s["w"][..., :1]))
    return {"kept": torch.where(live, at, torch.full_like(at, -1)).int(), "weights": w, "ctx": keep[:, 0, 0].int(),
            "k": y[:, 0], "v": y[:, 1]}


def _handles(s):
    """What a user's program makes once: the pool's and the rotary embedding's handles, workspaces, split counts."""
    import paper_2609_17475_gb300 as jf
    h, c = s["own"], s["c"]
    if h:
        return jf, h
    if c["op"] == "rope":
        h["rope"] = jf.Rope(c["rot"], s["sections"], base=1e7, layout=c["layout"], pairing=c["pairing"])
        return jf, h
    h["pool"] = jf.KVPool(s["pool"], c["page"], c["hkv"], c["d"], format=jf.JF_FMT_E4M3_B32)
    if c["op"] == "decode":
        n = h["splits"] = jf.default_num_splits(c["batch"], c["hkv"], format=jf.JF_FMT_E4M3_B32)
        h["ws"] = (jf.decode_weights_workspace(c["batch"], c["hq"], c["hkv"], c["d"], n, s["top"]) if c["weights"]
                   else jf.decode_workspace(c["batch"], c["hq"], c["hkv"], c["d"], n))
    elif c["op"] == "prefill":
        n = h["splits"] = jf.default_prefill_splits([c["q_start"]], [c["chunk"]], c["hq"], c["hkv"])
        # a long chunk balances its waves by itself, a short one spreads its history
        h["one"] = c["chunk"] >= 1024
        h["ws"] = (jf.prefill_chunk_workspace(h["pool"], c["q_start"], c["chunk"], c["hq"]) if h["one"]
                   else jf.prefill_batch_workspace(c["chunk"], c["hq"], c["d"], n, format=jf.JF_FMT_E4M3_B32))
    return jf, h


def _own_rope(s):
    jf, h = _handles(s)
    jf.jf_rope_axes(h["rope"], s["pos"], s["q"], s["q_out"], s["k"], s["k_out"], inverse=s["c"]["inverse"])
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_append(s):
    jf, h = _handles(s)
    jf.jf_kv8_append(h["pool"], s["table"], s["start"], s["rows"], s["k"], s["v"], s["err"])
    jf.jf_kv8_read(h["pool"], s["table"], s["first"], s["size"], s["k_out"], s["v_out"], s["err"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_decode(s):
    jf, h = _handles(s)
    scale = 1 / math.sqrt(s["c"]["d"])
    if not s["c"]["weights"]:
        jf.jf_paged_decode_attn(h["pool"], s["table"], s["ctx"], s["q"], scale, s["out"], h["ws"], h["splits"])
        return {"out": s["out"]}
    jf.jf_paged_decode_weights_attn(h["pool"], s["table"], s["ctx"], s["q"], scale, s["out"], s["w"], s["w_out"], h["ws"],
                                    h["splits"])
    return {"out": s["out"], "weights": s["w_out"]}


def _own_prefill(s):
    jf, h = _handles(s)
    c = s["c"]
    scale = 1 / math.sqrt(c["d"])
    if h["one"]:
        jf.jf_prefill_chunk_attn(h["pool"], s["table"][0], s["q"], c["q_start"], scale, True, s["out"], h["ws"])
    else:
        jf.jf_prefill_batch_attn(h["pool"], s["table"], [c["q_start"]], [c["chunk"]], s["q"], scale, True, s["out"],
                                 h["ws"], h["splits"])
    return {"out": s["out"]}


def _own_evict(s):
    jf, h = _handles(s)
    c = s["c"]
    jf.jf_kv8_evict(h["pool"], s["table"], s["ctx"], s["w"], c["budget"], c["sinks"], c["recent"], s["dst"], s["ctx_out"],
                    s["w_out"], s["kept"], s["err"])
    jf.jf_kv8_read(h["pool"], s["dst"], s["first"], s["size"], s["k_out"], s["v_out"], s["err"])
    return {"kept": s["kept"], "weights": s["w_out"], "ctx": s["ctx_out"], "k": s["k_out"], "v": s["v_out"]}


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------
def work(case):
    c = case
    d = c["d"]
    if c["op"] == "rope":
        n = c["tokens"] * (c["hq"] + c["hkv"])
        return {"bytes": 4 * n * d + 4 * c["axes"] * c["tokens"], "flops": 3 * n * c["rot"]}
    row = c["hkv"] * d                                     # elements of a K or V row
    if c["op"] == "append":
        n = c["batch"] * c["rows"]
        back = sum(m % BLOCK for m in _lens(c)) + n        # positions whose values come back
        return {"bytes": n * row * 2 * (2 + 1) + back * row * 2 * 2, "flops": 4 * n * row}
    if c["op"] == "prefill":
        n = c["q_start"] + c["chunk"]
        pairs = c["chunk"] * c["q_start"] + c["chunk"] * (c["chunk"] + 1) // 2
        return {"bytes": 2 * n * row + 4 * c["chunk"] * c["hq"] * d, "flops": 4 * pairs * c["hq"] * d}
    lens = _lens(c)
    if c["op"] == "decode":
        more = 8 * c["hkv"] * sum(lens) if c["weights"] else 0
        scales = 2 * 4 * c["hkv"] * sum(-(-n // BLOCK) for n in lens)
        return {"bytes": 2 * row * sum(lens) + scales + 4 * c["batch"] * c["hq"] * d + more,
                "flops": 4 * c["hq"] * d * sum(lens)}
    keep = sum(min(n, c["budget"]) for n in lens)
    # weights once, each kept position's codes once in and once out, its values back, its index and weight
    return {"bytes": 4 * c["hkv"] * sum(lens) + keep * row * 2 * (1 + 1 + 2) + 8 * c["hkv"] * keep,
            "flops": c["hkv"] * sum(lens) + 4 * keep * row}


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits, apart from the plain forms
# ---------------------------------------------------------------------------------------------
def _e4m3_table():
    """The 256 values of e4m3: sign, 4 exponent bits (bias 7), 3 mantissa bits; S.1111.111 is not a number."""
    b = np.arange(256)
    ex, man = (b >> 3) & 15, b & 7
    x = np.where(ex == 0, man / 8 * 2.0 ** -6, (1 + man / 8) * 2.0 ** (ex.astype(np.float64) - 7))
    x = np.where((b & 127) == 127, np.nan, x)
    return torch.from_numpy(np.where(b >= 128, -x, x)).cuda()


def _request64(s, b, n):
    """K and V [2, n, Hkv, D] of request b's first n positions in 64 bits."""
    c = s["c"]
    codes, scales = _record(s["pool"], c)
    pages = -(-n // c["page"])
    at = s["table"][b, :pages].long()
    x = _e4m3_table()[codes[at].int()]                                             # [pages, 2, Hkv, P, D]
    x = x * scales[at].double().repeat_interleave(BLOCK, -1)[..., None]
    return x.permute(1, 0, 3, 2, 4).reshape(2, pages * c["page"], c["hkv"], c["d"])[:, :n]


def _two64(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exponent64(x):
    """Least e of [E_MIN, E_MAX] with all of x (over the first and the last axis) <= 448 * 2^e."""
    amax = x.abs().amax(0).amax(-1)
    powers = _two64(torch.arange(E_MIN, E_MAX, device="cuda"))
    return E_MIN + (amax[..., None] > 448 * powers).sum(-1)


def _block64(x, extra=None):
    """x [n <= 32, ...] rounded to e4m3 under one power of two for all but the last axis and the rows; `extra`: the least
    exponent it may have."""
    e = _exponent64(x)
    if extra is not None:
        e = torch.maximum(e, extra)
    two = _two64(e)[..., None]
    y = (x / two).clamp(-448, 448)
    step = torch.full_like(y, 2.0 ** -9)                                            # of the least normal numbers and below
    for k in range(-5, 9):
        step = torch.where(y.abs() >= 2.0 ** k, torch.full_like(y, 2.0 ** (k - 3)), step)
    return torch.round(y / step) * step * two


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["op"] == "rope":
        turn = s["pos"].double()[s["axis"].tolist()] * s["freq"].double()[:, None]  # [pairs, tokens]
        if c["inverse"]:
            turn = -turn
        z = torch.polar(torch.ones_like(turn), turn).t()[:, None]
        out = {}
        for name in ("q", "k"):
            x = s[name].double().clone()
            half = c["rot"] // 2
            i = torch.arange(half, device="cuda")
            a, b = (i, i + half) if c["pairing"] == "half" else (2 * i, 2 * i + 1)
            y = torch.complex(x[..., a], x[..., b]) * z
            x[..., a], x[..., b] = y.real, y.imag
            out[name] = x
        return out
    if c["op"] == "append":
        codes, scales = _record(s["pool"], c)
        ks, vs = [], []
        start, r = _lens(c), c["rows"]
        for b, n in enumerate(start):
            new = torch.stack([s["k"], s["v"]], 1).double()[b * r:(b + 1) * r]      # [r, 2, Hkv, D]
            f = n // BLOCK * BLOCK
            if n > f:
                old = _request64(s, b, n)[:, f:].permute(1, 0, 2, 3)
                page = int(s["table"][b, f // c["page"]])
                had = torch.log2(scales[page, :, :, f % c["page"] // BLOCK].double()).round().long()
                x = torch.cat([old, new])
            else:
                x, had = new, None
            for i in range(0, len(x), BLOCK):
                part = x[i:i + BLOCK]
                fresh = part[n - f:] if i == 0 else part
                low = None
                if i == 0 and had is not None:
                    # the rows that were there do not lower the scale, nor raise it
                    low = torch.maximum(had, _exponent64(fresh))
                y = _block64(part, low)
                ks.append(y[:, 0])
                vs.append(y[:, 1])
        return {"k": torch.cat(ks), "v": torch.cat(vs)}
    grp = c.get("hq", c["hkv"]) // c["hkv"]
    if c["op"] == "prefill":
        n = c["q_start"] + c["chunk"]
        kv = _request64(s, 0, n)
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        last = c["q_start"] + torch.arange(c["chunk"], device="cuda")
        for h in range(c["hq"]):
            x = s["q"][:, h].double() @ kv[0, :, h // grp].t() / math.sqrt(c["d"])
            x.masked_fill_(torch.arange(n, device="cuda") > last[:, None], -math.inf)
            out[:, h] = torch.softmax(x, -1) @ kv[1, :, h // grp]
        return {"out": out}
    if c["op"] == "decode":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        w = torch.zeros(len(out), c["hkv"], s["top"], dtype=torch.float64, device="cuda")
        for b, n in enumerate(_lens(c)):
            if n == 0:
                continue
            kv = _request64(s, b, n)
            for h in range(c["hq"]):
                p = torch.softmax(kv[0, :, h // grp] @ s["q"][b, h].double() / math.sqrt(c["d"]), 0)
                out[b, h] = p @ kv[1, :, h // grp]
                w[b, h // grp, :n] += p
            if c["weights"]:
                w[b, :, :n] += s["w"][b, :, :n].double()
        return {"out": out, "weights": w} if c["weights"] else {"out": out}
    # eviction: each head's kept places by weight in falling order, equal weights in rising order of place
    ks, vs = [], []
    kept = torch.zeros(c["batch"], c["hkv"], c["budget"], dtype=torch.float64, device="cuda")
    weights = s["w"].double().cpu().numpy()
    for b, n in enumerate(_lens(c)):
        m = min(n, c["budget"])
        kv = _request64(s, b, n)
        rows = []
        for h in range(c["hkv"]):
            t = np.arange(n)
            safe = (t < c["sinks"]) | (t >= n - c["recent"])
            best = np.lexsort((t, -weights[b, h, :n], ~safe))[:m]
            at = torch.from_numpy(np.sort(best)).cuda()
            kept[b, h, :m] = s["w"][b, h, at].double()
            rows.append(kv[:, at, h])
        x = torch.stack(rows, 2).permute(1, 0, 2, 3)                                # [m, 2, Hkv, D]
        y = torch.cat([_block64(x[i:i + BLOCK]) for i in range(0, m, BLOCK)])
        ks.append(y[:, 0])
        vs.append(y[:, 1])
    return {"kept": None, "weights": kept, "ctx": None, "k": torch.cat(ks), "v": torch.cat(vs)}
