"""Latent attention over a paged cache: keys and values of all heads come from one latent vector a token.

A position holds c (R channels) and r (64 rotated key channels, shared by all heads), bf16, as one row of R + 64 values; a
page is a run of rows.  Three attentions read it:

* decode, the absorbed form: a head's query is (q_lat [R], q_rot [64]); s_t = scale (q_lat . c_t + q_rot . r_t), the output
  sum_t softmax(s)_t c_t.
* prefix: the same for groups of requests whose first positions are one shared run of pages, each request's own
  positions after them.
* prefill, the expanded form: k_t = (W_k c_t, r_t), v_t = W_v c_t with 128 + 64 and 128 channels a head, causal.

Each case names one operator and its sizes; ``run`` computes it in plain torch operations, or, where ``own`` is true,
through the framework's entry points.
"""
import math

import torch

own = False

ROT = 64            # rotated key channels of a position
NOPE = 128          # a head's other key channels, and its value channels, in the expanded form
SCALE = 1 / math.sqrt(NOPE + ROT)


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------
def listed():
    return [
        # the append of one decode step of 32 requests, read back: the launches' latency
        dict(name="append_step_32", op="append", batch=32, lo=1025, hi=65535, rows=1, r=512, page=256),
        # a 2,048-row prompt chunk after an odd number of positions
        dict(name="append_chunk_2048", op="append", batch=1, lo=30725, hi=30725, rows=2048, r=512, page=256),
        # single-token attention at the benchmark's smallest context
        dict(name="decode_4096", op="decode", batch=1, lo=4096, hi=4096, empty=False, h=16, r=512, page=256),
        # a small latent, an odd number of heads, short ragged contexts
        dict(name="decode_ragged_5", op="decode", batch=5, lo=1, hi=3001, empty=True, h=20, r=256, page=64),
        # a mixed batch of 32 requests, one of them without a position yet
        dict(name="decode_mixed_32", op="decode", batch=32, lo=1025, hi=65535, empty=True, h=16, r=512, page=64),
        # one long request with all heads on this GPU: bytes and products weigh the same
        dict(name="decode_128k_heads_128", op="decode", batch=1, lo=131072, hi=131072, empty=False, h=128, r=512, page=256),
        # two prompts, a few continuations of each, all heads
        dict(name="prefix_2x4_heads_128", op="prefix", groups="4,4", prefix="4001,7000", lo=1, hi=300, h=128, r=512,
             page=128),
        # 64 continuations of one long prompt, some of them just begun
        dict(name="prefix_64", op="prefix", groups="64", prefix="32768", lo=0, hi=2047, h=16, r=512, page=256),
        # a short last chunk after an odd prefix
        dict(name="prefill_77", op="prefill", q_start=4001, chunk=77, h=16, r=512, page=128),
        # a prompt's chunk of 2,048 queries after 30,720 positions
        dict(name="prefill_2048", op="prefill", q_start=30720, chunk=2048, h=16, r=512, page=256),
        # a whole prompt of odd length, all heads
        dict(name="prefill_whole_4095", op="prefill", q_start=0, chunk=4095, h=128, r=512, page=256),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "decode", "decode", "prefix", "prefix", "prefill", "prefill"])
    r, page = rng.choice([256, 512]), rng.choice([64, 128, 256])
    if op == "append":
        batch = _log(rng, 1, 64)
        return dict(op="append", batch=batch, lo=_log(rng, 1, 1000), hi=_log(rng, 1001, 32768),
                    rows=_log(rng, 1, max(1, 2048 // batch)), r=r, page=page)
    if op == "decode":
        batch, h = rng.choice([1, 1, 2, 5, 16, 33]), rng.choice([1, 5, 8, 16, 20, 40, 64, 100, 128])
        # no more work than the long request's
        hi = _log(rng, 64, min(131072, 131072 * 128 // (batch * h), 65535 * 8 // batch))
        return dict(op="decode", batch=batch, lo=max(1, hi // rng.choice([1, 3, 20])), hi=hi,
                    empty=batch > 1 and rng.random() < 0.5, h=h, r=r, page=page)
    if op == "prefix":
        h = rng.choice([4, 8, 16, 20, 64, 128])
        groups = [_log(rng, 1, 64) for _ in range(rng.choice([1, 1, 2, 3]))]
        top = max(64, min(32768, 64 * 16 * 32768 // (sum(groups) * h)))
        return dict(op="prefix", groups=",".join(map(str, groups)),
                    prefix=",".join(str(_log(rng, 32, top)) for _ in groups), lo=rng.choice([0, 1]), hi=_log(rng, 1, min(2047, 64 * 2047 // sum(groups))), h=h, r=r,
                    page=page)
    h = rng.choice([1, 4, 16])
    return dict(op="prefill", q_start=rng.choice([0, _log(rng, 1, 30720)]), chunk=_log(rng, 1, 2000), h=h, r=r, page=page)


def _counts(text):
    return [int(x) for x in text.split(",")]


def _lens(case):
    """Lengths spread evenly over the logarithm of [lo, hi] (the first one lo itself, which may be 0)."""
    n = sum(_counts(case["groups"])) if case["op"] == "prefix" else case["batch"]
    lo, hi = max(1, case["lo"]), case["hi"]
    lens = [int(round(lo * (hi / lo) ** (i / (n - 1)))) if n > 1 else hi for i in range(n)]
    if case["lo"] == 0:
        lens[0] = 0
    if case.get("empty"):
        lens[1] = 0
    return lens


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _rows(g, n, gain):
    """n positions [n, R + 64]: normalised latents under their channels' gains, and rotated keys."""
    c = torch.randn(n, len(gain), generator=g, device="cuda") * gain
    return torch.cat([c, torch.randn(n, ROT, generator=g, device="cuda")], 1).bfloat16()


def _tables(g, need):
    """Page tables [B, max] of distinct pages in no order (-1 past a request's pages), and the pool's pages."""
    total = max(1, sum(need))
    perm = torch.randperm(total, generator=g, device="cuda").int()
    table = torch.full((len(need), max(max(need), 1)), -1, dtype=torch.int32, device="cuda")
    off = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[off:off + n]
        off += n
    return table, total


def _fill(g, pool, table, lens, gain, page):
    """lens[b] random positions of each request into its pages."""
    for b, n in enumerate(lens):
        if n:
            t = torch.arange(n, device="cuda")
            pool[table[b, t // page].long(), t % page] = _rows(g, n, gain)


def prepare(case, seed):
    g, c = _gen(seed), dict(case)
    r, page = c["r"], c["page"]
    if c["op"] == "prefix":
        c["groups"], c["prefix"] = _counts(c["groups"]), _counts(c["prefix"])
    d = r + ROT
    s = {"c": c, "own": {}}
    gain = torch.exp(0.5 * torch.randn(r, generator=g, device="cuda"))

    def pool_of(pages):   # slots that hold no position keep stale bytes
        stale = torch.randint(0, 256, (pages, page * d * 2), dtype=torch.uint8, device="cuda", generator=g)
        return stale, stale.view(torch.bfloat16).view(pages, page, d)

    if c["op"] == "append":
        start, n = _lens(c), c["rows"]
        s["table"], pages = _tables(g, [-(-(m + n) // page) for m in start])
        s["bytes"], s["pool"] = pool_of(pages)
        total = len(start) * n
        # the latent and the key part are slices of one projection's output, as a layer leaves them
        s["rows"] = _rows(g, total, gain)
        s["latent"], s["rot"] = s["rows"][:, :r], s["rows"][:, r:]
        s["start"], s["offsets"] = _ints(start), _ints([i * n for i in range(len(start) + 1)])
        req = torch.arange(len(start), device="cuda").repeat_interleave(n)
        s["pos"] = s["start"].long()[req] + torch.arange(total, device="cuda") % n
        s["req"] = req
        s["out"] = torch.zeros(total, r, dtype=torch.bfloat16, device="cuda")
        s["out_rot"] = torch.zeros(total, ROT, dtype=torch.bfloat16, device="cuda")
        s["err"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        return s
    if c["op"] == "prefill":
        n = c["q_start"] + c["chunk"]
        s["table"], pages = _tables(g, [-(-n // page)])
        s["bytes"], s["pool"] = pool_of(pages)
        _fill(g, s["pool"], s["table"], [n], gain, page)
        s["q"] = torch.randn(c["chunk"], c["h"], NOPE + ROT, generator=g, device="cuda").bfloat16()
        w = torch.randn(2, c["h"], NOPE, r, generator=g, device="cuda") / math.sqrt(1.65 * r)
        s["w_k"], s["w_v"] = w[0].bfloat16(), w[1].bfloat16()
        s["out"] = torch.zeros(c["chunk"], c["h"], NOPE, dtype=torch.bfloat16, device="cuda")
        return s
    lens = _lens(case)
    shared = c["prefix"] if c["op"] == "prefix" else []
    table, pages = _tables(g, [-(-n // page) for n in shared + lens])
    s["bytes"], s["pool"] = pool_of(pages)
    _fill(g, s["pool"], table, shared + lens, gain, page)
    s["prefix_table"], s["table"] = table[:len(shared)].contiguous(), table[len(shared):].contiguous()
    s["prefix_lens"], s["ctx"] = _ints(shared), _ints(lens)
    s["lens"] = lens
    s["offsets"] = [sum(c["groups"][:i]) for i in range(len(shared) + 1)] if shared else None
    # absorbed queries: W_k^T q of a query of 128 channels
    q = torch.randn(len(lens), c["h"], d, generator=g, device="cuda")
    q[..., :r] *= math.sqrt(NOPE / (1.65 * r))
    s["q"] = q.bfloat16()
    s["out"] = torch.zeros(len(lens), c["h"], r, dtype=torch.bfloat16, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def run(state):
    op = state["c"]["op"]
    if own:
        return {"append": _own_append, "decode": _own_decode, "prefix": _own_prefix, "prefill": _own_prefill}[op](state)
    return {"append": _append, "decode": _decode, "prefix": _prefix, "prefill": _prefill}[op](state)


def _positions(s, table_row, n):
    """Positions 0 .. n - 1 of a request as rows in 32 bits [n, R + 64]."""
    pages = -(-n // s["c"]["page"])
    return s["pool"][table_row[:pages].long()].flatten(0, 1)[:n].float()


def _softmax(x):
    w = torch.exp(x - x.amax(-1, keepdim=True))
    return w / w.sum(-1, keepdim=True)


def _append(s):
    c = s["c"]
    page = s["table"][s["req"], s["pos"] // c["page"]].long()
    s["pool"][page, s["pos"] % c["page"]] = torch.cat([s["latent"], s["rot"]], 1)
    x = s["pool"][page, s["pos"] % c["page"]]
    return {"latent": x[:, :c["r"]].contiguous(), "rot": x[:, c["r"]:].contiguous()}


def _attend(q, kv, r):
    """q [rows, R + 64] over positions kv [n, R + 64], in 32 bits."""
    return _softmax(q @ kv.t() * SCALE) @ kv[:, :r]


def _decode(s):
    r = s["c"]["r"]
    out = torch.zeros(s["out"].shape, device="cuda")
    for b, n in enumerate(s["lens"]):
        if n:
            out[b] = _attend(s["q"][b].float(), _positions(s, s["table"][b], n), r)
    return {"out": out.bfloat16()}


def _prefix(s):
    c, r = s["c"], s["c"]["r"]
    out = torch.zeros(s["out"].shape, device="cuda")
    for g, n in enumerate(c["prefix"]):
        shared = _positions(s, s["prefix_table"][g], n)
        for b in range(s["offsets"][g], s["offsets"][g + 1]):
            kv = torch.cat([shared, _positions(s, s["table"][b], s["lens"][b])])
            out[b] = _attend(s["q"][b].float(), kv, r)
    return {"out": out.bfloat16()}


def _prefill(s):
    c, r = s["c"], s["c"]["r"]
    n = c["q_start"] + c["chunk"]
    kv = _positions(s, s["table"][0], n)
    seen = torch.arange(n, device="cuda") <= c["q_start"] + torch.arange(c["chunk"], device="cuda")[:, None]
    out = torch.empty(s["out"].shape, dtype=s["out"].dtype, device="cuda")
    for h in range(c["h"]):
        q = s["q"][:, h].float()
        k = torch.cat([kv[:, :r] @ s["w_k"][h].float().t(), kv[:, r:]], 1)
        v = kv[:, :r] @ s["w_v"][h].float().t()
        x = (q @ k.t()).mul_(SCALE).masked_fill_(~seen, -math.inf)
        out[:, h] = (_softmax(x) @ v).bfloat16()
    return {"out": out}


def _handles(s):
    """What a user's program makes once: the pool's handle and a workspace."""
    import paper_2609_17475_gb300 as jf
    h, c = s["own"], s["c"]
    if not h:
        h["pool"] = jf.KVPool(s["bytes"], c["page"], 1, c["r"] + ROT, format=jf.JF_FMT_LATENT16)
        if c["op"] == "decode":
            h["ws"] = jf.latent_decode_workspace(c["batch"], c["h"], c["r"])
        elif c["op"] == "prefix":
            h["ws"] = jf.latent_decode_workspace(sum(c["groups"]), c["h"], c["r"], num_groups=len(c["groups"]))
        elif c["op"] == "prefill":
            h["ws"] = jf.latent_prefill_workspace(c["q_start"], c["chunk"], c["h"])
    return jf, h


def _own_append(s):
    jf, h = _handles(s)
    jf.jf_latent_append(h["pool"], s["table"], s["start"], s["offsets"], s["latent"], s["rot"], s["err"])
    jf.jf_latent_read(h["pool"], s["table"], s["start"], s["offsets"], s["out"], s["out_rot"], s["err"])
    return {"latent": s["out"], "rot": s["out_rot"]}


def _own_decode(s):
    jf, h = _handles(s)
    jf.jf_latent_decode_attn(h["pool"], s["table"], s["ctx"], s["q"], SCALE, s["out"], h["ws"])
    return {"out": s["out"]}


def _own_prefix(s):
    jf, h = _handles(s)
    jf.jf_latent_prefix_decode_attn(h["pool"], s["prefix_table"], s["prefix_lens"], s["offsets"], s["table"], s["ctx"],
                                    s["q"], SCALE, s["out"], h["ws"])
    return {"out": s["out"]}


def _own_prefill(s):
    jf, h = _handles(s)
    jf.jf_latent_prefill_attn(h["pool"], s["table"][0], s["q"], s["c"]["q_start"], s["w_k"], s["w_v"], SCALE, True, s["out"],
                              h["ws"])
    return {"out": s["out"]}


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------
def work(case):
    c = case
    r = c["r"]
    row = 2 * (r + ROT)                                      # bytes of a position
    if c["op"] == "append":
        return {"bytes": 4 * c["batch"] * c["rows"] * row, "flops": 0}       # rows in, into the pool, out of it and back
    if c["op"] == "prefill":
        n, h = c["q_start"] + c["chunk"], c["h"]
        pairs = c["chunk"] * c["q_start"] + c["chunk"] * (c["chunk"] + 1) // 2
        expanded = 2 * n * r * 2 * NOPE * h + 2 * pairs * h * (2 * NOPE + ROT)
        absorbed = 2 * c["chunk"] * r * 2 * NOPE * h + 2 * pairs * h * (2 * r + ROT)
        return {"bytes": n * row + 2 * c["chunk"] * h * (2 * NOPE + ROT) + 4 * h * NOPE * r, "flops": min(expanded, absorbed)}
    lens = _lens(c)
    heads = len(lens) * c["h"]
    if c["op"] == "decode":
        held, seen = sum(lens), sum(lens)
    else:
        prefix = _counts(c["prefix"])
        held = sum(prefix) + sum(lens)
        seen = sum(n * p for n, p in zip(_counts(c["groups"]), prefix)) + sum(lens)
    return {"bytes": held * row + heads * (row + 2 * r), "flops": 2 * seen * c["h"] * (2 * r + ROT)}


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits, apart from the plain forms
# ---------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    c, r, page = s["c"], case["r"], case["page"]
    if c["op"] == "append":
        return {"latent": s["latent"].double().contiguous(), "rot": s["rot"].double().contiguous()}

    def at(table_row, first, last):   # positions first .. last - 1
        t = torch.arange(first, last, device="cuda")
        return s["pool"][table_row[t // page].long(), t % page].double()

    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    if c["op"] == "prefill":
        kv = at(s["table"][0], 0, c["q_start"] + c["chunk"])
        lat, rot = kv[:, :r], kv[:, r:]
        step = 512
        for h in range(c["h"]):
            w_k, w_v = s["w_k"][h].double(), s["w_v"][h].double()
            k, v = lat @ w_k.t(), lat @ w_v.t()
            for i in range(0, c["chunk"], step):
                q = s["q"][i:i + step, h].double()
                last = c["q_start"] + i + len(q)             # positions that any of these queries sees
                x = (q[:, :NOPE] @ k[:last].t() + q[:, NOPE:] @ rot[:last].t()) / math.sqrt(NOPE + ROT)
                own_last = torch.arange(last - len(q), last, device="cuda")[:, None]
                x[torch.arange(last, device="cuda") > own_last] = -math.inf
                out[i:i + step, h] = torch.softmax(x, -1) @ v[:last]
        return {"out": out}
    for b, n in enumerate(s["lens"]):
        runs = [(s["table"][b], n)]
        if c["op"] == "prefix":
            g = max(i for i, o in enumerate(s["offsets"]) if o <= b)
            runs.insert(0, (s["prefix_table"][g], c["prefix"][g]))
        # the runs' softmax sums joined under their common maximum
        q = s["q"][b].double()
        top = torch.full((c["h"], 1), -math.inf, dtype=torch.float64, device="cuda")
        num, den = torch.zeros(c["h"], r, dtype=torch.float64, device="cuda"), torch.zeros_like(top)
        for row, m in runs:
            for i in range(0, m, 16384):
                kv = at(row, i, min(m, i + 16384))
                x = (q[:, :r] @ kv[:, :r].t() + q[:, r:] @ kv[:, r:].t()) / math.sqrt(NOPE + ROT)
                new = torch.maximum(top, x.amax(1, keepdim=True))
                w = torch.exp(x - new)
                num = num * torch.exp(top - new) + w @ kv[:, :r]
                den = den * torch.exp(top - new) + w.sum(1, keepdim=True)
                top = new
        if any(m for _, m in runs):
            out[b] = num / den
    return {"out": out}
