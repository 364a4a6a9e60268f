"""A long image-and-text session through one attention layer with an 8-bit cache.

The layer's queries, keys and values are drawn at random; everything between them and the layer's output runs
through the library: a prompt of text and image patches is turned by its time, height and width positions, appended
to the paged cache and attended in chunks, and the attention weights that its last queries draw are added up; then
tokens are generated one at a time, their weights are added too, and whenever the cache has grown past its budget the
positions that drew the least weight are evicted and their pages given back.

    python examples/long_session.py --prompt 8192 --tokens 512 --budget 4096
"""
import argparse
import math
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2609_17475_gb300 as jf  # noqa: E402


def positions(n, image_side, start=0):
    """int32 [3, n] time, height and width of n tokens: text, and an image of image_side^2 patches in every 1,024
    tokens, whose patches share a time and spread over height and width."""
    t = torch.arange(start, start + n)
    p = t[None].repeat(3, 1)
    at = t % 1024
    image = at < image_side * image_side
    base = t - at
    p[0] = torch.where(image, base, t)
    p[1] = torch.where(image, base + at // image_side, t)
    p[2] = torch.where(image, base + at % image_side, t)
    return p.int()


class Session:
    """One request's cache: its pool, its page table, its weights, and the calls that use them."""

    def __init__(self, hq=24, hkv=4, d=256, page=256, max_positions=16384, budget=4096, sinks=4, recent=512,
                 device="cuda"):
        self.hq, self.hkv, self.d, self.page = hq, hkv, d, page
        self.budget, self.sinks, self.recent = budget, sinks, recent
        pages = -(-max_positions // page) + -(-budget // page)
        self.pool = jf.KVPool.allocate(pages, page, hkv, d, device=device, format=jf.JF_FMT_E4M3_B32)
        self.free = list(range(pages))
        self.pages = []
        self.table = torch.full((1, pages), -1, dtype=torch.int32, device=device)
        # a quarter of each head's channels is rotated, three axes interleaved
        r = d // 4
        side = 3 * (r // 2) // 8
        self.rope = jf.Rope(r, [r // 2 - 2 * side, side, side], base=1e7, layout="interleaved")
        self.length = 0          # positions in the cache
        self.seen = 0            # tokens so far: the next token's place in time
        self.weights = torch.zeros(1, hkv, max_positions, device=device)
        self.splits = jf.default_num_splits(1, hkv, format=jf.JF_FMT_E4M3_B32)
        self.ws = jf.decode_weights_workspace(1, hq, hkv, d, self.splits, max_positions, device=device)
        self.err = torch.zeros(1, dtype=torch.int32, device=device)
        self.device = device

    def _ints(self, *x):
        return torch.tensor(x, dtype=torch.int32, device=self.device)

    def _reserve(self, length):
        while len(self.pages) * self.page < length:
            self.pages.append(self.free.pop())
            self.table[0, len(self.pages) - 1] = self.pages[-1]

    def extend(self, q, k, v, pos):
        """Turns and appends n tokens' rows: q [n, Hq, D], k and v [n, Hkv, D] bf16, pos [3, n]."""
        n = q.shape[0]
        self._reserve(self.length + n)
        jf.jf_rope_axes(self.rope, pos, q, None, k, None)
        jf.jf_kv8_append(self.pool, self.table, self._ints(self.length), self._ints(0, n), k, v, self.err)
        self.length += n
        self.seen += n

    def prompt(self, q, k, v, pos):
        """One chunk of the prompt: its attention output [n, Hq, D]."""
        self.extend(q, k, v, pos)
        n, out = q.shape[0], torch.empty_like(q)
        ws = jf.prefill_chunk_workspace(self.pool, self.length - n, n, self.hq, device=self.device)
        jf.jf_prefill_chunk_attn(self.pool, self.table[0], q, self.length - n, 1 / math.sqrt(self.d), True, out, ws)
        return out

    def observe(self, q):
        """Adds up the weights that the last n positions' queries draw, q [n, Hq, D] as `prompt` has turned them: a
        batch of n single-token calls over one request's pages, each up to its own position."""
        n = q.shape[0]
        ctx = torch.arange(self.length - n + 1, self.length + 1, dtype=torch.int32, device=self.device)
        table = self.table.repeat(n, 1)
        weights = torch.zeros(n, self.hkv, self.length, device=self.device)
        splits = jf.default_num_splits(n, self.hkv, format=jf.JF_FMT_E4M3_B32)
        ws = jf.decode_weights_workspace(n, self.hq, self.hkv, self.d, splits, self.length, device=self.device)
        jf.jf_paged_decode_weights_attn(self.pool, table, ctx, q, 1 / math.sqrt(self.d), torch.empty_like(q), None, weights,
                                        ws, splits)
        self.weights[0, :, :self.length] += weights.sum(0)
        self.err |= ws[:4].view(torch.int32)

    def step(self, q, k, v, pos):
        """One generated token: its attention output [1, Hq, D]; its weights are added up."""
        self.extend(q, k, v, pos)
        out = torch.empty_like(q)
        jf.jf_paged_decode_weights_attn(self.pool, self.table, self._ints(self.length), q, 1 / math.sqrt(self.d), out,
                                        self.weights, self.weights, self.ws, self.splits)
        return out

    def evict(self):
        """Keeps `budget` positions; the old pages are free again.  Returns the kept positions [Hkv, budget]."""
        n = min(self.length, self.budget)
        fresh = [self.free.pop() for _ in range(-(-n // self.page))]
        dst = self._ints(*fresh).view(1, -1)
        kept = torch.empty(1, self.hkv, self.budget, dtype=torch.int32, device=self.device)
        weights = torch.empty(1, self.hkv, self.budget, device=self.device)
        length = self._ints(0)
        jf.jf_kv8_evict(self.pool, self.table, self._ints(self.length), self.weights, self.budget, self.sinks,
                        self.recent, dst, length, weights, kept, self.err)
        self.weights.zero_()
        self.weights[:, :, :self.budget] = weights
        self.free += self.pages
        self.pages = fresh
        self.table.fill_(-1)
        self.table[0, :len(fresh)] = dst[0]
        self.length = n
        return kept[0]

    def status(self):
        return int(self.err.item()) | jf.workspace_status(self.ws)


def run(prompt=8192, tokens=512, budget=4096, chunk=2048, hq=24, hkv=4, d=256, page=256, seed=0, verbose=True, window=64):
    g = torch.Generator(device="cuda").manual_seed(seed)
    draw = lambda n, h: torch.randn(n, h, d, generator=g, device="cuda").bfloat16()  # noqa: E731
    slack = 256     # the cache grows this far past its budget before it is cut
    s = Session(hq, hkv, d, page, max(prompt, budget + slack) + tokens, budget, recent=budget // 8)
    pos = positions(prompt + tokens, 16).cuda()
    torch.cuda.synchronize()
    t = time.perf_counter()
    for at in range(0, prompt, chunk):
        n = min(chunk, prompt - at)
        q = draw(n, hq)
        s.prompt(q, draw(n, hkv), draw(n, hkv), pos[:, at:at + n])
    if prompt:
        s.observe(q[-window:])
    torch.cuda.synchronize()
    t_prompt, cuts = time.perf_counter() - t, 0
    t = time.perf_counter()
    outs = []
    for i in range(tokens):
        at = prompt + i
        outs.append(s.step(draw(1, hq), draw(1, hkv), draw(1, hkv), pos[:, at:at + 1]))
        if s.length > budget + slack:
            s.evict()
            cuts += 1
    torch.cuda.synchronize()
    t_tokens = time.perf_counter() - t
    if s.status():
        raise RuntimeError(f"device status {s.status()}")
    if verbose:
        print(f"prompt of {prompt} positions: {1e3 * t_prompt:.1f} ms; {tokens} tokens: {1e6 * t_tokens / tokens:.0f} us "
              f"each; {cuts} evictions; {s.length} positions left in {len(s.pages)} pages")
    return s, torch.cat(outs)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--prompt", type=int, default=8192)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--budget", type=int, default=4096)
    a = ap.parse_args()
    run(a.prompt, a.tokens, a.budget)
