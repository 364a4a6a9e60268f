"""The session example: rotary axes, append, chunked attention, weighed steps and eviction used together."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

from oracle import kv8 as O
from oracle import rope as R
from tests import kv8_cases as C

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
spec = importlib.util.spec_from_file_location("long_session", os.path.join(ROOT, "examples", "long_session.py"))
E = importlib.util.module_from_spec(spec)
spec.loader.exec_module(E)


def test_session_equals_the_oracles():
    """A prompt in two chunks and six steps: pool bytes and outputs against the oracles' rotation, cache and
    attention.  The rotated rows are taken from the GPU (they round to bf16) after they are checked themselves."""
    hq, hkv, d, page = 6, 2, 128, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    draw = lambda n, h: torch.randn(n, h, d, generator=g, device="cuda").bfloat16()  # noqa: E731
    s = E.Session(hq, hkv, d, page, max_positions=320, budget=128, recent=16)
    pos = E.positions(206, 8).cuda()
    L, pool = O.Layout(hkv, page, d), None
    pool = O.new_pool(L, s.pool.num_pages)
    done, scale = 0, float(np.float32(1 / math.sqrt(d)))
    for n in (130, 70, 1, 1, 1, 1, 1, 1):
        q, k, v = draw(n, hq), draw(n, hkv), draw(n, hkv)
        p = pos[:, done:done + n]
        want = [R.rotate(x.double().cpu().numpy(), p.cpu().numpy(), s.rope.axis, s.rope.inv_freq, "half") for x in (q, k)]
        out = (s.prompt if n > 1 else s.step)(q, k, v, p)        # q and k are turned in place
        for x, w in zip((q, k), want):
            err = np.abs(x.double().cpu().numpy() - w)
            assert (err <= np.abs(w) * 2.0 ** -8 + 8 * 2.0 ** -21).all()
        q64, k64, v64 = (x.double().cpu().numpy() for x in (q, k, v))
        O.append(pool, L, s.table.cpu().numpy(), [done], [0, n], k64, v64)
        done += n
        assert np.array_equal(s.pool.data.cpu().numpy(), pool)
        kk, vv = O.read(pool, L, s.table[0].tolist(), done)
        ref, w, mass = O.attend(kk, vv, q64, scale, done - n + 1 + np.arange(n))
        got = out.double().cpu().numpy()
        for h in range(hq):
            slack = 2.0 ** -10 * (np.abs(q64[:, h]) @ np.abs(kk[:, h // 3]).T * scale).max(-1)[:, None]
            bound = C.out_bound(ref[:, h], mass[:, h], done, np.abs(vv).max()) + mass[:, h] * slack + 2.0 ** -12
            assert (np.abs(got[:, h] - ref[:, h]) <= bound).all()
    assert s.status() == 0
    # six steps' weights: each adds up to the query heads of its KV head
    total = s.weights[0, :, :done].double().sum(-1)
    assert (total - 6 * 3).abs().max() < 1e-3 and not s.weights[0, :, done:].any()


def test_session_evicts_and_gives_pages_back():
    s, out = E.run(prompt=700, tokens=600, budget=512, chunk=256, hq=8, hkv=2, d=128, page=64, verbose=False)
    assert torch.isfinite(out.float()).all() and out.shape == (600, 8, 128)
    assert 512 <= s.length <= 512 + 256 and len(s.pages) == -(-s.length // 64)
    assert sorted(s.pages + s.free) == list(range(s.pool.num_pages))      # no page lost or held twice
    before = s.length
    kept = s.evict()
    assert s.length == 512 and kept.shape == (2, 512)
    k = kept.cpu().numpy()
    assert (np.diff(k, axis=1) > 0).all() and (k[:, :4] == np.arange(4)).all()
    assert (k[:, -64:] == np.arange(before - 64, before)).all() and s.status() == 0
