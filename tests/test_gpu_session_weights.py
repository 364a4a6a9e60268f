"""The session example's first cut goes by the prompt's last queries, not by one generated token's."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

from oracle import kv8 as O

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
spec = importlib.util.spec_from_file_location("long_session", os.path.join(ROOT, "examples", "long_session.py"))
E = importlib.util.module_from_spec(spec)
spec.loader.exec_module(E)


def test_a_prompts_last_queries_add_up_weights():
    """observe(): what the prompt's last queries draw, each from the positions up to its own."""
    hq, hkv, d, page, n, last = 6, 2, 128, 64, 300, 20
    g = torch.Generator(device="cuda").manual_seed(8)
    draw = lambda h: torch.randn(n, h, d, generator=g, device="cuda").bfloat16()  # noqa: E731
    s = E.Session(hq, hkv, d, page, max_positions=320, budget=128, recent=16)
    q = draw(hq)
    s.prompt(q, draw(hkv), draw(hkv), E.positions(n, 8).cuda())
    assert not s.weights.any()
    L = O.Layout(hkv, page, d)
    k, v = O.read(s.pool.data.cpu().numpy(), L, s.table[0].tolist(), n)
    scale = float(np.float32(1 / math.sqrt(d)))
    _, w, _ = O.attend(k, v, q[-last:].double().cpu().numpy(), scale, n - last + 1 + np.arange(last))
    want = w.sum(0).reshape(hkv, hq // hkv, n).sum(1)
    for times in (1, 2):
        s.observe(q[-last:])
        # a weight: 2^-20 for its exponential, row sum and score (|score| < 2^5 in fp32), and fp32 sums of 60 of them
        got = s.weights[0, :, :n].double().cpu().numpy()
        assert (np.abs(got - times * want) <= times * want * (2.0 ** -16) + 2.0 ** -30).all()
    assert not s.weights[0, :, n:].any() and s.status() == 0


def test_the_run_cuts_by_them():
    """In a run the weights before the first generated token are those of a window of queries."""
    seen = []
    step = E.Session.step

    def spy(self, *a):
        seen.append(float(self.weights.sum()))
        return step(self, *a)
    E.Session.step = spy
    try:
        E.run(prompt=700, tokens=2, budget=512, chunk=256, hq=8, hkv=2, d=128, page=64, verbose=False)
    finally:
        E.Session.step = step
    assert abs(seen[0] - 8 * 64) < 1e-2          # 64 queries of 8 heads, a weight of one each
