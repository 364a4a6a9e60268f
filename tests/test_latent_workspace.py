"""One workspace for all chunks of a prompt: a short chunk prefers more heads at a time than a long one, and takes
fewer where the workspace holds no more."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2609_17475_gb300 as jf
from oracle import latent as O
from paper_2609_17475_gb300 import binding as B
from tests import latent_cases as T
from tests.latent_cases import f64, gpu, ints


def need(q_start, C, H, sms=152):
    return B.jf_latent_prefill_workspace_bytes(q_start, C, H, sms)


def test_what_a_call_needs_depends_on_its_last_position_and_grows_with_it():
    rng = np.random.default_rng(1)
    least = 0
    for n in [1, 2, 63, 64, 255, 256, 257, 1000, 4095, 4096, 4097, 32768, 1 << 20]:
        one = {need(n - C, C, 1) for C in {1, n, *rng.integers(1, n + 1, 5).tolist()}}
        assert len(one) == 1 and min(one) >= least
        least = max(one)
        for H in (1, 16, 128, 1024):
            assert all(need(n - C, C, H) >= least for C in (1, min(n, 50), n))


def test_short_last_chunks_prefer_more():
    """What makes sharing a workspace more than a matter of its size."""
    assert need(4046, 50, 128) > need(0, 4096, 128) and need(32668, 100, 128) > need(24576, 8192, 128)


def test_a_workspace_that_does_not_hold_a_head_is_refused():
    p, f = B._Pool(0x10000, 8, 64, 1, 576, 64, B.JF_FMT_LATENT16), ctypes.c_void_p(0x20000)
    for start, C, H in ((0, 16, 4), (1000, 1, 128)):
        least = B.jf_latent_prefill_workspace_bytes(start, C, 1, 0)
        assert B.lib().jf_latent_prefill_attn(ctypes.byref(p), f, f, start, C, H, f, f, 0.1, 1, f, f, least - 1, None) == \
            B.JF_ERR_WORKSPACE_TOO_SMALL


@pytest.mark.gpu
@pytest.mark.parametrize("H,chunks,first", [(128, [2000, 1500, 500, 37, 1], 0), (40, [3000, 300, 7], 1), (24, [600, 50], 1)])
def test_one_workspace_for_a_prompts_chunks(H, chunks, first):
    """Sized by the longest chunk at the prompt's end, or for one head alone, with bytes past it that stay as they
    are; outputs as with a workspace of their own."""
    rng = np.random.default_rng(H)
    R, n = 256, sum(chunks)
    table, pool = T.filled(rng, R, 64, [n])
    kv, g = O.gather(pool, table[0], n), T.gpu_pool(pool)
    w = T.bf16(rng.standard_normal((2, H, 128, R)) / np.sqrt(1.65 * R))
    wk, wv, row = gpu(w[0]), gpu(w[1]), ints(table[0])
    size = jf.jf_latent_prefill_workspace_bytes(n - chunks[0], chunks[0], 1 if first else H)
    raw = torch.full((size + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    ws = raw[:size]
    ws[:256] = 0
    at = 0
    for C in chunks:
        q = T.bf16(rng.standard_normal((C, H, 192)))
        outs = []
        for space in (ws, jf.latent_prefill_workspace(at, C, H)):
            out = torch.full((C, H, 128), float("nan"), device="cuda").bfloat16()
            jf.jf_latent_prefill_attn(g, row, gpu(q), at, wk, wv, T.SCALE, True, out, space)
            assert jf.workspace_status(space) == 0
            outs.append(f64(out))
        assert (raw[size:] == 0x5A).all()
        # the same sums in another division: two bf16 roundings, and values and weights of 2^-11 each
        for h in range(0, H, 7):
            ref, mass, _ = O.prefill(q[:, h:h + 1], kv[:at + C], at, w[0][h:h + 1], w[1][h:h + 1], T.SCALE, True)
            for got in outs:
                assert np.linalg.norm(got[:, h:h + 1] - ref) <= 0.004 * np.linalg.norm(ref)
            assert (np.abs(outs[0][:, h] - outs[1][:, h]) <= 2.0 ** -7 * np.abs(ref[:, 0]) + 2.0 ** -9 * mass[:, 0]).all()
        at += C
