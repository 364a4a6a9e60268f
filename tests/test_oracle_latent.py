"""The fp64 latent attention against other ways of computing it."""
import numpy as np
import pytest
import torch

from oracle import latent as O
from tests import latent_cases as T


def sdpa(q, k, v, scale, mask=None):
    q, k, v = (torch.from_numpy(np.ascontiguousarray(x)).double()[None] for x in (q, k, v))
    return torch.nn.functional.scaled_dot_product_attention(q, k, v, attn_mask=mask, scale=scale)[0].numpy()


def test_decode_is_attention_with_latents_as_values():
    rng = np.random.default_rng(0)
    kv, q = T.rows(rng, 37, 256), T.queries(rng, 1, 5, 256)[0]
    out, mass = O.decode(q, kv, 0.07)
    assert np.allclose(out, sdpa(q, kv, kv[:, :256], 0.07), atol=1e-12)
    assert (mass >= np.abs(out) - 1e-12).all()
    assert (O.decode(q, kv[:0], 0.07)[0] == 0).all()
    one, _ = O.decode(q, kv[:1], 0.07)
    assert np.allclose(one, np.broadcast_to(kv[0, :256], one.shape))


@pytest.mark.parametrize("causal", [True, False])
def test_prefill_is_attention_over_expanded_keys(causal):
    rng = np.random.default_rng(1)
    kv, q = T.rows(rng, 21, 256), rng.standard_normal((6, 3, 192))
    w = rng.standard_normal((2, 3, 128, 256)) / 16
    out, _, _ = O.prefill(q, kv, 15, w[0], w[1], 0.07, causal)
    mask = torch.from_numpy(np.arange(21) <= 15 + np.arange(6)[:, None]) if causal else None
    for h in range(3):
        k, v = O.expand(kv, w[0, h], w[1, h])
        assert np.allclose(out[:, h], sdpa(q[:, h], k, v, 0.07, mask), atol=1e-12)


def test_absorbed_and_expanded_forms_agree():
    rng = np.random.default_rng(2)
    kv, q = T.rows(rng, 50, 512), rng.standard_normal((1, 4, 192))
    w = rng.standard_normal((2, 4, 128, 512)) / 22
    expanded, _, _ = O.prefill(q, kv, 49, w[0], w[1], 0.07, True)
    lat = np.concatenate([np.einsum("hk,hkr->hr", q[0, :, :128], w[0]), q[0, :, 128:]], 1)
    out, _ = O.decode(lat, kv, 0.07)
    assert np.allclose(np.einsum("hr,hvr->hv", out, w[1]), expanded[0], atol=1e-11)


def test_gather_follows_the_page_table():
    pool = np.arange(4 * 2 * 3, dtype=float).reshape(4, 2, 3)
    assert np.array_equal(O.gather(pool, [3, 0, -1], 3), np.concatenate([pool[3], pool[0, :1]]))
    assert O.gather(pool, [1], 0).shape == (0, 3)


def test_bounds_count_their_terms():
    """Weights rounded to bf16 by hand stay inside the bound, a tenth of it would not do."""
    rng = np.random.default_rng(3)
    kv, q = T.rows(rng, 300, 256), T.queries(rng, 1, 8, 256)[0]
    ref, mass = O.decode(q, kv, T.SCALE)
    w = np.exp(T.SCALE * (q @ kv.T))
    p = T.bf16(w)
    got = T.bf16(p @ kv[:, :256] / p.sum(1, keepdims=True))
    bound = T.decode_bound(ref, mass, T.score_error(q, kv, T.SCALE, 320))
    assert (np.abs(got - ref) <= bound).all() and (np.abs(got - ref) > bound / 10).any()
