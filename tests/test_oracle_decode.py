"""Pins of the decode oracle: reductions to the block oracle on contiguous prompts, closed forms, brute force."""
import numpy as np
import pytest

from oracle import zo_block as ob
from oracle import zo_decode as od


def _cache(rng, lens, g, P, dh, extra=2):
    pages = [-(-n // P) for n in lens]
    n_pages, width = sum(pages) + extra, max(max(pages), 1)
    perm = rng.permutation(n_pages)
    table = np.full((len(lens), width), -1, np.int32)
    at = 0
    for i, n in enumerate(pages):
        table[i, :n] = perm[at:at + n]
        at += n
    return rng.normal(size=(n_pages, g, P, dh)), rng.normal(size=(n_pages, g, P, dh)), table


@pytest.mark.parametrize("H,g,dh,P", [(4, 2, 16, 16), (3, 3, 8, 4), (6, 1, 10, 2)])
def test_prompt_through_the_cache_is_packed_attention(H, g, dh, P):
    rng = np.random.default_rng(H * 100 + dh)
    lens = [5, 0, 1, 19]
    cu = np.concatenate([[0], np.cumsum(lens)])
    T = cu[-1]
    q, k, v = (rng.normal(size=(T, n * dh)) for n in (H, g, g))
    gq, gk = 1 + 0.1 * rng.normal(size=dh), 1 + 0.1 * rng.normal(size=dh)
    K, V, table = _cache(rng, lens, g, P, dh)
    before = K.copy()
    q2, K, V = od.cache_append(q, k, v, cu, H, gq, gk, 1e-6, 1e4, K, V, table, lens)
    qr, kr = ob.qk_norm_rope(q, k, cu, H, g, dh, gq, gk, 1e-6, 1e4)
    np.testing.assert_allclose(q2, qr, rtol=1e-12, atol=1e-12)
    o = od.attention_paged(q2, cu, H, 0.3, K, V, table, lens)
    np.testing.assert_allclose(o, ob.attention(qr, kr, v, cu, H, g, dh, 0.3), rtol=1e-10, atol=1e-12)
    used = np.zeros(K.shape[0], bool)
    used[table[table >= 0]] = True
    assert (K[~used] == before[~used]).all()          # pages of no sequence stay as they were
    last = table[3, 18 // P]
    assert (K[last, :, 18 % P + 1:] == before[last, :, 18 % P + 1:]).all()


def test_token_by_token_is_the_whole_prompt():
    rng = np.random.default_rng(5)
    H, g, dh, P, n = 4, 2, 8, 4, 11
    q, k, v = (rng.normal(size=(n, m * dh)) for m in (H, g, g))
    K, V, table = _cache(rng, [n], g, P, dh)
    whole, Kw, Vw = od.cache_append(q, k, v, [0, n], H, None, None, 0.0, 1e4, K, V, table, [n])
    o = od.attention_paged(whole, [0, n], H, 0.5, Kw, Vw, table, [n])
    for t in range(n):
        qt, K, V = od.cache_append(q[t:t + 1], k[t:t + 1], v[t:t + 1], [0, 1], H, None, None, 0.0, 1e4, K, V, table, [t + 1])
        np.testing.assert_allclose(qt[0], whole[t], rtol=1e-12)
        np.testing.assert_allclose(od.attention_paged(qt, [0, 1], H, 0.5, K, V, table, [t + 1])[0], o[t], rtol=1e-12)
    assert (K == Kw).all() and (V == Vw).all()


def test_pages_outside_the_pool_are_not_seen():
    rng = np.random.default_rng(6)
    K, V, table = _cache(rng, [12], 1, 4, 6)
    q = rng.normal(size=(1, 6))
    table[0, 1] = 99
    o = od.attention_paged(q, [0, 1], 1, 1.0, K, V, table, [12])
    keep = np.concatenate([K[table[0, 0], 0], K[table[0, 2], 0]]), np.concatenate([V[table[0, 0], 0], V[table[0, 2], 0]])
    p = np.exp(keep[0] @ q[0])
    np.testing.assert_allclose(o[0], p @ keep[1] / p.sum(), rtol=1e-12)
    assert (od.attention_paged(q, [0, 1], 1, 1.0, K, V, np.full_like(table, -1), [12]) == 0).all()
    assert (od.attention_paged(q, [0, 1], 1, 1.0, K, V, table, [0]) == 0).all()


def test_filters_keep_what_their_definitions_say():
    z = np.log(np.array([0.1, 0.4, 0.05, 0.25, 0.2]))          # probabilities at temperature 1
    kept = lambda k=0, p=1.0, m=0.0, t=1.0: list(od.kept_tokens(z, t, k, p, m)[0])
    assert kept() == [1, 3, 4, 0, 2]
    assert kept(k=2) == [1, 3] and kept(k=99) == [1, 3, 4, 0, 2]
    assert kept(p=0.39) == [1] and kept(p=0.41) == [1, 3] and kept(p=0.84) == [1, 3, 4] and kept(p=0.0) == [1]
    assert kept(k=2, p=0.6) == [1] and kept(k=2, p=0.63) == [1, 3]     # 0.4 / 0.65 = 0.615
    assert kept(m=0.5) == [1, 3, 4] and kept(m=0.6) == [1, 3] and kept(m=1.0) == [1] and kept(m=2.0) == [1]
    assert kept(t=0.0) == [1] and kept(t=float("nan")) == [1]
    tied = np.array([1.0, 2.0, 2.0, 2.0, 0.0])
    assert list(od.kept_tokens(tied, 1.0, 2, 1.0, 0.0)[0]) == [1, 2]


def test_draw_is_the_inverse_of_the_running_sum():
    z = np.log(np.array([[0.1, 0.4, 0.0, 0.5]]) + 1e-300)
    z[0, 2] = -np.inf
    draw = lambda u, **k: od.sample(z, [1.0], k.get("k"), k.get("p"), k.get("m"), [u])
    assert [int(draw(u)[0][0]) for u in (0.0, 0.099, 0.101, 0.499, 0.501, 0.9999, 1.0)] == [0, 0, 1, 1, 3, 3, 3]
    assert int(draw(0.05, k=[2])[0][0]) == 1 and abs(draw(0.05, k=[2])[1][0] - 0.4 / 0.9) < 1e-12
    tok, prob, kept = od.sample(np.full((1, 4), -np.inf), [1.0], None, None, None, [0.5])
    assert tok[0] == -1 and prob[0] == 0 and kept[0] == 0
    many = [int(od.sample(z, [1.0], None, None, None, [u])[0][0]) for u in (np.arange(2000) + 0.5) / 2000]
    np.testing.assert_allclose(np.bincount(many, minlength=4) / 2000, [0.1, 0.4, 0.0, 0.5], atol=1e-3)


def test_infinite_and_nan_logits():
    z = np.array([[np.nan, np.inf, 0.0, np.inf, -np.inf]])
    tok, prob, kept = od.sample(z, [1.0], None, None, None, [0.6])
    assert tok[0] == 3 and prob[0] == 0.5 and kept[0] == 3            # -inf and NaN are no tokens, 0.0 has weight 0
    low = np.full((1, 3), np.finfo(np.float32).min)
    assert [int(od.sample(low, [1.0], None, None, None, [u])[0][0]) for u in (0.1, 0.5, 0.9)] == [0, 1, 2]


def test_embed_rows():
    E, Ep = np.arange(12.0).reshape(4, 3), 100 + np.arange(6.0).reshape(2, 3)
    x = od.embed_rows([2, -1, 4, 0], [1, 0, 7, 9], E, Ep)
    assert (x == [E[2] + Ep[1], Ep[0], [0, 0, 0], E[0]]).all()
