"""The oracle of the operators on shared prefixes, against torch and against itself."""
import numpy as np
import torch

from oracle import shared


def _cache(rng, ctx, nrow, n_kv, hd):
    need = [(c + r + 15) // 16 for c, r in zip(ctx, nrow)]
    nb = sum(need) + 1
    pt, o = np.full((len(ctx), max(need)), -1, np.int32), 0
    perm = rng.permutation(nb)
    for i, k in enumerate(need):
        pt[i, :k] = perm[o:o + k]
        o += k
    return rng.normal(0, 1, (nb, n_kv, 16, hd)), rng.normal(0, 1, (nb, n_kv, 16, hd)), pt


def test_attention_and_mass_against_torch():
    rng = np.random.default_rng(1)
    ctx, nrow = [20, 3], [3, 2]
    k, v, pt = _cache(rng, ctx, nrow, 2, 32)
    q = rng.normal(0, 1, (5, 4, 32))
    out, lse, _, _ = shared.attention(q, k, v, pt, ctx, nrow)
    prev = rng.random(k.shape[:3])
    mass, _, on = shared.mass(q, k, lse, pt, ctx, nrow, [2, 2], 0.5, prev)
    want = np.zeros_like(mass)
    r = 0
    for b in range(2):
        T = ctx[b] + nrow[b]
        K, V = (torch.from_numpy(shared.tokens(p, pt[b, :(T + 15) // 16], 0, T)) for p in (k, v))
        for j in range(nrow[b]):
            s = torch.from_numpy(q[r, :2]) @ K.T / 32 ** 0.5
            s[:, ctx[b] + j + 1:] = -torch.inf
            np.testing.assert_allclose(out[r, :2], (torch.softmax(s, -1) @ V).numpy(), rtol=1e-12, atol=1e-14)
            np.testing.assert_allclose(lse[r, :2], torch.logsumexp(s, -1).numpy(), rtol=1e-13)
            if j < 2:
                for t in range(T):
                    want[pt[b, t // 16], 0, t % 16] += torch.softmax(s, -1)[:, t].sum().item()
            r += 1
        for t in range(T):
            assert on[pt[b, t // 16], 0, t % 16]
            if t < ctx[b]:
                want[pt[b, t // 16], 0, t % 16] += 0.5 * prev[pt[b, t // 16], 0, t % 16]
    np.testing.assert_allclose(mass[:, 0], want[:, 0], rtol=1e-12, atol=1e-14)
    assert on.sum() == 2 * (23 + 5)


def test_chosen():
    w = np.array([5, 0, 3, 3, np.nan, 1, 3, -np.inf, 9], np.float32)
    np.testing.assert_array_equal(shared.chosen(w, 4, 0, 0), [0, 2, 3, 8])
    np.testing.assert_array_equal(shared.chosen(w, 5, 2, 0), [0, 1, 2, 3, 8])
    np.testing.assert_array_equal(shared.chosen(w, 7, 0, 1), [0, 1, 2, 3, 5, 6, 8])
    np.testing.assert_array_equal(shared.chosen(w, 8, 0, 0), [0, 1, 2, 3, 5, 6, 7, 8])
    np.testing.assert_array_equal(shared.chosen(w, 3, 2, 1), [0, 1, 8])
    np.testing.assert_array_equal(shared.chosen(w, 99, 2, 1), np.arange(9))


def test_evicted_keys_are_those_of_their_new_positions():
    """Keys rotated by their positions before, are rotated by their new ones after; scores of queries at the
    same distance from them are the same."""
    rng = np.random.default_rng(2)
    ctx, base, hd = [40, 18], 1e4, 32
    raw = rng.normal(0, 1, (2, 40, hd))
    k, v, pt = _cache(rng, ctx, [0, 0], 1, hd)
    k, v = k[None], v[None]
    freq = base ** (-2.0 * np.arange(hd // 2) / hd)

    def rot(x, p):
        c, s = np.cos(p * freq), np.sin(p * freq)
        return np.concatenate([x[:hd // 2] * c - x[hd // 2:] * s, x[hd // 2:] * c + x[:hd // 2] * s])

    for b in range(2):
        for t in range(ctx[b]):
            k[0, pt[b, t // 16], 0, t % 16] = rot(raw[b, t], t)
    mass = rng.random(k.shape[:4]).astype(np.float32)
    v0 = v.copy()
    kept, pair = shared.evict(k, v, mass, pt, ctx, [17, 18], [2, 0], [3, 0], pt, base)
    assert kept.shape == (1, 1, 35)
    for b, (a, n) in enumerate([(0, 17), (17, 18)]):
        for d, t in enumerate(kept[0, 0, a:a + n]):
            np.testing.assert_allclose(k[0, pt[b, d // 16], 0, d % 16], rot(raw[b, t], d), atol=1e-12)
            np.testing.assert_array_equal(v[0, pt[b, d // 16], 0, d % 16], v0[0, pt[b, t // 16], 0, t % 16])
    assert (pair[0, pt[1, 0]] == 0).all() and (kept[0, 0, 17:] == np.arange(18)).all()
