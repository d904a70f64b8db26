"""The oracle of shared prefixes and of the choice among beams, against torch and by hand."""
import numpy as np
import torch

from oracle import beams, cache


def test_attention_over_prefix_and_own_is_attention_over_both():
    g = np.random.default_rng(1)
    q, k, v = g.normal(size=(5, 8)), g.normal(size=(30, 8)), g.normal(size=(30, 8))
    for before in (0, 7, 25):
        got = beams.attend(q, (k[:before], v[:before]), (k[before:], v[before:]), 5, 0.3, True)
        for a, b in zip(got, cache.attend(q, k, v, 0.3, True)):
            np.testing.assert_allclose(a, b, rtol=1e-12, atol=1e-14)
    s = torch.from_numpy(0.3 * q @ k.T)
    got = beams.attend(q, (k[:10], v[:10]), (k[10:], v[10:]), 5, 0.3, False)
    np.testing.assert_allclose(got[0], (torch.softmax(s, 1) @ torch.from_numpy(v)).numpy(), rtol=1e-12)
    np.testing.assert_allclose(got[1], torch.logsumexp(s, 1).numpy(), rtol=1e-12)
    # padded queries see nothing; a query before the first own token sees the prefix alone
    O, lse, _ = beams.attend(q, (k[:10], v[:10]), (k[10:12], v[10:12]), 4, 0.3, True)
    assert np.isneginf(lse[4]) and (O[4] == 0).all()
    np.testing.assert_allclose(lse[0], torch.logsumexp(torch.from_numpy(0.3 * k[:10] @ q[0]), 0).item(), rtol=1e-12)
    O, lse, _ = beams.attend(q, (k[:0], v[:0]), (k[:2], v[:2]), 4, 0.3, True)
    assert np.isneginf(lse[:2]).all() and np.isfinite(lse[2:4]).all()


def test_select_against_torch():
    g = torch.Generator().manual_seed(2)
    x, scores = torch.randn(4, 50, generator=g, dtype=torch.float64), -torch.rand(4, generator=g, dtype=torch.float64)
    total = scores[:, None] + torch.log_softmax(x, 1)
    want, at = torch.topk(total.view(-1), 9)
    parents, tokens, sums, ended = beams.select(x.numpy(), scores.numpy(), 9, end_token=int(at[3]) % 50)
    assert parents == (at // 50).tolist() and tokens == (at % 50).tolist() and ended[3]
    np.testing.assert_allclose(sums, want.numpy(), rtol=1e-12)


def test_select_by_hand():
    inf, nan = np.inf, np.nan
    x = np.array([[1.0, 2.0, 2.0, 1.0], [0.0, 0.0, -inf, 0.0], [nan, 9.0, 9.0, 9.0], [9.0, inf, 9.0, 9.0], [-inf] * 4, [5.0] * 4])
    p, t, s, e = beams.select(x, [0.0, 0.0, 0.0, 0.0, 0.0, -inf], 9, end_token=3)
    assert p == [0, 0, 1, 1, 1, 0, 0, -1, -1] and t == [1, 2, 0, 1, 3, 0, 3, -1, -1] and e == [False, False, False, False, True, False, True, False, False]
    np.testing.assert_allclose(s[2], -np.log(3.0))
    # ended beams: end_token alone, whatever their logits; equal sums: the lower beam
    p, t, s, e = beams.select(x, [-1.0, -1.0, -0.5, -1.0, -1.0, -1.0], 4, [True, False, True, False, True, False], 0)
    assert p == [2, 0, 4, 1] and t == [0, 0, 0, 0] and s[:3] == [-0.5, -1.0, -1.0] and e == [True, True, True, True]
    assert beams.origin([1, 0, -1, 9, 2]) == [1, 0, 2, 3, 2]
