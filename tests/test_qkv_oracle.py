"""Pins of the float64 reference of the operators around the attention (CPU)."""
import numpy as np
import pytest
import torch

from oracle import qkv as O


def freqs(rot):
    return 10000.0 ** (-np.arange(0, rot, 2) / rot)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [0, 4, 8])
def test_norm_rope_against_complex_numbers_and_autograd(rot, interleaved):
    rng = np.random.default_rng(0)
    x, w, dy = rng.normal(size=(5, 3, 8)), rng.normal(size=8), rng.normal(size=(5, 3, 8))
    pos = np.array([0, 1, 7, -3, 100000])
    f = freqs(rot) if rot else None
    tx, tw = torch.from_numpy(x).requires_grad_(), torch.from_numpy(w).requires_grad_()
    y = tx * torch.rsqrt(tx.square().mean(-1, keepdim=True) + 1e-5) * tw
    if rot:
        ia, ib = ((slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot)))
        ang = torch.from_numpy(pos[:, None] * f[None])[:, None]
        z = torch.complex(y[..., ia], y[..., ib]) * torch.polar(torch.ones_like(ang), ang)
        y = y.clone()
        y[..., ia], y[..., ib] = z.real, z.imag
    np.testing.assert_allclose(O.norm_rope(x, w, 1e-5, pos, f, interleaved), y.detach().numpy(), rtol=0, atol=1e-13)
    y.backward(torch.from_numpy(dy))
    dx, dw, _, _ = O.norm_rope_bwd(x, w, 1e-5, pos, f, interleaved, dy)
    np.testing.assert_allclose(dx, tx.grad.numpy(), rtol=0, atol=1e-12)
    np.testing.assert_allclose(dw, tw.grad.numpy(), rtol=0, atol=1e-11)


def test_gradient_against_differences():
    rng = np.random.default_rng(1)
    x, w, dy = rng.normal(size=(2, 2, 4)), rng.normal(size=4), rng.normal(size=(2, 2, 4))
    pos, f = np.array([3, 11]), freqs(4)
    dx, dw, _, _ = O.norm_rope_bwd(x, w, 1e-3, pos, f, False, dy)
    loss = lambda a, b: float((O.norm_rope(a, b, 1e-3, pos, f, False) * dy).sum())  # noqa: E731
    h = 1e-6
    for i in np.ndindex(*x.shape):
        e = np.zeros_like(x)
        e[i] = h
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * h) - dx[i]) < 1e-8
    for i in range(4):
        e = np.zeros(4)
        e[i] = h
        assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * h) - dw[i]) < 1e-8


def test_rotation_keeps_lengths_and_relative_positions():
    rng = np.random.default_rng(2)
    q, k = rng.normal(size=(1, 1, 8)), rng.normal(size=(1, 1, 8))
    turned = lambda x, t: O.norm_rope(x, None, 0, np.array([t]), freqs(8), False)[0, 0]  # noqa: E731
    assert abs(np.linalg.norm(turned(q, 12345)) - np.linalg.norm(q)) < 1e-12
    assert abs(turned(q, 105) @ turned(k, 100) - turned(q, 5) @ turned(k, 0)) < 1e-12


def small_cache(rng, lens, page=4, hkv=2, d=4, spare=2):
    need = [-(-n // page) for n in lens]
    pages = sum(need) + spare
    ids = rng.permutation(pages)
    table = np.full((len(lens), max(need) + 1), -1)
    for b, n in enumerate(need):
        table[b, :n] = ids[sum(need[:b]):sum(need[:b]) + n]
    return rng.normal(size=(pages, page, hkv, d)), rng.normal(size=(pages, page, hkv, d)), table


@pytest.mark.parametrize("causal", [True, False])
def test_paged_attention_is_the_packed_one_on_gathered_keys(causal):
    rng = np.random.default_rng(3)
    lens, new = [9, 4, 1, 0], [3, 4, 1, 2]
    kc, vc, table = small_cache(rng, lens)
    cu = np.concatenate([[0], np.cumsum(new)])
    q = rng.normal(size=(cu[-1], 4, 4))
    o, l, _ = O.paged_fwd(q, kc, vc, table, lens, cu, causal, 0.5)
    o2, l2 = O.paged_by_varlen(q, kc, vc, table, lens, cu, causal, 0.5)
    np.testing.assert_allclose(o, o2, atol=1e-13)
    np.testing.assert_allclose(l, l2, atol=1e-13)
    assert np.all(o[-2:] == 0) and np.all(np.isneginf(l[:, -2:]))  # a sequence without keys


def test_missing_pages_hide_their_keys():
    rng = np.random.default_rng(4)
    kc, vc, table = small_cache(rng, [9])
    q, cu = rng.normal(size=(2, 2, 4)), np.array([0, 2])
    gone = table.copy()
    gone[0, 1] = 99  # keys 4 .. 7
    o, l, _ = O.paged_fwd(q, kc, vc, gone, [9], cu, True, 0.5)
    for i in range(2):
        js = [j for j in range(9) if not 4 <= j < 8 and j <= i + 7]
        kk = np.array([kc[table[0, j // 4], j % 4] for j in js])
        vv = np.array([vc[table[0, j // 4], j % 4] for j in js])
        for h in range(2):
            p = np.exp(0.5 * kk[:, h] @ q[i, h])
            np.testing.assert_allclose(o[i, h], p @ vv[:, h] / p.sum(), atol=1e-13)
            assert abs(l[h, i] - np.log(p.sum())) < 1e-12


def test_append_stores_the_last_tokens_and_nothing_else():
    rng = np.random.default_rng(5)
    lens, new = np.array([6, 2, 3]), [2, 2, 0]
    kc, vc, table = small_cache(rng, lens)
    table[1, 0] = -7  # no page: not stored
    cu = np.array([0, 2, 4, 4])
    k, v = rng.normal(size=(5, 2, 4)), rng.normal(size=(5, 2, 4))
    k2, v2, stored = O.append(k, v, kc, vc, table, lens, cu)
    assert stored == [(table[0, 1], 0, 0), (table[0, 1], 1, 1)]
    assert (k2 != kc).any(axis=(2, 3)).sum() == 2 and np.array_equal(v2[table[0, 1], 1], v[1])
