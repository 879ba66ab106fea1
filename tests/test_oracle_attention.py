"""Pins for the attention and rotary oracle: library attention and its derivatives in float64, differences, closed forms."""
import numpy as np
import pytest
import torch

import oracle


def _case(seed, lens_q, lens_k, H, K, D):
    rng = np.random.default_rng(seed)
    nq, nk = sum(lens_q), sum(lens_k)
    cut = lambda lens, n: oracle.groups(rng.permutation(n), np.concatenate([[0], np.cumsum(lens)]), len(lens), n, max(lens))
    r = lambda n, h: rng.standard_normal((n, h, D))
    return r(nq, H), r(nk, K), r(nk, K), r(nq, H), cut(lens_q, nq), cut(lens_k, nk), rng


@pytest.mark.parametrize("H,K,D", [(1, 1, 1), (4, 2, 8), (3, 1, 5)])
def test_library_attention_and_its_gradient(H, K, D):
    q, k, v, g, qg, kg, rng = _case(1, [3, 1, 7], [4, 2, 1], H, K, D)
    mask = np.ones(7, np.uint8)
    mask[kg[0][1]] = 0
    out, lse, _, _ = oracle.attention(q, k, v, qg, kg, 0.3, mask)
    (dq, dk, dv), _ = oracle.attention_backward(q, k, v, g, qg, kg, 0.3, mask)
    tq, tk, tv = (torch.from_numpy(x).requires_grad_() for x in (q, k, v))
    total = 0
    for rq, rk in zip(qg, kg):
        rk = rk[mask[rk] != 0]
        heads = lambda x, r: x[torch.from_numpy(r)].transpose(0, 1)
        rep = lambda x: x.repeat_interleave(H // K, 0)
        o = torch.nn.functional.scaled_dot_product_attention(heads(tq, rq), rep(heads(tk, rk)), rep(heads(tv, rk)), scale=0.3)
        assert np.allclose(o.detach().transpose(0, 1).numpy(), out[rq], atol=1e-12)
        z = 0.3 * heads(tq, rq) @ rep(heads(tk, rk)).transpose(1, 2)
        assert np.allclose(torch.logsumexp(z, -1).detach().T.numpy(), lse[rq], atol=1e-12)
        total = total + (o.transpose(0, 1) * torch.from_numpy(g[rq])).sum()
    total.backward()
    for mine, theirs in ((dq, tq), (dk, tk), (dv, tv)):
        assert np.allclose(mine, theirs.grad.numpy(), atol=1e-12)


def test_gradient_is_that_of_differences():
    q, k, v, g, qg, kg, rng = _case(2, [4, 2], [3, 6], 2, 1, 4)
    grads, _ = oracle.attention_backward(q, k, v, g, qg, kg, 0.7)
    loss = lambda *x: (oracle.attention(*x, qg, kg, 0.7)[0] * g).sum()
    at, h = (q, k, v), 1e-6
    for i in range(3):
        d = rng.standard_normal(at[i].shape)
        up, down = (tuple(x + s * h * d if j == i else x for j, x in enumerate(at)) for s in (1, -1))
        assert abs((loss(*up) - loss(*down)) / (2 * h) - (grads[i] * d).sum()) < 1e-7


def test_closed_forms():
    q, k, v, g, qg, kg, _ = _case(3, [2, 3], [1, 5], 2, 2, 3)
    out, lse, _, _ = oracle.attention(q, k, v, qg, kg, 1.0)
    assert np.allclose(out[qg[0]], v[kg[0]])                                    # one key: its value
    flat, lse0, _, _ = oracle.attention(0 * q, k, v, qg, kg, 1.0)
    assert np.allclose(flat[qg[1]], v[kg[1]].mean(0)) and np.allclose(lse0[qg[1]], np.log(5))
    none, lse1, _, _ = oracle.attention(q, k, v, qg, kg, 1.0, np.zeros(6))
    assert (none == 0).all() and (lse1 == -np.inf).all()
    (dq, dk, dv), _ = oracle.attention_backward(q, k, v, g, qg, kg, 1.0, np.zeros(6))
    assert not dq.any() and not dk.any() and not dv.any()


def test_groups_are_cut_to_the_rows_that_are_there():
    got = oracle.groups([2, 0, 9, 1], [-3, 2, 8], 2, 4, 3)
    assert [list(r) for r in got] == [[2, 0], [1]]
    assert [list(r) for r in oracle.groups(None, [0, 5, 9], 1, 9, 3)] == [[0, 1, 2]]


@pytest.mark.parametrize("half", [True, False])
def test_rotary_is_a_rotation_by_the_distance(half):
    rng = np.random.default_rng(4)
    x = rng.standard_normal((2, 1, 14))
    f = rng.uniform(0.01, 2, (2, 3))
    p = np.array([[5, -7], [100, 3]])
    y = oracle.rotary(x, p, f, half)
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1)) and (y[..., 12:] == x[..., 12:]).all()
    assert np.allclose(oracle.rotary(y, p, f, half, inverse=True), x)
    moved = oracle.rotary(x, p + 11, f, half)
    assert np.allclose((y[0] * y[1])[..., :12].sum(), (moved[0] * moved[1])[..., :12].sum())
    z = x[0, 0, 0] + 1j * x[0, 0, 3 if half else 1]
    assert np.allclose(y[0, 0, 0] + 1j * y[0, 0, 3 if half else 1], z * np.exp(5j * f[0, 0]))
