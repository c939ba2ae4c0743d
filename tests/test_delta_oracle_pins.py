"""The fp64 oracle of the gated delta rule and of the norms between two blocks, held to closed forms, to the plain operator's oracle and
to differences.  No GPU."""
import numpy as np
import pytest

from oracle import delta_oracle as orc
from oracle import la_oracle


def draw(rng, B, H, Hk, N, d):
    q, k = (rng.standard_normal((B, Hk, N, d)) for _ in range(2))
    k /= np.linalg.norm(k, axis=-1, keepdims=True)
    return q, k, rng.standard_normal((B, H, N, d)), -rng.random((B, H, N)), rng.random((B, H, N))


def test_unit_key_is_overwritten():
    """beta = 1, no decay, one key: the state holds the last value alone."""
    v = np.arange(12.0).reshape(1, 1, 3, 4)
    k = np.zeros((1, 1, 3, 4))
    k[..., 2] = 1.0
    o, S = orc.delta_fwd(2 * k, k, v, np.zeros((1, 1, 3)), np.ones((1, 1, 3)), scale=0.5)
    assert np.array_equal(o, v) and np.array_equal(S[0, 0, 2], v[0, 0, 2]) and not S[0, 0, [0, 1, 3]].any()


def test_orthogonal_keys_are_the_plain_operator():
    """With keys orthogonal to one another nothing is taken out, and a constant decay is lambda.  The plain operator's oracle takes q, k
    and beta v rounded to fp32, half a step of 2^-24 each: its sums are off by at most three times that of the sums of magnitudes (the
    second half of the bound is for products of roundings and for its own)."""
    rng = np.random.default_rng(0)
    N = d = 8
    k = np.linalg.qr(rng.standard_normal((N, d)))[0].reshape(1, 1, N, d)
    q, v = rng.standard_normal((2, 1, 1, N, d))
    beta = rng.random((1, 1, N))
    lam = 0.9
    o, S = orc.delta_fwd(q, k, v, np.full((1, 1, N), np.log(lam)), beta)
    ref, ref_S = la_oracle.fwd_rec(q, k, beta[..., None] * v, np.array([lam]), want_state=True)
    most, most_S = la_oracle.fwd_rec(abs(q), abs(k), abs(beta[..., None] * v), np.array([lam]), want_state=True)
    for got, want, size in ((o, ref, most), (S, ref_S, most_S)):
        assert np.all(abs(got - want) <= 3.5 * 2.0 ** -24 * size)


def test_forgetting_and_idle_tokens():
    rng = np.random.default_rng(1)
    q, k, v, g, beta = draw(rng, 1, 2, 2, 10, 4)
    g[:, :, 5] = -np.inf                                        # nothing before token 5 is seen from it on
    whole, _ = orc.delta_fwd(q, k, v, g, beta)
    tail, _ = orc.delta_fwd(*(x[:, :, 5:] for x in (q, k, v, g, beta)))
    assert np.array_equal(whole[:, :, 5:], tail)
    g[:, :, 7:], beta[:, :, 7:] = 0, 0                          # padding leaves the state as it is
    _, S = orc.delta_fwd(q, k, v, g, beta)
    _, at6 = orc.delta_fwd(*(x[:, :, :7] for x in (q, k, v, g, beta)))
    assert np.array_equal(S, at6)


@pytest.mark.parametrize("Hk", [1, 2])
def test_delta_adjoint_against_differences(Hk):
    rng = np.random.default_rng(2 + Hk)
    B, H, N, d, scale = 2, 2, 5, 3, 0.7
    args = list(draw(rng, B, H, Hk, N, d))
    do, s0, ds = rng.standard_normal((B, H, N, d)), rng.standard_normal((B, H, d, d)), rng.standard_normal((B, H, d, d))

    def loss(*a):
        o, S = orc.delta_fwd(*a[:5], scale=scale, kv_in=a[5])
        return np.sum(o * do) + np.sum(S * ds)

    grads = orc.delta_bwd(*args, do, scale=scale, kv_in=s0, grad_kv_out=ds)
    for i, x in enumerate(args + [s0]):
        step = 1e-6 * rng.standard_normal(x.shape)
        moved = [list(args) + [s0], list(args) + [s0]]
        moved[0][i], moved[1][i] = x + step, x - step
        want = (loss(*moved[0]) - loss(*moved[1])) / 2
        assert np.isclose(np.sum(grads[i] * step), want, rtol=1e-6, atol=1e-12)


@pytest.mark.parametrize("gate,post_norm,eps", [(0, True, 0.0), (1, True, 1e-5), (2, False, 1e-3), (None, True, 1e-6)])
def test_norm_adjoint_against_differences(gate, post_norm, eps):
    rng = np.random.default_rng(7)
    rows, D = 3, 6
    x, y, u = rng.standard_normal((3, rows, D))
    w = list(1 + 0.3 * rng.standard_normal((3, D)))
    dh, dn = rng.standard_normal((2, rows, D))
    more = {"eps": eps, "gate": gate or 0, "post_norm": post_norm}

    def loss(x, y, u, *w):
        h, n = orc.block_norm_fwd(x, y, None if gate is None else u, *w, **more)
        return np.sum(h * dh) + np.sum(n * dn)

    grads = orc.block_norm_bwd(x, y, None if gate is None else u, *w, dh, dn, **more)
    args = [x, y, u] + w
    for i, a in enumerate(args):
        if i == 2 and gate is None:
            assert grads[i] is None
            continue
        step = 1e-6 * rng.standard_normal(a.shape)
        up, down = list(args), list(args)
        up[i], down[i] = a + step, a - step
        assert np.isclose(np.sum(grads[i] * step), (loss(*up) - loss(*down)) / 2, rtol=1e-6, atol=1e-12)


def test_norm_by_hand():
    x, y = np.zeros((2, 2)), np.array([[3.0, 4.0], [0.0, 0.0]])
    h, n = orc.block_norm_fwd(x, y, s=np.array([2.0, 1.0]))
    r = np.sqrt(12.5)
    assert np.allclose(h, [[6 / r, 4 / r], [0, 0]]) and np.allclose(n, [[6 / np.sqrt(26), 4 / np.sqrt(26)], [0, 0]])
    _, n = orc.block_norm_fwd(x, y, eps=12.5, post_norm=False)
    assert np.allclose(n[0], [3 / 5, 4 / 5])
