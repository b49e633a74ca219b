"""Pins of the checkers for norm and rotation and for attention over a paged cache."""
import numpy as np
import pytest

from oracle import attention as att
from oracle import paged, rotation


def _case(seed, D=16, rot=16, tokens=5, heads=3):
    rng = np.random.default_rng(seed)
    return (rng.normal(size=(tokens, heads, D)), rng.uniform(0.5, 1.5, D), rng.integers(0, 5000, tokens),
            10000.0 ** (-np.arange(rot // 2) / max(rot // 2, 1)))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(16, 16), (24, 16), (8, 0), (64, 32)])
def test_rotation_keeps_pairs_and_goes_back(D, rot, interleaved):
    x, _, pos, f = _case(1, D, rot)
    y = rotation.turn(x, pos, f, rot, interleaved)
    np.testing.assert_allclose(rotation.pair_sizes(y, rot, interleaved), rotation.pair_sizes(x, rot, interleaved), rtol=1e-12)
    np.testing.assert_allclose(rotation.turn(y, pos, f, rot, interleaved, back=True), x, atol=1e-12)
    np.testing.assert_array_equal(y[..., rot:], x[..., rot:])


@pytest.mark.parametrize("interleaved", [False, True])
def test_dot_products_depend_on_the_distance_alone(interleaved):
    x, _, _, f = _case(2, tokens=2)
    for d in (0, 3, 41):
        dots = []
        for p in (0, 7, 1000):
            y = rotation.turn(x, [p, p + d], f, 16, interleaved)
            dots.append((y[0] * y[1]).sum(-1))
        np.testing.assert_allclose(dots[1], dots[0], atol=1e-10)
        np.testing.assert_allclose(dots[2], dots[0], atol=1e-10)


def test_hand_example():
    # rms of (3, 4, 0, 0 ..) over 8 values is 5 / sqrt(8); a quarter turn takes (a, b) to (-b, a)
    x = np.zeros((1, 1, 16))
    x[0, 0, 0], x[0, 0, 8] = 3.0, 4.0
    y = rotation.norm_rotate(x, np.full(16, 2.0), [1], np.full(8, np.pi / 2), 16, False, 0.0)
    np.testing.assert_allclose(y[0, 0, [0, 8]], np.array([-4.0, 3.0]) * 2.0 * 4.0 / 5.0, atol=1e-12)
    y = rotation.norm_rotate(np.roll(x, 0), None, [1], np.full(8, np.pi / 2), 16, True, 0.0)
    np.testing.assert_allclose(y[0, 0, [0, 1, 8, 9]], [0.0, 3.0, 0.0, 4.0], atol=1e-12)


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_gradients_by_differences(norm, interleaved):
    x, g, pos, f = _case(3, D=24, rot=16)
    gamma = g if norm else None
    dy = np.random.default_rng(4).normal(size=x.shape)
    fun = lambda x_, g_: (rotation.norm_rotate(x_, g_, pos, f, 16, interleaved, 1e-3) * dy).sum()
    dx, dg = rotation.norm_rotate_bwd(x, gamma, pos, f, 16, interleaved, 1e-3, dy)
    h = 1e-6
    for at in [(0, 0, 0), (1, 2, 7), (4, 1, 15), (2, 0, 20)]:
        e = np.zeros_like(x)
        e[at] = h
        assert abs((fun(x + e, gamma) - fun(x - e, gamma)) / (2 * h) - dx[at]) < 1e-7
    if norm:
        for i in (0, 9, 23):
            e = np.zeros_like(g)
            e[i] = h
            assert abs((fun(x, g + e) - fun(x, g - e)) / (2 * h) - dg[i]) < 1e-7
    else:
        assert dg is None


@pytest.mark.parametrize("stride", [1, 3, 64, 1 << 30])
@pytest.mark.parametrize("page_size", [1, 5, 16])
def test_paged_attention_is_the_plain_one_in_shuffled_pages(page_size, stride):
    rng = np.random.default_rng(5)
    B, n, H, d = 2, 70, 3, 8
    q, k, v = (rng.normal(size=(B, H, n, d)) for _ in range(3))
    per = (n + page_size - 1) // page_size
    order = rng.permutation(B * per + 2)
    table = order[: B * per].reshape(B, per)
    K, V = (np.full((B * per + 2, page_size, H, d), np.nan) for _ in range(2))
    for b in range(B):
        for p in range(n):
            K[table[b, p // page_size], p % page_size], V[table[b, p // page_size], p % page_size] = k[b, :, p], v[b, :, p]
    ref, ref_lse = att.strided_attention(q, k, v, stride) if stride > 1 else att.strided_attention(q, k, v, n)
    new = (n, 4)                                   # the first sequence whole, of the second the last four
    Q = np.concatenate([q[0].transpose(1, 0, 2), q[1][:, n - 4:].transpose(1, 0, 2)])
    out, lse, weight = paged.paged_attention(Q, K, V, [0, n, n + 4], [n, n], table, stride)
    np.testing.assert_allclose(out[:n], ref[0].transpose(1, 0, 2), atol=1e-12)
    np.testing.assert_allclose(out[n:], ref[1][:, n - 4:].transpose(1, 0, 2), atol=1e-12)
    np.testing.assert_allclose(lse[:, n:], ref_lse[1][:, n - 4:], atol=1e-12)
    assert (weight >= np.abs(out) - 1e-12).all()


def test_paged_attention_leaves_out_what_is_not_there():
    K = np.random.default_rng(6).normal(size=(3, 4, 1, 8))
    V, Q = K + 1, np.ones((4, 2, 8))
    out, lse, _ = paged.paged_attention(Q, K, V, [0, 2, 4], [1, 4], np.array([[0, -1], [7, 1]]), 64)
    assert (out[0] == 0).all() and np.isneginf(lse[:, 0]).all()          # position -1
    np.testing.assert_allclose(out[1], np.repeat(V[0, 0], 2, 0))          # itself alone
    assert (out[2:] == 0).all() and np.isneginf(lse[:, 2:]).all()        # its page does not exist
