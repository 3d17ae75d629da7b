"""The fp64 definitions of the attention block's operators against closed forms, published numbers and differences."""
import numpy as np
import pytest

from oracle import attn_oracle as ao


def test_philox_known_answers():
    """the vectors that the authors of the generator publish with it"""
    assert ao.philox4x32((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    f = 0xFFFFFFFF
    assert ao.philox4x32((f, f, f, f), (f, f)) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert ao.philox4x32((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420,
                                                                                                    0x24126EA1]


def test_dropout_shares():
    mask, f = ao.dropout_mask(64, 67, 0.25, 5, 9)
    assert f == 4.0 / 3.0 and abs(mask.mean() - 0.75) < 5 * np.sqrt(0.1875 / mask.size)
    assert ao.dropout_mask(2, 9, 0.0, 1, 1)[0].all() and not ao.dropout_mask(2, 9, 1.0, 1, 1)[0].any()
    assert (ao.dropout_mask(4, 16, 0.5, -1, 3)[0] == ao.dropout_mask(4, 16, 0.5, 2 ** 64 - 1, 3)[0]).all()


@pytest.mark.parametrize("neighbours", [False, True])
def test_rotation_keeps_relative_positions(neighbours):
    rng = np.random.default_rng(0)
    f = 10.0 ** -np.arange(3)
    q, k = rng.normal(size=(1, 1, 8)), rng.normal(size=(1, 1, 8))
    dots = []
    for p in (3, 1000):
        a, b = (ao.rotate(x, ao.angles([[p + s]], f), neighbours) for x, s in ((q, 0), (k, 5)))
        dots.append((a * b).sum())
        assert np.allclose(a[..., 6:], q[..., 6:]) and np.isclose((a * a).sum(), (q * q).sum())
    assert np.isclose(*dots)
    assert np.allclose(ao.rotate(ao.rotate(q, ao.angles([[7]], f), neighbours), -ao.angles([[7]], f), neighbours), q)


def test_axes():
    t = ao.angles([[1, 2], [10, 20]], [0.5, 0.25, 2.0], [0, 1, 9])
    assert np.allclose(t, [[0.5, 2.5, 20.0], [1.0, 5.0, 40.0]])


@pytest.mark.parametrize("norm", [False, True])
def test_norm_rope_gradients_are_differences(norm):
    rng = np.random.default_rng(1)
    x, dy, w = rng.normal(size=(3, 20)), rng.normal(size=(3, 20)), rng.normal(size=10)
    t = ao.angles([[1, 5, 2]], [1.0, 0.3])
    dx, dw = ao.head_norm_rope_bwd(dy, x, 2, w, norm, 1e-3, t, False)

    def loss(x, w):
        return (ao.head_norm_rope_fwd(x, 2, w, norm, 1e-3, t, False) * dy).sum()
    h = 1e-6
    for at in [(0, 0), (1, 7), (2, 19), (2, 12)]:
        e = np.zeros_like(x)
        e[at] = h
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * h) - dx[at]) < 1e-7
    if norm:
        for at in (0, 9):
            e = np.zeros_like(w)
            e[at] = h
            assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * h) - dw[at]) < 1e-7


def test_masks():
    assert ao.seen(3, 3, True, 0, 0).tolist() == [[1, 0, 0], [1, 1, 0], [1, 1, 1]]
    assert ao.seen(4, 4, True, 2, 1).tolist() == [[1, 0, 0, 0], [1, 1, 0, 0], [1, 1, 1, 0], [1, 0, 1, 1]]
    assert ao.seen(3, 3, False, 1, 0).tolist() == [[1, 0, 0], [0, 1, 0], [0, 0, 1]]
    assert ao.seen(3, 1, True, 0, 0).tolist() == [[0], [0], [1]] and ao.seen(1, 3, True, 0, 0).all()


def test_attention_closed_forms():
    v = np.arange(6.0).reshape(3, 2)
    o, lse, p = ao.attention_fwd(np.zeros((3, 4)), np.ones((3, 4)), v, 0.5, ao.seen(3, 3, True, 0, 0))
    assert np.allclose(o, [v[0], v[:2].mean(0), v.mean(0)]) and np.allclose(lse, np.log([1, 2, 3]))
    o, lse, p = ao.attention_fwd(np.ones((2, 4)), np.ones((1, 4)), v[:1], 0.5, ao.seen(2, 1, True, 0, 0))
    assert (o[0] == 0).all() and lse[0] == -np.inf and np.allclose(o[1], v[0]) and lse[1] == 2.0


def test_attention_gradients_are_differences():
    rng = np.random.default_rng(2)
    q, k, v, do = (rng.normal(size=(n, 6)) for n in (4, 5, 5, 4))
    mask = ao.seen(4, 5, True, 2, 1)

    def loss(q, k, v):
        return (ao.attention_fwd(q, k, v, 0.7, mask)[0] * do).sum()
    o, _, p = ao.attention_fwd(q, k, v, 0.7, mask)
    grads = ao.attention_bwd(do, q, k, v, o, p, 0.7)[:3]
    h = 1e-6
    for n, (x, g) in enumerate(zip((q, k, v), grads)):
        for at in [(0, 0), (3, 5), (2, 1)]:
            e = [np.zeros_like(y) for y in (q, k, v)]
            e[n][at] = h
            up, down = loss(*(y + d for y, d in zip((q, k, v), e))), loss(*(y - d for y, d in zip((q, k, v), e)))
            assert abs((up - down) / (2 * h) - g[at]) < 1e-7
