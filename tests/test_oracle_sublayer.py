"""Pins of the plain implementations around the pool layer: finite differences, hand values and closed cases."""
import numpy as np
import pytest

from oracle import sublayer_oracle as O


def test_norm_of_a_hand_row():
    h, y = O.rmsnorm(np.array([[1.0, 2.0]]), np.array([[2.0, 2.0]]), np.array([1.0, 0.5]), 0.0)
    assert np.array_equal(h, [[3.0, 4.0]])
    assert np.allclose(y, [[3.0 / np.sqrt(12.5), 2.0 / np.sqrt(12.5)]], rtol=1e-15)


def test_norm_gradients_against_differences():
    g = np.random.default_rng(1)
    h, w, dy, dh = g.standard_normal((3, 7)), g.standard_normal(7), g.standard_normal((3, 7)), g.standard_normal((3, 7))
    dx, dw = O.rmsnorm_bwd(h, w, dy, dh, 1e-3)

    def objective(h, w):
        return np.sum(O.rmsnorm(h, None, w, 1e-3)[1] * dy) + np.sum(h * dh)
    step = 1e-6
    for i in np.ndindex(h.shape):
        d = np.zeros_like(h)
        d[i] = step
        assert abs((objective(h + d, w) - objective(h - d, w)) / (2 * step) - dx[i]) < 1e-7
    for i in range(7):
        d = np.zeros(7)
        d[i] = step
        assert abs((objective(h, w + d) - objective(h, w - d)) / (2 * step) - dw[i]) < 1e-7


@pytest.mark.parametrize("router", ["norm", "softmax"])
def test_balance_gradients_against_differences(router):
    g = np.random.default_rng(2)
    z = g.standard_normal((11, 5))
    idx = np.argsort(-z, axis=1)[:, :2]
    off = [1, 4, 4, 9, 10]                                # a token in front, an empty sequence, one behind
    args = (idx, off, 0.3, router)
    _, loss, dz, ds = O.seq_balance_loss(z, *args, 1.2, 1.7, 1e-6)
    step = 1e-6
    for i in np.ndindex(z.shape):
        d = np.zeros_like(z)
        d[i] = step
        hi, lo = (O.seq_balance_loss(z + s * d, *args, 1.2, 1.7, 1e-6)[1] for s in (1, -1))
        assert abs((hi - lo) / (2 * step) - dz[i]) < 1e-8
    hi, lo = (O.seq_balance_loss(z, *args, 1.2 + s * step, 1.7, 1e-6)[1] for s in (1, -1))
    assert abs((hi - lo) / (2 * step) - ds) < 1e-8
    assert not dz[0].any() and not dz[10].any()


def test_balance_of_even_use_is_alpha():
    # every expert picked equally often and all probabilities alike: f = 1, sum P = 1, whatever the lengths
    z = np.zeros((8, 4))
    idx = np.array([[t % 4] for t in range(8)])
    counts, loss, dz, _ = O.seq_balance_loss(z, idx, [0, 4, 8], 0.25, "softmax", 1.0, 1.0, 0.0)
    assert np.array_equal(counts, np.ones((2, 4))) and abs(loss - 0.25) < 1e-15 and np.abs(dz).max() < 1e-17


def test_one_sequence_is_the_layer_loss():
    from oracle import unipool_oracle as P
    g = np.random.default_rng(3)
    x, w = g.standard_normal((40, 6)), g.standard_normal((8, 6))
    r = P.route(x, w, 2, 1.1, 2.0, 1e-6)
    want = P.pool_aux_loss(r["counts"][None], r["psum"][None], 40, 2, 0.02)[2]
    counts, loss, _, _ = O.seq_balance_loss(P.router_logits(x, w), r["idx"], [0, 40], 0.02, "norm", 1.1, 2.0, 1e-6)
    assert np.array_equal(counts[0], r["counts"])
    by_hand = 0.02 * 8 * np.sum(r["counts"] / 80.0 * r["psum"] / 40.0)
    assert abs(loss - by_hand) < 1e-14
    assert abs(loss - want) < 1e-14


def test_e4m3_grid():
    v = O.e4m3_values()
    assert v[0x38] == 1.0 and v[0x7e] == 448.0 and v[0x01] == 2.0 ** -9 and v[0x08] == 2.0 ** -6 and np.isnan(v[0x7f])
    assert np.array_equal(O.to_e4m3(v[:127]), np.arange(127))
    assert list(O.to_e4m3(np.array([1.0625, 1.1875, -1.0625, 2.0 ** -10, 3 * 2.0 ** -10, 447.0]))) == [0x38, 0x3a, 0xb8, 0x00, 0x02, 0x7e]


def test_mx8_scales_and_blocks():
    v = np.zeros((5, 96))
    v[0, 0], v[0, 33] = 448.0, 449.0                     # scale 1, then the next power of two
    v[1, 64] = np.inf
    v[2, 5] = np.nan
    v[3, 7] = 1e-45
    v[4, :] = 2.0 ** -100
    q, s = O.to_mx8(v)
    assert s.shape == (1, 5, 4)
    assert list(s[0, 0]) == [127, 128, 0, 127] and list(s[0, 1]) == [0, 0, 255, 127] and s[0, 2, 0] == 255 and s[0, 3, 0] == 0
    back = O.from_mx8(q, s)
    assert back[0, 0] == 448.0 and abs(back[0, 33] - 449.0) <= 449.0 * 2.0 ** -4
    assert np.isnan(back[1, 64:]).all() and np.isnan(back[2, :32]).all() and (back[3] == 0).all()
    assert np.array_equal(back[4], v[4])
    w = np.random.default_rng(4).standard_normal((6, 160))
    q, s = O.to_mx8(w)
    assert s.shape == (2, 6, 4) and (s[1, :, 1:] == 127).all()
    e = np.repeat(np.transpose(s, (1, 0, 2)).reshape(6, -1)[:, :5].astype(int) - 127, 32, axis=1)
    assert (np.abs(O.from_mx8(q, s) - w) <= np.maximum(np.abs(w) * 2.0 ** -4, 2.0 ** (e - 10.0))).all()


def test_balance_of_a_token_without_a_direction():
    z = np.array([[1.0, 2.0], [0.0, 0.0], [-1.0, 3.0]])
    idx = np.array([[1], [0], [1]])
    counts, loss, dz, ds = O.seq_balance_loss(z, idx, [0, 3], 0.3, "norm", 2.0, 1.5, 0.0)
    near = O.seq_balance_loss(z, idx, [0, 3], 0.3, "norm", 2.0, 1.5, 1e-12)
    assert np.array_equal(counts, [[1, 2]]) and not dz[1].any() and np.isfinite(loss)
    assert abs(loss - near[1]) < 1e-11 and abs(ds - near[3]) < 1e-11 and np.abs(dz - near[2]).max() < 1e-11
