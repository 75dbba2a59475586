"""CPU pins of the oracle's routing from scores, 8-bit float rows and gradient clipping:
hand-worked values, torch autograd in fp64, central differences and torch's e4m3 type."""
import numpy as np
import pytest
import torch

import oracle as O


def test_group_limited_selection_by_hand():
    # 2 groups of 3; the second group's two best sum to more, the first holds the best
    z = np.array([[4.0, -4.0, -4.0, 1.0, 1.0, -9.0]])
    s = O.scores(z, "sigmoid")[0]
    idx, gate, _ = O.route_scored(z, 2, "sigmoid", 2, 1, 2)
    assert idx.tolist() == [[3, 4]] and np.allclose(gate, 0.5)
    idx, gate, _ = O.route_scored(z, 2, "sigmoid", 2, 1, 1, renorm=False, scale=3.0)
    assert idx.tolist() == [[0, 1]] and np.allclose(gate, 3 * s[[0, 1]])
    # a selection bias moves the choice, not the gate
    idx, gate, _ = O.route_scored(z, 2, "sigmoid", sel_bias=np.array([0, 2.0, 0, 0, 0, 1.0]), renorm=False)
    assert idx.tolist() == [[1, 5]] and np.allclose(gate, s[[1, 5]])
    # ties go to the lower expert and the lower group
    assert O.route_scored(np.zeros((1, 6)), 3, "softmax", 3, 2, 1)[0].tolist() == [[0, 1, 2]]


def test_scores_of_infinities_and_nothing():
    inf = np.inf
    z = np.array([[inf, inf, 0.0], [-inf, -inf, -inf], [np.nan, 1.0, -inf], [800.0, -800.0, 0.0]])
    np.testing.assert_allclose(O.scores(z, "softmax"), [[0.5, 0.5, 0], [0, 0, 0], [0, 1, 0], [1, 0, 0]], atol=1e-300)
    assert np.isfinite(O.scores(z, "sigmoid")).all()
    idx, gate, _ = O.route_scored(z, 2)
    assert idx.tolist() == [[0, 1], [0, 1], [1, 0], [0, 2]]
    np.testing.assert_allclose(gate[1], 0)
    # scores too small for fp64 still share their sum
    np.testing.assert_allclose(O.route_scored(np.array([[-900.0, -900.0, -2000.0]]), 2, "sigmoid")[1], 0.5)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_gradient(score, renorm):
    rng = np.random.default_rng(3)
    z, dg = rng.standard_normal((5, 12)) * 2, rng.standard_normal((5, 4))
    idx, gate, _ = O.route_scored(z, 4, score, 3, 2, 2, renorm, 2.5, rng.standard_normal(12) * 0.1)
    got = O.route_scored_backward(z, idx, dg, score, renorm, 2.5)
    t = torch.tensor(z, requires_grad=True)
    s = torch.sigmoid(t) if score == "sigmoid" else torch.softmax(t, 1)
    sel = s.gather(1, torch.tensor(idx))
    g = 2.5 * (sel / sel.sum(1, keepdim=True) if renorm else sel)
    np.testing.assert_allclose(g.detach(), gate, rtol=1e-12)
    g.backward(torch.tensor(dg))
    np.testing.assert_allclose(got, t.grad, rtol=1e-10, atol=1e-14)
    for t_, e in ((0, 3), (4, 11), (2, int(idx[2, 0]))):
        up, down = z.copy(), z.copy()
        up[t_, e] += 1e-5
        down[t_, e] -= 1e-5
        diff = (O.gates_of(up, idx, score, renorm, 2.5) - O.gates_of(down, idx, score, renorm, 2.5)) / 2e-5
        assert abs((diff * dg).sum() - got[t_, e]) < 1e-8
    # an expert named twice takes both shares; an entry outside takes no part
    twice = O.route_scored_backward(z[:1], [[2, 2]], [[1.0, 1.0]], score, False, 1.0)
    once = O.route_scored_backward(z[:1], [[2, -1]], [[2.0, 5.0]], score, False, 1.0)
    np.testing.assert_allclose(twice, once, rtol=1e-12)


def test_bias_update_by_hand():
    np.testing.assert_allclose(O.bias_update([4, 0, 2], [0.5, 0.5, 0.5], 0.25), [0.25, 0.75, 0.5])


def test_fp8_against_torch():
    rng = np.random.default_rng(0)
    q = np.concatenate((rng.standard_normal(4000) * np.exp(2 * rng.standard_normal(4000)), [0.0, 448, -448, 2.0 ** -10,
                                                                                          3 * 2.0 ** -10, 17.0, 19.0, 432.0]))
    q = np.clip(q, -448, 448).astype(np.float32)
    want = torch.tensor(q).to(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(O.fp8_nearest(q), want)


def test_fp8_blocks():
    rng = np.random.default_rng(1)
    W = rng.standard_normal((200, 200))
    W[:128, 128:] = 0
    val, scale = O.fp8_rows(W, 128)
    assert scale.shape == (2, 2) and scale[0, 1] == 0 and scale[0, 0] == np.float32(np.abs(W[:128, :128]).max() / 448)
    assert np.abs(val[:128, :128]).max() == 448
    # half a step: 2^-4 of the value, or of the smallest normal value's step below it
    e = O.fp8_spread(scale, 200, 200, 128)
    assert np.all(np.abs(val * e - W) <= np.maximum(2.0 ** -4 * np.abs(W), 2.0 ** -10 * e) * (1 + 1e-6))
    W[150, 150] = np.inf
    assert np.isnan(O.fp8_rows(W, 128)[1][1, 1]) and np.isnan(O.fp8_round(W, 128)[128:, 128:]).all()
    v, s = O.fp8_rows(np.full((1, 8), 2.0 ** -140))       # below the floor of the scales
    assert s[0, 0] == 2.0 ** -126 and not v.any()


def test_fp8_forward():
    """Activations that are codes times a power of two pass as they are; H is quantised
    between the products, and where its rows are codes too the output is torch's."""
    rng = np.random.default_rng(2)
    x = rng.choice([448.0, 0.5, -3.0, 0.0, 26.0], (5, 160))
    x[:, 0] = x[:, 128] = 448
    Wg, Wu, Wd = rng.standard_normal((130, 160)) / 500, rng.standard_normal((130, 160)) / 500, rng.standard_normal((160, 130))
    H, out = O.swiglu_fp8_fwd(x, Wg, Wu, Wd)
    t = torch.tensor(x)
    np.testing.assert_allclose(H, torch.nn.functional.silu(t @ torch.tensor(Wg).T) * (t @ torch.tensor(Wu).T), rtol=1e-10, atol=1e-13)
    np.testing.assert_array_equal(out, O.fp8_round(H) @ Wd.T)
    big = np.abs(H).max() * 1e3                          # one gate saturates, and up makes H a code
    Hs, out = O.swiglu_fp8_fwd(np.array([[448.0] + [0.0] * 127]), np.full((1, 128), big), np.full((1, 128), 2.0), Wd[:, :1])
    np.testing.assert_allclose(out, Hs * Wd[:, 0], rtol=1e-7)


def test_clip_by_hand():
    assert O.grad_sumsq([np.array([3.0]), None, np.array([[4.0]])]) == 25
    assert O.clip_coefficient(25.0, 1.0, 0.0) == 0.2 and O.clip_coefficient(25.0, 6.0) == 1.0
    assert O.clip_coefficient(0.0, 0.0, 0.0) == 1.0 and O.clip_coefficient(0.0, 0.0) == 0.0
    assert O.clip_coefficient(np.inf, 1.0) == 0.0 and np.isnan(O.clip_coefficient(np.nan, 1.0))
