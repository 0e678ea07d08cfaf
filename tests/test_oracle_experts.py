"""Pins of the experts' oracle: grouping against a stable sort, the gradients
against differences, the 4-bit format against values worked by hand."""
import numpy as np
import pytest

import oracle.experts as X


def test_group_is_a_stable_sort():
    rng = np.random.default_rng(0)
    topk = rng.integers(-1, 7, (53, 3)).astype(np.int32)
    pos = rng.permutation(159).astype(np.int32).reshape(53, 3)
    rows, tokens, off = X.group(topk, pos, 6)
    key = np.where((topk < 0) | (topk >= 6), 6, topk).reshape(-1)
    order = np.argsort(key, kind="stable")
    n = int((key < 6).sum())
    assert np.array_equal(rows[:n], pos.reshape(-1)[order[:n]]) and (rows[n:] == -1).all()
    assert np.array_equal(tokens[:n], order[:n] // 3) and (tokens[n:] == -1).all()
    assert np.array_equal(off, np.searchsorted(key[order], np.arange(7)))


@pytest.mark.parametrize("kind", [X.SILU, X.GELU])
def test_slope_is_the_activations_derivative(kind):
    g = np.linspace(-9, 9, 301)
    e = 1e-5
    num = (X.act(g + e, kind) - X.act(g - e, kind)) / (2 * e)
    # the second-order difference is off by e^2 a'''/6 and by rounding 2^-52 |a| / e
    assert np.abs(num - X.act_slope(g, kind)).max() < 1e-9


@pytest.mark.parametrize("kind", [X.SILU, X.GELU])
def test_gradients_against_differences(kind):
    """The block's gradients as the library's calls compose them, against
    central differences of a loss sum(c * out)."""
    rng = np.random.default_rng(1)
    d, f, off = 5, 4, np.array([0, 3, 3, 7])
    x, w_in = rng.standard_normal((7, d)), rng.standard_normal((3, 2 * f, d))
    w_down, c = rng.standard_normal((3, d, f)), rng.standard_normal((7, d))

    def forward(x, w_in, w_down):
        gu, _ = X.per_expert(x, off, w_in)
        h = X.act(gu[:, :f], kind) * gu[:, f:]
        return gu, h, X.per_expert(h, off, w_down)[0]

    gu, h, _ = forward(x, w_in, w_down)
    dh, _ = X.per_expert(c, off, w_down.transpose(0, 2, 1))
    dgu = np.concatenate([dh * gu[:, f:] * X.act_slope(gu[:, :f], kind),
                          dh * X.act(gu[:, :f], kind)], 1)
    grads = {"x": X.per_expert(dgu, off, w_in.transpose(0, 2, 1))[0],
             "w_in": X.outer_sums(dgu, x, off)[0], "w_down": X.outer_sums(c, h, off)[0]}
    at = {"x": x, "w_in": w_in, "w_down": w_down}
    for name, grad in grads.items():
        for _ in range(25):
            i = tuple(rng.integers(0, n) for n in grad.shape)
            e, v = 1e-5, []
            for s in (e, -e):
                moved = {k: a.copy() for k, a in at.items()}
                moved[name][i] += s
                v.append((c * forward(**moved)[2]).sum())
            assert abs((v[0] - v[1]) / (2 * e) - grad[i]) < 1e-6 * (1 + abs(grad[i])), (name, i)
    assert not grads["w_in"][1].any()  # the expert without rows


def test_quantize_by_hand():
    x = np.zeros((1, 96))
    # largest 6 = 1.5 * 2^2: scale 2^0, every value over 1 as it stands
    x[0, :12] = [6, -6, 5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, 0.26, -0.5, -0.0]
    # largest 7.9: still scale 1, saturates; 2^-3 of it in the third block
    x[0, 32:36] = [7.9, 4.9, 5.1, -7]
    x[0, 64:66] = [1, 0.15]
    codes, scales = X.quantize(x)
    assert scales.tolist() == [[127, 127, 125]]
    v = X.dequantize(codes, scales)[0]
    assert v[:12].tolist() == [6, -6, 4, 4, 2, 2, 1, 1, 0, 0.5, -0.5, 0]
    assert v[32:36].tolist() == [6, 4, 6, -6]
    assert v[64:66].tolist() == [1, 0.125]
    assert codes[0, 5] >> 4 == 8  # -0 keeps its sign


def test_quantize_extremes():
    x = np.zeros((5, 32))
    x[1, 3] = np.inf
    x[2, 3] = np.nan
    x[3, 3] = 2.0 ** -130           # below the least scale: 2^-127 * 0.125 rounds to 0
    x[4, 3] = 2.0 ** 127 * 1.9375   # the largest exponent of bf16
    codes, scales = X.quantize(x)
    assert scales[:, 0].tolist() == [0, 255, 255, 0, 252]
    v = X.dequantize(codes, scales)
    assert np.isnan(v[1:3]).all() and not v[0].any() and not v[3].any()
    assert v[4, 3] == 6 * 2.0 ** 125


def test_every_value_is_nearest():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((4, 64)) * 2.0 ** rng.integers(-20, 20, (4, 1))
    codes, scales = X.quantize(x)
    v = X.dequantize(codes, scales)
    step = np.repeat(2.0 ** (scales.astype(float) - 127), 32, -1)
    grid = X.E2M1[None, None, :] * step[..., None]
    assert np.array_equal(np.abs(v - x), np.abs(grid - x[..., None]).min(-1))
