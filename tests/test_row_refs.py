"""The 64-bit forms of the row operators against differences, and against values worked out by hand."""
import math

import numpy as np
import pytest

from tests import row_refs as refs


def _slopes(f, x, aim, step=1e-5):
    """d sum(aim * f(x)) / dx by central differences"""
    out = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        hi, lo = x.copy(), x.copy()
        hi[i] += step
        lo[i] -= step
        out[i] = ((f(hi) - f(lo)) * aim).sum() / (2 * step)
    return out


# central differences of functions whose third derivatives are below 100 here: 100 step^2 / 6 of truncation, and 1e-16 / step of rounding
NEAR = dict(rtol=1e-7, atol=5e-9)


@pytest.mark.parametrize("rows,cols", [(1, 5), (4, 7)])
def test_layer_norm_gradients(rows, cols):
    rng = np.random.default_rng(rows)
    x, res, dy, more = (rng.standard_normal((rows, cols)) for _ in range(4))
    w, b = rng.standard_normal(cols), rng.standard_normal(cols)
    got = refs.layer_norm(x, res, w, b)
    t, mean, rstd = got["total"][0], got["mean"][0], got["rstd"][0]
    grad = refs.layer_norm_backward(dy, t, mean, rstd, w, more)
    want = _slopes(lambda v: refs.layer_norm(v, res, w, b)["y"][0], x, dy) + more
    np.testing.assert_allclose(grad["dx"][0], want, **NEAR)
    np.testing.assert_allclose(grad["dweight"][0], _slopes(lambda v: refs.layer_norm(x, res, v, b)["y"][0], w, dy), **NEAR)
    np.testing.assert_allclose(grad["dbias"][0], _slopes(lambda v: refs.layer_norm(x, res, w, v)["y"][0], b, dy), **NEAR)


def test_layer_norm_by_hand():
    got = refs.layer_norm(np.array([[1.0, 3.0]]), None, np.array([2.0, 2.0]), np.array([0.0, 1.0]), eps=0.0)
    assert got["y"][0].tolist() == [[-2.0, 3.0]] and got["mean"][0].tolist() == [2.0] and got["rstd"][0].tolist() == [1.0]


@pytest.mark.parametrize("tanh", [False, True])
def test_gelu_gradients(tanh):
    rng = np.random.default_rng(3)
    x, dy, b = rng.standard_normal((3, 6)) * 2, rng.standard_normal((3, 6)), rng.standard_normal(6)
    grad = refs.bias_gelu_backward(dy, x, b, tanh)
    np.testing.assert_allclose(grad["dx"][0], _slopes(lambda v: refs.bias_gelu(v, b, tanh)["y"][0], x, dy), **NEAR)
    np.testing.assert_allclose(grad["dbias"][0], _slopes(lambda v: refs.bias_gelu(x, v, tanh)["y"][0], b, dy), **NEAR)


def test_gelu_by_hand():
    x = np.array([[0.0, 1.0, -1.0]])
    assert refs.bias_gelu(x)["y"][0][0, 0] == 0.0
    np.testing.assert_allclose(refs.bias_gelu(x)["y"][0][0, 1:], [0.8413447460685429, -0.15865525393145707], rtol=1e-14)
    th = math.tanh(math.sqrt(2 / math.pi) * 1.044715)
    np.testing.assert_allclose(refs.bias_gelu(x, tanh=True)["y"][0][0, 1:], [0.5 * (1 + th), -0.5 * (1 - th)], rtol=1e-14)


@pytest.mark.parametrize("T", [1.0, 2.5])
def test_distill_gradient(T):
    rng = np.random.default_rng(7)
    z, t = rng.standard_normal((4, 9)) * 2, rng.standard_normal((4, 3)) * 2
    index = np.array([[0, 4, 8], [2, 2, 5], [-1, 3, 9], [-1, -1, 77]])          # distinct, one twice, one entry, none
    w = np.array([1.0, 0.5, -2.0, 1.0])
    got = refs.distill(z, t, index, T, w)
    want = _slopes(lambda v: refs.distill(v, t, index, T)["loss"][0][:, None], z, w[:, None])
    np.testing.assert_allclose(got["dlogits"][0], want, **NEAR)
    assert got["loss"][0][3] == 0 and not got["dlogits"][0][3].any()
    np.testing.assert_allclose(got["dlogits"][0].sum(1), 0, atol=1e-12)


def test_distill_by_hand():
    # the teacher halves its mass between two of four columns that are all alike to the student: log 2 and q - p
    got = refs.distill(np.zeros((1, 4)), np.zeros((1, 2)), np.array([[1, 3]]), 1.0)
    np.testing.assert_allclose(got["loss"][0], [math.log(2.0)], rtol=1e-15)
    np.testing.assert_allclose(got["dlogits"][0], [[0.25, -0.25, 0.25, -0.25]], rtol=1e-15)
    # a teacher's list that holds what the student says itself, the whole of it: nothing to learn
    z = np.array([[1.0, -2.0, 0.5]])
    got = refs.distill(z, z, np.array([[0, 1, 2]]), 3.0)
    np.testing.assert_allclose(got["loss"][0], [0.0], atol=1e-14)
    np.testing.assert_allclose(got["dlogits"][0], np.zeros((1, 3)), atol=1e-15)
    # a masked column has no share and costs nothing unless the teacher wants it
    z = np.array([[0.0, -np.inf, 0.0]])
    assert np.isfinite(refs.distill(z, np.zeros((1, 1)), np.array([[0]]), 1.0)["loss"][0]).all()
    got = refs.distill(z, np.zeros((1, 1)), np.array([[1]]), 1.0)
    assert got["loss"][0][0] == np.inf and got["dlogits"][0].tolist() == [[0.5, -1.0, 0.5]]
