"""The fp64 oracles of the operators around the layers, against explicit
loops and central differences."""
import math

import numpy as np
import pytest

from oracle import block_norm as ON
from oracle import dense_embed as OE
from oracle import grad_clip as OG

EPS = 1e-3


def test_embed_forward_and_gradient():
    rng = np.random.default_rng(1)
    T, ids = rng.standard_normal((6, 3)), np.array([2, 5, 2, -1, 0, 6, 2])
    Y = OE.forward(ids, T, 1.5)
    for t, v in enumerate(ids):
        assert np.array_equal(Y[t], 1.5 * T[v] if 0 <= v < 6 else np.zeros(3))
    dY = rng.standard_normal(Y.shape)
    dT = OE.backward(ids, dY, 6, 1.5)
    # <Y, dY> is linear in T
    for v in range(6):
        for c in range(3):
            E = np.zeros_like(T)
            E[v, c] = 1.0
            assert dT[v, c] == pytest.approx(float(np.sum(OE.forward(ids, E, 1.5) * dY)), abs=1e-12)
    assert not OE.backward(ids, dY, 6, 1.5, pad=2)[2].any()


def _norm_inputs(rng, b, n, post, pre, gate):
    d = {"X": rng.standard_normal((b, n)), "F": rng.standard_normal((b, n))}
    d["post_w"], d["post_b"] = (1 + 0.3 * rng.standard_normal((2, n))) if post != "none" else (None, None)
    d["pre_w"], d["pre_b"] = (1 + 0.3 * rng.standard_normal((2, n))) if pre != "none" else (None, None)
    d["gate"] = None if gate == "none" else rng.standard_normal(n if gate == "channel" else (b, n))
    return d


@pytest.mark.parametrize("post", ["none", "rms", "layer"])
@pytest.mark.parametrize("pre", ["none", "rms", "layer"])
@pytest.mark.parametrize("gate", ["none", "channel", "token"])
def test_norm_gradient_by_differences(post, pre, gate):
    rng = np.random.default_rng(2)
    b, n, a, beta = 2, 5, 0.9, 0.7
    d = _norm_inputs(rng, b, n, post, pre, gate)
    CX, CH = rng.standard_normal((2, b, n))

    def fwd(**k):
        v = {**d, **k}
        return ON.forward(v["X"], v["F"], post, v["post_w"], v["post_b"], v["gate"], pre, v["pre_w"], v["pre_b"], EPS,
                          a, beta)

    def loss(**k):
        Xn, H = fwd(**k)
        return float(np.sum(Xn * CX) + (np.sum(H * CH) if H is not None else 0.0))

    Xn, _ = fwd()
    got = ON.backward(Xn, d["F"], post, d["post_w"], d["post_b"], d["gate"], pre, d["pre_w"], CX,
                      None if pre == "none" else CH, EPS, a, beta)
    for name in ("X", "F", "gate", "post_w", "post_b", "pre_w", "pre_b"):
        if d[name] is None:
            continue
        for i in np.ndindex(d[name].shape):
            h, v = 1e-5, []
            for sign in (1, -1):
                x = d[name].copy()
                x[i] += sign * h
                v.append(loss(**{name: x}))
            assert got["d" + name][i] == pytest.approx((v[0] - v[1]) / (2 * h), abs=1e-7), (name, i)


def test_norm_without_a_block_before():
    rng = np.random.default_rng(3)
    X = rng.standard_normal((3, 4))
    Xn, H = ON.forward(X, None, "none", None, None, None, "rms", None, None, 0.0 + EPS, 0.5, 2.0)
    assert Xn is X
    assert np.allclose(H[1], X[1] / math.sqrt(np.mean(X[1] ** 2) + EPS))


def test_clip():
    g = [np.array([3.0]), np.zeros(0), np.array([[0.0, -4.0]])]
    n, out = OG.clip(g, 2.0, 5.0)
    assert n == 10.0 and out[0][0] == 3.0 and out[2][0, 1] == -4.0
    n, out = OG.clip(g, 1.0, 5.0)
    assert n == 5.0 and out[0][0] == 3.0
    n, out = OG.clip([np.array([math.inf, 1.0])], 2.0, 1.0)
    assert math.isnan(n) and out[0][1] == 2.0
