"""Pins of the layer oracle: closed forms, invariants and a second way of computing the same thing (CPU)."""
import math

import numpy as np
import pytest

from oracle import layer_oracle as L


def test_norms_closed_forms():
    x = np.array([3.0, 4.0, 0.0, 0.0])
    np.testing.assert_allclose(L.norm(x, "rms", np.ones(4), eps=0.0), x / 2.5)
    np.testing.assert_allclose(L.norm([1.0, -1.0], "layer", np.ones(2), np.array([1.0, 2.0]), eps=0.0), [2.0, 1.0])
    np.testing.assert_allclose(L.norm(x, "rms", np.zeros(4), eps=0.0, w0=1.0), x / 2.5)
    assert np.all(L.norm(np.zeros(4), "rms", np.ones(4)) == 0)


def test_norm_residual_composes():
    g = np.random.default_rng(0)
    res, y, gate = g.normal(size=(3, 8)), g.normal(size=(3, 8)), g.normal(size=8)
    r, h = L.norm_residual(res, y, gate, pre_w=np.ones(8), post="none", res_scale=2.0, out_scale=0.5, gate_act="tanh")
    np.testing.assert_allclose(r, 2 * res + 0.5 * np.tanh(gate) * y)
    np.testing.assert_allclose((h * h).mean(1), 1.0, rtol=1e-5)
    r, h = L.norm_residual(res, pre="none")
    assert np.array_equal(r, res) and np.array_equal(h, res)


@pytest.mark.parametrize("style", ["half", "pairs"])
def test_rotation_keeps_lengths_and_adds_angles(style):
    g = np.random.default_rng(1)
    x, a, b = g.normal(size=10), g.normal(size=4), g.normal(size=4)
    once = L.rotate(L.rotate(x, np.cos(a), np.sin(a), style), np.cos(b), np.sin(b), style)
    np.testing.assert_allclose(once, L.rotate(x, np.cos(a + b), np.sin(a + b), style), atol=1e-12)
    assert math.isclose(np.linalg.norm(once), np.linalg.norm(x)) and np.array_equal(once[8:], x[8:])
    quarter = L.rotate(np.arange(4.0), np.zeros(2), np.ones(2), style)
    np.testing.assert_allclose(quarter, [-2, -3, 0, 1] if style == "half" else [-1, 0, -3, 2])


def test_append_then_gather_gives_the_tokens_back():
    g = np.random.default_rng(2)
    k, v, q = g.normal(size=(7, 2, 4)), g.normal(size=(7, 2, 4)), g.normal(size=(7, 4, 4))
    table = np.array([[3, 1], [0, 2]])
    kp, vp, _ = L.kv_append(np.zeros((4, 2, 4, 4)), np.zeros((4, 2, 4, 4)), [0, 5, 7], [5, 2], table, 9, q, k, v)
    assert np.array_equal(L.gather(kp, table[0], 5), k[:5]) and np.array_equal(L.gather(vp, table[1], 2), v[5:])
    kp, vp, qo = L.kv_append(np.zeros((4, 2, 4, 4)), np.zeros((4, 2, 4, 4)), [0, 5, 7], [3, 2], table, 9, q, k, v)
    assert np.all(qo[:2] == 0) and np.array_equal(L.gather(kp, table[0], 3), k[2:5])     # two rows of padding in front


def test_attention_against_a_mask_over_everything_and_invariants():
    g = np.random.default_rng(3)
    q, kp, vp = g.normal(size=(4, 4, 8)), g.normal(size=(5, 2, 4, 8)), g.normal(size=(5, 2, 4, 8))
    args = (np.array([0, 1, 4]), np.array([2, 6]), np.array([[1, 0], [3, 2]]), np.array([4]), 3, 0.3)
    out, mass = L.attention(q, kp, vp, *args)
    flat_k = np.concatenate([kp[p].transpose(1, 0, 2) for p in (4, 3, 2)])              # prefix page, then the second sequence's
    flat_v = np.concatenate([vp[p].transpose(1, 0, 2) for p in (4, 3, 2)])
    for t, seen in ((1, 4), (2, 5), (3, 6)):
        ok = np.array([i < 3 or 4 <= i < 4 + seen for i in range(12)])
        for h in range(4):
            w = np.where(ok, np.exp(flat_k[:, h // 2] @ q[t, h] * 0.3), 0.0)
            np.testing.assert_allclose(out[t, h], (w / w.sum()) @ flat_v[:, h // 2])
    np.testing.assert_allclose(L.attention(q, kp, np.ones_like(vp), *args)[0], 1.0)
    assert np.all(mass >= np.abs(out) - 1e-12)
    nothing = L.attention(q[:1], kp, vp, np.array([0, 1]), np.array([0]), np.zeros((1, 1), int), np.zeros(0, int), 0, 1.0)[0]
    assert np.all(nothing == 0)


def test_planted_mistakes_are_seen():
    g = np.random.default_rng(4)
    q, kp, vp = g.normal(size=(2, 2, 8)), g.normal(size=(2, 1, 4, 8)), g.normal(size=(2, 1, 4, 8))
    good = L.attention(q, kp, vp, [0, 2], [3], np.array([[1]]), np.array([0]), 4, 0.3)[0]
    for wrong in (L.attention(q, kp, vp, [0, 2], [4], np.array([[1]]), np.array([0]), 4, 0.3)[0],    # sees one token more
                  L.attention(q, kp, vp, [0, 2], [3], np.array([[1]]), np.array([0]), 3, 0.3)[0],    # one prefix token less
                  L.attention(q, kp, vp, [0, 2], [3], np.array([[0]]), np.array([0]), 4, 0.3)[0],    # the wrong page
                  L.attention(q, kp, vp, [0, 2], [3], np.array([[1]]), np.array([0]), 4, 0.31)[0]):
        assert np.abs(wrong - good).max() > 1e-3
