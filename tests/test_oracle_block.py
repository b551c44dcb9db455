"""The oracle's norms around a block: against their definition on hand-made rows, and their gradients against differences."""
import numpy as np
import pytest

from oracle import block

CASES = [(post, pre, gate, with_u, with_dr) for post in block.KINDS for pre in block.KINDS for gate in (False, True)
         for with_u in (True, False) for with_dr in (True, False)
         if (with_u or (post == "none" and pre != "none" and not gate)) and (with_dr or pre != "none")]


def test_by_hand():
    x, u = np.array([[1.0, 2.0, 3.0, 6.0]]), np.array([[1.0, 1.0, -1.0, -1.0]])
    out = block.norm_forward(x, u, "rms", "layer", 1e-300, 1e-300, 2.0, {"gate": [1.0, 0.0, 1.0, 0.5]})
    np.testing.assert_allclose(out["r"], [[3.0, 2.0, 1.0, 5.0]])       # the root mean square of u is 1
    np.testing.assert_allclose(out["stats"], [[0.0, 1.0, 2.75, 1 / np.sqrt(2.1875)]])
    np.testing.assert_allclose(out["n"], (np.array([[3.0, 2.0, 1.0, 5.0]]) - 2.75) / np.sqrt(2.1875))


@pytest.mark.parametrize("post,pre,gate,with_u,with_dr", CASES)
def test_gradients_against_differences(post, pre, gate, with_u, with_dr):
    g = np.random.default_rng(7)
    rows, cols, scale, eps = 3, 7, 0.6, 1e-3
    draw = lambda *s: g.normal(size=s)
    at = {"x": draw(rows, cols), "u": draw(rows, cols) if with_u else None}
    at.update({k: draw(cols) + 1 for k in ("post_gamma", "post_beta", "pre_gamma", "pre_beta")})
    at["gate"] = draw(cols) if gate else None
    dr, dn = draw(rows, cols) if with_dr else None, draw(rows, cols) if pre != "none" else None

    def loss(a):
        o = block.norm_forward(a["x"], a["u"], post, pre, eps, eps, scale, a)
        return (0 if dr is None else (dr * o["r"]).sum()) + (0 if dn is None else (dn * o["n"]).sum())
    o = block.norm_forward(at["x"], at["u"], post, pre, eps, eps, scale, at)
    got = block.norm_backward(dr, dn, o["r"], at["u"], o["stats"], post, pre, scale, at)
    names = {"x": "dx", "u": "du"}
    for name, value in at.items():
        key = names.get(name, name)
        if value is None or key not in got:
            continue
        diff, h = np.zeros_like(value), 1e-5
        for i in np.ndindex(value.shape):
            up, down = value.copy(), value.copy()
            up[i] += h
            down[i] -= h
            diff[i] = (loss({**at, name: up}) - loss({**at, name: down})) / (2 * h)
        np.testing.assert_allclose(got[key], diff, rtol=1e-6, atol=1e-6, err_msg=name)
    if with_u and not gate:      # the gate's gradient at 1
        one = {**at, "gate": np.ones(cols)}
        diff = np.array([(loss({**one, "gate": one["gate"] + d}) - loss({**one, "gate": one["gate"] - d})) / 2e-5
                         for d in 1e-5 * np.eye(cols)])
        np.testing.assert_allclose(got["gate"], diff, rtol=1e-6, atol=1e-6)


@pytest.mark.parametrize("post,pre", [("none", "rms"), ("layer", "layer"), ("rms", "layer"), ("layer", "rms")])
def test_bounds_cover_an_evaluation_in_single_precision(post, pre):
    """numpy's pairwise fp32 sums of 640 columns pass through fewer than 40 additions."""
    g = np.random.default_rng(11)
    rows, cols, eps = 9, 640, 1e-5
    f32 = lambda t: None if t is None else t.astype(np.float32)
    x, u, dr, dn = (f32(g.normal(0.3, 2.0, size=(rows, cols))) for _ in range(4))
    p = {k: f32(g.normal(1.0, 0.3, size=cols)) for k in ("post_gamma", "post_beta", "gate", "pre_gamma", "pre_beta")}
    d = lambda t: t.astype(np.float64)
    want = block.norm_forward(d(x), d(u), post, pre, eps, eps, 0.5, p)
    bound = block.norm_forward_bound(d(x), d(u), post, pre, eps, eps, 0.5, p, 60)
    one = np.float32(1)

    def normed(t, kind):
        mean = t.mean(axis=1, keepdims=True) if kind == "layer" else np.zeros((rows, 1), np.float32)
        return (t - mean), one / np.sqrt(((t - mean) ** 2).mean(axis=1, keepdims=True) + np.float32(eps))
    v = u
    if post != "none":
        c, s = normed(u, post)
        v = c * s * p["post_gamma"] + p["post_beta"]
    r = x + np.float32(0.5) * p["gate"] * v
    c, s = normed(r, pre)
    n = c * s * p["pre_gamma"] + p["pre_beta"]
    assert r.dtype == n.dtype == np.float32
    assert np.all(np.abs(r - want["r"]) <= bound["r"])
    assert np.all(np.abs(n - want["n"]) <= bound["n"])
    assert np.all(bound["n"] <= 1e-3 * np.abs(want["n"]).max())


def test_clip():
    assert block.gradient_norm([np.array([3.0]), np.array([[4.0]])]) == 5.0
    assert block.clip_factor(5.0, 1.0) == 0.2 and block.clip_factor(5.0, 10.0) == 1.0
    assert block.clip_factor(5.0, 1.0, scale=0.1) == 0.1 and block.clip_factor(float("inf"), 1.0) == 1.0
