"""CPU: the 64-bit reference of the gated delta rule and the group norm against closed forms and differences."""
import numpy as np
import pytest

import delta_reference as dr

ORDER = ("q", "k", "v", "g", "beta", "H0")


def test_rule_gradients_are_the_differences_of_the_forward():
    s = dr.rule_inputs(1, 2, 7, 4, 3, 5, Nqk=2)
    s = {n: np.asarray(x, np.float64) for n, x in s.items()}

    def loss(s):
        y, HT, _ = dr.rule_fwd(*(s[n] for n in ORDER))
        return (y * s["dy"]).sum() + (HT * s["dHT"]).sum()

    grads = dict(zip(ORDER, dr.rule_bwd(*(s[n] for n in ORDER), s["dy"], s["dHT"])))
    r = np.random.default_rng(2)
    for n in ORDER:
        d = r.standard_normal(s[n].shape)
        h = 1e-5
        diff = (loss(dict(s, **{n: s[n] + h * d})) - loss(dict(s, **{n: s[n] - h * d}))) / (2 * h)
        # (central differences: h^2 of third derivatives, 2^-53 / h of rounding)
        assert abs(diff - (grads[n] * d).sum()) <= 1e-7 * (1 + abs(diff)), n


def test_rule_replaces_what_a_key_holds():
    """beta = 1, g = 0 and unit keys: a step makes the state answer its key with its value, whatever it held."""
    s = dr.rule_inputs(3, 1, 5, 2, 8, 4)
    k = s["k"].astype(np.float64)
    k /= np.linalg.norm(k, axis=-1, keepdims=True)
    _, HT, _ = dr.rule_fwd(s["q"], k, s["v"], 0 * s["g"], 0 * s["beta"] + 1, s["H0"])
    assert np.abs(np.einsum("bnk,bnkv->bnv", k[:, -1], HT) - s["v"][:, -1]).max() < 1e-12


@pytest.mark.parametrize("act", ["none", "silu", "gate"])
@pytest.mark.parametrize("center", [False, True])
def test_group_norm_gradients_are_the_differences_of_the_forward(act, center):
    r = np.random.default_rng(4)
    t = {"x": r.standard_normal((2, 3, 12)), "a": r.standard_normal((2, 3, 12)) if act == "gate" else None,
         "w": r.standard_normal(12), "b": r.standard_normal(12)}
    dout = r.standard_normal((2, 3, 12))
    f = lambda t: dr.group_norm(t["x"], t["a"], t["w"], t["b"], 3, 1e-3, center, act == "silu", dout)
    g = f(t)
    for n in t:
        if t[n] is None:
            continue
        d, h = r.standard_normal(t[n].shape), 1e-5
        diff = ((f(dict(t, **{n: t[n] + h * d}))["out"] - f(dict(t, **{n: t[n] - h * d}))["out"]) * dout).sum() / (2 * h)
        assert abs(diff - (g["d" + n] * d).sum()) <= 1e-7 * (1 + abs(diff)), n
