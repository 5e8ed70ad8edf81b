"""GPU: the gated delta rule on magnitudes far from one.

The rule is linear in (v, H0) and its gradients in (dy, dHT), so inputs times a power of two give results times that
power, to the bit as long as nothing leaves the range of fp32: no tolerance is needed there.  Where inputs of unlike
size meet, the 64-bit reference at the tolerances of the small tests, of the largest entry that a tensor has met."""
import numpy as np
import pytest

import delta_reference as dr
import gpu_util as gu
import test_gpu_delta as small

pytestmark = pytest.mark.gpu

# columns of V per workgroup: 16 (few states) and 32
SIZES = [(2, 130, 3, 64, 64), (2, 70, 2, 128, 32), (3, 65, 2, 32, 256), (33, 66, 4, 64, 32), (17, 70, 2, 128, 128)]


def times(s, **exponents):
    return {n: x if n not in exponents or x is None else x * np.float32(2.0 ** exponents[n]) for n, x in s.items()}


def same_but_for(got, base, **exponents):
    import torch
    for n, x in base.items():
        want = x * 2.0 ** exponents.get(n, 0)
        assert torch.isfinite(got[n]).all() and torch.equal(got[n], want), (n, float((got[n].float() - want.float()).abs().max()))


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,N,K,V", SIZES)
def test_values_and_states_of_any_size(io, B, T, N, K, V):
    """From 2^-60 to 2^60."""
    s = dr.rule_inputs(61, B, T, N, K, V, io=io)
    base = small.run(s, io)
    for e in (-60, -20, 13, 60):
        print("case", io, B, T, N, K, V, e, flush=True)
        got = small.run(times(s, v=e, H0=e), io, use_ckpt=e != 13)
        same_but_for(got, base, **dict.fromkeys(("y", "HT", "dq", "dk", "dg", "dbeta"), e))


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,N,K,V", SIZES)
def test_gradients_of_any_size(io, B, T, N, K, V):
    """From 2^-60 to 2^110: the results are linear in (dy, dHT)."""
    s = dr.rule_inputs(64, B, T, N, K, V, io=io)
    base = small.run(s, io)
    for e in (-60, -20, 13, 60, 110):
        print("case", io, B, T, N, K, V, e, flush=True)
        got = small.run(times(s, dy=e, dHT=e), io, use_ckpt=e != 13)
        same_but_for(got, base, **dict.fromkeys(("dq", "dk", "dv", "dg", "dbeta", "dH0"), e))


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,N,K,V", SIZES)
@pytest.mark.parametrize("e", [-60, -13, 13, 60])
def test_queries_of_any_size(io, B, T, N, K, V, e):
    """(Entries of q far below its largest are not always exact as fp16, so the bits may differ.)"""
    s = times(dr.rule_inputs(65, B, T, N, K, V, io=io), q=e, dHT=e)
    small.check(small.run(s, io), dr.rule(s), (io, B, T, N, K, V, e))


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,N,K,V", SIZES)
@pytest.mark.parametrize("e", [-20, -10, 10, 20])
def test_keys_of_any_size(io, B, T, N, K, V, e):
    """Betas that make up for it: u is 2^-2e, the state 2^-e of what it is with unit keys."""
    s = times(dr.rule_inputs(68, B, T, N, K, V, io=io), k=e, beta=-2 * e, H0=-e, dHT=e)
    small.check(small.run(s, io), dr.rule(s), (io, B, T, N, K, V, e))


@pytest.mark.parametrize("T", [13, 65, 130])
def test_queries_that_add_up(T):
    """Products q.k of thousands, the same query and loss at every step: dU is the sum of all of them."""
    s = dr.rule_inputs(66, 2, T, 3, 64, 64, io="bf16")
    s["k"][:, ::2] = 0.125
    s["q"][:] = 1000
    s["dy"][:] = 1
    s["g"][:] = s["g"] * np.float32(0.05)
    want, got = dr.rule(s), small.run(s, "bf16")
    # the aligned keys take most of Q^T e^G dY away again: dH0 is the difference of it and K^T e^G dV, sums over a
    # chunk of up to sum_t |q_t dy_t| an entry, each off by F32 of that
    err = np.abs(gu.to_np(got["dH0"]) - want.pop("dH0")).max()
    assert err <= small.F32 * 1000 * min(T, 64), err
    small.check(got, want, T)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("e", [20, 60])
def test_dq_beside_a_large_gradient_of_the_state(io, e):
    """dq_t = H_t dy_t has nothing to do with dHT."""
    s = dr.rule_inputs(67, 2, 100, 3, 64, 64, io=io)
    base, got = small.run(s, io), small.run(times(s, dHT=e), io)
    import torch
    assert torch.equal(got["dq"], base["dq"])


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("T", [12, 13, 65, 130])
@pytest.mark.parametrize("size", [1e4, 1.9e4])
def test_a_state_along_a_key(io, T, size):
    """k^T H and with it the updates are sqrt(K) times larger than the state."""
    s = dr.rule_inputs(62, 2, T, 3, 64, 64, io=io)
    s["H0"][:] = size
    s["k"][:, ::5] = 0.125
    s["g"][:] = s["g"] * np.float32(0.05)
    want = dr.rule(s)
    got = small.run(s, io)
    # (the final state is what is left of one of `size`: its error is one of that)
    err = np.abs(gu.to_np(got["HT"]) - want.pop("HT")).max()
    assert err <= small.F32 * size, err
    # dg = <dH, e^g H> is formed from sums over the chunk's steps of q.(H dy) and -k.(H dv), which cancel.  bf16 io: H in
    # them is one fp16 value, off by at most 2^-12 of the largest state, each entry on its own; such errors E make
    # sum_t q_t.(E dy_t) of a standard deviation of at most 2^-12 max|H| sqrt(sum_t |q_t|^2 |dy_t|^2), and k, dv
    # likewise.  Four of them, beside what every bf16 result may be off.
    if io == "bf16":
        dg, norm2 = want.pop("dg"), lambda n: (s.get(n, want.get(n)).astype(np.float64) ** 2).sum(-1)
        per_step = norm2("q") * norm2("dy") + norm2("k") * norm2("dv")
        chunk = max(per_step[:, t:t + 64].sum(1).max() for t in range(0, T, 64))
        lim = small.BF16 * (np.abs(dg) + np.abs(dg).max()) + 4 * 2.0 ** -12 * size * chunk ** 0.5
        assert (np.abs(gu.to_np(got["dg"]) - dg) <= lim).all(), (T, size)
    small.check(got, want, (io, T, size))
    y = gu.to_np(small.run(s, io, backward=False)["y"])
    assert np.abs(y - want["y"]).max() <= 2 * small.BF16 * np.abs(want["y"]).max()


@pytest.mark.parametrize("bad", [np.inf, np.nan])
@pytest.mark.parametrize("where", ["dy", "dHT", "v", "H0"])
@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_what_is_not_finite_stays_in_its_column(io, where, bad):
    """One infinity or NaN: y, HT, dv, dH0 of the other columns are as if it had not been there, and so is all of the
    other heads and batch rows; what it reaches is not finite."""
    B, T, N, V, t, col = 2, 200, 3, 64, 100, 5
    s = dr.rule_inputs(63, B, T, N, 64, V, io=io)
    want = dr.rule(s)
    if where in ("dy", "v"):
        s[where][1, t, 2, col] = bad
    else:
        s[where][1, 2, 7, col] = bad
    got = small.run(s, io)
    top = {n: np.abs(w).max() for n, w in want.items()}
    for n, w in want.items():
        g = gu.to_np(got[n])
        ok = np.ones(w.shape, bool)  # what has to be right
        if n in ("y", "dv"):
            ok[1, :, 2, col] = False
        elif n in ("HT", "dH0"):
            ok[1, 2, :, col] = False
        else:
            ok[1, :, 2] = False
            if n == "dq" and where in ("dy", "dHT"):  # (dq_t is H_t dy_t: of one step, or of none)
                ok[1, :, 2] = True
                ok[1, t, 2] = where == "dHT"
        lim = small.BF16 * (np.abs(w) + top[n]) if "bfloat16" in str(got[n].dtype) else np.full(w.shape, small.F32 * top[n])
        assert np.isfinite(g[ok]).all() and (np.abs(g - w)[ok] <= lim[ok]).all(), (n, float(np.nanmax(np.abs(g - w)[ok] / lim[ok])))
    g = {n: gu.to_np(x) for n, x in got.items()}
    if where in ("dy", "dHT"):
        assert not np.isfinite(g["dH0"][1, 2, :, col]).all() and not np.isfinite(g["dv"][1, :t - 63, 2, col]).any()
        assert not np.isfinite(g["dk"][1, :t - 63, 2]).all(-1).any()
    else:
        assert not np.isfinite(g["HT"][1, 2, :, col]).all() and not np.isfinite(g["y"][1, t:, 2, col]).any()


# (B, N, K, V): 16 and 32 columns of V per workgroup, all sizes of K
LONG = [(2, 3, 64, 64), (2, 2, 128, 32), (3, 2, 32, 256), (33, 4, 64, 32), (17, 2, 128, 128), (33, 4, 32, 32)]


def check_chunks(got, want, names, label):
    """Every 64 steps by the largest entry there."""
    for t in range(0, want["y"].shape[1], 64):
        small.check({n: got[n][:, t:t + 64] for n in names}, {n: want[n][:, t:t + 64] for n in names}, (label, t))


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("B,N,K,V", LONG)
@pytest.mark.parametrize("first,last", [(128, 192), (0, 64), (256, 300)])
def test_keys_and_queries_far_from_one_in_some_steps(io, B, N, K, V, first, last):
    """... between chunks where they are near it."""
    print("case", io, B, N, K, V, first, flush=True)
    s = dr.rule_inputs(69, B, 300, N, K, V, io=io)
    s["q"][:, first:last] *= np.float32(2.0 ** -14)
    s["k"][:, first:last] *= np.float32(2.0 ** -9)
    s["beta"][:, first:last] *= np.float32(2.0 ** 18)
    s["v"][:, first:last] *= np.float32(2.0 ** -9)
    want, got = dr.rule(s), small.run(s, io)
    small.check({n: got[n] for n in ("HT", "dH0")}, {n: want[n] for n in ("HT", "dH0")}, (io, "states"))
    check_chunks(got, want, ("y", "dq", "dv"), (io, K, V, first))


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("B,N,K,V", LONG)
def test_states_and_gradients_that_change_their_size(io, B, N, K, V):
    """v and dy 2^20 times larger for some steps, a reset behind them: both recurrences go up and down again."""
    print("case", io, B, N, K, V, flush=True)
    s = dr.rule_inputs(70, B, 400, N, K, V, io=io)
    for n in ("v", "dy"):
        s[n][:, 150:170] *= np.float32(2.0 ** 20)
    s["g"][:, 140] = s["g"][:, 200] = -np.inf
    want, got = dr.rule(s), small.run(s, io)
    small.check({"HT": got["HT"]}, {"HT": want["HT"]}, (io, "states"))
    check_chunks(got, want, ("y", "dq"), (io, K, V))
    # bf16 io: the steps 128 to 139, which alone reach what is in front of them, share their 64 steps with losses 2^20
    # times larger and are held to 2^-25 of those, in dy and once more in Z.  What dH is off by in front of them, at
    # most the sum of |q_t| times that, twice, decays by e^g (the rule does not expand), and keys of unit length hand
    # it on to dv, times beta below one.
    lost = 2 * 2.0 ** -25 * np.abs(s["dy"]).max() * np.abs(s["q"][:, 128:140]).max(-1).sum(1).max() if io == "bf16" else 0.0
    decay = np.exp(s["g"][:, :128][:, ::-1].cumsum(1)[:, ::-1])  # from step t to 128
    off = small.F32 * np.abs(want["dH0"]).max() + lost * decay[:, 0].max()
    assert np.abs(gu.to_np(got["dH0"]) - want["dH0"]).max() <= off
    for t in range(0, 400, 64):
        g, w = gu.to_np(got["dv"][:, t:t + 64]), want["dv"][:, t:t + 64]
        more = np.abs(s["k"][:, t:t + 64]).sum(-1).max() * lost * decay[:, t:t + 64].max() if t < 128 else 0.0
        rel = small.BF16 * (np.abs(w) + np.abs(w).max()) if io == "bf16" else small.F32 * np.abs(w).max()
        assert (np.abs(g - w) <= rel + more).all(), t


@pytest.mark.parametrize("B,N,K,V", LONG)
def test_an_infinity_far_behind(B, N, K, V):
    """... in v and in dy of one column each: other columns of all chunks are right, also where the state was scaled anew."""
    s = dr.rule_inputs(73, B, 300, N, K, V, io="bf16")
    want = dr.rule(s)
    s["v"][0, 70, 0, 3], s["dy"][0, 230, 0, 9] = np.inf, -np.inf
    got = small.run(s, "bf16")
    keep = [c for c in range(V) if c not in (3, 9)]
    pick = lambda x, n: x[..., keep] if n in ("y", "dv", "HT", "dH0") else x[:, :, 1:]
    names = ("y", "dv", "HT", "dH0", "dq", "dk", "dbeta")
    small.check({n: pick(got[n], n) for n in names}, {n: pick(want[n], n) for n in names}, (K, V))


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("B,N,K,V", LONG)
def test_padding_of_zeros(io, B, N, K, V):
    """Two chunks of zeros behind a sequence and one in front: the same bits as without those behind."""
    import torch
    s = dr.rule_inputs(74, B, 300, N, K, V, io=io)
    for n in ("q", "k", "v", "dy", "g", "beta"):
        s[n][:, :64] = 0
        s[n][:, 172:] = 0
    short = {n: x if n in ("H0", "dHT") else x[:, :172] for n, x in s.items()}
    got, want = small.run(s, io), small.run(short, io)
    for n in ("HT", "dH0"):
        assert torch.equal(got[n], want[n]), n
    for n in ("y", "dq", "dv", "dk", "dg", "dbeta"):
        assert torch.equal(got[n][:, :172], want[n]), n
    small.check(want, dr.rule(short), (io, B, N, K, V))
