"""The gated delta rule, the group norm and the windowed convolution in 64 bits (numpy), from their formulas,
and inputs for them.  Gradients of the rule step by step backwards; tests/test_delta_reference.py holds them
to differences of the forward."""
import numpy as np


def rule_fwd(q, k, v, g, beta, H0=None):
    """q, k [B,T,Nqk,K], v [B,T,N,V], g, beta [B,T,N] -> y [B,T,N,V], HT [B,N,K,V], tape."""
    B, T, N, V = v.shape
    K, rep = q.shape[3], N // q.shape[2]
    q, k = np.repeat(q, rep, 2).astype(np.float64), np.repeat(k, rep, 2).astype(np.float64)
    H = np.zeros((B, N, K, V)) if H0 is None else np.asarray(H0, np.float64)
    y, tape = np.zeros((B, T, N, V)), []
    for t in range(T):
        Hd = np.exp(np.asarray(g[:, t], np.float64))[..., None, None] * H
        delta = v[:, t] - np.matmul(k[:, t, :, None], Hd)[:, :, 0]
        H = Hd + k[:, t, ..., None] * (beta[:, t, :, None] * delta)[:, :, None]
        y[:, t] = np.matmul(q[:, t, :, None], H)[:, :, 0]
        tape.append((Hd, delta, H))
    return y, H, tape


def rule_bwd(q, k, v, g, beta, H0, dy, dHT=None):
    """dq, dk, dv, dg, dbeta, dH0."""
    B, T, N, V = v.shape
    Nqk, K = q.shape[2], q.shape[3]
    rep = N // Nqk
    _, H, tape = rule_fwd(q, k, v, g, beta, H0)
    q, k = np.repeat(q, rep, 2).astype(np.float64), np.repeat(k, rep, 2).astype(np.float64)
    dH = np.zeros((B, N, K, V)) if dHT is None else np.asarray(dHT, np.float64)
    dq, dk, dv = np.zeros((B, T, N, K)), np.zeros((B, T, N, K)), np.zeros((B, T, N, V))
    dg, db = np.zeros((B, T, N)), np.zeros((B, T, N))
    for t in range(T - 1, -1, -1):
        Hd, delta, H = tape[t]
        bt, y = beta[:, t, :, None].astype(np.float64), dy[:, t].astype(np.float64)
        dq[:, t] = np.matmul(H, y[..., None])[..., 0]
        dH = dH + q[:, t, ..., None] * y[:, :, None]
        du = np.matmul(k[:, t, :, None], dH)[:, :, 0]
        db[:, t] = (du * delta).sum(-1)
        dv[:, t] = bt * du
        dk[:, t] = np.matmul(dH, (bt * delta)[..., None])[..., 0] - np.matmul(Hd, dv[:, t][..., None])[..., 0]
        dH = dH - k[:, t, ..., None] * dv[:, t][:, :, None]
        dg[:, t] = (dH * Hd).sum((-1, -2))
        dH = np.exp(np.asarray(g[:, t], np.float64))[..., None, None] * dH
    share = lambda x: x.reshape(B, T, Nqk, rep, K).sum(3)
    return share(dq), share(dk), dv, dg, db, dH


def bf16(x):
    """Rounded to bfloat16, to nearest even."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)


def rule_inputs(seed, B, T, N, K, V, Nqk=None, io="f32", carry=True, memory=20.0):
    """Keys of unit length, gates of a memory of about `memory` steps; io tensors as they are stored."""
    r = np.random.default_rng(seed)
    Nqk = Nqk or N
    unit = lambda x: x / np.linalg.norm(x, axis=-1, keepdims=True)
    st = bf16 if io == "bf16" else (lambda x: np.asarray(x, np.float32))
    s = {"q": st(unit(r.standard_normal((B, T, Nqk, K))) * K ** -0.5), "k": st(unit(r.standard_normal((B, T, Nqk, K)))),
         "v": st(r.standard_normal((B, T, N, V))), "dy": st(r.standard_normal((B, T, N, V))),
         "g": (-np.exp(0.5 * r.standard_normal((B, T, N))) / memory).astype(np.float32),
         "beta": (1 / (1 + np.exp(-r.standard_normal((B, T, N))))).astype(np.float32), "H0": None, "dHT": None}
    if carry:
        s["H0"] = (0.3 * r.standard_normal((B, N, K, V))).astype(np.float32)
        s["dHT"] = (0.3 * r.standard_normal((B, N, K, V))).astype(np.float32)
    return s


RULE_NAMES = ("dq", "dk", "dv", "dg", "dbeta", "dH0")


def rule(s):
    """y, HT and the gradients, by name."""
    y, HT, _ = rule_fwd(s["q"], s["k"], s["v"], s["g"], s["beta"], s["H0"])
    grads = rule_bwd(s["q"], s["k"], s["v"], s["g"], s["beta"], s["H0"], s["dy"], s["dHT"])
    return dict(zip(RULE_NAMES, grads), y=y, HT=HT)


def silu(z):
    return z / (1 + np.exp(-z))


def silu_slope(z):
    s = 1 / (1 + np.exp(-z))
    return s * (1 + z * (1 - s))


def group_norm(x, a, w, b, groups, eps, center, act_silu, dout=None):
    """out, and with dout also dx, da, dw, db, by name."""
    B, T, D = x.shape
    x = x.astype(np.float64).reshape(B, T, groups, D // groups)
    wg = np.ones(D) if w is None else w.astype(np.float64)
    bg = np.zeros(D) if b is None else b.astype(np.float64)
    xc = x - (x.mean(-1, keepdims=True) if center else 0.0)
    s = 1 / np.sqrt((xc * xc).mean(-1, keepdims=True) + eps)
    xh = (xc * s).reshape(B, T, D)
    n = xh * wg + bg
    a = None if a is None else a.astype(np.float64)
    out = silu(n) if act_silu else n if a is None else n * silu(a)
    res = {"out": out}
    if dout is None:
        return res
    d = dout.astype(np.float64)
    dn = d * silu_slope(n) if act_silu else d if a is None else d * silu(a)
    if a is not None:
        res["da"] = d * n * silu_slope(a)
    p, h = (dn * wg).reshape(x.shape), xh.reshape(x.shape)
    dx = p - h * (p * h).mean(-1, keepdims=True) - (p.mean(-1, keepdims=True) if center else 0.0)
    res.update(dx=(dx * s).reshape(B, T, D), dw=(dn * xh).sum((0, 1)), db=dn.sum((0, 1)))
    return res


def conv_window(x, w, bias, win):
    """out, and the window behind the last step."""
    B, T, C = x.shape
    xx = np.concatenate([np.zeros((B, 3, C)) if win is None else win.astype(np.float64), x.astype(np.float64)], 1)
    u = sum(xx[:, j:j + T] * w[:, j].astype(np.float64) for j in range(4))
    return silu(u + (0.0 if bias is None else bias.astype(np.float64))), xx[:, T:]
