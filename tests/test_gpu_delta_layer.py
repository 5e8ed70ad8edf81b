"""GPU: group norm with an activation and the windowed convolution against their 64-bit formulas, and the mixer of a
gated-delta-rule layer as a program runs it: convolution, norm of q and k, rule, gated norm of each head.

Tolerances: fp32 results a few roundings and the hardware's exp2 and reciprocal (1 ulp each), sums over L <= 1024
channels in registers: 16 x 2^-24 = 1e-6 of the largest entry, 1e-5 for sums over tokens; bf16 results half a step of
their own value, 2^-8, and as much of fp32's."""
import numpy as np
import pytest

from paper_2603_14360_amd import binding as mb
import delta_reference as dr
import gpu_util as gu

pytestmark = pytest.mark.gpu

EPS = 1e-5


def dev(x, io):
    import torch
    if x is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(x, np.float32)).to("cuda")
    return t.to(torch.bfloat16) if io == "bf16" else t


def store(x, io):
    return dr.bf16(x) if io == "bf16" else np.asarray(x, np.float32)


def check(got, want, label):
    for n, w in want.items():
        g = gu.to_np(got[n])
        assert g.shape == w.shape and np.isfinite(g).all(), (label, n)
        if w.size:
            rel = 2.0 ** -8 if "bfloat16" in str(got[n].dtype) else 0.0
            top = (1e-5 if n in ("dw", "db") else 1e-6) * np.abs(w).max() + 1e-30
            assert (np.abs(g - w) <= rel * np.abs(w) + top).all(), (label, n, float((np.abs(g - w) / (rel * np.abs(w) + top)).max()))


# (B, T, groups, channels of one): single lanes to two vectors a lane, tokens side by side and in slices
SHAPES = [(2, 3, 1, 8), (3, 37, 84, 16), (2, 41, 7, 24), (1, 5, 5, 40), (2, 65, 16, 64), (2, 33, 16, 128), (1, 9, 3, 200),
          (2, 4, 2, 512), (2, 7, 1, 520), (1, 3, 4, 1024), (1, 2100, 2, 8), (2, 0, 2, 16), (1, 1, 1, 64), (1, 3, 300, 8)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,G,L", SHAPES)
@pytest.mark.parametrize("act,center,affine", [("none", False, 1), ("gate", False, 1), ("silu", True, 2), ("gate", True, 2), ("none", True, 0)])
def test_group_norm(io, B, T, G, L, act, center, affine):
    import torch
    print("case", io, B, T, G, L, act, center, affine, flush=True)
    r = np.random.default_rng(B + T + G + L)
    D = G * L
    x, dout = store(r.standard_normal((B, T, D)) + 0.3, io), store(r.standard_normal((B, T, D)), io)
    a = store(r.standard_normal((B, T, D)), io) if act == "gate" else None
    w = store(1 + 0.2 * r.standard_normal(D), io) if affine > 0 else None
    b = store(0.2 * r.standard_normal(D), io) if affine > 1 else None
    mode = (mb.M2RNN_NORM_CENTER if center else 0) | (mb.M2RNN_NORM_SILU if act == "silu" else 0)
    xd, ad, wd, bd, dd = (dev(t, io) for t in (x, a, w, b, dout))
    new = lambda: torch.full_like(xd, float("nan"))
    got = {"out": new(), "dx": new(), "da": new() if act == "gate" else None,
           "dw": torch.full((D,), float("nan"), device="cuda"), "db": torch.full((D,), float("nan"), device="cuda")}
    ws = torch.full((max(256, mb.m2rnn_group_norm_workspace_bytes(B, T, D)),), 255, dtype=torch.uint8, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    mb.m2rnn_group_norm_fwd(xd, ad, wd, bd, G, EPS, mode, got["out"], stream=st)
    mb.m2rnn_group_norm_bwd(xd, ad, wd, bd, G, EPS, mode, dd, got["dx"], got["da"], got["dw"], got["db"], ws, stream=st)
    want = dr.group_norm(x, a, w, b, G, EPS, center, act == "silu", dout)
    check(got, want, (io, B, T, G, L, act))
    # in place, and without the sums over tokens
    out, dx = xd.clone(), dd.clone()
    da = None if ad is None else ad.clone()
    mb.m2rnn_group_norm_fwd(out, ad, wd, bd, G, EPS, mode, out, stream=st)
    mb.m2rnn_group_norm_bwd(xd, da, wd, bd, G, EPS, mode, dx, dx, da, None, None, None, stream=st)
    assert torch.equal(out, got["out"]) and torch.equal(dx, got["dx"]) and (da is None or torch.equal(da, got["da"]))


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_group_norm_of_equal_channels(io):
    """No variance: nothing but the bias is left, and gradients stay finite."""
    import torch
    x = dev(np.full((2, 3, 64), 0.75), io)
    b = dev(np.arange(64) / 64, io)
    out, dx = torch.empty_like(x), torch.empty_like(x)
    mb.m2rnn_group_norm_fwd(x, None, None, b, 4, EPS, mb.M2RNN_NORM_CENTER, out)
    mb.m2rnn_group_norm_bwd(x, None, None, b, 4, EPS, mb.M2RNN_NORM_CENTER, x, dx, None, None, None, None)
    assert torch.equal(out, b.expand_as(out)) and not dx.any()


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,C,bias,win", [(3, 1, 8, True, True), (2, 2, 24, False, True), (2, 3, 64, True, True), (5, 4, 1472, True, True),
                                            (2, 37, 520, False, True), (1, 200, 64, True, False), (64, 1, 1472, True, True), (2, 0, 16, True, True)])
def test_window(io, B, T, C, bias, win):
    import torch
    print("case", io, B, T, C, flush=True)
    r = np.random.default_rng(B + T + C)
    x, w = store(r.standard_normal((B, T, C)), io), store(0.5 * r.standard_normal((C, 4)), io)
    bs = store(0.5 * r.standard_normal(C), io) if bias else None
    wn = store(r.standard_normal((B, 3, C)), io) if win else None
    xd, wd, bd, nd = (dev(t, io) for t in (x, w, bs, wn))
    st = torch.cuda.current_stream().cuda_stream
    out, nxt = torch.full_like(xd, float("nan")), torch.full((B, 3, C), float("nan"), dtype=xd.dtype, device="cuda")
    mb.m2rnn_conv_silu_window_fwd(xd, wd, bd, nd, out, nxt, stream=st)
    wo, wl = dr.conv_window(x, w, bs, wn)
    check({"out": out}, {"out": wo}, (io, B, T, C))
    assert (gu.to_np(nxt) == wl).all()
    if win:  # in place
        out2 = torch.empty_like(out)
        mb.m2rnn_conv_silu_window_fwd(xd, wd, bd, nd, out2, nd, stream=st)
        assert torch.equal(out2, out) and torch.equal(nd, nxt)
    elif T:  # from zeros: the call without a window
        plain = torch.empty_like(out)
        mb.m2rnn_conv_silu_fwd(xd, wd, bd, plain, stream=st)
        assert torch.equal(plain, out)


class Mixer:
    """x -> conv -> q, k, v -> unit q, k -> rule -> norm of each head times SiLU(a)."""

    def __init__(self, N, K, V, io, seed=30):
        r = np.random.default_rng(seed)
        self.N, self.K, self.V, self.io, self.C = N, K, V, io, N * (2 * K + V)
        self.np = {"w": store(0.5 * r.standard_normal((self.C, 4)), io), "bias": store(0.1 * r.standard_normal(self.C), io),
                   "wn": store(1 + 0.1 * r.standard_normal(N * V), io), "unit": store(np.full(N * K, K ** -0.5), io)}
        self.d = {n: dev(x, io) for n, x in self.np.items()}

    def run(self, x, g, beta, a, state, win, backward=None):
        """One segment; state and window are carried in place.  With backward = dout: (out, grads)."""
        import torch
        B, T = x.shape[:2]
        N, K, V, io, d = self.N, self.K, self.V, self.io, self.d
        st = torch.cuda.current_stream().cuda_stream
        u = torch.empty_like(x)
        mb.m2rnn_conv_silu_window_fwd(x, d["w"], d["bias"], win, u, win, stream=st)
        qr, kr, v = (t.contiguous() for t in u.split([N * K, N * K, N * V], -1))
        q, k = torch.empty_like(qr), torch.empty_like(kr)
        for src, dst in ((qr, q), (kr, k)):
            mb.m2rnn_group_norm_fwd(src, None, d["unit"], None, N, 1e-6, 0, dst, stream=st)
        p = mb.Delta(B, T, N, K, V, io, backward=backward is not None)
        if state is not None:
            p.HT = state
        heads = lambda t: t.view(B, T, N, -1)
        y, HT = p.fwd(heads(q), heads(k), heads(v), g, beta, state)
        y = y.view(B, T, N * V)
        out = torch.empty_like(y)
        mb.m2rnn_group_norm_fwd(y, a, d["wn"], None, N, EPS, 0, out, stream=st)
        if backward is None:
            return out
        dy, da, dqr, dkr, dx = torch.empty_like(y), torch.empty_like(a), torch.empty_like(q), torch.empty_like(k), torch.empty_like(x)
        new = lambda *s: torch.empty(s, dtype=torch.float32, device="cuda")
        dwn, dw, db = new(N * V), new(self.C, 4), new(self.C)
        ws = torch.empty(max(mb.m2rnn_group_norm_workspace_bytes(B, T, N * V), mb.m2rnn_conv_silu_workspace_bytes(B, T, self.C)),
                         dtype=torch.uint8, device="cuda")
        mb.m2rnn_group_norm_bwd(y, a, d["wn"], None, N, EPS, 0, backward, dy, da, dwn, None, ws, stream=st)
        dq, dk, dv, dg, dbeta, _ = p.bwd(heads(q), heads(k), heads(v), g, beta, state, heads(dy))
        for src, dsrc, dst in ((qr, dq, dqr), (kr, dk, dkr)):
            mb.m2rnn_group_norm_bwd(src, None, d["unit"], None, N, 1e-6, 0, dsrc.view(B, T, N * K), dst, None, None, None, None, stream=st)
        du = torch.cat([dqr, dkr, dv.view(B, T, N * V)], -1)
        mb.m2rnn_conv_silu_bwd(x, d["w"], d["bias"], du, dx, dw, db, ws, stream=st)
        return out, {"dx": dx, "da": da, "dg": dg, "dbeta": dbeta, "dwn": dwn, "dw": dw, "db": db}

    def reference(self, x, g, beta, a, dout=None):
        """The whole layer in 64 bits on the CPU, gradients by torch's differentiation of the recurrence."""
        import torch
        N, K, V = self.N, self.K, self.V
        t = {n: torch.from_numpy(np.asarray(z, np.float64)).requires_grad_() for n, z in
             dict(x=x, g=g, beta=beta, a=a, w=self.np["w"], bias=self.np["bias"], wn=self.np["wn"]).items()}
        B, T = x.shape[:2]
        xx = torch.cat([torch.zeros(B, 3, self.C, dtype=torch.double), t["x"]], 1)
        u = sum(xx[:, j:j + T] * t["w"][:, j] for j in range(4)) + t["bias"]
        q, k, v = (u * torch.sigmoid(u)).split([N * K, N * K, N * V], -1)
        unit = lambda z: z / (z.square().mean(-1, keepdim=True) + 1e-6).sqrt() * K ** -0.5
        q, k, v = unit(q.view(B, T, N, K)), unit(k.view(B, T, N, K)), v.view(B, T, N, V)
        H, ys = torch.zeros(B, N, K, V, dtype=torch.double), []
        for i in range(T):
            H = torch.exp(t["g"][:, i])[..., None, None] * H
            e = t["beta"][:, i, :, None] * (v[:, i] - (k[:, i, ..., None] * H).sum(2))
            H = H + k[:, i, ..., None] * e[:, :, None]
            ys.append((q[:, i, ..., None] * H).sum(2))
        y = torch.stack(ys, 1)
        n = (y / (y.square().mean(-1, keepdim=True) + EPS).sqrt()).reshape(B, T, N * V) * t["wn"]
        out = n * t["a"] * torch.sigmoid(t["a"])
        if dout is None:
            return out.detach().numpy()
        names = ["x", "a", "g", "beta", "wn", "w", "bias"]
        grads = torch.autograd.grad(out, [t[n] for n in names], torch.from_numpy(np.asarray(dout, np.float64)))
        return out.detach().numpy(), dict(zip(("dx", "da", "dg", "dbeta", "dwn", "dw", "db"), (z.numpy() for z in grads)))


def mixer_inputs(m, B, T, seed):
    r = np.random.default_rng(seed)
    return (store(r.standard_normal((B, T, m.C)), m.io), (-np.exp(0.5 * r.standard_normal((B, T, m.N))) / 20).astype(np.float32),
            (1 / (1 + np.exp(-r.standard_normal((B, T, m.N))))).astype(np.float32), store(r.standard_normal((B, T, m.N * m.V)), m.io),
            store(r.standard_normal((B, T, m.N * m.V)), m.io))


def close(got, want, io, label):
    # fp32: four operators, 1e-5 each.  bf16: five tensors on the way rounded to 2^-8, and the gradients' as many
    # again; each rounding reaches a result through maps of gain near one, the norms' by up to the ratio of a head's
    # largest channel to its root mean square, below four: 2-norm 4 sqrt(10) 2^-9 (rms of a rounding 2^-9)
    lim = 4e-5 if io == "f32" else 4 * 10 ** 0.5 * 2.0 ** -9
    err = np.linalg.norm(gu.to_np(got) - want) / np.linalg.norm(want)
    assert err <= lim, (label, io, err)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("N,K,V,T", [(2, 32, 32, 75), (3, 64, 128, 130)])
def test_mixer_trains(io, N, K, V, T):
    m = Mixer(N, K, V, io)
    x, g, beta, a, dout = mixer_inputs(m, 2, T, 31)
    out, grads = m.run(dev(x, io), dev(g, "f32"), dev(beta, "f32"), dev(a, io), None, None, backward=dev(dout, io))
    want, wgrads = m.reference(x, g, beta, a, dout)
    close(out, want, io, "out")
    for n in grads:
        close(grads[n], wgrads[n], io, n)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_mixer_serves(io):
    """A prompt of 70 steps in two segments, then tokens one by one, state and window carried in place."""
    import torch
    m = Mixer(3, 64, 64, io)
    parts = [40, 30, 1, 1, 1, 2, 1]
    x, g, beta, a, _ = mixer_inputs(m, 2, sum(parts), 32)
    xd, gd, bd, ad = dev(x, io), dev(g, "f32"), dev(beta, "f32"), dev(a, io)
    state = torch.zeros(2, 3, 64, 64, device="cuda")
    win = torch.zeros(2, 3, m.C, dtype=xd.dtype, device="cuda")
    t, outs = 0, []
    for T in parts:
        seg = [z[:, t:t + T].contiguous() for z in (xd, gd, bd, ad)]
        outs.append(m.run(*seg, state, win))
        t += T
    close(torch.cat(outs, 1), m.reference(x, g, beta, a), io, "out")
