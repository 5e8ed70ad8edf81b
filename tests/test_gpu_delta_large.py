"""GPU: the gated delta rule, the group norm and the windowed convolution on tensors of more than 2^32 bytes (all of
it zero but the end, which is compared with the 64-bit reference at the tolerances of the small tests), segments whose
gradients are handed on in place, and the norm and the window under graph capture."""
import numpy as np
import pytest

from paper_2603_14360_amd import binding as mb
import delta_reference as dr
import gpu_util as gu
import test_gpu_delta as small
import test_gpu_delta_layer as layer

pytestmark = pytest.mark.gpu


@pytest.fixture
def torch():
    import torch
    yield torch
    torch.cuda.empty_cache()


@pytest.mark.parametrize("io,T", [("bf16", (1 << 19) + 65), ("f32", (1 << 18) + 65)])
@pytest.mark.parametrize("use_ckpt", [True, False])
def test_one_long_sequence(torch, io, T, use_ckpt):
    """With g = beta = 0 and k = 0 in front, the last 65 steps are a sequence of their own, which begins with a chunk."""
    print("case", io, T, use_ckpt, flush=True)
    N, K, V, end = 32, 64, 128, 65
    s = dr.rule_inputs(41, 1, end, N, K, V, io=io, carry=False)
    d = small.device(s, io)
    names = ("q", "k", "v", "g", "beta", "dy")
    many = {n: torch.zeros((1, T) + d[n].shape[2:], dtype=d[n].dtype, device="cuda") for n in names}
    assert many["v"].nbytes > 1 << 32
    for n in names:
        many[n][:, -end:] = d[n]
    p = mb.Delta(1, T, N, K, V, io)
    args = [many[n] for n in names[:5]] + [None]
    got = dict(zip(("y", "HT"), p.fwd(*args)))
    if not use_ckpt:
        p.ckpt.fill_(255)
    got.update(zip(dr.RULE_NAMES, p.bwd(*args, many["dy"], use_ckpt=use_ckpt)))
    torch.cuda.synchronize()
    for n, x in got.items():
        if n not in ("HT", "dH0"):
            assert not x[:, :-end].any(), n
            got[n] = x[:, -end:]
    small.check(got, dr.rule(s), (io, T))


@pytest.mark.parametrize("io,T", [("bf16", (1 << 21) + 3), ("f32", (1 << 20) + 3)])
def test_large_norm(torch, io, T):
    G, L, end = 17, 64, 3
    D = G * L
    r = np.random.default_rng(42)
    x, a, dout = (layer.store(r.standard_normal((1, end, D)), io) for _ in range(3))
    w = layer.store(1 + 0.2 * r.standard_normal(D), io)
    big = {}
    for n, z in (("x", x), ("a", a), ("dout", dout)):
        big[n] = torch.zeros(1, T, D, dtype=layer.dev(z, io).dtype, device="cuda")
        big[n][:, -end:] = layer.dev(z, io)
    assert big["x"].nbytes > 1 << 32
    wd = layer.dev(w, io)
    got = {n: torch.full_like(big["x"], float("nan")) for n in ("out", "dx", "da")}
    got.update({n: torch.empty(D, device="cuda") for n in ("dw", "db")})
    ws = torch.empty(mb.m2rnn_group_norm_workspace_bytes(1, T, D), dtype=torch.uint8, device="cuda")
    mb.m2rnn_group_norm_fwd(big["x"], big["a"], wd, None, G, layer.EPS, 0, got["out"])
    mb.m2rnn_group_norm_bwd(big["x"], big["a"], wd, None, G, layer.EPS, 0, big["dout"], got["dx"], got["da"], got["dw"],
                            got["db"], ws)
    torch.cuda.synchronize()
    for n in ("out", "dx", "da"):
        assert not got[n][:, :-end].any(), n
        got[n] = got[n][:, -end:]
    layer.check(got, dr.group_norm(x, a, w, None, G, layer.EPS, False, False, dout), (io, T))


@pytest.mark.parametrize("io,T", [("bf16", 730003), ("f32", 365003)])
def test_large_window(torch, io, T):
    C, end = 1472, 5
    r = np.random.default_rng(43)
    x, w = layer.store(r.standard_normal((1, end, C)), io), layer.store(0.5 * r.standard_normal((C, 4)), io)
    win = layer.store(r.standard_normal((1, 3, C)), io)
    xd = torch.zeros(2, T, C, dtype=layer.dev(x, io).dtype, device="cuda")
    assert xd.nbytes > 1 << 32
    xd[1, :end], xd[1, -end:] = layer.dev(x, io)[0], layer.dev(x, io)[0]
    wd = torch.zeros(2, 3, C, dtype=xd.dtype, device="cuda")
    wd[1] = layer.dev(win, io)[0]
    out, nxt = torch.full_like(xd, float("nan")), torch.full_like(wd, float("nan"))
    mb.m2rnn_conv_silu_window_fwd(xd, layer.dev(w, io), None, wd, out, nxt)
    torch.cuda.synchronize()
    assert not out[0].any() and not out[1, end + 3:-end].any() and not nxt[0].any()
    first, _ = dr.conv_window(x, w, None, win)
    last, behind = dr.conv_window(x, w, None, None)
    layer.check({"first": out[1:, :end], "last": out[1:, -end:]}, {"first": first, "last": last}, (io, T))
    assert (gu.to_np(nxt[1:]) == behind).all()


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("K,V", [(32, 32), (64, 128), (128, 16)])
def test_gradients_of_segments_in_place(torch, io, K, V):
    """Three segments of a sequence, backward from the last: dH0 of a call takes the place of its dHT."""
    parts = [64, 20, 66]
    s = dr.rule_inputs(44, 2, sum(parts), 4, K, V, Nqk=2, io=io)
    d = small.device(s, io)
    cut = lambda n, t, T: d[n][:, t:t + T].contiguous()
    state, calls, t = d["H0"], [], 0
    for T in parts:
        p, seg = mb.Delta(2, T, 4, K, V, io, Nqk=2), [cut(n, t, T) for n in ("q", "k", "v", "g", "beta")]
        calls.append((p, seg + [state], cut("dy", t, T)))
        state = p.fwd(*seg, state)[1]
        t += T
    grad, parts_of = d["dHT"].clone(), []
    for p, args, dy in reversed(calls):
        p.dH0 = grad
        parts_of.insert(0, p.bwd(*args, dy, grad)[:5])
    got = {n: torch.cat([x[i] for x in parts_of], 1) for i, n in enumerate(dr.RULE_NAMES[:5])}
    want = dr.rule(s)
    small.check(dict(got, HT=state, dH0=grad), {n: want[n] for n in list(got) + ["HT", "dH0"]}, (io, K, V))


# 64 states in 128 workgroups: more than 16 chunks go in several launches
@pytest.mark.parametrize("K", [32, 64, 128])
@pytest.mark.parametrize("T", [1024, 1025, 2200])
def test_few_long_sequences(torch, K, T):
    print("case", K, T, flush=True)
    s = dr.rule_inputs(46, 2, T, 32, K, 32, Nqk=16, io="bf16")
    want = dr.rule(s)
    a, b = small.run(s, "bf16"), small.run(s, "bf16", use_ckpt=False)
    small.check(a, want, (K, T))
    assert all(torch.equal(a[n], b[n]) for n in a)
    c = small.run(s, "bf16", backward=False)
    assert torch.equal(a["y"], c["y"]) and torch.equal(a["HT"], c["HT"])
    d = small.device(s, "bf16")  # the state in place
    p = mb.Delta(2, T, 32, K, 32, "bf16", Nqk=16, backward=False)
    p.HT = d["H0"]
    y, HT = p.fwd(*(d[n] for n in ("q", "k", "v", "g", "beta", "H0")))
    assert torch.equal(a["y"], y) and torch.equal(a["HT"], HT)


def test_norm_and_window_captured(torch):
    """Replayed three times on other inputs, with eager work in between; the window is carried in place."""
    B, T, G, L, io = 2, 65, 6, 64, "bf16"
    D = G * L
    r = np.random.default_rng(45)
    draw = lambda *shape: layer.dev(layer.store(r.standard_normal(shape), io), io)
    t = {"x": draw(B, T, D), "a": draw(B, T, D), "dout": draw(B, T, D), "win": draw(B, 3, D)}
    cw, w = draw(D, 4), draw(D)
    ws = torch.empty(mb.m2rnn_group_norm_workspace_bytes(B, T, D), dtype=torch.uint8, device="cuda")

    def buffers():
        new = lambda: torch.full((B, T, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        return {"u": new(), "out": new(), "dx": new(), "da": new(), "dw": torch.empty(D, device="cuda"), "db": torch.empty(D, device="cuda")}

    def call(i, o, win):
        st = torch.cuda.current_stream().cuda_stream
        mb.m2rnn_conv_silu_window_fwd(i["x"], cw, None, win, o["u"], win, stream=st)
        mb.m2rnn_group_norm_fwd(o["u"], i["a"], w, None, G, layer.EPS, 0, o["out"], stream=st)
        mb.m2rnn_group_norm_bwd(o["u"], i["a"], w, None, G, layer.EPS, 0, i["dout"], o["dx"], o["da"], o["dw"], o["db"], ws, stream=st)

    out = buffers()
    call(t, out, t["win"].clone())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(t, out, t["win"])
    for _ in range(3):
        for n in ("x", "a", "dout"):
            t[n].copy_(draw(*t[n].shape))
        want, win = buffers(), t["win"].clone()
        call(t, want, win)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(t["win"], win)
        for n in want:
            assert torch.equal(out[n], want[n]), n


@pytest.mark.parametrize("io,B,T,N,Nqk,K,V", [("bf16", 2, 1100, 32, 16, 32, 32), ("bf16", 3, 130, 4, 2, 64, 256), ("bf16", 2, 65, 3, 3, 128, 64),
                                              ("f32", 2, 70, 4, 2, 64, 32), ("bf16", 2, 33, 2, 1, 16, 16)])
@pytest.mark.parametrize("use_ckpt", [True, False])
def test_room_of_exactly_the_queried_size(torch, io, B, T, N, Nqk, K, V, use_ckpt):
    """Checkpoints and workspace end where the queries say: what lies in front of and behind them stays as it was."""
    print("case", io, B, T, N, Nqk, K, V, use_ckpt, flush=True)
    s = dr.rule_inputs(47, B, T, N, K, V, Nqk=Nqk, io=io)
    d, want = small.device(s, io), small.run(s, io, use_ckpt=use_ckpt)
    desc = mb.make_desc(B=B, T=T, N=N, K=K, V=V, io=mb.M2RNN_BF16 if io == "bf16" else mb.M2RNN_F32, Nqk=Nqk)
    st, guard = torch.cuda.current_stream().cuda_stream, 4096

    def room(n):
        whole = torch.full((n + 2 * guard,), 0xA5, dtype=torch.uint8, device="cuda")
        return whole, whole[guard:guard + n]

    kept = [room(mb.m2rnn_delta_ckpt_bytes(desc)), room(mb.m2rnn_delta_workspace_bytes(desc, 0)),
            room(mb.m2rnn_delta_workspace_bytes(desc, 1 if use_ckpt else 2))]
    got = {n: torch.full_like(x, float("nan")) for n, x in want.items()}
    args = [d[n] for n in ("q", "k", "v", "g", "beta", "H0")]
    mb.m2rnn_delta_fwd(desc, *args, got["y"], got["HT"], kept[0][1] if use_ckpt else None, kept[1][1], stream=st)
    mb.m2rnn_delta_bwd(desc, *args, kept[0][1] if use_ckpt else None, d["dy"], d["dHT"], *(got[n] for n in dr.RULE_NAMES),
                       kept[2][1], stream=st)
    torch.cuda.synchronize()
    for whole, _ in kept:
        assert (whole[:guard] == 0xA5).all() and (whole[-guard:] == 0xA5).all()
    for n in want:
        assert torch.equal(got[n], want[n]), n


def test_long_parts_captured(torch):
    """A forward of several launches, captured, replayed on other inputs with eager work in between."""
    T, N, K, V = 2200, 64, 64, 32
    first = dr.rule_inputs(48, 1, T, N, K, V, io="bf16")
    d = small.device(first, "bf16")
    names = ("q", "k", "v", "g", "beta", "H0")
    p, other = (mb.Delta(1, T, N, K, V, "bf16", backward=False) for _ in range(2))
    p.fwd(*(d[n] for n in names))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = p.fwd(*(d[n] for n in names))
    for seed in (49, 50, 51):
        s = small.device(dr.rule_inputs(seed, 1, T, N, K, V, io="bf16"), "bf16")
        want = other.fwd(*(s[n] for n in names))
        for n in names:
            d[n].copy_(s[n])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, w) for x, w in zip(out, want)), seed


@pytest.mark.parametrize("K", [32, 64, 128])
@pytest.mark.parametrize("V", [32, 64])
def test_many_states_without_checkpoints(torch, K, V):
    s = dr.rule_inputs(52, 33, 70, 4, K, V, Nqk=2, io="bf16")
    y, HT, _ = dr.rule_fwd(*(s[n] for n in ("q", "k", "v", "g", "beta", "H0")))
    a, b = small.run(s, "bf16"), small.run(s, "bf16", backward=False)
    small.check(b, {"y": y, "HT": HT}, (K, V))
    assert torch.equal(a["y"], b["y"]) and torch.equal(a["HT"], b["HT"])
