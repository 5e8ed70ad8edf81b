"""GPU: the gated delta rule through the C ABI against the 64-bit reference (delta_reference.py), which reads the
storage-rounded inputs.

Tolerances, of the largest entry of a tensor.  fp32 results are sums of at most 2 C + K + V = 384 products, each
rounded to 2^-24 once as a product, once as an operand and once as a sum: 3 sqrt(384) 2^-24 = 3.5e-6 where roundings
are independent; states are carried over chunks by maps that do not expand, so over some ten chunks three times that:
1e-5.  (The states of bf16 io too: their chain runs on operands of 22 bits, of which four are rounded per chunk.)
bf16 results are off by half a step of their own value, 2^-8, and by what operands of 11 bits leave: two roundings of
2^-12 in each of the products, whose terms add up to no more than eight times the largest entry: 2^-8."""
import numpy as np
import pytest

from paper_2603_14360_amd import binding as mb
import delta_reference as dr
import gpu_util as gu

pytestmark = pytest.mark.gpu

F32 = 1e-5
BF16 = 2.0 ** -8


def check(got, want, label):
    """got: tensors by name, want: arrays."""
    bad = {}
    for n, w in want.items():
        g = gu.to_np(got[n])
        assert g.shape == w.shape and np.isfinite(g).all(), (label, n)
        if not w.size:
            continue
        top = np.abs(w).max()
        err = np.abs(g - w)
        if "bfloat16" in str(got[n].dtype):
            over = (err / (BF16 * np.abs(w) + BF16 * top + 1e-30)).max()
        else:
            over = (err / (F32 * top + 1e-30)).max()
        if not over <= 1:
            bad[n] = float(over)
    assert not bad, (label, bad)


def device(s, io):
    import torch
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    put = lambda n: None if s[n] is None else torch.from_numpy(np.ascontiguousarray(s[n], np.float32)).to("cuda")
    d = {n: put(n) for n in s}
    for n in ("q", "k", "v", "dy"):
        d[n] = d[n].to(dt)
    return d


def run(s, io, use_ckpt=True, backward=True):
    """The results by name; every output buffer starts as NaN."""
    import torch
    B, T, Nqk, K = s["q"].shape
    N, V = s["v"].shape[2:]
    d = device(s, io)
    delta = mb.Delta(B, T, N, K, V, io, Nqk=Nqk, backward=backward)
    for x in vars(delta).values():
        if torch.is_tensor(x):
            x.fill_(float("nan") if x.is_floating_point() else 255)
    args = [d[n] for n in ("q", "k", "v", "g", "beta", "H0")]
    y, HT = delta.fwd(*args)
    out = {"y": y, "HT": HT}
    if backward:
        if not use_ckpt:
            delta.ckpt.fill_(255)
        out.update(zip(dr.RULE_NAMES, delta.bwd(*args, d["dy"], d["dHT"], use_ckpt=use_ckpt)))
    torch.cuda.synchronize()
    return out


DIMS = [(K, V) for K in (16, 32, 64, 128) for V in (16, 32, 64, 128, 256)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("K,V", DIMS)
def test_every_size(io, K, V):
    print("case", io, K, V, flush=True)
    s = dr.rule_inputs(K + V, 2, 83, 3, K, V, io=io)
    check(run(s, io), dr.rule(s), (io, K, V))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("K,V", [(64, 64), (128, 128), (32, 16)])
@pytest.mark.parametrize("T", [1, 2, 15, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300])
def test_lengths(io, K, V, T):
    print("case", io, K, V, T, flush=True)
    s = dr.rule_inputs(T, 1, T, 2, K, V, io=io, carry=T % 2 == 1)
    check(run(s, io, use_ckpt=T != 129), dr.rule(s), (io, T))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("N,Nqk", [(4, 1), (6, 2), (4, 4)])
@pytest.mark.parametrize("use_ckpt", [True, False])
def test_heads_that_share_q_and_k(io, N, Nqk, use_ckpt):
    s = dr.rule_inputs(N, 3, 70, N, 64, 32, Nqk=Nqk, io=io)
    check(run(s, io, use_ckpt=use_ckpt), dr.rule(s), (io, N, Nqk))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 3, 5, 8, 9, 16, 17])
@pytest.mark.parametrize("K,V,Nqk", [(16, 16, 4), (32, 64, 1), (64, 32, 2), (128, 128, 4), (128, 256, 1), (16, 32, 2), (64, 16, 4)])
def test_without_checkpoints(io, T, K, V, Nqk):
    s = dr.rule_inputs(T + K, 3, T, 4, K, V, Nqk=Nqk, io=io)
    y, HT, _ = dr.rule_fwd(*(s[n] for n in ("q", "k", "v", "g", "beta", "H0")))
    check(run(s, io, backward=False), {"y": y, "HT": HT}, (io, T, K, V))


# enough states for the workgroups with 32 columns (bf16), where the sizes above run on those with 16
@pytest.mark.parametrize("K,V", [(K, V) for K in (32, 64, 128) for V in (32, 64, 128, 256)])
def test_many_states(K, V):
    T = 130 if V < 256 else 65
    N = 4 if V < 128 else 2
    B = -(-129 // (N * (V // 32)))
    s = dr.rule_inputs(K * V, B, T, N, K, V, Nqk=2, io="bf16")
    check(run(s, "bf16", use_ckpt=V != 64), dr.rule(s), (K, V))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("K", [16, 32, 64, 128])
@pytest.mark.parametrize("B,N,V,T", [(128, 4, 64, 1), (65, 4, 128, 3)])
def test_many_states_step_by_step(io, K, B, N, V, T):
    s = dr.rule_inputs(K + T, B, T, N, K, V, Nqk=1, io=io)
    y, HT, _ = dr.rule_fwd(*(s[n] for n in ("q", "k", "v", "g", "beta", "H0")))
    check(run(s, io, backward=False), {"y": y, "HT": HT}, (io, K, V))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("T", [7, 150])
@pytest.mark.parametrize("what", ["resets", "open", "shut", "padded", "still", "strong", "same_key", "beta_two"])
def test_gates_and_betas_at_their_ends(io, T, what):
    s = dr.rule_inputs(9, 2, T, 3, 64, 64, io=io)
    if what == "resets":       # the state forgets everything, at single steps and at the first one
        s["g"][:, ::5] = -np.inf
    elif what == "open":       # no forgetting at all
        s["g"][:] = 0
    elif what == "shut":
        s["g"][:] = -np.inf
    elif what == "padded":     # the steps of a padded batch: neither gate nor update
        s["g"][1, T // 2:], s["beta"][1, T // 2:] = 0, 0
    elif what == "still":
        s["beta"][:] = 0
    elif what == "strong":     # sums of g over a chunk far below what exp can hold
        s["g"][:] = -30 - 40 * np.random.default_rng(1).random(s["g"].shape)
    elif what == "same_key":   # every step asks and writes the same row
        s["k"][:] = s["k"][:, :1]
    elif what == "beta_two":   # reflections
        s["beta"][:] = 2
    want = dr.rule(s)
    got = run(s, io)
    if what in ("resets", "shut", "strong"):
        # where nothing is carried over (e^-30 = 9e-14 of it at most), dg = <dH, e^g H> is zero beside the terms
        # that it is formed from, the chunk's q.dq and k.dk, whose sums cancel: off by 2^-24 (fp32) or 2^-11 of
        # up to 64 of them
        terms = sum(np.abs(s[n].astype(float) * want["d" + n]).sum(-1).max() for n in ("q", "k"))
        lim = 64 * terms * (2.0 ** -24 if io == "f32" else 2.0 ** -11)
        assert np.abs(gu.to_np(got["dg"]) - want["dg"]).max() <= lim
        del want["dg"]
    check(got, want, (io, what))
    if what == "padded":       # the state behind the padding is the one in front of it
        short = {n: None if x is None else x if n in ("H0", "dHT") else x[:, :T // 2] for n, x in s.items()}
        y, HT, _ = dr.rule_fwd(*(short[n] for n in ("q", "k", "v", "g", "beta", "H0")))
        check({"HT": got["HT"][1]}, {"HT": HT[1]}, "padded")


@pytest.mark.parametrize("scale", [1e-6, 1e4])
@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_gradients_of_any_size(io, scale):
    s = dr.rule_inputs(10, 2, 100, 3, 64, 64, io=io)
    s["dy"] = (s["dy"] * np.float32(2.0 ** round(np.log2(scale)))).astype(np.float32)
    s["dHT"] = s["dHT"] * np.float32(scale)
    check(run(s, io), dr.rule(s), (io, scale))


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_a_gradient_at_the_end_alone(io):
    """Only the last step has a loss: what reaches the first ones is many orders smaller."""
    s = dr.rule_inputs(11, 1, 400, 2, 64, 32, io=io, memory=20.0)
    s["dy"][:, :-1] = 0
    s["dHT"] = None
    want = dr.rule(s)
    got = run(s, io)
    check(got, want, io)
    check({"dv": got["dv"][:, :200]}, {"dv": want["dv"][:, :200]}, io)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_nothing_to_do(io):
    import torch
    s = dr.rule_inputs(12, 2, 0, 3, 32, 32, io=io)
    got = run(s, io)
    d = device(s, io)
    assert torch.equal(got["HT"], d["H0"]) and torch.equal(got["dH0"], d["dHT"])
    s["H0"] = s["dHT"] = None
    got = run(s, io)
    assert not got["HT"].any() and not got["dH0"].any()
    assert mb.Delta(0, 5, 2, 32, 32, io).fwd(*[None] * 5)[0].numel() == 0


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("T,bad", [(5, 3), (200, 100)])
def test_a_nan_stays_behind(io, T, bad):
    """A NaN in a step reaches no y of an earlier chunk, no other head and no other batch row."""
    s = dr.rule_inputs(13, 2, T, 3, 64, 64, io=io)
    clean = run(s, io, backward=False)
    s["v"][1, bad, 2, 5] = np.nan
    got = run(s, io, backward=False)
    first = bad if T <= 8 else bad - 63
    for n in ("y", "HT"):
        a, b = gu.to_np(got[n]), gu.to_np(clean[n])
        assert (a[0] == b[0]).all()
    y, z = gu.to_np(got["y"]), gu.to_np(clean["y"])
    assert (y[1, :, :2] == z[1, :, :2]).all() and (y[1, :first, 2] == z[1, :first, 2]).all()
    assert np.isnan(y[1, bad:, 2, 5]).all() and np.isnan(gu.to_np(got["HT"])[1, 2, :, 5]).any()


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_the_same_call_gives_the_same_bits(io):
    import torch
    s = dr.rule_inputs(14, 2, 200, 6, 64, 64, Nqk=2, io=io)
    a, b = run(s, io), run(s, io)
    assert all(torch.equal(a[n], b[n]) for n in a)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_a_chain_of_calls_is_one_sequence(io):
    """Segments of 70, 1, 1, 8 and 40 steps with the state handed on in place, against one call's reference."""
    import torch
    parts = [70, 1, 1, 8, 40]
    s = dr.rule_inputs(15, 2, sum(parts), 4, 64, 128, Nqk=2, io=io)
    y, HT, _ = dr.rule_fwd(*(s[n] for n in ("q", "k", "v", "g", "beta", "H0")))
    d = device(s, io)
    state, t, ys = d["H0"].clone(), 0, []
    for T in parts:
        delta = mb.Delta(2, T, 4, 64, 128, io, Nqk=2, backward=False)
        seg = [d[n][:, t:t + T].contiguous() for n in ("q", "k", "v", "g", "beta")]
        delta.HT = state
        ys.append(delta.fwd(*seg, state)[0])
        t += T
    check({"y": torch.cat(ys, 1), "HT": state}, {"y": y, "HT": HT}, io)


def test_two_streams_at_once():
    """Calls that share nothing but inputs, each with buffers and a stream of its own."""
    import torch
    s = dr.rule_inputs(16, 2, 300, 4, 64, 64, io="bf16")
    d = device(s, "bf16")
    args = [d[n] for n in ("q", "k", "v", "g", "beta", "H0")]
    plans = [mb.Delta(2, 300, 4, 64, 64, "bf16") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in plans]
    torch.cuda.synchronize()
    out = []
    for p, st in zip(plans, streams):
        with torch.cuda.stream(st):
            out.append(dict(zip(("y", "HT") + dr.RULE_NAMES, p.fwd(*args) + p.bwd(*args, d["dy"], d["dHT"]))))
    torch.cuda.synchronize()
    want = run(s, "bf16")
    for o in out:
        assert all(torch.equal(o[n], want[n]) for n in want)


@pytest.mark.parametrize("io,T", [("bf16", 200), ("f32", 100), ("bf16", 1)])
def test_graph_capture_and_replay(io, T):
    """A forward and backward captured once and replayed on other inputs, with eager work in between."""
    import torch
    B, N, K, V = 2, 4, 64, 64
    first = dr.rule_inputs(17, B, T, N, K, V, io=io)
    d = device(first, io)
    args = [d[n] for n in ("q", "k", "v", "g", "beta", "H0")]
    p = mb.Delta(B, T, N, K, V, io)
    call = lambda: p.fwd(*args) + p.bwd(*args, d["dy"], d["dHT"])
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for seed in (18, 19, 20):
        s = dr.rule_inputs(seed, B, T, N, K, V, io=io)
        want = run(s, io)
        for n, x in device(s, io).items():
            d[n].copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        for n, x in zip(("y", "HT") + dr.RULE_NAMES, out):
            assert torch.equal(x, want[n]), (seed, n)


def test_offsets_beyond_32_bits():
    """Tensors of more than 2^32 bytes, states of more than 2^31: the last sequence against the reference."""
    import torch
    B, T, N, K, V = 2300, 65, 64, 64, 256
    s = dr.rule_inputs(21, 1, T, N, K, V, io="bf16", carry=False)
    d = device(s, "bf16")
    one = [d[n] for n in ("q", "k", "v", "g", "beta")]
    many = [torch.zeros((B,) + x.shape[1:], dtype=x.dtype, device="cuda") for x in one]
    assert many[2].nbytes > 1 << 32
    for x, m in zip(one, many):
        m[-1].copy_(x[0])
    p = mb.Delta(B, T, N, K, V, "bf16", backward=False)
    y, HT = p.fwd(*many)
    torch.cuda.synchronize()
    wy, wH, _ = dr.rule_fwd(*(s[n] for n in ("q", "k", "v", "g", "beta")))
    check({"y": y[-1:], "HT": HT[-1:]}, {"y": wy, "HT": wH}, "large")
    assert not y[:-1].any() and not HT[:-1].any()


def test_tensors_that_do_not_fit_are_refused():
    """Another size, type or memory order: an exception, and nothing is launched."""
    import torch
    s = dr.rule_inputs(22, 2, 10, 4, 32, 64, Nqk=2, io="bf16")
    d = device(s, "bf16")
    p = mb.Delta(2, 10, 4, 32, 64, "bf16", Nqk=2)
    names = ("q", "k", "v", "g", "beta", "H0")
    good = [d[n] for n in names]
    p.y.fill_(7)
    for i, n in enumerate(names):
        x = good[i]
        for bad, why in ((x[:1], "size"), (x.double(), "dtype"), (x.cpu(), "not on the GPU"),
                         (x.transpose(0, 1).contiguous().transpose(0, 1), "contiguous")):
            args = good[:i] + [bad] + good[i + 1:]
            with pytest.raises(ValueError, match="%s .*%s" % (n, why)):
                p.fwd(*args)
            with pytest.raises(ValueError, match="%s .*%s" % (n, why)):
                p.bwd(*args, d["dy"], d["dHT"])
    with pytest.raises(ValueError, match="dy"):
        p.bwd(*good, d["dy"].float(), None)
    with pytest.raises(mb.M2RNNError):
        p.fwd(None, *good[1:])
    torch.cuda.synchronize()
    assert (p.y == 7).all()
    x = torch.zeros(2, 3, 16, device="cuda")
    for kw in (dict(w=torch.zeros(8, device="cuda")), dict(out=torch.zeros(2, 3, 16, device="cuda").bfloat16()),
               dict(a=x[:, :2]), dict(b=torch.zeros(16))):
        a = dict(dict(x=x, a=None, w=None, b=None, groups=2, eps=1e-5, mode=0, out=x.clone()), **kw)
        with pytest.raises(ValueError):
            mb.m2rnn_group_norm_fwd(**a)
