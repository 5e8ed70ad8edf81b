"""GPU: what the calls of the gated delta rule and the group norm refuse (nothing is launched then: outputs keep what they
held), and the stream that calls beside Delta run on."""
import pytest

from paper_2603_14360_amd import binding as mb
import delta_reference as dr
import test_gpu_delta as small

pytestmark = pytest.mark.gpu


def others(x):
    """Buffers that do not fit in x's place, and why."""
    import torch
    flat = x.flatten()
    yield flat[:-1].clone(), "size"
    yield x.double(), "dtype"
    yield x.cpu(), "not on the GPU"
    wide = torch.empty(x.shape + (2,), dtype=x.dtype, device=x.device)
    yield wide[..., 0], "contiguous"


def test_outputs_of_the_rule():
    import torch
    s = dr.rule_inputs(81, 2, 10, 4, 32, 64, Nqk=2, io="bf16")
    d = small.device(s, "bf16")
    args = [d[n] for n in ("q", "k", "v", "g", "beta", "H0")]
    p = mb.Delta(2, 10, 4, 32, 64, "bf16", Nqk=2)
    mine = ("y", "HT") + dr.RULE_NAMES
    for n in mine:
        getattr(p, n).fill_(7)
    for n in mine:
        good = getattr(p, n)
        for bad, why in others(good):
            setattr(p, n, bad)
            with pytest.raises(ValueError, match="%s .*%s" % (n, why)):
                p.fwd(*args) if n in ("y", "HT") else p.bwd(*args, d["dy"], d["dHT"])
        setattr(p, n, good)
    calls = (lambda: p.fwd(*args), lambda: p.bwd(*args, d["dy"], d["dHT"]))
    for n in ("ckpt", "workspace"):
        good = getattr(p, n)
        # (what there is of the workspace the library compares itself)
        short = ValueError if n == "ckpt" else mb.M2RNNError
        for bad, refused in ((good[:1024].clone(), short), (good.cpu(), ValueError), (good[::2], ValueError)):
            setattr(p, n, bad)
            for call in calls:
                with pytest.raises(refused):
                    call()
        setattr(p, n, good)
    torch.cuda.synchronize()
    for n in mine:
        assert (getattr(p, n) == 7).all(), n


def test_tensors_of_the_backward_of_a_norm():
    import torch
    D = 64
    new = lambda *shape: torch.full(shape, 7.0, device="cuda")
    good = dict(x=new(2, 3, D), a=new(2, 3, D), w=new(D), b=new(D), groups=4, eps=1e-5, mode=0, dout=new(2, 3, D), dx=new(2, 3, D),
                da=new(2, 3, D), dw=new(D), db=new(D),
                workspace=torch.full((mb.m2rnn_group_norm_workspace_bytes(2, 3, D),), 7, dtype=torch.uint8, device="cuda"))
    for n in ("a", "w", "b", "dout", "dx", "da", "dw", "db"):
        for bad, why in others(good[n]):
            with pytest.raises(ValueError, match="%s .*%s" % (n, why)):
                mb.m2rnn_group_norm_bwd(**dict(good, **{n: bad}))
    with pytest.raises(ValueError, match="workspace is not on the GPU"):
        mb.m2rnn_group_norm_bwd(**dict(good, workspace=good["workspace"].cpu()))
    with pytest.raises(mb.M2RNNError):
        mb.m2rnn_group_norm_bwd(**dict(good, workspace=good["workspace"][:-16].clone()))
    torch.cuda.synchronize()
    for n in ("dx", "da", "dw", "db"):
        assert (good[n] == 7).all(), n


def test_calls_without_a_stream_run_on_the_current_one():
    """As Delta does: a capture holds them all, in order, and replays them on other inputs."""
    import torch
    B, T, G, L = 2, 9, 4, 64
    D = G * L
    gen = torch.Generator(device="cuda").manual_seed(82)
    new = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    x, cw, win, w, dout, ws = new(B, T, D), new(D, 4), new(B, 3, D), new(D), new(B, T, D), new(1 << 16)

    def call():
        u, out, dx, dw, nxt = (torch.empty_like(t) for t in (x, x, x, w, win))
        mb.m2rnn_conv_silu_window_fwd(x, cw, None, win, u, nxt)
        mb.m2rnn_group_norm_fwd(u, None, w, None, G, 1e-5, 0, out)
        mb.m2rnn_group_norm_bwd(u, None, w, None, G, 1e-5, 0, dout, dx, None, dw, None, ws)
        return u, out, dx, dw, nxt

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for _ in range(3):
        for t in (x, win, dout):
            t.copy_(new(*t.shape))
        want = call()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("io,T", [("bf16", 12), ("f32", 16)])
def test_twelve_steps_without_a_workspace(io, T):
    """Many small heads, which go by chunks from 8 steps on where there is room for it."""
    import torch
    B, N, K, V = 11, 50, 64, 16
    s = dr.rule_inputs(83, B, T, N, K, V, Nqk=10, io=io)
    d = small.device(s, io)
    desc = mb.make_desc(B=B, T=T, N=N, K=K, V=V, Nqk=10, io=mb.M2RNN_BF16 if io == "bf16" else mb.M2RNN_F32)
    assert mb.m2rnn_delta_route_string(desc, 0) != "step"
    got = {"y": torch.full_like(d["v"], float("nan")), "HT": torch.full_like(d["H0"], float("nan"))}
    mb.m2rnn_delta_fwd(desc, *(d[n] for n in ("q", "k", "v", "g", "beta", "H0")), got["y"], got["HT"], None, None,
                       stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    y, HT, _ = dr.rule_fwd(*(s[n] for n in ("q", "k", "v", "g", "beta", "H0")))
    small.check(got, {"y": y, "HT": HT}, (io, T))
    small.check(small.run(s, io, backward=False), {"y": y, "HT": HT}, (io, T))
