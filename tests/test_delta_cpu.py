"""CPU-only: sizes, routes and refusals of the gated delta rule, the group norm and the windowed convolution.
Nothing is launched: every call here is refused, or has nothing to do."""
import ctypes

import pytest

from paper_2603_14360_amd import binding as mb


class Buf:
    def __init__(self, addr=0x100000, nbytes=1 << 40):
        self.addr, self.nbytes = addr, nbytes

    def data_ptr(self):
        return self.addr


A, BIG = 0x1000, Buf()


def desc(**kw):
    return mb.make_desc(**dict(dict(B=2, T=70, N=4, K=32, V=32, io=mb.M2RNN_BF16), **kw))


def fwd(d, q=A, k=A, v=A, g=A, beta=A, H0=None, y=A, HT=A, ckpt=None, ws=BIG):
    return mb.m2rnn_delta_fwd(d, q, k, v, g, beta, H0, y, HT, ckpt, ws, check=False)


def bwd(d, q=A, k=A, v=A, g=A, beta=A, H0=None, ckpt=A, dy=A, dHT=None, dq=A, dk=A, dv=A, dg=A, dbeta=A, dH0=A, ws=BIG):
    return mb.m2rnn_delta_bwd(d, q, k, v, g, beta, H0, ckpt, dy, dHT, dq, dk, dv, dg, dbeta, dH0, ws, check=False)


BAD = [(dict(K=24), 2), (dict(K=256), 2), (dict(V=48), 2), (dict(V=512), 2), (dict(N=0), 2), (dict(Nqk=3), 2),
       (dict(Nqk=0), 2), (dict(B=-1), 2), (dict(T=-1), 2), (dict(io=5), 3), (dict(flags=1), 2), (dict(chunk=16), 7),
       (dict(B=1 << 30, N=1 << 20), 2), (dict(B=1 << 20, N=64, T=1 << 20), 2), (dict(B=1, N=64, T=1 << 25), 2),
       (dict(N=1 << 18, Nqk=1), 2)]


@pytest.mark.parametrize("kw,code", BAD)
def test_bad_descriptors_are_refused(kw, code):
    d = desc(**kw)
    assert fwd(d) == code and bwd(d) == code
    assert mb.m2rnn_delta_ckpt_bytes(d) == mb.m2rnn_delta_workspace_bytes(d, 0) == mb.m2rnn_delta_workspace_bytes(d, 2) == 0
    assert mb.m2rnn_delta_route_string(d, 0) == "invalid descriptor"


@pytest.mark.parametrize("name", ["q", "k", "v", "g", "beta", "y"])
def test_forward_needs_its_tensors(name):
    assert fwd(desc(), **{name: None}) == 1
    assert fwd(desc(), **{name: A + 8}) == 4


@pytest.mark.parametrize("name", ["q", "k", "v", "g", "beta", "dy", "dq", "dk", "dv", "dg", "dbeta"])
def test_backward_needs_its_tensors(name):
    assert bwd(desc(), **{name: None}) == 1
    assert bwd(desc(), **{name: A + 4}) == 4


@pytest.mark.parametrize("name", ["H0", "HT", "ckpt"])
def test_optional_tensors_are_aligned(name):
    assert fwd(desc(), **{name: A + 4}) == 4


@pytest.mark.parametrize("name", ["H0", "dHT", "dH0", "ckpt"])
def test_optional_tensors_of_the_backward_are_aligned(name):
    assert bwd(desc(), **{name: A + 4}) == 4


@pytest.mark.parametrize("io", [mb.M2RNN_F32, mb.M2RNN_BF16])
@pytest.mark.parametrize("Nqk", [4, 2])
@pytest.mark.parametrize("T", [1, 9, 64, 1000])
def test_workspace(io, Nqk, T):
    d = desc(T=T, Nqk=Nqk, io=io)
    for ckpt, bwd_mode in ((A, 1), (None, 2)):
        need = mb.m2rnn_delta_workspace_bytes(d, bwd_mode)
        assert need > 0
        assert bwd(d, ckpt=ckpt, ws=Buf(nbytes=need - 1)) == 5 and bwd(d, ckpt=ckpt, ws=None) == 1
    assert mb.m2rnn_delta_workspace_bytes(d, 2) == mb.m2rnn_delta_workspace_bytes(d, 1) + mb.m2rnn_delta_ckpt_bytes(d)
    need = mb.m2rnn_delta_workspace_bytes(d, 0)
    assert fwd(d, ckpt=A, ws=Buf(nbytes=need - 1)) == 5 and fwd(d, ckpt=A, ws=None) == 1
    if mb.m2rnn_delta_route_string(d, 0) != "step":
        assert fwd(d, ws=Buf(nbytes=need - 1)) == 5 and fwd(d, ws=None) == 1


def test_an_empty_batch_has_nothing_to_do():
    d = desc(B=0)
    assert fwd(d, q=None, k=None, v=None, g=None, beta=None, y=None, HT=None, ws=None) == 0
    assert bwd(d, *[None] * 16) == 0


def test_one_token_runs_the_recurrence():
    assert mb.m2rnn_delta_route_string(desc(T=1), 0) == "step"
    assert mb.m2rnn_delta_route_string(desc(T=1), 1) != "step"
    assert mb.m2rnn_delta_route_string(desc(T=4096), 0) != "step"


def test_group_norm_refusals():
    L, p = mb.lib(), ctypes.c_void_p(A)
    odd = ctypes.c_void_p(A + 4)

    def f(B=2, T=5, D=64, G=4, io=1, mode=0, x=p, a=None, w=p, b=p, eps=1e-5, out=p):
        return L.m2rnn_group_norm_fwd(B, T, D, G, io, mode, x, a, w, b, eps, out, None)

    def r(B=2, T=5, D=64, G=4, io=1, mode=0, x=p, a=None, w=p, b=p, eps=1e-5, dout=p, dx=p, da=None, dw=p, db=p, ws=p,
          n=1 << 30):
        return L.m2rnn_group_norm_bwd(B, T, D, G, io, mode, x, a, w, b, eps, dout, dx, da, dw, db, ws, n, None)

    for call in (f, r):
        for kw in (dict(D=60), dict(G=0), dict(G=5), dict(G=16), dict(D=2048, G=1), dict(eps=-1.0), dict(eps=float("nan")),
                   dict(mode=4), dict(mode=-1), dict(mode=mb.M2RNN_NORM_SILU, a=p), dict(B=-1), dict(T=-1)):
            assert call(**kw) == 2, kw
        assert call(io=2) == 3
        assert call(x=None) == 1 and call(x=odd) == 4 and call(w=odd) == 4 and call(b=odd) == 4
    assert f(out=None) == 1 and f(out=odd) == 4 and f(a=odd) == 4
    assert r(dout=None) == 1 and r(dx=None) == 1 and r(a=p) == 1 and r(a=p, da=odd) == 4
    assert r(ws=None) == 1 and r(n=16) == 5 and r(dw=odd) == 4
    assert mb.m2rnn_group_norm_workspace_bytes(2, 5, 60) == 0 < mb.m2rnn_group_norm_workspace_bytes(2, 5, 64)


def test_window_refusals():
    L, p, odd = mb.lib(), ctypes.c_void_p(A), ctypes.c_void_p(A + 2)

    def f(B=2, T=5, C=64, io=1, x=p, w=p, bias=None, win=p, out=p, win_out=p):
        return L.m2rnn_conv_silu_window_fwd(B, T, C, io, x, w, bias, win, out, win_out, None)

    assert f(C=12) == 2 and f(T=-1) == 2 and f(io=3) == 3
    assert f(x=None) == f(w=None) == f(out=None) == 1
    for n in ("x", "w", "bias", "win", "out", "win_out"):
        assert f(**{n: odd}) == 4
    assert f(B=0) == 0


def cpu(*shape, dtype="float32"):
    import torch
    return torch.zeros(shape, dtype=getattr(torch, dtype))


def test_tensors_that_are_not_on_the_gpu_are_refused():
    """... before anything is launched; an address on the host would be read by the GPU."""
    x, w = cpu(2, 3, 16), cpu(16)
    with pytest.raises(ValueError, match="x is not on the GPU"):
        mb.m2rnn_group_norm_fwd(x, None, w, None, 2, 1e-5, 0, cpu(2, 3, 16))
    with pytest.raises(ValueError, match="x is not on the GPU"):
        mb.m2rnn_conv_silu_window_fwd(x, cpu(16, 4), None, None, cpu(2, 3, 16), None)
    for bad in (cpu(2, 16), cpu(2, 3, 16, dtype="float16"), cpu(2, 3, 16, dtype="float64")):
        with pytest.raises(ValueError, match="x: expected"):
            mb.m2rnn_group_norm_fwd(bad, None, w, None, 2, 1e-5, 0, cpu(2, 3, 16))
    with pytest.raises(TypeError):
        mb.m2rnn_group_norm_fwd(A, None, w, None, 2, 1e-5, 0, cpu(2, 3, 16))
    d = desc()
    args = [ctypes.addressof(d)] + [cpu(2, 70, 4, 32, dtype="bfloat16")] * 3 + [cpu(2, 70, 4)] * 2
    with pytest.raises(ValueError, match="q is not on the GPU"):
        mb._call().delta_fwd(*args, None, A, A, None, A, 0, 1 << 40, -1)
    with pytest.raises(ValueError, match="q is not on the GPU"):
        mb._call().delta_bwd(*args, None, A, A, None, A, A, A, A, A, A, A, 0, 1 << 40, -1)
    with pytest.raises(TypeError):
        mb._call().delta_fwd(*args)


def test_a_norm_of_more_channels_than_its_sums_can_count_is_refused():
    L, p = mb.lib(), ctypes.c_void_p(A)
    D = 1 << 30
    assert L.m2rnn_group_norm_fwd(1, 1, D, D // 8, 1, 0, p, None, p, p, 1e-5, p, None) == 2
    assert L.m2rnn_group_norm_bwd(1, 1, D, D // 8, 1, 0, p, None, p, p, 1e-5, p, p, None, p, p, p, 1 << 60, None) == 2
    assert mb.m2rnn_group_norm_workspace_bytes(1, 1, D) == 0


def test_a_count_beyond_32_bits_is_not_cut_to_one_that_fits():
    x = cpu(2, 3, 16)
    for groups, mode in (((1 << 32) + 2, 0), (2, 1 << 32), (-(1 << 32) + 2, 0)):
        with pytest.raises(ValueError, match="too large"):
            mb.m2rnn_group_norm_fwd(x, None, cpu(16), None, groups, 1e-5, mode, x)


@pytest.mark.parametrize("V", [16, 32, 256])
@pytest.mark.parametrize("io", [mb.M2RNN_F32, mb.M2RNN_BF16])
def test_as_many_states_as_a_launch_can_have(V, io):
    """16 workgroups of 256 threads for each eight states: 2^32 threads from 2^20 - 7 states on."""
    most = (1 << 20) - 8
    assert mb.m2rnn_delta_workspace_bytes(desc(B=most, N=1, K=16, V=V, T=1, io=io), 0) > 0
    for B in (most + 1, most + 7, most + 8):
        d = desc(B=B, N=1, K=16, V=V, T=1, io=io)
        assert mb.m2rnn_delta_workspace_bytes(d, 0) == 0 and fwd(d) == 2 and bwd(d) == 2


def test_outputs_and_rooms_are_checked_as_inputs_are():
    """A tensor in any place of a call, the others addresses: one on the host is refused by its name."""
    d = desc()
    io, f = "bfloat16", "float32"
    qk, v, gates, state = (2, 70, 4, 32), (2, 70, 4, 32), (2, 70, 4), (2, 4, 32, 32)
    grads = [("dq", qk, io), ("dk", qk, io), ("dv", v, io), ("dg", gates, io), ("dbeta", gates, io), ("dH0", state, f)]
    backward = [("q", qk, io), ("k", qk, io), ("v", v, io), ("g", gates, f), ("beta", gates, f), ("H0", state, f),
                ("ckpt", (1 << 20,), "uint8"), ("dy", v, io), ("dHT", state, f)] + grads + [("workspace", (1 << 20,), "uint8")]
    forward = backward[:6] + [("y", v, io), ("HT", state, f), ("ckpt", (1 << 20,), "uint8"), ("workspace", (1 << 20,), "uint8")]
    for call, places in ((mb._call().delta_fwd, forward), (mb._call().delta_bwd, backward)):
        for i, (name, shape, dtype) in enumerate(places):
            args = [A] * len(places)
            args[i] = cpu(*shape, dtype=dtype)
            with pytest.raises(ValueError, match="%s is not on the GPU" % name):
                call(ctypes.addressof(d), *args, 0, 1 << 20, -1)


def test_the_backward_of_a_norm_checks_its_tensors():
    x, w = cpu(2, 3, 16), cpu(16)
    with pytest.raises(ValueError, match="x is not on the GPU"):
        mb.m2rnn_group_norm_bwd(x, None, w, None, 2, 1e-5, 0, x, cpu(2, 3, 16), None, None, None, None)
    with pytest.raises(ValueError, match="x: expected"):
        mb.m2rnn_group_norm_bwd(cpu(2, 16), None, w, None, 2, 1e-5, 0, x, x, None, None, None, None)
    with pytest.raises(ValueError, match="too large"):
        mb.m2rnn_group_norm_bwd(x, None, w, None, (1 << 32) + 2, 1e-5, 0, x, x, None, None, None, None)
    with pytest.raises(TypeError):
        mb.m2rnn_group_norm_bwd(A, None, w, None, 2, 1e-5, 0, x, x, None, None, None, None)


def test_calls_beside_delta_take_torchs_current_stream(monkeypatch):
    """... of x's GPU, unless they are given one; 0 is the null stream."""
    import torch

    class OnGpu:
        is_cuda = True

        def get_device(self):
            return 3

    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 1000 + device, raising=False)
    assert mb._stream_for(OnGpu(), None) == 1003 and mb._stream_for(OnGpu(), 0) == 0 and mb._stream_for(OnGpu(), 77) == 77
    assert mb._stream_for(cpu(1), None) == 0 and mb._stream_for(A, None) == 0


@pytest.mark.parametrize("T", [1, 70, 1000])
def test_the_fp32_backward_asks_for_what_it_uses(T):
    """Gates, T and P are kept with the checkpoints there: a backward needs room for a state a chunk and U's rows."""
    d = desc(T=T, io=mb.M2RNN_F32, K=64, V=32)
    up = lambda n: -(-n // 256) * 256
    assert mb.m2rnn_delta_workspace_bytes(d, 1) == up(2 * 4 * -(-T // 32) * 64 * 32 * 4) + up(2 * T * 4 * 32 * 4)


@pytest.mark.parametrize("io", [mb.M2RNN_F32, mb.M2RNN_BF16])
def test_few_steps_go_the_faster_way(io):
    """Fewer steps by the recurrence where heads are small and many, whose chunks are cheap; more where the states are large."""
    route = lambda **kw: mb.m2rnn_delta_route_string(desc(io=io, **kw), 0)
    for B, N, K, V, most in ((1, 32, 128, 128, 12), (16, 16, 128, 128, 16), (4, 16, 64, 64, 12), (64, 16, 64, 64, 16), (1, 84, 64, 16, 12),
                             (64, 84, 64, 16, 6), (64, 16, 32, 32, 8), (32, 16, 32, 32, 12), (256, 16, 16, 16, 12), (256, 16, 16, 64, 12)):
        assert route(B=B, N=N, K=K, V=V, T=most) == "step" != route(B=B, N=N, K=K, V=V, T=most + 1), (B, N, K, V)


def test_twelve_steps_need_no_workspace():
    """... whichever way is the faster one; an empty batch of them has nothing to do, and launches nothing."""
    none = dict(q=None, k=None, v=None, g=None, beta=None, y=None, HT=None, ws=None)
    for io, most in ((mb.M2RNN_BF16, 12), (mb.M2RNN_F32, 16)):
        assert fwd(desc(B=0, N=1, K=64, V=16, T=most, io=io), **none) == 0
        assert fwd(desc(B=2, N=4, K=64, V=64, T=most + 1, io=io), ws=None) == 1
