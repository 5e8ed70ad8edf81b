"""GPU: what the calls of the gated delta rule and the group norm refuse.  Nothing here is launched: outputs keep what they
held."""
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
