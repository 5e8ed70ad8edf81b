"""Gated delta rule, group norm with an activation, and the convolution that goes on from a window, as
calls to be timed and compared.

  delta_train    forward (keeping chunk states) and backward of the gated delta rule
  delta_prefill  its forward over prompts, no chunk states kept
  delta_decode   one token per sequence: the recurrent form, the state handed in and out
  norm_train     group norm of a token's channels with an activation, forward and backward
  norm_infer     its forward alone
  window         causal conv1d(4) + SiLU that starts from the last three inputs and hands on its own

Together they are the mixer of a gated-delta-rule layer, which hybrids put beside the layer whose scan
this library computes: convolution, norm of q and k, delta rule, gated norm of each head.

Sizes are those of the benchmark's workloads (8 x 4096 with 16 heads of 64 x 64, 4 x 8192 with 8 of
128 x 128, 1 x 65536 with 32 of 64 x 64, fp32 4 x 512 with 8 of 32 x 32), of the paper's layer
(1472 convolution channels, 84 heads of 16 values) and generic ones: heads of 128 x 128, q and k shared
by several heads, odd lengths.  q and k have unit length, as the rule needs it (q scaled by K^-1/2 on
top); log gates are spread from a memory of two steps to one of some hundreds; beta is a sigmoid.
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_CHUNK = 64  # of the plain form
_EPS = 1e-5


# ------------------------------------------------------------------ cases
def _delta(kind, B, T, N, K, V, Nqk=0, io="bf16", carry=False, name=None):
    """carry: an initial state is given (and, in training, the gradient of the final one)."""
    c = {"kind": kind, "B": B, "T": T, "N": N, "Nqk": Nqk or N, "K": K, "V": V, "io": io, "carry": carry}
    return c if name is None else dict(c, name=name)


def _norm(kind, B, T, G, L, act, center, affine=True, io="bf16", name=None):
    """G groups of L channels.  act: "gate" (SiLU of a second input), "silu" or "none"; affine: weight
    and bias per channel, or a weight alone."""
    c = {"kind": kind, "B": B, "T": T, "G": G, "L": L, "act": act, "center": center, "affine": affine, "io": io}
    return c if name is None else dict(c, name=name)


def _window(B, T, C, io="bf16", bias=True, name=None):
    c = {"kind": "window", "B": B, "T": T, "C": C, "io": io, "bias": bias}
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # training steps at the benchmark's headline sizes and at its large state
        _delta("delta_train", 8, 4096, 16, 64, 64, name="delta_train_headline"),
        _delta("delta_train", 4, 8192, 8, 128, 128, name="delta_train_wide"),
        # segments of odd length of a model whose heads share q and k, the state carried across
        _delta("delta_train", 8, 1000, 12, 64, 128, Nqk=4, carry=True, name="delta_train_segments"),
        # fp32 storage, for debugging and for comparing with another implementation
        _delta("delta_train", 4, 512, 8, 32, 32, io="f32", carry=True, name="delta_train_fp32"),
        # a few prompts of odd length, and one long document on few states
        _delta("delta_prefill", 4, 777, 32, 128, 128, Nqk=16, carry=True, name="delta_prefill_prompts"),
        _delta("delta_prefill", 1, 65536, 32, 64, 64, name="delta_prefill_long"),
        # serving, one sequence and a large batch: latency, and the state's traffic
        _delta("delta_decode", 1, 1, 32, 128, 128, Nqk=16, carry=True, name="delta_decode_one"),
        _delta("delta_decode", 256, 1, 16, 128, 128, carry=True, name="delta_decode_batch"),
        # the gated norm behind a layer of 16 heads of 128 in training, and of the paper's 84 heads of 16
        # values, with a mean, over the token that each of 64 sequences is served
        _norm("norm_train", 8, 4096, 16, 128, "gate", False, name="norm_train_heads"),
        _norm("norm_infer", 64, 1, 84, 16, "silu", True, name="norm_serve_small"),
        # the convolution of q, k and v of the paper's layer: a token for each of 64 sequences, and the
        # next segment of a few prompts
        _window(64, 1, 1472, name="window_decode"),
        _window(4, 777, 1472, name="window_segment"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_MOST = 4 * 8192 * 8 * 128 * 128  # state elements times steps of one drawn case


def draw(rng):
    kind = rng.choice(["delta_train"] * 4 + ["delta_prefill"] * 2 + ["delta_decode"] * 2 + ["norm", "norm", "window"])
    io = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "window":
        return _window(rng.randint(1, 64), rng.choice([1, rng.randint(2, 8), _log_int(rng, 8, 512)]),
                       8 * _log_int(rng, 8, 256), io=io, bias=rng.random() < 0.5)
    if kind == "norm":
        G = rng.choice([1, 4, 7, 16, 32, 84])
        L = 8 * rng.randint(1, min(40, 4096 // (8 * G)))
        return _norm(rng.choice(["norm_train", "norm_train", "norm_infer"]), rng.randint(1, 8), _log_int(rng, 1, 4096),
                     G, L, rng.choice(["gate", "gate", "silu", "none"]), rng.random() < 0.5,
                     affine=rng.random() < 0.5, io=io)
    K, V = rng.choice([(64, 64), (64, 64), (128, 128), (128, 128), (64, 128), (128, 64), (128, 256), (32, 32), (32, 64),
                       (16, 16), (16, 64)])
    Nqk = rng.choice([1, 2, 4, 8, 16])
    N = Nqk * rng.choice([1, 1, 2, 3])
    if kind == "delta_decode":
        return _delta(kind, _log_int(rng, 1, 256), 1, N, K, V, Nqk=Nqk, io=io, carry=True)
    T = _log_int(rng, 2, min(8192, _MOST // (N * K * V)))
    B = _log_int(rng, 1, min(64, _MOST // (T * N * K * V)))
    return _delta(kind, B, T, N, K, V, Nqk=Nqk, io=io, carry=rng.random() < 0.5)


# ------------------------------------------------------------------ inputs
def _randn(g, *shape, scale=1.0, mean=0.0, dtype=torch.float32):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    return x.mul_(scale).add_(mean).to(dtype)


def _unit(g, *shape, scale=1.0, dtype=torch.float32):
    x = _randn(g, *shape)
    return x.mul_(scale / x.norm(dim=-1, keepdim=True)).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    c, dt = case, _DT[case["io"]]
    s = {"case": dict(c)}
    if c["kind"] == "window":
        s["x"] = _randn(g, c["B"], c["T"], c["C"], dtype=dt)
        s["w"] = _randn(g, c["C"], 4, scale=0.5, dtype=dt)
        s["bias"] = _randn(g, c["C"], scale=0.5, dtype=dt) if c["bias"] else None
        s["win"] = _randn(g, c["B"], 3, c["C"], dtype=dt)
        s["out"], s["win_out"] = torch.empty_like(s["x"]), torch.empty_like(s["win"])
        return s
    if c["kind"] in ("norm_train", "norm_infer"):
        B, T, D = c["B"], c["T"], c["G"] * c["L"]
        s["x"] = _randn(g, B, T, D, mean=0.25, dtype=dt)
        s["a"] = _randn(g, B, T, D, dtype=dt) if c["act"] == "gate" else None
        s["w"] = _randn(g, D, scale=0.1, mean=1.0, dtype=dt)
        s["b"] = _randn(g, D, scale=0.1, dtype=dt) if c["affine"] else None
        s["out"] = torch.empty_like(s["x"])
        if c["kind"] == "norm_train":
            s["dout"] = _randn(g, B, T, D, dtype=dt)
            s["dx"] = torch.empty_like(s["x"])
            s["da"] = None if s["a"] is None else torch.empty_like(s["a"])
            s["dw"] = torch.empty(D, device="cuda", dtype=torch.float32)
            s["db"] = torch.empty_like(s["dw"]) if c["affine"] else None
            if own:
                nbytes = _library().m2rnn_group_norm_workspace_bytes(B, T, D)
                s["workspace"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        return s
    B, T, N, Nqk, K, V = (c[n] for n in ("B", "T", "N", "Nqk", "K", "V"))
    s["q"] = _unit(g, B, T, Nqk, K, scale=K ** -0.5, dtype=dt)
    s["k"] = _unit(g, B, T, Nqk, K, dtype=dt)
    s["v"] = _randn(g, B, T, N, V, dtype=dt)
    # a head's memory, 2 to 500 steps, with a spread over its tokens
    rate = torch.rand(N, generator=g, device="cuda").mul_(math.log(250.0)).exp_().mul_(1 / 500.0)
    s["g"] = _randn(g, B, T, N, scale=0.5).exp_().mul_(-rate)
    s["beta"] = torch.sigmoid_(_randn(g, B, T, N))
    s["H0"] = _randn(g, B, N, K, V, scale=0.1) if c["carry"] else None
    train = c["kind"] == "delta_train"
    s["dy"] = _randn(g, B, T, N, V, dtype=dt) if train else None
    s["dHT"] = _randn(g, B, N, K, V, scale=0.1) if train and c["carry"] else None
    if own:
        s["delta"] = _library().Delta(B, T, N, K, V, c["io"], Nqk=Nqk, backward=train)
    return s


# ------------------------------------------------------------------ the calls
def _library():
    from paper_2603_14360_amd import binding
    return binding


def _own_norm(s, c):
    mb, stream = _library(), torch.cuda.current_stream().cuda_stream
    mode = (mb.M2RNN_NORM_CENTER if c["center"] else 0) | (mb.M2RNN_NORM_SILU if c["act"] == "silu" else 0)
    mb.m2rnn_group_norm_fwd(s["x"], s["a"], s["w"], s["b"], c["G"], _EPS, mode, s["out"], stream=stream)
    if c["kind"] == "norm_infer":
        return {"out": s["out"]}
    mb.m2rnn_group_norm_bwd(s["x"], s["a"], s["w"], s["b"], c["G"], _EPS, mode, s["dout"], s["dx"], s["da"], s["dw"],
                            s["db"], s["workspace"], stream=stream)
    return {n: s[n] for n in ("out", "dx", "da", "dw", "db") if s[n] is not None}


def _own_delta(s, c):
    y, HT = s["delta"].fwd(s["q"], s["k"], s["v"], s["g"], s["beta"], s["H0"])
    if c["kind"] != "delta_train":
        return {"y": y, "HT": HT}
    grads = s["delta"].bwd(s["q"], s["k"], s["v"], s["g"], s["beta"], s["H0"], s["dy"], s["dHT"])
    return dict(zip(("dq", "dk", "dv", "dg", "dbeta", "dH0"), grads), y=y, HT=HT)


def run(state):
    s, c = state, state["case"]
    if c["kind"] == "window":
        if not own:
            return _plain_window(s, c)
        _library().m2rnn_conv_silu_window_fwd(s["x"], s["w"], s["bias"], s["win"], s["out"], s["win_out"],
                                              stream=torch.cuda.current_stream().cuda_stream)
        return {"out": s["out"], "win": s["win_out"]}
    if c["kind"] in ("norm_train", "norm_infer"):
        return _own_norm(s, c) if own else _plain_norm(s, c)
    if own:
        return _own_delta(s, c)
    return _plain_step(s, c) if c["T"] == 1 else _plain_delta(s, c)


# ------------------------------------------------------------------ plain forms, in 32 bits
def _plain_window(s, c):
    T = c["T"]
    x = torch.cat([s["win"], s["x"]], dim=1).float()
    w = s["w"].float()
    u = x[:, 0:T] * w[:, 0] + x[:, 1:T + 1] * w[:, 1] + x[:, 2:T + 2] * w[:, 2] + x[:, 3:T + 3] * w[:, 3]
    if s["bias"] is not None:
        u = u + s["bias"].float()
    dt = s["x"].dtype
    return {"out": (u / (1 + torch.exp(-u))).to(dt), "win": x[:, T:T + 3].to(dt)}


def _plain_norm(s, c):
    dt, shape, groups = s["x"].dtype, s["x"].shape, (c["B"], c["T"], c["G"], c["L"])
    x, w = s["x"].float().view(groups), s["w"].float().view(c["G"], c["L"])
    mu = x.mean(-1, keepdim=True) if c["center"] else torch.zeros((), device="cuda")
    xc = x - mu
    r = 1 / torch.sqrt((xc * xc).mean(-1, keepdim=True) + _EPS)
    xh = xc * r
    n = xh * w
    if s["b"] is not None:
        n = n + s["b"].float().view(c["G"], c["L"])
    a = None if s["a"] is None else s["a"].float().view(groups)
    z = a if a is not None else n
    sg = 1 / (1 + torch.exp(-z))
    silu = z * sg
    out = n if c["act"] == "none" else silu if c["act"] == "silu" else n * silu
    res = {"out": out.reshape(shape).to(dt)}
    if c["kind"] == "norm_infer":
        return res
    d = s["dout"].float().view(groups)
    slope = sg * (1 + z * (1 - sg))
    dn = d if c["act"] == "none" else d * slope if c["act"] == "silu" else d * silu
    p = dn * w
    dx = p - xh * (p * xh).mean(-1, keepdim=True)
    if c["center"]:
        dx = dx - p.mean(-1, keepdim=True)
    res["dx"] = (dx * r).reshape(shape).to(dt)
    if a is not None:
        res["da"] = (d * n * slope).reshape(shape).to(dt)
    # (sums over as many terms as there are tokens: in 64 bits)
    res["dw"] = (dn * xh).double().sum((0, 1)).flatten().float()
    if s["b"] is not None:
        res["db"] = dn.double().sum((0, 1)).flatten().float()
    return res


def _plain_step(s, c):
    """One token: the recurrence as it is written."""
    rep = c["N"] // c["Nqk"]
    q, k = (s[n][:, 0].float().repeat_interleave(rep, 1) for n in ("q", "k"))
    H = torch.exp(s["g"][:, 0])[..., None, None] * s["H0"]
    r = s["v"][:, 0].float() - (k[..., None] * H).sum(2)
    H = H + k[..., None] * (s["beta"][:, 0][..., None] * r)[:, :, None, :]
    y = (q[..., None] * H).sum(2)
    return {"y": y[:, None].to(s["v"].dtype), "HT": H}


def _heads(x, rep, T):
    """[B,T,H,..] -> [B H rep, chunks, _CHUNK, ..], zeros behind the last step."""
    x = x.repeat_interleave(rep, 2).transpose(1, 2)
    x = torch.cat([x, x.new_zeros(x.shape[:2] + (-T % _CHUNK,) + x.shape[3:])], 2)
    return x.reshape((x.shape[0] * x.shape[1], -1, _CHUNK) + x.shape[3:])


def _steps(x, B, T, dt):
    """The way back: [B N, chunks, _CHUNK, ..] -> [B,T,N,..]."""
    x = x.reshape((B, -1, x.shape[1] * _CHUNK) + x.shape[3:])[:, :, :T]
    return x.transpose(1, 2).to(dt).contiguous()


def _plain_delta(s, c):
    """The rule by chunks of 64 steps.  With G the running sum of g inside a chunk, e_ij = exp(G_i - G_j) and
    H the state in front of it, the steps' updates u solve (I + A) u = beta (v - e^G H^T k), A strictly lower
    triangular with beta_i e_ij k_i.k_j: one triangular inverse T per chunk, then products."""
    B, T, N, K, V, dt, rep = c["B"], c["T"], c["N"], c["K"], c["V"], s["v"].dtype, c["N"] // c["Nqk"]
    q, k = _heads(s["q"].float(), rep, T), _heads(s["k"].float(), rep, T)
    v, beta = _heads(s["v"].float(), 1, T), _heads(s["beta"], 1, T)[..., None]
    G = _heads(s["g"].double(), 1, T).cumsum(2)
    lower = torch.ones(_CHUNK, _CHUNK, device="cuda", dtype=torch.bool).tril()
    e = (G[..., :, None] - G[..., None, :]).masked_fill_(~lower, -math.inf).exp_().float()
    ge, gl, gc = G.exp().float()[..., None], (G[..., -1:] - G).exp().float()[..., None], G[..., -1].exp().float()
    strict = e.tril(-1)
    P, D = e * (q @ k.transpose(-1, -2)), strict * (k @ k.transpose(-1, -2))
    A = beta * D
    Ti = torch.eye(_CHUNK, device="cuda").expand(A.shape).clone()
    for i in range(1, _CHUNK):  # rows of the inverse, each from those above it
        Ti[..., i, :i] = -(A[..., i:i + 1, :i] @ Ti[..., :i, :i])[..., 0, :]
    kl, kg, qg = (k * gl).transpose(-1, -2).contiguous(), k * ge, q * ge
    M, chunks = q.shape[0], q.shape[1]
    H = s["H0"].reshape(M, K, V) if s["H0"] is not None else torch.zeros(M, K, V, device="cuda")
    Hs = torch.empty(M, chunks, K, V, device="cuda")
    U = torch.empty_like(v)
    for i in range(chunks):  # states, which have to be in order
        Hs[:, i] = H
        U[:, i] = Ti[:, i] @ (beta[:, i] * (v[:, i] - kg[:, i] @ H))
        H = gc[:, i, None, None] * H + kl[:, i] @ U[:, i]
    y = qg @ Hs + P @ U
    res = {"y": _steps(y, B, T, dt), "HT": H.reshape(B, N, K, V)}
    if c["kind"] != "delta_train":
        return res
    dy = _heads(s["dy"].float(), 1, T)
    dH = s["dHT"].reshape(M, K, V) if s["dHT"] is not None else torch.zeros(M, K, V, device="cuda")
    dHs, Z = torch.empty_like(Hs), torch.empty_like(v)
    dU, TT = P.transpose(-1, -2).contiguous() @ dy, Ti.transpose(-1, -2).contiguous()
    qgT, bkT = qg.transpose(-1, -2).contiguous(), (beta * kg).transpose(-1, -2).contiguous()
    klT = kl.transpose(-1, -2).contiguous()
    for i in range(chunks - 1, -1, -1):  # gradients of the states behind the chunks
        dHs[:, i] = dH
        Z[:, i] = TT[:, i] @ (dU[:, i] + klT[:, i] @ dH)
        dH = gc[:, i, None, None] * dH + qgT[:, i] @ dy[:, i] - bkT[:, i] @ Z[:, i]
    HsT, UT = Hs.transpose(-1, -2).contiguous(), U.transpose(-1, -2).contiguous()
    S1, S2 = e * (dy @ UT), strict * (Z @ UT)
    S2b = (beta * S2).transpose(-1, -2).contiguous()
    dq = ge * (dy @ HsT) + S1 @ k
    asks = -(ge * (Z @ HsT) + S2 @ k)
    kept = gl * (U @ dHs.transpose(-1, -2).contiguous()) + S1.transpose(-1, -2).contiguous() @ q - S2b @ k
    dk = beta * asks + kept
    dbeta = (Z * v).sum(-1) + (k * asks).sum(-1)
    # (differences that sums over a chunk leave: in 64 bits)
    dG = (q.double() * dq + k.double() * (beta * asks - kept)).sum(-1)
    last = gc.double() * (Hs.double() * dHs).sum((-1, -2)) + (U.double() * (kl.transpose(-1, -2) @ dHs)).sum((-1, -2))
    dg = dG.flip(2).cumsum(2).flip(2) + last[..., None]
    share = lambda x: x.reshape(B, N // rep, rep, chunks, _CHUNK, K).sum(2).reshape(-1, chunks, _CHUNK, K)
    res["dq"], res["dk"] = _steps(share(dq), B, T, dt), _steps(share(dk), B, T, dt)
    res["dv"] = _steps(beta * Z, B, T, dt)
    res["dg"], res["dbeta"] = _steps(dg, B, T, dt), _steps(dbeta, B, T, dt)
    res["dH0"] = dH.reshape(B, N, K, V)
    return res


# ------------------------------------------------------------------ bytes and operations
def work(case):
    """Bytes: every input once, every output once.  Flops of the recurrence: H^T k, k u^T, H^T q forward;
    q dy^T, dH^T k, dH u, H dy, H u', k u'^T and <H, dH> backward, two each per state element and step."""
    c, io = case, 2 if case["io"] == "bf16" else 4
    if c["kind"] == "window":
        n = c["B"] * c["T"] * c["C"]
        return {"bytes": io * (2 * n + 6 * c["B"] * c["C"] + 5 * c["C"]), "flops": 12 * n}
    if c["kind"] in ("norm_train", "norm_infer"):
        D = c["G"] * c["L"]
        n, gate = c["B"] * c["T"] * D, int(c["act"] == "gate")
        if c["kind"] == "norm_infer":
            return {"bytes": io * (n * (2 + gate) + 2 * D), "flops": 10 * n}
        return {"bytes": io * (n * (4 + 2 * gate) + 2 * D) + 8 * D, "flops": 30 * n}
    B, T, N = c["B"], c["T"], c["N"]
    qk, v, gates, state = 2 * B * T * c["Nqk"] * c["K"] * io, B * T * N * c["V"] * io, 2 * B * T * N, B * N * c["K"] * c["V"] * 4
    states = 2 if c["carry"] else 1
    nbytes, flops = qk + 2 * v + 4 * gates + states * state, 6
    if c["kind"] == "delta_train":
        # dy in; dq, dk, dv, dg, dbeta, dH0 out; (dHT in)
        nbytes += qk + 2 * v + io * gates + states * state
        flops += 14
    return {"bytes": nbytes, "flops": flops * B * T * N * c["K"] * c["V"]}


# ------------------------------------------------------------------ the definition, in 64 bits
def _silu(z):
    return z * torch.sigmoid(z)


def _exact_window(s, c):
    x = torch.cat([s["win"], s["x"]], dim=1).double().transpose(1, 2)
    u = torch.stack([(x[:, :, t:t + 4] * s["w"].double()).sum(-1) for t in range(c["T"])], 1)
    if s["bias"] is not None:
        u = u + s["bias"].double()
    return {"out": _silu(u), "win": x[:, :, c["T"]:].transpose(1, 2)}


def _exact_norm(s, c):
    """The formula, and its gradients by differentiation of it."""
    leaves = {n: s[n].double().requires_grad_() for n in ("x", "a", "w", "b") if s[n] is not None}
    B, T, G, L = c["B"], c["T"], c["G"], c["L"]
    x = leaves["x"].reshape(B, T, G, L)
    if c["center"]:
        x = x - x.mean(-1, keepdim=True)
    n = (x / (x.square().mean(-1, keepdim=True) + _EPS).sqrt()).reshape(B, T, G * L) * leaves["w"]
    if "b" in leaves:
        n = n + leaves["b"]
    out = _silu(n) if c["act"] == "silu" else n * _silu(leaves["a"]) if c["act"] == "gate" else n
    res = {"out": out.detach()}
    if c["kind"] == "norm_train":
        names = sorted(leaves)
        grads = torch.autograd.grad(out, [leaves[n] for n in names], s["dout"].double())
        res.update({"d" + n: d for n, d in zip(names, grads)})
    return {n: res[n] for n in ("out", "dx", "da", "dw", "db") if n in res}


def _exact_delta(s, c):
    """Step by step, and back step by step; states are kept every 64 steps and made again in between."""
    B, T, N, K, V, rep = c["B"], c["T"], c["N"], c["K"], c["V"], c["N"] // c["Nqk"]
    M, S = B * N, 64
    flat = lambda x, r=1: x.double().repeat_interleave(r, 2).transpose(0, 1).reshape(T, M, *x.shape[3:])
    q, k, v, beta, gate = flat(s["q"], rep), flat(s["k"], rep), flat(s["v"]), flat(s["beta"]), flat(s["g"]).exp()
    state = lambda x: torch.zeros(M, K, V, device="cuda", dtype=torch.double) if x is None else x.double().reshape(M, K, V)
    H, y, kept = state(s["H0"]), torch.empty_like(v), []
    train = c["kind"] == "delta_train"

    def step(H, t):
        Hd = gate[t, :, None, None] * H
        delta = v[t] - torch.bmm(k[t][:, None], Hd)[:, 0]
        return Hd, delta, torch.baddbmm(Hd, k[t][:, :, None], (beta[t][:, None] * delta)[:, None])

    for t in range(T):
        if train and t % S == 0:
            kept.append(H)
        H = step(H, t)[2]
        y[t] = torch.bmm(q[t][:, None], H)[:, 0]
    back = lambda x: x.reshape(T, B, N, *x.shape[2:]).transpose(0, 1)
    res = {"y": back(y), "HT": H.reshape(B, N, K, V)}
    if not train:
        return res
    dy, dH = flat(s["dy"]), state(s["dHT"])
    dq, dk, dv, dg, db = (torch.empty_like(x) for x in (q, k, v, gate, beta))
    for t0 in range((T - 1) // S * S, -1, -S):
        tape, H = [], kept[t0 // S]
        for t in range(t0, min(t0 + S, T)):
            tape.append(step(H, t))
            H = tape[-1][2]
        for t in range(min(t0 + S, T) - 1, t0 - 1, -1):
            Hd, delta, H = tape[t - t0]
            u = beta[t][:, None] * delta
            dq[t] = torch.bmm(H, dy[t][:, :, None])[:, :, 0]
            dH = torch.baddbmm(dH, q[t][:, :, None], dy[t][:, None])
            du = torch.bmm(k[t][:, None], dH)[:, 0]
            db[t] = (du * delta).sum(-1)
            dv[t] = beta[t][:, None] * du
            dk[t] = torch.bmm(dH, u[:, :, None])[:, :, 0] - torch.bmm(Hd, dv[t][:, :, None])[:, :, 0]
            dH = torch.baddbmm(dH, k[t][:, :, None], -dv[t][:, None])
            dg[t] = (dH * Hd).sum((-1, -2))
            dH = gate[t, :, None, None] * dH
    share = lambda x: x.reshape(B, T, N // rep, rep, K).sum(3)
    res["dq"], res["dk"], res["dv"], res["dg"], res["dbeta"] = share(back(dq)), share(back(dk)), back(dv), back(dg), back(db)
    res["dH0"] = dH.reshape(B, N, K, V)
    return res


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "window":
        return _exact_window(s, c)
    if c["kind"] in ("norm_train", "norm_infer"):
        return _exact_norm(s, c)
    return _exact_delta(s, c)
