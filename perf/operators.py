"""What the row operators of transformer blocks on sparse tensors are measured on: layer norm, rotary positions at the
rows' coordinates, and the gated feed-forward block, forward and backward, over the sizes a program calls them at.

A case is a dict of plain values; ``op`` names the operator:

  norm      layer norm of feature rows; ``train``: forward with its statistics, then the backward pass with the gradients
            of the weight and the bias, else the forward alone;
  rotary    the rows' queries and keys (``heads`` of ``d`` channels inside rows of ``ld``) rotated at their coordinates;
            ``train``: then the gradient of the rotated rows rotated back;
  ffn       (act(X Wg) * (X Wu)) Wd; ``train``: forward and backward with all gradients, else the forward alone.

``own`` chooses between the plain form (elementary torch operations in 32 bits) and the library's calls.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def listed():
    return [
        # serving: the rows of one small sample through a norm (latency of one call)
        dict(name="norm_infer_2k_c32", op="norm", n=2000, c=32, dtype="f32", train=False),
        # training: the finest level of two indoor rooms (2 cm) at the width of the bf16 networks
        dict(name="norm_train_scene_c256_bf16", op="norm", n=300_000, c=256, dtype="bf16", train=True),
        # training: a 3D video of three frames in float32
        dict(name="norm_train_video_c96", op="norm", n=120_011, c=96, dtype="f32", train=True),
        # training: wide rows of an odd width (no 16-byte groups), as of concatenated features
        dict(name="norm_train_odd_c1027_bf16", op="norm", n=20_011, c=1027, dtype="bf16", train=True),
        # serving: queries and keys of a small sample, three axes, some channels left unrotated
        dict(name="rotary_infer_2k", op="rotary", n=2000, heads=8, d=16, ld=128, D=3, axes="2,2,2", pairing="adjacent",
             scale=1.0, far=0, dtype="f32", train=False),
        # queries and keys of 8 heads each, as they lie in the rows of one projection (queries, keys, values)
        dict(name="rotary_scene_qk_bf16", op="rotary", n=300_000, heads=16, d=32, ld=768, D=3, axes="6,5,5",
             pairing="halves", scale=0.5, far=0, dtype="bf16", train=False),
        # training on a 3D video: three axes of space and one of time, far from the origin
        dict(name="rotary_train_video", op="rotary", n=120_011, heads=6, d=64, ld=384, D=4, axes="8,8,8,8",
             pairing="adjacent", scale=1.0, far=1_000_000, dtype="f32", train=True),
        # serving: a single row (a global feature)
        dict(name="ffn_infer_one_c256_bf16", op="ffn", n=1, c=256, hidden=1024, act="silu", dtype="bf16", train=False),
        # serving: one room at 5 cm
        dict(name="ffn_infer_room_c64_bf16", op="ffn", n=12_007, c=64, hidden=256, act="gelu", dtype="bf16",
             train=False),
        # training: two indoor rooms at 2 cm, 256 channels: the largest by arithmetic
        dict(name="ffn_train_scene_c256_bf16", op="ffn", n=300_000, c=256, hidden=1024, act="silu", dtype="bf16",
             train=True),
        # training: a 3D video in float32
        dict(name="ffn_train_video_c64", op="ffn", n=120_011, c=64, hidden=256, act="silu", dtype="f32", train=True),
        # training: odd widths, two thirds of the usual hidden width, as parameter counts are matched
        dict(name="ffn_train_odd_c100_bf16", op="ffn", n=30_011, c=100, hidden=267, act="gelu_tanh", dtype="bf16",
             train=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "rotary", "ffn", "ffn"])
    dtype = rng.choice(["f32", "bf16"])
    train = rng.random() < 0.6
    if op == "norm":
        c = rng.choice([_log(rng, 3, 2048), 8 * _log(rng, 2, 256)])
        return dict(op=op, n=_log(rng, 1, min(300_000, 76_800_000 // c)), c=c, dtype=dtype, train=train)
    if op == "rotary":
        d, D = 2 * _log(rng, 2, 64), rng.randint(1, 4)
        heads = rng.randint(1, 16)
        left, axes = d // 2, []
        for a in range(D):
            axes.append(rng.randint(0 if a else 1, max(1, left // (D - a))) if left else 0)
            left -= axes[-1]
        ld = heads * d * rng.choice([1, 1, 3]) + rng.choice([0, 0, 5])
        return dict(op=op, n=_log(rng, 1, min(300_000, 150_000_000 // ld)), heads=heads, d=d, ld=ld, D=D,
                    axes=",".join(map(str, axes)), pairing=rng.choice(["adjacent", "halves"]),
                    scale=rng.choice([1.0, 0.5, 0.02]), far=rng.choice([0, 0, 30_000, 1_000_000]), dtype=dtype,
                    train=train)
    c = rng.choice([_log(rng, 8, 512), 32 * rng.randint(1, 12)])
    hidden = rng.choice([4 * c, max(8, 8 * c // 3), _log(rng, 16, 2048)])
    most = (300_000 * 256 * 1024) // (c * hidden) // (8 if dtype == "f32" else 1)
    return dict(op=op, n=_log(rng, 1, max(1, min(300_000, most))), c=c, hidden=hidden,
                act=rng.choice(["silu", "gelu", "gelu_tanh", "relu", "sigmoid"]), dtype=dtype, train=train)


# --------------------------------------------------------------------------- #
# inputs
# --------------------------------------------------------------------------- #
def _axes(case):
    return [int(v) for v in case["axes"].split(",")]


def prepare(case, seed):
    g = torch.Generator(DEV).manual_seed(int(seed) * 7919 + 17)
    dt = TYPES[case["dtype"]]
    n = case["n"]

    def normal(*shape, by=1.0):
        return (torch.randn(shape, generator=g, device=DEV) * by).to(dt)

    s = dict(case=case)
    if case["op"] == "norm":
        c = case["c"]
        # a convolution's rows: each row of its own size and offset, some channels larger than others
        row = 0.25 + 2.0 * torch.rand((n, 1), generator=g, device=DEV)
        col = 0.5 + torch.rand((1, c), generator=g, device=DEV)
        s["X"] = ((torch.randn((n, c), generator=g, device=DEV) * col + 0.3) * row).to(dt)
        s["gamma"] = 1.0 + 0.2 * torch.randn(c, generator=g, device=DEV)
        s["beta"] = 0.1 * torch.randn(c, generator=g, device=DEV)
        if case["train"]:
            s["dY"] = normal(n, c)
    elif case["op"] == "rotary":
        D, H, d, ld = case["D"], case["heads"], case["d"], case["ld"]
        rows = normal(n, ld)
        s["X"] = rows[:, :H * d].view(n, H, d)   # heads inside wider rows
        x = torch.randint(-400, 400, (n, D), generator=g, device=DEV, dtype=torch.int32) + int(case["far"])
        b = torch.randint(0, 4, (n, 1), generator=g, device=DEV, dtype=torch.int32)
        s["coords"] = torch.cat([b, x], 1).contiguous()
        if case["train"]:
            s["dY"] = normal(n, H, d)
    else:
        c, f = case["c"], case["hidden"]
        s["X"] = normal(n, c)
        s["Wg"] = normal(c, f, by=c ** -0.5)
        s["Wu"] = normal(c, f, by=c ** -0.5)
        s["Wd"] = normal(f, c, by=f ** -0.5)
        if case["train"]:
            s["dY"] = normal(n, c)
    return s


# --------------------------------------------------------------------------- #
# one pass
# --------------------------------------------------------------------------- #
def run(state):
    case = state["case"]
    if own:
        return {"norm": _own_norm, "rotary": _own_rotary, "ffn": _own_ffn}[case["op"]](state, case)
    return {"norm": _norm, "rotary": _rotary, "ffn": _ffn}[case["op"]](state, case)


def _own_norm(s, case):
    from paper_1904_08755_amd import gsc
    if not case["train"]:
        return gsc.gsc_layer_norm_fwd(s["X"], s["gamma"], s["beta"], EPS, stats=False)[0]
    Y, mean, rstd = gsc.gsc_layer_norm_fwd(s["X"], s["gamma"], s["beta"], EPS)
    dX, dgamma, dbeta = gsc.gsc_layer_norm_bwd(s["X"], s["dY"], mean, rstd, s["gamma"])
    return dict(Y=Y, mean=mean, rstd=rstd, dX=dX, dgamma=dgamma, dbeta=dbeta)


def _own_rotary(s, case):
    from paper_1904_08755_amd import gsc
    kw = dict(scale=[case["scale"]] * case["D"], pairing=case["pairing"])
    Y = gsc.gsc_rotary(s["X"], s["coords"], _axes(case), **kw)
    if not case["train"]:
        return Y
    return dict(Y=Y, dX=gsc.gsc_rotary(s["dY"], s["coords"], _axes(case), inverse=True, **kw))


def _own_ffn(s, case):
    from paper_1904_08755_amd import gsc
    Y = gsc.gsc_gated_ffn_fwd(s["X"], s["Wg"], s["Wu"], s["Wd"], act=case["act"])
    if not case["train"]:
        return Y
    dX, dWg, dWu, dWd = gsc.gsc_gated_ffn_bwd(s["X"], s["Wg"], s["Wu"], s["Wd"], s["dY"], act=case["act"])
    return dict(Y=Y, dX=dX, dWg=dWg, dWu=dWu, dWd=dWd)


def _norm(s, case):
    x = s["X"].float()
    mean = x.mean(1)
    xc = x - mean[:, None]
    rstd = torch.rsqrt((xc * xc).mean(1) + EPS)
    xh = xc * rstd[:, None]
    Y = (xh * s["gamma"] + s["beta"]).to(s["X"].dtype)
    if not case["train"]:
        return Y
    dy = s["dY"].float()
    g = dy * s["gamma"]
    dx = (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) * rstd[:, None]
    return dict(Y=Y, mean=mean, rstd=rstd, dX=dx.to(s["X"].dtype), dgamma=(dy * xh).sum(0), dbeta=dy.sum(0))


def _turns(case, coords):
    """cos and sin (n, 1, d/2) of every pair's angle, the angle in 64 bits; 1 and 0 where no axis turns the pair."""
    parts = [coords[:, 1 + a, None].double() * (case["scale"] * torch.exp2(
        torch.arange(p, device=coords.device, dtype=torch.float64) * (-math.log2(10000.0) / max(p, 1))))
        for a, p in enumerate(_axes(case))]
    t = torch.cat(parts, 1)
    rest = case["d"] // 2 - t.shape[1]
    t = torch.cat([t, t.new_zeros((t.shape[0], rest))], 1)[:, None]
    return t.cos().float(), t.sin().float()


def _turned(x, cos, sin, pairing):
    v = x.float()
    if pairing == "halves":
        h = v.shape[2] // 2
        p, q = v[..., :h], v[..., h:]
        return torch.cat([p * cos - q * sin, p * sin + q * cos], 2).to(x.dtype)
    p, q = v[..., 0::2], v[..., 1::2]
    return torch.stack([p * cos - q * sin, p * sin + q * cos], 3).flatten(2).to(x.dtype)


def _rotary(s, case):
    cos, sin = _turns(case, s["coords"])
    Y = _turned(s["X"], cos, sin, case["pairing"])
    if not case["train"]:
        return Y
    return dict(Y=Y, dX=_turned(s["dY"], cos, -sin, case["pairing"]))


def _gate(act, g):
    """act(g) and its derivative."""
    if act == "relu":
        return g.clamp(min=0), (g > 0).float()
    if act in ("silu", "sigmoid"):
        p = 1 / (1 + torch.exp(-g))
        return (p, p * (1 - p)) if act == "sigmoid" else (g * p, p * (1 + g * (1 - p)))
    if act == "gelu":
        p = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * p, p + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)


def _ffn(s, case):
    dt = s["X"].dtype
    X, Wg, Wu, Wd = (s[k].float() for k in ("X", "Wg", "Wu", "Wd"))
    G, U = X @ Wg, X @ Wu
    a, da = _gate(case["act"], G)
    H = a * U
    Y = (H @ Wd).to(dt)
    if not case["train"]:
        return Y
    dY = s["dY"].float()
    dH = dY @ Wd.t()
    dG, dU = dH * U * da, dH * a
    return dict(Y=Y, dX=(dG @ Wg.t() + dU @ Wu.t()).to(dt), dWg=(X.t() @ dG).to(dt), dWu=(X.t() @ dU).to(dt),
                dWd=(H.t() @ dY).to(dt))


# --------------------------------------------------------------------------- #
# the least work, and 64-bit results
# --------------------------------------------------------------------------- #
def work(case):
    n, size, train = case["n"], 4 if case["dtype"] == "f32" else 2, case["train"]
    if case["op"] == "norm":
        c = case["c"]
        return {"bytes": n * c * size * (5 if train else 2) + c * (24 if train else 8) + (16 * n if train else 0),
                "flops": n * c * (20 if train else 8)}
    if case["op"] == "rotary":
        v = n * case["heads"] * case["d"]
        return {"bytes": v * size * (4 if train else 2) + n * 4 * (1 + case["D"]) * (2 if train else 1),
                "flops": v * 3 * (2 if train else 1)}
    c, f = case["c"], case["hidden"]
    return {"bytes": (n * c * (5 if train else 2) + 3 * c * f * (3 if train else 1)) * size,
            "flops": 2 * n * c * f * (9 if train else 3)}


EXACT_ROWS = 32768


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "rotary": _exact_rotary, "ffn": _exact_ffn}[case["op"]](s, case)


def _exact_norm(s, case):
    gamma, beta = (s[k].double().requires_grad_() for k in ("gamma", "beta"))
    X = s["X"].double().requires_grad_()
    c = case["c"]
    mean = torch.sum(X, 1) / c
    var = torch.sum(torch.square(X - mean.unsqueeze(1)), 1) / c
    rstd = 1.0 / torch.sqrt(var + EPS)
    Y = torch.addcmul(beta, (X - mean.unsqueeze(1)) * rstd.unsqueeze(1), gamma)
    if not case["train"]:
        return Y.detach()
    dX, dgamma, dbeta = torch.autograd.grad(Y, (X, gamma, beta), s["dY"].double())
    return dict(Y=Y.detach(), mean=mean.detach(), rstd=rstd.detach(), dX=dX, dgamma=dgamma, dbeta=dbeta)


def _exact_rotary(s, case):
    def turned(x, sign):
        """Each pair as a complex number, times exp(i sign t)."""
        z = x.double().clone()
        at, d = 0, case["d"]
        for a, p in enumerate(_axes(case)):
            for j in range(p):
                lo, hi = (at, at + d // 2) if case["pairing"] == "halves" else (2 * at, 2 * at + 1)
                t = sign * s["coords"][:, 1 + a].double() * (case["scale"] * 10000.0 ** (-j / p))
                w = torch.complex(x[..., lo].double(), x[..., hi].double()) * torch.polar(torch.ones_like(t), t)[:, None]
                z[..., lo], z[..., hi] = w.real, w.imag
                at += 1
        return z

    Y = turned(s["X"], 1.0)
    return dict(Y=Y, dX=turned(s["dY"], -1.0)) if case["train"] else Y


def _exact_ffn(s, case):
    W = [s[k].double().requires_grad_(case["train"]) for k in ("Wg", "Wu", "Wd")]
    act = {"silu": lambda g: g * torch.sigmoid(g), "sigmoid": torch.sigmoid, "relu": torch.relu,
           "gelu": lambda g: 0.5 * g * torch.erfc(-g / math.sqrt(2.0)),
           "gelu_tanh": lambda g: g * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3))}[case["act"]]
    Ys, dXs = [], []
    for r in range(0, case["n"], EXACT_ROWS):
        X = s["X"][r:r + EXACT_ROWS].double().requires_grad_(case["train"])
        Y = torch.mm(act(torch.mm(X, W[0])) * torch.mm(X, W[1]), W[2])
        Ys.append(Y.detach())
        if case["train"]:
            Y.backward(s["dY"][r:r + EXACT_ROWS].double())
            dXs.append(X.grad)
    if not case["train"]:
        return torch.cat(Ys)
    return dict(Y=torch.cat(Ys), dX=torch.cat(dXs), dWg=W[0].grad, dWu=W[1].grad, dWd=W[2].grad)
