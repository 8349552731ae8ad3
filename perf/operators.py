"""Timed cases of the operators around the table-lookup layers: the linear layers that stay dense (a matrix product with bias,
activation and residual in its epilogue) and the layer norms between them, forward and backward.

A case is a dict of plain values; `path` names the entry point:

  dense           lut.dense_linear            Y = act(X W + b) + R, with X W + b kept where a backward pass follows
  dense_backward  lut.dense_linear_backward   gradients of X, W and b
  norm            lut.layer_norm              y = norm(x + r) w + b, with the sum and the statistics where they are kept
  norm_backward   lut.layer_norm_backward     gradients of x, w and b

N rows, D inputs, M outputs, `type` of the matrices; vectors (bias, weight, statistics) are fp32.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")
EPS = 1e-5


def listed():
    return [
        # one token through a feed-forward layer's first half: serving, where the weights' bytes and launches count
        dict(name="dense_token_bf16", path="dense", N=1, D=1024, M=4096, type="bf16", activation="gelu", bias=True, residual=False,
             keep=False),
        # the attention output of a short sentence, BERT-base width: little work, two row tiles at most
        dict(name="dense_sentence_f32", path="dense", N=37, D=768, M=768, type="f32", activation="none", bias=True, residual=True,
             keep=False),
        # BERT-base QKV at batch 32 x 128 tokens, in the type that the table-lookup layers compute in
        dict(name="dense_qkv_f32", path="dense", N=4096, D=768, M=2304, type="f32", activation="none", bias=True, residual=False,
             keep=False),
        # sizes that are no multiple of anything, rows that are not aligned
        dict(name="dense_odd_f16", path="dense", N=1001, D=515, M=1030, type="f16", activation="silu", bias=True, residual=True,
             keep=False),
        # a training step's feed-forward half, the values before the activation kept
        dict(name="dense_ffn_bf16", path="dense", N=16384, D=1024, M=4096, type="bf16", activation="gelu", bias=True,
             residual=False, keep=True),
        # the size of the largest table-lookup benchmark as a dense layer with a residual
        dict(name="dense_large_bf16", path="dense", N=16384, D=4096, M=4096, type="bf16", activation="none", bias=True,
             residual=True, keep=False),
        # the same layers' backward passes, small and large
        dict(name="dense_backward_f32", path="dense_backward", N=4096, D=768, M=2304, type="f32", activation="gelu"),
        dict(name="dense_backward_large_bf16", path="dense_backward", N=8192, D=4096, M=4096, type="bf16",
             activation="gelu_tanh"),
        # one token's norm behind a residual: latency
        dict(name="norm_token_f32", path="norm", N=1, D=768, type="f32", residual=True, keep=False),
        # a training step's norm, the sum and the statistics kept
        dict(name="norm_large_bf16", path="norm", N=16384, D=4096, type="bf16", residual=True, keep=True),
        # BERT-base at batch 32 x 128, and the large one with the gradient that comes by the residual added
        dict(name="norm_backward_f32", path="norm_backward", N=4096, D=768, type="f32", residual=False),
        dict(name="norm_backward_large_bf16", path="norm_backward", N=16384, D=4096, type="bf16", residual=True),
    ]


def _log_uniform(rng, low, high):
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def _width(rng, low, high):
    """A layer width: mostly whole vectors, one in four of any size."""
    n = _log_uniform(rng, low, high)
    return n if rng.random() < 0.25 else max(low, n // 64 * 64)


def draw(rng):
    path = rng.choice(("dense", "dense", "dense_backward", "norm", "norm_backward"))
    kind = rng.choice(tuple(TYPES))
    if path.startswith("norm"):
        N, D = _log_uniform(rng, 1, 16384), _width(rng, 64, 4096)
        case = dict(path=path, N=N, D=D, type=kind, residual=rng.random() < 0.5)
        if path == "norm":
            case["keep"] = rng.random() < 0.5
        return _afforded(case)
    N, D, M = _log_uniform(rng, 1, 16384), _width(rng, 64, 4096), _width(rng, 64, 4096)
    case = dict(path=path, N=N, D=D, M=M, type=kind, activation=rng.choice(ACTIVATIONS))
    if path == "dense":
        case.update(bias=rng.random() < 0.75, residual=rng.random() < 0.5, keep=rng.random() < 0.3)
    return _afforded(case)


def _afforded(case):
    """No more bytes or operations than the largest listed cases."""
    while work(case)["bytes"] > 540e6 or work(case)["flops"] > 550e9:
        case["N"] = case["N"] * 3 // 4
    return case


def _inputs(case, seed):
    """Activations of unit size with one in a hundred ten times larger, weights that keep the size, biases and gradients."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    T, N, D = TYPES[case["type"]], case["N"], case["D"]

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=g, device="cuda") * std

    def outliers(t):
        return torch.where(torch.rand(t.shape, generator=g, device="cuda") < 0.01, t * 10, t)

    s = {"X": outliers(normal(N, D)).to(T)}
    if case["path"].startswith("dense"):
        M = case["M"]
        s["W"] = normal(D, M, std=1 / math.sqrt(D)).to(T)
        s["b"] = normal(M, std=0.1)
        if case["path"] == "dense_backward":
            s["Z"] = (s["X"].float() @ s["W"].float() + s["b"]).to(T)
            s["G"] = normal(N, M).to(T)
        else:
            s["b"] = s["b"] if case["bias"] else None
            s["R"] = normal(N, M).to(T) if case["residual"] else None
        return s
    s["w"], s["b"] = 1 + normal(D, std=0.1), normal(D, std=0.1)
    s["R"] = normal(N, D).to(T) if case["residual"] else None
    if case["path"] == "norm_backward":
        s["G"] = normal(N, D).to(T)
        x = s["X"].float()
        mean = x.mean(dim=1, keepdim=True)
        s["statistics"] = torch.cat((mean, ((x - mean) ** 2).mean(dim=1, keepdim=True).add(EPS).rsqrt()), dim=1)
    return s


def prepare(case, seed):
    return dict(_inputs(case, seed), case=case)


def _activation(z, kind):
    if kind == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if kind == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if kind == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if kind == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _slope(z, kind):
    if kind == "relu":
        return (z > 0).float()
    if kind == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if kind == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    if kind == "silu":
        e = 1 / (1 + torch.exp(-z))
        return e * (1 + z * (1 - e))
    return torch.ones_like(z)


def _plain_dense(s, case):
    z = s["X"].float() @ s["W"].float()
    if s["b"] is not None:
        z = z + s["b"]
    y = _activation(z, case["activation"])
    if s["R"] is not None:
        y = y + s["R"].float()
    T = s["X"].dtype
    return [y.to(T), z.to(T)] if case["keep"] else [y.to(T)]


def _plain_dense_backward(s, case):
    dz = s["G"].float()
    if case["activation"] != "none":
        dz = dz * _slope(s["Z"].float(), case["activation"])
    T = s["X"].dtype
    return [(dz @ s["W"].float().t()).to(T), (s["X"].float().t() @ dz).to(T), dz.sum(dim=0)]


def _plain_norm(s, case):
    x = s["X"].float()
    if s["R"] is not None:
        x = x + s["R"].float()
    mean = x.sum(dim=1, keepdim=True) / case["D"]
    far = x - mean
    rstd = 1 / torch.sqrt((far * far).sum(dim=1, keepdim=True) / case["D"] + EPS)
    T = s["X"].dtype
    y = (far * rstd * s["w"] + s["b"]).to(T)
    if not case["keep"]:
        return [y]
    statistics = torch.cat((mean, rstd), dim=1)
    return [y, statistics] if s["R"] is None else [y, statistics, x.to(T)]


def _plain_norm_backward(s, case):
    mean, rstd = s["statistics"][:, :1], s["statistics"][:, 1:]
    h, g = (s["X"].float() - mean) * rstd, s["G"].float()
    q = g * s["w"]
    dx = rstd * (q - q.sum(dim=1, keepdim=True) / case["D"] - h * ((q * h).sum(dim=1, keepdim=True) / case["D"]))
    if s["R"] is not None:
        dx = dx + s["R"].float()
    return [dx.to(s["X"].dtype), (g * h).sum(dim=0), g.sum(dim=0)]


def _own(s, case):
    import paper_2302_03213_amd as lut
    X, path = s["X"], case["path"]
    if path == "dense":
        Z = torch.empty((case["N"], case["M"]), dtype=X.dtype, device=X.device) if case["keep"] else None
        Y = lut.dense_linear(X, s["W"], bias=s["b"], activation=_named(case), residual=s["R"], preactivation=Z)
        return [Y, Z] if case["keep"] else [Y]
    if path == "dense_backward":
        kept = s["Z"] if case["activation"] != "none" else None
        return list(lut.dense_linear_backward(X, s["W"], s["G"], preactivation=kept, activation=_named(case)))
    if path == "norm":
        if not case["keep"]:
            return [lut.layer_norm(X, s["w"], s["b"], EPS, residual=s["R"])]
        statistics = torch.empty((case["N"], 2), device=X.device)
        total = None if s["R"] is None else torch.empty_like(X)
        Y = lut.layer_norm(X, s["w"], s["b"], EPS, residual=s["R"], total=total, statistics=statistics)
        return [Y, statistics] if total is None else [Y, statistics, total]
    return list(lut.layer_norm_backward(s["G"], X, s["statistics"], weight=s["w"], residual=s["R"]))


def _named(case):
    return None if case["activation"] == "none" else case["activation"]


def run(state):
    case = state["case"]
    if own:
        return _own(state, case)
    return {"dense": _plain_dense, "dense_backward": _plain_dense_backward, "norm": _plain_norm,
            "norm_backward": _plain_norm_backward}[case["path"]](state, case)


def work(case):
    N, D, e = case["N"], case["D"], 4 if case["type"] == "f32" else 2
    if case["path"] == "dense":
        M = case["M"]
        written = N * M * (2 if case["keep"] else 1)
        return {"bytes": e * (N * D + D * M + written + (N * M if case["residual"] else 0)) + (4 * M if case["bias"] else 0),
                "flops": 2 * N * D * M}
    if case["path"] == "dense_backward":
        M = case["M"]
        read = N * D + D * M + N * M * (1 if case["activation"] == "none" else 2)
        return {"bytes": e * (read + N * D + D * M) + 4 * M, "flops": 4 * N * D * M}
    if case["path"] == "norm":
        matrices = 2 + (1 if case["residual"] else 0) + (1 if case["residual"] and case["keep"] else 0)
        return {"bytes": e * N * D * matrices + 8 * D + (8 * N if case["keep"] else 0), "flops": 8 * N * D}
    return {"bytes": e * N * D * (4 if case["residual"] else 3) + 8 * N + 12 * D, "flops": 14 * N * D}


def exact(case, seed):
    """The definitions in 64 bits: torch's own functions and their derivatives by autograd."""
    s = {k: None if v is None else v.double() for k, v in _inputs(case, seed).items()}
    functional = torch.nn.functional
    activation = {"none": lambda z: z, "relu": functional.relu, "gelu": functional.gelu, "silu": functional.silu,
                  "gelu_tanh": lambda z: functional.gelu(z, approximate="tanh")}
    if case["path"] == "dense":
        z = torch.addmm(s["b"] if s["b"] is not None else s["X"].new_zeros(case["M"]), s["X"], s["W"])
        y = activation[case["activation"]](z)
        y = y if s["R"] is None else y + s["R"]
        return [y, z] if case["keep"] else [y]
    if case["path"] == "dense_backward":
        Z = s["Z"].requires_grad_()
        dz, = torch.autograd.grad(activation[case["activation"]](Z), Z, s["G"])
        return [dz @ s["W"].t(), s["X"].t() @ dz, dz.sum(dim=0)]
    D = case["D"]
    if case["path"] == "norm":
        x = s["X"] if s["R"] is None else s["X"] + s["R"]
        y = functional.layer_norm(x, (D,), s["w"], s["b"], EPS)
        if not case["keep"]:
            return [y]
        var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        statistics = torch.cat((mean, (var + EPS) ** -0.5), dim=1)
        return [y, statistics] if s["R"] is None else [y, statistics, x]
    leaves = [s[k].requires_grad_() for k in ("X", "w", "b")]
    dx, dw, db = torch.autograd.grad(functional.layer_norm(leaves[0], (D,), leaves[1], leaves[2], EPS), leaves, s["G"])
    return [dx if s["R"] is None else dx + s["R"], dw, db]
