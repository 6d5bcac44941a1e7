"""Timed cases of the training-step operators around the attributed linears.

Five calls, each a pass of its own: the linear layer with bias, activation and residual in its epilogue, its
backward pass (the factor B = dY act'(Z) that the attribution reads, dX, dW, db), the embedding lookup, its
gradient by sorted tokens, and the global gradient norm with clipping. ``run`` computes them either in a plain
form (elementary torch operations in 32 bits) or through the package's entry points (``own``).
"""
import math

import numpy as np
import torch

own = False

_T = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}
_ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token through a gate projection: the weights are all there is to read
        dict(name="linear_token", op="linear_forward", M=1, d_in=4096, d_out=14336, dtype="bf16", act="silu",
             bias=False, residual=False, keep_z=False, gap=0),
        # a small fp32 layer, as in the repository's smallest workload, an odd number of tokens
        dict(name="linear_small_f32", op="linear_forward", M=2047, d_in=256, d_out=256, dtype="f32", act="relu",
             bias=True, residual=False, keep_z=True, gap=0),
        # eight examples of 512 tokens through an up projection of a 2048-wide block, pre-activation kept
        dict(name="linear_up", op="linear_forward", M=4096, d_in=2048, d_out=8192, dtype="bf16", act="gelu_tanh",
             bias=True, residual=False, keep_z=True, gap=0),
        # eight examples of 1024 tokens through a down projection that adds the residual stream
        dict(name="linear_down_large", op="linear_forward", M=8192, d_in=14336, d_out=4096, dtype="bf16", act="none",
             bias=True, residual=True, keep_z=False, gap=0),
        # backward of an up projection, ragged batch (examples packed without padding), strided gradients
        dict(name="linear_up_backward", op="linear_backward", M=1999, d_in=2048, d_out=8192, dtype="bf16",
             act="silu", bias=True, grads="bf16", gap=64),
        # backward of an fp32 layer of odd widths
        dict(name="linear_odd_backward_f32", op="linear_backward", M=1021, d_in=1000, d_out=1363, dtype="f32",
             act="gelu", bias=True, grads="f32", gap=0),
        # the lookup of a prompt's tokens, and of a training batch
        dict(name="embedding_prompt", op="embedding_forward", n=509, vocab=32000, d=2048, dtype="bf16", index="i64",
             scale=1.0),
        dict(name="embedding_batch", op="embedding_forward", n=32768, vocab=131072, d=4096, dtype="bf16", index="i32",
             scale=64.0),
        # the gradient of a table after one small batch, and after a large one
        dict(name="embedding_grad", op="embedding_backward", n=4096, vocab=32000, d=2048, dtype="bf16", index="i64",
             scale=1.0, grads="f32"),
        dict(name="embedding_grad_large", op="embedding_backward", n=65536, vocab=131072, d=4096, dtype="bf16",
             index="i32", scale=64.0, grads="bf16"),
        # the gradients of one small fp32 layer stack, and of a stack of 2048-wide blocks
        dict(name="clip_small", op="clip", layers=4, d=256, ff=512, dtype="f32", max_norm=1.0),
        dict(name="clip_blocks", op="clip", layers=8, d=2048, ff=8192, dtype="bf16", max_norm=1.0),
    ]


def _log_int(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v))


def _width(rng, lo, hi):
    """A layer width: mostly multiples of 64, now and then any number."""
    v = _log_int(rng, lo, hi)
    return v if rng.random() < 0.2 else max(64, v // 64 * 64)


def draw(rng):
    op = rng.choice(["linear_forward", "linear_forward", "linear_backward", "embedding_forward",
                     "embedding_backward", "clip"])
    if op in ("linear_forward", "linear_backward"):
        dtype = rng.choice(["bf16", "bf16", "f32"])
        top = 9e11 if dtype == "bf16" else 2e11
        while True:
            M, di, do = _log_int(rng, 1, 8192), _width(rng, 64, 14336), _width(rng, 64, 14336)
            if (2 if op == "linear_forward" else 4) * M * di * do <= top:
                break
        case = dict(op=op, M=M, d_in=di, d_out=do, dtype=dtype, act=rng.choice(_ACTS), bias=rng.random() < 0.5,
                    gap=rng.choice([0, 0, 64, 24]))
        if op == "linear_forward":
            return dict(case, residual=rng.random() < 0.5, keep_z=rng.random() < 0.5)
        # fp32 gradients from bf16 layers where the factor is the incoming gradient itself
        return dict(case, grads="f32" if dtype == "f32" or (case["act"] == "none" and rng.random() < 0.5) else "bf16")
    if op in ("embedding_forward", "embedding_backward"):
        dtype = rng.choice(["bf16", "bf16", "f32"])
        case = dict(op=op, n=_log_int(rng, 1, 65536), vocab=_log_int(rng, 1000, 131072), d=_width(rng, 64, 4096),
                    dtype=dtype, index=rng.choice(["i32", "i64"]), scale=rng.choice([1.0, 8.0, 0.25]))
        return dict(case, grads=rng.choice(["f32", dtype])) if op == "embedding_backward" else case
    return dict(op="clip", layers=rng.randint(1, 6), d=_width(rng, 64, 2048), ff=_width(rng, 64, 8192),
                dtype=rng.choice(["bf16", "f32"]), max_norm=rng.choice([0.5, 1.0, 1e6]))


# ------------------------------------------------------------------------------------------------ inputs
def _normal(gen, shape, sigma, dtype):
    out = torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, sigma, generator=gen)
    return out.to(_T[dtype])


def _rows(gen, n, d, gap, sigma, dtype, masked=False):
    """n rows of d values in rows of d + gap; masked: one token in a hundred is padding, a zero row."""
    wide = _normal(gen, (n, d + gap), sigma, dtype)
    if masked:
        wide *= (torch.rand((n, 1), generator=gen, device="cuda") >= 0.01).to(wide.dtype)
    return wide[:, :d]


def _tokens(gen, n, vocab, index):
    """Token ids of log-uniform rank (word frequencies fall about as 1/rank); one in fifty is padding, -1."""
    u = torch.rand((n,), generator=gen, device="cuda", dtype=torch.float64)
    ids = torch.exp(u * math.log(vocab + 1.0)).floor().long() - 1
    ids = ids.clamp(0, vocab - 1)
    pad = torch.rand((n,), generator=gen, device="cuda") < 0.02
    return torch.where(pad, torch.full_like(ids, -1), ids).to(torch.int32 if index == "i32" else torch.int64)


def _block_shapes(case):
    """A stack of blocks: four d x d and three d x ff matrices and two vectors of d each."""
    d, ff = case["d"], case["ff"]
    one = [(d, d)] * 4 + [(ff, d), (ff, d), (d, ff)] + [(d,), (d,)]
    return one * case["layers"]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    op, dev = case["op"], "cuda"
    s = dict(case=case)
    if op == "linear_forward":
        M, di, do, dt, gap = case["M"], case["d_in"], case["d_out"], case["dtype"], case["gap"]
        s["X"] = _rows(gen, M, di, gap, 1.0, dt)
        s["W"] = _normal(gen, (do, di), 1.0 / math.sqrt(di), dt)
        s["bias"] = _normal(gen, (do,), 0.1, dt) if case["bias"] else None
        s["R"] = _rows(gen, M, do, gap, 1.0, dt) if case["residual"] else None
        s["Y"] = torch.empty((M, do), dtype=_T[dt], device=dev)
        s["Z"] = torch.empty((M, do), dtype=_T[dt], device=dev) if case["keep_z"] else None
    elif op == "linear_backward":
        M, di, do, dt, gap = case["M"], case["d_in"], case["d_out"], case["dtype"], case["gap"]
        s["dY"] = _rows(gen, M, do, gap, 1e-3, dt, masked=True)
        s["Z"] = _rows(gen, M, do, 0, 1.0, dt) if case["act"] != "none" else None
        s["X"] = _rows(gen, M, di, gap, 1.0, dt)
        s["W"] = _normal(gen, (do, di), 1.0 / math.sqrt(di), dt)
        s["B"] = torch.empty((M, do), dtype=_T[dt], device=dev) if case["act"] != "none" else None
        s["dX"] = torch.empty((M, di), dtype=_T[dt], device=dev)
        s["dW"] = torch.empty((do, di), dtype=_T[case["grads"]], device=dev)
        s["db"] = torch.empty((do,), dtype=_T[case["grads"]], device=dev) if case["bias"] else None
    elif op == "embedding_forward":
        s["E"] = _normal(gen, (case["vocab"], case["d"]), 0.02, case["dtype"])
        s["tokens"] = _tokens(gen, case["n"], case["vocab"], case["index"])
        s["out"] = torch.empty((case["n"], case["d"]), dtype=_T[case["dtype"]], device=dev)
    elif op == "embedding_backward":
        s["tokens"] = _tokens(gen, case["n"], case["vocab"], case["index"])
        s["dout"] = _rows(gen, case["n"], case["d"], 0, 1e-3, case["dtype"])
        s["dE"] = torch.empty((case["vocab"], case["d"]), dtype=_T[case["grads"]], device=dev)
    else:
        # the gradients live in one flat bucket, each tensor on a boundary of 64 values, zeros between
        sizes = [math.prod(x) for x in _block_shapes(case)]
        starts = np.cumsum([0] + [(n + 63) // 64 * 64 for n in sizes])
        s["flat"] = _normal(gen, (int(starts[-1]),), 1e-2, case["dtype"])
        s["clipped"] = torch.zeros_like(s["flat"])
        keep = torch.zeros_like(s["flat"])
        for a, n in zip(starts, sizes):
            keep[a:a + n] = 1
        s["flat"] *= keep
        s["views"] = [(s["flat"][a:a + n], s["clipped"][a:a + n]) for a, n in zip(starts, sizes)]
        s["norm"] = torch.empty((1,), dtype=torch.float32, device=dev)
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a user's program keeps beside its tensors: the layer's descriptor, the tensor list, a workspace."""
    import paper_2609_38767_gb300 as tda
    case, op = s["case"], s["case"]["op"]
    if op in ("linear_forward", "linear_backward"):
        act = {"none": tda.TDA_ACT_NONE, "relu": tda.TDA_ACT_RELU, "gelu": tda.TDA_ACT_GELU,
               "gelu_tanh": tda.TDA_ACT_GELU_TANH, "silu": tda.TDA_ACT_SILU}[case["act"]]
        s["L"] = tda.LinearDesc(case["d_in"], case["d_out"], act,
                                tda.TDA_BF16 if case["dtype"] == "bf16" else tda.TDA_F32)
        kind = tda.TDA_LINEAR_FORWARD if op == "linear_forward" else tda.TDA_LINEAR_BACKWARD
        s["wsb"] = tda.tda_linear_workspace_size(kind, s["L"], case["M"])
    elif op == "embedding_backward":
        s["wsb"] = tda.tda_embedding_workspace_size(case["vocab"], case["d"], case["n"])
    elif op == "clip":
        s["list"] = tda.tensor_list([a for a, _ in s["views"]], [b for _, b in s["views"]])
        s["wsb"] = tda.tda_grad_clip_workspace_size(s["list"], len(s["views"]))
    else:
        s["wsb"] = 0
    s["ws"] = torch.empty((max(s["wsb"], 1),), dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------------------------------------ the passes
def _act(name, z):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if name == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    if name == "silu":
        g = 1.0 / (1.0 + torch.exp(-z))
        return g * (1.0 + z * (1.0 - g))
    return torch.ones_like(z)


def _run_plain(s):
    case, op = s["case"], s["case"]["op"]
    if op == "linear_forward":
        dt = _T[case["dtype"]]
        z = s["X"].float() @ s["W"].float().t()
        if s["bias"] is not None:
            z = z + s["bias"].float()
        y = _act(case["act"], z)
        if s["R"] is not None:
            y = y + s["R"].float()
        return {"Y": y.to(dt), "Z": z.to(dt)} if case["keep_z"] else {"Y": y.to(dt)}
    if op == "linear_backward":
        dt, gt = _T[case["dtype"]], _T[case["grads"]]
        b = s["dY"].float()
        if case["act"] != "none":
            b = b * _act_slope(case["act"], s["Z"].float())
        out = {"dX": (b @ s["W"].float()).to(dt), "dW": (b.t() @ s["X"].float()).to(gt)}
        if case["act"] != "none":
            out["B"] = b.to(dt)
        if case["bias"]:
            out["db"] = b.sum(0).to(gt)
        return out
    if op == "embedding_forward":
        ids = s["tokens"].long()
        rows = s["E"][ids.clamp(min=0)].float() * case["scale"]
        return (rows * (ids >= 0).unsqueeze(1)).to(_T[case["dtype"]])
    if op == "embedding_backward":
        ids = s["tokens"].long()
        rows = s["dout"].float() * (ids >= 0).unsqueeze(1) * case["scale"]
        grad = torch.zeros((case["vocab"], case["d"]), dtype=torch.float32, device=rows.device)
        return grad.index_add_(0, ids.clamp(min=0), rows).to(_T[case["grads"]])
    g = s["flat"].float()
    norm = torch.sqrt((g * g).sum())
    coef = torch.clamp(case["max_norm"] / norm, max=1.0)
    return {"norm": norm.reshape(1), "clipped": (g * coef).to(_T[case["dtype"]])}


def _run_own(s):
    import paper_2609_38767_gb300 as tda
    case, op = s["case"], s["case"]["op"]
    if op == "linear_forward":
        X, W, R, Y, Z = s["X"], s["W"], s["R"], s["Y"], s["Z"]
        tda.tda_linear_forward(s["L"], X, X.stride(0), case["M"], W, W.stride(0), s["bias"], R,
                               R.stride(0) if R is not None else 0, Y, Y.stride(0), Z,
                               Z.stride(0) if Z is not None else 0, s["ws"], s["wsb"])
        return {"Y": Y, "Z": Z} if case["keep_z"] else {"Y": Y}
    if op == "linear_backward":
        dY, Z, X, W, B, dX, dW = s["dY"], s["Z"], s["X"], s["W"], s["B"], s["dX"], s["dW"]
        tda.tda_linear_backward(s["L"], dY, dY.stride(0), Z, Z.stride(0) if Z is not None else 0, case["M"], X,
                                X.stride(0), W, W.stride(0), B, B.stride(0) if B is not None else 0, dX, dX.stride(0),
                                dW, dW.stride(0), s["db"], tda.TDA_BF16 if case["grads"] == "bf16" else tda.TDA_F32,
                                0.0, s["ws"], s["wsb"])
        out = {"dX": dX, "dW": dW}
        if B is not None:
            out["B"] = B
        if s["db"] is not None:
            out["db"] = s["db"]
        return out
    dt = {"bf16": tda.TDA_BF16, "f32": tda.TDA_F32}
    if op in ("embedding_forward", "embedding_backward"):
        it = tda.TDA_I32 if case["index"] == "i32" else tda.TDA_I64
        V, d, n = case["vocab"], case["d"], case["n"]
        if op == "embedding_forward":
            tda.tda_embedding_forward(dt[case["dtype"]], s["E"], d, V, d, it, s["tokens"], n, case["scale"], s["out"], d)
            return s["out"]
        tda.tda_embedding_backward(dt[case["dtype"]], s["dout"], d, V, d, it, s["tokens"], n, case["scale"],
                                   dt[case["grads"]], s["dE"], d, 0.0, s["ws"], s["wsb"])
        return s["dE"]
    tda.tda_grad_clip(s["list"], len(s["views"]), case["max_norm"], s["norm"], s["ws"], s["wsb"])
    return {"norm": s["norm"], "clipped": s["clipped"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------ floors
def _distinct(n, vocab):
    """Expected number of different ids among n tokens of the inputs' distribution."""
    v = np.arange(vocab, dtype=np.float64)
    p = np.log((v + 2) / (v + 1)) / math.log(vocab + 1.0)
    return float(np.sum(-np.expm1(0.98 * n * np.log1p(-p))))


def work(case):
    op = case["op"]
    if op in ("linear_forward", "linear_backward"):
        M, di, do, e = case["M"], case["d_in"], case["d_out"], _BYTES[case["dtype"]]
        if op == "linear_forward":
            each = M * di + do * di + M * do * (1 + case["residual"] + case["keep_z"]) + do * case["bias"]
            return {"bytes": each * e, "flops": 2 * M * di * do}
        g = _BYTES[case["grads"]]
        each = M * do * (1 + 2 * (case["act"] != "none")) + 2 * M * di + do * di
        return {"bytes": each * e + (do * di + do * case["bias"]) * g, "flops": 4 * M * di * do}
    if op in ("embedding_forward", "embedding_backward"):
        n, V, d, e = case["n"], case["vocab"], case["d"], _BYTES[case["dtype"]]
        ids = n * (4 if case["index"] == "i32" else 8)
        if op == "embedding_forward":
            return {"bytes": ids + (_distinct(n, V) + n) * d * e, "flops": n * d}
        return {"bytes": ids + 0.98 * n * d * e + V * d * _BYTES[case["grads"]], "flops": n * d}
    total = sum(math.prod(x) for x in _block_shapes(case))
    return {"bytes": 2 * total * _BYTES[case["dtype"]] + 4, "flops": 3 * total}


# ------------------------------------------------------------------------------------------------ 64 bits
def _phi(z):
    return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))


def exact(case, seed):
    """The definitions in 64 bits on the same inputs."""
    s = prepare(case, seed)
    op, D = case["op"], torch.float64
    if op in ("linear_forward", "linear_backward"):
        a = math.sqrt(2.0 / math.pi)

        def value(z):
            return {"none": lambda: z, "relu": lambda: z.clamp(min=0), "gelu": lambda: z * _phi(z),
                    "gelu_tanh": lambda: z * torch.special.expit(2 * a * (z + 0.044715 * z ** 3)),
                    "silu": lambda: z * torch.special.expit(z)}[case["act"]]()

        if op == "linear_forward":
            z = torch.einsum("mk,nk->mn", s["X"].to(D), s["W"].to(D))
            z = z if s["bias"] is None else z + s["bias"].to(D)
            y = value(z)
            y = y if s["R"] is None else y + s["R"].to(D)
            return {"Y": y, "Z": z} if case["keep_z"] else {"Y": y}
        b = s["dY"].to(D)
        if case["act"] != "none":
            z = s["Z"].to(D).requires_grad_(True)
            (slope,) = torch.autograd.grad(value(z).sum(), z)
            b = b * slope
        out = {"dX": torch.einsum("mn,nk->mk", b, s["W"].to(D)), "dW": torch.einsum("mn,mk->nk", b, s["X"].to(D))}
        if case["act"] != "none":
            out["B"] = b
        if case["bias"]:
            out["db"] = b.sum(0)
        return out
    if op in ("embedding_forward", "embedding_backward"):
        live = (s["tokens"] >= 0).nonzero().squeeze(1)
        ids = s["tokens"][live].long()
        if op == "embedding_forward":
            out = torch.zeros((case["n"], case["d"]), dtype=D, device="cuda")
            out[live] = case["scale"] * s["E"][ids].to(D)
            return out
        grad = torch.zeros((case["vocab"], case["d"]), dtype=D, device="cuda")
        return grad.index_put_((ids,), case["scale"] * s["dout"][live].to(D), accumulate=True)
    g = s["flat"].to(D)
    norm = torch.linalg.vector_norm(g)
    return {"norm": norm.reshape(1), "clipped": g * min(1.0, case["max_norm"] / float(norm))}
