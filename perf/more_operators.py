"""Timed cases of what a transformer block has beside its linear layers.

Four calls, each a pass of its own: masked attention with capped scores and distance biases, its backward pass
(with the gradient of a learned relative position bias by buckets), the root-mean-square norm with the residual's
addition, and its backward pass. ``run`` computes them either in a plain form (elementary torch operations in 32
bits) or through the package's entry points (``own``).
"""
import math

import numpy as np
import torch

own = False

_T = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}


# ------------------------------------------------------------------------------------------------ cases
def _att(op, N, T, H, KV, hd, dtype="bf16", mask="causal", window=0, cap=0.0, buckets=0, reach=0, slope=False, **more):
    """mask: "full", "causal", "docs" (causal inside packed documents), "docs_prefix" (the same, a document's first
    tokens seen by all of it) or "docs_full" (no order inside a document)."""
    return dict(op=op, N=N, T=T, H=H, KV=KV, hd=hd, dtype=dtype, mask=mask, window=window, cap=cap, buckets=buckets,
                reach=reach, slope=slope, **more)


def listed():
    return [
        # one short query example through a layer of a 2048-wide block: latency
        _att("attention", 1, 37, 32, 8, 64, name="attention_query"),
        # eight examples of 1024 tokens, heads of a 4096-wide block with shared keys
        _att("attention", 8, 1024, 32, 8, 128, name="attention_block"),
        # one long example of the same block
        _att("attention", 1, 8192, 32, 8, 128, name="attention_long"),
        # packed documents of an instruction-tuned model, prompts seen whole, capped scores and a learned bias
        _att("attention", 4, 2047, 32, 8, 64, mask="docs_prefix", cap=30.0, buckets=32, reach=128,
             name="attention_packed"),
        # a small fp32 model with biases that fall with distance, an odd length
        _att("attention", 4, 515, 8, 8, 64, dtype="f32", slope=True, name="attention_small_f32"),
        # the backward passes of the eight examples, of the packed documents, of the small model
        _att("attention_backward", 8, 1024, 32, 8, 128, name="attention_block_backward"),
        _att("attention_backward", 4, 2047, 32, 8, 64, mask="docs_prefix", cap=30.0, buckets=32, reach=128,
             name="attention_packed_backward"),
        _att("attention_backward", 2, 515, 8, 8, 64, dtype="f32", slope=True, name="attention_small_backward_f32"),
        # a query example's norm, and a large batch's, with the residual's addition
        dict(name="norm_query", op="norm", M=509, d=2048, dtype="bf16", residual=True),
        dict(name="norm_batch", op="norm", M=32768, d=4096, dtype="bf16", residual=True),
        # the backward pass of a batch, and of a ragged one of odd width in fp32
        dict(name="norm_batch_backward", op="norm_backward", M=8192, d=4096, dtype="bf16", residual=True),
        dict(name="norm_odd_backward_f32", op="norm_backward", M=1999, d=1363, dtype="f32", residual=False),
    ]


def _log_int(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v))


def _width(rng, lo, hi):
    """A row length: mostly multiples of 64, now and then any number."""
    v = _log_int(rng, lo, hi)
    return v if rng.random() < 0.2 else max(64, v // 64 * 64)


def draw(rng):
    op = rng.choice(["attention", "attention", "attention_backward", "attention_backward", "norm", "norm_backward"])
    if op in ("norm", "norm_backward"):
        return dict(op=op, M=_log_int(rng, 1, 32768), d=_width(rng, 64, 4096), dtype=rng.choice(["bf16", "bf16", "f32"]),
                    residual=rng.random() < 0.6)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    top = {"bf16": 2.7e8, "f32": 1.5e7}[dtype] * (2 if op == "attention" else 1)
    while True:
        N, T, KV, G = _log_int(rng, 1, 8), _log_int(rng, 1, 8192), rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 2, 4, 8])
        if N * T * T * KV * G <= top and KV * G <= 32:
            break
    buckets = rng.choice([0, 0, 16, 32])
    return _att(op, N, T, KV * G, KV, rng.choice([32, 64, 64, 80, 96, 128, 128] + ([36] if dtype == "f32" else [])),
                dtype=dtype, mask=rng.choice(["causal", "causal", "full", "docs", "docs_prefix", "docs_full"]),
                window=rng.choice([0, 0, 0, 100, 511]), cap=rng.choice([0.0, 0.0, 20.0, 50.0]), buckets=buckets,
                reach=rng.choice([32, 128, 300]) if buckets else 0, slope=rng.random() < 0.25)


# ------------------------------------------------------------------------------------------------ inputs
def _normal(gen, shape, sigma, dtype):
    out = torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, sigma, generator=gen)
    return out.to(_T[dtype])


def _ranged(case):
    return case["mask"].startswith("docs") or case["window"] > 0


def _documents(gen, case):
    """Ids of packed documents, about five to a row and at least 16 tokens long on average, -1 in the padding at a
    row's end (up to a tenth of it); and which tokens are prompt (about the first quarter of a document)."""
    N, T = case["N"], case["T"]
    mean = max(16.0, T / 5)
    begins = torch.rand((N, T), generator=gen, device="cuda") < 1.0 / mean
    doc = begins.long().cumsum(1)
    at = torch.arange(T, device="cuda").expand(N, T)
    first = torch.where(begins, at, torch.zeros_like(at)).cummax(1).values
    share = torch.rand((N, T), generator=gen, device="cuda") * mean / 2
    prompt = (at - first) < share.gather(1, first)
    pad = (torch.rand((N, 1), generator=gen, device="cuda") * 0.1 * T).long()
    doc = torch.where(at >= T - pad, torch.full_like(doc, -1), doc)
    return doc.to(torch.int32).contiguous(), prompt.to(torch.int32).contiguous()


def _bucket_map(case):
    """Distance i - j, held within +-reach, to its bucket: small distances one each, larger ones by their logarithm;
    half of the buckets for later keys unless the mask hides them."""
    n, reach = case["buckets"], case["reach"]
    ids = np.zeros(2 * reach + 1, dtype=np.int32)
    both = case["mask"] in ("full", "docs_full", "docs_prefix")
    side = n // 2 if both else n
    near = side // 2
    for dist in range(-reach, reach + 1):
        a = abs(dist) if both else max(dist, 0)
        b = a if a < near else min(side - 1, near + int(math.log(a / near) / math.log(reach / near) * (side - near) + 1e-9))
        ids[dist + reach] = b + (side if both and dist < 0 else 0)
    return ids


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    op, dt = case["op"], case["dtype"]
    s = dict(case=case)
    if op in ("norm", "norm_backward"):
        M, d = case["M"], case["d"]
        s["w"] = (1.0 + _normal(gen, (d,), 0.1, "f32")).to(_T[dt])
        s["eps"] = 1e-5
        s["r"] = _normal(gen, (M, d), 1.0, dt) if case["residual"] else None
        if op == "norm":
            s["x"] = _normal(gen, (M, d), 0.5, dt)
            s["h"] = torch.empty_like(s["x"]) if case["residual"] else None
            s["y"] = torch.empty_like(s["x"])
            s["rstd"] = torch.empty((M,), dtype=torch.float32, device="cuda")
        else:
            s["h"] = _normal(gen, (M, d), 1.2, dt)
            s["rstd"] = torch.rsqrt(s["h"].float().square().mean(1) + s["eps"])
            s["dy"] = _normal(gen, (M, d), 1e-2, dt)
            s["dx"] = torch.empty_like(s["h"])
            s["dw"] = torch.empty((d,), dtype=torch.float32, device="cuda")
    else:
        N, T, H, KV, hd = (case[k] for k in ("N", "T", "H", "KV", "hd"))
        s["scale"] = 1.0 / math.sqrt(hd)
        # queries, keys and values as one linear layer leaves them, side by side in a token's row
        s["qkv"] = _normal(gen, (N * T, (H + 2 * KV) * hd), 1.2, dt)
        if _ranged(case):
            s["doc"], s["prompt"] = _documents(gen, case)
            s["range"] = torch.empty((N, T, 2), dtype=torch.int32, device="cuda")
        if case["buckets"]:
            s["bucket"] = torch.from_numpy(_bucket_map(case)).cuda()
            s["table"] = _normal(gen, (case["buckets"], H), 1.0, dt)
        if case["slope"]:
            s["slope"] = torch.exp2(-8.0 * torch.arange(1, H + 1, device="cuda", dtype=torch.float32) / H)
        if op == "attention":
            s["O"] = torch.empty((N * T, H * hd), dtype=_T[dt], device="cuda")
            s["lse"] = torch.empty((N, H, T), dtype=torch.float32, device="cuda")
        else:
            # what the forward pass left, and the gradient of its output
            kept = _attention(s, torch.float32)
            s["O"], s["lse"] = kept["O"].to(_T[dt]), kept["lse"]
            s["dO"] = _normal(gen, (N * T, H * hd), 1e-2, dt)
            if _ranged(case):
                s["dO"] *= (s["doc"].reshape(-1, 1) >= 0).to(s["dO"].dtype)
            s["dqkv"] = torch.empty_like(s["qkv"])
            if case["buckets"]:
                s["dtable"] = torch.empty_like(s["table"])
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a user's program keeps beside its tensors: descriptor and workspace."""
    import paper_2609_38767_gb300 as tda
    case, op = s["case"], s["case"]["op"]
    s["kind"] = tda.TDA_BF16 if case["dtype"] == "bf16" else tda.TDA_F32
    s["wsb"] = 0
    if op == "norm_backward":
        s["wsb"] = tda.tda_rmsnorm_workspace_size(case["M"], case["d"])
    elif op != "norm":
        s["L"] = tda.AttentionDesc(case["N"], case["T"], case["H"], case["KV"], case["hd"], s["kind"], s["scale"],
                                   cap=case["cap"], causal=case["mask"] in ("causal", "docs", "docs_prefix"),
                                   n_buckets=case["buckets"], max_distance=case["reach"])
        kind = tda.TDA_ATTENTION_FORWARD if op == "attention" else tda.TDA_ATTENTION_BACKWARD
        s["wsb"] = tda.tda_attention_workspace_size(kind, s["L"])
    s["ws"] = torch.empty((max(s["wsb"], 1),), dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------------------------------------ the passes
def _ranges(s):
    """The keys [lo, hi) that each token sees: its document's, up to itself or to the end of the document's prompt
    where that is later, and less than `window` tokens away."""
    case = s["case"]
    N, T = case["N"], case["T"]
    at = torch.arange(T, device="cuda").expand(N, T)
    if case["mask"].startswith("docs"):
        doc = s["doc"].long()
        new = torch.ones_like(doc, dtype=torch.bool)
        new[:, 1:] = doc[:, 1:] != doc[:, :-1]
        first = torch.where(new, at, torch.zeros_like(at)).cummax(1).values
        last = torch.ones_like(new)
        last[:, :-1] = new[:, 1:]
        end = torch.where(last, at + 1, torch.full_like(at, T)).flip(1).cummin(1).values.flip(1)
        live = doc >= 0
    else:
        first, end, live = torch.zeros_like(at), torch.full_like(at, T), torch.ones_like(at, dtype=torch.bool)
    hi = end if case["mask"] in ("full", "docs_full") else at + 1
    if case["mask"] == "docs_prefix":
        # a document's prompt: its tokens up to the first that is not prompt
        stop = torch.where((s["prompt"] == 0) | last, at + (s["prompt"] != 0).long(), torch.full_like(at, T))
        stop = stop.flip(1).cummin(1).values.flip(1).gather(1, first)
        hi = torch.maximum(hi, stop)
    lo = first
    if case["window"]:
        lo, hi = torch.maximum(lo, at - case["window"] + 1), torch.minimum(hi, at + case["window"])
    lo, hi = torch.where(live, lo, torch.zeros_like(lo)), torch.where(live, hi, torch.zeros_like(hi))
    return torch.stack([lo, hi], 2).to(torch.int32)


def _split(s, kind):
    case = s["case"]
    N, T, H, KV, hd = (case[k] for k in ("N", "T", "H", "KV", "hd"))
    x = s["qkv"].to(kind).view(N, T, H + 2 * KV, hd).transpose(1, 2)
    return x[:, :H].reshape(N, KV, H // KV * T, hd), x[:, H:H + KV], x[:, H + KV:]


def _scores(s, q, k):
    """Scores [N][H][T][T] with -inf where a key is not seen, the slope of the cap, the ranges."""
    case = s["case"]
    N, T, H = case["N"], case["T"], case["H"]
    z = (q @ k.transpose(2, 3)).view(N, H, T, T) * s["scale"]
    bend = None
    if case["cap"]:
        t = torch.tanh(z / case["cap"])
        z, bend = case["cap"] * t, 1.0 - t * t
    at = torch.arange(T, device="cuda")
    dist = at[:, None] - at[None, :]
    if case["buckets"]:
        reach = case["reach"]
        z = z + s["table"].to(z.dtype)[s["bucket"].long()[dist.clamp(-reach, reach) + reach]].permute(2, 0, 1)
    if case["slope"]:
        z = z - s["slope"].to(z.dtype)[:, None, None] * dist.abs()
    found = None
    if _ranged(case):
        found = _ranges(s)
        seen = (at >= found[..., 0:1]) & (at < found[..., 1:2])
        z = torch.where(seen[:, None], z, torch.full_like(z[:1, :1, :1, :1], -math.inf))
    elif case["mask"] == "causal":
        z = torch.where(dist >= 0, z, torch.full_like(z[:1, :1, :1, :1], -math.inf))
    return z, bend, found


def _softmax(z):
    top = z.amax(3, keepdim=True).clamp(min=-1e30)
    p = torch.exp(z - top)
    total = p.sum(3, keepdim=True)
    return p / total.clamp(min=1e-30), (top + torch.log(total)).squeeze(3)


def _attention(s, kind):
    case = s["case"]
    N, T, H, KV, hd = (case[k] for k in ("N", "T", "H", "KV", "hd"))
    q, k, v = _split(s, kind)
    z, _, found = _scores(s, q, k)
    p, lse = _softmax(z)
    out = {"O": (p.view(N, KV, -1, T) @ v).view(N, H, T, hd).transpose(1, 2).reshape(N * T, H * hd), "lse": lse}
    return out if found is None else dict(out, range=found)


def _attention_backward(s, kind):
    case = s["case"]
    N, T, H, KV, hd = (case[k] for k in ("N", "T", "H", "KV", "hd"))
    q, k, v = _split(s, kind)
    do = s["dO"].to(kind).view(N, T, H, hd).transpose(1, 2).reshape(N, KV, -1, hd)
    z, bend, found = _scores(s, q, k)
    p = _softmax(z)[0].view(N, KV, -1, T)
    dv = p.transpose(2, 3) @ do
    dp = do @ v.transpose(2, 3)
    ds = (p * (dp - (p * dp).sum(3, keepdim=True))).view(N, H, T, T)
    out = {}
    if case["buckets"]:
        # sums along the diagonals: one more zero per row shifts each row by one
        skew = torch.nn.functional.pad(ds.sum(0).flip(2), (0, T)).view(H, -1)[:, :T * (2 * T - 1)]
        along = skew.view(H, T, 2 * T - 1).double().sum(1)  # by i - j + T - 1
        reach = case["reach"]
        ids = s["bucket"].long()[(torch.arange(2 * T - 1, device="cuda") - (T - 1)).clamp(-reach, reach) + reach]
        out["dtable"] = torch.zeros((case["buckets"], H), dtype=torch.float64, device="cuda").index_add_(0, ids, along.t())
    if bend is not None:
        ds = ds * bend
    ds = (ds * s["scale"]).view(N, KV, -1, T)
    rows = lambda x, heads: x.reshape(N, heads, T, hd).transpose(1, 2).reshape(N * T, heads * hd)  # noqa: E731
    out.update(dQ=rows(ds @ k, H), dK=rows(ds.transpose(2, 3) @ q, KV), dV=rows(dv, KV))
    return out if found is None else dict(out, range=found)


def _run_plain(s):
    case, op, dt = s["case"], s["case"]["op"], _T[s["case"]["dtype"]]
    if op == "attention":
        out = _attention(s, torch.float32)
        return dict(out, O=out["O"].to(dt))
    if op == "attention_backward":
        return {k: v if k == "range" else v.to(dt) for k, v in _attention_backward(s, torch.float32).items()}
    w = s["w"].float()
    if op == "norm":
        # the norm reads the sum as it is stored
        h = s["x"] if s["r"] is None else (s["x"].float() + s["r"].float()).to(dt)
        rstd = torch.rsqrt(h.float().square().mean(1) + s["eps"])
        out = {"y": (h.float() * rstd[:, None] * w).to(dt), "rstd": rstd}
        return out if s["r"] is None else dict(out, h=h)
    n = s["h"].float() * s["rstd"][:, None]
    g = s["dy"].float() * w
    dx = s["rstd"][:, None] * (g - n * (g * n).mean(1, keepdim=True))
    if s["r"] is not None:
        dx = dx + s["r"].float()
    return {"dx": dx.to(dt), "dw": (s["dy"].float() * n).double().sum(0).float()}


def _run_own(s):
    import paper_2609_38767_gb300 as tda
    case, op = s["case"], s["case"]["op"]
    if op == "norm":
        x, r, h, y, M, d = s["x"], s["r"], s["h"], s["y"], case["M"], case["d"]
        tda.tda_rmsnorm_forward(s["kind"], x, d, r, d, M, d, s["w"], s["eps"], h, d, y, d, s["rstd"])
        out = {"y": y, "rstd": s["rstd"]}
        return out if r is None else dict(out, h=h)
    if op == "norm_backward":
        M, d = case["M"], case["d"]
        tda.tda_rmsnorm_backward(s["kind"], s["h"], d, s["rstd"], s["w"], s["dy"], d, s["r"], d, M, d, s["dx"], d, s["dw"],
                                 tda.TDA_F32, 0.0, s["ws"], s["wsb"])
        return {"dx": s["dx"], "dw": s["dw"]}
    N, T, H, KV, hd = (case[k] for k in ("N", "T", "H", "KV", "hd"))
    out, a, b, ld = {}, H * hd, (H + KV) * hd, (H + 2 * KV) * hd
    if _ranged(case):
        docs = case["mask"].startswith("docs")
        tda.tda_attention_ranges(N, T, s["doc"] if docs else None, s["prompt"] if case["mask"] == "docs_prefix" else None,
                                 case["mask"] not in ("full", "docs_full"), case["window"], s["range"])
        out["range"] = s["range"]
    qkv, rng, bucket, table, slope = s["qkv"], s.get("range"), s.get("bucket"), s.get("table"), s.get("slope")
    q, k, v = qkv, qkv[:, a:], qkv[:, b:]
    if op == "attention":
        tda.tda_attention_forward(s["L"], q, ld, k, ld, v, ld, rng, bucket, table, slope, s["O"], a, s["lse"], s["ws"],
                                  s["wsb"])
        return dict(out, O=s["O"], lse=s["lse"])
    g = s["dqkv"]
    dq, dk, dv = g[:, :a], g[:, a:b], g[:, b:]
    tda.tda_attention_backward(s["L"], q, ld, k, ld, v, ld, rng, bucket, table, slope, s["O"], a, s["lse"], s["dO"], a, dq, ld,
                               dk, ld, dv, ld, s.get("dtable"), s["kind"], 0.0, s["ws"], s["wsb"])
    out.update(dQ=dq, dK=dk, dV=dv)
    return dict(out, dtable=s["dtable"]) if case["buckets"] else out


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------ floors
def _pairs(case):
    """Expected number of (query, key) pairs of one head over all rows, from a fixed sample of document lengths."""
    N, T, w = case["N"], case["T"], case["window"] or case["T"]
    if not case["mask"].startswith("docs"):
        i = np.arange(T)
        lo, hi = np.maximum(0, i - w + 1), i + 1 if case["mask"] == "causal" else np.minimum(T, i + w)
        return N * float(np.sum(hi - lo))
    total, rng, mean, rows = 0.0, np.random.RandomState(7), max(16.0, T / 5), 32
    i = np.arange(T)
    for _ in range(rows):
        begins = rng.rand(T) < 1.0 / mean
        first = np.maximum.accumulate(np.where(begins, i, 0))
        new = np.append(begins[1:], True)
        end = np.minimum.accumulate(np.where(new, i + 1, T)[::-1])[::-1]
        live = T - int(rng.rand() * 0.1 * T)
        end = np.minimum(end, max(live, 1))
        hi = end if case["mask"] == "docs_full" else i + 1
        if case["mask"] == "docs_prefix":
            hi = np.maximum(hi, np.minimum(end, first + np.ceil((rng.rand(T) * mean / 2)[first])))
        lo, hi = np.maximum(first, i - w + 1), np.minimum(hi, i + w)
        total += float(np.sum((hi - lo)[:live]))
    return N * total / rows


def work(case):
    op, e = case["op"], _BYTES[case["dtype"]]
    if op == "norm":
        M, d = case["M"], case["d"]
        return {"bytes": M * d * e * (4 if case["residual"] else 2) + d * e + 4 * M, "flops": 4 * M * d}
    if op == "norm_backward":
        M, d = case["M"], case["d"]
        return {"bytes": M * d * e * (4 if case["residual"] else 3) + d * (e + 4) + 4 * M, "flops": 9 * M * d}
    N, T, H, KV, hd = (case[k] for k in ("N", "T", "H", "KV", "hd"))
    pairs, small = _pairs(case) * H, (24 * N * T if _ranged(case) else 0) + 2 * case["buckets"] * H * e
    if op == "attention":
        return {"bytes": N * T * ((2 * H + 2 * KV) * hd * e + 4 * H) + small, "flops": 4 * pairs * hd}
    return {"bytes": N * T * ((4 * H + 4 * KV) * hd * e + 4 * H) + small, "flops": 10 * pairs * hd}


# ------------------------------------------------------------------------------------------------ 64 bits
def _seen(s):
    """Which keys a query sees, [N][T][T], from the documents themselves."""
    case = s["case"]
    N, T = case["N"], case["T"]
    at = torch.arange(T, device="cuda")
    seen = (at[:, None] >= at[None, :]).expand(N, T, T)
    if case["mask"] in ("full", "docs_full"):
        seen = torch.ones_like(seen)
    if case["mask"].startswith("docs"):
        doc = s["doc"].long()
        edge = torch.zeros_like(doc)
        edge[:, 1:] = (doc[:, 1:] != doc[:, :-1]).long()
        run_of = edge.cumsum(1)
        if case["mask"] == "docs_prefix":
            # prompt tokens with no other token of their document before them
            off = (s["prompt"] == 0).long().cumsum(1)
            before = off - (s["prompt"] == 0).long()  # others in the row before this token
            lead = before.gather(1, (run_of[:, :, None] > run_of[:, None, :]).sum(2).clamp(max=T - 1))
            seen = seen | ((s["prompt"] != 0) & (before == lead))[:, None, :]
        seen = seen & (run_of[:, :, None] == run_of[:, None, :]) & (doc >= 0)[:, :, None]
    if case["window"]:
        seen = seen & ((at[:, None] - at[None, :]).abs() < case["window"])
    return seen


def _range_of(seen):
    T = seen.shape[2]
    n = seen.sum(2)
    lo = torch.where(n > 0, seen.to(torch.uint8).argmax(2), torch.zeros_like(n))
    return torch.stack([lo, lo + n], 2).to(torch.int32)


def exact(case, seed):
    """The definitions in 64 bits on the same inputs."""
    s = prepare(case, seed)
    op, D = case["op"], torch.float64
    if op in ("norm", "norm_backward"):
        w = s["w"].to(D).requires_grad_(True)
        if op == "norm":
            h = s["x"].to(D) if s["r"] is None else (s["x"].to(D) + s["r"].to(D)).to(s["x"].dtype).to(D)
        else:
            h = s["h"].to(D).requires_grad_(True)
        rms = (torch.linalg.vector_norm(h, dim=1, keepdim=True) ** 2 / case["d"] + s["eps"]) ** 0.5
        y = h / rms * w
        if op == "norm":
            out = {"y": y, "rstd": (1.0 / rms).squeeze(1)}
            return out if s["r"] is None else dict(out, h=h)
        dx, dw = torch.autograd.grad(y, (h, w), s["dy"].to(D))
        return {"dx": dx if s["r"] is None else dx + s["r"].to(D), "dw": dw}
    N, T, H, KV, hd = (case[k] for k in ("N", "T", "H", "KV", "hd"))
    need = op == "attention_backward"
    parts = s["qkv"].to(D).view(N, T, H + 2 * KV, hd).split([H, KV, KV], 2)
    q, k, v = (x.contiguous().requires_grad_(need) for x in parts)
    z = torch.einsum("nikgd,njkd->nkgij", q.view(N, T, KV, H // KV, hd), k).reshape(N, H, T, T) * s["scale"]
    if case["cap"]:
        z = case["cap"] * torch.tanh(z / case["cap"])
    at = torch.arange(T, device="cuda")
    apart = at[:, None] - at[None, :]
    wanted = [q, k, v]
    if case["buckets"]:
        table = s["table"].to(D).requires_grad_(need)
        wanted.append(table)
        one = table.t()[:, s["bucket"].long()]  # [H][2 reach + 1]
        z = z + one[:, (apart.clamp(-case["reach"], case["reach"]) + case["reach"]).reshape(-1)].view(H, T, T)
    if case["slope"]:
        z = z - s["slope"].to(D).view(H, 1, 1) * apart.abs()
    seen = _seen(s)
    z = z.masked_fill(~seen[:, None], -math.inf)
    none = ~seen.any(2)[:, None, :, None]
    lse = torch.logsumexp(z.masked_fill(none, 0.0), 3, keepdim=True)
    p = torch.exp(z - lse)
    out = {}
    if _ranged(case):
        out["range"] = _range_of(seen)
    o = torch.einsum("nkgij,njkd->nikgd", p.view(N, KV, H // KV, T, T), v).reshape(N * T, H * hd)
    if not need:
        return dict(out, O=o, lse=lse.masked_fill(none, -math.inf).squeeze(3))
    got = torch.autograd.grad(o, wanted, s["dO"].to(D))
    out.update(dQ=got[0].reshape(N * T, -1), dK=got[1].reshape(N * T, -1), dV=got[2].reshape(N * T, -1))
    return dict(out, dtable=got[3]) if case["buckets"] else out
