"""Masked attention and its gradients from the definition in 64 bits, with error bounds of a kernel that computes
them in its own precision. What a rounding costs: at most half a step, 2^-8 of a bf16 value, 2^-24 of an fp32 one."""
import math

import torch

D = torch.float64


def seen_by(rng, T, N, causal, device):
    at = torch.arange(T, device=device)
    if rng is None:
        return ((at[:, None] >= at[None, :]) if causal else torch.ones(T, T, dtype=torch.bool, device=device)).expand(N, T, T)
    r = rng.to(device).long()
    return (at >= r[..., :1].clamp(min=0)) & (at < r[..., 1:].clamp(max=T))


def attention(q, k, v, seen, scale, cap=0.0, bias=None):
    """q [N][H][T][d], k and v [N][KV][T][d], bias [H][T][T] or None. Returns a dict of the intermediate values."""
    G = q.shape[1] // k.shape[1]
    q, k, v = q.to(D), k.to(D).repeat_interleave(G, 1), v.to(D).repeat_interleave(G, 1)
    live = seen.any(2)
    q = torch.where(live[:, None, :, None], q, 0.0)  # what nothing reads may be anything
    used = seen.any(1)
    k, v = torch.where(used[:, None, :, None], k, 0.0), torch.where(used[:, None, :, None], v, 0.0)
    x = scale * q @ k.transpose(2, 3)
    mag = scale * q.abs() @ k.abs().transpose(2, 3)
    bend = torch.ones_like(x)
    c = x
    if cap:
        t = torch.tanh(x / cap)
        c, bend = cap * t, 1 - t * t
    s = c if bias is None else c + bias.to(D)
    s = torch.where(seen[:, None], s, -math.inf)
    lse = torch.logsumexp(s, 3)
    none = lse == -math.inf
    p = torch.where(seen[:, None], torch.exp(s - torch.where(none, 0.0, lse)[..., None]), 0.0)
    return dict(q=q, k=k, v=v, x=x, mag=mag, bend=bend, s=s, lse=lse, p=p, o=p @ v, seen=seen[:, None], live=live)


def gradients(f, do, scale, KV, bucket=None, reach=0, n_buckets=0):
    """dQ, dK, dV, dtable and the intermediate values."""
    do = torch.where(f["live"][:, None, :, None], do.to(D), 0.0)
    p, v = f["p"], f["v"]
    dp = do @ v.transpose(2, 3)
    delta = (do * f["o"]).sum(3, keepdim=True)
    ds = p * (dp - delta) * (f["seen"].sum(3, keepdim=True) > 1)
    dx = scale * ds * f["bend"]
    N, H, T, d = do.shape
    shared = lambda g: g.view(N, KV, H // KV, T, d).sum(2)  # noqa: E731
    out = dict(dQ=dx @ f["k"], dK=shared(dx.transpose(2, 3) @ f["q"]), dV=shared(p.transpose(2, 3) @ do), ds=ds, dx=dx, dp=dp,
               delta=delta, do=do)
    if n_buckets:
        out["dtable"] = by_bucket(ds, bucket, reach, n_buckets)
    return out


def by_bucket(x, bucket, reach, n_buckets):
    """Sums of [N][H][T][T] over the pairs of each bucket: [n_buckets][H]."""
    T = x.shape[3]
    at = torch.arange(T, device=x.device)
    ids = bucket.to(x.device).long()[(at[:, None] - at[None, :]).clamp(-reach, reach) + reach].reshape(-1)
    ok = (ids >= 0) & (ids < n_buckets)
    out = torch.zeros((n_buckets, x.shape[1]), dtype=x.dtype, device=x.device)
    return out.index_add_(0, ids[ok], x.sum(0).flatten(1).t()[ok])


def bias_of(T, H, bucket, reach, table, slope, device):
    at = torch.arange(T, device=device)
    apart = at[:, None] - at[None, :]
    b = torch.zeros((H, T, T), dtype=D, device=device)
    if table is not None:
        ids = bucket.to(device).long()[apart.clamp(-reach, reach) + reach]
        ok = (ids >= 0) & (ids < table.shape[0])
        b += torch.where(ok[..., None], table.to(D)[ids.clamp(0, table.shape[0] - 1)], 0.0).permute(2, 0, 1)
    if slope is not None:
        b -= slope.to(D)[:, None, None] * apart.abs()
    return b


class Bounds:
    """u: the rounding of outputs, and of P and dX before a product with bf16 operands (0 for fp32: part of g then).
    g: relative error of an fp32 sum of products. The tensor pipe truncates its sums every 16 products by at most 2^-22
    of sum |products|: 2^-22 (T + d) / 16 in all. fp32 sums on the CUDA cores: 2^-24 per addition.
    A score's error: that of its sum, two roundings more, and 2^-21 (exp2's argument and the functions) of its size, of
    the cap's and of the bias's."""

    def __init__(self, f, dtype, T, d, cap, bias):
        bf = dtype == torch.bfloat16
        self.u = 2.0 ** -8 if bf else 2.0 ** -24
        self.up = 2.0 ** -8 if bf else 0.0
        self.g = 2.0 ** -22 * ((T + d) / 16 + 8) if bf else 2.0 ** -24 * (T + d + 16)
        size = f["x"].abs() + cap + (0 if bias is None else bias.abs()) + torch.where(f["lse"] > -math.inf, f["lse"].abs(), 0.0)[..., None]
        self.e = f["mag"] * (2.0 ** -22 * (d / 16 + 4) if bf else 2.0 ** -24 * (d + 4)) + 2.0 ** -21 * (size + 4)
        self.e = torch.where(f["seen"], self.e, 0.0)
        self.f = f

    def lse(self):
        f = self.f
        return (f["p"] * self.e).sum(3) + 2.0 ** -22 * (f["lse"].abs().nan_to_num(posinf=0.0) + 4) + self.g

    def o(self):
        f = self.f
        off = f["p"] * (2 * self.e + 2 * (f["p"] * self.e).sum(3, keepdim=True) + self.up + 2 * self.g)
        return off @ f["v"].abs() + self.u * f["o"].abs() + 1e-37

    def grads(self, r, scale, KV, bucket=None, reach=0, n_buckets=0, grad_u=None, summed=False):
        """summed: dO . O is the sum of P dP in fp32, not taken from the stored O."""
        f = self.f
        N, H, T, d = r["do"].shape
        dp_mag = r["do"].abs() @ f["v"].abs().transpose(2, 3)
        delta_off = (r["do"].abs() * (self.o() + self.g * f["o"].abs())).sum(3, keepdim=True)
        p_off = 2 * self.e + 2 * (f["p"] * self.e).sum(3, keepdim=True) + 2.0 ** -20
        if summed:
            delta_off = (f["p"] * (p_off * r["dp"].abs() + self.g * dp_mag + 2.0 ** -24 * T * r["dp"].abs())).sum(3, keepdim=True)
        many = f["seen"].sum(3, keepdim=True) > 1
        ds_off = many * f["p"] * (p_off * (r["dp"] - r["delta"]).abs() + self.g * dp_mag + delta_off
                                  + 2.0 ** -22 * (r["dp"].abs() + r["delta"].abs()))
        # the slope of the cap, 1 - t^2, is off by 2 |t| times t's error
        dx_off = scale * (ds_off * f["bend"] + r["ds"].abs() * 2.0 ** -19) + (self.up + 2.0 ** -22) * r["dx"].abs()
        shared = lambda g: g.view(N, KV, H // KV, T, d).sum(2)  # noqa: E731
        g2 = self.g * H / KV
        out = dict(
            dQ=dx_off @ f["k"].abs() + self.g * (r["dx"].abs() @ f["k"].abs()) + self.u * r["dQ"].abs() + 1e-37,
            dK=shared((dx_off + g2 * r["dx"].abs()).transpose(2, 3) @ f["q"].abs()) + self.u * r["dK"].abs() + 1e-37,
            dV=shared((f["p"] * (p_off + self.up + g2)).transpose(2, 3) @ r["do"].abs()) + self.u * r["dV"].abs() + 1e-37)
        if n_buckets:
            out["dtable"] = (by_bucket(ds_off + 2.0 ** -24 * (T + 64) * r["ds"].abs(), bucket, reach, n_buckets)
                             + (grad_u if grad_u is not None else self.u) * r["dtable"].abs() + 1e-37)
        return out
