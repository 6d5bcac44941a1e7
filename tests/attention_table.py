"""Bounds of a position bias's gradient that see a missing or doubled diagonal in long examples.

dtable is a sum of dS over rows. Where O was stored in few bits, dO . O of row i is off by

    sum_d dO_id rho_id O_id + sum_j eta_ij P_ij dP_ij,   |rho| <= u, |eta| <= up,

rho from storing O and eta from rounding P for the product with V, all of them roundings to the nearest of unrelated numbers:
independent, with mean zero. It enters dS of all of the row's pairs, so a bucket's sum with the row's weight in it, w_i = the sum of
P_ij over the bucket's pairs. By Hoeffding's inequality such a sum exceeds 8 sqrt(the sum of the squares of its terms' bounds) with a
chance below 2 exp(-32). The rows' errors from scores and lse (p_off) are taken at their worst within a row and so between rows; what
has a sign of its own, the tensor pipe's truncated sums, is added up as it is."""
import torch


def by_row(x, bucket, reach, n_buckets):
    """Sums of [N][H][T][T] over each row's pairs of each bucket: [N][H][T][n_buckets]."""
    T = x.shape[3]
    at = torch.arange(T, device=x.device)
    ids = bucket.to(x.device).long()[(at[:, None] - at[None, :]).clamp(-reach, reach) + reach]
    ids = torch.where((ids >= 0) & (ids < n_buckets), ids, n_buckets)
    out = torch.zeros((*x.shape[:3], n_buckets + 1), dtype=x.dtype, device=x.device)
    return out.scatter_add_(3, ids.expand(x.shape), x)[..., :n_buckets]


def table_bound(f, b, r, bucket, reach, n_buckets, grad_u, summed=False):
    """f: attention()'s values, b: their Bounds, r: gradients()' values; grad_u: the rounding of dtable; summed: every row's dO . O
    is the sum of P dP in fp32."""
    T, P, d = f["p"].shape[3], f["p"], f["q"].shape[3]
    e = b.e
    p_off = 2 * e + 2 * (P * e).sum(3, keepdim=True) + 2.0 ** -20
    many = f["seen"].sum(3, keepdim=True) > 1
    dp_mag = r["do"].abs() @ f["v"].abs().transpose(2, 3)
    weight = by_row(many * P, bucket, reach, n_buckets)
    rows = by_row(many * P * (p_off * (r["dp"] - r["delta"]).abs() + (P * p_off * r["dp"].abs()).sum(3, keepdim=True)), bucket, reach,
                  n_buckets)
    spread = rows.square()
    if not summed:
        stored = (b.u * r["do"] * f["o"]).square().sum(3, keepdim=True) + (b.up * P * r["dp"]).square().sum(3, keepdim=True)
        spread = spread + weight.square() * stored * 1.02  # the stored O's own errors, to first order
    # sums of products, of P dP over a row, and of dS along the diagonals: fp32, 2^-24 a step
    straight = many * P * (2 * b.g * (dp_mag + (r["do"].abs() * f["o"].abs()).sum(3, keepdim=True))
                           + 2.0 ** -22 * (r["dp"].abs() + r["delta"].abs())) + 2.0 ** -24 * (T / 128 + 300) * r["ds"].abs()
    if summed:
        straight = straight + many * P * (2.0 ** -24 * (T + d) * (P * r["dp"].abs()).sum(3, keepdim=True))
    straight = by_row(straight, bucket, reach, n_buckets).sum((0, 2)).t()
    return 8 * spread.sum((0, 2)).sqrt().t() + straight + grad_u * r["dtable"].abs() + 1e-30
