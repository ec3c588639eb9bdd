"""Attention of given rows over the keys that each of them sees, in 64 bits, with a bound on what the kernels may be off by.

With u = 2^-24, z the logits, A = scale max_n sum_c |q_c k_nc| and S = sum_n p_n |v_n|:
  a logit is off by dz = (d + 4) u A (products and sums of d terms in fp32, the scale's rounding);
  a weight by 2 dz + u (4 |z|_max + n + 96) relative to itself: its own logit's error and the denominator's, the exponent's
  product, difference and exponential twice (log2 e times 2 u |z| each way is below 4), the n additions of the denominator and,
  of the product with V, as many again: n more; the merges of token groups and splits, at most 64 + 8 factors and additions;
  fp32: |out| is off by S times that, and by u |out| for the division
  bf16: the weights are rounded (u_b = 2^-8 each) and their denominator with them (u_b): 2 u_b S more, and u_b |out| for the output
  lse: dz + u (4 |z|_max + n + 96), and for bf16 u_b for the denominator of rounded weights
"""
import math

import torch

U, UB = 2.0 ** -24, 2.0 ** -8


def attend(q, k, v, sees, scale=None):
    """q [r, d], k and v [n, d], sees [r, n] -> out [r, d], its bound, lse [r], its bound; a row that sees nothing: zeros, -inf.
    What k and v hold where no row sees it is not looked at."""
    bf16 = q.dtype == torch.bfloat16
    q, k, v = q.double(), k.double(), v.double()
    d, n = q.shape[1], k.shape[0]
    scale = scale or 1.0 / math.sqrt(d)
    used = sees.any(0)
    k, v = torch.where(used[:, None], k, 0.0), torch.where(used[:, None], v, 0.0)
    if n == 0:
        z, a = q.new_full((q.shape[0], 0), 0.0), q.new_zeros((q.shape[0], 1))
        empty = torch.ones(q.shape[0], dtype=torch.bool, device=q.device)
        return torch.zeros_like(q), torch.zeros_like(q), q.new_full((q.shape[0],), -math.inf), q.new_zeros(q.shape[0])
    z = ((q @ k.T.contiguous()) * scale).masked_fill(~sees, -math.inf)
    a = scale * ((q.abs() @ k.abs().T.contiguous()) * sees).amax(1, keepdim=True)
    top = z.amax(1, keepdim=True)
    empty = top[:, 0] == -math.inf
    e = torch.exp(z - top.clamp(min=-1e300))
    total = e.sum(1, keepdim=True)
    p = e / torch.where(total > 0, total, 1.0)
    out, mass = p @ v, p @ v.abs()
    zmax = torch.where(sees & (z > -math.inf), z.abs(), 0.0).amax(1, keepdim=True)
    rel = 2 * (d + 4) * U * a + U * (4 * zmax + 2 * n + 96)
    bound = mass * rel + U * out.abs() + 1e-37
    lse = torch.where(empty, -math.inf, (top + torch.log(total))[:, 0])
    lse_bound = ((d + 4) * U * a + U * (8 * zmax + n + 96))[:, 0] + U * torch.where(empty, 0.0, lse).abs()
    if bf16:
        bound = bound + 2 * UB * mass + UB * (out.abs() + bound)
        lse_bound = lse_bound + UB
    return out, bound, lse, lse_bound


def check(got, out, bound, what=""):
    got = got.double()
    assert torch.isfinite(got).all(), "%s: non-finite" % what
    off = (got - out).abs()
    bad = off > bound
    assert not bad.any(), "%s: %d of %d outside; worst %.3g times the bound" % (what, int(bad.sum()), bad.numel(), float((off / bound).max()))


def check_lse(got, lse, bound, what=""):
    got = got.double()
    empty = lse == -math.inf
    assert torch.equal(got == -math.inf, empty), what
    off = (got - lse)[~empty].abs()
    assert (off <= bound[~empty]).all(), "%s: lse off by %.3g times its bound" % (what, float((off / bound[~empty]).max()))
