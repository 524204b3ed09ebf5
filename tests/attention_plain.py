"""Attention over a CSR pattern in 64 bits, straight from the formulas, with the bounds that the kernels' results are held to.

Bounds, element by element.  u = 2^-24 (half a step of fp32), r = 2^-8 (half a step of bfloat16; 0 for fp32 operands).  A dot product of d
terms in fp32 is off by at most (d + 2) u sum|terms|, in any order; the exponent's argument takes that, and the roundings of the
factor scale log2(e) and of the multiplication: with S_ij = scale sum_e |q_ie k_je|, the weight's relative error is at most
e_ij = 2 (d + 6) u S_ij + 8 u (|lse_i| + 8) -- exp(x) ~ 1 + 2x for the x that occur here; exp2 is good to 2 ulp; lse_i = log l + max adds its own
roundings, 4 u (|lse| + 4).  Sums over n weights add 2 (n + 8) u sum|terms| (rescaled partial sums twice).
  O:  sum_j p |v| (2 e_i + 2 (n + 8) u + r) + r |O|        (e_i = max_j e_ij, twice: weights and their sum; r: the weight's rounding, the result's)
  lse: e_i + 8 u (|lse| + 8)
  dV: sum_i p |dO| (e + 2 (n + 8) u + r) + r |dV|
  ds = p (dp - delta): |ds| e + p (d + 4) u (sum|dO v| + sum|dO O|) 2, and r |ds|; dQ, dK: scale sum of that times |k| or |q|,
  2 (n + 8) u sum|terms|, and r |result|
"""
import numpy as np
import torch

U = 2.0 ** -24


def csr(mask):
    """row_ptr, col_idx (int32) of a [M, K] truth-valued mask, columns ascending."""
    row_ptr = np.zeros(mask.shape[0] + 1, np.int32)
    row_ptr[1:] = np.cumsum(mask.sum(1))
    return torch.from_numpy(row_ptr), torch.from_numpy(np.nonzero(mask)[1].astype(np.int32))


def stacked(masks, shape):
    """row_ptr [*shape, M + 1] and col_idx [*shape, longest] of several masks, padded with zeros."""
    parts = [csr(m) for m in masks]
    longest = max(1, max(c.numel() for _, c in parts))
    col = torch.zeros((len(parts), longest), dtype=torch.int32)
    for i, (_, c) in enumerate(parts):
        col[i, :c.numel()] = c
    return torch.stack([r for r, _ in parts]).view(*shape, -1), col.view(*shape, -1)


def _half_step(dtype):
    return 0.0 if dtype == torch.float32 else torch.finfo(dtype).eps / 2


def forward(mask, q, k, v, scale):
    """mask [B, H, M, K]; q [B, H, M, d], k, v [B, Hkv, K, d].  (O, lse, bound of O, bound of lse), float64 on q's device.
    Rows of k and v that a row's mask leaves out do not enter, whatever they hold."""
    r, d = _half_step(q.dtype), q.shape[-1]
    group = q.shape[1] // k.shape[1]
    q, k, v = q.double(), k.double().repeat_interleave(group, 1), v.double().repeat_interleave(group, 1)
    k, v = torch.nan_to_num(k, 0.0, 0.0, 0.0), torch.nan_to_num(v, 0.0, 0.0, 0.0)
    q = torch.where(mask.any(3, keepdim=True), q, 0.0)
    s = (q @ k.transpose(2, 3) * scale).masked_fill(~mask, -np.inf)
    lse = torch.logsumexp(s, 3)
    some = mask.any(3)
    p = torch.where(mask, torch.exp(s - torch.where(some, lse, 0.0).unsqueeze(3)), 0.0)
    o = p @ v
    S = torch.where(mask, q.abs() @ k.abs().transpose(2, 3) * abs(scale), 0.0)
    flat = torch.where(some, lse, 0.0)
    n = mask.sum(3)
    e = 2 * (d + 6) * U * S.amax(3) + 8 * U * (flat.abs() + 8) if s.shape[3] else torch.zeros_like(flat)
    bound = (p @ v.abs()) * (2 * e + 2 * (n + 8) * U + r).unsqueeze(3) + r * o.abs() + 1e-30
    return o, lse, bound, e + 8 * U * (flat.abs() + 8)


def backward(mask, q, k, v, o, lse, do, scale):
    """(dQ, dK, dV) and their bounds, from the O and lse that are given."""
    r, d = _half_step(q.dtype), q.shape[-1]
    B, H, M, _ = q.shape
    Hkv, K = k.shape[1], k.shape[2]
    group = H // Hkv
    q, k, v, o, do = q.double(), k.double().repeat_interleave(group, 1), v.double().repeat_interleave(group, 1), o.double(), do.double()
    k, v = torch.nan_to_num(k, 0.0, 0.0, 0.0), torch.nan_to_num(v, 0.0, 0.0, 0.0)
    some = mask.any(3, keepdim=True)
    q, o, do = (torch.where(some, t, 0.0) for t in (q, o, do))
    lse = torch.where(some.squeeze(3), lse.double(), 0.0).unsqueeze(3)
    s = q @ k.transpose(2, 3) * scale
    p = torch.where(mask, torch.exp(s - lse), 0.0)
    dp, delta = do @ v.transpose(2, 3), (do * o).sum(3, keepdim=True)
    ds = p * (dp - delta)
    S = torch.where(mask, q.abs() @ k.abs().transpose(2, 3) * abs(scale), 0.0)
    e = 2 * (d + 6) * U * S + 8 * U * (lse.abs() + 8)
    T = do.abs() @ v.abs().transpose(2, 3) + (do * o).abs().sum(3, keepdim=True)
    err_p = p * (e + r)
    err_ds = ds.abs() * (e + r) + 2 * p * (d + 4) * U * T
    n, m = mask.sum(3, keepdim=True), mask.sum(2).unsqueeze(3) * group
    dq, dk, dv = ds @ k * scale, ds.transpose(2, 3) @ q * scale, p.transpose(2, 3) @ do
    bq = abs(scale) * (err_ds @ k.abs() + 2 * (n + 8) * U * (ds.abs() @ k.abs()))
    bk = abs(scale) * (err_ds.transpose(2, 3) @ q.abs() + 2 * (m + 8) * U * (ds.abs().transpose(2, 3) @ q.abs()))
    bv = err_p.transpose(2, 3) @ do.abs() + 2 * (m + 8) * U * (p.transpose(2, 3) @ do.abs())
    fold = lambda t: t.view(B, Hkv, group, K, d).sum(2)  # noqa: E731
    dk, dv, bk, bv = (fold(t) for t in (dk, dv, bk, bv))
    return (dq, dk, dv), (bq + r * dq.abs() + 1e-30, bk + r * dk.abs() + 1e-30, bv + r * dv.abs() + 1e-30)


def inside(got, want, bound):
    """Worst |got - want| / bound (infinities and NaN have to be the same)."""
    got = got.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    off = torch.where(same, 0.0, (got - want).abs() / bound)
    return float(torch.nan_to_num(off, nan=np.inf).max()) if off.numel() else 0.0
