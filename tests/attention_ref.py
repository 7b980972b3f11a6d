"""A plain 64-bit attention and the bounds that the kernels' outputs are held to.

The kernels' steps, each with its rounding: logits as 128-term fp32 sums (an error of at most
128 * 2^-24 * A, A = scale * sum |q_i k_i|; a relative error of that size in every numerator and in
the sum), numerators rounded to bf16 for the product with v (2^-8 of each term), fp32 sums over L keys
(L * 2^-24), base-2 exponentials and logarithms good to 2^-21, the output rounded to bf16 (2^-8).
With V = sum_j p_j |v_j| of the exact probabilities:
    |out - exact| <= (2^-8 + 2 * 2^-17 A + L 2^-24 + 2^-20) V + 2^-8 |exact|
    |lse - exact| <= 2^-17 A + (L + 8) 2^-24 + 2^-22 (|lse| + A + 1)
A is at least the largest logit, whose product with log2 e and back costs the last term.
"""
import math

import torch


def rows(q, k, v, positions, scale=None):
    """q [n, Hq, D], k, v [L, Hkv, D] (any type), positions [n] (the last key row i sees; a row of
    position -1 or less sees none) -> out [n, Hq, D], lse [Hq, n], and their bounds, in float64."""
    n, hq, d = q.shape
    L, hkv, _ = k.shape
    scale = 1.0 / math.sqrt(d) if not scale else scale
    out = torch.zeros((n, hq, d), dtype=torch.float64, device=q.device)
    lse = torch.full((hq, n), -math.inf, dtype=torch.float64, device=q.device)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    if n == 0 or L == 0:
        return out, lse, tol, tol_lse
    seen = torch.arange(L, device=q.device) <= positions.to(q.device)[:, None]
    for h in range(hq):
        g = h // (hq // hkv)
        qq, kk, vv = q[:, h].double(), k[:, g].double(), v[:, g].double()
        s = (qq @ kk.T) * scale
        a = ((qq.abs() @ kk.abs().T) * abs(scale)).masked_fill(~seen, 0).amax(1)
        s = s.masked_fill(~seen, -math.inf)
        l = torch.logsumexp(s, 1)
        p = torch.exp(s - l[:, None]).nan_to_num(0.0)
        vz = torch.where(seen.any(0)[:, None], vv, 0)
        out[:, h] = p @ vz
        lse[h] = l
        mass = p @ vz.abs()
        tol[:, h] = (2.0 ** -8 + 2 * 2.0 ** -17 * a[:, None] + L * 2.0 ** -24 + 2.0 ** -20) * mass \
            + 2.0 ** -8 * out[:, h].abs() + 1e-30
        tol_lse[h] = 2.0 ** -17 * a + (L + 8) * 2.0 ** -24 + 2.0 ** -22 * (l.abs() + a + 1)
    return out, lse, tol, tol_lse


def assert_close(got, want, tol, what):
    got = got.double()
    bad = ~((got - want).abs() <= tol)
    if bool(bad.any()):
        i = tuple(int(x) for x in bad.nonzero()[0])
        worst = ((got - want).abs() / tol).nan_to_num(math.inf).max()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values out of bounds, first at {i}: "
                             f"{got[i].item()} for {want[i].item()} +- {tol[i].item()}; worst ratio {worst.item()}")
