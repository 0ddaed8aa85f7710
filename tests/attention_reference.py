"""Plain 64-bit forms of the scored attentions and of the cache in 8 bits, and how far a kernel may be from them.

Bounds (relative to the weighted magnitudes M = sum_j p_j |v_j| of an output, beside the rounding of the result itself, half a step of its
type): the weights p = exp(x - m) carry the absolute error of x twice (in p and in the sum).  x is a sum of d products, each partial sum
rounded to fp32 (and in cases of fp32 queries beside 8-bit rows a product short of 2^-24 of itself): (d + 4) * 2^-24 of scale * sum |q k|.
A cap adds 2^-20 of itself (one reciprocal and one exponential of 2^-22 each; of fp32 calls and caps above 512, where |x| is below a quarter of
the cap, 2^-21 of x: a power series), a bias 2^-22 of its size, exp2 2^-22, and the sum over n rows
n * 2^-24 (its partial sums).  Weights in two bf16 terms are short of 2^-15; in one, of half a step: 2^-8."""
import math

import torch

BLOCK = 32


def e4m3_scale(most: float) -> float:
    """Smallest 2^k, k >= -120, with most <= 448 * 2^k, by search."""
    k = -120
    while most > 448.0 * 2.0 ** k:
        k += 1
    return 2.0 ** k


def to_e4m3(x: torch.Tensor) -> torch.Tensor:
    """float64 -> codes: nearest-even, beyond +-448 clamped, NaN kept.  (The scaled values have 24 bits at most: torch's conversion from fp32 is exact.)"""
    return torch.where(x.isnan(), x, x.clamp(-448.0, 448.0)).float().to(torch.float8_e4m3fn)


def quantize_block(rows: torch.Tensor):
    """rows [n][d], any float type -> codes (as float64 numbers), scale."""
    x = rows.double()
    fin = x[torch.isfinite(x)].abs()
    scale = e4m3_scale(float(fin.max()) if fin.numel() else 0.0)
    return to_e4m3(x / scale).double(), scale


def append_row(codes, scale, row, inside):
    """The block's codes [n >= inside][d] (float64) and scale after `row` became its row `inside`."""
    x = row.double()
    fin = x[torch.isfinite(x)].abs()
    want = e4m3_scale(float(fin.max()) if fin.numel() else 0.0)
    new = want if inside == 0 else max(scale, want)
    codes = codes.clone()
    if inside and new != scale:
        codes[:inside] = to_e4m3(codes[:inside] * (scale / new)).double()
    codes[inside] = to_e4m3(x / new).double()
    return codes, new


def attend(q, k, v, scale, cap, slope, distance, hidden, out_dtype, weight_error):
    """One head: q [n][d], k, v [m][d], distance and hidden [n][m] (or None).  -> reference [n][d] float64, tolerance [n][d]."""
    q, k, v = q.double(), k.double(), v.double()
    d = q.shape[-1]
    x = q @ k.T * scale
    err = (d + 4) * 2.0 ** -24 * scale * (q.abs() @ k.abs().T)
    if cap > 0:
        near = x.abs() < cap / 4 if cap > 512 or out_dtype == torch.float32 else torch.zeros_like(x, dtype=torch.bool)
        err = err + torch.where(near, x.abs() * 2.0 ** -21, cap * 2.0 ** -20)
        x = cap * torch.tanh(x / cap)
    if slope is not None:
        x = x - slope * distance
        err = err + slope * distance * 2.0 ** -22
    if hidden is not None:
        x = x.masked_fill(hidden, -math.inf)
        err = err.masked_fill(hidden, 0.0)
    p = torch.softmax(x, -1)
    ref = p @ v
    # only what weighs counts: a weight's own error, weighted, and the sum's
    e = p * (err + 2.0 ** -21)
    off = e @ v.abs() + (e.sum(-1, keepdim=True) + x.shape[-1] * 2.0 ** -24 + weight_error) * (p @ v.abs())
    return ref, off * (1 + 2.0 ** -7) + ref.abs() * torch.finfo(out_dtype).eps / 2 + 1e-30


def check(got, ref, tol, what=""):
    assert got.shape == ref.shape
    fine = torch.isfinite(ref)
    g = got.double()
    assert torch.equal(fine, torch.isfinite(g)), (what, "finite values")
    assert torch.equal(ref.isnan(), g.isnan()), (what, "NaN")
    assert torch.equal(ref[~fine & ~ref.isnan()], g[~fine & ~ref.isnan()]), (what, "infinities")
    over = ((g - ref).abs() / tol)[fine]
    worst = float(over.max()) if over.numel() else 0.0
    assert worst <= 1.0, (what, worst)
    return worst
