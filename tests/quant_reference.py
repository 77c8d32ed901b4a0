"""Plain 64-bit forms of the 4-bit cache's operators, for the tests: the format from its definition, and
attention over the values that codes and scales stand for."""

import math

import numpy as np
import torch

GROUP = 32


def quantise(x):
    """Packed codes uint8 [..., d / 2] and bf16 scales [..., d / 32] of rows x [..., d] (CPU tensor)."""
    x = x.float().numpy()
    y = x.reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    amax = np.abs(y).max(-1)                                  # (a NaN stays one)
    with np.errstate(all="ignore"):
        scale = torch.from_numpy((amax / np.float32(7)).astype(np.float32)).bfloat16()
        s = scale.float().numpy()[..., None]
        code = np.clip(np.rint((y / s).astype(np.float32)), -7, 7)
    good = np.isfinite(amax)[..., None] & (s > 0)
    code = np.where(good, code, 0).astype(np.int64).reshape(x.shape) + 8
    packed = (code[..., 0::2] | (code[..., 1::2] << 4)).astype(np.uint8)
    scale = torch.where(torch.from_numpy(np.isfinite(amax)), scale, torch.full_like(scale, math.nan))
    return torch.from_numpy(packed), scale


def values(codes, scales):
    """The fp64 values of packed codes and scales (CPU tensors)."""
    c = codes.to(torch.int64)
    n = torch.stack([c & 15, c >> 4], -1).flatten(-2).double() - 8
    return n * scales.double().repeat_interleave(GROUP, -1)


def attend(q, k, v, visible):
    """q [r, d], k and v [n, d], visible bool [r, n]: o, lse and sum p |v| / sum p, fp64."""
    x = q.double() @ k.T / math.sqrt(q.shape[-1])
    x = x.masked_fill(~visible, -math.inf)
    m = x.amax(1, keepdim=True)
    p = torch.exp(x - m)
    v = torch.where(visible.any(0)[:, None], v, torch.zeros_like(v))   # rows nobody sees may hold anything
    l = p.sum(1, keepdim=True)
    return (p @ v) / l, (m + torch.log(l)).squeeze(1), (p @ v.abs()) / l


def check(o, lse, want_o, want_lse, spread, v_max, what=""):
    """o (bf16) and lse (fp32) of a call against the 64-bit ones; spread: sum p |v| / sum p, v_max: max |v|.

    An output is rounded to bf16 once: half a unit in its last of 8 places, 2^-8 of it at most.  The weights
    are rounded to 11 bits (2^-11 each at most) and their exponents carry the scores' fp32 error (about 2^-22
    of sum |q k| / sqrt(d), some 2^-13 of a weight at the scores these tests have): together within 2^-10 of
    sum p |v|.  fp16 has no weights below 2^-30 of the largest (2^-24, lifted by 2^6), so where
    every heavier row holds zeros an output may miss 2^-31 of the largest |v|.
    The normaliser is a sum of fp32 weights with a relative error of 2^-22 each, and n 2^-24 from adding
    them up, and a log."""
    o, lse = o.double().cpu(), lse.double().cpu()
    tol = 2.0 ** -8 * want_o.abs() + 2.0 ** -10 * spread + 2.0 ** -31 * v_max + 1e-37
    assert torch.isfinite(o).all(), f"{what}: not finite"
    worst = ((o - want_o).abs() / tol).max().item()
    assert worst <= 1, f"{what}: {worst:.2f} times the tolerance"
    tol = 5e-5 + 1e-5 * want_lse.abs()
    worst = ((lse - want_lse).abs() / tol).max().item()
    assert worst <= 1, f"{what}: lse {worst:.2f} times the tolerance"
