"""Plain 64-bit forms of the feed-forward operators and the error bounds their tests use.

Bounds, derived from the arithmetic (u = 2^-8: half an ulp of bf16 (8 significant bits) at a power of two, relative; e = 2^-23: an ulp of fp32):
  product   the tensor cores add 16 exact products at a time to an fp32 accumulator: at most K/16 + 16 additions (K splits included),
            each off by at most 2 e of what has been added up so far, which is at most S = |A| |B|:  (K/8 + 32) e S
  logistic  exponential and reciprocal in hardware, a few ulps: 2^-20 relative; every activation is z times something in [0, 1] plus terms
            bounded by |z|: 2^-20 (1 + |z|); slopes of the activations are below 1.13, so an error of z passes on with at most that
  slope     gelu's has z s (1 - s) dt/dz with dt/dz <= 1.6 (1 + 0.134 z^2), 1 - s off by e: 2^-20 (1 + |z|)^3, with z cut to 12
  rounding  u |result| once per output
"""
import math

import torch

U, E = 2.0 ** -8, 2.0 ** -23
ACTS = ("none", "relu", "gelu_tanh", "gelu_erf", "silu")


def act(z, name):
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "gelu_erf":
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def slope(z, name):
    if name == "relu":
        return torch.where(z <= 0, torch.zeros_like(z), torch.ones_like(z))
    if name == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    if name == "gelu_erf":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def product_bound(a, b):
    """a [M x K], b [K x N] in 64 bits -> bound of the fp32 product's error."""
    return (a.shape[1] / 8 + 32) * E * (a.abs() @ b.abs())


def act_bound(z, z_err, name):
    return z_err if name in ("none", "relu") else 1.13 * z_err + 2.0 ** -20 * (1 + z.abs())


def slope_bound(z, name):
    if name in ("none", "relu"):
        return torch.zeros_like(z)
    return 2.0 ** -20 * (1 + z.abs().clamp(max=12.0)) ** 3


def assert_within(got, want, bound, what):
    """|got - want| <= bound, element by element (non-finite values have to be the same ones)."""
    got, want = got.double(), want.double()
    fin = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    assert torch.equal(got[~fin & ~torch.isnan(want)], want[~fin & ~torch.isnan(want)]), f"{what}: infinities differ"
    off = (got - want).abs()[fin]
    bound = bound.expand_as(want)[fin]
    assert torch.all(off <= bound), f"{what}: off by {off.max().item():.3e} (worst ratio to the bound {(off / bound.clamp(min=1e-300)).max().item():.2f})"
