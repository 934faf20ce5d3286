"""What ccl_moe_tokens keeps of h between its two products: 16 significant bits, the value rounded to bf16 and what that rounding left.

The down projection takes differences of neighbouring features whose h agree to about seven bits, so that the part of h that one bf16
number holds nearly cancels and the rounding of Y (relative to the small difference) does not hide what is left.  A token has two entries
other than zero, so that the sums behind gate and up have two terms.

Bound (u, e as in ffn_reference.py): gate and up are fp32 sums of exact products, off by (H/8 + 64) e of the sum of magnitudes; the
activation adds 2^-20 (1 + |gate|); h's value is off by at most u |h| and its remainder, at most u |h|, is stored with an error of u of itself:
2^-16 |h|; the sums over I and the weight (1 within 4 e) add a few e of |h|; Y is rounded once."""
import pytest
import torch

from ffn_reference import E, U, act, assert_within
from test_gpu_moe_tokens import run

CASES = [(T, H, I) for T in (1, 4, 5, 8, 9, 16, 64) for H, I in ((136, 72), (512, 256))]


def problem(T, H, I, device):
    """x, router, gate, up, down and the result in 64 bits, its bound, and what Y would lose if h were rounded to bf16."""
    g = torch.Generator().manual_seed(T + H)

    def normal(*shape, s=1.0):
        return (torch.randn(*shape, generator=g) * s).to(torch.bfloat16)

    x = torch.zeros(T, H, dtype=torch.bfloat16)
    t = torch.arange(T)
    x[t, 7 * t % (H // 2)] = normal(T)
    x[t, H // 2 + 5 * t % (H // 2)] = normal(T)
    gate = normal(I // 2, H).repeat_interleave(2, 0)
    up = normal(I // 2, H).repeat_interleave(2, 0)
    up[:, H // 2:] = normal(I, H // 2, s=0.005)               # where neighbours differ
    row = torch.arange(H)
    down = torch.zeros(H, I, dtype=torch.bfloat16)
    down[row, row % (I // 2) * 2] = 1.0
    down[row, row % (I // 2) * 2 + 1] = -1.0
    router = normal(1, H, s=0.05)
    x, router, gate, up, down = (m.to(device) for m in (x, router, gate, up, down))
    x64, g64, u64, d64 = x.double(), gate.double(), up.double(), down.double()
    a, b = x64 @ g64.t(), x64 @ u64.t()
    ae, be = ((H / 8 + 64) * E * (x64.abs() @ m.abs().t()) for m in (g64, u64))
    h = act(a, "silu") * b
    he = (1.13 * ae + 2.0 ** -20 * (1 + a.abs())) * (b.abs() + be) + act(a, "silu").abs() * be
    he = he + 2.0 ** -16 * (h.abs() + he)
    want = h @ d64.t()
    err = he @ d64.abs().t() + 16 * E * ((h.abs() + he) @ d64.abs().t())
    lost = ((h.to(torch.bfloat16).double() - h) @ d64.t()).abs()
    return x, router, gate, up, down, want, err + U * (want.abs() + err), lost


@pytest.mark.parametrize("T,H,I", CASES)
def test_one_bf16_number_would_not_do(T, H, I):
    """The inputs below tell 16 bits from 8: the loss of a single rounding is above the bound for most results."""
    *_, bound, lost = problem(T, H, I, "cpu")
    assert (lost > bound).double().mean() > 0.5


@pytest.mark.gpu
@pytest.mark.parametrize("T,H,I", CASES)
def test_h_keeps_sixteen_bits(T, H, I):
    x, router, gate, up, down, want, bound, _ = problem(T, H, I, "cuda")
    y, _, _ = run(x, router, torch.cat([gate, up])[None].contiguous(), down[None], None, 1, True)
    assert_within(y, want, bound, "Y")
