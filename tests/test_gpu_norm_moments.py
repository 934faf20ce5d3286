"""ccl_norm's statistics where a row's columns are not alike, from few rows to many.

Bounds (h = 2^-24, half an ulp of fp32): a thread adds up to 32 + H/128 squares one after the other, every addition off by h of the sum so far, ten
more join the threads; the division by H, the product and the last difference are 8 h.  That is (50 + H/128) h for the variance, half as
much for its root, whose reciprocal is good to two ulps: 4 h.
  rstd   (29 + H/256) h
  mean   (50 + H/128) h of the mean magnitude
  y      |c| rstd (rstd's bound + 4 h) + rstd (the mean's bound) with c = x - mean, then 2^-8 of the value
A mean that is off by d adds d^2 to the variance: (50 + H/128)^2 h^2 of the mean magnitude squared, which is below 2^-32 of the variance at the
magnitudes used here (mean magnitude below 4 deviations).
"""
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from ffn_reference import U, assert_within
from test_gpu_gemm_epilogue import normal

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24


def check(X, layer, eps=1e-5):
    T, H = X.shape
    X = X.cuda()
    y, rstd = torch.empty_like(X), torch.empty(T, device="cuda")
    mean = torch.empty(T, device="cuda") if layer else None
    ccl.ccl_norm(ccl.Mat(T, H, 2), X, None, None, y, kind=ccl.NORM_LAYER if layer else ccl.NORM_RMS, eps=eps, mean=mean, rstd=rstd)
    x = X.double()
    mu = x.mean(1, keepdim=True) if layer else torch.zeros_like(x[:, :1])
    rs = (((x - mu) ** 2).mean(1, keepdim=True) + eps) ** -0.5
    rel, mean_err = (29 + H / 256) * EPS, (50 + H / 128) * EPS * x.abs().mean(1, keepdim=True)
    assert_within(rstd[:, None], rs, rs * rel, "rstd")
    if layer:
        assert_within(mean[:, None], mu, mean_err, "mean")
    want = (x - mu) * rs
    err = want.abs() * (rel + 4 * EPS) + rs * mean_err * layer
    assert_within(y, want, err + U * (want.abs() + err), "y")


@pytest.mark.parametrize("shift", [3.0, 30.0])
@pytest.mark.parametrize("T,H", [(1300, 8192), (1200, 15368), (1200, 16384), (200, 8191), (1300, 2048), (9, 16384), (40, 520), (9481, 512)])
def test_leading_columns_lie_elsewhere(T, H, shift):
    X = normal(T, H, 1.0, H).float()
    X[:, :256] += shift
    check(X.bfloat16(), True)


@pytest.mark.parametrize("layer", [True, False])
@pytest.mark.parametrize("size", [1e18, 3e18, 1.2e19])
@pytest.mark.parametrize("T,H", [(1300, 8192), (1200, 16384), (9, 8191), (9500, 264), (4, 1000), (4, 40000)])
def test_squares_whose_sum_leaves_fp32(T, H, size, layer):
    # mean squares of 1e36 to 1.4e38, their sums up to 6e42
    X = torch.full((T, H), size).bfloat16()
    X[:, ::2] *= -1
    X[1:, 3::7] *= 0.5
    check(X, layer)


@pytest.mark.parametrize("T,H", [(1300, 8192), (9, 8191), (4, 8192)])
def test_one_square_alone_leaves_fp32(T, H):
    X = normal(T, H, 1.0, 5)
    X[:, 300] = 1e20                                            # its square is 1e40, the mean of squares 1e36
    check(X, False)
