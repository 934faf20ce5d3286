"""ccl_norm and ccl_norm_grad against their formulas in 64 bits, in every layout the map accepts, from one column to rows longer than a CTA
holds.

Bounds (u = 2^-8 for the rounding to bf16, e = 2^-23 an ulp of fp32).  A sum over a row of H values is at most n = 64 + H/512 additions deep (32
values of a thread or its share of a long row, five exchanges, at most 32 warps), so it is off by n e times the sum of magnitudes.
  mean   d = n e mean|x|
  rstd   the squares are taken about a value d from the mean at most (each warp's own mean, then joined): the variance is off by
         (n + 8) e of itself and by 4 d^2 + 2 d sigma (n + 8) e at most; its root and reciprocal by half of that and 3 e
  y      |gamma| rstd (d + 2 e |x - mean|) + |(x - mean) rstd gamma| (error of rstd + 3 e) + 2 e |y|, then u
  dx     from the statistics as given: rstd (4 e (|g| + |mean g| + |h mean(g h)|) + n e mean|g| + |h| (n + 6) e mean|g h|) + 2 e |addend|, then u
  sums   over T rows: (T + 64) e of the sum of magnitudes (a CTA's rows one after the other, its warps, the CTAs' lines), then u
"""
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from ffn_reference import E, U, assert_within
from test_gpu_gemm_epilogue import fetch, normal, place, poisoned

pytestmark = pytest.mark.gpu


def depth(H):
    return 64 + H / 512


def stats64(x, layer, eps):
    mean = x.mean(1, keepdim=True) if layer else torch.zeros_like(x[:, :1])
    var = ((x - mean) ** 2).mean(1, keepdim=True)
    return mean, var, (var + eps) ** -0.5


def check_forward(m, layer=True, weights=True, eps=1e-5, inplace=False, seed=0, shift=0, std=1.0, offset=0.0):
    T, H = m.rows, m.cols
    X = (normal(T, H, std, seed).float() + offset).to(torch.bfloat16)
    gamma, beta = normal(1, H, 0.5, seed + 1)[0], normal(1, H, 0.5, seed + 2)[0]
    x = place(X, m)
    out, n = poisoned(m)
    if inplace:
        out[:n] = x.view(torch.int16)[:n]
        x = out
    if shift:                                                   # a base that is only 2-byte aligned
        x = torch.cat([x[:shift], x])[shift:]
    kind = ccl.NORM_LAYER if layer else ccl.NORM_RMS
    mean = torch.full((T + 8,), 3.0, device="cuda") if layer else None
    rstd = torch.full((T + 8,), 3.0, device="cuda")
    ccl.ccl_norm(m, x, gamma.cuda() if weights else None, beta.cuda() if weights and layer else None, out, kind=kind, eps=eps, mean=mean, rstd=rstd)
    torch.cuda.synchronize()
    x64 = X.double().cuda()
    w = gamma.double().cuda() if weights else torch.ones(H, dtype=torch.float64, device="cuda")
    b = beta.double().cuda() if weights and layer else torch.zeros(H, dtype=torch.float64, device="cuda")
    mu, var, rs = stats64(x64, layer, eps)
    k = depth(H)
    d = k * E * x64.abs().mean(1, keepdim=True) if layer else torch.zeros_like(mu)
    var_err = (k + 8) * E * var + 4 * d * d + 2 * d * var.sqrt() * (k + 8) * E
    rs_rel = 0.5 * var_err / (var + eps) + 3 * E
    c = x64 - mu
    y = c * rs * w + b
    err = w.abs() * rs * (d + 2 * E * c.abs()) + (c * rs * w).abs() * (rs_rel + 3 * E) + 2 * E * (y.abs() + b.abs())
    assert_within(fetch(out, n, m), y, err + U * (y.abs() + err), "y")
    assert_within(rstd[:T, None], rs, rs * rs_rel, "rstd")
    assert (rstd[T:] == 3.0).all()
    if layer:
        assert_within(mean[:T, None], mu, d + E * mu.abs(), "mean")
        assert (mean[T:] == 3.0).all()


def check_grad(m, layer=True, weights=True, addend=True, inplace=None, seed=0, shift=0, dx=True, sums=True):
    T, H = m.rows, m.cols
    X, G, A = normal(T, H, 1.5, seed), normal(T, H, 1.0, seed + 1), normal(T, H, 1.0, seed + 2)
    gamma = normal(1, H, 0.5, seed + 3)[0]
    x64, g64, a64 = X.double().cuda(), G.double().cuda(), A.double().cuda()
    mu, _, rs = stats64(x64, layer, 1e-5)
    mean, rstd = mu[:, 0].float(), rs[:, 0].float()
    x, dy, ad = place(X, m), place(G, m), place(A, m) if addend else None
    out, n = poisoned(m)
    if inplace:
        src = {"x": x, "dy": dy, "addend": ad}[inplace]
        out[:n] = src.view(torch.int16)[:n]
        x, dy, ad = (out if inplace == "x" else x), (out if inplace == "dy" else dy), (out if inplace == "addend" else ad)
    if shift:
        dy = torch.cat([dy[:shift], dy])[shift:]
    dgamma = torch.full((H + 64,), 3.0, dtype=torch.bfloat16, device="cuda") if sums else None
    dbeta = torch.full((H + 64,), 3.0, dtype=torch.bfloat16, device="cuda") if sums and layer else None
    ws = torch.full((ccl.ccl_norm_grad_workspace(m) // 4,), float("nan"), device="cuda") if sums else None
    ccl.ccl_norm_grad(m, x, gamma.cuda() if weights else None, mean if layer else None, rstd, dy, out if dx else None, ws,
                      kind=ccl.NORM_LAYER if layer else ccl.NORM_RMS, addend=ad, dgamma=dgamma, dbeta=dbeta)
    torch.cuda.synchronize()
    w = gamma.double().cuda() if weights else torch.ones(H, dtype=torch.float64, device="cuda")
    rs, k = rstd.double()[:, None], depth(H)
    h = (x64 - (mean.double()[:, None] if layer else 0)) * rs
    g = g64 * w
    s1 = g.mean(1, keepdim=True) if layer else torch.zeros_like(rs)
    s2 = (g * h).mean(1, keepdim=True)
    want = rs * (g - s1 - h * s2) + (a64 if addend else 0)
    err = rs * (4 * E * (g.abs() + s1.abs() + (h * s2).abs()) + k * E * g.abs().mean(1, keepdim=True)
                + h.abs() * (k + 6) * E * (g * h).abs().mean(1, keepdim=True)) + 2 * E * (a64.abs() if addend else 0)
    if dx:
        assert_within(fetch(out, n, m), want, err + U * (want.abs() + err), "dx")
    for t, terms, what in ((dgamma, g64 * h, "dgamma"), (dbeta, g64, "dbeta")):
        if t is not None:
            s, e = terms.sum(0), (T + 64) * E * terms.abs().sum(0)
            assert_within(t[:H], s, e + U * (s.abs() + e), what)
            assert (t[H:] == 3.0).all()


SIZES = [(1, 1), (3, 8), (1, 2048), (5, 7), (40, 64), (300, 104), (33, 264), (700, 512), (64, 1024), (31, 1544), (20, 1541), (150, 4096), (9, 8192), (5, 8191),
         (4, 16384), (3, 20000), (3, 33000), (2, 40001), (1, 257), (7, 300), (9, 1026), (65, 259), (5, 16377), (3, 16379)]


@pytest.mark.parametrize("T,H", SIZES)
def test_forward_row_major(T, H):
    m = ccl.Mat(T, H, 2)
    check_forward(m)
    check_forward(m, layer=False, seed=3)
    check_forward(m, weights=False, inplace=True, seed=4)
    check_forward(m, shift=1, seed=5)


@pytest.mark.parametrize("T,H", SIZES)
def test_grad_row_major(T, H):
    m = ccl.Mat(T, H, 2)
    check_grad(m)
    check_grad(m, layer=False, addend=False, seed=3)
    check_grad(m, inplace="dy", seed=4)
    check_grad(m, layer=False, inplace="x", seed=5)
    check_grad(m, inplace="addend", weights=False, seed=6)
    check_grad(m, shift=1, seed=7)
    check_grad(m, sums=False, seed=8)
    check_grad(m, dx=False, seed=9)


@pytest.mark.parametrize("T,H", [(5000, 96), (9481, 256), (9500, 264), (5003, 512), (4999, 520), (3000, 1024), (2501, 2048), (1301, 4104), (1300, 5000), (1250, 8192), (1203, 9000), (1301, 1541), (2500, 258), (1207, 4100), (301, 8190), (500, 9001),
                                 (1200, 16384)])
def test_many_rows(T, H):
    m = ccl.Mat(T, H, 2)
    check_forward(m, seed=11)
    check_forward(m, layer=False, inplace=True, seed=12)
    check_grad(m, seed=13)
    check_grad(m, layer=False, addend=False, inplace="dy", seed=14)
    check_grad(m, inplace="addend", weights=False, seed=15)
    check_grad(m, dx=False, seed=16)


@pytest.mark.parametrize("m", [ccl.Mat(1500, 1536, 2, 4, ccl.PART_COLS, ccl.CCL, 0), ccl.Mat(1300, 4096, 2, 2, ccl.PART_COLS, ccl.CCL, 4096),
                               ccl.Mat(9600, 312, 2, 13, ccl.PART_COLS, ccl.CCL, 0), ccl.Mat(1400, 2040, 2, 9, ccl.PART_COLS, ccl.CCL, 0),
                               ccl.Mat(1300, 768, 2, 32, ccl.PART_COLS, ccl.CCL, 0), ccl.Mat(1200, 8192, 2, 4, ccl.PART_ROWS, ccl.CCL, 0)],
                         ids=lambda m: f"{m.rows}x{m.cols}-P{m.P}-part{m.part}-{m.strip_align_bytes}")
def test_many_rows_in_strips(m):
    check_forward(m, seed=21)
    check_forward(m, layer=False, inplace=True, seed=22)
    check_grad(m, seed=23)
    check_grad(m, layer=False, addend=False, seed=24)


LAYOUTS = [
    ccl.Mat(130, 1536, 2, 4, ccl.PART_COLS, ccl.CCL, 0), ccl.Mat(130, 1536, 2, 4, ccl.PART_COLS, ccl.CCL, 4096),
    ccl.Mat(33, 1001, 2, 4, ccl.PART_COLS, ccl.CCL, 64), ccl.Mat(70, 72, 2, 5, ccl.PART_COLS, ccl.CCL, 0),
    ccl.Mat(130, 200, 2, 4, ccl.PART_ROWS, ccl.CCL, 4096), ccl.Mat(131, 200, 2, 4, ccl.PART_ROWS, ccl.CCL, 0),
    ccl.Mat(64, 512, 2, 4, ccl.PART_COLS, ccl.CCL_INTERLEAVED, 1024), ccl.Mat(50, 202, 2, 3, ccl.PART_COLS, ccl.CCL_INTERLEAVED, 128),
    ccl.Mat(64, 256, 2, 4, ccl.PART_ROWS, ccl.CCL_INTERLEAVED, 48), ccl.Mat(40, 64, 2, 4, ccl.PART_NONE, ccl.CCL, 0),
    ccl.Mat(3, 40000, 2, 4, ccl.PART_COLS, ccl.CCL, 0), ccl.Mat(3, 8200, 2, 9, ccl.PART_COLS, ccl.CCL, 16),
]


@pytest.mark.parametrize("m", LAYOUTS, ids=lambda m: f"{m.rows}x{m.cols}-P{m.P}-part{m.part}-lay{m.layout}-{m.strip_align_bytes}")
def test_layouts(m):
    check_forward(m)
    check_forward(m, layer=False, inplace=True, seed=2)
    check_grad(m, seed=3)
    check_grad(m, layer=False, addend=False, inplace="dy", seed=4)


def test_padding_is_left_alone():
    m = ccl.Mat(5, 30, 2, 5, ccl.PART_COLS, ccl.CCL, 64)
    n = ccl.ccl_buffer_bytes(m) // 2
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    y = torch.full((n,), 7.0, dtype=torch.bfloat16, device="cuda")
    ccl.ccl_norm(m, x, None, None, y, kind=ccl.NORM_RMS, eps=0.0)
    assert int((y == 1.0).sum()) == 150 and int((y == 7.0).sum()) == n - 150


@pytest.mark.parametrize("T,H", [(17, 520), (17, 4096), (17, 40000), (1300, 4096), (1300, 520)])
def test_mean_far_from_zero(T, H):
    # values about 100 with a spread of 1: E x^2 - (E x)^2 in fp32 would lose half of its digits
    check_forward(ccl.Mat(T, H, 2), offset=100.0, seed=21)


@pytest.mark.parametrize("column", [0, 3, 255, 256, 4095])
@pytest.mark.parametrize("T", [17, 1300])
def test_one_column_far_out(T, column):
    # a column hundreds of deviations away from the others, as residual streams have them
    m = ccl.Mat(T, 4096, 2)
    X = normal(T, 4096, 1.0, 31)
    X[:, column] = 1500.0
    y, mean, rstd = torch.empty(T, 4096, dtype=torch.bfloat16, device="cuda"), torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    ccl.ccl_norm(m, X.cuda(), None, None, y, mean=mean, rstd=rstd)
    mu, var, rs = stats64(X.double().cuda(), True, 1e-5)
    # (the bounds above; the mean's error is of the mean magnitude, here that of the one column spread over the row)
    d = depth(4096) * E * X.double().cuda().abs().mean(1, keepdim=True)
    assert_within(mean[:, None], mu, d + E * mu.abs(), "mean")
    assert_within(rstd[:, None], rs, rs * (0.5 * ((depth(4096) + 8) * E * var + 4 * d * d + 2 * d * var.sqrt() * (depth(4096) + 8) * E) / var + 3 * E), "rstd")


def test_constant_rows_and_extremes():
    m = ccl.Mat(4, 1000, 2)
    x = torch.zeros(4, 1000, dtype=torch.bfloat16, device="cuda")
    x[1] = 5.0
    x[2] = 1e18                                                 # squares that leave fp32
    x[2, ::2] = -1e18
    x[3, 7] = float("nan")
    y, rstd = torch.empty_like(x), torch.empty(4, device="cuda")
    ccl.ccl_norm(m, x, None, None, y, rstd=rstd)
    assert (y[0] == 0).all() and (y[1] == 0).all() and torch.isnan(y[3]).all()
    assert abs(rstd[0].item() - 1e-5 ** -0.5) < 1e-3 and abs(rstd[1].item() - 1e-5 ** -0.5) < 1e-3
    want = torch.where(torch.arange(1000, device="cuda") % 2 == 0, -1.0, 1.0)
    assert torch.allclose(y[2].float(), want)                   # (1e18)^2 = 1e36: still in range, the sum over the row 1e39 is not summed as such


def test_against_differences():
    T, H, eps, step = 6, 200, 1e-5, 1e-4
    X, G = normal(T, H, 1.0, 1).double().cuda(), normal(T, H, 1.0, 2).double().cuda()
    w, b = normal(1, H, 0.5, 3)[0].double().cuda(), normal(1, H, 0.5, 4)[0].double().cuda()
    D, dw = normal(T, H, 1.0, 5).double().cuda(), normal(1, H, 1.0, 6)[0].double().cuda()
    for layer in (True, False):
        def value(x, w):
            mu, _, rs = stats64(x, layer, eps)
            return (((x - mu) * rs * w + (b if layer else 0)) * G).sum()

        mu, _, rs = stats64(X, layer, eps)
        dx = torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
        dgamma = torch.empty(H, dtype=torch.bfloat16, device="cuda")
        m = ccl.Mat(T, H, 2)
        ws = torch.empty(ccl.ccl_norm_grad_workspace(m), dtype=torch.uint8, device="cuda")
        ccl.ccl_norm_grad(m, X.bfloat16(), w.bfloat16(), mu[:, 0].float() if layer else None, rs[:, 0].float(), G.bfloat16(), dx, ws,
                          kind=ccl.NORM_LAYER if layer else ccl.NORM_RMS, dgamma=dgamma)
        along = (value(X + step * D, w) - value(X - step * D, w)) / (2 * step)
        # bf16 rounding of each gradient entry (u of it), summed; the difference's own error is of the order of step^2
        assert abs((dx.double() * D).sum() - along) <= U * (dx.double() * D).abs().sum() + 1e-4 * (1 + along.abs())
        along = (value(X, w + step * dw) - value(X, w - step * dw)) / (2 * step)
        assert abs((dgamma.double() * dw).sum() - along) <= U * (dgamma.double() * dw).abs().sum() + 1e-4 * (1 + along.abs())


def test_same_bits_on_every_run_and_in_a_graph():
    T, H = 3000, 2048
    m = ccl.Mat(T, H, 2)
    x, dy, gamma = normal(T, H, 1.0, 1).cuda(), normal(T, H, 1.0, 2).cuda(), normal(1, H, 1.0, 3)[0].cuda()
    y, mean, rstd = torch.empty_like(x), torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(gamma)
    ws = torch.empty(ccl.ccl_norm_grad_workspace(m), dtype=torch.uint8, device="cuda")

    def step():
        ccl.ccl_norm(m, x, gamma, None, y, mean=mean, rstd=rstd)
        ccl.ccl_norm_grad(m, x, gamma, mean, rstd, dy, dx, ws, dgamma=dgamma, dbeta=dbeta)

    outs = []
    for _ in range(3):
        step()
        outs.append([t.clone() for t in (y, mean, rstd, dx, dgamma, dbeta)])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for t in (y, mean, rstd, dx, dgamma, dbeta):
        t.fill_(9.0)
    for _ in range(2):
        g.replay()
    outs.append([t.clone() for t in (y, mean, rstd, dx, dgamma, dbeta)])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o in outs[1:] for a, b in zip(outs[0], o))


def test_offsets_past_32_bits():
    # 2.2e9 elements: the last rows lie behind 4 GB
    T, H = 270000, 8192
    m = ccl.Mat(T, H, 2)
    x = torch.zeros(T, H, dtype=torch.bfloat16, device="cuda")
    last = normal(64, H, 1.0, 1)
    x[-64:] = last.cuda()
    rstd, mean = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    ccl.ccl_norm(m, x, None, None, x, mean=mean, rstd=rstd)
    mu, _, rs = stats64(last.double().cuda(), True, 1e-5)
    want = (last.double().cuda() - mu) * rs
    assert_within(x[-64:], want, 2 * U * want.abs() + 1e-5, "y")
    assert (x[:1000] == 0).all()
    dy = torch.zeros_like(x)
    dy[-64:] = 1.0
    dgamma, ws = torch.empty(H, dtype=torch.bfloat16, device="cuda"), torch.empty(ccl.ccl_norm_grad_workspace(m), dtype=torch.uint8, device="cuda")
    ccl.ccl_norm_grad(m, x, None, mean.zero_(), rstd.fill_(1.0), dy, None, ws, dgamma=dgamma)
    s = x[-64:].double().sum(0)
    assert_within(dgamma, s, 2 * U * s.abs() + 128 * E * x[-64:].double().abs().sum(0), "dgamma")
