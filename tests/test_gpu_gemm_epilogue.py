"""ccl_gemm_epilogue and ccl_gemm_act_grad against plain forms in 64 bits, for every kernel variant, layout and ragged size.
Tolerances: ffn_reference.py."""
import contextlib
import os

import numpy as np
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from helpers import gemm_desc
from ffn_reference import ACTS, E, U, act, act_bound, assert_within, product_bound, slope, slope_bound
from test_gpu_gemm import GUARD, from_layout, to_layout

pytestmark = pytest.mark.gpu


@contextlib.contextmanager
def forced(**kw):
    keys = {"CCL_GEMM_" + k.upper(): str(v) for k, v in kw.items()}
    old = {k: os.environ.get(k) for k in keys}
    os.environ.update(keys)
    try:
        yield
    finally:
        for k, v in old.items():
            if v is None:
                os.environ.pop(k, None)
            else:
                os.environ[k] = v


def normal(rows, cols, std, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, cols, generator=g) * std).to(torch.bfloat16)


def bits(t):
    return t.contiguous().view(torch.int16).numpy().view(np.uint16)


def place(t, m):
    """bf16 CPU matrix -> CUDA buffer in layout `m`"""
    return to_layout(bits(t), m)


def poisoned(m):
    n = ccl.ccl_buffer_bytes(m) // 2
    return torch.full((n + GUARD,), 0x7FC0, dtype=torch.int16, device="cuda"), n


def fetch(buf, n, m):
    assert (buf[n:] == 0x7FC0).all(), "wrote past the end"
    return torch.from_numpy(from_layout(buf[:n], m).view(np.int16).copy()).view(torch.bfloat16).cuda()


def workspace(nbytes):
    return torch.full((max(nbytes, 16) // 4,), float("nan"), dtype=torch.float32, device="cuda")


def stored(A, B, at, bt):
    return (A.t().contiguous() if at else A), (B.t().contiguous() if bt else B)


def check_forward(M, N, K, name, d, at, bt, bias=True, residual=True, preact=True, inplace=False, seed=0):
    A, B = normal(M, K, 1.0, seed), normal(K, N, 0.05, seed + 1)
    b = normal(1, N, 0.5, seed + 2)[0] if bias else None
    R = normal(M, N, 1.0, seed + 3) if residual else None
    sa, sb = stored(A, B, at, bt)
    c, n = poisoned(d.C)
    z = poisoned(d.C)[0] if preact else None
    r = None
    if residual:
        r = place(R, d.C)
        if inplace:
            c[:n] = r.view(torch.int16)[:n]
            r = c
    ccl.ccl_gemm_epilogue(d, place(sa, d.A), place(sb, d.B), c, workspace(ccl.ccl_gemm_epilogue_workspace(d)), act=getattr(ccl, "ACT_" + name.upper()),
                          bias=b.cuda() if bias else None, residual=r, preact=z)
    st, detail = ccl.ccl_gemm_status()
    assert st == ccl.OK, detail
    a64, b64 = A.double().cuda(), B.double().cuda()
    z64, z_err = a64 @ b64, product_bound(a64, b64)
    if bias:
        z64 = z64 + b.double().cuda()
        z_err = z_err + E * z64.abs()
    h, h_err = act(z64, name), act_bound(z64, z_err, name)
    want = h + R.double().cuda() if residual else h
    assert_within(fetch(c, n, d.C), want, h_err + (U + E) * (want.abs() + h_err) + 2 * E * h.abs(), "C")
    if preact:
        assert_within(fetch(z, n, d.C), z64, z_err + U * (z64.abs() + z_err), "pre-activation")


def check_grad(M, N, K, name, d, at, bt, dbias=True, inplace=False, seed=0):
    A, B, Z = normal(M, K, 1.0, seed), normal(K, N, 0.05, seed + 1), normal(M, N, 1.5, seed + 2)
    sa, sb = stored(A, B, at, bt)
    z = place(Z, d.C)
    dz, n = poisoned(d.C)
    if inplace:
        dz[:n] = z.view(torch.int16)[:n]
        z = dz
    db = torch.full((N + 64,), 3.0, dtype=torch.bfloat16, device="cuda") if dbias else None
    ccl.ccl_gemm_act_grad(d, place(sa, d.A), place(sb, d.B), z, dz, workspace(ccl.ccl_gemm_act_grad_workspace(d)), act=getattr(ccl, "ACT_" + name.upper()), dbias=db)
    st, detail = ccl.ccl_gemm_status()
    assert st == ccl.OK, detail
    a64, b64, z64 = A.double().cuda(), B.double().cuda(), Z.double().cuda()
    p, p_err = a64 @ b64, product_bound(a64, b64)
    s, s_err = slope(z64, name), slope_bound(z64, name)
    want, err = p * s, p_err * s.abs() + (p.abs() + p_err) * s_err + 2 * E * (p * s).abs()
    assert_within(fetch(dz, n, d.C), want, err + U * (want.abs() + err), "dZ")
    if dbias:
        total, t_err = want.sum(0), err.sum(0) + (M + 40) * E * want.abs().sum(0)
        assert_within(db[:N], total, t_err + U * (total.abs() + t_err), "dbias")
        assert (db[N:] == 3.0).all()


ROW = ("row", "row", "row")
CCLB = ("row", "ccl", "ccl")

# M, N, K, P, layouts, a_trans, b_trans, out_part
SHAPES = [
    (1, 8, 8, 1, ROW, 0, 0, 0),                # the smallest
    (1, 1000, 264, 1, ROW, 0, 1, 0),           # one token
    (7, 520, 1032, 1, ROW, 0, 0, 0),           # fewer rows than a swizzle group
    (130, 776, 200, 1, ROW, 0, 0, 0),          # ragged everywhere
    (333, 1000, 328, 2, CCLB, 0, 1, 2),        # two strips of 500? (500 is not a multiple of 8 -> 1008 below)
    (96, 1536, 512, 4, CCLB, 0, 0, 2),         # strips of 384
    (300, 640, 64, 2, ("ccl", "row", "ccl"), 0, 0, 1),       # an M partition: strips of rows
    (264, 512, 136, 1, ROW, 1, 0, 0),          # A stored [K x M]
    (520, 2048, 192, 4, CCLB, 0, 1, 2),
]
SHAPES[4] = (333, 1008, 328, 2, CCLB, 0, 1, 2)


@pytest.mark.parametrize("M,N,K,P,lay,at,bt,op", SHAPES)
def test_forward_and_grad_over_shapes(M, N, K, P, lay, at, bt, op):
    for i, name in enumerate(ACTS):
        for align in ((0, 4096) if "ccl" in lay else (0,)):
            d = gemm_desc(M, N, K, P, lay, at, bt, op, 1, align=align)
            check_forward(M, N, K, name, d, at, bt, bias=i != 1, residual=i != 2, preact=i != 3, seed=10 * i)
            check_grad(M, N, K, name, d, at, bt, dbias=i != 1, seed=10 * i + 5)


VARIANTS = [dict(ctas=c, bn=b, splitk=1, clusterk=0) for c, b in ((1, 128), (1, 192), (1, 256), (2, 128), (2, 192), (2, 256))] + \
           [dict(ctas=1, bn=b, splitk=s, clusterk=0) for b, s in ((128, 2), (256, 3))] + [dict(ctas=2, bn=256, splitk=4, clusterk=0)] + \
           [dict(ctas=1, bn=b, clusterk=k) for b in (128, 192, 256) for k in (2, 4, 8)]


@pytest.mark.parametrize("v", VARIANTS, ids=lambda v: "-".join(f"{k}{x}" for k, x in v.items()))
@pytest.mark.parametrize("M,N,K", [(200, 1032, 1096), (40, 264, 1600)])
def test_every_kernel_variant(v, M, N, K):
    with forced(**v):
        for lay, bt, P in ((ROW, 0, 1), (CCLB, 1, 3)):
            d = gemm_desc(M, N, K, P, lay, 0, bt, 2 if P > 1 else 0, 1)
            check_forward(M, N, K, "gelu_tanh", d, 0, bt, seed=3)
            check_forward(M, N, K, "silu", d, 0, bt, preact=False, inplace=True, seed=4)
            check_grad(M, N, K, "gelu_erf", d, 0, bt, seed=5)
            check_grad(M, N, K, "silu", d, 0, bt, inplace=True, seed=6)


def test_several_tiles_per_cta_and_a_grouped_raster():
    M, N, K, P = 1560, 4096, 136, 4
    for v in (dict(), dict(ctas=2, bn=256, splitk=1), dict(ctas=1, bn=128, splitk=1)):
        with forced(**v):
            d = gemm_desc(M, N, K, P, CCLB, 0, 0, 2, 1, align=4096)
            check_forward(M, N, K, "gelu_tanh", d, 0, 0, seed=1)
            check_grad(M, N, K, "gelu_tanh", d, 0, 0, seed=2)


# a product long enough to hide the drain is drained by eight warps, a shorter one by sixteen: both sides of the limit, whole and cut tiles
@pytest.mark.parametrize("ctas,bn", [(1, 128), (1, 192), (1, 256), (2, 128), (2, 192), (2, 256)])
@pytest.mark.parametrize("K", [1472, 1544])
def test_both_sides_of_the_drain_limit(ctas, bn, K):
    M, N = 1800, 2632                            # more tiles than the GPU takes at a time
    with forced(ctas=ctas, bn=bn, splitk=1, clusterk=0):
        d = gemm_desc(M, N, K, 1, ROW, 0, 0, 0, 0)
        check_forward(M, N, K, "gelu_tanh", d, 0, 0, seed=7)
        check_grad(M, N, K, "silu", d, 0, 0, seed=8)


# page-interleaved operands, an operand split along K, strips of unequal size, a 2-D partition
FULL = [
    dict(M=200, N=1024, K=256, P=4, lay=("row", "ileave", "ileave"), at=0, bt=0, op=2, align=4096),     # a chunk holds whole strip rows
    dict(M=72, N=8192, K=128, P=2, lay=("row", "ileave", "ileave"), at=0, bt=0, op=2, align=4096),      # a strip row spans whole chunks
    dict(M=136, N=896, K=128, P=2, lay=("row", "row", "ileave"), at=0, bt=0, op=2, align=256),          # strip rows of 3.5 chunks
    dict(M=200, N=512, K=512, P=4, lay=("ccl", "row", "row"), at=0, bt=0, op=0, align=0, parts=(2, 0, 0)),   # A split along K
    dict(M=333, N=512, K=128, P=5, lay=("ccl", "row", "ccl"), at=0, bt=0, op=1, align=0),               # strips of 67 rows, the last of 65
    dict(M=130, N=1000, K=72, P=9, lay=("row", "ccl", "ccl"), at=0, bt=0, op=2, align=0),               # strips of 112 columns, the last of 104
    dict(M=256, N=512, K=128, P=4, lay=ROW, at=0, bt=0, op=3, align=0, part_m=2),
]


@pytest.mark.parametrize("case", FULL)
def test_optional_layouts(case):
    c = dict(case)
    M, N, K, P, lay, at, bt, op = (c.pop(k) for k in ("M", "N", "K", "P", "lay", "at", "bt", "op"))
    for v in (dict(), dict(ctas=1, bn=128), dict(ctas=2, bn=256), dict(ctas=1, bn=256), dict(ctas=2, bn=128)):
        with forced(**v):
            d = gemm_desc(M, N, K, P, lay, at, bt, op, 1, **c)
            check_forward(M, N, K, "silu", d, at, bt, seed=7)
            check_grad(M, N, K, "gelu_tanh", d, at, bt, seed=8)


def test_plain_epilogue_gives_ccl_gemm_bits():
    for M, N, K in ((16, 1536, 2048), (300, 1032, 512)):
        A, B = normal(M, K, 1.0, 1), normal(K, N, 0.02, 2)
        d = gemm_desc(M, N, K)
        with forced(ctas=1, bn=128, splitk=1, clusterk=0):
            c1, n = poisoned(d.C)
            c2, _ = poisoned(d.C)
            ccl.ccl_gemm(d, A.cuda(), B.cuda(), c1)
            ccl.ccl_gemm_epilogue(d, A.cuda(), B.cuda(), c2)
        assert torch.equal(c1, c2)


def test_extreme_values_follow_the_formulas():
    """Infinities, NaN and magnitudes whose square overflows fp32, as a pre-activation."""
    M, N, K = 8, 64, 8
    vals = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1.0, -1.0, 30.0, -30.0, 300.0, -300.0, 1e20, -1e20, 3e38, -3e38, float("inf"), float("nan")])
    Z = vals.to(torch.bfloat16).repeat(M, N // 16)
    d = gemm_desc(M, N, K)
    A = torch.ones(M, K, dtype=torch.bfloat16)
    B = torch.zeros(K, N, dtype=torch.bfloat16)
    B[0] = 1.0
    for name in ACTS:
        dz, n = poisoned(d.C)
        ccl.ccl_gemm_act_grad(d, A.cuda(), B.cuda(), place(Z, d.C), dz, workspace(ccl.ccl_gemm_act_grad_workspace(d)), act=getattr(ccl, "ACT_" + name.upper()))
        got, z = fetch(dz, n, d.C).double(), Z.double().cuda()
        big = z.abs() >= 30
        want = torch.where(big & (z > 0), torch.ones_like(z), torch.where(big, torch.zeros_like(z), slope(z, name))) if name != "none" else torch.ones_like(z)
        cols = [i for i in range(N) if i % 16 < 14]                          # the finite ones
        assert_within(got[:, cols], want[:, cols], U * want[:, cols].abs() + 2.0 ** -18, name)
        if name not in ("none", "relu"):
            assert torch.isnan(got[:, 15]).all()                             # NaN stays
        # forward: the pre-activation comes in as a residual-free bias row
        c, n = poisoned(d.C)
        ccl.ccl_gemm_epilogue(d, A.cuda(), torch.zeros_like(B).cuda(), c, act=getattr(ccl, "ACT_" + name.upper()), bias=Z[0].cuda())
        got = fetch(c, n, d.C).double()
        want = torch.where(big & (z > 0), z, torch.where(big, torch.zeros_like(z), act(z, name))) if name != "none" else z
        assert_within(got[:, cols], want[:, cols], U * want[:, cols].abs() + 2.0 ** -18 * (1 + want[:, cols].abs().clamp(max=1.0)), name)
        assert torch.isnan(got[:, 15]).all() and (got[:, 14] == float("inf")).all()


def test_gradient_against_differences():
    """dbias and dZ against central differences of the 64-bit forward pass, along the bias and along single pre-activations."""
    M, N, K = 24, 72, 40
    for name in ("gelu_tanh", "gelu_erf", "silu"):
        d = gemm_desc(M, N, K)
        A, B, Z = normal(M, K, 1.0, 1), normal(K, N, 0.2, 2), normal(M, N, 1.0, 3)
        dz, n = poisoned(d.C)
        db = torch.empty(N, dtype=torch.bfloat16, device="cuda")
        ccl.ccl_gemm_act_grad(d, A.cuda(), B.cuda(), place(Z, d.C), dz, workspace(ccl.ccl_gemm_act_grad_workspace(d)), act=getattr(ccl, "ACT_" + name.upper()), dbias=db)
        up, z, h = A.double() @ B.double(), Z.double(), 1e-5
        diff = (up * act(z + h, name) - up * act(z - h, name)) / (2 * h)    # d/dz of sum(up * act(z))
        # central differences: h^2/6 of the third derivative (< 3) and 2^-52 of the value over h
        err = (product_bound(A.double(), B.double()) + up.abs() * (slope_bound(z, name) + 1e-10)) * 1.2
        assert_within(fetch(dz, n, d.C).cpu(), diff, err + U * (diff.abs() + err), name)
        t, te = diff.sum(0), err.sum(0) + (M + 40) * E * diff.abs().sum(0)
        assert_within(db.cpu(), t, te + U * (t.abs() + te), name + " dbias")


def test_the_same_bits_on_every_run_and_from_a_graph():
    M, N, K = 300, 1032, 1096
    A, B, Z = normal(M, K, 1.0, 1).cuda(), normal(K, N, 0.05, 2).cuda(), normal(M, N, 1.0, 3).cuda()
    bias = normal(1, N, 0.5, 4)[0].cuda()
    for v in (dict(ctas=1, bn=128, splitk=3, clusterk=0), dict(ctas=2, bn=256, splitk=1, clusterk=0), dict(ctas=1, bn=192, clusterk=4)):
        with forced(**v):
            d = gemm_desc(M, N, K)
            ws = workspace(max(ccl.ccl_gemm_act_grad_workspace(d), ccl.ccl_gemm_epilogue_workspace(d)))
            outs = [torch.empty(M * N, dtype=torch.bfloat16, device="cuda") for _ in range(3)] + [torch.empty(N, dtype=torch.bfloat16, device="cuda")]

            def step():
                ccl.ccl_gemm_epilogue(d, A, B, outs[0], ws, act=ccl.ACT_SILU, bias=bias, residual=Z, preact=outs[1])
                ccl.ccl_gemm_act_grad(d, A, B, outs[1], outs[2], ws, act=ccl.ACT_SILU, dbias=outs[3])

            step()
            torch.cuda.synchronize()
            first = [o.clone() for o in outs]
            side = torch.cuda.Stream()
            with torch.cuda.stream(side):
                step()
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(first, outs))
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
            for o in outs:
                o.fill_(float("nan"))
            ws.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(first, outs))
            assert ccl.ccl_gemm_status()[0] == ccl.OK
