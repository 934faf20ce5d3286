"""ccl_bias_act_grad against the formula in 64 bits, in every layout the map accepts and at sizes no vector divides.
Tolerances: ffn_reference.py."""
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from ffn_reference import ACTS, E, U, assert_within, slope, slope_bound
from test_gpu_gemm_epilogue import fetch, normal, place, poisoned

pytestmark = pytest.mark.gpu


def check(m, name, want_dz=True, want_db=True, inplace=None, seed=0, shift=0):
    M, N = m.rows, m.cols
    G, Z = normal(M, N, 1.0, seed), normal(M, N, 1.5, seed + 1)
    dy, z = place(G, m), place(Z, m)
    dz, n = poisoned(m)
    if inplace == "dy":
        dz[:n] = dy.view(torch.int16)[:n]
        dy = dz
    if inplace == "z":
        dz[:n] = z.view(torch.int16)[:n]
        z = dz
    if shift:                                                   # bases that are only 2-byte aligned
        dy = torch.cat([dy[:shift], dy])[shift:]
    db = torch.full((N + 64,), 3.0, dtype=torch.bfloat16, device="cuda") if want_db else None
    ccl.ccl_bias_act_grad(m, dy, z if name != "none" else None, dz if want_dz else None, db, act=getattr(ccl, "ACT_" + name.upper()))
    torch.cuda.synchronize()
    g64, z64 = G.double().cuda(), Z.double().cuda()
    want, err = g64 * slope(z64, name), g64.abs() * slope_bound(z64, name) + 2 * E * (g64 * slope(z64, name)).abs()
    if want_dz:
        assert_within(fetch(dz, n, m), want, err + U * (want.abs() + err), "dZ")
    if want_db:
        t, te = want.sum(0), err.sum(0) + (M + 8) * E * want.abs().sum(0)
        assert_within(db[:N], t, te + U * (t.abs() + te), "dbias")
        assert (db[N:] == 3.0).all()


SIZES = [(1, 1), (1, 8), (3, 7), (31, 24), (257, 40), (100, 2056), (1531, 264), (513, 1001), (64, 16384), (5000, 16)]


@pytest.mark.parametrize("M,N", SIZES)
def test_row_major(M, N):
    for i, name in enumerate(ACTS):
        check(ccl.Mat(M, N, 2), name, seed=i)
    check(ccl.Mat(M, N, 2), "silu", want_dz=False)
    check(ccl.Mat(M, N, 2), "silu", want_db=False)
    check(ccl.Mat(M, N, 2), "none", want_dz=False)
    check(ccl.Mat(M, N, 2), "gelu_tanh", inplace="dy")
    check(ccl.Mat(M, N, 2), "gelu_tanh", inplace="z")
    check(ccl.Mat(M, N, 2), "gelu_erf", shift=1)


LAYOUTS = [
    ccl.Mat(130, 1536, 2, 4, ccl.PART_COLS, ccl.CCL, 0), ccl.Mat(130, 1536, 2, 4, ccl.PART_COLS, ccl.CCL, 4096),
    ccl.Mat(33, 1001, 2, 4, ccl.PART_COLS, ccl.CCL, 64), ccl.Mat(70, 72, 2, 5, ccl.PART_COLS, ccl.CCL, 0),
    ccl.Mat(130, 200, 2, 4, ccl.PART_ROWS, ccl.CCL, 4096), ccl.Mat(131, 200, 2, 4, ccl.PART_ROWS, ccl.CCL, 0),
    ccl.Mat(64, 512, 2, 4, ccl.PART_COLS, ccl.CCL_INTERLEAVED, 1024), ccl.Mat(50, 202, 2, 3, ccl.PART_COLS, ccl.CCL_INTERLEAVED, 128),
    ccl.Mat(64, 256, 2, 4, ccl.PART_ROWS, ccl.CCL_INTERLEAVED, 48), ccl.Mat(40, 64, 2, 4, ccl.PART_NONE, ccl.CCL, 0),
]


@pytest.mark.parametrize("m", LAYOUTS, ids=lambda m: f"{m.rows}x{m.cols}-P{m.P}-part{m.part}-lay{m.layout}-{m.strip_align_bytes}")
def test_layouts(m):
    for i, name in enumerate(ACTS):
        check(m, name, seed=i)


def test_padding_is_left_alone():
    m = ccl.Mat(5, 30, 2, 5, ccl.PART_COLS, ccl.CCL, 64)
    n = ccl.ccl_buffer_bytes(m) // 2
    dy = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    dz = torch.full((n,), 7.0, dtype=torch.bfloat16, device="cuda")
    ccl.ccl_bias_act_grad(m, dy, None, dz)
    assert int((dz == 1.0).sum()) == 150 and int((dz == 7.0).sum()) == n - 150


def test_same_bits_on_every_run():
    dy, z = normal(3000, 520, 1.0, 1).cuda(), normal(3000, 520, 1.0, 2).cuda()
    m = ccl.Mat(3000, 520, 2)
    outs = []
    for _ in range(5):
        db = torch.empty(520, dtype=torch.bfloat16, device="cuda")
        ccl.ccl_bias_act_grad(m, dy, z, None, db, act=ccl.ACT_GELU_TANH)
        outs.append(db)
    assert all(torch.equal(outs[0], o) for o in outs)
