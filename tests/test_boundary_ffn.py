"""C-ABI boundary of the feed-forward operators on the CPU: descriptors, workspace sizes and refusals before any launch.  No GPU."""
import ctypes as C

import pytest

from paper_2606_11718_b200 import binding as ccl
from paper_2606_11718_b200 import build as ccl_build
from helpers import gemm_desc
from test_boundary import expect

P1, P2, P3, P4, P5, P6 = (C.c_void_p(i << 12) for i in range(1, 7))
NULL = None


@pytest.fixture(scope="module", autouse=True)
def built():
    ccl_build.build()


def status(code, rc):
    assert rc == code, (rc, ccl.lib().ccl_last_error())
    assert ccl.lib().ccl_last_error() != b""


def test_struct_sizes_match_c_layout():
    assert C.sizeof(ccl.Epilogue) == 8 + 3 * 8
    assert C.sizeof(ccl.MoeDesc) == 3 * 8 + 4 * 4 + 2 * 8


def epilogue(d, e=None, A=P1, B=P2, Cc=P3, ws=NULL, n=0):
    e = e if e is not None else ccl.Epilogue(0, None, None, None)
    return ccl.lib().ccl_gemm_epilogue(C.byref(d) if d else None, C.byref(e), A, B, Cc, ws, n, None)


def test_epilogue_refusals():
    d = gemm_desc(256, 512, 64)
    assert ccl.ccl_gemm_epilogue_workspace(d) >= 0
    status(ccl.ERR_INVALID_ARG, ccl.lib().ccl_gemm_epilogue(C.byref(d), None, P1, P2, P3, None, 0, None))
    status(ccl.ERR_INVALID_ARG, epilogue(None))
    status(ccl.ERR_INVALID_ARG, epilogue(d, A=NULL))
    status(ccl.ERR_INVALID_ARG, epilogue(d, Cc=NULL))
    status(ccl.ERR_INVALID_ARG, epilogue(d, ccl.Epilogue(5, None, None, None)))
    status(ccl.ERR_INVALID_ARG, epilogue(d, ccl.Epilogue(-1, None, None, None)))
    status(ccl.ERR_INVALID_ARG, epilogue(d, ccl.Epilogue(0, None, None, P3.value)))          # the pre-activation in C
    status(ccl.ERR_INVALID_ARG, epilogue(d, ccl.Epilogue(0, None, P4.value, P4.value)))      # ... in the residual
    for bad in (ccl.Epilogue(0, 4104, None, None), ccl.Epilogue(0, None, 4104, None), ccl.Epilogue(0, None, None, 4104)):
        status(ccl.ERR_ALIGN, epilogue(d, bad))
    status(ccl.ERR_ALIGN, epilogue(d, A=C.c_void_p(4104)))
    status(ccl.ERR_UNSUPPORTED, epilogue(gemm_desc(256, 500, 64)))
    bad = gemm_desc(256, 512, 64)
    bad.A = ccl.Mat(256, 72, 2)
    status(ccl.ERR_SHAPE, epilogue(bad))
    expect(ccl.ERR_SHAPE, ccl.ccl_gemm_epilogue_workspace, bad)
    status(ccl.ERR_INVALID_ARG, ccl.lib().ccl_gemm_epilogue_workspace(C.byref(d), None))


def test_act_grad_refusals():
    l, d = ccl.lib(), gemm_desc(256, 512, 64)
    need = ccl.ccl_gemm_act_grad_workspace(d)
    assert need >= 256 // 32 * 512 * 4                                       # a line of partial sums per 32 rows

    def call(act=ccl.ACT_SILU, A=P1, B=P2, Z=P3, dZ=P4, db=P5, ws=P6, n=1 << 30):
        return l.ccl_gemm_act_grad(C.byref(d), act, A, B, Z, dZ, db, ws, n, None)

    status(ccl.ERR_INVALID_ARG, call(act=9))
    status(ccl.ERR_INVALID_ARG, call(Z=NULL))
    status(ccl.ERR_INVALID_ARG, call(dZ=NULL))
    status(ccl.ERR_WORKSPACE, call(ws=NULL))
    status(ccl.ERR_WORKSPACE, call(n=need - 1))
    status(ccl.ERR_ALIGN, call(ws=C.c_void_p(4100)))
    status(ccl.ERR_ALIGN, call(Z=C.c_void_p(4098)))
    status(ccl.ERR_ALIGN, call(db=C.c_void_p(4097)))
    status(ccl.ERR_INVALID_ARG, l.ccl_gemm_act_grad_workspace(None, C.byref(C.c_size_t())))


def test_bias_act_grad_refusals():
    l, m = ccl.lib(), ccl.Mat(16, 24, 2)

    def call(m=m, act=ccl.ACT_SILU, dy=P1, z=P2, dz=P3, db=P4):
        return l.ccl_bias_act_grad(C.byref(m) if m else None, act, dy, z, dz, db, None)

    status(ccl.ERR_INVALID_ARG, call(m=None))
    status(ccl.ERR_INVALID_ARG, call(act=5))
    status(ccl.ERR_INVALID_ARG, call(dy=NULL))
    status(ccl.ERR_INVALID_ARG, call(z=NULL))
    status(ccl.ERR_INVALID_ARG, call(dz=NULL, db=NULL))
    status(ccl.ERR_ALIGN, call(dz=C.c_void_p(4097)))
    status(ccl.ERR_UNSUPPORTED, call(m=ccl.Mat(16, 24, 4)))
    status(ccl.ERR_SHAPE, call(m=ccl.Mat(4, 9, 2, 4, ccl.PART_COLS, ccl.CCL)))


def test_moe_refusals():
    l = ccl.lib()

    def call(ws=P6, n=1 << 40, X=P1, Y=P5, ids=None, res=None, **kw):
        d = ccl.MoeDesc(**{**dict(T=4, E=16, topk=2, H=64, I=32), **kw})
        return l.ccl_moe_tokens(C.byref(d), X, P2, P3, P4, res, Y, ids, None, ws, n, None)

    for kw in (dict(T=0), dict(H=0), dict(I=-8), dict(E=0), dict(topk=0), dict(gu_strips=0), dict(gu_stride_bytes=64), dict(d_stride_bytes=-16)):
        status(ccl.ERR_INVALID_ARG, call(**kw))
    status(ccl.ERR_SHAPE, call(topk=17))
    status(ccl.ERR_SHAPE, call(gu_strips=3))
    for kw in (dict(T=65), dict(E=513), dict(E=64, topk=17), dict(H=8200), dict(I=32776), dict(H=60), dict(I=36)):
        status(ccl.ERR_UNSUPPORTED, call(**kw))
    status(ccl.ERR_ALIGN, call(gu_stride_bytes=4 * 64 * 32 + 8))
    status(ccl.ERR_ALIGN, call(X=C.c_void_p(4104)))
    status(ccl.ERR_ALIGN, call(ids=C.c_void_p(4098)))
    status(ccl.ERR_INVALID_ARG, call(X=NULL))
    status(ccl.ERR_INVALID_ARG, call(Y=NULL))
    need = ccl.ccl_moe_tokens_workspace(ccl.MoeDesc(4, 16, 2, 64, 32))
    status(ccl.ERR_WORKSPACE, call(n=need - 1))
    status(ccl.ERR_WORKSPACE, call(ws=NULL))
    status(ccl.ERR_INVALID_ARG, l.ccl_moe_tokens(None, P1, P2, P3, P4, None, P5, None, None, P6, 1 << 30, None))


def test_moe_plans_fit_shared_memory_over_the_whole_range():
    for T in (1, 8, 9, 33, 64):
        for E in (1, 8, 60, 512):
            for topk in (1, 4, 16):
                for H in (8, 520, 2048, 4104, 8192):
                    for I in (8, 768, 32768):
                        if topk <= E:
                            assert ccl.ccl_moe_tokens_workspace(ccl.MoeDesc(T, E, topk, H, I)) > 0
