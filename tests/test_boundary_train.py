"""C-ABI boundary of the normalisation and of the AdamW step on the CPU: descriptors, workspace sizes and refusals before any launch.  No GPU."""
import ctypes as C

import pytest
import torch

from paper_2606_11718_b200 import binding as ccl
from paper_2606_11718_b200 import build as ccl_build
from test_boundary import expect
from test_boundary_ffn import NULL, P1, P2, P3, P4, P5, P6, status

P7, P8, P9 = (C.c_void_p(i << 12) for i in range(7, 10))


@pytest.fixture(scope="module", autouse=True)
def built():
    ccl_build.build()


def test_struct_sizes_match_c_layout():
    assert C.sizeof(ccl.AdamwTensor) == 9 * 8
    assert C.sizeof(ccl.AdamwDesc) == 5 * 8 + 8 + 8 + 3 * 8


def test_norm_refusals():
    l, m = ccl.lib(), ccl.Mat(16, 24, 2)

    def call(m=m, kind=0, eps=1e-5, x=P1, g=P2, b=P3, y=P4, mean=P5, rstd=P6):
        return l.ccl_norm(C.byref(m) if m else None, kind, eps, x, g, b, y, mean, rstd, None)

    status(ccl.ERR_INVALID_ARG, call(m=None))
    status(ccl.ERR_INVALID_ARG, call(kind=2))
    status(ccl.ERR_INVALID_ARG, call(x=NULL))
    status(ccl.ERR_INVALID_ARG, call(y=NULL))
    for eps in (-1e-9, float("nan"), float("inf")):
        status(ccl.ERR_INVALID_ARG, call(eps=eps))
    status(ccl.ERR_INVALID_ARG, call(kind=1, mean=NULL))                                 # beta
    status(ccl.ERR_INVALID_ARG, call(kind=1, b=NULL))                                    # means
    status(ccl.ERR_UNSUPPORTED, call(m=ccl.Mat(16, 24, 4)))
    status(ccl.ERR_UNSUPPORTED, call(m=ccl.Mat(1, 1 << 31, 2)))
    status(ccl.ERR_SHAPE, call(m=ccl.Mat(4, 9, 2, 4, ccl.PART_COLS, ccl.CCL)))
    status(ccl.ERR_ALIGN, call(x=C.c_void_p(4097)))
    status(ccl.ERR_ALIGN, call(g=C.c_void_p(4097)))
    status(ccl.ERR_ALIGN, call(rstd=C.c_void_p(4098)))


def test_norm_grad_refusals():
    l, m = ccl.lib(), ccl.Mat(8192, 2048, 2)
    need = ccl.ccl_norm_grad_workspace(m)
    assert need >= 2 * 2048 * 4

    def call(m=m, kind=0, x=P1, g=P2, mean=P3, rstd=P4, dy=P5, add=P6, dx=P7, dg=P8, db=P9, ws=P1, n=1 << 30):
        return l.ccl_norm_grad(C.byref(m) if m else None, kind, x, g, mean, rstd, dy, add, dx, dg, db, ws, n, None)

    status(ccl.ERR_INVALID_ARG, call(m=None))
    status(ccl.ERR_INVALID_ARG, call(kind=-1))
    for k in ("x", "dy", "rstd", "mean"):
        status(ccl.ERR_INVALID_ARG, call(**{k: NULL}))
    status(ccl.ERR_INVALID_ARG, call(kind=1))                                            # dbeta
    status(ccl.ERR_INVALID_ARG, call(dx=NULL, dg=NULL, db=NULL))
    status(ccl.ERR_INVALID_ARG, call(dx=P2))                                             # in gamma
    status(ccl.ERR_WORKSPACE, call(ws=NULL))
    status(ccl.ERR_WORKSPACE, call(n=need - 1))
    status(ccl.ERR_ALIGN, call(ws=C.c_void_p(4104)))
    status(ccl.ERR_ALIGN, call(dg=C.c_void_p(4097)))
    status(ccl.ERR_ALIGN, call(mean=C.c_void_p(4098)))
    status(ccl.ERR_UNSUPPORTED, call(m=ccl.Mat(16, 24, 1)))
    status(ccl.ERR_INVALID_ARG, l.ccl_norm_grad_workspace(C.byref(m), None))
    expect(ccl.ERR_UNSUPPORTED, ccl.ccl_norm_grad_workspace, ccl.Mat(16, 24, 4))


def test_norm_grad_workspace_is_bounded():
    # a line of two sums a column for every CTA, one an SM (eight where rows start at eight places of a 16-byte piece), or none
    for rows in (1, 300, 1 << 20):
        for cols in (1, 8, 520, 8192, 8191, 100000):
            assert ccl.ccl_norm_grad_workspace(ccl.Mat(rows, cols, 2)) <= min(max(rows, 8), 148) * 8 * (cols + 14)


def test_adamw_refusals():
    l = ccl.lib()
    base = dict(n=100, param=P1, param_bf16=P2, grad=P3, m=P4, v=P5, m_scale=P6, v_scale=P7, grad_fp32=0)

    def call(tensors=1, bits=32, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, wd=0.1, step=1, gs=None, lr_dev=None, step_dev=None, desc=True, **kw):
        d = ccl.AdamwDesc(lr, b1, b2, eps, wd, step)
        d.state_bits, d.grad_scale_dev, d.lr_dev, d.step_dev = bits, gs, lr_dev, step_dev
        t = ccl.AdamwTensor(**{k: (v.value if isinstance(v, C.c_void_p) else v) for k, v in {**base, **kw}.items()})
        return l.ccl_adamw(C.byref(d) if desc else None, C.byref(t) if tensors else None, 1 if tensors >= 0 else -1, None)

    status(ccl.ERR_INVALID_ARG, call(desc=False))
    status(ccl.ERR_INVALID_ARG, call(tensors=0))
    status(ccl.ERR_INVALID_ARG, call(tensors=-1))
    status(ccl.ERR_UNSUPPORTED, call(bits=16))
    for kw in (dict(lr=-1.0), dict(lr=float("nan")), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(eps=0.0), dict(eps=1e-60), dict(wd=-1.0), dict(wd=float("inf")),
               dict(step=0), dict(step=-5), dict(lr_dev=4096)):
        status(ccl.ERR_INVALID_ARG, call(**kw))
    for kw in (dict(n=-1), dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(bits=8, m_scale=None), dict(bits=8, v_scale=None)):
        status(ccl.ERR_INVALID_ARG, call(**kw))
    status(ccl.ERR_UNSUPPORTED, call(n=(1 << 40) + 1))
    for kw in (dict(param=4098), dict(m=4098), dict(grad=4098, grad_fp32=1), dict(grad=4097), dict(param_bf16=4097), dict(bits=8, v_scale=4098), dict(gs=4098),
               dict(step_dev=4100)):
        status(ccl.ERR_ALIGN, call(**kw))
    assert call(n=0, param=None) == ccl.OK                                               # nothing to do: nothing is launched
    assert l.ccl_adamw(C.byref(ccl.AdamwDesc()), None, 0, None) == ccl.OK


def test_adamw_tensor_list_refusals(monkeypatch):
    monkeypatch.setattr(ccl, "_current_device", lambda: -1)                                # CPU tensors say -1: the other checks then run here
    f, h = lambda n: torch.zeros(n), lambda n: torch.zeros(n, dtype=torch.bfloat16)       # noqa: E731
    q = lambda n: torch.zeros(n, dtype=torch.float8_e4m3fn)                               # noqa: E731

    def make(p=None, g=None, m=None, v=None, **kw):
        return ccl.AdamwTensors(p or [f(300)], g or [h(300)], m or [f(300)], v or [f(300)], **kw)

    assert make().count == 1 and make().bits == 32
    assert make(m=[q(300)], v=[q(300)], m_scales=[f(2)], v_scales=[f(2)]).bits == 8
    assert ccl.AdamwTensors([], [], [], []).count == 0
    bad = [dict(p=[h(300)]), dict(g=[f(299)]), dict(m=[q(300)]), dict(v=[f(300), f(300)]), dict(copies=[f(300)]), dict(copies=[]), dict(m_scales=[f(2)], v_scales=[f(2)]),
           dict(m=[q(300)], v=[q(300)], m_scales=[f(1)], v_scales=[f(2)]), dict(m=[q(300)], v=[q(300)], m_scales=[f(2)]), dict(g=[None]),
           dict(p=[torch.zeros(20, 30).t()], g=[h(600)], m=[f(600)], v=[f(600)])]
    for kw in bad:
        with pytest.raises(ValueError):
            make(**kw)
    x = f(600)
    with pytest.raises(ValueError, match="overlap"):
        make(p=[x[:300]], m=[x[299:599]])
    with pytest.raises(ValueError, match="overlap"):
        ccl.AdamwTensors([x[:300], x[:300]], [h(300)] * 2, [f(300), f(300)], [f(300), f(300)])
    monkeypatch.undo()
    with pytest.raises(ValueError):
        make()                                                                           # not on a GPU


def test_xent_refusals():
    l = ccl.lib()

    def desc(T=16, V=100, H=64, W=None, trans=1):
        return ccl.XentDesc(T, V, H, W if W is not None else (ccl.Mat(V, H, 2) if trans else ccl.Mat(H, V, 2)), trans)

    def fwd(d, X=P1, W=P2, t=P3, loss=P4, lse=P5, ws=P6, n=1 << 40):
        return l.ccl_linear_xent(C.byref(d) if d else None, X, W, t, loss, lse, ws, n, None)

    def grad(d, X=P1, W=P2, t=P3, lse=P4, dl=P5, dx=P6, dw=P7, ws=P8, n=1 << 40):
        return l.ccl_linear_xent_grad(C.byref(d) if d else None, X, W, t, lse, dl, dx, dw, ws, n, None)

    strips = ccl.Mat(64, 96, 2, 4, ccl.PART_COLS, ccl.CCL)
    for call, size in ((fwd, ccl.ccl_linear_xent_workspace), (grad, ccl.ccl_linear_xent_grad_workspace)):
        status(ccl.ERR_INVALID_ARG, call(None))
        for kw in (dict(T=0), dict(V=0), dict(H=-8)):
            status(ccl.ERR_INVALID_ARG, call(desc(**kw, W=ccl.Mat(100, 64, 2))))
        status(ccl.ERR_SHAPE, call(desc(W=ccl.Mat(101, 64, 2))))
        status(ccl.ERR_SHAPE, call(desc(W=ccl.Mat(64, 100, 2))))
        for d in (desc(H=60), desc(T=1 << 31), desc(W=ccl.Mat(100, 64, 4)), desc(W=ccl.Mat(100, 64, 2, 4, ccl.PART_ROWS, ccl.CCL)), desc(V=100, trans=0),
                  desc(V=96, W=ccl.Mat(64, 96, 2, 8, ccl.PART_COLS, ccl.CCL), trans=0), desc(V=96, W=ccl.Mat(64, 96, 2, 4, ccl.PART_COLS, ccl.CCL_INTERLEAVED, 48), trans=0),
                  desc(V=96, W=ccl.Mat(64, 96, 2, 4, ccl.PART_ROWS, ccl.CCL), trans=0), desc(V=100, W=ccl.Mat(64, 100, 2, 3, ccl.PART_COLS, ccl.CCL), trans=0),
                  desc(V=96, W=ccl.Mat(64, 96, 2, 4, ccl.PART_COLS, ccl.CCL, 3082), trans=0)):
            status(ccl.ERR_UNSUPPORTED, call(d))
        for k in ("X", "W", "t"):
            status(ccl.ERR_INVALID_ARG, call(desc(), **{k: NULL}))
        for k, v in (("X", 4104), ("W", 4104), ("t", 4098), ("lse", 4098), ("ws", 4104)):
            status(ccl.ERR_ALIGN, call(desc(), **{k: C.c_void_p(v)}))
        for d in (desc(), desc(V=96, W=strips, trans=0)):
            need = size(d)
            assert need > 0
            status(ccl.ERR_WORKSPACE, call(d, n=need - 1))
            status(ccl.ERR_WORKSPACE, call(d, ws=NULL))
        expect(ccl.ERR_UNSUPPORTED, size, desc(H=60))
    status(ccl.ERR_INVALID_ARG, fwd(desc(), loss=NULL, lse=NULL))
    status(ccl.ERR_ALIGN, fwd(desc(), loss=C.c_void_p(4098)))
    status(ccl.ERR_INVALID_ARG, grad(desc(), lse=NULL))
    status(ccl.ERR_INVALID_ARG, grad(desc(), dl=NULL))
    status(ccl.ERR_INVALID_ARG, grad(desc(), dx=NULL, dw=NULL))
    status(ccl.ERR_INVALID_ARG, grad(desc(), dx=P1))
    status(ccl.ERR_INVALID_ARG, grad(desc(), dw=P2))
    status(ccl.ERR_ALIGN, grad(desc(), dw=C.c_void_p(4104)))
    assert C.sizeof(ccl.XentDesc) == 3 * 8 + C.sizeof(ccl.Mat) + 8


def test_xent_workspace_is_bounded():
    # the gradient's piece is 512 MB at most, or 256 columns, and dX's fp32 sums come beside it
    for T in (1, 100, 8192, 1 << 20):
        for V in (1, 1000, 131072, 131071):
            for H in (64, 4096):
                d = ccl.XentDesc(T, V, H)
                assert ccl.ccl_linear_xent_workspace(d) <= T * (V // 128 + 2) * 8 * 4 + T * 4 + 512
                assert ccl.ccl_linear_xent_grad_workspace(d) <= max(1 << 29, T * 512) + 16 * T * H * 4 * 2 + 16 * 64 * max(T, V) * H + 4096


@pytest.mark.parametrize("rows", [16, 8192])
def test_norm_grad_refuses_gradients_in_each_others_place(rows):
    l, m = ccl.lib(), ccl.Mat(rows, 2048, 2)

    def call(dx=P7, dg=P8, db=P9):
        return l.ccl_norm_grad(C.byref(m), 0, P1, P2, P3, P4, P5, P6, dx, dg, db, P1, 1 << 30, None)

    for bad in (dict(dg=P2), dict(db=P2), dict(dg=P9), dict(dx=P8), dict(dx=P9), dict(dx=P2)):
        status(ccl.ERR_INVALID_ARG, call(**bad))
