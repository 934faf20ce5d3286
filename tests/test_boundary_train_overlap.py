"""Outputs and workspaces that lie over other buffers of the same call are refused before any launch.  No GPU."""
import ctypes as C

import pytest

from paper_2606_11718_b200 import binding as ccl
from paper_2606_11718_b200 import build as ccl_build
from test_boundary_ffn import status

INVALID = ccl.ERR_INVALID_ARG


@pytest.fixture(scope="module", autouse=True)
def built():
    ccl_build.build()


def places(*names):
    """An address for every name, far from all others."""
    return {k: (i + 1) << 40 for i, k in enumerate(names)}


def p(v):
    return C.c_void_p(v)


def overlaps(call, at, sizes, outputs, inputs, allowed=()):
    """Each output over each other buffer: at the same place, its last bytes over the other's first ones, the other's last bytes over its first (16-byte
    aligned places all of them)."""
    for o in outputs:
        for b in (*outputs, *inputs):
            if b == o:
                continue
            for shift in (0, (sizes[b] - 1) // 16 * 16, -((sizes[o] - 1) // 16 * 16)):
                if shift == 0 and (o, b) in allowed:
                    continue
                status(INVALID, call(**{**at, o: at[b] + shift}))


@pytest.mark.parametrize("trans", [1, 0])
@pytest.mark.parametrize("T", [16, 400])
def test_xent(T, trans):
    V, H = 960, 64
    w = ccl.Mat(V, H, 2) if trans else ccl.Mat(H, V, 2, 4, ccl.PART_COLS, ccl.CCL)
    d, l = ccl.XentDesc(T, V, H, w, w_trans=trans), ccl.lib()
    at = places("X", "W", "targets", "loss", "lse", "ws")
    need = ccl.ccl_linear_xent_workspace(d)
    sizes = dict(X=2 * T * H, W=2 * V * H, targets=4 * T, loss=4 * T, lse=4 * T, ws=need)

    def forward(X, W, targets, loss, lse, ws):
        return l.ccl_linear_xent(C.byref(d), p(X), p(W), p(targets), p(loss), p(lse), p(ws), need, None)

    overlaps(forward, at, sizes, ("loss", "lse", "ws"), ("X", "W", "targets"))
    at = places("X", "W", "targets", "lse", "dloss", "dX", "dW", "ws")
    grad_need = ccl.ccl_linear_xent_grad_workspace(d)
    sizes = dict(X=2 * T * H, W=2 * V * H, targets=4 * T, lse=4 * T, dloss=4 * T, dX=2 * T * H, dW=2 * V * H, ws=grad_need)

    def grad(X, W, targets, lse, dloss, dX, dW, ws):
        return l.ccl_linear_xent_grad(C.byref(d), p(X), p(W), p(targets), p(lse), p(dloss), p(dX), p(dW), p(ws), grad_need, None)

    overlaps(grad, at, sizes, ("dX", "dW", "ws"), ("X", "W", "targets", "lse", "dloss"))


@pytest.mark.parametrize("T,H", [(16, 512), (8192, 2048), (300, 1541)])
def test_norm(T, H):
    m, l = ccl.Mat(T, H, 2), ccl.lib()
    at = places("X", "gamma", "beta", "Y", "mean", "rstd")
    sizes = dict(X=2 * T * H, gamma=2 * H, beta=2 * H, Y=2 * T * H, mean=4 * T, rstd=4 * T)

    def forward(X, gamma, beta, Y, mean, rstd):
        return l.ccl_norm(C.byref(m), 0, 1e-5, p(X), p(gamma), p(beta), p(Y), p(mean), p(rstd), None)

    overlaps(forward, at, sizes, ("Y", "mean", "rstd"), ("X", "gamma", "beta"), allowed=(("Y", "X"),))


@pytest.mark.parametrize("T,H", [(16, 512), (8192, 2048), (300, 1541)])
def test_norm_grad(T, H):
    m, l = ccl.Mat(T, H, 2), ccl.lib()
    need = ccl.ccl_norm_grad_workspace(m)
    big, outputs = 2 * T * H, ("dX", "dgamma", "dbeta") + (("ws",) if need else ())
    at = places("X", "gamma", "mean", "rstd", "dY", "addend", "dX", "dgamma", "dbeta", "ws")
    sizes = dict(X=big, gamma=2 * H, mean=4 * T, rstd=4 * T, dY=big, addend=big, dX=big, dgamma=2 * H, dbeta=2 * H, ws=need)

    def grad(X, gamma, mean, rstd, dY, addend, dX, dgamma, dbeta, ws):
        return l.ccl_norm_grad(C.byref(m), 0, p(X), p(gamma), p(mean), p(rstd), p(dY), p(addend), p(dX), p(dgamma), p(dbeta), p(ws), 1 << 30, None)

    overlaps(grad, at, sizes, outputs, ("X", "gamma", "mean", "rstd", "dY", "addend"), allowed=(("dX", "X"), ("dX", "dY"), ("dX", "addend")))
