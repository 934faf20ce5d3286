"""Operands of the normalisation, the linear cross entropy and the AdamW step that the GPU cannot use as they are: refused by the binding, nothing
written; and calls in other places than the tested ones: several at once on streams, two graphs side by side."""
import pytest
import torch

from paper_2606_11718_b200 import binding as ccl

pytestmark = pytest.mark.gpu

T, H, V = 40, 64, 300


def bf(*shape, **kw):
    return torch.ones(*shape, dtype=torch.bfloat16, device="cuda", **kw)


def fp(*shape):
    return torch.ones(*shape, device="cuda")


def refused(f, *args, **kw):
    with pytest.raises(ValueError):
        f(*args, **kw)


def variants(t):
    """Forms of an operand that are not what a call takes."""
    yield t.cpu()
    yield t.half() if t.dtype is torch.bfloat16 else t.double()
    yield t.view(-1)[:-1]
    yield torch.stack([t, t], -1)[..., 0]                       # every other element


def test_norm():
    m = ccl.Mat(T, H, 2)
    good = dict(X=bf(T, H), gamma=bf(H), beta=bf(H), Y=bf(T, H) * 5, mean=fp(T), rstd=fp(T))
    for k, t in good.items():
        for bad in variants(t):
            refused(ccl.ccl_norm, m, **{**good, k: bad})
    assert (good["Y"] == 5).all()
    ccl.ccl_norm(m, **good)
    assert (good["Y"] == 1).all()
    refused(ccl.ccl_norm, m, None, None, None, good["Y"])


def test_norm_grad():
    m = ccl.Mat(T, H, 2)
    good = dict(X=bf(T, H), gamma=bf(H), mean=fp(T), rstd=fp(T), dy=bf(T, H), dx=bf(T, H) * 5, addend=bf(T, H), dgamma=bf(H), dbeta=bf(H))
    for k, t in good.items():
        for bad in variants(t):
            refused(ccl.ccl_norm_grad, m, **{**good, k: bad})
    refused(ccl.ccl_norm_grad, m, **good, ws=torch.empty(1000))
    assert (good["dx"] == 5).all()
    ccl.ccl_norm_grad(m, **good)


def test_xent():
    d = ccl.XentDesc(T, V, H)
    targets = torch.zeros(T, dtype=torch.int32, device="cuda")
    ws = torch.empty(ccl.ccl_linear_xent_workspace(d), dtype=torch.uint8, device="cuda")
    good = dict(X=bf(T, H), W=bf(V, H), targets=targets, loss=fp(T) * 5, lse=fp(T) * 5, ws=ws)
    for k, t in good.items():
        for bad in variants(t) if k != "ws" else (ws.cpu(), torch.stack([ws, ws], -1)[..., 0]):
            refused(ccl.ccl_linear_xent, d, **{**good, k: bad})
    refused(ccl.ccl_linear_xent, d, **{**good, "targets": targets.long()})
    assert (good["loss"] == 5).all() and (good["lse"] == 5).all()
    ws = torch.empty(ccl.ccl_linear_xent_grad_workspace(d), dtype=torch.uint8, device="cuda")
    good = dict(X=bf(T, H), W=bf(V, H), targets=targets, lse=fp(T), dloss=fp(T), dX=bf(T, H) * 5, dW=bf(V, H) * 5, ws=ws)
    for k, t in good.items():
        for bad in variants(t) if k != "ws" else (ws.cpu(),):
            refused(ccl.ccl_linear_xent_grad, d, **{**good, k: bad})
    with pytest.raises(ccl.CclError) as e:
        ccl.ccl_linear_xent_grad(d, **{**good, "ws": ws[:1000]})
    assert e.value.status == ccl.ERR_WORKSPACE
    assert (good["dX"] == 5).all() and (good["dW"] == 5).all()


def test_adamw():
    good = [[fp(100)], [bf(100)], [fp(100)], [fp(100)]]
    for k in range(4):
        for bad in variants(good[k][0]):
            refused(ccl.AdamwTensors, *(good[:k] + [[bad]] + good[k + 1:]))
    tensors = ccl.AdamwTensors(*good)
    for kw in (dict(grad_scale=torch.ones(1)), dict(grad_scale=torch.ones(1, device="cuda", dtype=torch.float64)), dict(step=torch.ones(1, device="cuda")),
               dict(step=torch.ones(1, device="cuda", dtype=torch.int64), lr=torch.ones(1))):
        refused(ccl.ccl_adamw, ccl.AdamwDesc(), tensors, **kw)
    with pytest.raises(ccl.CclError) as e:
        ccl.ccl_adamw(ccl.AdamwDesc(), tensors, lr=fp(1))       # a rate on the device goes with a step there
    assert e.value.status == ccl.ERR_INVALID_ARG
    assert (good[0][0] == 1).all()


def problem(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s, std=1.0: (torch.randn(*s, generator=g, device="cuda") * std).to(torch.bfloat16)     # noqa: E731
    T, H, V = 600, 520, 3001
    p = dict(x=normal(T, H), w=normal(V, H, std=0.05), dy=normal(T, H), gamma=normal(H), d=ccl.XentDesc(T, V, H), m=ccl.Mat(T, H, 2),
             tg=torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32), y=bf(T, H), mean=fp(T), rstd=fp(T), dx=bf(T, H), dgamma=bf(H), loss=fp(T), lse=fp(T),
             dX=bf(T, H), dW=bf(V, H), dloss=fp(T) / T)
    need = max(ccl.ccl_norm_grad_workspace(p["m"]), ccl.ccl_linear_xent_workspace(p["d"]), ccl.ccl_linear_xent_grad_workspace(p["d"]))
    p["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    return p


def run(p):
    ccl.ccl_norm(p["m"], p["x"], p["gamma"], None, p["y"], mean=p["mean"], rstd=p["rstd"])
    ccl.ccl_linear_xent(p["d"], p["y"], p["w"], p["tg"], p["loss"], p["lse"], p["ws"])
    ccl.ccl_linear_xent_grad(p["d"], p["y"], p["w"], p["tg"], p["lse"], p["dloss"], p["dX"], p["dW"], p["ws"])
    ccl.ccl_norm_grad(p["m"], p["x"], p["gamma"], p["mean"], p["rstd"], p["dX"], p["dx"], p["ws"], dgamma=p["dgamma"], addend=p["dy"])
    return [p[k] for k in ("y", "loss", "lse", "dX", "dW", "dx", "dgamma")]


def test_several_at_once_on_streams():
    ps = [problem(k) for k in range(3)]
    want = [[t.clone() for t in run(p)] for p in ps]
    for p in ps:
        for t in run(p):
            t.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ps]
    for _ in range(5):
        for p, s in zip(ps, streams):
            with torch.cuda.stream(s):
                run(p)
    torch.cuda.synchronize()
    for p, w in zip(ps, want):
        for k, t in zip(("y", "loss", "lse", "dX", "dW", "dx", "dgamma"), w):
            assert torch.equal(p[k], t), k
    assert ccl.ccl_gemm_status()[0] == ccl.OK


def test_two_graphs_with_workspaces_of_their_own():
    ps = [problem(k + 7) for k in range(2)]
    want = [[t.clone() for t in run(p)] for p in ps]
    graphs = []
    for p in ps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run(p)
        graphs.append(g)
    for p in ps:
        for k in ("y", "loss", "lse", "dX", "dW", "dx", "dgamma"):
            p[k].zero_()
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for p, w in zip(ps, want):
        for k, t in zip(("y", "loss", "lse", "dX", "dW", "dx", "dgamma"), w):
            assert torch.equal(p[k], t), k
