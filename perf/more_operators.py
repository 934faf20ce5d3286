"""Measured cases of what a training step has around its feed-forward blocks: the normalisation of the residual stream and
its gradient, the cross entropy over a large vocabulary without its logits being kept and its gradient, and the AdamW update of many
tensors.

Each operator has a plain form (elementary torch operations, rounded once at the end) and the framework's own call; `own` says
which of the two `run` makes.
"""
import math
import random

import torch

own = False

BF16 = torch.bfloat16
F8 = torch.float8_e4m3fn
IGNORE = -100
BLOCK = 256                                             # elements that share a scale of the 8-bit states
F8_MAX = 448.0
F8_LEAST = 2.0 ** -9
DROPPED = 1e-30                                         # blocks whose largest state is smaller than this are kept as zeros


# ---------------------------------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------------------------------

def _norm(name, T, H, kind="layer", P=1):
    """Normalised rows, their means and reciprocal deviations.  P > 1: rows stored in P strips of H / P columns."""
    return {"name": name, "op": "norm", "T": T, "H": H, "kind": kind, "P": P}


def _norm_grad(name, T, H, kind="layer", P=1, addend=True):
    """The rows' gradient (plus the residual stream's, `addend`) and those of weight and bias."""
    return {"name": name, "op": "norm_grad", "T": T, "H": H, "kind": kind, "P": P, "addend": addend}


def _xent(name, T, V, H, P=1, ignored=0.0):
    """Each token's loss and log of its partition sum.  P = 1: weight kept as [V x H], P > 1: [H x V] in P strips of columns."""
    return {"name": name, "op": "xent", "T": T, "V": V, "H": H, "P": P, "ignored": ignored}


def _xent_grad(name, T, V, H, P=1, ignored=0.0):
    """Gradients of the hidden states and of the weight."""
    return {"name": name, "op": "xent_grad", "T": T, "V": V, "H": H, "P": P, "ignored": ignored}


def _adamw(name, bits, count, least, most, shapes=1, grad="bf16", clip=False, copy=True):
    """A step over `count` tensors of `least` to `most` elements; copy: with the bfloat16 weights the products read."""
    return {"name": name, "op": "adamw", "bits": bits, "count": count, "least": least, "most": most, "shapes": shapes, "grad": grad,
            "clip": clip, "copy": copy}


def listed():
    return [
        # One decoded token of a 2048-wide block: the smallest call, all latency.
        _norm("norm_one_token", 1, 2048, "rms"),
        # A training batch of the dense 70B-size residual stream.
        _norm("norm_train", 8192, 8192),
        # The same going backward, the residual stream's own gradient added.
        _norm_grad("norm_grad_train", 8192, 8192),
        # A short ragged batch of odd width, no residual beside it.
        _norm_grad("norm_grad_ragged", 777, 1541, "rms", addend=False),
        # Scoring a few tokens against a vocabulary no tile divides.
        _xent("xent_few_tokens", 19, 50001, 2048),
        # A training batch at a vocabulary of 131072, padding in it ignored.
        _xent("xent_train", 8192, 131072, 4096, ignored=0.1),
        # The gradient of a short ragged batch.
        _xent_grad("xent_grad_ragged", 777, 50001, 1544, ignored=0.2),
        # The gradient of a training batch at the dense 70B-size width, the weight in four strips.
        _xent_grad("xent_grad_train", 4096, 131072, 8192, P=4, ignored=0.05),
        # All small tensors of a model -- norms, biases, routers -- after a clipped gradient: many, odd sizes.
        _adamw("adamw_many_small", 32, 300, 64, 40000, grad="fp32", clip=True),
        # A dense 70B-size projection, states in 32 bits.
        _adamw("adamw_70b_matrix", 32, 1, 8192 * 28672, 8192 * 28672),
        # The matrices of a few 2048-wide blocks, states in 8 bits.
        _adamw("adamw8_blocks", 8, 24, 2048 * 2048, 2048 * 8192, clip=True),
        # A small model's tensors, states in 8 bits, odd sizes.
        _adamw("adamw8_odd", 8, 40, 100, 1000000, copy=False),
    ]


def _log_int(rng, lo, hi, multiple=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v // multiple * multiple))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "xent", "xent_grad", "adamw"])
    if op == "adamw":
        least = _log_int(rng, 1, 1 << 20)
        most = _log_int(rng, least, 1 << 24)
        case = _adamw("", rng.choice([8, 32]), _log_int(rng, 1, 300 if most < 1 << 18 else 12), least, most, shapes=rng.randint(1, 1 << 30),
                      grad=rng.choice(["bf16", "fp32"]), clip=rng.random() < 0.5, copy=rng.random() < 0.7)
    elif op in ("norm", "norm_grad"):
        P = rng.choice([1, 1, 2, 4])
        T, H = _log_int(rng, 1, 8192), _log_int(rng, 32, 8192, 8 * P if rng.random() < 0.7 else P)
        kind = rng.choice(["layer", "rms"])
        case = _norm("", T, H, kind, P) if op == "norm" else _norm_grad("", T, H, kind, P, rng.random() < 0.5)
    else:
        P = rng.choice([1, 1, 2, 4])
        T, V, H = _log_int(rng, 1, 4096), _log_int(rng, 1000, 131072, 8 * P if P > 1 else 1), _log_int(rng, 64, 8192, 8)
        case = (_xent if op == "xent" else _xent_grad)("", T, V, H, P, rng.choice([0.0, 0.1, 0.3]))
    del case["name"]
    return case


def _sizes(case):
    """Elements of each tensor of an update."""
    r = random.Random(case["shapes"])
    return [_log_int(r, case["least"], case["most"]) for _ in range(case["count"])]


# ---------------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0, dtype=BF16):
        return torch.randn(*shape, generator=g, device="cuda", dtype=dtype).mul_(std)

    s = {"case": case}
    if case["op"] == "adamw":
        return _prepare_adamw(s, case, g)
    T, H, P = case["T"], case["H"], case["P"]
    if case["op"] in ("norm", "norm_grad"):
        # a residual stream: channels of different sizes, a few large ones, rows off centre
        scale = torch.exp(torch.randn(H, generator=g, device="cuda"))
        x = (normal(T, H, dtype=torch.float32) * scale + normal(T, 1, std=0.5, dtype=torch.float32)).to(BF16)
        s["x"] = _strips(x, P)
        s["gamma"] = (1 + 0.2 * torch.randn(H, generator=g, device="cuda")).to(BF16)
        s["beta"] = normal(H, std=0.1) if case["kind"] == "layer" else None
        s["eps"] = 1e-5
        if case["op"] == "norm_grad":
            s["dy"] = normal(P, T, H // P)
            s["addend"] = normal(P, T, H // P) if case["addend"] else None
            mean, rstd = _statistics(x.float(), case["kind"], s["eps"])
            s["mean"], s["rstd"] = mean if case["kind"] == "layer" else None, rstd
        return s
    V = case["V"]
    s["w"] = normal(V, H, std=0.02) if P == 1 else normal(P, H, V // P, std=0.02)
    targets = torch.randint(0, V, (T,), generator=g, device="cuda")
    # hidden states that lean towards their targets, from not at all to nearly certain
    x = normal(T, H, dtype=torch.float32)
    lean = 16.0 * torch.rand(T, 1, generator=g, device="cuda") / (0.02 * 0.02 * H)
    x += lean * (s["w"][targets] if P == 1 else s["w"][targets // (V // P), :, targets % (V // P)]).float()
    s["x"] = x.to(BF16)
    keep = torch.rand(T, generator=g, device="cuda") >= case["ignored"]
    s["targets"] = torch.where(keep, targets, IGNORE).to(torch.int32)
    if case["op"] == "xent_grad":
        s["lse"] = _lse(s["x"].float() @ _vocab_rows(s).float().t())
        s["dloss"] = keep.float() / max(1, T)
    return s


def _prepare_adamw(s, case, g):
    """All tensors lie in one arena, each from a multiple of BLOCK elements on (zeros between them)."""
    sizes = _sizes(case)
    starts, n = [], 0
    for k in sizes:
        starts.append(n)
        n += -(-k // BLOCK) * BLOCK
    s["sizes"], s["starts"] = sizes, starts
    tensor = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), torch.tensor([-(-k // BLOCK) * BLOCK for k in sizes], device="cuda"))
    used = torch.arange(n, device="cuda") - torch.tensor(starts, device="cuda")[tensor] < torch.tensor(sizes, device="cuda")[tensor]
    del tensor

    def normal(std):
        return torch.randn(n, generator=g, device="cuda").mul_(std).mul_(used)

    s["p"] = normal(0.02)
    grad = normal(1e-3)
    # gradients of very different sizes side by side, as rows of an embedding have them
    grad.mul_(torch.exp(2.0 * torch.randn(n // BLOCK, 1, generator=g, device="cuda")).expand(-1, BLOCK).reshape(-1))
    s["g"] = grad.to(BF16) if case["grad"] == "bf16" else grad
    s["copy"] = s["p"].to(BF16) if case["copy"] else None
    m = normal(3e-4)
    v = normal(1e-3).square_()
    if case["bits"] == 8:
        s["m"], s["ms"] = _to_8bit(m)
        s["v"], s["vs"] = _to_8bit(v.sqrt_(), least=True)
    else:
        s["m"], s["v"] = m, v
    s["clip"] = torch.rand(1, generator=g, device="cuda").mul_(0.5).add_(0.5) if case["clip"] else None
    s["hyper"] = {"lr": 3e-4, "beta1": 0.9, "beta2": 0.95, "eps": 1e-8, "weight_decay": 0.1, "step": 100}
    return s


def _strips(t, P):
    """[rows][columns] -> [P strips][rows][columns of a strip]"""
    return t.reshape(t.shape[0], P, -1).permute(1, 0, 2).contiguous()


def _rows(t):
    """[P strips][rows][columns of a strip] -> [rows][columns]"""
    return t.permute(1, 0, 2).reshape(t.shape[1], -1)


# ---------------------------------------------------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------------------------------------------------

def _statistics(x, kind, eps):
    mean = x.mean(1) if kind == "layer" else torch.zeros_like(x[:, 0])
    d = x - mean[:, None]
    return mean, 1 / torch.sqrt((d * d).mean(1) + eps)


def _plain_norm(s):
    case = s["case"]
    x = _rows(s["x"]).float()
    mean, rstd = _statistics(x, case["kind"], s["eps"])
    y = (x - mean[:, None]) * rstd[:, None] * s["gamma"].float()
    if s["beta"] is not None:
        y = y + s["beta"].float()
    out = {"y": _strips(y.to(BF16), case["P"]), "rstd": rstd}
    return {**out, "mean": mean} if case["kind"] == "layer" else out


def _plain_norm_grad(s):
    case = s["case"]
    layer = case["kind"] == "layer"
    x, dy, rstd = _rows(s["x"]).float(), _rows(s["dy"]).float(), s["rstd"][:, None]
    h = (x - s["mean"][:, None]) * rstd if layer else x * rstd
    g = dy * s["gamma"].float()
    dx = g - h * (g * h).mean(1, keepdim=True)
    if layer:
        dx = dx - g.mean(1, keepdim=True)
    dx = dx * rstd
    if s["addend"] is not None:
        dx = dx + _rows(s["addend"]).float()
    out = {"dx": _strips(dx.to(BF16), case["P"]), "dgamma": (dy * h).sum(0).to(BF16)}
    return {**out, "dbeta": dy.sum(0).to(BF16)} if layer else out


def _vocab_rows(s):
    """The weight as [V x H]."""
    return s["w"] if s["case"]["P"] == 1 else s["w"].permute(0, 2, 1).reshape(s["case"]["V"], -1)


def _lse(z):
    top = z.amax(1)
    return top + torch.log(torch.exp(z - top[:, None]).sum(1))


def _plain_xent(s):
    z = s["x"].float() @ _vocab_rows(s).float().t()
    lse = _lse(z)
    target = s["targets"].long()
    at = torch.gather(z, 1, target.clamp(min=0)[:, None])[:, 0]
    return {"loss": torch.where(target == IGNORE, torch.zeros_like(lse), lse - at), "lse": lse}


def _plain_xent_grad(s):
    case = s["case"]
    x, w, target = s["x"].float(), _vocab_rows(s).float(), s["targets"].long()
    scale = torch.where(target == IGNORE, torch.zeros_like(s["dloss"]), s["dloss"])
    z = x @ w.t()
    dz = torch.exp(z.sub_(s["lse"][:, None])).mul_(scale[:, None])
    dz.scatter_add_(1, target.clamp(min=0)[:, None], -scale[:, None])
    dw = (dz.t() @ x).to(BF16)
    if case["P"] > 1:
        dw = dw.view(case["P"], -1, case["H"]).permute(0, 2, 1).contiguous()
    return {"dx": (dz @ w).to(BF16), "dw": dw}


def _to_8bit(x, least=False):
    """Values of `x` in blocks of BLOCK as e4m3 and a scale a block; least: none but zeros become zero."""
    b = x.view(-1, BLOCK)
    top = b.abs().amax(1)
    kept = ~(top < DROPPED)
    zero = torch.zeros_like(top)
    inverse = torch.where(kept, torch.div(torch.full_like(top, F8_MAX), top), zero)
    q = (b * inverse[:, None]).to(F8)
    if least:
        q = torch.where((b > 0) & (q.float() == 0), torch.full_like(b, F8_LEAST), q.float()).to(F8)
    return q.view(-1), torch.where(kept, top * (1 / F8_MAX), zero)


def _from_8bit(q, scale):
    return (q.view(-1, BLOCK).float() * scale[:, None]).view(-1)


def _plain_adamw(s):
    """In place, every operation rounded by itself."""
    h, case = s["hyper"], s["case"]
    grad = s["g"].float()
    if s["clip"] is not None:
        grad = grad * s["clip"]
    if case["bits"] == 8:
        m, r = _from_8bit(s["m"], s["ms"]), _from_8bit(s["v"], s["vs"])
        v = r * r
    else:
        m, v = s["m"], s["v"]
    m = m * h["beta1"] + grad * (1 - h["beta1"])
    v = v * h["beta2"] + grad * (1 - h["beta2"]) * grad
    r = torch.sqrt(v)
    step = torch.div(m, r * (1 / math.sqrt(1 - h["beta2"] ** h["step"])) + h["eps"])
    p = s["p"] * (1 - h["lr"] * h["weight_decay"]) - step * (h["lr"] / (1 - h["beta1"] ** h["step"]))
    s["p"].copy_(p)
    if case["bits"] == 8:
        q, scale = _to_8bit(m)
        s["m"].copy_(q), s["ms"].copy_(scale)
        q, scale = _to_8bit(r, least=True)
        s["v"].copy_(q), s["vs"].copy_(scale)
    else:
        s["m"].copy_(m), s["v"].copy_(v)
    if s["copy"] is not None:
        s["copy"].copy_(p)
    return _updated(s)


def _updated(s):
    out = {"p": s["p"]}
    if s["case"]["bits"] == 8:
        out["m"], out["sqrt_v"] = _from_8bit(s["m"], s["ms"]), _from_8bit(s["v"], s["vs"])
    else:
        out["m"], out["v"] = s["m"], s["v"]
    return {**out, "copy": s["copy"]} if s["copy"] is not None else out


_PLAIN = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "xent": _plain_xent, "xent_grad": _plain_xent_grad, "adamw": _plain_adamw}


# ---------------------------------------------------------------------------------------------------------------------
# The framework's calls.  What a program builds once for a shape (descriptor, workspace, output buffers, the list of an update's
# tensors) is kept with the state; the calls take the tensors as they are.
# ---------------------------------------------------------------------------------------------------------------------

def _workspace(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


def _norm_plan(s, case):
    from paper_2606_11718_b200 import binding as ccl
    T, H, P = case["T"], case["H"], case["P"]
    split = (P, ccl.PART_COLS, ccl.CCL, 0) if P > 1 else (1, ccl.PART_NONE, ccl.ROWMAJOR, 0)
    m, layer = ccl.Mat(T, H, 2, *split), case["kind"] == "layer"
    plan = {"ccl": ccl, "m": m, "kind": ccl.NORM_LAYER if layer else ccl.NORM_RMS, "out": torch.empty_like(s["x"])}
    if case["op"] == "norm":
        plan["rstd"] = torch.empty(T, device="cuda")
        plan["mean"] = torch.empty(T, device="cuda") if layer else None
    else:
        plan["dgamma"] = torch.empty(H, dtype=BF16, device="cuda")
        plan["dbeta"] = torch.empty(H, dtype=BF16, device="cuda") if layer else None
        plan["ws"] = _workspace(ccl.ccl_norm_grad_workspace(m))
    return plan


def _xent_plan(s, case):
    from paper_2606_11718_b200 import binding as ccl
    T, V, H, P = case["T"], case["V"], case["H"], case["P"]
    w = ccl.Mat(V, H, 2) if P == 1 else ccl.Mat(H, V, 2, P, ccl.PART_COLS, ccl.CCL, 0)
    d = ccl.XentDesc(T, V, H, w, w_trans=int(P == 1), ignore_index=IGNORE)
    plan = {"ccl": ccl, "d": d}
    if case["op"] == "xent":
        plan["loss"], plan["lse"] = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        plan["ws"] = _workspace(ccl.ccl_linear_xent_workspace(d))
    else:
        plan["dx"], plan["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
        plan["ws"] = _workspace(ccl.ccl_linear_xent_grad_workspace(d))
    return plan


def _adamw_plan(s, case):
    from paper_2606_11718_b200 import binding as ccl
    parts = list(zip(s["starts"], s["sizes"]))

    def views(t):
        return None if t is None else [t[a:a + k] for a, k in parts]

    def scales(t):
        return [t[a // BLOCK:a // BLOCK + -(-k // BLOCK)] for a, k in parts] if case["bits"] == 8 else None

    tensors = ccl.AdamwTensors(views(s["p"]), views(s["g"]), views(s["m"]), views(s["v"]), copies=views(s["copy"]),
                               m_scales=scales(s.get("ms")), v_scales=scales(s.get("vs")))
    return {"ccl": ccl, "tensors": tensors, "d": ccl.AdamwDesc(**s["hyper"])}


_PLANS = {"norm": _norm_plan, "norm_grad": _norm_plan, "xent": _xent_plan, "xent_grad": _xent_plan, "adamw": _adamw_plan}


def _own(s):
    case = s["case"]
    plan = s.get("plan")
    if plan is None:
        plan = s["plan"] = _PLANS[case["op"]](s, case)
    ccl = plan["ccl"]
    if case["op"] == "norm":
        ccl.ccl_norm(plan["m"], s["x"], s["gamma"], s["beta"], plan["out"], kind=plan["kind"], eps=s["eps"], mean=plan["mean"], rstd=plan["rstd"])
        out = {"y": plan["out"], "rstd": plan["rstd"]}
        return {**out, "mean": plan["mean"]} if plan["mean"] is not None else out
    if case["op"] == "norm_grad":
        ccl.ccl_norm_grad(plan["m"], s["x"], s["gamma"], s["mean"], s["rstd"], s["dy"], plan["out"], plan["ws"], kind=plan["kind"],
                          addend=s["addend"], dgamma=plan["dgamma"], dbeta=plan["dbeta"])
        out = {"dx": plan["out"], "dgamma": plan["dgamma"]}
        return {**out, "dbeta": plan["dbeta"]} if plan["dbeta"] is not None else out
    if case["op"] == "xent":
        ccl.ccl_linear_xent(plan["d"], s["x"], s["w"], s["targets"], plan["loss"], plan["lse"], plan["ws"])
        return {"loss": plan["loss"], "lse": plan["lse"]}
    if case["op"] == "xent_grad":
        ccl.ccl_linear_xent_grad(plan["d"], s["x"], s["w"], s["targets"], s["lse"], s["dloss"], plan["dx"], plan["dw"], plan["ws"])
        return {"dx": plan["dx"], "dw": plan["dw"]}
    ccl.ccl_adamw(plan["d"], plan["tensors"], grad_scale=s["clip"])
    return _updated(s)


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------------

def work(case):
    if case["op"] == "adamw":
        n = float(sum(_sizes(case)))
        state = 16.0 if case["bits"] == 32 else 4.0 + 16.0 / BLOCK
        return {"bytes": n * (8 + state + (2 if case["grad"] == "bf16" else 4) + (2 if case["copy"] else 0)), "flops": 15.0 * n}
    T, H = float(case["T"]), float(case["H"])
    layer = case.get("kind") == "layer"
    if case["op"] == "norm":
        return {"bytes": 4 * T * H + (2 + 2 * layer) * H + (4 + 4 * layer) * T, "flops": 8 * T * H}
    if case["op"] == "norm_grad":
        return {"bytes": (6 + 2 * case["addend"]) * T * H + (4 + 2 * layer) * H + (4 + 4 * layer) * T, "flops": 14 * T * H}
    V = float(case["V"])
    if case["op"] == "xent":
        return {"bytes": 2 * (T * H + V * H) + 12 * T, "flops": 2 * T * H * V}
    return {"bytes": 4 * (T * H + V * H) + 12 * T, "flops": 6 * T * H * V}


# ---------------------------------------------------------------------------------------------------------------------
# The same results in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------------------------------

def _whole64(t):
    return torch.cat(list(t.double()), dim=1)


def _cut64(t, P):
    return torch.stack(t.chunk(P, dim=1))


def _exact_norm(s, case):
    x, gamma, layer = _whole64(s["x"]), s["gamma"].double(), case["kind"] == "layer"
    mean = x.sum(1) / case["H"] if layer else x.new_zeros(x.shape[0])
    if case["op"] == "norm":
        rstd = (((x - mean[:, None]) ** 2).sum(1) / case["H"] + s["eps"]) ** -0.5
        y = torch.einsum("th,t,h->th", x - mean[:, None], rstd, gamma)
        if layer:
            return {"y": _cut64(y + s["beta"].double(), case["P"]), "rstd": rstd, "mean": mean}
        return {"y": _cut64(y, case["P"]), "rstd": rstd}
    # the gradient by automatic differentiation of the definition
    with torch.enable_grad():
        x.requires_grad_(True)
        w = gamma.clone().requires_grad_(True)
        b = torch.zeros_like(gamma).requires_grad_(True)
        c = x - x.mean(1, keepdim=True) if layer else x
        y = c * torch.rsqrt((c * c).mean(1, keepdim=True) + s["eps"]) * w + b
        dx, dw, db = torch.autograd.grad(y, (x, w, b), _whole64(s["dy"]))
    if case["addend"]:
        dx = dx + _whole64(s["addend"])
    out = {"dx": _cut64(dx, case["P"]), "dgamma": dw}
    return {**out, "dbeta": db} if layer else out


def _exact_xent(s, case):
    P, H = case["P"], case["H"]
    w = s["w"].double() if P == 1 else torch.cat([strip.double().T for strip in s["w"]])
    x, t = s["x"].double(), s["targets"].long()
    kept = t != IGNORE
    rows = torch.arange(case["T"], device="cuda")[kept]
    logits = torch.nn.functional.linear(x, w)
    if case["op"] == "xent":
        lse = torch.logsumexp(logits, 1)
        loss = torch.zeros_like(lse)
        loss[kept] = lse[kept] - logits[rows, t[kept]]
        return {"loss": loss, "lse": lse}
    dz = torch.softmax(logits, 1)
    dz[rows, t[kept]] -= 1
    dz *= (s["dloss"].double() * kept)[:, None]
    dw = torch.matmul(dz.T, x)
    return {"dx": torch.matmul(dz, w), "dw": dw if P == 1 else torch.stack([part.T for part in dw.split(case["V"] // P)])}


def _exact_adamw(s, case):
    h = s["hyper"]
    b1, b2, t = h["beta1"], h["beta2"], h["step"]
    g = s["g"].double()
    if case["clip"]:
        g = g * s["clip"].double()
    eight = case["bits"] == 8
    m, v = s["m"].double(), s["v"].double()
    if eight:
        m = m * s["ms"].double().repeat_interleave(BLOCK)
        v = (v * s["vs"].double().repeat_interleave(BLOCK)) ** 2
    m = torch.lerp(g, m, b1)
    v = torch.lerp(g ** 2, v, b2)
    m_hat, v_hat = m / (1 - b1 ** t), v / (1 - b2 ** t)
    p = s["p"].double()
    p = p - h["lr"] * (h["weight_decay"] * p + m_hat / (v_hat.sqrt() + h["eps"]))
    out = {"p": p}
    # (the 8-bit states stand for roundings to four bits: the values beneath them are no result)
    out["m"], out["sqrt_v" if eight else "v"] = (None, None) if eight else (m, v)
    return {**out, "copy": p} if case["copy"] else out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adamw":
        return _exact_adamw(s, case)
    return _exact_norm(s, case) if case["op"] in ("norm", "norm_grad") else _exact_xent(s, case)
