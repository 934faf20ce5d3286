"""Measured cases of the feed-forward operators around the GEMM: the GEMM with bias, activation and residual in its
epilogue, the two passes of its gradient, and a mixture-of-experts layer for a few tokens.

Each operator has a plain form (elementary torch operations in 32 bits, rounded once at the end) and the framework's own
call; `own` says which of the two `run` makes.
"""
import math

import torch

own = False

BF16 = torch.bfloat16
ACTS = ("none", "relu", "gelu_tanh", "gelu_erf", "silu")


# ---------------------------------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------------------------------

def _epilogue(name, M, N, K, act, b_trans=False, P=1, bias=True, residual=False, preact=False):
    """C = act(A B + bias) + residual.  P > 1: B, C, residual and pre-activation in P strips of N / P columns each."""
    return {"name": name, "op": "epilogue", "M": M, "N": N, "K": K, "act": act, "b_trans": b_trans, "P": P, "bias": bias,
            "residual": residual, "preact": preact}


def _act_grad(name, M, N, K, act, b_trans=True, P=1, dbias=True):
    """dZ = (A B) * act'(Z), and the column sums of dZ."""
    return {"name": name, "op": "act_grad", "M": M, "N": N, "K": K, "act": act, "b_trans": b_trans, "P": P, "dbias": dbias}


def _bias_grad(name, M, N, act):
    """dZ = dY * act'(Z), and the column sums of dZ (act "none": the sums alone)."""
    return {"name": name, "op": "bias_grad", "M": M, "N": N, "act": act}


def _moe(name, T, E, topk, H, I, norm=True, residual=False):
    """Router, top-k, gated expert feed-forward and weighted sum for T tokens."""
    return {"name": name, "op": "moe", "T": T, "E": E, "topk": topk, "H": H, "I": I, "norm": norm, "residual": residual}


def listed():
    return [
        # One decoded token through the up projection of a small dense block: the smallest call, all latency.
        _epilogue("up_one_token", 1, 8192, 2048, "gelu_tanh"),
        # Sixteen decoded tokens through the down projection of the dense 70B-size block, added to the residual stream.
        _epilogue("down_16_tokens", 16, 8192, 28672, "none", residual=True),
        # A ragged prefill: token count and widths that no tile divides, weight kept as [N x K].
        _epilogue("prefill_ragged", 333, 1000, 1544, "silu", b_trans=True, residual=True),
        # A training step's up projection at the dense 70B size, weights and activations in four strips, the
        # pre-activation kept for the gradient.
        _epilogue("train_up_70b", 4096, 28672, 8192, "gelu_tanh", P=4, preact=True),
        # The gradient through a 2048-wide block's activation: the product with the down projection's transpose.
        _act_grad("dgrad_block", 4096, 8192, 2048, "gelu_tanh"),
        # The same for a short ragged batch with the exact activation, weight kept as [K x N].
        _act_grad("dgrad_ragged", 777, 1544, 1000, "gelu_erf", b_trans=False),
        # An output layer's own activation gradient, and its bias's gradient.
        _bias_grad("bias_grad_silu", 8192, 8192, "silu"),
        # The gradient of a bias that no activation follows, a ragged batch.
        _bias_grad("bias_grad_plain", 1531, 2056, "none"),
        # One decoded token through a 128-expert layer, eight experts a token, added to the residual stream.
        _moe("moe_one_token", 1, 128, 8, 2048, 768, residual=True),
        # A handful of sequences on a layer of another make: odd widths, weights of the chosen experts not renormalised.
        _moe("moe_seven_odd", 7, 60, 4, 1544, 712, norm=False),
        # The largest decode batch taken: nearly every expert is read.
        _moe("moe_64_tokens", 64, 128, 8, 2048, 768, residual=True),
    ]


def _log_int(rng, lo, hi, multiple=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v // multiple * multiple))


def draw(rng):
    op = rng.choice(["epilogue", "act_grad", "bias_grad", "moe"])
    if op == "bias_grad":
        M = _log_int(rng, 1, 8192)
        return _drop_name(_bias_grad("", M, _log_int(rng, 64, 8192, 8), rng.choice(ACTS)))
    if op == "moe":
        E = rng.choice([8, 16, 60, 64, 128])
        H = _log_int(rng, 512, 2048, 8)
        T = _log_int(rng, 1, 64)
        topk = rng.randint(1, 8)
        return _drop_name(_moe("", T, E, topk, H, _log_int(rng, 128, 768, 8), norm=rng.random() < 0.5, residual=rng.random() < 0.5))
    P = rng.choice([1, 1, 2, 4])
    N = _log_int(rng, 128, 28672, 8 * P)
    K = _log_int(rng, 64, 8192, 8)
    M = _log_int(rng, 1, 4096)
    act = rng.choice(ACTS)
    if op == "act_grad":
        return _drop_name(_act_grad("", M, N, K, act, b_trans=rng.random() < 0.5, P=P, dbias=rng.random() < 0.8))
    return _drop_name(_epilogue("", M, N, K, act, b_trans=rng.random() < 0.5, P=P, bias=rng.random() < 0.8,
                                residual=rng.random() < 0.5, preact=rng.random() < 0.3))


def _drop_name(case):
    del case["name"]
    return case


# ---------------------------------------------------------------------------------------------------------------------
# Inputs: activations and gradients ~ N(0, 1), weights ~ N(0, 0.02), biases ~ N(0, 0.1), all bf16
# ---------------------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda", dtype=BF16).mul_(std)

    s = {"case": case}
    if case["op"] == "moe":
        T, E, H, I = case["T"], case["E"], case["H"], case["I"]
        s["x"] = normal(T, H)
        s["router"] = normal(E, H, std=0.02)
        s["w_gu"] = normal(E, 2 * I, H, std=0.02)           # expert e: I gate rows, then I up rows
        s["w_down"] = normal(E, H, I, std=0.02)
        s["residual"] = normal(T, H) if case["residual"] else None
        return s
    M, N = case["M"], case["N"]
    if case["op"] == "bias_grad":
        s["dy"] = normal(M, N)
        s["z"] = normal(M, N) if case["act"] != "none" else None
        return s
    P, K = case["P"], case["K"]
    s["a"] = normal(M, K)
    # a weight kept as [N x K], or as [K x N] in P strips of columns
    s["w"] = normal(N, K, std=0.02) if case["b_trans"] else normal(P, K, N // P, std=0.02)
    if case["op"] == "epilogue":
        s["bias"] = normal(N, std=0.1) if case["bias"] else None
        s["residual"] = normal(P, M, N // P) if case["residual"] else None
    else:
        s["z"] = normal(P, M, N // P)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------------------------------------------------

_SQRT_2_PI = math.sqrt(2.0 / math.pi)


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(_SQRT_2_PI * (z + 0.044715 * z * z * z)))
    if act == "gelu_erf":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu_tanh":
        t = torch.tanh(_SQRT_2_PI * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * _SQRT_2_PI * (1 + 3 * 0.044715 * z * z)
    if act == "gelu_erf":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _rows(t):
    """[P strips][rows][columns of a strip] -> [rows][columns]"""
    return t.permute(1, 0, 2).reshape(t.shape[1], -1)


def _strips(t, P):
    """[rows][columns] -> [P strips][rows][columns of a strip]"""
    return t.reshape(t.shape[0], P, -1).permute(1, 0, 2).contiguous()


def _product(s, dtype):
    w = s["w"].to(dtype).t() if s["case"]["b_trans"] else _rows(s["w"]).to(dtype)
    return s["a"].to(dtype) @ w


def _plain_epilogue(s):
    case = s["case"]
    z = _product(s, torch.float32)
    if s["bias"] is not None:
        z = z + s["bias"].float()
    c = _act(z, case["act"])
    if s["residual"] is not None:
        c = c + _rows(s["residual"]).float()
    out = {"c": _strips(c.to(BF16), case["P"])}
    if case["preact"]:
        out["z"] = _strips(z.to(BF16), case["P"])
    return out


def _plain_act_grad(s):
    case = s["case"]
    dz = _product(s, torch.float32) * _act_slope(_rows(s["z"]).float(), case["act"])
    out = {"dz": _strips(dz.to(BF16), case["P"])}
    if case["dbias"]:
        out["dbias"] = dz.sum(0).to(BF16)
    return out


def _plain_bias_grad(s):
    dz = s["dy"].float()
    if s["z"] is None:
        return {"dbias": dz.sum(0).to(BF16)}
    dz = dz * _act_slope(s["z"].float(), s["case"]["act"])
    return {"dz": dz.to(BF16), "dbias": dz.sum(0).to(BF16)}


def _plain_moe(s):
    case = s["case"]
    I, k = case["I"], case["topk"]
    x = s["x"].float()
    p = torch.exp(x @ s["router"].float().t())
    p = p / p.sum(1, keepdim=True)
    w, ids = torch.sort(p, dim=1, descending=True, stable=True)        # equal values: the lowest expert first
    w, ids = w[:, :k], ids[:, :k]
    if case["norm"]:
        w = w / w.sum(1, keepdim=True)
    gu = (s["w_gu"][ids].float() @ x[:, None, :, None])[..., 0]       # [T, k, 2 I]
    h = _act(gu[..., :I], "silu") * gu[..., I:]
    y = ((s["w_down"][ids].float() @ h[..., None])[..., 0] * w[..., None]).sum(1)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(BF16)}


_PLAIN = {"epilogue": _plain_epilogue, "act_grad": _plain_act_grad, "bias_grad": _plain_bias_grad, "moe": _plain_moe}


# ---------------------------------------------------------------------------------------------------------------------
# The framework's calls.  What a program builds once for a shape (descriptor, workspace, output buffers) is kept with
# the state; the calls take the tensors as they are.
# ---------------------------------------------------------------------------------------------------------------------

def _empty(n):
    return torch.empty(n, dtype=BF16, device="cuda")


def _gemm_plan(case):
    from paper_2606_11718_b200 import binding as ccl
    M, N, K, P = case["M"], case["N"], case["K"], case["P"]
    d = ccl.GemmDesc()
    d.M, d.N, d.K = M, N, K
    split = (P, ccl.PART_COLS, ccl.CCL, 0) if P > 1 else (1, ccl.PART_NONE, ccl.ROWMAJOR, 0)
    d.A = ccl.Mat(M, K, 2)
    d.B = ccl.Mat(N, K, 2) if case["b_trans"] else ccl.Mat(K, N, 2, *split)
    d.C = ccl.Mat(M, N, 2, *split)
    d.a_trans, d.b_trans, d.out_part, d.P, d.grouped_raster = 0, int(case["b_trans"]), ccl.PART_COLS, P, 1
    plan = {"ccl": ccl, "d": d, "act": getattr(ccl, "ACT_" + case["act"].upper()), "out": torch.empty(P, M, N // P, dtype=BF16, device="cuda")}
    if case["op"] == "epilogue":
        plan["z"] = torch.empty_like(plan["out"]) if case["preact"] else None
        need = ccl.ccl_gemm_epilogue_workspace(d)
    else:
        plan["dbias"] = _empty(N) if case["dbias"] else None
        need = ccl.ccl_gemm_act_grad_workspace(d)
    plan["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    return plan


def _bias_grad_plan(case):
    from paper_2606_11718_b200 import binding as ccl
    return {"ccl": ccl, "m": ccl.Mat(case["M"], case["N"], 2), "act": getattr(ccl, "ACT_" + case["act"].upper()),
            "dz": torch.empty(case["M"], case["N"], dtype=BF16, device="cuda") if case["act"] != "none" else None,
            "dbias": _empty(case["N"])}


def _moe_plan(case):
    from paper_2606_11718_b200 import binding as ccl
    d = ccl.MoeDesc(case["T"], case["E"], case["topk"], case["H"], case["I"], norm_topk=int(case["norm"]))
    return {"ccl": ccl, "d": d, "y": torch.empty(case["T"], case["H"], dtype=BF16, device="cuda"),
            "ws": torch.empty(ccl.ccl_moe_tokens_workspace(d), dtype=torch.uint8, device="cuda")}


_PLANS = {"epilogue": _gemm_plan, "act_grad": _gemm_plan, "bias_grad": _bias_grad_plan, "moe": _moe_plan}


def _own(s):
    case = s["case"]
    plan = s.get("plan")
    if plan is None:
        plan = s["plan"] = _PLANS[case["op"]](case)
    ccl = plan["ccl"]
    if case["op"] == "epilogue":
        ccl.ccl_gemm_epilogue(plan["d"], s["a"], s["w"], plan["out"], plan["ws"], act=plan["act"], bias=s["bias"],
                              residual=s["residual"], preact=plan["z"])
        return {"c": plan["out"], "z": plan["z"]} if case["preact"] else {"c": plan["out"]}
    if case["op"] == "act_grad":
        ccl.ccl_gemm_act_grad(plan["d"], s["a"], s["w"], s["z"], plan["out"], plan["ws"], act=plan["act"], dbias=plan["dbias"])
        return {"dz": plan["out"], "dbias": plan["dbias"]} if case["dbias"] else {"dz": plan["out"]}
    if case["op"] == "bias_grad":
        ccl.ccl_bias_act_grad(plan["m"], s["dy"], s["z"], plan["dz"], plan["dbias"], act=plan["act"])
        return {"dbias": plan["dbias"]} if plan["dz"] is None else {"dz": plan["dz"], "dbias": plan["dbias"]}
    ccl.ccl_moe_tokens(plan["d"], s["x"], s["router"], s["w_gu"], s["w_down"], plan["y"], plan["ws"], residual=s["residual"])
    return {"y": plan["y"]}


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------------

def work(case):
    if case["op"] == "moe":
        T, E, k, H, I = (case[n] for n in ("T", "E", "topk", "H", "I"))
        read = E * (1.0 - (1.0 - k / E) ** T)                  # experts that at least one of T tokens chooses, on average
        bytes_ = 2.0 * (read * 3 * H * I + E * H + T * H * (3 if case["residual"] else 2))
        return {"bytes": bytes_, "flops": 2.0 * T * (E * H + k * 3 * H * I)}
    M, N = case["M"], case["N"]
    if case["op"] == "bias_grad":
        return {"bytes": 2.0 * (M * N * (1 if case["act"] == "none" else 3) + N), "flops": 2.0 * M * N}
    K = case["K"]
    if case["op"] == "epilogue":
        tiles = 1 + int(case["residual"]) + int(case["preact"])
        vec = int(case["bias"])
    else:
        tiles, vec = 2, int(case["dbias"])
    return {"bytes": 2.0 * (M * K + K * N + tiles * M * N + vec * N), "flops": 2.0 * M * N * K}


# ---------------------------------------------------------------------------------------------------------------------
# The same results in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------------------------------

_DEFINED = {
    "none": lambda z: z,
    "relu": torch.nn.functional.relu,
    "gelu_tanh": lambda z: torch.nn.functional.gelu(z, approximate="tanh"),
    "gelu_erf": torch.nn.functional.gelu,
    "silu": torch.nn.functional.silu,
}


def _weight64(s):
    if s["case"]["b_trans"]:
        return s["w"].double().T
    return torch.cat(list(s["w"].double()), dim=1)


def _unstrip64(t):
    return torch.cat(list(t.double()), dim=1)


def _strip64(t, P):
    return torch.stack(t.chunk(P, dim=1))


def _pull_back(z, act, dy):
    """Gradient of sum(act(z) * dy) with respect to z."""
    with torch.enable_grad():
        z = z.clone().requires_grad_(True)
        (dz,) = torch.autograd.grad(_DEFINED[act](z), z, dy)
    return dz


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "moe":
        T, E, k, I = case["T"], case["E"], case["topk"], case["I"]
        x = s["x"].double()
        logits = torch.nn.functional.linear(x, s["router"].double())
        prob = torch.softmax(logits, dim=1)
        chosen = torch.zeros(T, E, dtype=torch.bool, device="cuda")
        left = prob.clone()
        for _ in range(k):
            best = left.max(1, keepdim=True).values
            first = (left == best).to(torch.int8).argmax(1, keepdim=True)
            chosen.scatter_(1, first, True)
            left.scatter_(1, first, -1.0)
        weight = torch.where(chosen, prob, torch.zeros_like(prob))
        if case["norm"]:
            weight = weight / weight.sum(1, keepdim=True)
        y = s["residual"].double() if s["residual"] is not None else torch.zeros_like(x)
        for e in range(E):
            t = chosen[:, e].nonzero()[:, 0]
            if t.numel():
                gate, up = torch.nn.functional.linear(x[t], s["w_gu"][e].double()).split(I, dim=1)
                out = torch.nn.functional.linear(torch.nn.functional.silu(gate) * up, s["w_down"][e].double())
                y[t] += weight[t, e, None] * out
        return {"y": y}
    if case["op"] == "bias_grad":
        dy = s["dy"].double()
        if s["z"] is None:
            return {"dbias": dy.sum(0)}
        dz = _pull_back(s["z"].double(), case["act"], dy)
        return {"dz": dz, "dbias": dz.sum(0)}
    product = torch.matmul(s["a"].double(), _weight64(s))
    if case["op"] == "act_grad":
        dz = _pull_back(_unstrip64(s["z"]), case["act"], product)
        out = {"dz": _strip64(dz, case["P"])}
        if case["dbias"]:
            out["dbias"] = dz.sum(0)
        return out
    if s["bias"] is not None:
        product += s["bias"].double()
    c = _DEFINED[case["act"]](product)
    if s["residual"] is not None:
        c = c + _unstrip64(s["residual"])
    out = {"c": _strip64(c, case["P"])}
    if case["preact"]:
        out["z"] = _strip64(product, case["P"])
    return out
