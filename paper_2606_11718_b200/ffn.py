"""The feed-forward operators put together as a program would use them.

``Block``  a feed-forward block  y = x + act(x W1 + b1) W2 + b2  with its forward and backward pass: every bias, activation, slope
           and residual is in the epilogue of a GEMM; weights and inner activations are kept in CCL strips.
``MoeLayer``  a mixture-of-experts layer for decode steps of a few tokens, one launch a step.

``python -m paper_2606_11718_b200.ffn`` times a training step of the first and decode steps of the second.
"""
import argparse

import torch

from . import binding as ccl

BF16 = torch.bfloat16


def _buffer(m):
    return torch.empty(ccl.ccl_buffer_bytes(m) // 2, dtype=BF16, device="cuda")


class Block:
    """y = x + act(x W1 + b1) W2 + b2 for `tokens` rows; W1 [H x I] and W2 [I x H] row-major bfloat16.  With strips > 1 W1, the inner
    activation and its gradient are stored in that many column strips (I / strips a multiple of 64).  The inner activations of the last
    forward pass and the workspace are kept in the object: its calls go to one stream, or wait for each other."""

    def __init__(self, w1, b1, w2, b2, tokens, act=ccl.ACT_GELU_TANH, strips=1):
        H, I = w1.shape
        T, P = tokens, strips
        if P > 1 and I % (64 * P):
            raise ValueError("Block: the inner width must be a multiple of 64 * strips")
        self.T, self.H, self.I, self.act = T, H, I, act
        inner = (P, ccl.PART_COLS, ccl.CCL, 0) if P > 1 else (1, ccl.PART_NONE, ccl.ROWMAJOR, 0)
        x, h, w1m, w2m = ccl.Mat(T, H, 2), ccl.Mat(T, I, 2, *inner), ccl.Mat(H, I, 2, *inner), ccl.Mat(I, H, 2)
        self.b1, self.b2, self.w2 = b1, b2, w2.contiguous()
        self.w1 = _buffer(w1m)
        ccl.ccl_repack(w1m, w1.contiguous(), self.w1)

        def desc(M, N, K, A, B, C, at=0, bt=0, part=ccl.PART_NONE):
            d = ccl.GemmDesc()
            d.M, d.N, d.K, d.A, d.B, d.C = M, N, K, A, B, C
            d.a_trans, d.b_trans, d.out_part, d.P, d.grouped_raster = at, bt, part if P > 1 else ccl.PART_NONE, P, int(P > 1)
            return d

        self.up = desc(T, I, H, x, w1m, h, part=ccl.PART_COLS)                        # z = x W1 + b1, h = act(z)
        self.down = desc(T, H, I, h, w2m, x)                                          # y = h W2 + b2 + x
        self.d_inner = desc(T, I, H, x, w2m, h, bt=1, part=ccl.PART_COLS)             # dz = (dy W2^T) * act'(z), db1
        self.d_x = desc(T, H, I, h, w1m, x, bt=1)                                     # dx = dz W1^T + dy
        self.d_w1 = desc(H, I, T, x, h, w1m, at=1, part=ccl.PART_COLS)                # dW1 = x^T dz
        self.d_w2 = desc(I, H, T, h, x, w2m, at=1)                                    # dW2 = h^T dy
        self.x_mat, self.w1_mat = x, w1m
        self.z, self.h, self.dz = _buffer(h), _buffer(h), _buffer(h)
        need = max(ccl.ccl_gemm_epilogue_workspace(self.up), ccl.ccl_gemm_epilogue_workspace(self.down), ccl.ccl_gemm_epilogue_workspace(self.d_x),
                   ccl.ccl_gemm_act_grad_workspace(self.d_inner), ccl.ccl_gemm_workspace(self.d_w1), ccl.ccl_gemm_workspace(self.d_w2))
        self.ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")

    def forward(self, x, y=None):
        """x, y: [tokens x H] row-major; y may be x (the residual stream updated in place, when no gradient is wanted)."""
        y = torch.empty_like(x) if y is None else y
        ccl.ccl_gemm_epilogue(self.up, x, self.w1, self.h, self.ws, act=self.act, bias=self.b1, preact=self.z)
        ccl.ccl_gemm_epilogue(self.down, self.h, self.w2, y, self.ws, bias=self.b2, residual=x)
        return y

    def backward(self, x, dy):
        """Gradients of the last forward pass: dx [tokens x H], dw1 (row-major), db1, dw2, db2."""
        dx, dw1_strips, dw2 = torch.empty_like(x), _buffer(self.w1_mat), torch.empty_like(self.w2)
        db1, db2 = torch.empty_like(self.b1), torch.empty_like(self.b2)
        ccl.ccl_bias_act_grad(self.x_mat, dy, None, None, db2)
        ccl.ccl_gemm_act_grad(self.d_inner, dy, self.w2, self.z, self.dz, self.ws, act=self.act, dbias=db1)
        ccl.ccl_gemm(self.d_w2, self.h, dy, dw2, self.ws)
        ccl.ccl_gemm(self.d_w1, x, self.dz, dw1_strips, self.ws)
        ccl.ccl_gemm_epilogue(self.d_x, self.dz, self.w1, dx, self.ws, residual=dy)
        dw1 = torch.empty(self.H, self.I, dtype=BF16, device="cuda")
        ccl.ccl_repack(self.w1_mat, dw1_strips, dw1, 1)
        return {"dx": dx, "dw1": dw1, "db1": db1, "dw2": dw2, "db2": db2}


class MoeLayer:
    """Decode steps through a mixture-of-experts layer: router [E x H], w_gu [E x 2I x H] (gate rows, then up rows), w_down [E x H x I].
    Steps on different streams may overlap: each has a workspace of its own, from torch's allocator for its stream."""

    def __init__(self, router, w_gu, w_down, topk, norm_topk=True):
        self.weights = (router, w_gu, w_down)
        self.E, self.H = router.shape
        self.I, self.topk, self.norm = w_down.shape[2], topk, int(norm_topk)
        self.plans = {}                                                               # tokens -> descriptor, bytes of workspace

    def step(self, x, out=None):
        """out = x + layer(x) for x [T x H], T <= 64; out may be x."""
        T = x.shape[0]
        if T not in self.plans:
            d = ccl.MoeDesc(T, self.E, self.topk, self.H, self.I, norm_topk=self.norm)
            self.plans[T] = d, ccl.ccl_moe_tokens_workspace(d)
        d, ws_bytes = self.plans[T]
        ws = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda")
        out = torch.empty_like(x) if out is None else out
        ccl.ccl_moe_tokens(d, x, *self.weights, out, ws, residual=x)
        return out


def _ms(fn, reps):
    for _ in range(3):
        fn()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda.synchronize()
    a.record()
    for _ in range(reps):
        fn()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b) / reps


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--inner", type=int, default=8192)
    ap.add_argument("--strips", type=int, default=4)
    ap.add_argument("--experts", type=int, default=128)
    ap.add_argument("--topk", type=int, default=8)
    ap.add_argument("--expert-inner", type=int, default=768)
    args = ap.parse_args()
    T, H, I = args.tokens, args.hidden, args.inner

    def normal(*shape, std=1.0):
        return torch.randn(*shape, device="cuda", dtype=BF16).mul_(std)

    block = Block(normal(H, I, std=0.02), normal(I, std=0.02), normal(I, H, std=0.02), normal(H, std=0.02), T, strips=args.strips)
    x, dy = normal(T, H), normal(T, H)
    fwd = _ms(lambda: block.forward(x), 20)
    both = _ms(lambda: (block.forward(x), block.backward(x, dy)), 20)
    flops = 4.0 * T * H * I
    print(f"block {T} tokens, {H} -> {I} -> {H}, {args.strips} strips: forward {fwd * 1e3:.0f} us ({flops / fwd / 1e9:.0f} TFLOP/s), "
          f"forward and backward {both * 1e3:.0f} us ({3 * flops / both / 1e9:.0f} TFLOP/s)")
    E, Ie = args.experts, args.expert_inner
    layer = MoeLayer(normal(E, H, std=0.02), normal(E, 2 * Ie, H, std=0.02), normal(E, H, Ie, std=0.02), args.topk)
    for tokens in (1, 4, 16, 64):
        xs = [normal(tokens, H) for _ in range(8)]
        turn = iter(range(1 << 30))
        ms = _ms(lambda: layer.step(xs[next(turn) % 8]), 40)
        print(f"mixture of experts, {tokens} token(s), {args.topk} of {E} experts of {H} x {Ie}: {ms * 1e3:.1f} us a step")
    status, detail = ccl.ccl_gemm_status()
    assert status == ccl.OK, detail


if __name__ == "__main__":
    main()
