"""A decoder's blocks around their layers, as they run while a few sequences are generated, on one MI355X:

    python -m paper_2406_11235_amd.example_layers [tokens n f experts]

1. a feed-forward block in 8 bits: norm, rotation and 8-bit rows in one launch; gate and up in one product; silu(gate) .* up,
   rotation and 8-bit rows in one launch; down;
2. what stands between that block and the next one in one launch: the norm behind the block, its gate, the residual's
   scale and sum, the norm in front of the next block;
3. a mixture-of-experts layer with 8-bit experts;
4. the same between it and a trellis-coded layer, the result rotated for that layer, and the layer itself.
The rows of all 8-bit weights are made by the row quantizer too.  Weights are i.i.d. Gaussian; torch is used for memory and
for the dense check in 64 bits only.
"""
import math
import sys

import torch

from . import (BF16, CODE_3INST, F16, F32, I8, NORM_RMS, qtip_decode_matmat, qtip_dequantize, qtip_matmul_i8,
               qtip_matmul_i8_workspace, qtip_moe_i8, qtip_moe_i8_workspace, qtip_norm_residual, qtip_quantize_rows_i8)


def largest_pow2_divisor(v, cap=16384):
    return min(cap, v & -v)


class Rows8:
    """A matrix as 8-bit rows with a scale each."""

    def __init__(self, rows, n):
        self.n, self.ld = n, -(-n // 16) * 16
        self.q = torch.empty(rows, self.ld, dtype=torch.int8, device="cuda")
        self.scale = torch.empty(rows, device="cuda")

    def of(self, W, signs=None, block=0):
        qtip_quantize_rows_i8(W, None, F32, W.shape[0], self.n, self.n, signs, block, self.q, self.ld, self.scale)
        return self

    def values(self):
        return self.q[:, :self.n].double() * self.scale.double()[:, None]


def main(tokens=5, n=1024, f=2048, experts=8, top_k=2, seed=0):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, device=dev, generator=g)
    signs = lambda length: (torch.randint(0, 2, (length,), device=dev, generator=g) * 2 - 1).to(torch.int8)
    vector = lambda: 1 + 0.1 * normal(n)
    eps, half = 1e-6, dict(dtype=torch.bfloat16, device=dev)

    # ---- what a model keeps
    bn, bf = largest_pow2_divisor(n), largest_pow2_divisor(f)
    sn, sf, st = signs(n), signs(f), signs(n)
    W_up, W_down = normal(2 * f, n) / math.sqrt(n), normal(n, f) / math.sqrt(f)
    up, down = Rows8(2 * f, n).of(W_up, sn, bn), Rows8(n, f).of(W_down, sf, bf)
    E_up = Rows8(experts * 2 * f, n).of(normal(experts * 2 * f, n) / math.sqrt(n))
    E_down = Rows8(experts * n, f).of(normal(experts * n, f) / math.sqrt(f))
    router = (normal(experts, n) / math.sqrt(n)).bfloat16()
    w_first, w_post, w_pre, w_post2, w_pre2 = (vector() for _ in range(5))
    m = 512  # the trellis-coded layer: random streams stand for a rotated matrix
    codes = torch.randint(-2 ** 31, 2 ** 31 - 1, ((m // 16) * (n // 16) * 16,), dtype=torch.int32, device=dev, generator=g)

    # ---- the tokens, and room for what passes between the calls
    h = normal(tokens, n).bfloat16()                        # the residual stream
    gate = torch.rand(tokens, n, device=dev, generator=g).bfloat16()
    x8, u8 = Rows8(tokens, n), Rows8(tokens, f)
    z, y, x = torch.empty(tokens, 2 * f, **half), torch.empty(tokens, n, **half), torch.empty(tokens, n, **half)
    h1, h2, y2 = torch.empty_like(h), torch.empty_like(h), torch.empty(tokens, n, **half)
    xt = torch.empty(tokens, n, dtype=torch.float16, device=dev)
    out = torch.empty(tokens, m, device=dev)
    ids = torch.empty(tokens, top_k, dtype=torch.int32, device=dev)
    weights = torch.empty(tokens, top_k, device=dev)
    room = max(qtip_matmul_i8_workspace(2 * f, n, tokens), qtip_matmul_i8_workspace(n, f, tokens),
               qtip_moe_i8_workspace(tokens, n, f, experts, top_k))
    ws = torch.empty(room, dtype=torch.uint8, device=dev)

    # 1. x8 = rows8(V_n S_n norm(h)); z = [gate; up]; u8 = rows8(V_f S_f (silu(gate) .* up)); y = down
    qtip_norm_residual(None, n, BF16, h, n, BF16, None, 0, tokens, n, NORM_RMS, None, None, w_first, None, eps, 1.0, sn, bn, None,
                       x8.q, x8.ld, I8, x8.scale)
    qtip_matmul_i8(up.q, up.ld, up.scale, 2 * f, n, x8.q, x8.ld, x8.scale, tokens, None, z, 2 * f, BF16, ws, ws.numel())
    qtip_quantize_rows_i8(z, z[:, f:].data_ptr(), BF16, tokens, f, 2 * f, sf, bf, u8.q, u8.ld, u8.scale)
    qtip_matmul_i8(down.q, down.ld, down.scale, n, f, u8.q, u8.ld, u8.scale, tokens, None, y, n, BF16, ws, ws.numel())
    # 2. h1 = h + 0.5 gate .* norm(y); x = norm(h1)
    qtip_norm_residual(y, n, BF16, h, n, BF16, gate, n, tokens, n, NORM_RMS, w_post, None, w_pre, None, eps, 0.5, None, 0, h1, x, n,
                       BF16, None)
    # 3. the experts
    qtip_moe_i8(x, n, BF16, tokens, n, router, None, experts, top_k, 1, E_up.q, E_up.scale, f, E_down.q, E_down.scale, y2, n, ids,
                weights, ws, ws.numel())
    # 4. h2 = h1 + 0.5 norm(y2); xt = V_n S_t norm(h2), for the trellis-coded layer
    qtip_norm_residual(y2, n, BF16, h1, n, BF16, None, 0, tokens, n, NORM_RMS, w_post2, None, w_pre2, None, eps, 0.5, st, bn, h2, xt,
                       n, F16, None)
    qtip_decode_matmat(codes, 16, 2, 1, CODE_3INST, None, m, n, xt, tokens, None, out)
    torch.cuda.synchronize()

    # ---- the same in 64 bits, from each step's own inputs (dense weights, no rotation: it cancels)
    norm = lambda v, w: v / (v.square().mean(dim=1, keepdim=True) + eps).sqrt() * w.double()
    silu = lambda v: v / (1 + torch.exp(-v))

    def far(got, want):
        return float((got.double() - want).norm() / want.norm())

    zd = norm(h.double(), w_first) @ W_up.double().t().contiguous()
    checks = {"gate and up, 8 bits": (far(z, zd), 0.02)}
    yd = (silu(z[:, :f].double()) * z[:, f:].double()) @ W_down.double().t().contiguous()
    checks["down, 8 bits"] = (far(y, yd), 0.02)
    h1d = h.double() + 0.5 * gate.double() * norm(y.double(), w_post)
    checks["residual"] = (far(h1, h1d), 4e-3)
    checks["norm"] = (far(x, norm(h1d, w_pre)), 4e-3)
    y2d = torch.zeros(tokens, n, dtype=torch.float64, device=dev)
    Eu, Ed = E_up.values().view(experts, 2 * f, n), E_down.values().view(experts, n, f)
    for t in range(tokens):
        for j in range(top_k):
            zt = Eu[ids[t, j]] @ x[t].double()
            y2d[t] += float(weights[t, j]) * (Ed[ids[t, j]] @ (silu(zt[:f]) * zt[f:]))
    checks["experts"] = (far(y2, y2d), 4e-3)
    checks["residual behind the experts"] = (far(h2, h1.double() + 0.5 * norm(y2.double(), w_post2)), 4e-3)
    Wd = torch.empty(m, n, dtype=torch.float16, device=dev)
    qtip_dequantize(codes, 16, 2, 1, CODE_3INST, None, m, n, Wd)
    checks["trellis-coded layer"] = (far(out, xt.double() @ Wd.double().t().contiguous()), 1e-5)
    for name, (error, bar) in checks.items():
        print(f"{name}: relative error {error:.2e}")
        assert error < bar, (name, error)
    return checks


if __name__ == "__main__":
    main(*[int(a) for a in sys.argv[1:5]])
