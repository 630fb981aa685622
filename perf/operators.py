"""The operators of 8-bit layers and of what stands around a layer, as cases that can be timed and compared.

Four kinds of work, all through the package's public entry points:
  rows      rows of activations (or of weights) to 8 bits with a scale each, qtip_quantize_rows_i8: as they are,
            gated (silu(x) .* up), or after the random Hadamard transform;
  matmul    the product of 8-bit rows with 8-bit weights, a scale per token and per channel, qtip_matmul_i8;
  norm      what stands between two blocks, qtip_norm_residual: the norm behind a block, its gate, the residual's scale
            and sum, the norm in front of the next block, its result in 16 or 32 bits, rotated, or in 8 bits;
  moe       a mixture-of-experts layer for a few tokens, qtip_moe_i8: router, choice, experts in 8-bit weights, sum.

Where `own` is false, the same in elementary torch operations in 32 bits.
"""
import math
from types import SimpleNamespace

import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"f16": 2, "bf16": 2, "f32": 4, "i8": 1}
MAX_ROWS = 4096 * 8192             # values of a case of rows or norm
MAX_PRODUCT = 8192 * 28672 * 4096  # multiplications of a product
MAX_WEIGHTS = 8192 * 28672
MAX_EXPERTS = 8 * 3 * 14336 * 4096 // 2  # bytes of all experts of a drawn layer


def rows(name, T, n, dtype, gated=False, block=0):
    case = {"kind": "rows", "T": T, "n": n, "dtype": dtype, "gated": gated, "block": block}
    return {"name": name} | case if name else case


def matmul(name, m, n, B, out, bias=False):
    case = {"kind": "matmul", "m": m, "n": n, "B": B, "out": out, "bias": bias}
    return {"name": name} | case if name else case


def norm(name, T, n, y_type, h_type, out, layer=False, post=True, gate="none", block=0):
    case = {"kind": "norm", "T": T, "n": n, "y_type": y_type, "h_type": h_type, "out": out, "layer": layer, "post": post,
            "gate": gate, "block": block}
    return {"name": name} | case if name else case


def moe(name, T, n, f, E, top_k, dtype):
    case = {"kind": "moe", "T": T, "n": n, "f": f, "E": E, "top_k": top_k, "dtype": dtype}
    return {"name": name} | case if name else case


def listed():
    return [
        # one token's activations in front of an 8-bit layer of the benchmark's width, rotated: latency
        rows("rows_1x28672_f16_rht4096", 1, 28672, "f16", block=4096),
        # a prompt of no round length between the two products of a gated feed-forward block
        rows("rows_997x14336_bf16_gated", 997, 14336, "bf16", gated=True),
        # an attention projection kept at 8 bits, generating token by token
        matmul("matmul_4096x4096_b1_f16", 4096, 4096, 1, "f16", bias=True),
        # the benchmark's feed-forward shape, sixteen sequences generated together: the weights' bytes count
        matmul("matmul_8192x28672_b16_f32", 8192, 28672, 16, "f32"),
        # a prompt of no round length
        matmul("matmul_14336x4096_b997_bf16", 14336, 4096, 997, "bf16"),
        # a batch of long prompts: the matrix cores count
        matmul("matmul_8192x28672_b4096_bf16", 8192, 28672, 4096, "bf16"),
        # between two blocks while generating one token, the result rotated for a trellis-coded layer: latency
        norm("norm_1x4096_f16_rht4096", 1, 4096, "f16", "f16", "f16", post=False, block=4096),
        # norms behind and in front of a block with a gate of its own per token, the result in 8 bits, a long prompt
        norm("norm_4096x8192_bf16_gate_i8", 4096, 8192, "bf16", "bf16", "i8", gate="rows"),
        # layer norms of a width that divides into nothing, residual stream in 32 bits, one scale per channel
        norm("norm_997x5003_f32_layer", 997, 5003, "bf16", "f32", "bf16", layer=True, gate="channels"),
        # few large experts, one token: two experts' weights
        moe("moe_t1_8x14336x4096_top2_bf16", 1, 4096, 14336, 8, 2, "bf16"),
        # many small experts, sixteen sequences generated together: most experts have a token or two
        moe("moe_t16_64x1024x2048_top8_f16", 16, 2048, 1024, 64, 8, "f16"),
        # as many tokens as the layer takes at once, every expert has several
        moe("moe_t64_32x2048x4096_top4_bf16", 64, 4096, 2048, 32, 4, "bf16"),
    ]


def spread(rng, low, high):
    """A whole number whose logarithm is uniform."""
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    case = drawn(rng)
    while 3072 in case.values():  # (a size that nothing else here has)
        case = drawn(rng)
    return case


def drawn(rng):
    kind = rng.choice(["rows", "matmul", "norm", "moe"])
    if kind == "rows":
        if rng.random() < 0.5:
            block = 1 << rng.randint(4, 13)
            n = block * spread(rng, 1, 28672 // block)
        else:
            block, n = 0, spread(rng, 64, 28672)
        return rows(None, spread(rng, 1, MAX_ROWS // 2 // n), n, rng.choice(["f16", "bf16", "f32"]), rng.random() < 0.4, block)
    if kind == "matmul":
        m, n = spread(rng, 64, 28672), spread(rng, 64, 28672)
        if rng.random() < 0.5:
            m, n = -(-m // 16) * 16, -(-n // 64) * 64
        n = min(n, MAX_WEIGHTS // m)
        return matmul(None, m, n, spread(rng, 1, 4096), rng.choice(["f16", "bf16", "f32"]), rng.random() < 0.5)
    if kind == "norm":
        if rng.random() < 0.4:
            block = 1 << rng.randint(4, 13)
            n = block * spread(rng, 1, 28672 // block)
        else:
            block, n = 0, spread(rng, 64, 28672)
        y_type = rng.choice(["f16", "bf16", "f32"])
        return norm(None, spread(rng, 1, MAX_ROWS // 2 // n), n, y_type, rng.choice([y_type, "f32"]),
                    rng.choice(["i8", "f16", "bf16"]), rng.random() < 0.4, rng.random() < 0.5,
                    rng.choice(["none", "rows", "channels"]), block)
    E = spread(rng, 4, 128)
    n, f = 16 * spread(rng, 16, 512), 16 * spread(rng, 8, 512)
    while 3 * E * n * f > MAX_EXPERTS:
        n, f = max(256, n // 32 * 16), max(128, f // 32 * 16)
    return moe(None, spread(rng, 1, 64), n, f, E, rng.randint(1, min(8, E)), rng.choice(["f16", "bf16"]))


def work(case):
    c = SimpleNamespace(**case)
    if c.kind == "rows":
        return {"bytes": c.T * c.n * (BYTES[c.dtype] * (2 if c.gated else 1) + 1) + 4 * c.T + (c.n if c.block else 0),
                "flops": c.T * c.n * (3 + (6 if c.gated else 0) + (math.log2(c.block) + 1 if c.block else 0))}
    if c.kind == "matmul":
        return {"bytes": c.m * c.n + c.B * c.n + 4 * c.m * (2 if c.bias else 1) + 4 * c.B + c.B * c.m * BYTES[c.out],
                "flops": 2 * c.m * c.n * c.B}
    if c.kind == "norm":
        per = BYTES[c.y_type] * (2 if c.gate == "rows" else 1) + 2 * BYTES[c.h_type] + BYTES[c.out]
        vectors = 4 * ((2 if c.layer else 1) * (2 if c.post else 1)) + (BYTES[c.y_type] if c.gate == "channels" else 0)
        return {"bytes": c.T * c.n * per + c.n * (vectors + (1 if c.block else 0)) + (4 * c.T if c.out == "i8" else 0),
                "flops": c.T * c.n * (6 + (4 if c.post else 0) + (math.log2(c.block) + 1 if c.block else 0))}
    # each chosen expert is read once: as many as T tokens choose on average where all are equally likely
    experts = c.E * (1 - (1 - c.top_k / c.E) ** c.T)
    return {"bytes": experts * (3 * c.f * c.n + 4 * (2 * c.f + c.n)) + c.E * c.n * BYTES[c.dtype] + 2 * c.T * c.n * BYTES[c.dtype]
            + 8 * c.T * c.top_k, "flops": 6 * c.T * c.top_k * c.f * c.n + 2 * c.T * c.E * c.n}


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def signs_of(g, n):
    return (torch.randint(0, 2, (n,), device="cuda", generator=g) * 2 - 1).to(torch.int8)


def sylvester(block, dtype):
    H = torch.ones(1, 1, dtype=dtype, device="cuda")
    while H.shape[0] < block:
        H = torch.cat((torch.cat((H, H), 1), torch.cat((H, -H), 1)), 0)
    return H


def padded(v):
    return -(-v // 16) * 16


def activations(g, T, n):
    """Rows as a model has them: a few channels are much larger than the others."""
    x = normal(g, T, n)
    return x * (1 + 20 * (torch.rand(n, device="cuda", generator=g) < 0.005))


def prepare(case, seed):
    c = SimpleNamespace(**case)
    g = generator(seed)
    s = SimpleNamespace(c=c)
    if own:
        import paper_2406_11235_amd as q
        s.q, s.type = q, {"f16": q.F16, "bf16": q.BF16, "f32": q.F32, "i8": q.I8}
    if c.kind == "rows":
        s.x = activations(g, c.T, c.n).to(TYPES[c.dtype])
        s.up = normal(g, c.T, c.n).to(TYPES[c.dtype]) if c.gated else None
        s.signs = signs_of(g, c.n) if c.block else None
        s.H = sylvester(c.block, torch.float32) if c.block else None
        s.xq = torch.empty(c.T, padded(c.n), dtype=torch.int8, device="cuda")
        s.scale = torch.empty(c.T, device="cuda")
        s.values = torch.empty(c.T, c.n, dtype=torch.float16, device="cuda")
    elif c.kind == "matmul":
        # weights and activations as the row quantizer leaves them: the largest of a row is 127 (what stands between a
        # row's end and the next row's begin is anything)
        s.ld = padded(c.n)
        s.W = torch.randint(-127, 128, (c.m, s.ld), device="cuda", generator=g, dtype=torch.int8)
        s.w_scale = 0.02 / 127 * (1 + torch.rand(c.m, device="cuda", generator=g))
        s.X = (normal(g, c.B, s.ld) * 32).clamp_(-127, 127).round_().to(torch.int8)
        s.x_scale = 4 / 127 * (0.5 + torch.rand(c.B, device="cuda", generator=g))
        s.bias = normal(g, c.m) if c.bias else None
        s.Y = torch.empty(c.B, c.m, dtype=TYPES[c.out], device="cuda")
        if own:
            s.ws = torch.empty(max(1, s.q.qtip_matmul_i8_workspace(c.m, c.n, c.B)), dtype=torch.uint8, device="cuda")
    elif c.kind == "norm":
        s.y = activations(g, c.T, c.n).to(TYPES[c.y_type])
        s.h = (3 * activations(g, c.T, c.n)).to(TYPES[c.h_type])
        s.gate = {"none": None, "rows": torch.rand(c.T, c.n, device="cuda", generator=g),
                  "channels": normal(g, c.n) * 0.3}[c.gate]
        s.gate = None if s.gate is None else s.gate.to(TYPES[c.y_type])
        s.post = 1 + 0.2 * normal(g, c.n) if c.post else None
        s.post_bias = 0.1 * normal(g, c.n) if c.post and c.layer else None
        s.pre = 1 + 0.2 * normal(g, c.n)
        s.pre_bias = 0.1 * normal(g, c.n) if c.layer else None
        s.signs = signs_of(g, c.n) if c.block else None
        s.H = sylvester(c.block, torch.float32) if c.block else None
        s.eps, s.res_scale = 1e-5, 0.7
        s.h_out = torch.empty_like(s.h)
        s.ld = padded(c.n) if c.out == "i8" else c.n
        s.x = torch.empty(c.T, s.ld, dtype=torch.int8 if c.out == "i8" else TYPES[c.out], device="cuda")
        s.scale = torch.empty(c.T, device="cuda") if c.out == "i8" else None
        s.values = torch.empty(c.T, c.n, dtype=torch.float16, device="cuda") if c.out == "i8" else None
    else:
        dt = TYPES[c.dtype]
        s.x = activations(g, c.T, c.n).to(dt)
        s.router = (normal(g, c.E, c.n) / math.sqrt(c.n)).to(dt)
        s.W_up = torch.randint(-127, 128, (c.E, 2 * c.f, c.n), device="cuda", generator=g, dtype=torch.int8)
        s.up_scale = (1 + torch.rand(c.E, 2 * c.f, device="cuda", generator=g)) / (100 * math.sqrt(c.n))
        s.W_down = torch.randint(-127, 128, (c.E, c.n, c.f), device="cuda", generator=g, dtype=torch.int8)
        s.down_scale = (1 + torch.rand(c.E, c.n, device="cuda", generator=g)) / (100 * math.sqrt(c.f))
        s.y = torch.empty(c.T, c.n, dtype=dt, device="cuda")
        s.ids = torch.empty(c.T, c.top_k, dtype=torch.int32, device="cuda")
        s.weights = torch.empty(c.T, c.top_k, device="cuda")
        if own:
            s.ws = torch.empty(s.q.qtip_moe_i8_workspace(c.T, c.n, c.f, c.E, c.top_k), dtype=torch.uint8, device="cuda")
    return s


def run(s):
    return (run_own if own else run_plain)(s)


def run_own(s):
    c, q, t = s.c, s.q, s.type
    if c.kind == "rows":
        q.qtip_quantize_rows_i8(s.x, s.up, t[c.dtype], c.T, c.n, c.n, s.signs, c.block, s.xq, padded(c.n), s.scale)
        torch.mul(s.xq[:, :c.n], s.scale[:, None], out=s.values)
        return {"values": s.values, "scale": s.scale}
    if c.kind == "matmul":
        q.qtip_matmul_i8(s.W, s.ld, s.w_scale, c.m, c.n, s.X, s.ld, s.x_scale, c.B, s.bias, s.Y, c.m, t[c.out], s.ws, s.ws.numel())
        return {"Y": s.Y}
    if c.kind == "norm":
        q.qtip_norm_residual(s.y, c.n, t[c.y_type], s.h, c.n, t[c.h_type], s.gate, c.n if c.gate == "rows" else 0, c.T, c.n,
                             q.NORM_LAYER if c.layer else q.NORM_RMS, s.post, s.post_bias, s.pre, s.pre_bias, s.eps,
                             s.res_scale, s.signs, c.block, s.h_out, s.x, s.ld, t[c.out], s.scale)
        if c.out == "i8":
            torch.mul(s.x[:, :c.n], s.scale[:, None], out=s.values)
            return {"h": s.h_out, "values": s.values, "scale": s.scale}
        return {"h": s.h_out, "x": s.x}
    q.qtip_moe_i8(s.x, c.n, t[c.dtype], c.T, c.n, s.router, None, c.E, c.top_k, 1, s.W_up, s.up_scale, c.f, s.W_down,
                  s.down_scale, s.y, c.n, s.ids, s.weights, s.ws, s.ws.numel())
    return {"y": s.y, "ids": s.ids, "weights": s.weights}


def rotated(v, signs, H, block):
    T, n = v.shape
    return ((v * signs).view(-1, block) @ H).view(T, n) * (1 / math.sqrt(block))


def to_8_bits(v):
    a = v.abs().amax(dim=1, keepdim=True)
    scale = a / 127
    return (v * (127 / a)).round() * scale, scale[:, 0]


def normed(v, layer, eps, weight, bias):
    if layer:
        v = v - v.mean(dim=1, keepdim=True)
    v = v * torch.rsqrt(v.square().mean(dim=1, keepdim=True) + eps) * weight
    return v if bias is None else v + bias


def run_plain(s):
    c = s.c
    if c.kind == "rows":
        v = s.x.float()
        if c.gated:
            v = v * torch.sigmoid(v) * s.up.float()
        if c.block:
            v = rotated(v, s.signs.float(), s.H, c.block)
        values, scale = to_8_bits(v)
        return {"values": values.half(), "scale": scale}
    if c.kind == "matmul":
        Y = s.X[:, :c.n].float() @ s.W[:, :c.n].float().t() * s.x_scale[:, None] * s.w_scale
        return {"Y": (Y if s.bias is None else Y + s.bias).to(TYPES[c.out])}
    if c.kind == "norm":
        a = s.y.float()
        if c.post:
            a = normed(a, c.layer, s.eps, s.post, s.post_bias)
        if s.gate is not None:
            a = a * s.gate.float()
        h = s.h.float() + s.res_scale * a
        x = normed(h, c.layer, s.eps, s.pre, s.pre_bias)
        if c.block:
            x = rotated(x, s.signs.float(), s.H, c.block)
        h = h.to(TYPES[c.h_type])
        if c.out == "i8":
            values, scale = to_8_bits(x)
            return {"h": h, "values": values.half(), "scale": scale}
        return {"h": h, "x": x.to(TYPES[c.out])}
    x = s.x.float()
    logits = x @ s.router.float().t()
    best, ids = torch.sort(logits, dim=1, descending=True, stable=True)
    ids = ids[:, :c.top_k]
    weights = torch.softmax(best[:, :c.top_k], dim=1)
    if c.T * c.top_k <= c.E:  # the chosen experts' weights alone, one product for each
        at = ids.reshape(-1)
        z = (s.W_up[at].float() @ x.repeat_interleave(c.top_k, dim=0)[:, :, None])[:, :, 0] * s.up_scale[at]
        h = z[:, :c.f] * torch.sigmoid(z[:, :c.f]) * z[:, c.f:]
        out = (s.W_down[at].float() @ h[:, :, None])[:, :, 0] * s.down_scale[at]
        y = (out.view(c.T, c.top_k, c.n) * weights[:, :, None]).sum(dim=1)
    else:  # all experts for all tokens, and those that count
        z = (s.W_up.float() @ x.t()) * s.up_scale[:, :, None]
        h = z[:, :c.f] * torch.sigmoid(z[:, :c.f]) * z[:, c.f:]
        out = (s.W_down.float() @ h) * s.down_scale[:, :, None]
        share = torch.zeros(c.T, c.E, device="cuda").scatter_(1, ids, weights)
        y = (out * share.t()[:, None, :]).sum(dim=0).t().contiguous()
    return {"y": y.to(TYPES[c.dtype]), "ids": ids.int(), "weights": weights}


def exact(case, seed):
    """From the definitions, in 64 bits."""
    s = prepare(case, seed)
    c, d = s.c, torch.float64

    def transform(v):
        H = sylvester(c.block, d)
        v = v * s.signs.to(d)
        for at in range(0, c.n, c.block):
            v[:, at:at + c.block] = v[:, at:at + c.block] @ H / math.sqrt(c.block)
        return v

    def eight_bits(v):
        scale = v.abs().max(dim=1).values / 127
        return torch.round(v / scale[:, None]) * scale[:, None], scale

    def statistics(v):
        mean = v.sum(dim=1, keepdim=True) / c.n if c.layer else torch.zeros(c.T, 1, dtype=d, device="cuda")
        return mean, ((v - mean) ** 2).sum(dim=1, keepdim=True) / c.n

    def affine(v, weight, bias):
        mean, var = statistics(v)
        v = (v - mean) / (var + s.eps).sqrt() * weight.to(d)
        return v + bias.to(d) if bias is not None else v

    if c.kind == "rows":
        v = s.x.to(d)
        if c.gated:
            v = v / (1 + torch.exp(-v)) * s.up.to(d)
        values, scale = eight_bits(transform(v) if c.block else v)
        return {"values": values, "scale": scale}
    if c.kind == "matmul":
        Y = torch.empty(c.B, c.m, dtype=d, device="cuda")
        X = s.X[:, :c.n].to(d)
        for at in range(0, c.m, 4096):
            Y[:, at:at + 4096] = X @ s.W[at:at + 4096, :c.n].to(d).t().contiguous()
        Y = Y * (s.x_scale.to(d)[:, None] * s.w_scale.to(d)[None, :])
        return {"Y": Y + s.bias.to(d) if c.bias else Y}
    if c.kind == "norm":
        a = affine(s.y.to(d), s.post, s.post_bias) if c.post else s.y.to(d)
        h = s.h.to(d) + s.res_scale * (a * s.gate.to(d) if c.gate != "none" else a)
        x = affine(h, s.pre, s.pre_bias)
        x = transform(x) if c.block else x
        if c.out == "i8":
            values, scale = eight_bits(x)
            return {"h": h, "values": values, "scale": scale}
        return {"h": h, "x": x}
    x = s.x.to(d)
    logits = x @ s.router.to(d).t().contiguous()
    ids = torch.argsort(logits, dim=1, descending=True, stable=True)[:, :c.top_k]
    e = torch.exp(logits - logits.max(dim=1, keepdim=True).values)
    weights = e.gather(1, ids)
    weights = weights / weights.sum(dim=1, keepdim=True)
    y = torch.zeros(c.T, c.n, dtype=d, device="cuda")
    for expert in torch.unique(ids).tolist():
        token, slot = torch.nonzero(ids == expert, as_tuple=True)
        z = x[token] @ (s.W_up[expert].to(d) * s.up_scale[expert].to(d)[:, None]).t().contiguous()
        gate, up = z[:, :c.f], z[:, c.f:]
        h = gate / (1 + torch.exp(-gate)) * up
        out = h @ (s.W_down[expert].to(d) * s.down_scale[expert].to(d)[:, None]).t().contiguous()
        y[token] += out * weights[token, slot][:, None]
    return {"y": y, "ids": ids.int(), "weights": weights}
