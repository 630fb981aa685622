"""qtip_quantize_rows_i8 and qtip_norm_residual against plain 64-bit statements."""
import math

import pytest

from layers_util import EPS, EPS32, LEAST, TYPES, Rim, generator, normal, normed, rotate, signs_of, silu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2406_11235_amd as q
    q.lib()
    return q


def type_of(q, name):
    return {"f16": q.F16, "bf16": q.BF16, "f32": q.F32, "i8": q.I8}[name]


def check_i8(got, scale, want, error):
    """8-bit rows against 64-bit values that binary32 has to `error`: the scale is the largest's 127th part, and a
    value times 127 / largest is at most half a step off, but for its own error and that of three roundings."""
    import torch
    top = want.abs().amax(dim=1)
    top_error = error.amax(dim=1)
    assert bool(((scale.double() - top / 127).abs() <= top_error / 127 + 2 * EPS32 * top / 127).all())
    steps = want * (127 / top)[:, None]
    # (the largest's own error moves every step)
    slack = (error + want.abs() * (top_error / top)[:, None]) * (127 / top)[:, None] + 4 * EPS32 * 127
    off = (got.double() - steps).abs()
    assert bool((off <= 0.5 + slack).all()), float((off - slack).max())
    assert int(got.abs().max()) <= 127
    assert bool((got.abs().amax(dim=1) == 127).all())
    assert torch.isfinite(scale).all()


# n, rows, block (0: as it is), rows apart by n + pad values, values in front of the first row
SHAPES = [(1, 1, 0, 0, 0), (1, 3, 0, 5, 1), (2, 5, 0, 0, 0), (3, 2, 0, 1, 3), (63, 4, 0, 2, 0), (255, 3, 0, 0, 1), (1000, 7, 0, 0, 0),
          (1024, 3, 0, 0, 0), (1025, 2, 0, 0, 0), (2047, 3, 0, 1, 0), (4096, 2, 0, 0, 0), (4097, 2, 0, 3, 2), (5003, 3, 0, 0, 0),
          (8192, 2, 0, 0, 0), (8200, 600, 0, 0, 0), (14336, 3, 0, 0, 0), (16385, 2, 0, 0, 1), (28672, 1, 0, 0, 0),
          (32767, 2, 0, 0, 0), (32768, 1, 0, 0, 0),
          (16, 1, 16, 0, 0), (48, 3, 16, 8, 4), (96, 2, 32, 0, 0), (192, 2, 64, 0, 0), (384, 2, 128, 0, 0), (768, 3, 256, 0, 0),
          (1536, 2, 512, 0, 0), (1024, 700, 1024, 0, 0), (14336, 3, 2048, 0, 0), (28672, 2, 4096, 0, 0), (8192, 2, 8192, 0, 0),
          (24576, 2, 8192, 0, 0), (16384, 2, 16384, 0, 0), (32768, 2, 16384, 0, 0),
          # few long rows, rotated, that begin anywhere and end within a wave
          (20496, 3, 16, 1, 1), (20528, 3, 16, 1, 3), (28672, 40, 2048, 0, 0), (28672, 30, 1024, 5, 0), (18432, 2, 2048, 0, 1)]


@pytest.mark.parametrize("n,rows,block,pad,lead", SHAPES)
@pytest.mark.parametrize("dtype,gated", [("f16", False), ("bf16", True), ("f32", False), ("f32", True)])
def test_quantize_rows(q, n, rows, block, pad, lead, dtype, gated):
    import torch
    g = generator(n * 7 + rows)
    x = Rim(rows, n, TYPES[dtype], n + pad, lead).set(normal(g, rows, n) * torch.exp(normal(g, rows, 1)))
    up = Rim(rows, n, TYPES[dtype], n + pad, lead).set(normal(g, rows, n)) if gated else None
    signs = signs_of(g, n) if block else None
    out = Rim(rows, n, torch.int8, n + 2 * pad, lead)
    scale = Rim(1, rows, torch.float32, fill=-1.0)
    q.qtip_quantize_rows_i8(x.pointer, up.pointer if gated else None, type_of(q, dtype), rows, n, n + pad, signs, block,
                            out.pointer, n + 2 * pad, scale.pointer)
    torch.cuda.synchronize()
    v = x.view.double()
    error = torch.zeros_like(v)
    if gated:
        # exp(-v) from its argument's rounding and two units of the instruction, a sum, a division and two products
        error = (8 + v.abs()) * 2 * EPS32 * (silu(v) * up.view.double()).abs()
        v = silu(v) * up.view.double()
    if block:
        # a sum of `block` terms in log2(block) + a few steps, each rounding no more than the sum of magnitudes
        p = math.log2(block)
        weight = (v.abs().reshape(-1, block).sum(dim=1, keepdim=True) / math.sqrt(block))
        moved = error.reshape(-1, block).sum(dim=1, keepdim=True) / math.sqrt(block)
        error = ((2 * p + 8) * EPS32 * weight + moved).expand(-1, block).reshape(rows, n)
        v = rotate(v, signs, block)
    check_i8(out.view, scale.view[0], v, error)
    assert out.rim_is_whole() and scale.rim_is_whole()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_rows_that_have_no_scale(q, dtype):
    import torch
    n, inf = 500, float("inf")
    x = torch.zeros(8, n, dtype=TYPES[dtype], device="cuda")
    x[1, 7] = inf
    x[2, 499] = -inf
    x[3, 0] = float("nan")
    x[4] = torch.finfo(TYPES[dtype]).max
    x[5] = -torch.finfo(TYPES[dtype]).tiny
    x[6, 3] = torch.finfo(TYPES[dtype]).smallest_normal * 2 ** -6  # (below the smallest normal number)
    x[7, 1], x[7, 2] = inf, float("nan")
    out = torch.full((8, n), 9, dtype=torch.int8, device="cuda")
    scale = torch.full((8,), -1.0, device="cuda")
    q.qtip_quantize_rows_i8(x, None, type_of(q, dtype), 8, n, n, None, 0, out, n, scale)
    torch.cuda.synchronize()
    assert float(scale[0]) == 0 and int(out[0].abs().max()) == 0
    for row in (1, 2, 3, 7):
        assert math.isnan(float(scale[row])) and int(out[row].abs().max()) == 0
    assert bool((out[4] == 127).all()) and bool((out[5] == -127).all())
    assert float(scale[4]) == float((x[4, 0].double() / 127).float())  # (correctly rounded)
    assert int(out[6, 3]) == 127 and int(out[6].abs().sum()) == 127


def test_gated_by_halves_of_one_product(q):
    """up beside x in the same rows, as a product with stacked weights leaves them."""
    import torch
    g = generator(3)
    rows, n = 5, 1000
    both = normal(g, rows, 2 * n).bfloat16()
    out, scale = torch.empty(rows, n, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    q.qtip_quantize_rows_i8(both, both.data_ptr() + 2 * n, q.BF16, rows, n, 2 * n, None, 0, out, n, scale)
    x, up = both[:, :n].contiguous(), both[:, n:].contiguous()
    out2, scale2 = torch.empty_like(out), torch.empty_like(scale)
    q.qtip_quantize_rows_i8(x, up, q.BF16, rows, n, n, None, 0, out2, n, scale2)
    torch.cuda.synchronize()
    assert torch.equal(out, out2) and torch.equal(scale, scale2)


NORM_SHAPES = [(1, 1, 0, 0), (3, 2, 0, 1), (77, 4, 0, 3), (1000, 5, 0, 0), (1024, 3, 0, 0), (2050, 3, 0, 0), (4096, 2, 0, 0),
               (5003, 3, 0, 0), (8192, 700, 0, 0), (12000, 2, 0, 1), (28672, 1, 0, 0), (32768, 2, 0, 0), (32767, 1, 0, 0),
               (16, 2, 16, 0), (1000 * 16, 2, 128, 4), (4096, 1, 4096, 0), (28672, 2, 4096, 0), (16384, 2, 16384, 0)]
KINDS = [("rms, post, gate", False, True, "rows", 0.7, True), ("layer, post, gate for all", True, True, "channels", -1.5, True),
         ("rms, no post", False, False, "none", 1.0, True), ("layer without biases", True, True, "none", 0.25, False)]


@pytest.mark.parametrize("n,rows,block,pad", NORM_SHAPES)
@pytest.mark.parametrize("kind", KINDS, ids=[k[0] for k in KINDS])
@pytest.mark.parametrize("y_type,h_type,x_type", [("f16", "f16", "f16"), ("bf16", "bf16", "i8"), ("bf16", "f32", "bf16"),
                                                  ("f32", "f32", "f32"), ("f16", "f32", "i8")])
def test_norm_residual(q, n, rows, block, pad, kind, y_type, h_type, x_type):
    import torch
    _, layer, post, gate, res_scale, bias = kind
    g = generator(n + 3 * rows)
    ld = n + pad
    y = Rim(rows, n, TYPES[y_type], ld, pad).set(normal(g, rows, n) + 0.5)
    h = Rim(rows, n, TYPES[h_type], ld, pad).set(normal(g, rows, n) * 3)
    gates = None if gate == "none" else Rim(rows if gate == "rows" else 1, n, TYPES[y_type], ld).set(normal(g, rows if gate == "rows" else 1, n))
    vector = lambda: 1 + 0.3 * normal(g, n)
    post_w, pre_w = vector() if post else None, vector()
    post_b, pre_b = 0.2 * normal(g, n) if bias and post else None, 0.2 * normal(g, n) if bias else None
    signs = signs_of(g, n) if block else None
    h_out = Rim(rows, n, TYPES[h_type], ld, pad)
    x = Rim(rows, n, torch.int8 if x_type == "i8" else TYPES[x_type], ld + 1, pad)
    scale = Rim(1, rows, torch.float32, fill=-1.0)
    q.qtip_norm_residual(y.pointer, ld, type_of(q, y_type), h.pointer, ld, type_of(q, h_type),
                         None if gates is None else gates.pointer, ld if gate == "rows" else 0, rows, n,
                         q.NORM_LAYER if layer else q.NORM_RMS, post_w, post_b, pre_w, pre_b, 1e-5, res_scale, signs, block,
                         h_out.pointer, x.pointer, ld + 1, type_of(q, x_type), scale.pointer if x_type == "i8" else None)
    torch.cuda.synchronize()

    # Errors, to first order: a sum over a row has at most 128 roundings in line (32 a thread, 6 in a wave, 16 waves and a few
    # operations around them), so a norm's factor is off by at most that many halves of a unit; and a centred value by
    # that many of the values' mean size.
    many = 128 * EPS32

    def norm_error(v, error, weight, bias):
        centred = v - v.mean(dim=1, keepdim=True) if layer else v
        error = error + many * v.abs().mean(dim=1, keepdim=True) if layer else error
        if layer:
            error = error + error.mean(dim=1, keepdim=True)
        r = 1 / (centred.square().mean(dim=1, keepdim=True) + 1e-5).sqrt()
        # (the factor moves with the root mean square of the errors)
        moved = centred.abs() * r ** 2 * (error.square().mean(dim=1, keepdim=True).sqrt())
        e = (error * r + moved * 1 + many * centred.abs() * r) * weight.double().abs()
        return e if bias is None else e + 2 * EPS32 * bias.double().abs()

    a = y.view.double()
    error = torch.zeros_like(a)
    if post:
        error = norm_error(a, error, post_w, post_b)
        a = normed(a, layer, 1e-5, post_w, post_b)
    if gates is not None:
        error = error * gates.view.double().abs()
        a = a * gates.view.double()
    error = abs(res_scale) * (error + 4 * EPS32 * a.abs()) + EPS32 * h.view.double().abs()
    want_h = h.view.double() + res_scale * a
    error = error + EPS32 * want_h.abs()
    assert bool(((h_out.view.double() - want_h).abs() <= error + EPS[h_type] * (want_h.abs() + error) + LEAST[h_type]).all())
    error = norm_error(want_h, error, pre_w, pre_b)
    want = normed(want_h, layer, 1e-5, pre_w, pre_b)
    if block:
        weight = want.abs().reshape(-1, block).sum(dim=1, keepdim=True) / math.sqrt(block)
        moved = error.reshape(-1, block).sum(dim=1, keepdim=True) / math.sqrt(block)
        error = ((2 * math.log2(block) + 8) * EPS32 * weight + moved).expand(-1, block).reshape(rows, n)
        want = rotate(want, signs, block)
    if x_type == "i8":
        if n > 1:
            check_i8(x.view, scale.view[0], want, error)
    else:
        assert bool(((x.view.double() - want).abs() <= error + EPS[x_type] * (want.abs() + error) + LEAST[x_type]).all())
    for buffer in (y, h, h_out, x, scale):
        assert buffer.rim_is_whole()


def test_norm_residual_in_place_and_in_parts(q):
    """h_out = h; without h, without y, without x, without h_out."""
    import torch
    g = generator(11)
    rows, n = 4, 777
    y, h, w = normal(g, rows, n).half(), normal(g, rows, n).half(), 1 + normal(g, n) * 0.1
    call = lambda y, h, gate, post, pre, h_out, x: q.qtip_norm_residual(
        y, n, q.F16, h, n, q.F16, gate, n, rows, n, q.NORM_RMS, post, None, pre, None, 1e-6, 0.5, None, 0, h_out, x, n, q.F16,
        None)
    h_out, x = torch.empty_like(h), torch.empty_like(h)
    call(y, h, None, w, w, h_out, x)
    place, x2 = h.clone(), torch.empty_like(h)
    call(y, place, None, w, w, place, x2)
    alone = torch.empty_like(h)
    call(y, h, None, w, None, alone, None)
    only_x = torch.empty_like(h)
    call(y, h, None, w, w, None, only_x)
    no_h, no_h_x = torch.empty_like(h), torch.empty_like(h)
    call(y, None, None, None, None, no_h, no_h_x)
    no_y, no_y_x = torch.empty_like(h), torch.empty_like(h)
    call(None, h, None, None, w, no_y, no_y_x)
    torch.cuda.synchronize()
    assert torch.equal(place, h_out) and torch.equal(x2, x) and torch.equal(alone, h_out) and torch.equal(only_x, x)
    assert torch.equal(no_h, (y.float() * 0.5).half()) and torch.equal(no_h_x, no_h)
    assert torch.equal(no_y, h)
    want = normed(h.double(), False, 1e-6, w, None)
    assert bool(((no_y_x.double() - want).abs() <= (EPS["f16"] + 128 * EPS32) * want.abs() * (1 + EPS["f16"]) + LEAST["f16"]).all())


def test_norm_residual_keeps_what_is_not_finite_in_its_row(q):
    import torch
    g = generator(12)
    rows, n = 6, 1000
    y, h = normal(g, rows, n).bfloat16(), normal(g, rows, n).bfloat16()
    clean = [torch.empty_like(h), torch.empty(rows, n, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")]
    dirty = [torch.empty_like(c) for c in clean]
    w = torch.ones(n, device="cuda")
    for buffers in (clean, dirty):
        q.qtip_norm_residual(y, n, q.BF16, h, n, q.BF16, None, 0, rows, n, q.NORM_RMS, w, None, w, None, 1e-6, 1.0, None, 0,
                             buffers[0], buffers[1], n, q.I8, buffers[2])
        torch.cuda.synchronize()
        y[1, 5], h[3, 999], y[4, 0] = float("inf"), float("nan"), float("-inf")
    for row in (0, 2, 5):
        assert torch.equal(clean[0][row], dirty[0][row]) and torch.equal(clean[1][row], dirty[1][row])
        assert float(clean[2][row]) == float(dirty[2][row])
    assert all(math.isnan(float(dirty[2][row])) for row in (1, 3, 4))


def test_rows_of_zeros_through_a_norm(q):
    import torch
    n = 640
    z = torch.zeros(2, n, dtype=torch.float16, device="cuda")
    w, out = torch.ones(n, device="cuda"), torch.full((2, n), 5, dtype=torch.int8, device="cuda")
    scale, h = torch.full((2,), 7.0, device="cuda"), torch.empty_like(z)
    for norm in (q.NORM_RMS, q.NORM_LAYER):
        q.qtip_norm_residual(z, n, q.F16, z, n, q.F16, None, 0, 2, n, norm, w, None, w, None, 1e-6, 1.0, None, 0, h, out, n,
                             q.I8, scale)
        torch.cuda.synchronize()
        assert int(out.abs().max()) == 0 and float(scale.abs().max()) == 0 and int(h.abs().max()) == 0
