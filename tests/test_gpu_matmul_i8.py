"""qtip_matmul_i8 against the exact sum in 64 bits."""
import pytest

from layers_util import EPS, EPS32, LEAST, TYPES, Rim, generator, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2406_11235_amd as q
    q.lib()
    return q


def type_of(q, name):
    return {"f16": q.F16, "bf16": q.BF16, "f32": q.F32}[name]


def up16(v):
    return -(-v // 16) * 16


def check(q, m, n, B, out, bias=True, values="uniform", w_pad=0, x_pad=0, y_pad=0, y_lead=0, seed=0):
    import torch
    g = generator(seed + m + 3 * n + 7 * B)
    ldw, ldx = up16(n) + w_pad, up16(n) + x_pad
    # (rows that are never looked at stand in front of and behind both; what is behind a row's end is not zero)
    W = torch.randint(-128, 128, (m + 2, ldw), device="cuda", generator=g, dtype=torch.int8)
    X = torch.randint(-128, 128, (B + 2, ldx), device="cuda", generator=g, dtype=torch.int8)
    if values == "largest":
        W.fill_(-128)
        X.fill_(-128)
    elif values == "one":  # single products: every position is seen once
        X.zero_()
        at = torch.arange(B, device="cuda") * 37 % n
        X[1:B + 1].scatter_(1, at[:, None], 1)
    w_scale, x_scale = torch.rand(m, device="cuda", generator=g) + 0.5, torch.rand(B, device="cuda", generator=g) * 1e-3
    b = normal(g, m) if bias else None
    Y = Rim(B, m, TYPES[out], m + y_pad, y_lead)
    need = q.qtip_matmul_i8_workspace(m, n, B)
    ws = torch.full((need + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    q.qtip_matmul_i8(W[1:], ldw, w_scale, m, n, X[1:], ldx, x_scale, B, b, Y.pointer, m + y_pad, type_of(q, out),
                     ws if need else None, need)
    torch.cuda.synchronize()
    # (binary64 holds every partial sum exactly)
    sums = X[1:B + 1, :n].double() @ W[1:m + 1, :n].double().t().contiguous()
    want = sums * x_scale.double()[:, None] * w_scale.double()
    error = 4 * EPS32 * want.abs()
    if bias:
        want = want + b.double()
    error = error + EPS32 * want.abs()
    off = (Y.view.double() - want).abs()
    assert bool((off <= error + EPS[out] * (want.abs() + error) + LEAST[out]).all()), float(off.max())
    assert Y.rim_is_whole()
    assert bool((ws[need:] == 0xA5).all())


SMALL = [(1, 1, 1), (1, 17, 3), (5, 16, 2), (16, 64, 16), (17, 65, 17), (33, 127, 1), (48, 128, 31), (100, 129, 5), (64, 1000, 33),
         (250, 2049, 64), (257, 512, 65), (130, 4096, 100), (16, 31000, 2), (1, 4096, 300), (511, 640, 129), (1000, 96, 257)]


@pytest.mark.parametrize("m,n,B", SMALL)
@pytest.mark.parametrize("out,bias", [("f32", True), ("f16", False), ("bf16", True)])
def test_small_and_ragged(q, m, n, B, out, bias):
    check(q, m, n, B, out, bias)


@pytest.mark.parametrize("m,n,B", [(33, 127, 1), (257, 512, 65), (300, 4096, 16), (513, 1040, 700), (2048, 4112, 40)])
@pytest.mark.parametrize("w_pad,x_pad,y_pad,y_lead", [(16, 0, 0, 0), (0, 48, 3, 0), (128, 16, 8, 4), (0, 0, 1, 1)])
def test_strides(q, m, n, B, w_pad, x_pad, y_pad, y_lead):
    for out in ("f32", "f16"):
        check(q, m, n, B, out, True, "uniform", w_pad, x_pad, y_pad, y_lead)


@pytest.mark.parametrize("m,n,B", [(4096, 4096, 1), (4096, 4096, 2), (8192, 28672, 16), (14336, 4096, 997), (8192, 8192, 64),
                                   (1024, 1024, 1), (4096, 14336, 24), (4096, 14336, 48), (4096, 14336, 130), (512, 28672, 256),
                                   (2049, 2047, 511), (4096, 4096, 4096), (28672, 512, 1024), (777, 16400, 333)])
def test_large(q, m, n, B):
    check(q, m, n, B, "bf16", False)


@pytest.mark.parametrize("B", [1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64, 65, 96, 127, 128, 129, 192, 193, 255, 256, 257, 384, 511, 512, 513])
def test_every_count_of_rows(q, B):
    check(q, 1024, 2048, B, "f32")
    check(q, 300, 1000, B, "f16")


@pytest.mark.parametrize("m,n", [(1, 16400), (64, 28672), (300, 16385), (4099, 16391), (8200, 17000)])
@pytest.mark.parametrize("B", [16, 17, 31, 32])
def test_long_rows_of_few_outputs(q, m, n, B):
    """Parts of the inputs below 33 rows."""
    check(q, m, n, B, "bf16", True)
    check(q, m, n, B, "f32", False, "uniform", 16, 32, 1, 3)


@pytest.mark.parametrize("m,n,B", [(64, 131071, 3), (64, 131071, 40), (300, 131056, 300), (1, 100000, 1)])
@pytest.mark.parametrize("values", ["largest", "uniform"])
def test_longest_rows_of_the_largest_values(q, m, n, B, values):
    check(q, m, n, B, "f32", False, values)


@pytest.mark.parametrize("m,n,B", [(64, 300, 320), (272, 4096, 4096), (256, 1111, 1200)])
def test_single_products(q, m, n, B):
    """One activation of 1 a row brings single weights out."""
    check(q, m, n, B, "f32", False, "one")


def test_rows_without_a_value_stay_so(q):
    """A scale of NaN, as the row quantizer gives rows that are not finite, is its row's alone; a scale of 0 gives the bias."""
    import torch
    g = generator(5)
    m, n = 300, 512
    for B in (3, 40, 300):
        W = torch.randint(-127, 128, (m, n), device="cuda", generator=g, dtype=torch.int8)
        X = torch.randint(-127, 128, (B, n), device="cuda", generator=g, dtype=torch.int8)
        xs, ws, bias = torch.ones(B, device="cuda"), torch.ones(m, device="cuda"), normal(g, m)
        xs[1], xs[2] = float("nan"), 0.0
        Y = torch.empty(B, m, device="cuda")
        space = torch.empty(q.qtip_matmul_i8_workspace(m, n, B) + 1, dtype=torch.uint8, device="cuda")
        q.qtip_matmul_i8(W, n, ws, m, n, X, n, xs, B, bias, Y, m, q.F32, space, space.numel())
        torch.cuda.synchronize()
        assert bool(torch.isnan(Y[1]).all()) and torch.equal(Y[2], bias)
        assert not bool(torch.isnan(Y[0]).any()) and not bool(torch.isnan(Y[3:]).any())


def test_offsets_beyond_32_bits(q):
    """Weights of more than 2^32 bytes and outputs of more than 2^32: last rows and columns are the right ones."""
    import torch
    g = generator(6)
    m, n, B = 70016, 65536, 5
    W = torch.empty(m, n, dtype=torch.int8, device="cuda")
    for at in range(0, m, 8192):
        W[at:at + 8192] = torch.randint(-127, 128, W[at:at + 8192].shape, device="cuda", generator=g, dtype=torch.int8)
    X = torch.randint(-127, 128, (B, n), device="cuda", generator=g, dtype=torch.int8)
    one = torch.ones(m, device="cuda")
    Y = torch.empty(B, m, device="cuda")
    space = torch.empty(q.qtip_matmul_i8_workspace(m, n, B) + 1, dtype=torch.uint8, device="cuda")
    q.qtip_matmul_i8(W, n, one, m, n, X, n, one, B, None, Y, m, q.F32, space, space.numel())
    torch.cuda.synchronize()
    for at in (0, 65520, m - 16):
        want = X.double() @ W[at:at + 16].double().t().contiguous()
        assert bool(((Y[:, at:at + 16].double() - want).abs() <= EPS32 * want.abs()).all())
    del W
    m, n, B = 34000, 128, 65600
    W = torch.randint(-127, 128, (m, n), device="cuda", generator=g, dtype=torch.int8)
    X = torch.randint(-127, 128, (B, n), device="cuda", generator=g, dtype=torch.int8)
    one = torch.ones(B, device="cuda")
    Y = torch.empty(B, m, dtype=torch.bfloat16, device="cuda")
    space = torch.empty(q.qtip_matmul_i8_workspace(m, n, B) + 1, dtype=torch.uint8, device="cuda")
    q.qtip_matmul_i8(W, n, one, m, n, X, n, one, B, None, Y, m, q.BF16, space, space.numel())
    torch.cuda.synchronize()
    for at in (0, 65500, B - 16):
        want = X[at:at + 16].double() @ W.double().t().contiguous()
        assert bool(((Y[at:at + 16].double() - want).abs() <= EPS["bf16"] * want.abs() * (1 + EPS32)).all())


def test_replayed_from_a_graph(q):
    """One call of every kind of product in a graph, replayed with other inputs: the eager calls' bits."""
    import torch
    g = generator(9)
    m, n = 1024, 2048
    W = torch.randint(-127, 128, (m, n), device="cuda", generator=g, dtype=torch.int8)
    ws = torch.rand(m, device="cuda", generator=g)
    jobs = []
    for B in (1, 40, 600):
        jobs.append((B, torch.zeros(B, n, dtype=torch.int8, device="cuda"), torch.rand(B, device="cuda", generator=g),
                     torch.empty(B, m, device="cuda"),
                     torch.empty(q.qtip_matmul_i8_workspace(m, n, B) + 1, dtype=torch.uint8, device="cuda")))

    def calls():
        for B, X, xs, Y, space in jobs:
            q.qtip_matmul_i8(W, n, ws, m, n, X, n, xs, B, None, Y, m, q.F32, space, space.numel())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for replay in range(3):
        for _, X, _, _, space in jobs:
            X.copy_(torch.randint(-127, 128, X.shape, device="cuda", generator=g, dtype=torch.int8))
        calls()
        torch.cuda.synchronize()
        want = [Y.clone() for _, _, _, Y, _ in jobs]
        for _, _, _, Y, space in jobs:
            Y.fill_(float("nan"))
            space.fill_(0xA5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for (_, _, _, Y, _), w in zip(jobs, want):
            assert torch.equal(Y, w), replay
