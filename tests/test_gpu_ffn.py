"""The dense feed-forward block, its gradient and its 8-bit forms against plain implementations in 64 bits.

Tolerances follow from the roundings that the header names, worst case, term by term:
  - a sum of K products in fp32 is off by at most K 2^-23 of the sum of the products' magnitudes (the tensor core
    may truncate where it aligns the addends: a whole step, 2^-23, per addition);
  - one rounding to bf16 is off by at most 2^-8 of the value;
  - the activation is off by at most 2^-16 of the value where |g| < 88 (exp and division, see fast_sigmoid()), and
    d silu / dg stays below 1.1, d^2 silu / dg^2 below 0.5.
Sums of integers are exact, so the 8-bit product has none: its fp32 result is compared bit for bit.
"""
import numpy as np
import pytest
import torch

import paper_2609_21483_b200 as pk

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -23
BF16 = 2.0 ** -8
ACT = 2.0 ** -16
TINY = 1e-30


def normal(shape, std, seed, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def block(T, H, I, seed=0):
    """x, gate_up, down, dy; weights scaled so that g, u and y are of order one whatever the widths."""
    return (normal((T, H), 1.0, seed), normal((2 * I, H), H ** -0.5, seed + 1), normal((H, I), I ** -0.5, seed + 2),
            normal((T, H), 0.01, seed + 3))


def abs_mm(a, b):
    return a.abs() @ b.abs()


def gated_and_bound(x, gate_up):
    """In 64 bits: g, u, h and how far the fp32 g, u and the unrounded h may be off."""
    H, I = x.shape[1], gate_up.shape[0] // 2
    xd, w = x.double(), gate_up.double()
    g, u = xd @ w[:I].T, xd @ w[I:].T
    eg, eu = H * STEP * abs_mm(xd, w[:I].T), H * STEP * abs_mm(xd, w[I:].T)
    s = torch.sigmoid(g)
    h = g * s * u
    eh = 1.1 * eg * (u.abs() + eu) + (g * s).abs() * eu + ACT * h.abs()
    return g, u, s, h, eg, eu, eh


def forward_and_bound(x, gate_up, down):
    _, _, _, h, _, _, eh = gated_and_bound(x, gate_up)
    I = h.shape[1]
    dd = down.double().T
    y = h @ dd
    eh = eh + BF16 * (h.abs() + eh)
    ey = eh @ dd.abs() + I * STEP * abs_mm(h, dd)
    return y, ey + BF16 * (y.abs() + ey) + TINY


def within(got, want, bound):
    d = (got.double() - want).abs()
    assert bool((d <= bound).all()), f"off by {float((d / bound).max()):.3f} of the bound at {int((d > bound).sum())} places"


SHAPES = [(1, 8, 8), (2, 64, 64), (1, 2048, 768), (7, 136, 72), (16, 512, 1024), (33, 1096, 344), (64, 256, 128), (127, 264, 520),
          (128, 2048, 1408), (129, 72, 2744), (256, 256, 128), (257, 520, 136), (300, 1096, 2744), (511, 128, 64), (1023, 4096, 648),
          (2100, 768, 1032), (700, 4008, 200), (1500, 264, 4104), (4500, 136, 72)]


@pytest.mark.parametrize("T,H,I", SHAPES)
def test_forward(T, H, I):
    x, gate_up, down, _ = block(T, H, I, seed=T)
    ffn = pk.GatedFFN(gate_up, down, max_tokens=T)
    y = ffn.forward(x)
    ffn.check()
    within(y, *forward_and_bound(x, gate_up, down))
    assert torch.equal(ffn.forward(x), y)
    ffn.close()


@pytest.mark.parametrize("T,H,I", SHAPES)
def test_backward(T, H, I):
    x, gate_up, down, dy = block(T, H, I, seed=T + 7)
    ffn = pk.GatedFFN(gate_up, down, max_tokens=T, backward=True)
    dx, dgu, dd = ffn.backward(x, dy)
    ffn.check()
    g, u, s, h, eg, eu, eh = gated_and_bound(x, gate_up)
    w, d, xd, dyd = gate_up.double(), down.double(), x.double(), dy.double()
    dh = dyd @ d
    edh = H * STEP * abs_mm(dyd, d)
    silu, slope = g * s, s * (1 + g * (1 - s))
    dg, du = dh * u * slope, dh * silu
    edg = edh * ((u.abs() + eu) * 1.1) + dh.abs() * (eu * 1.1 + (u.abs() + eu) * (0.5 * eg + 3 * ACT * (1 + g.abs()) * s))
    edu = edh * (silu.abs() + 1.1 * eg) + dh.abs() * (1.1 * eg + ACT * silu.abs())
    eh, edg, edu = (e + BF16 * (v.abs() + e) for e, v in ((eh, h), (edg, dg), (edu, du)))
    dgu64, edgu = torch.cat([dg, du], 1), torch.cat([edg, edu], 1)

    def product(a, b, ea=None, eb=None):
        want = a @ b
        e = a.shape[1] * STEP * abs_mm(a, b)
        if ea is not None:
            e = e + ea @ b.abs()
        if eb is not None:
            e = e + a.abs() @ eb
        return want, e + BF16 * (want.abs() + e) + TINY

    within(dx, *product(dgu64, w, ea=edgu))
    within(dgu, *product(dgu64.T, xd, ea=edgu.T))
    within(dd, *product(dyd.T, h, eb=eh))
    again = ffn.backward(x, dy)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dgu, dd)))
    # the forward pass of a handle that also does the gradient
    within(ffn.forward(x), *forward_and_bound(x, gate_up, down))
    ffn.close()


def test_backward_against_differences():
    """The gradients' projections on random directions against differences of the block in 64 bits."""
    T, H, I = 40, 136, 200
    x, gate_up, down, dy = block(T, H, I, seed=3)
    ffn = pk.GatedFFN(gate_up, down, max_tokens=T, backward=True)
    grads = ffn.backward(x, dy)
    ffn.check()
    ffn.close()

    def loss(xx, ww, dd):
        g, u = (xx @ ww.T).chunk(2, 1)
        return float(((g * torch.sigmoid(g) * u) @ dd.T * dy.double()).sum())

    at = [x.double(), gate_up.double(), down.double()]
    for k in range(3):
        v = torch.randn(at[k].shape, generator=torch.Generator().manual_seed(k)).double().cuda()
        eps = 1e-5
        hi, lo = ([p + sgn * eps * v if i == k else p for i, p in enumerate(at)] for sgn in (1, -1))
        want = (loss(*hi) - loss(*lo)) / (2 * eps)
        got = float((grads[k].double() * v).sum())
        # every entry of a gradient carries at most three roundings to bf16 (operands and result), each of them below
        # 2^-8 of the value or of the sum that it stands in; over n random signs they add up like sqrt(n): four times that
        n = grads[k].numel()
        rms = float(grads[k].double().pow(2).mean().sqrt())
        assert abs(got - want) <= 4 * 3 * BF16 * rms * n ** 0.5 + 1e-6 * abs(want)


@pytest.mark.parametrize("T", [0, 1, 5])
def test_rows_behind_the_batch_stay(T):
    H, I = 264, 136
    x, gate_up, down, dy = block(8, H, I, seed=9)
    ffn = pk.GatedFFN(gate_up, down, max_tokens=8, backward=True)
    buf, dbuf = (torch.full((8, H), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ffn.forward(x[:T], out=buf[:T])
    dgu, dd = (torch.full_like(t, 7.0) for t in (gate_up, down))
    ffn.backward(x[:T], dy[:T], dx=dbuf[:T], dgate_up=dgu, ddown=dd)
    ffn.check()
    assert bool((buf[T:] == 7.0).all()) and bool((dbuf[T:] == 7.0).all())
    if T == 0:
        assert not dgu.any() and not dd.any()
    else:
        assert torch.equal(buf[:T], ffn.forward(x[:T].clone()))
    ffn.close()


def test_extreme_gates():
    """g far out on both sides: the gate closes to zero or passes u through; one NaN or inf stays in its row."""
    T, H, I = 6, 64, 64
    x = torch.zeros(T, H, dtype=torch.bfloat16, device="cuda")
    gate_up = torch.zeros(2 * I, H, dtype=torch.bfloat16, device="cuda")
    down = torch.eye(H, I, dtype=torch.bfloat16, device="cuda")
    gate_up[:I, 0] = 1.0
    gate_up[I:, 1] = 1.0
    x[:, 0] = torch.tensor([-3e38, -200.0, -80.0, 200.0, float("nan"), 1.0], device="cuda")
    x[:, 1] = 2.0
    ffn = pk.GatedFFN(gate_up, down, max_tokens=T, backward=True)
    y = ffn.forward(x).float()
    dx, _, _ = ffn.backward(x, torch.ones_like(x))
    ffn.check()
    assert bool((y[:3].abs() < 1e-30).all())
    assert bool((y[3] == 400.0).all()) and bool(torch.isnan(y[4]).all())
    want = 2.0 / (1.0 + np.exp(-1.0))
    assert bool(((y[5] - want).abs() <= 2 * BF16 * want).all())
    assert bool(torch.isfinite(dx[[0, 1, 2, 3, 5]]).all()) and not bool(torch.isfinite(dx[4, 0]))
    ffn.close()


# ---------------------------------------------------------------------------------------- 8-bit integers

def exact_quantised(x):
    xd = x.double()
    scale = (xd.abs().amax(1) / 127.0).float()       # in 64 bits: torch divides fp32 by a number through its reciprocal
    q = (xd / scale.double()[:, None]).round().clamp(-127, 127)
    q[~((scale > 0) & torch.isfinite(scale))] = 0
    return q.to(torch.int8), scale


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7168), (3, 17), (5, 2048), (64, 14336), (7, 16400), (1300, 264), (2, 40008), (33, 1001)])
def test_quantize_rows(rows, cols, dtype):
    x = normal((rows, cols), 1.0, rows + cols, torch.float32)
    x = (x * torch.exp(normal((1, cols), 1.0, 5, torch.float32))).to(dtype)
    q, s = pk.quantize_rows(x)
    want_q, want_s = exact_quantised(x)
    assert torch.equal(s, want_s) and torch.equal(q, want_q)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(2049, 264), (5001, 675), (4099, 2048), (4096, 1), (2050, 7), (16386, 1024)])
def test_quantize_many_short_rows(rows, cols, dtype):
    """Rows that share a thread block: every one its own scale, the last ones of a broken block, a row with NaN among them."""
    x = normal((rows, cols), 1.0, cols, dtype) * (2.0 ** (torch.arange(rows, device="cuda") % 40 - 20))[:, None].to(dtype)
    q, s = pk.quantize_rows(x)
    want_q, want_s = exact_quantised(x)
    assert torch.equal(s, want_s) and torch.equal(q, want_q)
    x[rows - 2, 0], x[5] = float("nan"), 0.0
    q2, s2 = pk.quantize_rows(x)
    assert bool(torch.isnan(s2[rows - 2])) and not bool(q2[rows - 2].any()) and float(s2[5]) == 0.0 and not bool(q2[5].any())
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[rows - 2] = keep[5] = False
    assert torch.equal(q2[keep], q[keep]) and torch.equal(s2[keep], s[keep])


def test_quantize_rows_at_its_edges():
    """Ties, rows of zeros, infinities and NaN, the largest and the smallest numbers."""
    rows = [[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 126.5],            # scale 1: ties to even
            [254.0, 1.0, 3.0, 5.0, -1.0, -3.0, -5.0, 253.0],            # scale 2: the same ones
            [0.0] * 8, [-0.0] * 8,
            [float("inf")] + [1.0] * 7, [float("nan")] + [1.0] * 7, [1.0] * 7 + [-float("inf")],
            [3.3e38, -3.3e38, 1.0, 1e38, 0, 0, 0, 0], [1e-38, 5e-39, -2e-39, 1e-40, 0, 0, 0, 0],
            [2e-40, 1e-40, -3e-41, 1e-41, 0, 0, 0, 0], [1e-43, 5e-44, 0, 0, 0, 0, 0, 0], [1.4e-45, 0, 0, 0, 0, 0, 0, 0]]
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.tensor(rows, dtype=torch.float32, device="cuda").to(dtype)
        q, s = pk.quantize_rows(x)
        want_q, want_s = exact_quantised(x)
        assert torch.equal(s.view(torch.int32)[~torch.isnan(s)], want_s.view(torch.int32)[~torch.isnan(want_s)])
        assert torch.equal(torch.isnan(s), torch.isnan(want_s)) and torch.equal(q, want_q)


def int8_inputs(T, K, N, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.randint(-128, 128, (N, K), generator=g, device="cuda", dtype=torch.int8)
    q = torch.randint(-128, 128, (T, K), generator=g, device="cuda", dtype=torch.int8)
    return q, torch.rand(T, generator=g, device="cuda") + 0.01, w, torch.rand(N, generator=g, device="cuda") * 0.01


def exact_linear(q, sx, w, sw):
    return (q.double() @ w.double().T).float() * (sx[:, None] * sw[None, :])


INT8_SHAPES = [(700, 272, 9001), (1023, 400, 14336), (1500, 1040, 4120), (1, 16, 1), (1, 7168, 2048), (2, 144, 7), (15, 4096, 264), (33, 272, 4095), (64, 128, 128), (129, 1040, 130), (256, 512, 256),
               (257, 14336, 520), (1023, 2048, 1001), (2100, 400, 776)]


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,K,N", INT8_SHAPES)
def test_int8_linear(T, K, N, out):
    q, sx, w, sw = int8_inputs(T, K, N, T + K + N)
    lin = pk.Int8Linear(w, sw, max_tokens=T)
    y = lin.forward(q, sx, out_dtype=out)
    lin.check()
    assert torch.equal(y, exact_linear(q, sx, w, sw).to(out))
    # from bf16 and fp32: the rounding to 8 bits by quantize_rows()'s rule
    for dtype in (torch.bfloat16, torch.float32):
        x = normal((T, K), 1.0, T, dtype)
        xq, xs = exact_quantised(x)
        assert torch.equal(lin.forward(x, out_dtype=out), exact_linear(xq, xs, w, sw).to(out))
    lin.check()
    lin.close()


def test_int8_linear_largest_sums():
    """65536 products of -128 * -128 and of 127 * -128: the int32 sums next to their limit."""
    K, T, N = 65536, 3, 20
    q = torch.full((T, K), -128, dtype=torch.int8, device="cuda")
    q[1] = 127
    w = torch.full((N, K), -128, dtype=torch.int8, device="cuda")
    sx, sw = torch.ones(T, device="cuda"), torch.ones(N, device="cuda")
    lin = pk.Int8Linear(w, sw, max_tokens=T)
    assert torch.equal(lin.forward(q, sx, out_dtype=torch.float32), exact_linear(q, sx, w, sw))
    lin.check()
    lin.close()


def test_int8_linear_marks_rows_with_nan():
    T, K, N = 5, 64, 24
    _, _, w, sw = int8_inputs(T, K, N, 1)
    x = normal((T, K), 1.0, 2)
    x[1, 3] = float("nan")
    x[3, 5] = float("inf")
    x[4] = 0
    lin = pk.Int8Linear(w, sw, max_tokens=T)
    y = lin.forward(x)
    lin.check()
    assert bool(torch.isnan(y[[1, 3]]).all()) and bool(torch.isfinite(y[[0, 2]]).all()) and not y[4].any()
    lin.close()


@pytest.mark.parametrize("T,H,I", [(1, 16, 16), (1, 2048, 768), (7, 144, 80), (33, 1040, 336), (64, 512, 1408), (129, 272, 528), (300, 1104, 2752)])
def test_int8_ffn(T, H, I):
    """h is off by one rounding to bf16 and by half a step of its row's scale (8 bits); g and u come from exact sums, times
    two fp32 products of scales (three roundings of 2^-24 at most)."""
    x, gate_up, down, _ = block(T, H, I, seed=T + 1)
    (gq, gs), (dq, ds) = pk.quantize_rows(gate_up), pk.quantize_rows(down)
    ffn = pk.Int8FFN(gq, gs, dq, ds, max_tokens=T)
    y = ffn.forward(x)
    ffn.check()
    xq, xs = exact_quantised(x)
    gu = (xq.double() @ gq.double().T) * xs.double()[:, None] * gs.double()[None, :]
    g, u = gu.chunk(2, 1)
    h = g * torch.sigmoid(g) * u
    eh = (BF16 + ACT + 8 * 2.0 ** -24 * (1 + g.abs())) * h.abs()
    step = (h.abs() + eh).amax(1, keepdim=True) / 127.0
    dd = (dq.double() * ds.double()[:, None]).T
    want = h @ dd
    e = (eh + 0.5 * step * (1 + 2.0 ** -20)) @ dd.abs()
    within(y, want, e + (BF16 + 2.0 ** -22) * (want.abs() + e) + TINY)
    # the same chain from the operators that it is made of: equal but for values of h on a border of bf16, which the
    # fp32 activation may put on either side (one step of bf16, one step of 8 bits in q)
    lin_gu, lin_d = pk.Int8Linear(gq, gs, max_tokens=T), pk.Int8Linear(dq, ds, max_tokens=T)
    gf, uf = lin_gu.forward(x, out_dtype=torch.float32).chunk(2, 1)
    hf = (gf * torch.sigmoid(gf) * uf).to(torch.bfloat16)
    chain = lin_d.forward(hf).double()
    assert float((chain - y.double()).norm()) <= 2 * BF16 * float(y.double().norm())
    for m in (ffn, lin_gu, lin_d):
        m.check()
        m.close()


# ---------------------------------------------------------------------------------------- how the calls are made

def test_together_as_a_training_step_and_a_served_one():
    """Forward, gradient, an update of the weights in place, forward again; then the updated weights in 8 bits."""
    T, H, I = 200, 272, 528
    x, gate_up, down, dy = block(T, H, I, seed=21)
    ffn = pk.GatedFFN(gate_up, down, max_tokens=T, backward=True)
    before = ffn.forward(x)
    _, dgu, dd = ffn.backward(x, dy)
    gate_up.sub_(dgu * 0.5)
    down.sub_(dd * 0.5)
    after = ffn.forward(x)
    ffn.check()
    within(after, *forward_and_bound(x, gate_up, down))
    # a step against the gradient of sum(dy * y) makes that sum smaller
    assert float((after.double() * dy.double()).sum()) < float((before.double() * dy.double()).sum())
    (gq, gs), (dq, ds) = pk.quantize_rows(gate_up), pk.quantize_rows(down)
    served = pk.Int8FFN(gq, gs, dq, ds, max_tokens=T)
    y8 = served.forward(x)
    served.check()
    # a rounding to 8 bits is off by step / sqrt(12) on average, the step being the row's largest value over 127: 0.8 % of
    # the root mean square for the normal rows of x and of both weights (largest of some hundred: 3.5), 2 % for the products
    # in h, whose largest is up to 9 times theirs; together below 3 %
    assert float((y8.double() - after.double()).norm()) < 0.05 * float(after.double().norm())
    served.close()
    ffn.close()


@pytest.mark.parametrize("T", [1, 40, 300])
def test_captured_and_replayed(T):
    H, I = 272, 400
    x, gate_up, down, dy = block(T, H, I, seed=T)
    (gq, gs), (dq, ds) = pk.quantize_rows(gate_up), pk.quantize_rows(down)
    ffn, i8 = pk.GatedFFN(gate_up, down, max_tokens=T, backward=True), pk.Int8FFN(gq, gs, dq, ds, max_tokens=T)
    want = [ffn.forward(x), *ffn.backward(x, dy), i8.forward(x)]
    got = [torch.empty_like(t) for t in want]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ffn.forward(x, out=got[0])
        ffn.backward(x, dy, dx=got[1], dgate_up=got[2], ddown=got[3])
        i8.forward(x, out=got[4])
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        ffn.check()
        i8.check()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    # new inputs in the same buffers
    x2, _, _, dy2 = block(T, H, I, seed=T + 50)
    want = [ffn.forward(x2), *ffn.backward(x2, dy2), i8.forward(x2)]
    x.copy_(x2)
    dy.copy_(dy2)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ffn.close()
    i8.close()


def test_on_a_side_stream_and_back_to_back():
    T, H, I = 70, 520, 264
    x, gate_up, down, dy = block(T, H, I, seed=5)
    ffn = pk.GatedFFN(gate_up, down, max_tokens=T, backward=True)
    want = [ffn.forward(x), *ffn.backward(x, dy)]
    ffn.check()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(50):
            y = ffn.forward(x)
            grads = ffn.backward(x, dy)
    side.synchronize()
    ffn.check()
    assert torch.equal(y, want[0]) and all(torch.equal(a, b) for a, b in zip(grads, want[1:]))
    # each batch size of one handle gives what it gives alone
    for n in (1, 16, 33, 69):
        alone = pk.GatedFFN(gate_up, down, max_tokens=n)
        assert torch.equal(alone.forward(x[:n]), ffn.forward(x[:n]))
        alone.close()
    ffn.close()


@pytest.mark.parametrize("int8", [False, True])
def test_made_of_memory_that_is_still_written_to(int8):
    """The allocator gives a handle the block of a tensor whose last kernel has not run yet."""
    H, I, T = 256, 512, 16
    x, gate_up, down, _ = block(T, H, I, seed=13)
    (gq, gs), (dq, ds) = pk.quantize_rows(gate_up), pk.quantize_rows(down)
    make = (lambda: pk.Int8FFN(gq, gs, dq, ds, max_tokens=T)) if int8 else (lambda: pk.GatedFFN(gate_up, down, max_tokens=T))
    ffn = make()
    want = ffn.forward(x)
    ffn.check()
    nbytes = ffn.workspace.numel()
    ffn.close()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        before = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        torch.cuda._sleep(50_000_000)
        before.fill_(255)
        at = before.data_ptr()
        del before
        ffn = make()
        assert ffn.workspace.data_ptr() == at
        y = ffn.forward(x)
        ffn.check()
        assert torch.equal(y, want)
        ffn.close()


def test_refusals_on_the_device():
    x, gate_up, down, dy = block(8, 64, 64)
    ffn = pk.GatedFFN(gate_up, down, max_tokens=8)
    with pytest.raises(pk.WeaveError):
        ffn.backward(x, dy)                                       # no workspace for it was asked for
    with pytest.raises(pk.WeaveError):
        ffn.forward(torch.zeros(9, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(pk.WeaveError):
        ffn.forward(x, out=x)
    big = torch.zeros(8 * 64 + 1, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(pk.WeaveError):
        ffn.forward(big[1:].view(8, 64))                          # 2-byte aligned
    for bad in (x.float(), x.t().contiguous().t(), x.cpu(), x[:, :32].contiguous()):
        with pytest.raises(AssertionError):
            ffn.forward(bad)
    with pytest.raises(pk.WeaveError):
        pk.GatedFFN(torch.zeros(24, 20, dtype=torch.bfloat16, device="cuda"), torch.zeros(20, 12, dtype=torch.bfloat16, device="cuda"))
    ffn.check()
    ffn.close()


@pytest.mark.parametrize("int8", [False, True])
def test_a_wait_that_gives_up_ends_the_call(int8):
    """One thread block never arrives: every wait behind that barrier expires, the call ends with a status, and the handle
    works again."""
    T, H, I = 5, 1024, 2048          # a shape whose small batches run in one launch, in either form
    x, gate_up, down, _ = block(T, H, I, seed=6)
    if int8:
        ffn = pk.Int8FFN(*pk.quantize_rows(gate_up), *pk.quantize_rows(down), max_tokens=T)
    else:
        ffn = pk.GatedFFN(gate_up, down, max_tokens=T)
    want = ffn.forward(x)
    ffn.check()
    ffn.set_timeout_ms(20)
    ffn.debug_withhold_arrival(3)
    ffn.forward(x)
    assert ffn.status() == pk.ERR_TIMEOUT
    ffn.debug_withhold_arrival(-1)
    ffn.set_timeout_ms(4000)
    for _ in range(3):
        assert torch.equal(ffn.forward(x), want)
    ffn.check()
    with pytest.raises(pk.WeaveError):
        ffn.debug_withhold_arrival(-2)
    ffn.close()


def test_two_handles_on_two_streams():
    """Small and large batches of two handles side by side: what each computes does not change."""
    H, I = 528, 400
    x, gate_up, down, dy = block(300, H, I, seed=31)
    (gq, gs), (dq, ds) = pk.quantize_rows(gate_up), pk.quantize_rows(down)
    a, b = pk.GatedFFN(gate_up, down, max_tokens=300, backward=True), pk.Int8FFN(gq, gs, dq, ds, max_tokens=300)
    sizes = (1, 40, 300)
    want = {(k, n): m.forward(x[:n]) for k, m in (("a", a), ("b", b)) for n in sizes}
    grads = a.backward(x, dy)
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(40):
        for n in sizes:
            for (k, m), s in zip((("a", a), ("b", b)), streams):
                with torch.cuda.stream(s):
                    got.append((k, n, m.forward(x[:n])))
        with torch.cuda.stream(streams[0]):
            g = a.backward(x, dy)
    torch.cuda.synchronize()
    a.check()
    b.check()
    assert all(torch.equal(want[k, n], y) for k, n, y in got)
    assert all(torch.equal(p, q) for p, q in zip(g, grads))
    a.close()
    b.close()


def test_two_graphs_of_one_handle_in_turn():
    """Both use the handle's workspace; replayed in the order of a stream they do not disturb one another."""
    H, I = 272, 400
    x, gate_up, down, _ = block(200, H, I, seed=41)
    ffn = pk.GatedFFN(gate_up, down, max_tokens=200)
    outs = [torch.empty(n, H, dtype=torch.bfloat16, device="cuda") for n in (20, 200)]
    want = [ffn.forward(x[:n]) for n in (20, 200)]
    graphs = []
    for o in outs:
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ffn.forward(x[:o.shape[0]], out=o)
        graphs.append(g)
    for _ in range(20):
        for g, o in zip(graphs, outs):
            o.zero_()
            g.replay()
        eager = ffn.forward(x[:20])
    torch.cuda.synchronize()
    ffn.check()
    assert all(torch.equal(o, w) for o, w in zip(outs, want)) and torch.equal(eager, want[0])
    ffn.close()


@pytest.mark.parametrize("T", [1, 8, 9, 16, 24, 48, 100, 128])
def test_small_batches_of_every_plan(T):
    """Every number of K blocks per step, whole and broken last steps, one and several tiles per thread block."""
    for H, I in ((64, 64), (128, 24), (448, 136), (1088, 320), (192, 20000), (2968, 9600), (2048, 4736)):
        x, gate_up, down, _ = block(T, H, I, seed=T + H)
        ffn = pk.GatedFFN(gate_up, down, max_tokens=T)
        within(ffn.forward(x), *forward_and_bound(x, gate_up, down))
        ffn.check()
        ffn.close()


@pytest.mark.parametrize("T,H,I", [(130, 264, 8120), (257, 72, 6400), (270, 1016, 14840), (596, 136, 4104)])
def test_long_products_with_few_tiles(T, H, I):
    """K cut into parts that different thread blocks sum up: forward, gradient, 8-bit; twice, since the arrivals' counters go back to
    zero, and with another number of rows in between."""
    x, gate_up, down, dy = block(T, H, I, seed=T + I)
    ffn = pk.GatedFFN(gate_up, down, max_tokens=T, backward=True)
    y = ffn.forward(x)
    within(y, *forward_and_bound(x, gate_up, down))
    grads = ffn.backward(x, dy)
    within(ffn.forward(x[: T - 1]), *forward_and_bound(x[: T - 1], gate_up, down))
    assert torch.equal(ffn.forward(x), y)
    assert all(torch.equal(a, b) for a, b in zip(ffn.backward(x, dy), grads))
    ffn.check()
    # dx once more, in 64 bits from the kernel's own definition
    g, u, s, h, eg, eu, eh = gated_and_bound(x, gate_up)
    w, d, dyd = gate_up.double(), down.double(), dy.double()
    dh = dyd @ d
    edh = H * STEP * abs_mm(dyd, d)
    silu, slope = g * s, s * (1 + g * (1 - s))
    dg, du = dh * u * slope, dh * silu
    edg = edh * ((u.abs() + eu) * 1.1) + dh.abs() * (eu * 1.1 + (u.abs() + eu) * (0.5 * eg + 3 * ACT * (1 + g.abs()) * s))
    edu = edh * (silu.abs() + 1.1 * eg) + dh.abs() * (1.1 * eg + ACT * silu.abs())
    dgu, e = torch.cat([dg, du], 1), torch.cat([edg, edu], 1)
    e = e + BF16 * (dgu.abs() + e)
    want = dgu @ w
    bound = e @ w.abs() + 2 * I * STEP * abs_mm(dgu, w)
    within(grads[0], want, bound + BF16 * (want.abs() + bound) + TINY)
    ffn.close()
    # 8-bit: exact sums, results of 2 and of 4 bytes, widths that end on whole 16 bytes and not
    for n in (H, H + 1):
        q, sx, wq, sw = int8_inputs(T, I // 16 * 16, n, T)
        lin = pk.Int8Linear(wq, sw, max_tokens=T)
        for out in (torch.float32, torch.bfloat16):
            for rows in (T, T - 1, T):
                assert torch.equal(lin.forward(q[:rows], sx[:rows], out_dtype=out), exact_linear(q, sx, wq, sw).to(out)[:rows])
        lin.check()
        lin.close()


@pytest.mark.parametrize("T,H,I", [(48, 4096, 64), (130, 8112, 144), (257, 6400, 80), (300, 4096, 512), (520, 8192, 208)])
def test_long_first_products_with_few_tiles(T, H, I):
    """The same for the product that ends in the activation, in both types."""
    test_forward(T, H, I)
    test_int8_ffn(T, H, I)


def test_a_row_does_not_depend_on_the_batch():
    """The same token alone, in a small batch and in a large one: 8-bit products are the same bits, bf16 ones within a rounding."""
    H, I = 1024, 1408
    x, gate_up, down, _ = block(300, H, I, seed=51)
    (gq, gs), (dq, ds) = pk.quantize_rows(gate_up), pk.quantize_rows(down)
    lin = pk.Int8Linear(gq, gs, max_tokens=300)
    all_rows = lin.forward(x, out_dtype=torch.float32)
    for n in (1, 2, 3, 17, 128, 129):
        assert torch.equal(lin.forward(x[:n], out_dtype=torch.float32), all_rows[:n])
    lin.check()
    lin.close()
