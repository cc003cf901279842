"""The dense block on every form of its products: which one a shape takes is asked of the library, what comes out is compared with
64 bits."""
import pytest
import torch

import paper_2609_21483_b200 as pk
from paper_2609_21483_b200 import ffn as plans
from test_gpu_ffn import BF16, SHAPES, block, exact_linear, exact_quantised, int8_inputs, normal

pytestmark = pytest.mark.gpu


def n_sm():
    return torch.cuda.get_device_properties(0).multi_processor_count


def int8_chain(x, gq, gs, dq, ds):
    """Int8FFN by its definition in 64 bits, rounded where it rounds, and the rows whose scale of h does not hang on how the activation
    is computed (off by up to 2^-16 in fp32)."""
    xq, xs = exact_quantised(x)
    g, u = ((xq.double() @ gq.double().T) * xs.double()[:, None] * gs.double()[None, :]).chunk(2, 1)
    h = g * torch.sigmoid(g) * u
    hq, hs = exact_quantised(h.to(torch.bfloat16))
    top = h.abs().amax(1)
    sure = (top * (1 - 2.0 ** -15)).to(torch.bfloat16) == (top * (1 + 2.0 ** -15)).to(torch.bfloat16)
    return (hq.double() @ dq.double().T) * hs.double()[:, None] * ds.double()[None, :], sure


def near_chain(y, want, sure):
    """The result's rounding to bf16 is off by at most 2^-8 of each value, hence of the norm.  Beside it the fp32 activation is off by
    up to 2^-16 of a value of h, either way, and borders of bf16 lie at least 2^-8 of it apart: one value in 2^7 may fall to the
    other side of one (in few tokens twice as many, by chance), and with it to the next of its row's steps of 8 bits, the largest
    value over 127; the largest of some thousand products of normal numbers is below 9 times their root mean square.  A share of
    2^-6 off by 9 / 127 each: 9 / 127 / 8 of the norm."""
    assert 8 * int(sure.sum()) >= 7 * sure.numel() - 8
    assert float((y.double() - want)[sure].norm()) <= (BF16 + 9 / 127 / 8) * float(want[sure].norm())


LINEAR_WIDTHS = [(64, 129, 272, 200), (96, 129, 272, 4824), (128, 129, 272, 14344), (160, 129, 272, 9584), (192, 129, 1040, 11896),
                 (224, 300, 272, 14344), (256, 300, 1040, 8360), (224, 1023, 4096, 14333)]


@pytest.mark.parametrize("width,T,K,N", LINEAR_WIDTHS)
def test_8_bit_product_of_every_width(width, T, K, N):
    (p,) = plans.int8_linear_plan(K, N, T, x_type=plans.INT8, n_sm=n_sm())
    assert p["kernel"] == 0 and (n_sm() != 148 or p["width"] == width), p
    q, sx, w, sw = int8_inputs(T, K, N, N)
    lin = pk.Int8Linear(w, sw, max_tokens=T)
    assert torch.equal(lin.forward(q, sx, out_dtype=torch.float32), exact_linear(q, sx, w, sw))
    lin.check()
    lin.close()


GATED_WIDTHS = [(32, 129, 272, 208), (48, 129, 272, 2512), (64, 129, 272, 7120), (80, 129, 272, 4816), (96, 300, 272, 9568),
                (112, 300, 272, 7120), (128, 129, 1040, 8416), (128, 1023, 4096, 6400)]


@pytest.mark.parametrize("width,T,H,I", GATED_WIDTHS)
def test_8_bit_gated_product_of_every_width(width, T, H, I):
    p = plans.ffn_plan(H, I, T, int8=True, n_sm=n_sm())[0]
    assert p["kernel"] == 0 and (n_sm() != 148 or p["width"] == width), p
    x, gate_up, down, _ = block(T, H, I, seed=width)
    gq, gs, dq, ds = *pk.quantize_rows(gate_up), *pk.quantize_rows(down)
    ffn = pk.Int8FFN(gq, gs, dq, ds, max_tokens=T)
    near_chain(ffn.forward(x), *int8_chain(x, gq, gs, dq, ds))
    ffn.check()
    ffn.close()


# ---------------------------------------------------------------------------------------- the one launch for small batches, 8 bits

def form(p):
    """(blocks of K side by side, a tail of K, several tiles of a thread block)"""
    return p["blocks"], p["tail_n"] > 0, p["tiles"] > 1


SMALL_LINEAR = [((1, False, False), 17, 16, 4095), ((1, False, True), 2, 1424, 20000), ((2, False, False), 3, 896, 9001),
                ((2, False, True), 16, 896, 20000), ((2, True, False), 1, 1952, 9001), ((2, True, False), 33, 2480, 9001),
                ((2, True, True), 17, 1600, 20000), ((2, True, True), 33, 7184, 40001), ((4, False, False), 3, 2304, 4095),
                ((4, False, True), 8, 2304, 20000), ((4, True, False), 16, 2656, 4095), ((4, True, False), 33, 1952, 7),
                ((4, True, True), 1, 2480, 9001), ((4, True, True), 16, 4112, 20000), ((8, False, False), 2, 2304, 520),
                ((8, False, False), 17, 2304, 7), ((8, True, False), 1, 1072, 7), ((8, True, False), 3, 1072, 100),
                ((8, True, False), 16, 1424, 521)]


@pytest.mark.parametrize("want,T,K,N", SMALL_LINEAR)
def test_small_8_bit_products_of_every_form(want, T, K, N):
    """Bit for bit, from integers and from both types that the kernel rounds itself."""
    q, sx, w, sw = int8_inputs(T, K, N, K + N)
    lin = pk.Int8Linear(w, sw, max_tokens=T)
    for x_type, dtype in ((plans.INT8, None), (plans.BF16, torch.bfloat16), (plans.F32, torch.float32)):
        (p,) = plans.int8_linear_plan(K, N, T, x_type=x_type, n_sm=n_sm())
        assert n_sm() != 148 or (p["kernel"] == 1 and form(p) == want), p
        if dtype is None:
            x, scale, xq, xs = q, sx, q, sx
        else:
            x, scale = normal((T, K), 1.0, T + K, dtype), None
            xq, xs = exact_quantised(x)
        exact = exact_linear(xq, xs, w, sw)
        for out in (torch.float32, torch.bfloat16):
            assert torch.equal(lin.forward(x, scale, out_dtype=out), exact.to(out))
    lin.check()
    lin.close()


SMALL_BLOCKS = [((8, True, False), (8, True, False), 1, 1072, 1072), ((4, True, False), (8, True, False), 2, 1248, 1952),
                ((8, True, False), (8, True, False), 3, 1424, 1072), ((2, False, False), (8, True, False), 1, 896, 2480),
                ((1, False, True), (2, True, False), 64, 4112, 9616), ((1, False, True), (4, True, False), 3, 2832, 20016),
                ((4, True, False), (4, True, False), 33, 1072, 1600), ((2, False, False), (2, True, False), 64, 2304, 2832),
                ((2, False, True), (4, True, False), 33, 2304, 9616), ((2, True, False), (2, True, False), 16, 7184, 2480),
                ((2, True, True), (2, True, False), 33, 7184, 9616), ((2, True, True), (8, True, False), 2, 1600, 9616),
                ((4, True, True), (4, True, True), 8, 7184, 9616), ((4, True, False), (2, False, False), 3, 7184, 2304),
                ((8, True, True), (4, True, False), 8, 4112, 2480), ((8, True, True), (2, True, False), 2, 7184, 2480),
                ((4, False, False), (1, False, False), 17, 896, 544), ((8, False, False), (8, True, False), 1, 2304, 1072)]


@pytest.mark.parametrize("first,second,T,H,I", SMALL_BLOCKS)
def test_small_8_bit_blocks_of_every_form(first, second, T, H, I):
    ps = plans.ffn_plan(H, I, T, int8=True, n_sm=n_sm())
    assert n_sm() != 148 or ([p["kernel"] for p in ps] == [1, 1] and [form(p) for p in ps] == [first, second]), ps
    x, gate_up, down, _ = block(T, H, I, seed=T + I)
    gq, gs, dq, ds = *pk.quantize_rows(gate_up), *pk.quantize_rows(down)
    ffn = pk.Int8FFN(gq, gs, dq, ds, max_tokens=T)
    y = ffn.forward(x)
    near_chain(y, *int8_chain(x, gq, gs, dq, ds))
    assert torch.equal(ffn.forward(x), y)
    ffn.check()
    ffn.close()


# ---------------------------------------------------------------------------------------- bf16: nothing of K is lost

def near(got, want):
    """In the norm over some thousand values.  A result is a sum whose operands h, dg or du were rounded to bf16, and is rounded
    itself: errors of either kind are spread evenly over at most half a step, 2^-8 of the value, 2^-8 / sqrt(3) at the root of the
    mean square, and those of a sum's terms add up like the terms do: together sqrt(2 / 3) 2^-8 = 3.2e-3, and next to it fp32 sums.
    A block of 8 out of K = 20000 that is lost, or taken twice, makes 2e-2."""
    err = float((got.double() - want).norm() / want.norm())
    assert err <= 4e-3, err


def exact_forward(x, gate_up, down):
    g, u = (x.double() @ gate_up.double().T).chunk(2, 1)
    return (g * torch.sigmoid(g) * u) @ down.double().T


def exact_backward(x, gate_up, down, dy):
    I = down.shape[1]
    xd, w, d, dyd = x.double(), gate_up.double(), down.double(), dy.double()
    g, u = xd @ w[:I].T, xd @ w[I:].T
    s, dh = torch.sigmoid(g), dyd @ d
    dgu = torch.cat([dh * u * s * (1 + g * (1 - s)), dh * g * s], 1)
    return dgu @ w, dgu.T @ xd, dyd.T @ (g * s * u)


SMALL_WIDTHS = [(64, 64), (128, 24), (448, 136), (1088, 320), (192, 20000), (2968, 9600), (2048, 4736), (20000, 72), (1672, 12720)]
IN_PARTS = [(130, 264, 8120), (257, 72, 6400), (270, 1016, 14840), (596, 136, 4104), (48, 4096, 64), (130, 8112, 144), (257, 6400, 80),
            (300, 4096, 512), (520, 8192, 208)]
FORWARD = [s for s in SHAPES if s[0] * min(s[1:]) >= 2048] + IN_PARTS + \
          [(T, H, I) for T in (16, 33, 48, 100, 128) for H, I in SMALL_WIDTHS if T * min(H, I) >= 2048]


@pytest.mark.parametrize("T,H,I", FORWARD)
def test_forward_in_norm(T, H, I):
    x, gate_up, down, _ = block(T, H, I, seed=T + H)
    ffn = pk.GatedFFN(gate_up, down, max_tokens=T)
    near(ffn.forward(x), exact_forward(x, gate_up, down))
    ffn.check()
    ffn.close()


@pytest.mark.parametrize("T,H,I", [s for s in SHAPES if s[0] * min(s[1:]) >= 2048] + IN_PARTS)
def test_backward_in_norm(T, H, I):
    x, gate_up, down, dy = block(T, H, I, seed=T + I)
    ffn = pk.GatedFFN(gate_up, down, max_tokens=T, backward=True)
    for got, want in zip(ffn.backward(x, dy), exact_backward(x, gate_up, down, dy)):
        near(got, want)
    ffn.check()
    ffn.close()


def test_products_in_parts_are_reached():
    """Some of the shapes above cut K, in the forward pass's first and second product and in dx."""
    parts = [[p["parts"] for p in plans.ffn_plan(H, I, T, backward=b)] for T, H, I in IN_PARTS for b in (False, True)]
    assert any(p[0] > 1 for p in parts[::2]) and any(p[1] > 1 for p in parts[::2]) and any(p[2] > 1 for p in parts[1::2])


def test_a_row_of_the_block_does_not_depend_on_the_batch():
    """The same tokens in small batches, which the one launch takes, and in one of 300 on pairs of SMs.  8 bits: the same bits, as sums
    are exact and scales a row's own.  bf16: sums in another order, off by some 2^-18 of a value where a bf16 step is 2^-8 at least:
    one value of h, or of the result, in 2^9 falls to the next step, 2^-7 of it at most: 2^-11 of the norm each."""
    H, I, T = 1024, 1408, 300
    x, gate_up, down, _ = block(T, H, I, seed=52)
    gq, gs, dq, ds = *pk.quantize_rows(gate_up), *pk.quantize_rows(down)
    ffn, i8 = pk.GatedFFN(gate_up, down, max_tokens=T), pk.Int8FFN(gq, gs, dq, ds, max_tokens=T)
    all_rows, all_i8 = ffn.forward(x), i8.forward(x)
    for n in (1, 2, 3, 17, 128, 129):
        assert torch.equal(i8.forward(x[:n]), all_i8[:n])
        rows = ffn.forward(x[:n]).double()
        assert float((rows - all_rows[:n].double()).norm()) <= 2.0 ** -10 * float(rows.norm())
    for m in (ffn, i8):
        m.check()
        m.close()
