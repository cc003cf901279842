"""The dense block on every form of its products: which one a shape takes is asked of the library, what comes out is compared with
64 bits."""
import pytest
import torch

import paper_2609_21483_b200 as pk
from paper_2609_21483_b200 import ffn as plans
from test_gpu_ffn import BF16, block, exact_linear, exact_quantised, int8_inputs

pytestmark = pytest.mark.gpu


def n_sm():
    return torch.cuda.get_device_properties(0).multi_processor_count


def int8_chain(x, gq, gs, dq, ds):
    """Int8FFN by its definition in 64 bits: rounded where it rounds, sums exact."""
    xq, xs = exact_quantised(x)
    g, u = ((xq.double() @ gq.double().T) * xs.double()[:, None] * gs.double()[None, :]).chunk(2, 1)
    hq, hs = exact_quantised((g * torch.sigmoid(g) * u).to(torch.bfloat16))
    return (hq.double() @ dq.double().T) * hs.double()[:, None] * ds.double()[None, :]


def near_chain(y, want):
    """The result's rounding to bf16 is off by at most 2^-8 of each value, hence of the norm.  Beside it the fp32 activation is off by
    up to 2^-16 of a value of h, either way, and borders of bf16 lie at least 2^-8 of it apart: one value in 2^7 may fall to the
    other side of one, and one row's largest in 2^7, which moves the scale of its row.  Either moves what is concerned by one step
    of the row's 8 bits at most, its largest value over 127; the largest of some thousand products of normal numbers is below 9
    times their root mean square.  Two shares of 2^-7 off by 9 / 127 each: 9 / 127 / 8 of the norm."""
    assert float((y.double() - want).norm()) <= (BF16 + 9 / 127 / 8) * float(want.norm())


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
    near_chain(ffn.forward(x), int8_chain(x, gq, gs, dq, ds))
    ffn.check()
    ffn.close()
