"""What the dense block's calls are made of, asked of the routines that the calls themselves use: every product is a shape that
the tensor cores take, over the sizes that the header allows."""
import random

import pytest

from paper_2609_21483_b200 import ffn


def sizes(seed, unit, n=400):
    """Tokens and two widths, small ones and large ones alike."""
    rng = random.Random(seed)
    log = lambda lo, hi, step=1: max(step, step * int(lo * (hi / lo) ** rng.random() / step))
    return [(log(1, 20000), log(unit, 20000, unit), log(unit, 20000, unit)) for _ in range(n)]


def legal(p, int8):
    """N of a product with M = 128 in one CTA: multiples of 16 up to 256.  With M = 256 on a pair: multiples of 16 in bf16, of 32 in
    8-bit integers."""
    if p["kernel"] == 1:
        return all(n % 16 == 0 and 16 <= n <= 256 for n in (p["mma_n"], p["tail_n"] or 16))
    return p["mma_n"] % (32 if int8 else 16) == 0 and 32 <= p["mma_n"] <= 256


@pytest.mark.parametrize("n_sm", [148, 132, 2])
def test_every_product_is_a_legal_shape(n_sm):
    for T, H, I in sizes(1, 16):
        for int8 in (False, True):
            for p in ffn.ffn_plan(H, I, T, int8=int8, n_sm=n_sm):
                assert legal(p, int8), (T, H, I, int8, p)
        for p in ffn.ffn_plan(H, I, T, backward=True, n_sm=n_sm):
            assert legal(p, False), (T, H, I, p)
        for p in ffn.int8_linear_plan(H, I + T % 7, T, n_sm=n_sm):
            assert legal(p, True), (T, H, I + T % 7, p)


@pytest.mark.parametrize("T,K,N", [(1023, 4096, 14333), (1500, 1040, 4120), (2100, 400, 776), (257, 14336, 520), (700, 272, 9001)])
def test_8_bit_products_on_pairs(T, K, N):
    (p,) = ffn.int8_linear_plan(K, N, T)
    assert p["kernel"] == 0 and legal(p, True), p


@pytest.mark.parametrize("T,H,I", [(1023, 4096, 6400), (300, 4096, 512), (300, 1104, 2752), (520, 8192, 208), (257, 2048, 1408)])
def test_8_bit_blocks_on_pairs(T, H, I):
    for p in ffn.ffn_plan(H, I, T, int8=True):
        assert p["kernel"] == 0 and legal(p, True), p


def test_plans_are_refused_for_what_calls_refuse():
    for bad in (dict(hidden=60, ffn=64, T=8), dict(hidden=64, ffn=64, T=9, max_tokens=8), dict(hidden=64, ffn=64, T=0, max_tokens=8),
                dict(hidden=64, ffn=72, T=8, int8=True), dict(hidden=64, ffn=64, T=8, int8=True, backward=True)):
        with pytest.raises(ffn.WeaveError):
            ffn.ffn_plan(**bad)
    with pytest.raises(ffn.WeaveError):
        ffn.int8_linear_plan(24, 64, 8)
    with pytest.raises(ffn.WeaveError):
        ffn.int8_linear_plan(64, 64, 8, x_type=7)


def test_operands_that_run_along_n_are_whole_swizzle_atoms():
    """Where an operand's N (or M) runs along its rows, what a CTA gives to a product is whole atoms of its layout: 64 elements of
    bf16 with 128-byte swizzle, 32 with 64-byte swizzle.  Columns that stick out over the matrix are zeros, not missing."""
    seen = set()
    for T, H, I in sizes(2, 8) + [(2, 64, 64), (257, 2048, 1408), (777, 1096, 2744), (4096, 4096, 14336)]:
        for p in ffn.ffn_plan(H, I, T, backward=True):
            if p["mn_run"]:
                assert p["mn_atom"] in (32, 64) and p["mn_run"] % p["mn_atom"] == 0, (T, H, I, p)
                seen.add((p["mn_run"], p["mn_atom"]))
    assert seen == {(32, 32), (64, 64), (128, 64)}, seen
