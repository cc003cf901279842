"""CPU-side checks of the dense block's boundary: its symbols, its shape rules and what it refuses before it touches a GPU."""
import ctypes
import os
import re

import pytest

import paper_2609_21483_b200 as pk
from paper_2609_21483_b200 import ffn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, WORKSPACE = -1, -4


@pytest.fixture(scope="module")
def lib():
    pk.build()
    return ffn.load()


def test_every_declared_symbol_is_exported(lib):
    hdr = open(os.path.join(ROOT, "include", "weave_ffn.h")).read()
    hdr = re.sub(r"/\*.*?\*/", "", hdr, flags=re.S)
    declared = set(re.findall(r"\b(weave_(?:ffn|int8)_[a-z_0-9]+)\s*\(", hdr))
    assert declared == set(ffn.EXPORTS), declared ^ set(ffn.EXPORTS)
    for name in declared:
        assert getattr(lib, name) is not None


def test_block_shapes(lib):
    T, H, I = 4096, 4096, 14336
    fwd = pk.ffn_workspace_bytes(H, I, T)
    assert T * I * 2 <= fwd < T * I * 2 + (32 << 20)
    both = pk.ffn_workspace_bytes(H, I, T, backward=True)
    assert T * I * 6 <= both < T * I * 6 + (32 << 20)
    i8 = pk.ffn_workspace_bytes(H, I, T, int8=True)
    assert T * (H + 3 * I + 8) <= i8 < T * (H + 3 * I + 8) + (32 << 20)
    assert pk.ffn_workspace_bytes(8, 8, 1) > 0 and pk.ffn_workspace_bytes(16, 16, 1, int8=True) > 0
    # past 32 bits
    assert pk.ffn_workspace_bytes(65536, 65536, 1 << 22, backward=True) > 6 * (1 << 38)
    for bad in ((4, 8, 1), (8, 12, 1), (0, 8, 1), (8, -8, 1), (8, 8, 0), (8, 8, -1), (65544, 8, 1), (8, 8, (1 << 22) + 1)):
        assert pk.ffn_workspace_bytes(*bad) == 0, bad
    for bad in ((8, 16, 1), (16, 24, 1)):
        assert pk.ffn_workspace_bytes(*bad, int8=True) == 0, bad
    assert pk.ffn_workspace_bytes(16, 16, 1, int8=True, backward=True) == 0


def test_linear_shapes(lib):
    # partial sums have a place from 33 tokens on, and none where all columns make more than half a wave of tiles
    def step(f):
        return f(33) - f(32)
    assert 9 << 20 < step(lambda T: pk.int8_linear_workspace_bytes(4096, 4096, T)) < 10 << 20
    assert step(lambda T: pk.int8_linear_workspace_bytes(4096, 14336, T)) < 1 << 17
    assert 9 << 20 < step(lambda T: pk.ffn_workspace_bytes(4096, 1408, T)) < 10 << 20
    assert 9 << 20 < step(lambda T: pk.ffn_workspace_bytes(8192, 1408, T)) < 10 << 20
    assert step(lambda T: pk.ffn_workspace_bytes(8192, 14336, T)) < 1 << 17
    assert pk.int8_linear_workspace_bytes(16, 1, 1) > 0
    for bad in ((8, 1, 1), (0, 1, 1), (16, 0, 1), (16, 1, 0), (65552, 1, 1), (16, (1 << 22) + 1, 1), (16, 1, (1 << 22) + 1)):
        assert pk.int8_linear_workspace_bytes(*bad) == 0, bad


def _ffn(**kw):
    v = dict(hidden=64, ffn=64, max_tokens=8, weight_type=0, backward=0, gate_up=0x1000, down=0x10000, gate_up_scale=None,
             down_scale=None, workspace=0x100000, workspace_bytes=1 << 30)
    v.update(kw)
    return ffn._FfnConfig(**v)


@pytest.mark.parametrize("change,code", [
    (dict(hidden=60), INVALID), (dict(weight_type=1), INVALID), (dict(backward=2), INVALID), (dict(gate_up=None), INVALID),
    (dict(down=None), INVALID), (dict(workspace=None), INVALID), (dict(gate_up=0x1008), INVALID), (dict(down=0x10002), INVALID),
    (dict(workspace=0x100010), INVALID), (dict(gate_up_scale=0x2000), INVALID), (dict(weight_type=2), INVALID),
    (dict(weight_type=2, gate_up_scale=0x2000), INVALID), (dict(weight_type=2, gate_up_scale=0x2000, down_scale=0x3002), INVALID),
    (dict(weight_type=2, gate_up_scale=0x2000, down_scale=0x3000, backward=1), INVALID), (dict(workspace_bytes=100), WORKSPACE)])
def test_create_refuses_before_it_touches_a_gpu(lib, change, code):
    h = ctypes.c_void_p(1)
    assert lib.weave_ffn_create(ctypes.byref(_ffn(**change)), ctypes.byref(h)) == code
    assert not h.value


@pytest.mark.parametrize("change,code", [
    (dict(in_features=24), INVALID), (dict(weight=None), INVALID), (dict(scale=None), INVALID), (dict(weight=0x1008), INVALID),
    (dict(scale=0x2001), INVALID), (dict(workspace=0x100200), INVALID), (dict(workspace_bytes=0), WORKSPACE)])
def test_linear_create_refuses_before_it_touches_a_gpu(lib, change, code):
    v = dict(in_features=64, out_features=7, max_tokens=8, weight=0x1000, scale=0x2000, workspace=0x100000, workspace_bytes=1 << 30)
    v.update(change)
    h = ctypes.c_void_p(1)
    assert lib.weave_int8_linear_create(ctypes.byref(ffn._Int8LinearConfig(**v)), ctypes.byref(h)) == code
    assert not h.value


def test_calls_without_a_handle(lib):
    assert lib.weave_ffn_create(ctypes.byref(_ffn()), None) == INVALID
    assert lib.weave_ffn_create(None, ctypes.byref(ctypes.c_void_p())) == INVALID
    assert lib.weave_ffn_forward(None, None, None, 1, None) == INVALID
    assert lib.weave_ffn_backward(None, None, None, None, None, None, 1, None) == INVALID
    assert lib.weave_ffn_status(None) == INVALID and lib.weave_ffn_set_timeout_ms(None, 5) == INVALID
    assert lib.weave_ffn_debug_withhold_arrival(None, 0) == INVALID
    assert lib.weave_ffn_destroy(None) == 0 and lib.weave_int8_linear_destroy(None) == 0
    assert lib.weave_int8_linear_forward(None, None, 0, None, None, 0, 1, None) == INVALID
    assert lib.weave_int8_linear_status(None) == INVALID


def test_quantize_refuses(lib):
    f = lib.weave_int8_quantize
    a, q, s = 0x10000, 0x20000, 0x30000
    assert f(a, 2, 4, 4, q, s, None) == INVALID          # int8 input
    assert f(a, 0, -1, 4, q, s, None) == INVALID and f(a, 0, 4, 0, q, s, None) == INVALID
    assert f(a, 0, 1, (1 << 24) + 1, q, s, None) == INVALID
    assert f(None, 0, 4, 4, q, s, None) == INVALID and f(a, 0, 4, 4, None, s, None) == INVALID and f(a, 0, 4, 4, q, None, None) == INVALID
    assert f(a + 1, 0, 4, 4, q, s, None) == INVALID and f(a + 2, 1, 4, 4, q, s, None) == INVALID and f(a, 0, 4, 4, q, s + 2, None) == INVALID
    assert f(a, 0, 4, 4, a + 8, s, None) == INVALID      # q inside x
    assert f(a, 0, 4, 4, q, q + 12, None) == INVALID     # scale inside q
    assert f(a, 0, 0, 4, q, s, None) == 0                # no rows


def test_classes_need_a_gpu():
    import torch
    if torch.cuda.is_available():
        pytest.skip("CPU-only check")
    w = torch.zeros(16, 8, dtype=torch.bfloat16)
    with pytest.raises(RuntimeError):
        pk.GatedFFN(w, torch.zeros(8, 8, dtype=torch.bfloat16))
    with pytest.raises(RuntimeError):
        pk.Int8Linear(torch.zeros(16, 16, dtype=torch.int8), torch.zeros(16))
    with pytest.raises(RuntimeError):
        pk.Int8FFN(torch.zeros(32, 16, dtype=torch.int8), torch.zeros(32), torch.zeros(16, 16, dtype=torch.int8), torch.zeros(16))
    with pytest.raises(AssertionError):
        pk.quantize_rows(torch.zeros(2, 2))
