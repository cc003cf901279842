"""The dense block's calls in orders that a program may make them in, and what they refuse."""
import pytest
import torch

import paper_2609_21483_b200 as pk
from test_gpu_ffn import ACT, BF16, block

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("int8", [False, True])
def test_status_of_a_graph_replayed_on_another_stream(int8):
    """A captured call whose wait gives up, replayed on a stream that the handle never saw, behind work that is still running."""
    T, H, I = 5, 1024, 2048
    x, gate_up, down, _ = block(T, H, I, seed=61)
    if int8:
        ffn = pk.Int8FFN(*pk.quantize_rows(gate_up), *pk.quantize_rows(down), max_tokens=T)
    else:
        ffn = pk.GatedFFN(gate_up, down, max_tokens=T)
    want = ffn.forward(x)
    ffn.check()
    out = torch.empty_like(x)
    ffn.set_timeout_ms(20)
    ffn.debug_withhold_arrival(3)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ffn.forward(x, out=out)
    ffn.debug_withhold_arrival(-1)
    ffn.set_timeout_ms(4000)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
        graph.replay()
    assert ffn.status() == pk.ERR_TIMEOUT
    assert torch.equal(ffn.forward(x), want)
    ffn.check()
    ffn.close()


def test_an_output_on_top_of_scales_is_refused():
    H, I = 64, 96
    x, gate_up, down, _ = block(1, H, I, seed=62)
    gq, gs, dq, ds = *pk.quantize_rows(gate_up), *pk.quantize_rows(down)
    ffn = pk.Int8FFN(gq, gs, dq, ds, max_tokens=1)
    for scale in (gs, ds):
        before = scale.clone()
        with pytest.raises(pk.WeaveError):
            ffn.forward(x, out=scale.view(torch.bfloat16)[-H:].view(1, H))
        torch.cuda.synchronize()
        assert torch.equal(scale, before)
    ffn.check()
    ffn.close()


def test_the_largest_number_of_rows():
    """2^31 - 1 rows of one value each."""
    rows, part = (1 << 31) - 1, 1 << 28
    x = torch.empty(rows, 1, dtype=torch.bfloat16, device="cuda")
    value = lambda at: ((torch.arange(at, min(at + part, rows), device="cuda", dtype=torch.int32) & 255) - 127).to(torch.bfloat16)
    for at in range(0, rows, part):
        x[at:at + part, 0] = value(at)
    q, s = pk.quantize_rows(x)
    for at in range(0, rows, part):
        v = value(at)
        assert torch.equal(q[at:at + part, 0], (torch.sign(v) * 127).to(torch.int8))
        assert torch.equal(s[at:at + part], (v.double().abs() / 127.0).float())


@pytest.fixture(scope="module")
def long_copy():
    """A copy to the host of some 20 ms, which occupies no SM."""
    src, dst = torch.zeros(1 << 30, dtype=torch.uint8, device="cuda"), torch.empty(1 << 30, dtype=torch.uint8, pin_memory=True)
    return lambda: dst.copy_(src, non_blocking=True)


def behind_pending_work(nbytes, long_copy):
    """Leaves the allocator a block of the current stream that a kernel, which has yet to run there, still writes to."""
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    block = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    long_copy()
    block.fill_(255)


@pytest.mark.parametrize("call", ["forward", "backward", "int8_ffn", "linear", "quantize"])
def test_results_of_a_call_on_a_given_stream(call, long_copy):
    """What a call allocates for its results is ordered by the stream that the call runs on, not by the current one."""
    T, H, I = 1000, 1040, 1056
    x, gate_up, down, dy = block(T, H, I, seed=63)
    gq, gs, dq, ds = *pk.quantize_rows(gate_up), *pk.quantize_rows(down)
    ffn = pk.GatedFFN(gate_up, down, max_tokens=T, backward=True)
    i8, lin = pk.Int8FFN(gq, gs, dq, ds, max_tokens=T), pk.Int8Linear(gq, gs, max_tokens=T)
    run = {"forward": lambda **k: ffn.forward(x, **k), "backward": lambda **k: ffn.backward(x, dy, **k),
           "int8_ffn": lambda **k: i8.forward(x, **k), "linear": lambda **k: lin.forward(x, **k),
           "quantize": lambda **k: pk.quantize_rows(x, **k)}[call]
    as_tuple = lambda r: r if isinstance(r, tuple) else (r,)
    want = [t.clone() for t in as_tuple(run())]
    side = torch.cuda.Stream()
    for nbytes in sorted({t.numel() * t.element_size() for t in want}):
        behind_pending_work(nbytes, long_copy)
        got = as_tuple(run(stream=side.cuda_stream))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        del got
    # the current stream, by its number
    got = as_tuple(run(stream=torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for m in (ffn, i8, lin):
        m.check()
        m.close()


@pytest.mark.parametrize("T", [4, 200])
def test_gates_that_are_almost_closed(T):
    """sigmoid(g) where 1 + exp(-g) nears the largest fp32 number: tiny, but not zero, and a large u makes it count."""
    H, I = 64, 64
    gates = torch.tensor([-87.0, -87.5, -88.0, -88.5], device="cuda").repeat(T // 4)
    x = torch.zeros(T, H, dtype=torch.bfloat16, device="cuda")
    gate_up = torch.zeros(2 * I, H, dtype=torch.bfloat16, device="cuda")
    down = torch.eye(H, I, dtype=torch.bfloat16, device="cuda")
    gate_up[:I, 0], gate_up[I:, 1] = 1.0, 1.0
    x[:, 0], x[:, 1] = gates, 2.0 ** 100
    ffn = pk.GatedFFN(gate_up, down, max_tokens=T, backward=True)
    y = ffn.forward(x)
    dx, _, _ = ffn.backward(x, torch.ones_like(x))
    ffn.check()
    ffn.close()
    g = gates.double()
    s = torch.sigmoid(g)
    # the activation is off by 2^-16, h (dg, du) and the result by a rounding to bf16 each; all terms of a sum are alike
    off = lambda got, want: float((got.double() / want - 1).abs().max())
    assert off(y, (g * s * 2.0 ** 100)[:, None]) <= 2 * BF16 + 2 * ACT
    assert off(dx[:, 0], I * s * (1 + g * (1 - s)) * 2.0 ** 100) <= 2 * BF16 + 2 * ACT
    assert off(dx[:, 1], I * g * s) <= 2 * BF16 + 2 * ACT


@pytest.mark.parametrize("call,T,H,I", [("forward", 300, 520, 1032), ("forward", 257, 72, 6400), ("forward", 520, 8192, 208),
                                        ("backward", 257, 2048, 1408), ("backward", 777, 520, 1032), ("backward", 596, 136, 4104),
                                        ("int8_ffn", 300, 528, 1040), ("int8_ffn", 257, 80, 6400), ("int8_ffn", 520, 8192, 208)])
def test_a_wait_on_pairs_that_gives_up_ends_the_call(call, T, H, I):
    """One pair's stages never fill: its waits expire, those behind them see it, every launch of the call ends, and the handle works
    again, with K in parts (where others had arrived) as without."""
    x, gate_up, down, dy = block(T, H, I, seed=64)
    if call == "int8_ffn":
        ffn = pk.Int8FFN(*pk.quantize_rows(gate_up), *pk.quantize_rows(down), max_tokens=T)
    else:
        ffn = pk.GatedFFN(gate_up, down, max_tokens=T, backward=True)
    run = (lambda: ffn.backward(x, dy)) if call == "backward" else (lambda: (ffn.forward(x),))
    want = run()
    ffn.check()
    for cta in (0, 3):
        ffn.set_timeout_ms(20)
        ffn.debug_withhold_arrival(cta)
        run()
        assert ffn.status() == pk.ERR_TIMEOUT
        ffn.debug_withhold_arrival(-1)
        ffn.set_timeout_ms(4000)
        for _ in range(2):
            assert all(torch.equal(a, b) for a, b in zip(run(), want))
        ffn.check()
    ffn.close()


def test_streams_by_their_special_names():
    """The default stream as 0 and as cudaStreamLegacy (1), the thread's own (2), while another stream is current."""
    x, gate_up, down, dy = block(200, 264, 136, seed=65)
    ffn = pk.GatedFFN(gate_up, down, max_tokens=200, backward=True)
    want = (ffn.forward(x), *ffn.backward(x, dy), *pk.quantize_rows(x))
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        for stream in (0, 1, 2):
            got = (ffn.forward(x, stream=stream), *ffn.backward(x, dy, stream=stream), *pk.quantize_rows(x, stream=stream))
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    ffn.check()
    ffn.close()


@pytest.mark.parametrize("T", [2, 5, 200])
def test_a_row_with_nan_marks_itself_alone(T):
    """In both blocks: the others are the bits that they are without it, and a row of zeros gives zeros."""
    H, I = 272, 400
    x, gate_up, down, _ = block(T, H, I, seed=66)
    gq, gs, dq, ds = *pk.quantize_rows(gate_up), *pk.quantize_rows(down)
    for ffn in (pk.GatedFFN(gate_up, down, max_tokens=T), pk.Int8FFN(gq, gs, dq, ds, max_tokens=T)):
        want = ffn.forward(x)
        for bad in (float("nan"), float("inf"), -float("inf")):
            y = x.clone()
            y[T - 1, 7] = bad
            y[0] = 0
            got = ffn.forward(y)
            ffn.check()
            assert bool(torch.isnan(got[T - 1]).all()) and not bool(got[0].any()) and torch.equal(got[1:T - 1], want[1:T - 1])
        ffn.close()
