"""Calls on a stream that is not the current one: what they allocate is that stream's memory, neither taken from work that the
current stream has yet to finish nor given back to it before the call is done.

The addresses tell: the allocator keeps a stream's memory apart from every other's, so a tensor that a call on `side` made lies
where no tensor of the current stream did or will."""

import pytest
import torch

from paper_2505_06653_amd import binding
from test_gpu_linear import DEV, Matrix, randn

pytestmark = pytest.mark.gpu
MIB = 1 << 20


def spans(tensors):
    return [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in tensors]


def meet(a, b):
    return any(p < s and r < q for p, q in a for r, s in b)


def calls():
    """Name, and a function of a stream that returns all tensors that the call made."""
    m = Matrix(1001, 2080, 0.01)
    x, few, dy = randn((300, 2080), 1), randn((3, 2080), 2), randn((300, 1001), 3)
    logits, t = randn((40, 50000), 4, torch.float32), torch.arange(40, device=DEV)
    _, entropy, _, _, stats = binding.bof4_token_logprobs(logits, t)
    g = torch.ones(40, device=DEV)
    return [
        ("gemv_linear", lambda s: [m.linear("gemv", few, act="silu", stream=s)]),
        ("gemm_linear", lambda s: [m.linear("gemm", x, act="silu", stream=s)]),
        ("gemm_linear_backward", lambda s: [m.backward(dy, stream=s)]),
        ("token_logprobs", lambda s: list(binding.bof4_token_logprobs(logits, t, top=9, stream=s))),
        ("token_logprobs_backward", lambda s: [binding.bof4_token_logprobs_backward(logits, stats, t, g, entropy, g, stream=s)]),
    ]


NAMES = ["gemv_linear", "gemm_linear", "gemm_linear_backward", "token_logprobs", "token_logprobs_backward"]


def watched(monkeypatch):
    """The places of everything that torch.empty made, scratch among it (the tensors themselves are not kept)."""
    made, empty = [], torch.empty

    def spy(*args, **kw):
        t = empty(*args, **kw)
        if t.is_cuda and t.numel():
            made.append((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()))
        return t

    monkeypatch.setattr(torch, "empty", spy)
    return made


def check_places(monkeypatch, call):
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    side = torch.cuda.Stream()
    # memory that the current stream gave back: the call on another stream must not get it
    freed = [torch.zeros(size, dtype=torch.uint8, device=DEV) for size in (64, 512, 4096, MIB // 4, MIB, 4 * MIB, 30 * MIB, 300 * MIB)
             for _ in range(3)]
    before = spans(freed)
    del freed
    made = watched(monkeypatch)
    results = call(side)
    monkeypatch.undo()
    assert made and len(made) >= len(results) and not meet(made, before)
    # and what it made and dropped must not go to the current stream
    sizes = [t.numel() * t.element_size() for t in results] + [q - p for p, q in made]
    del results
    later = [torch.empty(size, dtype=torch.uint8, device=DEV) for size in sizes for _ in range(2)]
    assert not meet(spans(later), made)
    side.synchronize()


@pytest.mark.parametrize("which", range(5), ids=NAMES)
def test_memory_of_a_call_is_its_stream_s(monkeypatch, which):
    name, call = calls()[which]
    assert name == NAMES[which]
    call(None)
    check_places(monkeypatch, call)


def test_results_that_nobody_keeps_while_the_stream_is_busy():
    """Log probabilities alone are kept; the current stream goes on allocating and filling meanwhile."""
    logits, t = randn((300, 50000), 4, torch.float32), torch.arange(300, device=DEV)
    want = [r.clone() for r in binding.bof4_token_logprobs(logits, t, top=9)]
    work = randn((4096, 4096), 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(side):
            for _ in range(40):
                work @ work
        kept = [binding.bof4_token_logprobs(logits, t, top=9, stream=side)[i] for i in range(5)]
        other = [torch.full_like(r, 7) for r in want for _ in range(20)]
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, want)) and all(bool((o == 7).all()) for o in other)


def test_a_side_stream_inside_a_capture():
    logits, t = randn((7, 50000), 4, torch.float32), torch.arange(7, device=DEV)
    held, side = logits.clone(), torch.cuda.Stream()
    binding.bof4_token_logprobs(held, t, top=9)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        got = binding.bof4_token_logprobs(held, t, top=9, stream=side)
        main.wait_stream(side)
    for k in range(3):
        held.copy_(torch.roll(logits, k, 1))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, binding.bof4_token_logprobs(torch.roll(logits, k, 1), t, top=9)):
            assert torch.equal(a, b)


def check_dropped(call):
    """Results that the current stream still reads when they are dropped: the call's stream does not write there again before that
    is done."""
    work, main, side = randn((4096, 4096), 1), torch.cuda.current_stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    results = call(side)
    main.wait_stream(side)
    for _ in range(300):
        work @ work
    for r in results:
        r.clone()
    places, reading = spans(results), torch.cuda.Event()
    reading.record()
    del results
    again = call(side)
    if not reading.query():  # (the current stream was still at work when memory was found for the second call)
        assert not meet(spans(again), places)
    torch.cuda.synchronize()


@pytest.mark.parametrize("which", range(5), ids=NAMES)
def test_dropped_results_are_left_alone_until_the_current_stream_has_read_them(which):
    check_dropped(calls()[which][1])


def codec_calls():
    """The same of the codec's and the products' calls (those that return numbers of the host: no tensors)."""
    m = Matrix(1001, 2080, 0.01)
    w = randn(1001 * 2080, 1, scale=0.02)
    n, block, cb = w.numel(), 32, m.cb
    T = binding.bof4_opq_threshold(0.95, block)
    codes, scales, oi, ov, k = binding.bof4_quantize(w, block, cb, 1, opq_T=T, out_capacity=n // 20)
    x, few = randn((300, 2080), 1), randn((3, 2080), 2)
    args = (codes, scales, 1001, 2080, block, cb, oi, ov)
    return {
        "quantize": lambda s: list(binding.bof4_quantize(w, block, cb, 1, opq_T=T, out_capacity=n // 20, stream=s, trim=False)[:4]),
        "quantize_lloyd": lambda s: list(binding.bof4_quantize_lloyd(w, block, cb, 1, opq_T=T, out_capacity=n // 20, stream=s, trim=False)[:4]),
        "dequantize": lambda s: [binding.bof4_dequantize(codes, scales, n, block, cb, oi, ov, stream=s)],
        "gemv_outlier_table": lambda s: [binding.bof4_gemv_outlier_table(*args, stream=s)],
        "gemm_outlier_table": lambda s: [binding.bof4_gemm_outlier_table(*args, stream=s)],
        "gemm_pack": lambda s: [binding.bof4_gemm_pack(codes, scales, 1001, 2080, block, stream=s)],
        "gemv": lambda s: [binding.bof4_gemv(m.codes, m.scales, 1001, 2080, 32, cb, few, m.gemv_table, m.k, stream=s)],
        "gemm": lambda s: [binding.bof4_gemm(m.packed, 1001, 2080, cb, x, m.gemm_table, m.k, stream=s)],
        "lloyd_step": lambda s: [] if binding.bof4_lloyd_step(w, block, cb, 1, opq_T=T, stream=s) else None,
        "lloyd_step_mae": lambda s: [] if binding.bof4_lloyd_step_mae(w, block, cb, 1, opq_T=T, stream=s) else None,
        "quant_error": lambda s: [] if binding.bof4_quant_error(w, block, cb, 1, opq_T=T, stream=s) else None,
    }


CODEC = ["quantize", "quantize_lloyd", "dequantize", "gemv_outlier_table", "gemm_outlier_table", "gemm_pack", "gemv", "gemm", "lloyd_step",
         "lloyd_step_mae", "quant_error"]


@pytest.mark.parametrize("name", CODEC)
def test_memory_of_the_codec_s_and_the_products_calls_is_their_stream_s(monkeypatch, name):
    call = codec_calls()[name]
    call(None)
    check_places(monkeypatch, call)
    check_dropped(call)
