"""The attention half of a calibrated layer as a server drives it: recalibration under it, wrong shapes, ragged lengths,
several streams."""
import threading

import pytest
import torch

from paper_2311_01305_b200 import aweq, calibrate, serve, synth

pytestmark = pytest.mark.gpu


def calibrated():
    wl = synth.workloads(1.0 / 512)["opt125m_model_w8a8"]
    X, W = synth.generate(wl, "cuda")
    cal = calibrate.LayerCalibrator(wl, 8, X, W)
    cal.run()
    return cal, X["attn_in"]


def chunk(block, x, n_seq, n_q, own, table, held=0):
    """n_q tokens of each of n_seq sequences that hold ``held`` already."""
    i32 = dict(dtype=torch.int32, device="cuda")
    pos = (held + torch.arange(n_q, **i32)).repeat(n_seq)
    seq = torch.arange(n_seq, **i32).repeat_interleave(n_q)
    attend = block.attention(n_seq, n_q, max_own=own)
    return lambda: block(x, attend, table, torch.full((n_seq,), held + n_q, **i32), pos, seq)


def test_block_keeps_what_it_was_made_of():
    """A calibration that runs again writes 1/s, codes, pairs and biases in place."""
    cal, x = calibrated()
    block = serve.AttentionBlock(cal, 12, 4)
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    step = chunk(block, x[:10].contiguous(), 2, 5, 32, table)
    want = step()
    for out in cal.out.values():
        for t in out.values():
            if isinstance(t, torch.Tensor) and t.is_floating_point():
                t.mul_(1.5)
    assert torch.equal(step(), want)


def test_block_refuses_inputs_of_another_shape():
    """The codes of an input wider than the layer's would not fit the buffers made for them."""
    cal, x = calibrated()
    block, other = (serve.AttentionBlock(cal, 12, 4) for _ in range(2))
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    for bad in (torch.cat([x[:10], x[:10, :16]], 1), x[:10, :752].contiguous(), x[:9].contiguous(), x[:11].contiguous(), x[0]):
        with pytest.raises(ValueError):
            chunk(block, bad, 2, 5, 32, table)()
    i32 = dict(dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        block(x[:2].contiguous(), other.attention(2, 1, max_own=16), table, torch.ones(2, **i32), torch.zeros(2, **i32), torch.arange(2, **i32))


def test_block_on_two_streams_and_threads_at_a_time():
    """Calls of the same number of tokens that run side by side share nothing but the cache."""
    cal, x = calibrated()
    block = serve.AttentionBlock(cal, 12, 64)
    tables = torch.arange(64, dtype=torch.int32, device="cuda").view(2, 4, 8)
    calls = [chunk(block, x[80 * w:80 * w + 80].contiguous(), 4, 20, 32, tables[w]) for w in range(2)]
    want = [c() for c in calls]
    torch.cuda.synchronize()
    got = [[], []]

    def serve_one(w, stream):
        with torch.cuda.stream(stream):
            for _ in range(40):
                got[w].append(calls[w]())

    for streams in ([torch.cuda.Stream(), torch.cuda.Stream()], [torch.cuda.default_stream()] * 2):
        threads = [threading.Thread(target=serve_one, args=(w, streams[w])) for w in range(2)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        torch.cuda.synchronize()
    for w in range(2):
        assert len(got[w]) == 80 and all(torch.equal(g, want[w]) for g in got[w])


def test_block_keeps_buffers_for_the_longest_call_only():
    cal, x = calibrated()
    table = torch.arange(16, dtype=torch.int32, device="cuda").view(1, 16)

    def held_after(lengths):
        block = serve.AttentionBlock(cal, 12, 16)
        before = torch.cuda.memory_allocated()
        for n in lengths:
            chunk(block, x[:n].contiguous(), 1, n, 256, table)()
        torch.cuda.synchronize()
        return torch.cuda.memory_allocated() - before

    held_after([70])
    assert held_after(range(1, 71)) == held_after([70]) == held_after([70] + list(range(1, 70)))


def test_block_in_graphs_that_replay_side_by_side():
    cal, x = calibrated()
    block = serve.AttentionBlock(cal, 12, 64)
    tables = torch.arange(64, dtype=torch.int32, device="cuda").view(2, 4, 8)
    attends = [block.attention(4, 20, max_own=32) for _ in range(2)]
    i32 = dict(dtype=torch.int32, device="cuda")
    args = [torch.full((4,), 20, **i32), torch.arange(20, **i32).repeat(4), torch.arange(4, **i32).repeat_interleave(20)]
    inputs = [x[80 * w:80 * w + 80].contiguous() for w in range(2)]
    want = [block(inputs[w], attends[w], tables[w], *args) for w in range(2)]
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for w in range(2):
        with torch.cuda.graph(graphs[w]):
            outs.append(block(inputs[w], attends[w], tables[w], *args))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(30):
        for w in range(2):
            with torch.cuda.stream(streams[w]):
                graphs[w].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, t) for o, t in zip(outs, want))


def test_block_under_another_default_type():
    """A program that sets torch's default type to a 16-bit one: Steps are binary32 all the same."""
    cal, x = calibrated()
    block = serve.AttentionBlock(cal, 12, 4)
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    want = chunk(block, x[:10].contiguous(), 2, 5, 32, table)()
    torch.set_default_dtype(torch.bfloat16)
    try:
        got = chunk(serve.AttentionBlock(cal, 12, 4), x[:10].contiguous(), 2, 5, 32, table)()
    finally:
        torch.set_default_dtype(torch.float32)
    assert torch.equal(got, want)
