"""The attention half of a calibrated layer as a server drives it: recalibration under it, wrong shapes, ragged lengths,
several streams."""
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
