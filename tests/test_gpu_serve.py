"""The attention half of a calibrated decoder layer, run with the library's own products, cache and attention,
against the same layer built from its de-quantised codes in binary64."""
import pytest
import torch

from paper_2311_01305_b200 import aweq, calibrate, serve, synth

pytestmark = pytest.mark.gpu


def dequantised(cal, name):
    o = cal.out[name]
    return (o["codes"].double() - o["zp"].double()[:, None]) * o["step"].double()[:, None], o["bias_f32"].double()


def quantised(x, rinv):
    """Eq. 1-2 per token in the library's own arithmetic, de-quantised in binary64."""
    n = x.shape[0]
    codes, step, zp = torch.empty(x.shape, dtype=torch.uint8, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    aweq.aweq_quant_act(x.contiguous(), rinv, 8, aweq.PER_ROW, None, codes, step, zp)
    return (codes.double() - zp.double()[:, None]) * step.double()[:, None]


@pytest.mark.parametrize("with_rope", [True, False])
def test_attention_block_matches_its_dequantised_layer(with_rope):
    wl = synth.workloads(1.0 / 512)["opt125m_model_w8a8"]
    X, W = synth.generate(wl, "cuda")
    cal = calibrate.LayerCalibrator(wl, 8, X, W)
    cal.run()
    n_heads, d, page, prefix, n_seq, steps = 12, 64, 16, 70, 5, 3
    rope = aweq.aweq_rope_table(d, 128) if with_rope else None
    block = serve.AttentionBlock(cal, n_heads, 5 + n_seq, page, rope)
    order = torch.randperm(5 + n_seq, device="cuda").to(torch.int32)
    prefix_pages, table = order[:5], order[5:].view(n_seq, 1)
    i32 = dict(dtype=torch.int32, device="cuda")
    x0, x = X["attn_in"][:prefix], X["attn_in"][prefix:prefix + n_seq * steps].view(n_seq, steps, -1)
    st = aweq.new_status()
    got0 = block(x0, block.attention(1, prefix, max_own=prefix), prefix_pages.view(1, -1), torch.tensor([prefix], **i32),
                 torch.arange(prefix, **i32), torch.zeros(prefix, **i32), st)
    attend = block.attention(n_seq, 1, prefix_pages, prefix, page)
    got = [block(x[:, t].contiguous(), attend, table, torch.full((n_seq,), t + 1, **i32), torch.full((n_seq,), prefix + t, **i32),
                 torch.arange(n_seq, **i32), st) for t in range(steps)]
    assert aweq.read_out_of_range(st) == 0 and aweq.read_status(st)["wait_timeout"] == 0

    def rotate(y, pos):
        if rope is None:
            return y
        cs = rope.double()[pos][:, None]
        c, s, a, b = cs[..., :d // 2], cs[..., d // 2:], y[..., :d // 2], y[..., d // 2:]
        return torch.cat([a * c - b * s, a * s + b * c], -1)
    # 2^-11 per rounding to fp16: of q, k, v (three of them enter a score or a value), of the probabilities and of
    # the attended values; the last may move 8-bit codes of the o input by one step (2^-8 of a row's range each,
    # hardly any row has more than a few): a percent of the output's norm is far above all of it
    for b in range(n_seq):
        z = torch.cat([x0, x[b]])
        zq = quantised(z, cal.out["attn_in"]["rinv"])
        q, k, v = ((zq @ w.t() + bias).view(-1, n_heads, d) for w, bias in (dequantised(cal, n) for n in ("q", "k", "v")))
        pos = torch.arange(z.shape[0], device="cuda")
        score = torch.einsum("ihd,jhd->hij", rotate(q, pos), rotate(k, pos)) * d ** -0.5
        p = torch.softmax(score.masked_fill(pos[None, None] > pos[None, :, None], float("-inf")), -1)
        att = torch.einsum("hij,jhd->ihd", p, v).flatten(1).to(torch.float16)
        w, bias = dequantised(cal, "o")
        want = quantised(att, cal.out["o_in"]["rinv"]) @ w.t() + bias
        have = torch.cat([got0, torch.stack([g[b] for g in got])]).double()
        assert ((have - want).norm() / want.norm()).item() < 0.01


def test_the_example_runs(capsys):
    serve.main(n_seq=4, prefix=100, steps=3)
    line = capsys.readouterr().out
    assert "4 sequences after a prefix of 100 tokens" in line
    assert float(line.split("at most ")[1].split()[0]) < 0.2


def test_block_refuses_other_workloads():
    wl = synth.workloads(1.0 / 4096)["llama7b_layer_w4w3_g128"]
    X, W = synth.generate(wl, "cuda")
    with pytest.raises(ValueError):
        serve.AttentionBlock(calibrate.LayerCalibrator(wl, 4, X, W), 32, 4)
