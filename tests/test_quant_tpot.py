"""The multi-layer decode step over 8-bit caches (paper_2606_00024_amd.tpot)."""
from __future__ import annotations

import pytest
import torch

from paper_2606_00024_amd import tpot

TINY = tpot.ModelShape("tiny", layers=2, hidden=512, q_heads=8, kv_heads=2, ffn=1024, vocab=1000)


def test_kinds():
    with pytest.raises(SystemExit):
        tpot.main(["--kv", "fp4"])


@pytest.mark.gpu
@pytest.mark.parametrize("kv", ["e4m3", "int8"])
def test_step_appends_and_attends(kv):
    """The step's attention is a direct call's on the cache that its appends
    leave, and the appended token is the projected K and V, quantised."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_00024_amd import api
    step = tpot.Step(TINY, batch=2, seq_len=4096 + 17, kv=kv)
    for mode in ("nodet", "off", "on"):
        x = step.run(mode)
        torch.cuda.synchronize()
        assert torch.isfinite(x.float()).all()
    step.append(1, step.kv0)
    step.attention("on", 1)
    got, stop = step.out.clone(), step.stop[1].clone()
    L = step.layers[1]
    wl, cache = L["wl"], L["cache"]
    ref, _, ref_stop = api.decode_attention_quant(
        wl.q, cache, wl.page_table, wl.seq_lens, block_size=wl.spec.block_size, tau=wl.spec.tau,
        phi=wl.spec.phi, patience=wl.spec.patience, softmax_scale=wl.spec.softmax_scale,
        out_dtype=torch.bfloat16)
    assert torch.equal(got, ref) and torch.equal(stop, ref_stop)
    k, _ = api.quant_read(cache, wl.page_table, step.position, rows=2, dtype=torch.float32)
    scale = cache.k_scale[wl.page_table[:, 4112 // 64].long()][:, :, 0, None]     # the runs of token 4112
    want = step.kv0[:, :2 * 128].float().view(2, 2, 128)
    # half a step: e4m3 2^-4 of the value (or half its smallest step, 2^-10), int8 half a code
    tol = torch.maximum(want.abs() * 2.0 ** -4, scale * 2.0 ** -10) if kv == "e4m3" else scale * 0.5
    assert torch.all((k - want).abs() <= tol * (1 + 1e-6))
    assert (step.time_ms("on", steps=2, warmup=1) > 0).all()
    assert 0 <= step.skipped_pct("on") <= 100
