"""What a 4-bit variant holds on the device is what it says that it holds."""
import gc

import pytest
import torch

pytestmark = pytest.mark.gpu

SIZES = dict(layers=2, heads=16, kv_heads=8, head_dim=128, inner=4096, group=128, kv_group=64, page=64)


def _allocated():
    gc.collect()
    torch.cuda.synchronize()
    return torch.cuda.memory_stats()["requested_bytes.all.current"]   # without what the allocator rounds up


def test_a_model_holds_its_laid_out_weights_and_caches_only():
    from paper_2609_02109_amd import serve, step
    before = _allocated()
    model = step.Decoder(2, 500, **SIZES)
    held = _allocated() - before
    # beside them the page table and the two tables of angles
    more = 2 * 512 * 64 * 4 + 4096 + 512 * 12
    assert model.bytes <= held <= model.bytes + more
    drawn = model.drawn
    for layer, weights in zip(drawn, model.layers):
        for name, w in weights.items():
            assert torch.equal(serve.W4Weight(*layer[name]).packed, w.packed)


def test_options_hold_one_model_at_a_time():
    from paper_2609_02109_amd import step
    one = dict(SIZES, layers=8)
    step.options([1], 100, steps=1, **one)
    before = _allocated()
    torch.cuda.reset_peak_memory_stats()
    got = step.options([1, 2, 3], 100, steps=1, **one)
    peak = torch.cuda.memory_stats()["requested_bytes.all.peak"] - before
    assert max(o["gb"] for o in got) * 1e9 <= peak < 1.5e9 * max(o["gb"] for o in got)
