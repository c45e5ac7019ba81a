"""A prefill whose compaction goes to pages (CPU): what it says of the padded blocks that it does not have."""
import pytest
import torch

from paper_2412_14838_amd.pages import PagedCache
from paper_2412_14838_amd.pipeline import Compressor
from paper_2412_14838_amd.workloads import Workload

CFG = Workload(name="paged", L=2, Hq=4, Hkv=2, d=64, seqlens=(40, 60), dtype="bf16", w=16, P=7, mean_budget=16, layer_max=64, interval=2, seed=1)


def test_calls_over_the_padded_blocks_say_where_the_rows_are(monkeypatch):
    monkeypatch.setattr(PagedCache, "_on", lambda self, call, *args: None)
    without = Compressor(CFG, device="cpu", keep_cache=False)
    paged = Compressor(CFG, device="cpu", pages=PagedCache(without.desc, n_pages=4, device="cpu"))
    q, out = torch.zeros(2, 2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 4, 64)
    for comp, why in ((paged, "PagedCache"), (without, "keep_cache")):
        for call in (comp.pack, lambda: comp.decode_attention(0, q[0], out[0]), lambda: comp.decode_attention_layers(0, 2, q, out),
                     lambda: comp.gather(0, q, q), lambda: comp.gather_layers(0, [q], [q])):
            with pytest.raises(AttributeError, match=why):
                call()
        assert not hasattr(comp, "kb") and not hasattr(comp, "anything_else")
        with pytest.raises(AttributeError, match="anything_else"):
            comp.anything_else
    assert Compressor(CFG, device="cpu").kb.shape == (2, 2, 2, 80, 64)
