"""The binding of the attention half of a layer: errors for layouts that no cache can have (CPU tensors that pass for device ones, a
library that is not to be reached)."""
import pytest


@pytest.mark.parametrize("other", [dict(head_dim=0), dict(head_dim=96), dict(head_dim=-64), dict(kv_heads=0), dict(kv_heads=-2, page_tokens=-32), dict(kv_heads=1025), dict(kv_heads=2**40), dict(page_tokens=0), dict(page_tokens=96),
                                   dict(page_tokens=2**17), dict(page_tokens=2**36)])
def test_layouts_that_no_cache_can_have_are_refused(monkeypatch, other):
    import torch

    from paper_2603_27914_amd import binding

    monkeypatch.setattr(binding, "_need_here", lambda *t: None)
    monkeypatch.setattr(binding, "_stream", lambda: pytest.fail("the library was called"))
    f16, i32 = torch.float16, torch.int32

    class Bytes:  # as many as the layout needs
        dtype = torch.uint8

        def __init__(self, n):
            self.n = n

        def numel(self):
            return self.n

        def is_contiguous(self):
            return True

        def data_ptr(self):
            return 256

    layout = {"page_tokens": 32, "kv_heads": 2, "head_dim": 64, **other}
    cache = binding.Cache(Bytes(layout["kv_heads"] * (layout["page_tokens"] // 32) * (32 * layout["head_dim"] + 128)), **layout)
    x, slots = torch.zeros((3, 128), dtype=f16), torch.zeros(3, dtype=torch.int64)
    for call in (lambda: binding.itq3s_cache_append(x, x, x, cache=cache, slots=slots), lambda: binding.itq3s_cache_read(cache, slots),
                 lambda: binding.itq3s_cache_attention(x, cache, torch.zeros(2, dtype=i32), torch.zeros(1, dtype=i32), torch.zeros((1, 1), dtype=i32))):
        with pytest.raises(binding.Itq3sError):
            call()
