"""What the binding refuses before a call, without a GPU."""
import pytest
import torch

from paper_2609_34606_b200 import hsa


def test_rotation_of_more_tokens_than_32_bits_count():
    """Nothing of the tensor is read: it is one row, seen 2^32 + 3 times.  (Cut down to 32 bits that would be 3 tokens.)"""
    r = hsa.RotaryPositions(8, device="cpu")
    for n in ((1 << 32) + 3, 1 << 31):
        x = torch.zeros(1, 1, 8, dtype=torch.bfloat16).expand(n, 1, 8)
        with pytest.raises(ValueError, match="2\\^31"):
            hsa.hsa_rope(x, x, r.args(None, n))


def test_most_rows_of_more_than_32_bits(monkeypatch):
    cache = object.__new__(hsa.KV8Cache)
    cache.ctx, cache._index, cache.head_dim, cache.device = None, -1, 64, torch.device("cpu")
    monkeypatch.setattr(hsa, "_on_current", lambda t, name: None)
    t, held = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    assert cache._rows(t, 2, held, None, 3, "k") == 3 and cache._rows(t, 2, held, None, None, "k") == 1
    with pytest.raises(ValueError, match="2\\^31"):
        cache._rows(t, 2, held, None, (1 << 32) + 1, "k")
