"""Numbers that the parameter struct of the eviction cannot hold are refused, on the host, before anything else is looked at."""
import pytest
import torch


@pytest.mark.parametrize("name", ["limit", "budget", "keep_first", "keep_last"])
@pytest.mark.parametrize("value", [2 ** 31, 2 ** 32 + 100, 2 ** 63 - 1, -2 ** 31 - 1])
def test_numbers_beyond_32_bits(name, value):
    """2^32 + 100 as a limit that nobody reaches would otherwise be a limit of 100."""
    from paper_2511_14617_amd import binding
    k = torch.zeros((2, 1, 16, 64), dtype=torch.bfloat16)
    args = dict(limit=300, budget=100, keep_first=0, keep_last=0)
    args[name] = value
    with pytest.raises(ValueError, match=name + ": want a 32-bit number"):
        binding.seer_kv_evict(k, k, torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros((1, 1, 32)), **args)
