"""What the binding refuses before a library call is made, on the host."""
import pytest
import torch

from paper_2602_09323_b200 import binding, build


def test_a_cache_on_the_host_is_refused():
    build.build()
    n = binding.load_library().coopt_cache_bytes(4, 2, 64, binding.KV_FP8_E4M3)
    with pytest.raises(ValueError, match="CUDA"):
        binding.Cache(4, 2, 64, data=torch.zeros(n, dtype=torch.uint8))
    for wrong in (torch.zeros(n + 1, dtype=torch.uint8), torch.zeros(n, dtype=torch.int8), torch.zeros(2, n, dtype=torch.uint8).t()[:, 0]):
        with pytest.raises(ValueError):
            binding.Cache(4, 2, 64, data=wrong)
