"""Devices that the serving operators' handles cannot be made on, refused before anything is allocated or called."""
import pytest
import torch

from paper_2509_22622_amd import binding as B

MADE = dict(layers=1, q_heads=4, kv_heads=2, head_dim=64, page_tokens=16, n_pages=4)


@pytest.mark.parametrize("device", ["cpu", torch.device("cpu"), "meta"])
def test_a_pool_needs_a_gpu(device):
    with pytest.raises(ValueError, match="GPU"):
        B.PagedCache(**MADE, device=device)


@pytest.mark.parametrize("device", ["cpu", "meta"])
def test_a_weight_needs_a_gpu(device):
    with pytest.raises(ValueError, match="GPU"):
        B.Linear(torch.zeros(16, 64, dtype=torch.bfloat16, device=device))
