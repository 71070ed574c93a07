"""Adapters at the limits of their sizes: rank 0 with many tokens, rows of 2^24 values."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu


def _one(T, L=1):
    """Every token has adapter 0, with value 1."""
    from paper_2606_20855_gb300 import DeviceCSR
    return DeviceCSR(T, L, torch.arange(T + 1, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda"), torch.ones(T, device="cuda"))


@pytest.mark.parametrize("T", [512, 513, 65_535, 65_536, 200_000])
@pytest.mark.parametrize("N", [8, 13])
def test_rank_zero(T, N):
    """Nothing is added, whatever the number of tokens."""
    from paper_2606_20855_gb300 import adapters
    bf = torch.bfloat16
    base = torch.randn((T, N), device="cuda").to(bf)
    x, A, B = torch.ones((T, 16), dtype=bf, device="cuda"), torch.empty((1, 0, 16), dtype=bf, device="cuda"), torch.empty((1, N, 0), dtype=bf, device="cuda")
    assert torch.equal(adapters(x, A, B, _one(T), base, wait=True), base)
    assert not bool(adapters(x, A, B, _one(T), wait=True).any())


@pytest.mark.parametrize("T", [3, 520])
def test_longest_rows(T):
    from paper_2606_20855_gb300 import adapters
    N, r, K, bf = 1 << 24, 16, 16, torch.bfloat16
    x, A = torch.ones((T, K), dtype=bf, device="cuda"), torch.zeros((1, r, K), dtype=bf, device="cuda")
    A[0, 0, 0] = 1.0  # the only inner product that is not zero is 1
    B = torch.zeros((1, N, r), dtype=bf, device="cuda")
    B[0, :, 0] = (torch.arange(N, device="cuda") % 251).to(bf)
    y = adapters(x, A, B, _one(T), wait=True)
    assert torch.equal(y[0], B[0, :, 0]) and torch.equal(y[-1], B[0, :, 0])
