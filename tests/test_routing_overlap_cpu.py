"""Whether a result given by the caller shares memory with an input: views of one buffer, on the CPU."""
from __future__ import annotations

import pytest
import torch

from paper_2606_20855_gb300.routing import _overlap

BUF = torch.zeros(6, 40)


@pytest.mark.parametrize("a,b,meet", [
    (BUF[:3], BUF[3:], False),
    (BUF[:4], BUF[3:], True),
    (BUF[:, :16], BUF[:, 16:32], False),   # column blocks
    (BUF[:, :16], BUF[:, 15:32], True),
    (BUF[:, 20:], BUF[:, :20], False),
    (BUF[::2, :16], BUF[1::2, :16], False),  # every other row
    (BUF[::2, :16], BUF[:, 16:], False),
    (BUF[::2, :16], BUF[:, 15:], True),
    (BUF[:, 8:16], BUF[2, 4:8], False),      # a row of one in the gap of the other's
    (BUF[:, 8:16], BUF[2, 4:9], True),
    (BUF[:, :16], BUF.view(-1)[:41], True),
    (BUF.view(3, 2, 40)[:, :, :8], BUF[:, 8:], False),  # a stack of matrices
    (BUF.view(3, 2, 40)[:, :, :9], BUF[:, 8:], True),
    (BUF[:0], BUF, False),
    (BUF, BUF, True),
    (BUF, torch.zeros(6, 40), False),
])
def test_overlap(a, b, meet):
    assert _overlap(a, b) is meet and _overlap(b, a) is meet
    # against the addresses themselves
    def places(t):
        return set((torch.arange(BUF.numel() * 4).as_strided(t.shape, t.stride(), t.storage_offset())).flatten().tolist()) \
            if t.untyped_storage().data_ptr() == BUF.untyped_storage().data_ptr() else set()
    assert bool(places(a) & places(b)) is meet
