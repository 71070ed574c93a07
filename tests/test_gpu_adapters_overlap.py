"""Results of the adapters that the caller gives: apart from what is read, in one buffer with it or not."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu


def _inputs(T, dt=torch.bfloat16):
    from paper_2606_20855_gb300 import DeviceCSR
    g = torch.Generator(device="cuda").manual_seed(T)
    L, r, K, N = 3, 16, 64, 64

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(dt)
    col = (torch.arange(T, device="cuda") % L).to(torch.int32)
    return normal(T, 3 * K), normal(L, r, K), normal(L, N, r), DeviceCSR(T, L, torch.arange(T + 1, device="cuda"), col, torch.ones(T, device="cuda"))


@pytest.mark.parametrize("T", [20, 700])
def test_column_blocks_of_one_buffer(T):
    """x, base and the result side by side."""
    from paper_2606_20855_gb300 import adapters
    wide, A, B, S = _inputs(T)
    want = adapters(wide[:, :64].clone(), A, B, S, wide[:, 64:128].clone())
    assert adapters(wide[:, :64], A, B, S, wide[:, 64:128], out=wide[:, 128:]).data_ptr() == wide[:, 128:].data_ptr()
    assert torch.equal(wide[:, 128:], want)


@pytest.mark.parametrize("T", [20, 700])
def test_shared_memory_is_refused(T):
    from paper_2606_20855_gb300 import DeviceCSR, adapters
    wide, A, B, S = _inputs(T)
    x = wide[:, :64].contiguous()
    with pytest.raises(ValueError, match="x"):
        adapters(x, A, B, S, out=x)
    with pytest.raises(ValueError, match="x"):
        adapters(wide[:, :64], A, B, S, out=wide[:, 63:127])
    room = torch.zeros(T * 64 + A.numel() + B.numel(), dtype=torch.bfloat16, device="cuda")
    out = room[:T * 64].view(T, 64)
    for at, name in ((8, "A"), (T * 64 - 8, "B")):
        inside = [room[at:at + t.numel()].view(t.shape) if n == name else t for t, n in ((A, "A"), (B, "B"))]
        with pytest.raises(ValueError, match=name):
            adapters(x, *inside, S, out=out)
    vals = room.view(torch.float32)[:T]
    with pytest.raises(ValueError, match="S"):
        adapters(x, A, B, DeviceCSR(T, 3, S.rowptr, S.colidx, vals), out=out)
