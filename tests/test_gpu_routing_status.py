"""What a kernel that gives up a wait leaves to be read.  No wait runs out here: the word that the kernel would set is set by the test."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu


def _word(address):
    """An int32 tensor at an address of the GPU."""
    class At:
        __cuda_array_interface__ = {"shape": (1,), "typestr": "<i4", "data": (address, False), "version": 3}
    return torch.as_tensor(At(), device="cuda")


def _adapters_case(T):
    from paper_2606_20855_gb300 import DeviceCSR
    bf = torch.bfloat16
    S = DeviceCSR(T, 1, torch.arange(T + 1, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda"), torch.ones(T, device="cuda"))
    return torch.ones((T, 32), dtype=bf, device="cuda"), torch.ones((1, 16, 32), dtype=bf, device="cuda"), \
        torch.ones((1, 24, 16), dtype=bf, device="cuda"), S


def test_plan():
    from paper_2606_20855_gb300 import Routing, _abi, topk_route
    R = topk_route(torch.randn((50, 8), device="cuda"), 2)
    plan = Routing(R)
    assert plan.status.tolist() == [0] and plan.status.dtype == torch.int32
    plan.wait()
    plan.status.fill_(1)
    xs, W = torch.ones((100, 16), dtype=torch.bfloat16, device="cuda"), torch.ones((8, 16, 16), dtype=torch.bfloat16, device="cuda")
    plan.matmul(xs, W)  # a later product does not clear it
    with pytest.raises(_abi.WsError) as e:
        plan.wait()
    assert e.value.status_name == "WS_ERR_DEVICE"
    assert plan.offsets[-1] == 100 and Routing(R).status.tolist() == [0]


@pytest.mark.parametrize("shape", [(), (1,), (1, 1)])
def test_adapters_keep_it_where_the_caller_says(monkeypatch, shape):
    from paper_2606_20855_gb300 import _abi, adapters
    few, many = _adapters_case(20), _adapters_case(700)
    status = torch.zeros(shape, dtype=torch.int32, device="cuda")
    want = adapters(*many)
    for case in (few, many):
        adapters(*case, status=status, wait=True)
    assert int(status) == 0
    call = _abi.ws_adapters

    def gives_up(packed, scratch, size, stream):
        call(packed, scratch, size, stream)
        _word(scratch).fill_(1)

    with monkeypatch.context() as m:
        m.setattr(_abi, "ws_adapters", gives_up)
        adapters(*many, status=status)
        with pytest.raises(_abi.WsError):
            adapters(*many, wait=True)
    assert torch.equal(adapters(*many, status=status), want)  # and keeps it
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    adapters(*many, stream=s, status=status)
    s.synchronize()
    assert int(status) == 1


def test_a_status_that_cannot_hold_it_is_refused():
    from paper_2606_20855_gb300 import adapters
    for bad in (torch.zeros(1, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32)):
        with pytest.raises(TypeError):
            adapters(*_adapters_case(20), status=bad)
