"""eps between 0 and the smallest normal number of 32 bits is refused: the reciprocal takes it for 0, and 0 / eps would be NaN."""
from __future__ import annotations

import pytest

from paper_2606_20855_gb300 import _abi
from paper_2606_20855_gb300 import build as pkg_build
from tests.test_fused_abi_cpu import ADAMW, P


@pytest.mark.parametrize("eps", [5e-324, 1e-46, 1e-40, 1.1e-38])
def test_refused(eps):
    pkg_build.build()
    _abi.load()
    with pytest.raises(_abi.WsError, match="eps") as e:
        _abi.ws_adamw(_abi.ADAMW_CALL.pack(*{**ADAMW, "tensors": P, "grads": P, "count": 0, "eps": eps}.values()), 0)
    assert e.value.status_name == "WS_ERR_INVALID_ARG"


@pytest.mark.gpu
def test_smallest():
    """The smallest eps there is: nothing learnt, nothing changed; and at 0 a quotient of its own."""
    import torch

    from paper_2606_20855_gb300 import AdamW
    for eps in (1e-40, 1e-46):
        with pytest.raises(ValueError, match="eps"):
            AdamW([torch.ones(300, device="cuda")], eps=eps)
    p = torch.ones(300, device="cuda")
    opt = AdamW([p], lr=0.5, eps=1.2e-38, weight_decay=0.0)
    opt.step([torch.zeros(300, device="cuda")])
    assert bool((p == 1).all())
    grad = torch.full((300,), 0.25, device="cuda")
    first = torch.ones(300, device="cuda")
    AdamW([first], lr=0.5, eps=0.0, weight_decay=0.0).step([grad])
    assert bool(((first - 0.5).abs() < 1e-6).all())  # m / sqrt(v) is 1 in the first step, off by a few times 2^-22
