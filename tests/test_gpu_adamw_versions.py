"""A step writes parameters and copies in place: autograd is told so, as by any operation of torch."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 32])
def test_a_graph_of_the_old_values_is_refused(bits):
    from paper_2606_20855_gb300 import AdamW
    master = torch.ones(300, device="cuda").requires_grad_()
    half = torch.ones(300, dtype=torch.bfloat16, device="cuda")
    x = torch.ones(300, dtype=torch.bfloat16, device="cuda").requires_grad_()
    opt = AdamW([master], bits=bits, copies=[half])
    for value in ((master * master).sum(), (x * half).sum()):  # both keep what the step is about to write
        opt.step([torch.ones(300, dtype=torch.bfloat16, device="cuda")])
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            value.backward()


def test_only_what_was_written():
    from paper_2606_20855_gb300 import AdamW
    params = [torch.ones(n, device="cuda") for n in (5, 300, 7)]
    copies = [torch.ones(5, dtype=torch.float16, device="cuda"), None, torch.ones(7, dtype=torch.float16, device="cuda")]
    opt = AdamW(params, copies=copies)
    tensors = [*params, copies[0], copies[2]]

    def moved(grads):
        before = [t._version for t in tensors]
        opt.step(grads)
        return [t._version > b for t, b in zip(tensors, before)]

    grads = [torch.ones(p.numel(), device="cuda") for p in params]
    assert moved(grads) == [True] * 5
    assert moved([None, grads[1], None]) == [False, True, False, False, False]
    assert moved([grads[0], None, None]) == [True, False, False, True, False]
    assert moved([None, None, None]) == [False] * 5
