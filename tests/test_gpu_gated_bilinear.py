"""Gated blocks whose gate is the sum itself (WS_ACT_NONE, at the C entry alone): h = gate * up and its gradients."""
from __future__ import annotations

import pytest
import torch

from tests._fused import E32, TYPES, kept, near, plan_of, product, randn, spans

pytestmark = pytest.mark.gpu


def calls(plan, xs, Wg, Wu, bg, bu, gh):
    """h, gate, up and the gradients of xs, Wg, Wu, bg and bu, by ws_routing_gated and ws_routing_gated_backward."""
    from paper_2606_20855_gb300 import _abi
    (E, F, K), Z, dt = Wg.shape, xs.shape[0], xs.dtype
    code = {torch.bfloat16: _abi.WS_BF16, torch.float16: _abi.WS_F16}[dt]
    stream = torch.cuda.current_stream().cuda_stream

    def room(*shape):
        return torch.full(shape, 777.0, dtype=dt, device="cuda")

    h, gate, up, gxs, gWg, gWu, gbg, gbu = (room(*s) for s in ((Z, F), (Z, F), (Z, F), (Z, K), (E, F, K), (E, F, K), (E, F), (E, F)))
    w = (Wg.data_ptr(), K, F * K, Wu.data_ptr(), K, F * K)
    _abi.ws_routing_gated(plan._r, _abi.GATED_CALL.pack(F, K, xs.data_ptr(), K, *w, bg.data_ptr(), F, bu.data_ptr(), F, h.data_ptr(), F,
                                                        gate.data_ptr(), F, up.data_ptr(), F, code, 0), 0, 0, stream)
    need = _abi.ws_routing_gated_backward_scratch(Z, E, F, True)
    scratch = torch.full((need,), 0x7f, dtype=torch.uint8, device="cuda")
    _abi.ws_routing_gated_backward(plan._r, _abi.GATED_BACKWARD_CALL.pack(
        F, K, gh.data_ptr(), F, gate.data_ptr(), F, up.data_ptr(), F, xs.data_ptr(), K, *w, gxs.data_ptr(), K, gWg.data_ptr(), K, F * K,
        gWu.data_ptr(), K, F * K, gbg.data_ptr(), F, gbu.data_ptr(), F, code, 0), scratch.data_ptr(), need, stream)
    plan.wait()
    return h, gate, up, gxs, gWg, gWu, gbg, gbu


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("counts", [[1, 0, 2], [40, 0, 21, 5], [150, 260]])
def test_gradients(dt, counts):
    Z, E, F, K = sum(counts), len(counts), 136, 72
    plan, xs, gh = plan_of(counts), randn((Z, K), dt, 1), randn((Z, F), dt, 6)
    Wg, Wu, bg, bu = randn((E, F, K), dt, 2, 0.3), randn((E, F, K), dt, 3, 0.3), randn((E, F), dt, 4), randn((E, F), dt, 5)
    h, gate, up, gxs, gWg, gWu, gbg, gbu = calls(plan, xs, Wg, Wu, bg, bu, gh)
    for e, q in enumerate(spans(counts)):
        x, wg, wu, g = xs[q].double(), Wg[e].double(), Wu[e].double(), gh[q].double()
        z, z_off = product(x, wg, bg[e].double(), K)
        u, u_off = product(x, wu, bu[e].double(), K)
        near(gate[q], z, z_off, dt, "gate")
        near(up[q], u, u_off, dt, "up")
        near(h[q], z * u, u.abs() * z_off + z.abs() * u_off + z_off * u_off + E32 * (z * u).abs(), dt, "h")
        z, u = gate[q].double(), up[q].double()  # as they were kept
        dg, du = g * u, g * z
        dg_sure, du_sure = 2 * E32 * dg.abs(), 2 * E32 * du.abs()
        dg_off, du_off = kept(dg, dg_sure, dt), kept(du, du_sure, dt)
        mass = (dg.abs() + dg_off) @ wg.abs() + (du.abs() + du_off) @ wu.abs()
        near(gxs[q], dg @ wg + du @ wu, dg_off @ wg.abs() + du_off @ wu.abs() + 2 * F * E32 * mass, dt, "gxs")
        n = x.shape[0]
        for got, d, off in ((gWg, dg, dg_off), (gWu, du, du_off)):
            near(got[e], d.T @ x, off.T @ x.abs() + n * E32 * ((d.abs() + off).T @ x.abs()), dt, "gW")
        for got, d, sure in ((gbg, dg, dg_sure), (gbu, du, du_sure)):
            near(got[e], d.sum(0), sure.sum(0) + (n + 1) * E32 * (d.abs() + sure).sum(0), dt, "gbias")
