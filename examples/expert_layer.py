"""A layer of experts with low-rank adapters, trained for a few steps and then served one token at a time.

    python examples/expert_layer.py [steps]

Tokens choose two of eight experts (topk_route), are sorted by expert (Routing), go through the experts' two matrices
(matmul) and come back as weighted sums (combine); the gradients take the same way back.  Serving adds every request's
own adapter beside the projection that all share.  Prints the loss of every training step and how far a served step is
from the same layer in plain torch.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_20855_gb300 import DeviceCSR, Routing, adapters, topk_route, topk_route_backward  # noqa: E402

T, H, F, E, K = 1024, 256, 512, 8, 2  # tokens, width, experts' inner width, experts, experts a token


def one_expert(rows: int) -> DeviceCSR:
    """The routing matrix of a projection that all rows share."""
    return DeviceCSR(rows, 1, torch.arange(rows + 1, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda"),
                     torch.ones(rows, device="cuda"))


class Layer:
    def __init__(self, seed: int = 0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def normal(*shape, scale):
            return torch.randn(shape, generator=g, device="cuda") * scale

        # 32-bit masters; the products take 16-bit copies
        self.master = {"router": normal(E, H, scale=H ** -0.5), "up": normal(E, F, H, scale=H ** -0.5),
                       "down": normal(E, H, F, scale=F ** -0.5)}

    def weights(self):
        return {n: w.to(torch.bfloat16) for n, w in self.master.items()}

    def forward(self, x):
        w = self.weights()
        every = Routing(one_expert(x.shape[0]))
        logits = every.matmul(x, w["router"][None])
        R = topk_route(logits, K)
        plan = Routing(R)
        xs = plan.dispatch(x)
        up = plan.matmul(xs, w["up"])
        act = torch.relu(up)
        ys = plan.matmul(act, w["down"])
        return plan.combine(ys), (w, logits, R, plan, x, xs, up, act, ys, every)

    def backward(self, grad_y, kept):
        w, logits, R, plan, x, xs, up, act, ys, every = kept
        grad_ys, grad_vals = plan.combine_backward(grad_y, ys)
        grad_act, grad_down = plan.matmul_backward(grad_ys, act, w["down"])
        grad_xs, grad_up = plan.matmul_backward(grad_act * (up > 0), xs, w["up"])
        grad_logits = topk_route_backward(logits, R, grad_vals)
        grad_x, grad_router = every.matmul_backward(grad_logits, x, w["router"][None])
        return grad_x + plan.dispatch_backward(grad_xs), {"router": grad_router[0], "up": grad_up, "down": grad_down}


def train(layer: Layer, steps: int) -> list[float]:
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn((T, H), generator=g, device="cuda").to(torch.bfloat16)
    goal = torch.roll(x, 1, 1).float() * (x.float().mean(1, keepdim=True) > 0)
    losses = []
    for _ in range(steps):
        y, kept = layer.forward(x)
        off = y.float() - goal
        _, grads = layer.backward((off * (2 / off.numel())).to(torch.bfloat16), kept)
        # read back together: the loss, and whether a product's kernel gave up a wait (its result would be incomplete)
        loss, gave_up = torch.stack([off.square().mean(), (kept[3].status | kept[-1].status).float()[0]]).tolist()
        if gave_up:
            raise RuntimeError("a product's kernel gave up a wait")
        losses.append(loss)
        for name, grad in grads.items():
            layer.master[name] -= 20.0 * grad.float()
    return losses


def serve(layer: Layer, requests: int = 5, rank: int = 16) -> float:
    """One step of `requests` tokens, each with its own adapter beside a shared projection of the layer's output."""
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    x = torch.randn((requests, H), generator=g, device="cuda").to(torch.bfloat16)
    proj = (torch.randn((1, H, H), generator=g, device="cuda") * H ** -0.5).to(torch.bfloat16)
    A = (torch.randn((requests, rank, H), generator=g, device="cuda") * H ** -0.5).to(torch.bfloat16)
    B = (torch.randn((requests, H, rank), generator=g, device="cuda") * rank ** -0.5).to(torch.bfloat16)
    S = DeviceCSR(requests, requests, torch.arange(requests + 1, device="cuda"),
                  torch.arange(requests, dtype=torch.int32, device="cuda"), torch.full((requests,), 0.5, device="cuda"))
    y, (w, logits, R, *rest) = layer.forward(x)
    shared = Routing(one_expert(requests))
    base = shared.matmul(y, proj)
    out = adapters(y, A, B, S, base, out=base, wait=True)
    for plan in (rest[0], rest[-1], shared):
        plan.wait()

    cols, vals = R.colidx.view(-1, K).long(), R.vals.view(-1, K)
    want = torch.zeros((requests, H), device="cuda")
    for j in range(K):
        up = torch.einsum("th,tfh->tf", x.float(), w["up"].float()[cols[:, j]])
        want += vals[:, j, None] * torch.einsum("tf,thf->th", torch.relu(up), w["down"].float()[cols[:, j]])
    delta = torch.einsum("thr,tr->th", B.float(), torch.einsum("th,trh->tr", want, A.float()))
    want = want @ proj[0].float().T + 0.5 * delta
    return float((out.float() - want).norm() / want.norm())


def main(steps: int = 20) -> tuple[list[float], float]:
    layer = Layer()
    losses = train(layer, steps)
    for i, loss in enumerate(losses):
        print(f"step {i:3d}  loss {loss:.4f}")
    off = serve(layer)
    print(f"served step: relative distance from plain torch {off:.2e}")
    return losses, off


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 20)
