"""A sparse feed-forward block: a router chooses a few of many gated experts for every token, y = sum of w_e (silu(x Wg_e^T) * (x Wu_e^T)) Wd_e^T.

Products run on 8-bit floating point operands with a scale for every 128 elements along the axis that they sum over; the forward pass keeps 8-bit copies by
columns for the weight gradients, and the activation's input in 8 bits.  The experts' loads are balanced by a bias that counts for the choice only.

    python -m paper_2102_04782_amd.experts        # fits a small block to another one and serves single rows with it
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import binding as daq


@dataclass
class Saved:
    plan: daq.Plan
    logits: torch.Tensor
    weights: torch.Tensor
    chosen: torch.Tensor
    x: daq.Fp8          # by columns, for the router
    x_rows: daq.Fp8     # by columns, the rows in the order of the experts
    h: daq.Ckpt8        # [rows, gate | up]
    a: daq.Fp8          # by columns, in the order of the experts
    y: torch.Tensor     # the experts' rows, for the gradients of their weights in the sum


@dataclass
class Gradients:
    x: torch.Tensor
    w_router: torch.Tensor
    w_in: torch.Tensor
    w_out: torch.Tensor


class SparseFeedForward:
    """Weights in fp32, packed anew after every update: matrices for the forward pass, their transposes for the data gradients."""

    def __init__(self, d: int, f: int, experts: int, picks: int, groups: int = 1, top_groups: int = 1, seed: int = 0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        randn = lambda *shape: torch.randn(*shape, generator=g, device=device)
        self.w_router = randn(experts, d) * d ** -0.5
        self.w_in = randn(experts, 2 * f, d) * d ** -0.5      # gate | up
        self.w_out = randn(experts, d, f) * f ** -0.5
        self.bias = torch.zeros(experts, device=device)
        self.experts, self.picks, self.groups, self.top_groups = experts, picks, groups, top_groups
        self.form = {"scores": daq.SCORES_SIGMOID, "renormalize": True, "scale": 1.0}
        self.pack()

    def pack(self):
        self.q_router, self.q_router_t = daq.fp8_quantize_weights(self.w_router)
        self.q_in, self.q_in_t = daq.fp8_quantize_weights(self.w_in)
        self.q_out, self.q_out_t = daq.fp8_quantize_weights(self.w_out)

    def choose(self, x: torch.Tensor):
        """(logits, weights, experts, plan) of the tokens ``x``."""
        logits = daq.fp8_linear(x, self.q_router, dtype=torch.float32)
        weights, chosen = daq.route(logits, self.picks, bias=self.bias, groups=self.groups, top_groups=self.top_groups, **self.form)
        return logits, weights, chosen, daq.experts_plan(chosen, self.experts)

    def forward(self, x: torch.Tensor):
        """(y, what the backward pass needs)."""
        logits, weights, chosen, plan = self.choose(x)
        x_q, x_rows = daq.experts_quantize(x, plan)
        a, h8 = daq.ckpt8_act_forward(daq.experts_matmul(x_q, self.q_in, plan, dtype=x.dtype), daq.ACT_SILU, gated=True)
        a_q, a_c = daq.experts_quantize(a, plan, sorted_rows=True)
        y = daq.experts_matmul(a_q, self.q_out, plan, sorted_rows=True, dtype=x.dtype)
        saved = Saved(plan, logits, weights, chosen, daq.fp8_quantize(x, columns=True), x_rows, h8, a_c, y)
        return daq.experts_combine(y, plan, weights), saved

    def serve(self, x: torch.Tensor) -> torch.Tensor:
        """y of a few tokens, nothing kept."""
        _, weights, _, plan = self.choose(x)
        a, _ = daq.ckpt8_act_forward(daq.experts_linear(x, self.q_in, plan), daq.ACT_SILU, gated=True)
        return daq.experts_combine(daq.experts_linear(a, self.q_out, plan, sorted_rows=True), plan, weights)

    def backward(self, dout: torch.Tensor, s: Saved) -> Gradients:
        to = dout.dtype
        dy, dweights = daq.experts_combine_backward(dout, s.y, s.plan, s.weights)
        dy_q, dy_c = daq.experts_quantize(dy, s.plan, sorted_rows=True)
        da = daq.experts_matmul(dy_q, self.q_out_t, s.plan, sorted_rows=True, dtype=to)
        dh_q, dh_c = daq.experts_quantize(daq.ckpt8_act_backward(da, s.h, daq.ACT_SILU), s.plan, sorted_rows=True)
        dx = daq.experts_combine(daq.experts_matmul(dh_q, self.q_in_t, s.plan, sorted_rows=True, dtype=to), s.plan)
        dl_q, dl_c = daq.fp8_quantize_both(daq.route_backward(dweights, s.logits, s.chosen, **self.form))
        dx += daq.fp8_matmul(dl_q, self.q_router_t, dtype=to)
        return Gradients(dx, daq.fp8_matmul(dl_c, s.x, dtype=torch.float32), daq.experts_weight_grad(dh_c, s.x_rows, s.plan),
                         daq.experts_weight_grad(dy_c, s.a, s.plan))

    def update(self, g: Gradients, rate: float):
        self.w_router -= rate * g.w_router
        self.w_in -= rate * g.w_in
        self.w_out -= rate * g.w_out
        self.pack()

    def balance(self, plan: daq.Plan, rate: float = 0.001):
        """Experts with fewer rows than the mean are favoured from now on."""
        counts = plan.counts.float()
        self.bias += rate * torch.sign(counts.mean() - counts)


def main(d: int = 256, f: int = 256, experts: int = 8, picks: int = 2, tokens: int = 1024, steps: int = 60):
    block, goal = SparseFeedForward(d, f, experts, picks, seed=1), SparseFeedForward(d, f, experts, picks, seed=2)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    for step in range(steps):
        x = torch.randn(tokens, d, generator=g, device="cuda").to(torch.bfloat16)
        y, saved = block.forward(x)
        off = y.float() - goal.forward(x)[0].float()
        block.update(block.backward((off / tokens).to(torch.bfloat16), saved), rate=1.0)
        block.balance(saved.plan)
        if step % 10 == 0 or step == steps - 1:
            print(f"step {step:3d}  mean squared difference {float(off.square().mean()):.4f}  rows of the experts {saved.plan.counts.tolist()}", flush=True)
    one = torch.randn(1, d, generator=g, device="cuda").to(torch.bfloat16)
    print("one row:", [round(v, 3) for v in block.serve(one)[0, :6].tolist()], "goal:", [round(v, 3) for v in goal.serve(one)[0, :6].tolist()])


if __name__ == "__main__":
    main()
