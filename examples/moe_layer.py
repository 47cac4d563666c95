"""A Mixture-of-Experts layer on the library's operators, trained for a few steps.

    python examples/moe_layer.py [--steps 40] [--tokens 4096] [--dtype bf16]

One layer y_t = sum over a token's k experts of p_te W2_e (silu(g) * u), (g, u) =
W1_e x_t, with the DO-loss's surrogate added to the training loss:

    router scores -> do_fused          signatures F, distances D and the DO-loss
    signatures    -> do_expert_rows    the chosen experts' rows
    x, W1, p      -> do_expert_swiglu  gated activation; g and u kept in 8 bits
    h, W2         -> do_expert_matmul, do_expert_combine
    p, F, D       -> do_surrogate      loss and its gradient with respect to p

Backward: do_expert_swiglu_grad from the 8-bit values, do_expert_weight_grad for
both weights, and do_expert_matmul with the transposed W1 summed over the experts
for x.  Without gradients (serving) nothing is kept.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_32398_amd as dl  # noqa: E402


class _Experts(torch.autograd.Function):
    """(y, surrogate loss) of tokens x [N, H], probabilities p [N, E] and router scores [N, E].  training: keep
    what the backward pass reads (within a Function one cannot tell: the inputs say whether they require
    gradients, not whether any are recorded)."""

    @staticmethod
    def forward(ctx, x, p, scores, w1, w2, k, training):
        N = x.shape[0]
        bits, D, _ = dl.do_fused(scores[None], k, want_bits=True)
        rows = dl.do_expert_rows(bits, N, k)
        h, kept = dl.do_expert_swiglu(x, w1, rows, p, checkpoint=training)
        y = dl.do_expert_combine(dl.do_expert_matmul(h, w2, rows), rows)
        loss, dloss = dl.do_surrogate(p[None], k, bits, D, want_grad=training)
        if training:
            ctx.save_for_backward(x, p, w1, w2, dloss[0], *rows, *kept)
        return y, loss[0].float()

    @staticmethod
    def backward(ctx, dy, dl_do):
        if torch.is_grad_enabled():  # create_graph: the gradients' own derivatives would be left out silently
            raise RuntimeError("the experts' operators have no second derivative")
        x, p, w1, w2, dloss, *rest = ctx.saved_tensors
        rows, kept, dy = dl.ExpertRows(*rest[:-2]), dl.Act8(*rest[-2:]), dy.contiguous()
        da, h, dp = dl.do_expert_swiglu_grad(dy, w2, rows, kept, p)
        dw2 = dl.do_expert_weight_grad(dy, h, rows, gather_dy=True)
        dw1 = dl.do_expert_weight_grad(da, x, rows, gather_x=True)
        dx = dl.do_expert_combine(dl.do_expert_matmul(da, w1, rows, transposed=True), rows)
        return dx, dp + (dl_do * dloss).to(dp.dtype), None, dw1.to(w1.dtype), dw2.to(w2.dtype), None, None


class MoELayer(torch.nn.Module):
    """Router and experts: H wide, E experts of width F, k a token."""

    def __init__(self, H, F, E, k, dtype=torch.bfloat16, device="cuda", seed=0):
        super().__init__()
        g = torch.Generator()
        g.manual_seed(seed)

        def weight(*shape, fan):
            return torch.nn.Parameter((torch.randn(*shape, generator=g) * fan ** -0.5).to(device, dtype))

        self.k = k
        self.router = weight(E, H, fan=H)
        self.w1 = weight(E, 2 * F, H, fan=H)
        self.w2 = weight(E, H, F, fan=F)

    def forward(self, x):
        """y [N, H] and the surrogate loss of x [N, H]."""
        scores = torch.nn.functional.linear(x, self.router).float()
        p = torch.softmax(scores, dim=1)
        training = torch.is_grad_enabled() and any(t.requires_grad for t in (x, p, self.w1, self.w2))
        return _Experts.apply(x.contiguous(), p, scores.detach(), self.w1, self.w2, self.k, training)


def train(steps=40, tokens=4096, H=256, F=256, E=16, k=2, dtype=torch.bfloat16, weight=0.0, seed=0, log=print):
    """Fits the layer to 32 clusters of tokens, each with an output of its own; returns the losses of the steps."""
    gen = torch.Generator()
    gen.manual_seed(seed + 1)
    layer = MoELayer(H, F, E, k, dtype, seed=seed)
    masters = [q.detach().float().clone() for q in layer.parameters()]  # the optimizer's fp32 weights
    opt = torch.optim.Adam(masters, lr=3e-3)
    centre, answer = torch.randn(32, H, generator=gen).cuda(), torch.randn(32, H, generator=gen).cuda()
    losses = []
    for step in range(steps):
        c = torch.randint(32, (tokens,), generator=gen).cuda()
        x = centre[c] + 0.5 * torch.randn(tokens, H, generator=gen).cuda()
        y, do_loss = layer(x.to(dtype))
        fit = (y.float() - answer[c]).square().mean()
        (fit + weight * do_loss).backward()
        for m, q in zip(masters, layer.parameters()):
            m.grad, q.grad = q.grad.float(), None
        opt.step()
        with torch.no_grad():
            for m, q in zip(masters, layer.parameters()):
                q.copy_(m)
        losses.append(fit.item())
        if log and (step % 10 == 0 or step == steps - 1):
            log(f"step {step:3d}  mean square {losses[-1]:.4f}  surrogate {do_loss.item():.5g}")
    return layer, losses


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    ap.add_argument("--weight", type=float, default=0.0, help="of the surrogate loss")
    a = ap.parse_args()
    layer, _ = train(a.steps, a.tokens, dtype=torch.bfloat16 if a.dtype == "bf16" else torch.float32, weight=a.weight)
    with torch.no_grad():  # one token at a time, as in serving
        x = torch.randn(4, layer.w1.shape[2], device="cuda").to(layer.w1.dtype)
        one = torch.cat([layer(x[i:i + 1])[0] for i in range(4)])
        print("largest difference between four tokens alone and together:", (one - layer(x)[0]).abs().max().item())


if __name__ == "__main__":
    main()
