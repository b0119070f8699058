"""A mixture of SwiGLU experts in 8-bit integers: a prompt, tokens one at a time, and a few steps that train the router.

    python examples/experts.py [--tokens 512] [--experts 64] [--chosen 8] [--width 2048] [--hidden 1376]

Weights are random.  The experts are quantized once, a scale for each channel, as a server would when it loads them; the router's
matrix stays in fp32.  Its gradient comes from what the forward leaves in its workspace: the loss's gradient with respect to a
token's weights is <dL/dy, o_j>, and ssg_route_bwd takes it to the logits.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), os.pardir))
import paper_2409_12517_amd as ssg  # noqa: E402


class Experts:
    """E experts of k, their weights in 8-bit integers."""

    def __init__(self, E: int, k: int, d: int, f: int, generator: torch.Generator):
        self.E, self.k, self.d, self.f = E, k, d, f
        self.W1, self.W2, self.W3 = (self._weights(rows, K, generator) for rows, K in ((f, d), (f, d), (d, f)))

    def _weights(self, rows: int, K: int, generator: torch.Generator) -> torch.Tensor:
        q = torch.empty(ssg.ssg_i8_bytes(self.E * rows, K), dtype=torch.uint8, device="cuda")
        w = (torch.randn(self.E * rows, K, generator=generator, device="cuda") * K ** -0.5).bfloat16()
        ssg.ssg_i8_quantize(w, ssg.SSG_BF16, self.E * rows, K, K, q)
        return q

    def desc(self, T: int):
        return ssg.make_moe_desc(ssg.make_route_desc(T, self.E, self.k, score=ssg.SSG_ROUTE_SIGMOID), self.d, self.f, ssg.SSG_BF16)

    def forward(self, x: torch.Tensor, logits: torch.Tensor, bias: torch.Tensor):
        """y, and the descriptor and workspace that hold what the call went through."""
        desc = self.desc(x.shape[0])
        y = torch.empty_like(x)
        workspace = torch.empty(ssg.ssg_moe_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
        ssg.ssg_moe_fwd(desc, x, logits, bias, self.W1, self.W2, self.W3, y, workspace)
        return y, desc, workspace

    def router_gradient(self, desc, workspace: torch.Tensor, logits: torch.Tensor, dy: torch.Tensor) -> torch.Tensor:
        """dL/dlogits from dL/dy, the experts held."""
        T, k = desc.route.T, self.k
        view = ssg.ssg_moe_view_workspace(desc, workspace)

        def field(pointer, shape, dtype):
            return ssg.view_tensor(workspace, workspace.data_ptr(), pointer, shape, dtype)

        place = field(view.place, (T, k), torch.int32).long()
        o = field(view.o, (view.rows, self.d), torch.bfloat16)
        dweights = (o[place.clamp(min=0)].float() * dy.float()[:, None, :]).sum(-1) * (place >= 0)
        dlogits = torch.empty_like(logits)
        ssg.ssg_route_bwd(desc.route, logits, field(view.ids, (T, k), torch.int32), field(view.weights, (T, k), torch.float32), dweights, dlogits)
        return dlogits


def run(tokens: int = 512, experts: int = 64, chosen: int = 8, width: int = 2048, hidden: int = 1376, steps: int = 6, say=print) -> dict:
    if tokens < 5:
        raise ValueError("the workspace of a call of up to four tokens does not keep the experts' results")
    generator = torch.Generator(device="cuda").manual_seed(0)
    layer = Experts(experts, chosen, width, hidden, generator)
    # (what the tokens have in common makes some experts everybody's choice)
    x = (torch.randn(tokens, width, generator=generator, device="cuda") + 0.5 * torch.randn(width, generator=generator, device="cuda")).bfloat16()
    router = torch.randn(width, experts, generator=generator, device="cuda") * width ** -0.5
    bias = torch.zeros(experts, device="cuda")

    # a prompt, and its tokens again one at a time: the same bits
    logits = x.float() @ router
    y, desc, workspace = layer.forward(x, logits, bias)
    alone = torch.cat([layer.forward(x[t:t + 1], logits[t:t + 1].contiguous(), bias)[0] for t in range(tokens - 4, tokens)])
    same = torch.equal(alone, y[-4:])
    say(f"{tokens} tokens, {chosen} of {experts} experts of {width} x {hidden}: the last four one at a time give {'the same' if same else 'OTHER'} bits")

    # experts that have more than their share are chosen less: the bias counts for the choice, not for the weights
    def load():
        view = ssg.ssg_moe_view_workspace(desc, workspace)
        return ssg.view_tensor(workspace, workspace.data_ptr(), view.counts, (experts,), torch.int32).float()

    share, first = tokens * chosen / experts, load().max().item()
    for i in range(steps):
        bias -= 0.1 * 0.6 ** i * torch.sign(load() - share)
        y, desc, workspace = layer.forward(x, logits, bias)
    say(f"rows of the fullest expert: {first:.0f}, with a balance bias {load().max().item():.0f} (on average {share:.0f})")

    # the router learns towards a layer whose router is another one
    other = router + 0.5 * torch.randn(width, experts, generator=generator, device="cuda") * width ** -0.5
    target = layer.forward(x, x.float() @ other, bias)[0].float()
    losses = []
    for _ in range(steps):
        logits = x.float() @ router
        y, desc, workspace = layer.forward(x, logits, bias)
        dy = y.float() - target
        losses.append(dy.square().sum(1).mean().item())
        gradient = x.float().t() @ layer.router_gradient(desc, workspace, logits, dy)
        router = router - 0.02 * width ** -0.5 * gradient / gradient.square().mean().sqrt()
    say("loss of the router's steps: " + " ".join(f"{v:.4g}" for v in losses))
    return {"same": same, "fullest": (first, load().max().item()), "losses": losses}


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("tokens", 512), ("experts", 64), ("chosen", 8), ("width", 2048), ("hidden", 1376), ("steps", 6)):
        parser.add_argument("--" + name, type=int, default=value)
    run(**vars(parser.parse_args()))
