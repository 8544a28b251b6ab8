"""A small residual network on points, trained step by step with the library's operators: every block's convolution between a norm in
front of it and a norm, a gate and the residual behind it, activations kept in 8 bits for the backward pass, the log probabilities of the
points' labels at the end.

    python examples/train_segmentation.py [--steps 40] [--points 20000] [--full]      (--full: activations kept in full width)

The network's own arithmetic besides the library's is torch matrix products (stem, gates, head) and the optimiser's update.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2511_23227_amd as pcpp  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16


def make_scene(n, classes, seed=0):
    """Points in the unit cube with noisy colours; a point's label is the slab of its neighbourhood along x + y / 2, which a colour alone does not say."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    xyz = torch.rand(n, 3, generator=g, device="cuda")
    slab = ((xyz[:, 0] + 0.5 * xyz[:, 1]) / 1.5 * classes).long().clamp(max=classes - 1)
    colour = torch.nn.functional.one_hot(slab, classes).float() + 1.2 * torch.randn(n, classes, generator=g, device="cuda")
    return xyz, colour, slab.int()


class Network:
    """Parameters by name, the forward pass, and the gradients by hand."""

    def __init__(self, features, channels, classes, blocks, cells, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
        self.blocks, p = blocks, {}
        p["stem"] = normal(features, channels) / features ** 0.5
        for b in range(blocks):
            p[f"conv{b}"] = normal(cells, channels, channels) / (4 * channels) ** 0.5
            p[f"gate{b}"] = 0.1 * normal(channels, 1)
            p[f"post{b}"] = torch.full((channels,), 0.5, device="cuda")
        for b in range(blocks + 1):
            p[f"pre{b}"] = torch.ones(channels, device="cuda")
        p["head"] = normal(channels, classes) / channels ** 0.5
        self.p = p

    def forward(self, T, features, keep=True, packed=True):
        """Logits, and what the backward pass needs: per block the residual stream and, in 8 bits or in full, the convolution's input
        and output.  keep = False: an answer only."""
        p, kept = self.p, []
        x = features @ p["stem"]                       # the residual stream, fp32
        y = pcpp.pcpp_block_norm_fwd(x, w_pre=p["pre0"], dtype=BF16, pack_h=keep and packed)
        for b in range(self.blocks):
            h, h_packed = y.h, y.h_packed
            f = pcpp.pcpp_mvmr_fwd(h, p[f"conv{b}"].to(BF16), T, out_dtype=BF16)
            gate = (x @ p[f"gate{b}"]).to(BF16)
            r = x
            y = pcpp.pcpp_block_norm_fwd(r, f, gate, p[f"post{b}"], p[f"pre{b + 1}"], pack_f=keep and packed, pack_h=keep and packed)
            x = y.r
            if keep:
                kept.append((r, h_packed if packed else h, y.f_packed if packed else f, gate))
        logits = y.h.float() @ p["head"]
        return logits, (features, kept, x, y.h)

    def backward(self, T, kept, d_logits):
        p, grads = self.p, {}
        features, blocks, r, h = kept
        grads["head"] = h.float().t() @ d_logits
        dh, dr = (d_logits @ p["head"].t()).to(BF16), None
        for b in reversed(range(self.blocks)):
            x, h, f, gate = blocks[b]
            g = pcpp.pcpp_block_norm_bwd(dr, dh, r, f, gate, p[f"post{b}"], p[f"pre{b + 1}"])
            grads[f"post{b}"], grads[f"pre{b + 1}"] = g.dw_post, g.dw_pre
            weight = pcpp.pcpp_mvmr_bwd_weight_packed if isinstance(h, pcpp.Packed) else pcpp.pcpp_mvmr_bwd_weight
            grads[f"conv{b}"] = weight(h, g.df, T)
            dh = pcpp.pcpp_mvmr_bwd_input(g.df, p[f"conv{b}"].to(BF16), T, out_dtype=BF16)
            dgate = g.dgate.float()
            grads[f"gate{b}"] = x.t() @ dgate
            dr, r = g.dx + dgate @ p[f"gate{b}"].t(), x
        g = pcpp.pcpp_block_norm_bwd(dr, dh, r, w_pre=p["pre0"])
        grads["pre0"] = g.dw_pre
        grads["stem"] = features.t() @ g.dx
        return grads


def loss_and_gradients(net, T, features, labels, packed=True):
    """Mean of -log p(label), and its gradient by parameter."""
    logits, kept = net.forward(T, features, packed=packed)
    y = pcpp.pcpp_log_probs_fwd(logits, labels)
    d = torch.full_like(y.log_prob, -1.0 / labels.numel())
    d_logits = pcpp.pcpp_log_probs_bwd(logits, labels, y, d, out=logits)             # in place of the logits
    return -y.log_prob.mean(), net.backward(T, kept, d_logits)


def train(points=20_000, steps=40, channels=64, classes=8, blocks=3, packed=True, rate=0.01, report=print):
    """Losses of all steps, and the share of points whose most probable class is theirs at the end."""
    xyz, features, labels = make_scene(points, classes)
    radius = (20.0 / (points * 4.19)) ** (1 / 3)      # about twenty neighbours
    T = pcpp.pcpp_build_triplets(xyz, xyz, radius, 3)
    net = Network(features.shape[1], channels, classes, blocks, T.K)
    moments = {k: (torch.zeros_like(v), torch.zeros_like(v)) for k, v in net.p.items()}
    losses = []
    for step in range(1, steps + 1):
        loss, grads = loss_and_gradients(net, T, features, labels, packed)
        for k, g in grads.items():                     # Adam
            m, v = moments[k]
            m.mul_(0.9).add_(g, alpha=0.1)
            v.mul_(0.99).addcmul_(g, g, value=0.01)
            net.p[k] -= rate * (m / (1 - 0.9 ** step)) / ((v / (1 - 0.99 ** step)).sqrt() + 1e-8)
        losses.append(float(loss))
        if report and (step % 10 == 0 or step == 1):
            report(f"step {step}: loss {losses[-1]:.4f}")
    answer = pcpp.pcpp_log_probs_fwd(net.forward(T, features, keep=False)[0], labels, n_top=2)
    right = float((answer.top_index[:, 0] == labels).float().mean())
    if report:
        report(f"right {right:.3f}, entropy {float(answer.entropy.mean()):.3f}, log probability of the runner-up {float(answer.top_log_prob[:, 1].mean()):.2f}")
    return losses, right


if __name__ == "__main__":
    a = argparse.ArgumentParser()
    a.add_argument("--steps", type=int, default=40)
    a.add_argument("--points", type=int, default=20_000)
    a.add_argument("--full", action="store_true", help="keep activations in full width")
    o = a.parse_args()
    train(o.points, o.steps, packed=not o.full)
