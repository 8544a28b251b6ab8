"""The example's network: its gradients against automatic differentiation of the same network in 64 bits, and its training."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import train_segmentation
    return train_segmentation


def reference_loss(p, blocks, T, features, labels):
    """The network in binary64, parameters p."""
    o, i, k = (t.long().cpu() for t in (T.tri_o, T.tri_i, T.tri_k))
    norm = lambda v: v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-6)  # noqa: E731
    x = features @ p["stem"]
    h = p["pre0"] * norm(x)
    for b in range(blocks):
        w = p[f"conv{b}"]
        f = torch.zeros_like(h)
        for cell in range(w.shape[0]):
            at = k == cell
            f = f.index_add(0, o[at], h[i[at]] @ w[cell].t())
        x = x + torch.sigmoid(x @ p[f"gate{b}"]) * (p[f"post{b}"] * norm(f))
        h = p[f"pre{b + 1}"] * norm(x)
    return torch.nn.functional.cross_entropy(h @ p["head"], labels.long())


@pytest.mark.parametrize("packed", [True, False])
def test_gradients_of_the_network(example, packed):
    """bf16 convolutions round inputs, outputs and weights to 2^-8 of themselves, 8-bit copies the convolution's input and output to 2^-7 of the
    largest of 32 channels, about 2^-6 of a typical one; over two blocks, as independent errors, under 2 % of every gradient's norm in full width and under
    5 % with the copies, and 0.5 % of the loss."""
    pcpp = example.pcpp
    xyz, features, labels = example.make_scene(600, 5, seed=3)
    T = pcpp.pcpp_build_triplets(xyz, xyz, 0.2, 3)
    net = example.Network(5, 24, 5, 2, T.K, seed=4)
    loss, grads = example.loss_and_gradients(net, T, features, labels, packed)
    p = {k: v.double().cpu().requires_grad_() for k, v in net.p.items()}
    ref = reference_loss(p, 2, T, features.double().cpu(), labels.cpu())
    ref.backward()
    assert abs(float(loss) - float(ref)) <= 5e-3 * float(ref)
    assert set(grads) == set(p)
    for k, v in p.items():
        off = float((grads[k].double().cpu() - v.grad).norm() / v.grad.norm())
        assert off <= (0.05 if packed else 0.02), (k, off)


def test_training_learns(example):
    """Forty steps: the loss falls to under half of log(classes), and 8-bit copies do as well as full width, within a tenth."""
    few, right = example.train(points=6000, steps=40, channels=32, classes=6, blocks=2, report=None)
    full, _ = example.train(points=6000, steps=40, channels=32, classes=6, blocks=2, packed=False, report=None)
    assert few[-1] < 0.9 and right > 0.6
    assert abs(few[-1] - full[-1]) <= 0.1 * full[-1]
