"""The residual block on the layer operators: its gradients per node against autograd, and its training through the
compressed gradient path."""
import pytest
import torch

from paper_2103_08870_b200 import block as B
from paper_2103_08870_b200 import layers

pytestmark = pytest.mark.gpu


def test_gradients_are_those_of_autograd_up_to_the_rounding_to_8_bits():
    rows, width, hidden, K = 500, 264, 520, 3
    b = B.ResidualBlock(rows, width, hidden, K)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.randn(rows, width, generator=g, device="cuda").bfloat16()
    dy = torch.randn(rows, width, generator=g, device="cuda").bfloat16()
    start = torch.tensor([0, 130, 130, rows], device="cuda")
    y = b.forward(x).double()
    dx = b.backward(dy, start).double()
    layers.check()
    gamma, beta, w1, w2 = (t.double().clone().requires_grad_() for t in (b.gamma, b.beta, b.w1, b.w2))
    xd = x.double().requires_grad_()
    # the branch of the leaky ReLU is the kept activation's (where z is within its rounding of zero another branch is as good)
    slope = torch.where(b.a8.codes[:, :hidden] >= 128, B.SLOPE, 1.0).double()
    want = xd + (slope * (torch.nn.functional.layer_norm(xd, (width,), gamma, beta, B.EPS) @ w1.t())) @ w2.t()
    # e4m3 keeps four bits of an entry: a rounding errs by 2^-4 of it at most, 2^-5.3 in the mean square (uniform between the
    # neighbours, over a binade); up to seven such roundings, of operands or of products' inputs, follow one another.
    tol = 2 ** -5.3 * 7 ** 0.5
    assert (y - want).norm() <= tol * (want - xd).norm()
    for k in range(K):
        part = slice(int(start[k]), int(start[k + 1]))
        grads = torch.autograd.grad((want[part] * dy[part].double()).sum(), [gamma, beta, w1, w2], retain_graph=True)
        got = b.grads[k].double().split(b.numel)
        for a, w in zip(got, grads):
            if part.start == part.stop:
                assert (a == 0).all()
            else:
                assert (a - w.reshape(-1)).norm() <= tol * w.norm()
    (dxw,) = torch.autograd.grad((want * dy.double()).sum(), [xd])
    assert (dx - dxw).norm() <= tol * dxw.norm()


def test_training_through_the_compressed_path_lowers_the_loss():
    losses = B.train(B.ResidualBlock(1024, 128, 512, 4), 60)
    assert torch.isfinite(losses).all() and losses[-10:].mean() < 0.8 * losses[:5].mean()
