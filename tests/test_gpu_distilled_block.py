"""The training step of distilled_block.py: its gradients against automatic differentiation of the same block in 64 bits with the
masked weights, and its loss over steps."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import oracle                                                          # noqa: E402
from paper_2102_08124_amd.distilled_block import DistilledBlock       # noqa: E402

T, TOP = 2.0, 16


def _masked(wb):
    mask, _ = oracle.approx(wb.view(torch.int16).cpu().numpy().view(np.uint16), 2, 4)
    return wb.double().cpu() * torch.from_numpy(mask.astype(np.float64))


def _reference(block, x, teacher, index):
    """(loss, gradients) in 64 bits; W1 and W2 take the gradient of the masked weights as their own."""
    p = [_masked(wb).requires_grad_() for wb in block.wb]
    rest = [t.double().cpu().requires_grad_() for t in [block.bias] + block.norms[0] + block.norms[1]]
    xd = x.double().cpu().requires_grad_()

    def norm(t, w, b):
        var, mean = torch.var_mean(t, 1, correction=0, keepdim=True)
        return (t - mean) / torch.sqrt(var + 1e-5) * w + b

    u = norm(xd, rest[1], rest[2]) @ p[0].t() + rest[0]
    a = 0.5 * u * (1 + torch.erf(u / 2 ** 0.5))
    y = norm(a @ p[1].t() + xd, rest[3], rest[4])
    logits = y @ block.head.double().cpu().t()
    log_q = torch.log_softmax(logits / T, 1).gather(1, index.cpu())
    log_p = torch.log_softmax(teacher.double().cpu() / T, 1)
    loss = T * T * (log_p.exp() * (log_p - log_q)).sum(1)
    return loss.detach(), torch.autograd.grad(loss.mean(), p + rest + [xd])


def test_gradients_of_a_step():
    block = DistilledBlock(192, 64, 500, TOP, T, seed=3)
    x = torch.randn((192, 64), device="cuda").to(torch.bfloat16)
    teacher, index = block.teach(x)
    block.forward(x)
    dw1, dw2 = block.backward(x, teacher, index)
    torch.cuda.synchronize()
    loss, want = _reference(block, x, teacher, index)
    got = [dw1, dw2, block.dbias] + block.dnorms[0] + block.dnorms[1] + [block.dx]
    # seven roundings to bf16 (2^-8 each at most) on the longest way, and the loss a difference of logarithms of such logits
    for g, w in zip(got, want):
        g = g.double().cpu()
        assert float((g - w).norm() / w.norm()) < 8 * 2.0 ** -8
    assert float((block.loss.double().cpu() - loss).norm() / loss.norm()) < 8 * 2.0 ** -8


def test_the_student_comes_nearer_to_its_teacher():
    """A small step against the gradient lowers the loss, again and again."""
    block = DistilledBlock(256, 64, 700, TOP, T, rate=0.05, seed=4)
    x = torch.randn((256, 64), device="cuda").to(torch.bfloat16)
    lesson = block.teach(x)
    losses = []
    for _ in range(12):
        block.step(x, *lesson)
        losses.append(float(block.loss.mean()))
    assert all(b < a for a, b in zip(losses, losses[1:])), losses
