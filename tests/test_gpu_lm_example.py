"""The example's path from embedding to synchronisation: its gradient against automatic differentiation in 64 bits, and a
run in which the loss falls."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("vocab,width", [(1000, 64), (77, 5)])
def test_gradient_of_the_whole_step(vocab, width):
    import distill_language_model as ex
    R, N, K = 3, 40, 6
    gen = torch.Generator(device="cuda").manual_seed(1)
    student = ex.Student(vocab, width)
    flat = torch.randn((R, student.d), generator=gen, device="cuda") * 0.1
    grad = torch.full_like(flat, 7.0)
    tokens = torch.randint(0, vocab, (R, N), generator=gen, device="cuda")
    teacher = torch.randn((vocab, vocab), generator=gen, device="cuda") * 2
    ids, logp = ex.teacher_entries(teacher, tokens, K)
    loss = student.gradient(flat, grad, tokens, ids, logp)
    w = flat.double().cpu().requires_grad_()
    table, bias = student.views(w)
    total, want_loss = 0.0, []
    for r in range(R):
        h = table[r][tokens[r].cpu()] * student.scale
        lp = torch.log_softmax(h @ table[r].t() + bias[r], 1)
        i, q = ids.view(R, N, K)[r].cpu(), logp.view(R, N, K)[r].double().cpu().exp()
        rest = 1 - q.sum(1)
        keep = torch.ones(N, vocab, dtype=torch.bool).scatter_(1, i, False)
        log_tail = torch.logsumexp(lp.masked_fill(~keep, float("-inf")), 1)
        row = (q * (q.log() - lp.gather(1, i))).sum(1) + rest * (rest.log() - log_tail)
        want_loss.append(row)
        total = total + row.mean()
    total.backward()
    # fp32 products of up to 1000 terms of size 1, at most 40 places added: 1e-4 of the largest entry is a wide bound
    scale = float(w.grad.abs().max())
    assert float((grad.double().cpu() - w.grad).abs().max()) <= 1e-4 * scale
    assert float((loss.double().cpu() - torch.cat(want_loss).detach()).abs().max()) <= 1e-4


def test_the_loss_falls_over_compressed_rounds():
    import distill_language_model as ex
    got = ex.run(steps=60)
    first, last = got["losses"][0], got["losses"][-1]
    assert all(v == v for v in got["losses"]) and last < 0.6 * first, (first, last)
    assert got["in_top_5"] > 0.5
    again = ex.run(steps=3)
    assert again["losses"][0] == first           # the same inputs give the same bits
