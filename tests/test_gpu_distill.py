"""The operators around a quantized head, run together: the example of `distill.py`, and one of its steps against 64 bits."""
import numpy as np
import pytest
import torch

from paper_2407_02327_amd import distill
from tests import head_ref as R
from tests.gpu_util import say

pytestmark = pytest.mark.gpu


def test_the_student_approaches_its_teacher():
    say("distill example")
    first, last, before, after = distill.run(steps=40, tokens=256, width=256, vocabulary=2048, top=32, say=lambda *a: None)
    assert last < 0.5 * first and after > before


def test_a_step_against_64_bits():
    """What a step returns and leaves, from the logits that its INT8 head wrote: the loss, the gradient of the logits and, from the head's
    own gradient of its input, those of the norm."""
    say("distill step")
    g = torch.Generator(device="cuda").manual_seed(3)
    teacher = distill.Teacher(128, 256, 1040, 16, g)
    student = distill.Student(128, 256, 1040, 16, teacher.w * 0.5)
    hidden = torch.randn(128, 256, generator=g, device="cuda").half()
    logp, index = teacher(hidden)
    order = np.argsort(-R.f64(teacher.head.y), axis=1, kind="stable")[:, :16]
    assert np.array_equal(index.cpu().numpy(), order)
    losses = student.step(hidden, logp, index, rate=0.0)
    z, t, i = R.f64(student.head.y), R.f64(logp), index.cpu().numpy()
    want, _ = R.distill(z, t, i, 1.0)
    assert np.allclose(R.f64(losses), want, rtol=1e-5, atol=1e-5)
    grad = R.distill_grad(z, t, i, 1.0, R.f64(student.weight))
    assert np.allclose(R.f64(student.loss.dlogits), grad, rtol=2.0 ** -10, atol=2.0 ** -22)
    dy, x = R.f64(student.head.dx), R.f64(hidden)
    for got, w, b in zip((student.norm.dx, student.norm.dgamma, student.norm.dbeta), R.layernorm_grad(dy, x, np.ones(256), 1e-5),
                         R.layernorm_grad_bound(dy, x, np.ones(256), 1e-5)):
        R.assert_within(got, w, b + R.rounded(w, got.dtype), "norm")
