"""examples/heal.py: the operators together, on compressed layers the library installs."""
import importlib.util
import os

import pytest
import torch

from block_checks import f64
from oracle import block
from paper_2608_07814_gb300 import lx

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def heal():
    spec = importlib.util.spec_from_file_location("heal", os.path.join(ROOT, "examples", "heal.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_losses_fall(heal):
    """Adam on one batch with exact gradients of the last block's norms and gate: the
    distillation loss falls, and every token is counted with K experts."""
    history = heal.heal(steps=25)
    first, last = history[0], history[-1]
    assert last[0][1] < 0.9 * first[0][1]
    for _, counts in history:
        assert counts[-1] == heal.TOKENS and sum(counts[:-1]) == heal.TOKENS * heal.K


def test_a_step_is_the_definition(heal):
    """One step's distillation loss against the float64 definitions, from the layer's own
    outputs: norms (bf16 stored: 2^-8 of a value), head in fp64, loss.  The head multiplies
    256 bf16 values of error 2^-9 into logits of size about 3: 0.05 in a logit, and the loss
    is an average over the tokens of terms that change by no more than their logits."""
    teacher, student, first, x, head = heal.build()
    ids, top, lse = heal.targets(teacher, first, x, head, 2.0)
    r, h = lx.residual_norm(x, w_pre=first, eps=heal.EPS)
    rr = f64(x)
    for b in student:
        y = b.layer.moe_forward(h, heal.K)
        r, h = lx.residual_norm(r, y, w_post=b.w_post, gate=b.gate, w_pre=b.w_pre, eps=heal.EPS)
        rr, hh, _ = block.residual_norm(rr, f64(y), f64(b.w_post), f64(b.gate), f64(b.w_pre), eps=heal.EPS)
    loss, _ = lx.distill_loss(h @ head.t(), ids, top, temperature=2.0, teacher_lse=lse, want_grad=False)
    want, _ = block.distill(hh @ f64(head).T, ids.cpu().numpy(), f64(top), 2.0, f64(lse))
    assert abs(float(loss.double().mean()) - want.mean()) <= 0.05


def test_example_frees_its_layers(heal):
    teacher, student, *_ = heal.build()
    for b in teacher + student:
        b.layer.free()
    torch.cuda.synchronize()
