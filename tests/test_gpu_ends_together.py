"""The operators at the vocabulary's two ends used together (needs an MI355X)."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
EXAMPLE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "fit_drafter.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("fit_drafter", EXAMPLE)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_a_drafter_learns_to_be_accepted(example):
    found = example.run(steps=200)
    # it starts near the uniform distribution and nobody falls below the target's entropy, but for the noise of a batch's mean:
    # 1024 tokens whose ln p have a standard deviation of at most 3
    assert abs(found["loss"][0] - math.log(2000)) < 0.5
    assert found["entropy"] - 0.3 < found["loss"][-1] < found["loss"][0] - 0.3
    assert all(math.isfinite(n) and n > 0 for n in found["norm"])
    assert found["accepted"][1] > found["accepted"][0] + 0.1


def test_a_step_is_the_one_that_automatic_differentiation_takes(example):
    V, D, T, dev = 300, 32, 200, "cuda:0"
    gen = torch.Generator(device=dev)
    gen.manual_seed(3)
    drafter = example.Drafter(V, D, gen, dev)
    context = torch.randint(0, V, (T,), generator=gen, device=dev, dtype=torch.int32)
    following = torch.randint(0, V, (T,), generator=gen, device=dev, dtype=torch.int32)
    wide = [p.double().requires_grad_() for p in drafter.params]
    h = wide[0][context.long()] * drafter.scale
    loss = torch.nn.functional.cross_entropy(torch.relu(h @ wide[1]) @ wide[2], following.long())
    loss.backward()

    class Keeps:  # (an optimizer that does nothing)
        def step(self):
            pass

    got, norm = drafter.step(context, following, Keeps(), math.inf)
    want = math.sqrt(sum(float((p.grad ** 2).sum()) for p in wide))
    # products of 200 to 300 terms in fp32: 2^-24 a term, random in sign, twice in a row
    assert abs(float(got) - float(loss.detach())) < 1e-5 and abs(float(norm) - want) < 1e-4 * want
    for p, q in zip(drafter.params, wide):
        assert (p.grad.double() - q.grad).norm() <= 1e-4 * q.grad.norm()
    drafter.step(context, following, Keeps(), want / 10)
    for p, q in zip(drafter.params, wide):
        assert (p.grad.double() - q.grad / 10).norm() <= 1e-4 * q.grad.norm() / 10
