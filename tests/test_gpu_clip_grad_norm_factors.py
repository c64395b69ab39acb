"""GPU tests of focus_clip_grad_norm's factors next to powers of two, in place and with outputs of their own.

A factor below 2^-100 goes in as x 2^-100, x in fp32: just below 2^-100 x rounds to 1, and the gradients are scaled all the same. Bounds as
in the tests of ordinary factors: 2^-23 of the value, in bf16 2^-8 and 2^-23, and half a step of the smallest numbers.
"""
import math

import pytest
import torch

from gpu_common import announce, require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    return require_gpu()


# gradients of one element each and the bound: factors of 2^-100 (1 - 2^-27), 2^-100 (1 - 2^-29), 2^-100, a little above and below it
# and of 1 - 2^-27, which rounds to 1
CASES = {"below": ([2.0 ** 100, 2.0 ** 87], 1.0), "just below": ([2.0 ** 100, 2.0 ** 86], 1.0), "at": ([2.0 ** 100], 1.0),
         "above": ([2.0 ** 100 * (1 - 2.0 ** -8)], 1.0), "well below": ([2.0 ** 101], 1.0), "one": ([1.0, 2.0 ** -13], 1.0),
         "with a bound of another size": ([2.0 ** 60, 2.0 ** 47], 2.0 ** -40)}


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("name", CASES)
def test_in_place_and_beside(F, name, dt):
    announce(f"clip factor {name} {dt}")
    values, max_norm = CASES[name]
    before = [torch.tensor([v], dtype=dt, device="cuda") for v in values]
    if max(values) > 2.0 ** 90:  # too small to count in the norm
        before.append(torch.linspace(-1, 1, 1001, device="cuda").to(dt) * 2.0 ** 70)
    want = math.sqrt(sum(float(b.double().square().sum()) for b in before))
    factor = min(1.0, max_norm / want)
    here, out = [b.clone() for b in before], [torch.full_like(b, 7.0) for b in before]
    for grads, to in ((here, None), (before, out)):
        norm = F.clip_grad_norm(grads, max_norm, out=to)
        assert abs(norm.item() - want) <= 1e-9 * want
    for a, o, b in zip(here, out, before):
        assert torch.equal(a, o), name
        ref = b.double() * factor
        lim = (2.0 ** -23 + (2.0 ** -8 if dt == torch.bfloat16 else 0.0)) * ref.abs() + 2.0 ** (-149 if dt == torch.float32 else -134)
        assert ((a.double() - ref).abs() <= lim).all(), name
