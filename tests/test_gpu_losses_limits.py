"""GPU tests of the losses where their arguments or values are at a limit of what they may be."""
import math

import pytest
import torch

from test_gpu_losses import check_policy, losses, make  # noqa: F401

pytestmark = pytest.mark.gpu

# one workgroup a row for both; in slices; many rows, one workgroup each
ROWS = [(2, 5, 3001), (2, 5, 50257), (2, 60, 3001)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("low", ["-inf", "lowest"])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("scale,coef,tau", [(2.0 ** 16, 0.05, 1.0), (2.0 ** 20, 0.1, 0.6), (1.0, 1e4, 1.0)])
def test_masked_tokens_under_a_large_weight_of_the_kl(losses, rows, low, dtype, scale, coef, tau):
    """A token that the policy masks counts nothing, whatever the reference says of it, also where the KL's weight times the largest
    difference of two logits passes fp32."""
    inp, g = make(*rows, dtype, ref=True)
    x, z, y = inp["logits"], inp["ref_logits"], inp["tokens"]
    value = -math.inf if low == "-inf" else torch.finfo(x.dtype).min
    x[..., :100] = value
    z[..., :50] = value  # both mask these, the policy alone the next
    y.clamp_(min=200)
    x[0, 1, 150] = x[0, 1, 200:].float().amin() - 500  # nothing of it is left in the policy, and the reference masks it
    z[0, 1, 150] = torch.finfo(x.dtype).min
    check_policy(losses, inp, g, kl="full", tau=tau, reduction="sum", kl_coef=coef, scale=scale)
