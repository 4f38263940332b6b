"""sdsat_token_logprobs at the ends of the temperatures it takes."""
import math

import pytest
import torch

from operator_helpers import context, device_error
from paper_2403_18647_amd import binding as B
from test_gpu_token_logprobs import call, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [2.0 ** -127, 2.0 ** -100, 2.0 ** 40, 2.0 ** 126])
@pytest.mark.parametrize("V", [100, 5000])
def test_extreme_temperatures(T, V):
    """Logits of 0 and -1: the results at T = 2^-127 are 0, the log of the ties and -2^127."""
    ctx = context(batch=1, q=4, vocab=V)
    x = torch.full((4, V), -1.0, device="cuda")
    x[0, 3], x[1, V - 1], x[2, 5:7] = 0.0, 0.0, 0.0   # and a row of equal values
    tokens = torch.tensor([3, 0, 6, 9], dtype=torch.int32, device="cuda")
    check(x, tokens, T, 3, call(ctx, 1, 4, x, tokens, T, 3))
    assert device_error(ctx) == 0
    ctx.close()


@pytest.mark.parametrize("T", [3.0e-39, 3.5e-39, 4.2e-39, math.inf])
def test_temperatures_whose_scale_is_not_finite_are_refused(T):
    """1 / T is finite for the first three, log2(e) / T, by which the logits are scaled, is not."""
    ctx = context(batch=1, q=1, vocab=100)
    x, tokens = torch.zeros((1, 100), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    f, i = torch.empty(8, device="cuda"), torch.empty(8, dtype=torch.int32, device="cuda")
    with pytest.raises(B.SdsatError) as e:
        B.sdsat_token_logprobs(ctx.handle, 1, 1, x, tokens, T, 2, f, f, i, f)
    assert e.value.code == -1
    ctx.close()
