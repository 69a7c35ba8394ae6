"""Token log probabilities at the coldest and the hottest temperatures that are taken, of logits of their size."""
import pytest
import torch

from test_gpu_token_logprobs import TYPES, _check, _logits, _tok

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("power", [-126, -120, -100, 100, 120, 126])
def test_logits_of_the_temperatures_size(power, dtype):
    # (the products are exact in fp64; below 2^-126 the logits are subnormal)
    x = (_logits((2, 3, 20003), "f32", power % 7, 0.9).clamp(-3.9, 3.9).double() * 2.0 ** power).to(TYPES[dtype])
    _check(x, _tok(2, 3, 20003), 8, [2.0 ** power, 2.0 ** power if abs(power) == 126 else 1.5 * 2.0 ** power])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ordinary_logits_where_only_the_largest_counts(dtype):
    x = torch.zeros(1, 2, 5000)
    x[0, 0, 7], x[0, 1, [3, 4999]] = 1.0, 2.0
    tok = torch.tensor([[7, 4999]], dtype=torch.int32)
    _check(x.to(TYPES[dtype]), tok, 1, 2.0 ** -126)
    _check(x.to(TYPES[dtype]), tok, 3, 2.0 ** 126)
