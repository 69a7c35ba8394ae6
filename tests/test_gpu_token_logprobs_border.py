"""Token log probabilities of rows whose logits lie on both sides of where the sums' reference changes its form (2^26 in
log2 units): lanes, waves, steps and workgroups that saw one side are joined with those that saw the other."""
import math

import numpy as np
import pytest
import torch

from test_gpu_token_logprobs import _check, _tok

pytestmark = pytest.mark.gpu


def _rows(V, temperature, sign):
    """[1, 7, V] fp32: a few units in the last place around the border, at temperatures near a power of two 4 or so apart."""
    border = np.float32(sign * 2.0 ** 26 * temperature / math.log2(math.e))
    ulp = float(np.spacing(np.abs(border)))
    k = torch.zeros(7, V, dtype=torch.float64)
    k[0] = -1
    k[0, V - 1] = 1                                          # one entry above, in the last lane that has any
    k[1] = 1
    k[1, V // 2] = -1
    k[2] = torch.randint(-3, 4, (V,), generator=torch.Generator().manual_seed(V)).double()
    k[3] = torch.linspace(-6, 6, V, dtype=torch.float64).round()      # rises across it
    k[4] = -k[3]
    k[5] = -1
    k[5, -(V // 8):] = 0
    k[6] = -2
    k[6, : V // 16] = -20                                    # steps that raise the reference
    k[6, V // 2:] = 3
    return (float(border) + ulp * k).float()[None]


@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("temperature", [1.0, 0.37, 1e-6, 300.0])
@pytest.mark.parametrize("V", [64, 2048, 50257])
def test_rows_across_the_border(V, temperature, sign):
    x, tok = _rows(V, temperature, sign), _tok(1, 7, V, 2)
    tok[0, 0], tok[0, 1] = V - 1, V // 2
    _check(x, tok, 5, temperature)
    tok[0, 0], tok[0, 1] = 0, 1
    _check(x, tok, 0, temperature)


@pytest.mark.parametrize("sign", [-1, 1])
def test_rows_across_the_border_in_one_workgroup(sign):
    V = 20003
    x = _rows(V, 1.0, sign).expand(64, 7, V).reshape(32, 14, V).repeat(1, 3, 1)      # 1344 rows: a workgroup each
    _check(x, _tok(32, 42, V, 3), 3, rows=range(7))
