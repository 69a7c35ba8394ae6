"""Rows that an append writes again with a larger scale: code times old scale over new, also where the product itself is
beyond fp32's range, and where the old scale is far below the new one."""
import numpy as np
import pytest
import torch

import kv8_ref
from test_gpu_kv8 import F8, _mad

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("old,new,x", [(1.75 * 2.0 ** 119, 2.0 ** 120, 3.2e38),     # 448 of these are 5e38
                                       (2.0 ** 119, 2.0 ** 120, 3.2e38),
                                       (1.125 * 2.0 ** 118, 2.0 ** 120, -3.4e38),
                                       (2.0 ** -120, 2.0 ** 120, 3.2e38),
                                       (1.5, 2.0, 896.0), (2.0 ** -100, 1.0, 448.0)])
def test_rows_written_again(old, new, x):
    mad = _mad()
    d, block, n = 64, 16, 3
    codes = torch.arange(256, dtype=torch.uint8).repeat(3)[:n * d].view(1, 1, n, d)
    codes = torch.cat([codes, torch.zeros(1, 1, block - n, d, dtype=torch.uint8)], 2)
    k, v = codes.cuda().view(F8), codes.clone().cuda().view(F8)
    ks, vs = (torch.full((1, 1, 1), old, device="cuda") for _ in range(2))
    row = torch.zeros(1, 1, 1, d)
    row[..., 7] = x
    mad.kv8_append(row.cuda(), row.cuda(), mad.KV8(k, v, ks, vs, [n], block))
    torch.cuda.synchronize()
    # code times old / new: 4 bits times 3 at most here, exact in fp32 too
    want = kv8_ref.encode(kv8_ref.decode(codes[0, 0, :n].numpy()) * (old / new))
    for got, s in ((k, ks), (v, vs)):
        assert float(s) == new
        got = got.view(torch.uint8)[0, 0].cpu().numpy()
        nan = (want & 127) == 127
        assert np.array_equal(got[:n][~nan], want[~nan]) and np.all((got[:n][nan] & 127) == 127)
        assert got[n, 7] == kv8_ref.encode(x / new)
