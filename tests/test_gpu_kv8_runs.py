"""The 8-bit verify attention where workgroups' runs of keys cross unit borders (more units than workgroups, ragged
lengths of several slabs: two to eight units to a workgroup), for every number of query rows and both types, against
plain float64."""
import numpy as np
import pytest
import torch

from test_gpu_kv8 import _attend_case, _cache, _kv, _mad, _rows

pytestmark = pytest.mark.gpu


def _lens(B, top, seed):
    r = np.random.RandomState(seed)
    lens = [int(v) for v in r.randint(0, top, B)]
    lens[1], lens[B // 2] = 0, 3          # no rows; fewer than queries
    return lens


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,Hq,T", [(128, 64, 2), (128, 64, 3), (128, 64, 5), (128, 64, 6), (128, 64, 8), (64, 64, 4), (64, 64, 6), (64, 64, 8)])
def test_runs_over_unit_borders(d, Hq, T, dtype):
    B = 40
    _attend_case(B, T, Hq, 8, d, 32, dtype, _lens(B, 700, d + T), seed=d + T, scales="any")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_runs_over_unit_borders_with_an_odd_number_of_heads(dtype):
    _attend_case(64, 6, 40, 5, 128, 16, dtype, _lens(64, 400, 9), seed=9)


def test_the_same_bits_every_time():
    mad = _mad()
    B, T, Hq, Hkv, d, block = 40, 6, 64, 8, 128, 32
    lens = _lens(B, 700, 80)
    k, v, ks, vs = _cache(B, Hkv, 700, d, block, 81)
    kv = _kv(mad, k, v, ks, vs, lens, block)
    q = _rows((B, T, Hq, d), 82, 0.2).bfloat16().cuda()
    first = mad.verify_attn_kv8(q, kv)
    for _ in range(4):
        out, lse = mad.verify_attn_kv8(q, kv)
        torch.cuda.synchronize()
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
