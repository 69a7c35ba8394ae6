"""Sampling of large batches, whose rows' second launch gives several chunks to a workgroup, and of rows some of whose
chunks are masked throughout, against plain float64."""
import numpy as np
import pytest
import torch

import sample_ref
from test_gpu_sample import TYPES, _check, _logits, _mad

pytestmark = pytest.mark.gpu


def _run(x, probs, **kw):
    mad = _mad()
    u = torch.rand(x.shape[:2], generator=torch.Generator().manual_seed(x.shape[2]))
    out = torch.full(x.shape, float("nan"), device="cuda") if probs else None
    tok, p = mad.sample(x.cuda(), u.cuda(), probs=out, **kw)
    torch.cuda.synchronize()
    _check(x, u, tok.cpu(), None if p is None else p.cpu(), **kw)


@pytest.mark.parametrize("probs", [False, True])
def test_several_chunks_to_a_workgroup_top_p(probs):
    # 80 rows of 16 chunks: 3 to each of 5 workgroups, the last one takes 1
    _run(_logits("model", (16, 5, 128256), 201), probs, top_p=[0.8 + 0.012 * b for b in range(16)])


@pytest.mark.parametrize("probs", [False, True])
def test_several_chunks_to_a_workgroup_mixed(probs):
    # 256 rows of 5 chunks: 3 and 2; every row ends in the second launch
    B = 64
    kw = dict(temperature=[0.6 + 0.01 * b for b in range(B)], top_k=[(0, 129, 0, 3000)[b % 4] for b in range(B)],
              top_p=[(0.9, 1.0, 0.99, 1.0)[b % 4] for b in range(B)], min_p=[(0.0, 0.0, 0.01)[b % 3] for b in range(B)])
    _run(_logits("model", (B, 4, 40000), 202).to(torch.bfloat16), probs, **kw)


def test_several_chunks_to_a_workgroup_any_distribution():
    # 64 rows of 10 chunks, 2 to a workgroup: ends among thousands of equal or near values, over many bins, in few entries
    for i, kind in enumerate(("ties", "body", "wide", "masked", "lowest")):
        x = _logits(kind, (32, 2, 75000), 203 + i).to(TYPES[("bf16", "f32")[i % 2]])
        _run(x, i % 2 == 0, top_p=0.85)
        _run(x, i % 2 == 1, top_k=500)


@pytest.mark.parametrize("mask", [-1e4, -1e9, "lowest", -float("inf"), 2.5])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_chunks_of_one_value(dtype, mask):
    # whole chunks at a finite mask, or at a value among the others: the rest of the row decides as it would
    V = 40000
    x = _logits("model", (2, 1, V), 210)
    x[0, 0, 8192:24576] = torch.finfo(TYPES[dtype]).min if mask == "lowest" else mask
    x[1, 0, :30000] = torch.finfo(TYPES[dtype]).min if mask == "lowest" else mask
    x = x.to(TYPES[dtype])
    for i, kw in enumerate((dict(temperature=0), dict(top_k=1), dict(top_k=40), dict(top_k=100, top_p=0.9), dict(top_k=128, min_p=0.01),
                            dict(top_k=700), dict(top_k=700, top_p=0.9), dict(top_p=0.9), dict(top_p=0.99999), dict(min_p=0.05),
                            dict(top_p=0.9, min_p=0.3), dict())):
        _run(x, i % 2 == 0, **kw)


def test_no_uniform_is_near_an_edge():
    # the tokens above are compared exactly: no uniform lies where roundings decide
    x = _logits("model", (16, 5, 128256), 201)
    u = torch.rand(x.shape[:2], generator=torch.Generator().manual_seed(x.shape[2]))
    assert not any(sample_ref.near_edge(x[b, 0].double().numpy(), float(u[b, 0]), 2.0 ** -45, top_p=0.8 + 0.012 * b) for b in range(16))
