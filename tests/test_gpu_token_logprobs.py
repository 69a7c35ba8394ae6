"""Token log probabilities on the GPU against float64 (logprobs_ref.py): ranks and alternatives exactly, the numbers within
the bounds derived there."""
import numpy as np
import pytest
import torch

import logprobs_ref

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _check(x, tok, top_n, temperature=1.0, rows=None, got=None):
    """Runs the call (or takes its results) and compares rows (all, or the given ones) with the reference."""
    import paper_2608_30252_amd as mad
    B, T, V = x.shape
    dev = x.cuda() if x.device.type == "cpu" else x
    if got is None:
        got = mad.token_logprobs(dev, tok.cuda(), top_n, temperature)
    logp, rank, entropy, top_tok, top_logp = [None if t is None else t.double().cpu().numpy() for t in got]
    for b in range(B):
        temp = temperature[b] if isinstance(temperature, (list, tuple)) else temperature
        for t in (range(T) if rows is None else rows):
            r = logprobs_ref.row(dev[b, t].double().cpu().numpy(), int(tok[b, t]), top_n, temp)
            where = f"row ({b}, {t})"
            assert rank[b, t] == r["rank"], f"{where}: rank {rank[b, t]}, {r['rank']} expected"
            assert logprobs_ref.close(logp[b, t], r["logp"], r["S"]), f"{where}: logp {logp[b, t]!r}, {r['logp']!r} expected (bound {r['S']:.3g})"
            assert np.isnan(r["entropy"]) and np.isnan(entropy[b, t]) or abs(entropy[b, t] - r["entropy"]) <= r["tol_entropy"] + 1e-12, \
                f"{where}: entropy {entropy[b, t]!r}, {r['entropy']!r} expected (bound {r['tol_entropy']:.3g})"
            if top_n:
                assert np.array_equal(top_tok[b, t], r["top_tok"]), f"{where}: alternatives {top_tok[b, t]}, {r['top_tok']} expected"
                assert logprobs_ref.close(top_logp[b, t], r["top_logp"], np.full(top_n, r["S"])), where
    return got


def _logits(shape, dtype, seed, sigma=2.2):
    return (sigma * torch.randn(shape, generator=torch.Generator().manual_seed(seed))).to(TYPES[dtype])


def _tok(B, T, V, seed=0):
    return torch.randint(0, V, (B, T), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 63, 64, 65, 1000, 8191, 8192, 8193, 16389, 50257, 128256])
def test_vocabularies(V, dtype):
    # odd sizes put the rows at every alignment
    x = _logits((2, 5, V), dtype, V)
    _check(x, _tok(2, 5, V), min(V, 20), [0.7, 1.3])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("top_n", [0, 1, 2, 31, 63, 64])
def test_numbers_of_alternatives(top_n, dtype):
    x = _logits((3, 2, 40001), dtype, top_n)
    _check(x, _tok(3, 2, 40001), top_n)


def test_whole_small_vocabularies_in_order():
    _check(_logits((4, 9, 64), "bf16", 1), _tok(4, 9, 64), 64)
    _check(_logits((1, 3, 33), "f32", 2), _tok(1, 3, 33), 33)


def test_the_largest_vocabulary_and_one_workgroup_rows():
    x = _logits((1, 1, 1 << 20), "bf16", 3)
    _check(x, _tok(1, 1, 1 << 20), 64)
    x = _logits((64, 32, 9001), "bf16", 4)                # 2048 rows: a workgroup each
    _check(x, _tok(64, 32, 9001), 10, rows=[0, 17, 31])
    x = _logits((2, 1500, 700), "f32", 5)
    _check(x, _tok(2, 1500, 700), 3, rows=range(0, 1500, 37))


@pytest.mark.parametrize("top_n", [0, 1, 33])
def test_many_long_rows(top_n):
    # a workgroup to a row, steps of 32 entries; an odd vocabulary puts the rows at every alignment
    B, T, V = 9, 65, 65539
    g = torch.Generator(device="cuda").manual_seed(top_n)
    x = (2.2 * torch.randn((B, T, V), generator=g, device="cuda")).to(torch.bfloat16)
    x[0, 0] = torch.arange(V, device="cuda").div(256).floor()                    # rises, in equal values
    x[0, 1] = -x[0, 0]
    x[0, 2, ::3] = -float("inf")
    x[0, 3, 65000] = float("nan")
    x[0, 4, [7, 65538]] = float("inf")
    x[1, 0] = torch.finfo(torch.bfloat16).min
    x[1, 1], x[1, 1, 40000] = -float("inf"), 3.0
    x[1, 2] = 0.0
    x[1, 3] = 1e30 * torch.sign(x[1, 3].float())
    x[1, 4] = -float("inf")
    tok = _tok(B, T, V, 5)
    tok[0, 0], tok[0, 1], tok[1, 1], tok[1, 2] = 30000, 30000, 40000, 65538
    _check(x, tok, top_n, [0.5 + 0.2 * b for b in range(B)], rows=[0, 1, 2, 3, 4, 31, 64])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_few_different_values(dtype):
    """More equal values than the list of candidates holds: in one chunk, in a later one, everywhere."""
    V = 30011
    x = torch.zeros(1, 8, V)
    x[0, 1, 12000:20000] = 1.0                              # a later chunk rises above the first
    x[0, 2] = torch.arange(V).float().div(64).floor()       # rises all the way
    x[0, 3] = -x[0, 2]
    x[0, 4, ::2] = -1.0
    x[0, 5] = -1e30
    x[0, 6, :8200] = 2.0
    x[0, 7, 29000:] = 3.0
    _check(x.to(TYPES[dtype]), _tok(1, 8, V, 3), 64)
    _check(x.to(TYPES[dtype]), _tok(1, 8, V, 4), 1, 0.01)
    many = x.to(TYPES[dtype]).expand(64, 8, V).reshape(32, 16, V).repeat(1, 3, 1)   # 1536 rows: one workgroup goes through all chunks
    _check(many, _tok(32, 48, V, 5), 40, rows=range(8) if dtype == "bf16" else [1, 2, 6])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_and_special_values(dtype):
    low = torch.finfo(TYPES[dtype]).min
    inf, nan = float("inf"), float("nan")
    V = 20003
    x = _logits((1, 14, V), "f32", 7)
    x[0, 0, 100:] = -inf                                    # a mask that leaves 100
    x[0, 1, :V - 1] = -inf                                  # ... one
    x[0, 2] = -inf                                          # ... none
    x[0, 3, 50:] = low                                      # masked by the type's lowest value
    x[0, 4] = low                                           # all of them
    x[0, 5, 19999] = nan
    x[0, 6, 3] = inf
    x[0, 7, 5], x[0, 7, 15000], x[0, 7, 8] = inf, inf, -inf
    x[0, 8, 5], x[0, 8, 6] = inf, nan
    x[0, 9] = nan
    x[0, 10, :9000] = -inf                                  # a first chunk without anything
    x[0, 11, ::2], x[0, 11, 1::2] = 0.0, -0.0               # equal values
    x[0, 12, 7] = -low
    x[0, 13] = x[0, 13] * 1e30
    tok = _tok(1, 14, V, 1)
    tok[0, 0], tok[0, 1], tok[0, 3], tok[0, 6], tok[0, 7], tok[0, 10], tok[0, 12] = 200, V - 1, 60, 3, 15000, 8999, 7
    for top_n in (64, 1):
        _check(x.to(TYPES[dtype]), tok, top_n)
    tok[0, 1], tok[0, 7], tok[0, 6], tok[0, 2], tok[0, 0] = 5, 4, 8, -1, V
    _check(x.to(TYPES[dtype]), tok, 5, 2.5)


def test_tokens_outside_the_vocabulary():
    x = _logits((1, 6, 300), "f32", 8)
    _check(x, torch.tensor([[-1, 300, 2 ** 31 - 1, -2 ** 31, 0, 299]], dtype=torch.int32), 2)


@pytest.mark.parametrize("temperature", [1e-6, 0.01, 1.0, 50.0, 1e6])
def test_temperatures(temperature):
    _check(_logits((1, 3, 50257), "bf16", 9), _tok(1, 3, 50257), 8, temperature)


@pytest.mark.parametrize("scale", [1.0, 2.0 ** 20, 2.0 ** 26, 2.0 ** 30, 1e36])
def test_differences_of_far_logits_are_exact(scale):
    """Values a few units in the last place apart, around where the sums' reference changes its form and far beyond."""
    g = torch.Generator().manual_seed(14)
    near = torch.randint(0, 12, (1, 2, 20001), generator=g).float()
    x = scale * (0.6931471805599453 * (1 + near * 2.0 ** -23))
    x[0, 1] *= -1
    for temperature in (1.0, scale * 2.0 ** -23, scale * 2.0 ** -21):
        _check(x, _tok(1, 2, 20001), 30, temperature)


def test_sharp_and_shifted_rows():
    x = _logits((1, 4, 50257), "f32", 10)
    x[0, 0, 77] += 60.0                                     # a certain token
    x[0, 1] += 30000.0                                      # far from 0
    x[0, 2] -= 30000.0
    x[0, 3] *= 1e-3                                         # nearly even
    tok = torch.tensor([[77, 5, 6, 7]], dtype=torch.int32)
    _check(x, tok, 4)
    _check(x, torch.tensor([[76, 50256, 0, 9]], dtype=torch.int32), 4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_views(dtype):
    """Rows of padded vocabularies, all rows but the last, every second row, a row shared by all sequences."""
    big = _logits((3, 6, 1025), dtype, 11).cuda()
    _check(big[:, :-1], _tok(3, 5, 1025), 4)
    _check(big[:, 1::2, :1001], _tok(3, 3, 1001), 4)
    _check(big[1:, :, 3:1004], _tok(2, 6, 1001), 4)
    _check(big[:1].expand(3, 6, 1025), _tok(3, 6, 1025), 4)
    _check(big.transpose(0, 1), _tok(6, 3, 1025), 4)


def test_what_is_not_asked_for():
    import paper_2608_30252_amd as mad
    x = _logits((2, 3, 5000), "bf16", 12).cuda()
    tok = _tok(2, 3, 5000).cuda()
    full = mad.token_logprobs(x, tok, 7)
    none = mad.token_logprobs(x)
    assert none[0] is None and none[1] is None and none[3] is None and none[4] is None and torch.equal(none[2], full[2])
    only = mad.token_logprobs(x, None, 7)
    assert only[0] is None and torch.equal(only[3], full[3]) and torch.equal(only[4], full[4])
    outs = [torch.empty_like(t) for t in full]
    assert all(a is b for a, b in zip(mad.token_logprobs(x, tok, 7, 1.0, *outs), outs)) and all(torch.equal(a, b) for a, b in zip(outs, full))


@pytest.mark.parametrize("V,rows", [(50257, 3), (700, 1500)])
def test_calls_repeat_bit_for_bit_on_streams_and_in_graphs(V, rows):
    import bench
    import paper_2608_30252_amd as mad
    x, tok = _logits((2, rows, V), "bf16", 13).cuda(), _tok(2, rows, V).cuda()
    want = mad.token_logprobs(x, tok, 20, 0.8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        two = mad.token_logprobs(x, tok, 20, 0.8)
    one = mad.token_logprobs(x, tok, 20, 0.8)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, two, one))
    outs = [torch.empty_like(t) for t in want]
    graph = bench.graph_of(torch, lambda: mad.token_logprobs(x, tok, 20, 0.8, *outs))
    for _ in range(3):
        for t in outs:
            t.zero_()
        torch.randn(1 << 20, device="cuda").sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
