"""One workspace, sized once for a program's largest call, serves its smaller ones with the same results."""
import pytest
import torch

from test_gpu_kv4 import _bytes, _q

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
def test_attention_over_4_bits(d):
    import paper_2608_30252_amd as mad
    ws = torch.zeros(mad.workspace_bytes(mad.MAD_OP_VERIFY_KV4, 64, 64, 8, d, 6), dtype=torch.uint8, device="cuda")
    kv = [t.cuda() for t in _bytes(64, 8, 700, d, seed=3)]
    for B, Hq, Hkv, T in ((64, 64, 8, 6), (1, 64, 8, 6), (63, 64, 8, 1), (3, 32, 2, 4), (64, 8, 8, 2)):
        part = mad.KV4(*[t[:B, :Hkv].contiguous() for t in kv], [600 - 7 * b for b in range(B)])
        q = _q(B, T, Hq, d, "bf16", B).cuda()
        want, got = mad.verify_attn_kv4(q, part), mad.verify_attn_kv4(q, part, ws=ws)
        assert all(torch.equal(a, b) for a, b in zip(want, got)), (B, Hq, Hkv, T)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_log_probabilities(dtype):
    import paper_2608_30252_amd as mad
    ws = torch.zeros(mad.workspace_bytes(mad.MAD_OP_LOGPROBS, 64, T=64, max_keys=128256), dtype=torch.uint8, device="cuda")
    for B, T, V in ((64, 64, 300), (1, 1, 128256), (1, 1, 70000), (1, 1, 65000), (8, 9, 50257), (63, 8, 9001)):
        g = torch.Generator(device="cuda").manual_seed(V)
        x = torch.randn(B, T, V, generator=g, device="cuda").to(dtype)
        tok = torch.randint(0, V, (B, T), generator=g, device="cuda", dtype=torch.int32)
        want, got = mad.token_logprobs(x, tok, 20), mad.token_logprobs(x, tok, 20, ws=ws)
        assert all(torch.equal(a, b) for a, b in zip(want, got)), (B, T, V)
