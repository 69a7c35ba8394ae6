"""The target's pass over a 4-bit cache as it is used: a fused projection, head norms with the rotation, the append, the
attention, logits, sampling, the drafted block's acceptance, and the tokens' log probabilities -- over several steps, with a
rollback in between.  Every stage is compared with float64 computed from what the stage before left on the device."""
import numpy as np
import pytest
import torch

import kv4_ref
import logprobs_ref
from test_gpu_qk_norm_rope import _reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,Hq,Hkv", [(64, 8, 2), (128, 16, 2)])
def test_verify_steps_over_a_4_bit_cache(d, Hq, Hkv):
    import paper_2608_30252_amd as mad
    g = torch.Generator().manual_seed(d)
    B, T, D, V, base = 3, 4, 128, 1531, 1e4
    w_qkv = (torch.randn(((Hq + 2 * Hkv) * d, D), generator=g) * D ** -0.5).to(torch.bfloat16).cuda()
    w_out = (torch.randn((V, Hq * d), generator=g) * 6 * (Hq * d) ** -0.5).to(torch.bfloat16).cuda()
    gam = [(1 + 0.3 * torch.randn(d, generator=g)).to(torch.bfloat16).cuda() for _ in range(2)]
    kv = mad.KV4.empty(B, Hkv, 200, d)
    kv.length = [0, 0, 0]
    tokens = torch.randint(0, V, (B, T - 1), generator=g, dtype=torch.int32)
    shadow = {}

    def project(n_cap, n):
        """New rows of every sequence through projection, norm and rotation; appended; returns the queries."""
        x = torch.randn((B, n_cap, D), generator=g).to(torch.bfloat16).cuda()
        qkv = (x.view(-1, D) @ w_qkv.t()).view(B, n_cap, Hq + 2 * Hkv, d)
        q, k, v = torch.split(qkv, [Hq, Hkv, Hkv], 2)
        was = [t.double().cpu().numpy() for t in (q, k)]
        start = list(kv.length)
        mad.qk_norm_rope(q, k, start, gam[0], gam[1], q, k, n, rope_base=base)       # in place in the projection
        for t, w, gm in ((q, was[0], gam[0]), (k, was[1], gam[1])):
            for b in range(B):
                z, tol = _reference(w[b, :n[b]], gm.double().cpu().numpy(), start[b] + np.arange(n[b]), 1e-5, base, True)
                assert np.all(np.abs(t[b, :n[b]].double().cpu().numpy() - z) <= tol)
        mad.kv4_append(k, v, kv, n)
        for name, t, codes, scale in (("k", k, kv.k, kv.k_scale), ("v", v, kv.v, kv.v_scale)):
            for b in range(B):
                c, s = kv4_ref.encode(t[b, :n[b]].double().cpu().numpy())
                rows = slice(start[b], start[b] + n[b])
                assert np.array_equal(codes[b, :, rows].cpu().numpy(), c.transpose(1, 0, 2))
                assert np.array_equal(scale[b, :, rows].cpu().numpy(), s.transpose(1, 0, 2))
                for i in range(n[b]):
                    shadow[name, b, start[b] + i] = kv4_ref.values(c[i], s[i])
        kv.length = [l + m for l, m in zip(start, n)]
        return q

    project(70, [70, 33, 64])                                                        # prompts
    for step in range(3):
        q = project(T, [T] * B).contiguous()
        out, lse = mad.verify_attn_kv4(q, kv)
        o, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
        for b in range(B):
            for h in range(Hkv):
                kk, vv = (np.stack([shadow[name, b, i][h] for i in range(kv.length[b])]) for name in ("k", "v"))
                G = Hq // Hkv
                ref = kv4_ref.attend(q[b, :, h * G:(h + 1) * G].double().cpu().numpy(), kk, vv, kv.length[b], d ** -0.5)
                tol, tol_lse = kv4_ref.tolerances("bf16", d, kv.length[b], *ref)
                assert np.all(np.abs(o[b, :, h * G:(h + 1) * G] - ref[0]) <= tol) and np.all(np.abs(l[b, :, h * G:(h + 1) * G] - ref[1]) <= tol_lse)
        logits = (out.view(B * T, Hq * d) @ w_out.t()).float().view(B, T, V)
        u = torch.rand((B, T), generator=g).cuda()
        tok, probs = mad.sample(logits, u, 0.9, 50, 0.95, probs=torch.empty_like(logits))
        n_acc, nxt = mad.accept_stochastic(probs, probs[:, :-1].contiguous(), tokens.cuda(), u)
        emitted = torch.cat([tokens.cuda(), tok[:, -1:]], 1)
        for b in range(B):
            emitted[b, n_acc[b]] = nxt[b]
        logp, rank, entropy, top_tok, top_logp = mad.token_logprobs(logits, emitted, 5, 0.9)
        x = logits.double().cpu().numpy()
        for b in range(B):
            for t in range(T):
                r = logprobs_ref.row(x[b, t], int(emitted[b, t]), 5, 0.9)
                assert rank[b, t].item() == r["rank"] and np.array_equal(top_tok[b, t].cpu().numpy(), r["top_tok"])
                assert logprobs_ref.close(logp[b, t].item(), r["logp"], r["S"]) and abs(entropy[b, t].item() - r["entropy"]) <= r["tol_entropy"]
                assert logprobs_ref.close(top_logp[b, t].double().cpu().numpy(), r["top_logp"], np.full(5, r["S"]))
        # rejected rows are rolled back: the next step writes over them
        kv.length = [l - T + 1 + int(n_acc[b]) for b, l in enumerate(kv.length)]
        tokens = tok[:, :-1].cpu()
