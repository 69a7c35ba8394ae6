"""Speculative steps with stochastic acceptance over the 8-bit cache: the draft's tokens drawn from its filtered
distributions (mad_sample), the verify block's K/V appended (mad_kv8_append), attended with everything before it
(mad_verify_attn_kv8), the target's filtered distributions (mad_sample), and the accept rule on both
(mad_accept_stochastic).  What is rejected is written over by the next step.

A toy target: a token's query, keys and values are rows of tables, its logits the draft's (a table by the last token)
and a matrix product of the attention's output.  Every stage of every step is held to plain float64 on what the stage before it left on the device: the cache
byte for byte, attention within kv8_ref.out_tolerance, tokens exactly, probabilities to fp32 rounding, the accept
decisions exactly (the emitted token up to a uniform within 1e-9 of a bin's edge)."""
import numpy as np
import pytest
import torch

import kv8_ref
import sample_ref

pytestmark = pytest.mark.gpu

V, Hq, Hkv, GAMMA, STEPS = 700, 8, 2, 3, 6
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


class _Target:
    def __init__(self, d, dtype, seed):
        g = torch.Generator().manual_seed(seed)
        mk = lambda *s: torch.randn(s, generator=g).to(dtype)   # noqa: E731
        self.q, self.k, self.v = mk(V, Hq, d), mk(V, Hkv, d), mk(V, Hkv, d)
        self.out = (mk(Hq * d, V).float() * (8 / (Hq * d) ** 0.5)).cuda()
        self.draft = 3 * torch.randn((V, V), generator=g)       # the draft's logits by the last token
        self.dev = [t.cuda() for t in (self.q, self.k, self.v)]


@pytest.mark.parametrize("dtype,d,block,kw", [
    ("bf16", 128, 32, dict(temperature=0.8, top_k=40, top_p=0.95)),
    ("bf16", 64, 16, dict(temperature=1.2, top_p=0.9)),
    ("f32", 64, 64, dict(min_p=0.05)),
    ("f32", 128, 16, dict()),
])
def test_steps(dtype, d, block, kw):
    import oracle
    import paper_2608_30252_amd as mad
    B, T, cap, start = 3, GAMMA + 1, 120, [0, 17, 61]
    tg = _Target(d, TYPES[dtype], d + block)
    rng = np.random.default_rng(block)
    kv = mad.KV8.empty(B, Hkv, cap, d, block)
    ref = {n: (np.zeros((B, Hkv, cap, d), np.uint8), np.ones((B, Hkv, -(-cap // block)), np.float32)) for n in "kv"}

    def append(tok, n):
        """tok [B, rows] on the CPU."""
        kn, vn = (t[tok.cuda()].contiguous() for t in tg.dev[1:])
        mad.kv8_append(kn, vn, kv, n)
        for b in range(B):
            for name, new in (("k", tg.k), ("v", tg.v)):
                kv8_ref.append(ref[name][0][b], ref[name][1][b], new[tok[b]].double().numpy(), kv.length[b], n[b], block)

    # prompts of ragged lengths
    tok = torch.from_numpy(rng.integers(0, V, (B, max(start))))
    append(tok, start)
    kv.length = list(start)
    cur = torch.from_numpy(rng.integers(0, V, B))
    accepted = 0
    for step in range(STEPS):
        u = torch.from_numpy(rng.random((B, GAMMA + T)).astype(np.float32))
        # the draft: a token at a time
        q, drafted, last = [], [], cur
        for i in range(GAMMA):
            x = tg.draft[last].unsqueeze(1)
            prob = torch.empty((B, 1, V), device="cuda")
            t, _ = mad.sample(x.cuda(), u[:, i:i + 1].cuda(), probs=prob, **kw)
            for b in range(B):
                sample_ref.check_row(x[b, 0].double().numpy(), float(u[b, i]), int(t[b, 0]), prob[b, 0].cpu().numpy(),
                                     f"step {step}, draft {i}, sequence {b}", **kw)
            q.append(prob)
            last = t[:, 0].cpu().long()
            drafted.append(t)
        draft = torch.cat(drafted, 1).contiguous()
        # the target: the block behind the cache, then attention over all of it
        block_tok = torch.cat([cur[:, None], draft.cpu().long()], 1)
        append(block_tok, [T] * B)
        whole = mad.KV8(kv.k, kv.v, kv.k_scale, kv.v_scale, [n + T for n in kv.length], block)
        qs = tg.dev[0][block_tok.cuda()].contiguous()
        out, lse = mad.verify_attn_kv8(qs, whole)
        for name, codes, scale in (("k", kv.k, kv.k_scale), ("v", kv.v, kv.v_scale)):
            assert np.array_equal(codes.view(torch.uint8).cpu().numpy(), ref[name][0]), f"step {step}: {name} codes"
            assert np.array_equal(scale.cpu().numpy(), ref[name][1]), f"step {step}: {name} scales"
        for b in range(B):
            K, W = (kv8_ref.values(*(a[b] for a in ref[n]), block) for n in "kv")
            n = whole.length[b]
            o, _, mean, A, m = kv8_ref.attend(tg.q[block_tok[b]].double().numpy(), K, W, n, d ** -0.5)
            tol = kv8_ref.out_tolerance(o, mean, A, m, d, np.abs(W[:, :n]).max(), dtype == "bf16")
            kv8_ref.check_out(out[b].double().cpu().numpy(), o, tol, f"step {step}, sequence {b}")
        logits = (tg.draft.cuda()[block_tok.cuda()] + out.reshape(B, T, -1).float() @ tg.out).to(TYPES[dtype])
        p = torch.empty((B, T, V), device="cuda")
        mad.sample(logits, None, probs=p, **kw)
        for b in range(B):
            for t in range(T):
                sample_ref.check_row(logits[b, t].double().cpu().numpy(), None, None, p[b, t].cpu().numpy(),
                                     f"step {step}, row ({b}, {t})", **kw)
        # the accept rule on both distributions
        qq, ua = torch.cat(q, 1).contiguous(), u[:, GAMMA:].contiguous()
        n_acc, nxt = mad.accept_stochastic(p, qq, draft, ua.cuda())
        want_n, want_next = oracle.accept_stochastic(p.cpu().numpy(), qq.cpu().numpy(), draft.cpu().numpy(), ua.numpy())
        n_acc, nxt = n_acc.cpu().numpy(), nxt.cpu().numpy()
        assert np.array_equal(n_acc, want_n), f"step {step}"
        for b in range(B):
            if nxt[b] != want_next[b]:
                a = int(n_acc[b])
                r = p[b, a].double().cpu().numpy() - (qq[b, a].double().cpu().numpy() if a < GAMMA else 0.0)
                c = np.cumsum(np.maximum(r, 0.0))
                assert np.abs(c - float(ua[b, T - 1]) * c[-1]).min() <= 1e-9 * c[-1], f"step {step}, sequence {b}"
        accepted += int(n_acc.sum())
        kv.length = [n + 1 + int(a) for n, a in zip(kv.length, n_acc)]   # what was rejected is written over
        cur = torch.from_numpy(nxt.astype(np.int64))
    assert max(kv.length) + T <= cap
    assert 0 < accepted < STEPS * B * GAMMA                              # both ends of the rule were met
