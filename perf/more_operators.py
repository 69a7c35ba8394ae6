"""A 4-bit key/value cache with the attention over it, query and key norms with the position rotation, and token log
probabilities, as cases that can be timed and checked.

Four operators of a verifying target's pass, in the order of that pass, each in a plain form (elementary torch
operations) and as the framework's calls:
  rope     each head's RMS norm of new queries and keys, and the rotation at their positions (qk_norm_rope)
  append   new K/V rows into a cache in e2m1 with a power-of-two scale per row and 32 features (kv4_append)
  attn     the T-query attention over that cache, T = 1 a single token's (verify_attn_kv4)
  logp     given tokens' log probabilities and ranks, the rows' entropies, the top alternatives (token_logprobs)
Inputs are synthetic and made on the GPU from the seed: N(0, 1) rows of varying size with a few large channels, as
keys have; logits of a body N(0, 2.2^2) under a Zipf-like head of 256 tokens.
"""
import math
import random

import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]   # code & 7; bit 3 is the sign
GROUP = 32                                        # features that share a scale
EPS, BASE = 1e-5, 500000.0


def listed():
    return [
        # one sequence's new token: the smallest call, latency alone
        dict(name="rope_token", kind="rope", B=1, n=1, ragged=False, Hq=32, Hkv=8, d=64, dtype="bf16", norm=True, fused=True, pos="start", far=32768),
        # a serving batch in verification: gamma + 1 rows each at positions of their own, read from the device
        dict(name="rope_verify16", kind="rope", B=16, n=5, ragged=False, Hq=64, Hkv=8, d=128, dtype="bf16", norm=True, fused=True, pos="rows", far=120000),
        # two long prompts of uneven length, out of one fused projection: the largest write
        dict(name="rope_prompts", kind="rope", B=2, n=8192, ragged=True, Hq=64, Hkv=8, d=128, dtype="bf16", norm=True, fused=True, pos="start", far=0),
        # the target's verify pass of a serving batch: gamma + 1 rows each, at ragged lengths
        dict(name="append4_verify16", kind="append", B=16, n=5, ragged=False, Hkv=8, d=128, dtype="bf16", fused=True, lo=600, hi=12000, room=64),
        # two long prompts at once
        dict(name="append4_prompts", kind="append", B=2, n=16384, ragged=True, Hkv=8, d=128, dtype="bf16", fused=False, lo=0, hi=0, room=128),
        # one token over a short context: the smallest read
        dict(name="attn4_token_short", kind="attn", B=1, T=1, Hq=32, Hkv=8, d=64, dtype="bf16", lo=317, hi=317),
        # verification at a long prefix, 8 query heads per KV head, one sequence
        dict(name="attn4_verify_32k", kind="attn", B=1, T=5, Hq=64, Hkv=8, d=128, dtype="bf16", lo=32773, hi=32773),
        # a serving batch in verification: ragged prefixes
        dict(name="attn4_ragged16", kind="attn", B=16, T=6, Hq=64, Hkv=8, d=128, dtype="bf16", lo=600, hi=12000),
        # the fp32 form (parity and numerics work)
        dict(name="attn4_f32", kind="attn", B=4, T=3, Hq=32, Hkv=8, d=64, dtype="f32", lo=200, hi=6000),
        # a token just sampled, with the usual number of alternatives
        dict(name="logp_token", kind="logp", B=1, T=1, V=50257, dtype="bf16", top=20, warm=False, shifted=False),
        # 16 verified blocks at temperatures of their own: the accepted tokens' log probabilities, five alternatives
        dict(name="logp_block16", kind="logp", B=16, T=5, V=128256, dtype="f32", top=5, warm=True, shifted=False),
        # scoring two prompts: every row against the token after it, with the most likely one: the largest
        dict(name="logp_prompts", kind="logp", B=2, T=1024, V=128256, dtype="bf16", top=1, warm=False, shifted=True),
    ]


def _logu(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rope", "append", "attn", "attn", "logp", "logp"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "logp":
        V = rng.choice([50257, 128256, 32000, _logu(rng, 2000, 160000), _logu(rng, 2, 160000)])
        T = rng.choice([1, rng.randrange(2, 9), _logu(rng, 1, 2048)])
        B = max(1, min(_logu(rng, 1, 64), 100_000_000 // (T * V)))
        return dict(kind=kind, B=B, T=max(1, min(T, 200_000_000 // V)), V=V, dtype=dtype, top=min(V, rng.choice([0, 1, 5, 20, 64, rng.randrange(1, 65)])),
                    warm=rng.random() < 0.5, shifted=rng.random() < 0.5)
    Hkv, G = rng.choice([(8, 4), (8, 4), (8, 8), (8, 1), (2, 16), (4, 2), (3, 4)])
    d = rng.choice([64, 128, 128])
    c = dict(kind=kind, Hkv=Hkv, d=d, dtype=dtype)
    if kind == "attn":
        T = rng.randrange(1, min(8, 64 // G) + 1)
        B = _logu(rng, 1, 64)
        hi = _logu(rng, 64, max(64, min(65536, 100_000_000 // (B * Hkv * d))))
        return dict(c, Hq=Hkv * G, B=B, T=T, lo=max(16, hi // rng.choice([1, 2, 8])), hi=hi)
    n = _logu(rng, 1, 16384)
    c = dict(c, n=n, ragged=rng.random() < 0.5, fused=rng.random() < 0.5)
    if kind == "append":
        hi = _logu(rng, 1, 8000)
        return dict(c, B=_logu(rng, 1, max(1, min(64, 32768 // n))), lo=hi // rng.choice([1, 2, 8]), hi=hi, room=rng.randrange(0, 200))
    return dict(c, B=_logu(rng, 1, max(1, min(64, 16384 // n))), n=min(n, 16384), Hq=Hkv * G, norm=rng.random() < 0.7,
                pos=rng.choice(["start", "rows"]), far=_logu(rng, 1, 1_000_000) if rng.random() < 0.7 else 0)


# ---------------------------------------------------------------- inputs ----

def _rows(g, shape, channels):
    """N(0, 1) values [..., d] with `channels` of the d eight times as large, each row scaled by its own factor."""
    x = torch.randn(shape, generator=g, device=DEV)
    x *= torch.exp(0.5 * torch.randn(shape[:-1] + (1,), generator=g, device=DEV))
    at = torch.randperm(shape[-1], generator=g, device=DEV)[:channels]
    x[..., at] *= 8
    return x


def _heads(g, B, n, heads, d, channels, dt, fused):
    """New rows [B, n, H, d] of each of the kinds of heads: tensors of their own, or views of one fused projection."""
    parts = [_rows(g, (B, n, h, d), c).to(dt) for h, c in zip(heads, channels)]
    if not fused:
        return parts
    whole = torch.cat(parts, 2)
    return list(torch.split(whole, heads, 2))


def _cache(g, B, Hkv, cap, d, channels):
    """A filled cache: bytes [B, Hkv, cap, d / 2] (two codes, the even feature's in the low half) and [B, Hkv, cap, d / 32]
    scales (the exponent, biased by 127) that bring a row's 32 features to within 6."""
    codes = torch.empty((B, Hkv, cap, d // 2), dtype=torch.uint8, device=DEV)
    scale = torch.empty((B, Hkv, cap, d // GROUP), dtype=torch.uint8, device=DEV)
    for b in range(B):
        x = _rows(g, (Hkv, cap, d), channels).view(Hkv, cap, d // GROUP, GROUP)
        k = torch.ceil(torch.log2(x.abs().amax(3) / 6)).clamp(-100, 125)
        mag = (x / torch.exp2(k)[..., None]).abs()
        at = torch.bucketize(mag, torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=DEV))
        nib = (at + 8 * (x < 0)).view(Hkv, cap, d // 2, 2).to(torch.uint8)
        codes[b] = nib[..., 0] | (nib[..., 1] << 4)
        scale[b] = (k + 127).to(torch.uint8)
    return codes, scale


def _inputs(case, seed):
    rng = random.Random("%s %d" % (case["kind"], seed))
    g = torch.Generator(device=DEV).manual_seed(seed)
    B, dt = case["B"], TYPES[case["dtype"]]
    if case["kind"] == "logp":
        T, V = case["T"], case["V"]
        R = T + 1 if case["shifted"] else T
        m = min(256, V)
        head = 15 - 2 * torch.log(torch.arange(1, m + 1, device=DEV).float())
        x = torch.empty((B, R, V), dtype=dt, device=DEV)
        tok = torch.empty((B, R), dtype=torch.int32, device=DEV)
        for b in range(B):
            for r in range(0, R, 256):                                             # (a part at a time: fp32 copies)
                part = 2.2 * torch.randn((min(256, R - r), V), generator=g, device=DEV)
                at = torch.randint(0, V, (part.shape[0], 1), generator=g, device=DEV)
                at = (at + torch.arange(m, device=DEV) * max(1, V // m)) % V       # the row's likely tokens
                part.scatter_(1, at, head + 0.7 * torch.randn((part.shape[0], m), generator=g, device=DEV))
                x[b, r:r + part.shape[0]] = part.to(dt)
                # most tokens are likely ones, some any
                likely = torch.gather(at, 1, (torch.rand((part.shape[0], 1), generator=g, device=DEV) ** 4 * m).long())
                other = torch.randint(0, V, likely.shape, generator=g, device=DEV)
                rare = torch.rand(likely.shape, generator=g, device=DEV) < 0.1
                tok[b, r:r + part.shape[0]] = torch.where(rare, other, likely)[:, 0].to(torch.int32)
        temp = [round(rng.uniform(0.6, 1.3), 2) if case["warm"] else 1.0 for _ in range(B)]
        if case["shifted"]:
            return dict(x=x[:, :-1], tok=tok[:, 1:].contiguous(), temp=temp)       # each row scores the token after it
        return dict(x=x, tok=tok, temp=temp)
    Hkv, d = case["Hkv"], case["d"]
    if case["kind"] == "attn":
        lens = [max(rng.randint(case["lo"], case["hi"]), case["T"]) for _ in range(B)]
        cap = max(lens) + 5
        kc, ks = _cache(g, B, Hkv, cap, d, 4)
        vc, vs = _cache(g, B, Hkv, cap, d, 0)
        q = 0.5 * torch.randn((B, case["T"], case["Hq"], d), generator=g, device=DEV)
        return dict(lens=lens, kc=kc, ks=ks, vc=vc, vs=vs, q=q.to(dt))
    n_cap = case["n"]
    n = [rng.randint(max(1, n_cap // 3), n_cap) if case["ragged"] else n_cap for _ in range(B)]
    if case["kind"] == "append":
        lens = [rng.randint(case["lo"], case["hi"]) for _ in range(B)]
        cap = case["hi"] + n_cap + case["room"]
        kc, ks = _cache(g, B, Hkv, cap, d, 4)
        vc, vs = _cache(g, B, Hkv, cap, d, 0)
        k, v = _heads(g, B, n_cap, [Hkv, Hkv], d, [4, 0], dt, case["fused"])
        return dict(lens=lens, n=n, kc=kc, ks=ks, vc=vc, vs=vs, k=k, v=v)
    q, k, _ = _heads(g, B, n_cap, [case["Hq"], Hkv, Hkv], d, [4, 4, 0], dt, case["fused"])
    start = [rng.randint(0, case["far"]) for _ in range(B)]
    pos = torch.tensor(start, dtype=torch.int32, device=DEV)[:, None] + torch.arange(n_cap, dtype=torch.int32, device=DEV)
    if case["pos"] == "rows":                                                      # a slot shares the next token's position
        pos = pos - (torch.rand(pos.shape, generator=g, device=DEV) < 0.2).int() * (pos > 0).int()
    gam = [(1 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(dt) if case["norm"] else None for _ in range(2)]
    return dict(q=q, k=k, n=n, start=start, rows=pos, gq=gam[0], gk=gam[1])


def prepare(case, seed):
    s = dict(case, **_inputs(case, seed))
    B = case["B"]
    if case["kind"] == "logp":
        s["temp_dev"] = torch.tensor(s["temp"], dtype=torch.float64, device=DEV)
        shape, top = (B, case["T"]), (B, case["T"], case["top"])
        s["logp"], s["entropy"] = torch.empty(shape, device=DEV), torch.empty(shape, device=DEV)
        s["rank"] = torch.empty(shape, dtype=torch.int32, device=DEV)
        s["top_logp"] = torch.empty(top, device=DEV) if case["top"] else None
        s["top_tok"] = torch.empty(top, dtype=torch.int32, device=DEV) if case["top"] else None
        return s
    if case["kind"] == "attn":
        s["len_dev"] = torch.tensor(s["lens"], device=DEV)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:3], device=DEV)
    else:
        s["n_dev"] = torch.tensor(s["n"], device=DEV)
        names = ("k", "v") if case["kind"] == "append" else ("q", "k")
        # rows past a sequence's last keep these zeros
        s["to"] = [torch.zeros(s[x].shape, dtype=s[x].dtype, device=DEV) for x in names]
        if case["kind"] == "append":
            s["len_dev"] = torch.tensor(s["lens"], device=DEV)
    if own and case["kind"] in ("append", "attn"):
        import paper_2608_30252_amd as mad
        s["kv"] = mad.KV4(s["kc"], s["vc"], s["ks"], s["vs"], s["lens"])
    return s


# ------------------------------------------------------------------- run ----

def run(s):
    """An append returns the new rows as the values that the cache now holds for them (k, v), and the cache's bytes."""
    if own:
        import paper_2608_30252_amd as mad
        if s["kind"] == "rope":
            q, k = mad.qk_norm_rope(s["q"], s["k"], s["start"] if s["pos"] == "start" else s["rows"], s["gq"], s["gk"], s["to"][0], s["to"][1],
                                    n=s["n"], eps=EPS, rope_base=BASE)
            return {"q": q, "k": k}
        if s["kind"] == "append":
            mad.kv4_append(s["k"], s["v"], s["kv"], s["n"], k_held=s["to"][0], v_held=s["to"][1])
            return {"k": s["to"][0], "v": s["to"][1], "k_codes": s["kc"], "k_scale": s["ks"], "v_codes": s["vc"], "v_scale": s["vs"]}
        if s["kind"] == "attn":
            out, lse = mad.verify_attn_kv4(s["q"], s["kv"], s["out"], s["lse"])
            return {"out": out, "lse": lse}
        mad.token_logprobs(s["x"], s["tok"], s["top"], s["temp"], logp=s["logp"], rank=s["rank"], entropy=s["entropy"], top_tok=s["top_tok"],
                           top_logp=s["top_logp"])
        return _named(s, s["logp"], s["rank"], s["entropy"], s["top_tok"], s["top_logp"])
    if s["kind"] == "rope":
        for i, (x, gamma) in enumerate(((s["q"], s["gq"]), (s["k"], s["gk"]))):
            s["to"][i] = torch.where(_valid(s)[:, :, None, None], _rope(s, x, gamma), s["to"][i])
        return {"q": s["to"][0], "k": s["to"][1]}
    if s["kind"] == "append":
        s["to"][0] = _append_one(s, s["k"], s["kc"], s["ks"], s["to"][0])
        s["to"][1] = _append_one(s, s["v"], s["vc"], s["vs"], s["to"][1])
        return {"k": s["to"][0], "v": s["to"][1], "k_codes": s["kc"], "k_scale": s["ks"], "v_codes": s["vc"], "v_scale": s["vs"]}
    return _attn(s) if s["kind"] == "attn" else _logp(s)


def _named(s, logp, rank, entropy, top_tok, top_logp):
    got = {"logp": logp, "rank": rank, "entropy": entropy}
    return dict(got, top_tok=top_tok, top_logp=top_logp) if s["top"] else got


def _valid(s):
    return torch.arange(s["rows"].shape[1], device=DEV) < s["n_dev"][:, None]


def _rope(s, x, gamma):
    d = s["d"]
    y = x.float()
    if gamma is not None:
        y = y * torch.rsqrt((y * y).mean(3, keepdim=True) + EPS) * gamma.float()
    theta = BASE ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device=DEV) / d)
    angle = s["rows"].double()[:, :, None] * theta                                  # far positions: 64 bits
    c, sn = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
    a, b = y[..., :d // 2], y[..., d // 2:]
    return torch.cat([a * c - b * sn, b * c + a * sn], 3).to(x.dtype)


def _append_one(s, new, codes, scale, held):
    B, n, Hkv, d = new.shape
    x = new.float().reshape(B, n, Hkv, d // GROUP, GROUP)
    m, e = torch.frexp(x.abs().amax(4))                                             # m 2^e, m in [0.5, 1); 6 = 0.75 * 2^3
    k = torch.where(m > 0, e - 3 + (m > 0.75).to(e.dtype), -100).clamp(-100, 125)
    unit = ((k + 127) << 23).to(torch.int32).view(torch.float32)[..., None]         # 2^k, exactly
    y = (x / unit).abs().clamp_max(6)
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
    y = torch.round(y / step) * step                                                # ties to the even code
    nib = torch.where(y < 2, y * 2, torch.where(y < 4, y + 2, y / 2 + 4)).to(torch.uint8) + 8 * torch.signbit(x).to(torch.uint8)
    nib = nib.view(B, n, Hkv, d // 2, 2)
    two = nib[..., 0] | (nib[..., 1] << 4)
    # rows past a sequence's last stand for its first one again
    i = torch.arange(n, device=DEV)
    i = torch.where(i < s["n_dev"][:, None], i, 0)                                  # [B, n]
    b = torch.arange(B, device=DEV)[:, None]
    codes[b, :, s["len_dev"][:, None] + i] = two[b, i]
    scale[b, :, s["len_dev"][:, None] + i] = (k + 127).to(torch.uint8)[b, i]
    value = (torch.where(torch.signbit(x), -y, y) * unit).view(B, n, Hkv, d).to(held.dtype)
    return torch.where((torch.arange(n, device=DEV) < s["n_dev"][:, None])[:, :, None, None], value, held)


def _values(codes, scale):
    """The fp32 values of a cache's bytes."""
    table = torch.tensor(E2M1 + [-v for v in E2M1], device=DEV)
    x = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], 4)      # [B, Hkv, L, d / 2, 2]
    unit = (scale.int() << 23).view(torch.float32)
    return (x.view(*codes.shape[:3], -1, GROUP) * unit[..., None]).view(*codes.shape[:3], -1)


def _attn(s):
    B, T, Hq, Hkv, d = s["B"], s["T"], s["Hq"], s["Hkv"], s["d"]
    L = max(s["lens"])
    k, v = _values(s["kc"][:, :, :L], s["ks"][:, :, :L]), _values(s["vc"][:, :, :L], s["vs"][:, :, :L])
    q = s["q"].float().view(B, T, Hkv, Hq // Hkv, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, d)
    w = torch.matmul(q, k.transpose(2, 3).contiguous()) * d ** -0.5                      # [B, Hkv, T G, L]
    sees = torch.arange(L, device=DEV) < (s["len_dev"][:, None] - T + 1 + torch.arange(T, device=DEV))[:, :, None]
    sees = sees[:, None, :, None].expand(B, 1, T, Hq // Hkv, L).reshape(B, 1, -1, L)
    w = torch.where(sees, w, -torch.inf)
    top = w.amax(3, keepdim=True)
    w = torch.exp(w - top)
    z = w.sum(3, keepdim=True)
    back = lambda t: t.view(B, Hkv, T, Hq // Hkv, -1).permute(0, 2, 1, 3, 4).reshape(B, T, Hq, -1)   # noqa: E731
    return {"out": back(torch.matmul(w, v) / z).to(s["q"].dtype), "lse": back(top + torch.log(z))[..., 0]}


def _logp(s):
    x = s["x"].float()
    t = s["tok"].long()[:, :, None]
    at = torch.gather(x, 2, t)
    rank = (x > at).sum(2) + ((x == at) & (torch.arange(s["V"], device=DEV) < t)).sum(2)
    y = x / s["temp_dev"].float()[:, None, None]
    y = y - y.amax(2, keepdim=True)
    w = torch.exp(y)
    z = w.sum(2, keepdim=True)
    lp = y - torch.log(z)
    entropy = -(w / z * lp).sum(2)
    logp = torch.gather(lp, 2, t)[..., 0]
    if not s["top"]:
        return _named(s, logp, rank.to(torch.int32), entropy, None, None)
    order = torch.sort(x, dim=2, descending=True, stable=True).indices[:, :, :s["top"]]   # ties: the lower index first
    return _named(s, logp, rank.to(torch.int32), entropy, order.to(torch.int32), torch.gather(lp, 2, order))


# ------------------------------------------------------------ floors, 64 bits ----

def work(case):
    B, e = case["B"], 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "logp":
        rows = B * case["T"]
        return {"bytes": rows * (case["V"] * e + 4 + 12 + 8 * case["top"]), "flops": 5 * rows * case["V"]}
    Hkv, d = case["Hkv"], case["d"]
    row = d / 2 + d / GROUP                                                         # a cached row of one head
    if case["kind"] == "attn":
        keys = B * max((case["lo"] + case["hi"]) / 2, case["T"])
        return {"bytes": 2 * Hkv * keys * row + B * case["T"] * case["Hq"] * (2 * e * d + 4), "flops": 4 * keys * case["T"] * case["Hq"] * d}
    n = B * case["n"] * (2 / 3 if case["ragged"] else 1)
    if case["kind"] == "append":
        return {"bytes": 2 * Hkv * n * (2 * d * e + row), "flops": 4 * n * Hkv * d}
    return {"bytes": n * (case["Hq"] + Hkv) * 2 * d * e + (4 * n if case["pos"] == "rows" else 0), "flops": 8 * n * (case["Hq"] + Hkv) * d}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "rope":
        return {"q": _exact_rope(case, s, s["q"], s["gq"]), "k": _exact_rope(case, s, s["k"], s["gk"])}
    if case["kind"] == "append":
        k, v = _exact_append(case, s, s["k"], s["kc"], s["ks"]), _exact_append(case, s, s["v"], s["vc"], s["vs"])
        return {"k": k, "v": v, "k_codes": s["kc"], "k_scale": s["ks"], "v_codes": s["vc"], "v_scale": s["vs"]}
    return _exact_attn(case, s) if case["kind"] == "attn" else _exact_logp(case, s)


def _exact_rope(case, s, x, gamma):
    """Each pair as a complex number, turned by its position."""
    h = case["d"] // 2
    out = torch.zeros(x.shape, dtype=torch.float64, device=DEV)
    freq = torch.tensor([BASE ** (-j / h) for j in range(h)], dtype=torch.float64, device=DEV)
    for b in range(case["B"]):
        n = s["n"][b]
        for r in range(0, n, 4096):
            y = x[b, r:min(n, r + 4096)].double()
            if gamma is not None:
                y = y / torch.sqrt(y.square().sum(2, keepdim=True) / (2 * h) + EPS) * gamma.double()
            turn = torch.outer(s["rows"][b, r:min(n, r + 4096)].double(), freq)[:, None]
            z = torch.complex(y[..., :h], y[..., h:]) * torch.complex(torch.cos(turn), torch.sin(turn))
            out[b, r:min(n, r + 4096)] = torch.cat([z.real, z.imag], 2)
    return out


def _two_to(k):
    """2^k in 64 bits without a rounding (pow and exp2 have one on some devices)."""
    return ((k.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_append(case, s, new, codes, scale):
    """Sequence by sequence; brings the cache's bytes up to date and returns the values held."""
    d = case["d"]
    held = torch.zeros(new.shape, dtype=torch.float64, device=DEV)
    level = torch.tensor(E2M1, dtype=torch.float64, device=DEV)
    for b in range(case["B"]):
        n, at = s["n"][b], s["lens"][b]
        x = new[b, :n].double().transpose(0, 1).reshape(case["Hkv"], n, d // GROUP, GROUP)
        most = x.abs().amax(3)
        k = torch.ceil(torch.log2((most / 6).clamp_min(2.0 ** -100)))
        k += (most > 6 * _two_to(k)).double() - ((most <= 6 * _two_to(k - 1)) & (k > -100)).double()   # log2 may round
        a = x.abs() / _two_to(k)[..., None]
        up = torch.searchsorted(level, a.contiguous()).clamp_max(7)                 # the first level not below
        lo = (up - 1).clamp_min(0)
        to_up, to_lo = level[up] - a, a - level[lo]
        code = torch.where((to_up < to_lo) | ((to_up == to_lo) & (up % 2 == 0)), up, lo)
        held[b, :n] = (torch.copysign(level[code], x) * _two_to(k)[..., None]).reshape(case["Hkv"], n, d).transpose(0, 1)
        code = (code + 8 * torch.signbit(x)).reshape(case["Hkv"], n, d // 2, 2)
        codes[b, :, at:at + n] = (code[..., 0] + 16 * code[..., 1]).to(torch.uint8)
        scale[b, :, at:at + n] = (k + 127).to(torch.uint8)
    return held


def _exact_attn(case, s):
    B, T, Hq, Hkv, d = (case[n] for n in ("B", "T", "Hq", "Hkv", "d"))
    G = Hq // Hkv
    out = torch.empty((B, T, Hq, d), dtype=torch.float64, device=DEV)
    lse = torch.empty((B, T, Hq), dtype=torch.float64, device=DEV)
    level = torch.tensor(E2M1 + [-x for x in E2M1], dtype=torch.float64, device=DEV)

    def rows(codes, scale, b, h, n):
        c = codes[b, h, :n].long()
        x = torch.empty((n, d), dtype=torch.float64, device=DEV)
        x[:, 0::2], x[:, 1::2] = level[c % 16], level[c // 16]
        return x * _two_to(scale[b, h, :n].long() - 127).repeat_interleave(GROUP, 1)

    for b in range(B):
        n = s["lens"][b]
        for h in range(Hkv):
            k, v = rows(s["kc"], s["ks"], b, h, n), rows(s["vc"], s["vs"], b, h, n)
            q = s["q"][b, :, h * G:(h + 1) * G].double().reshape(T * G, d)
            a = (q @ k.t()) / math.sqrt(d)
            late = torch.arange(n, device=DEV)[None] > (n - T + torch.arange(T, device=DEV).repeat_interleave(G))[:, None]
            a.masked_fill_(late, -math.inf)
            z = torch.logsumexp(a, 1)
            out[b, :, h * G:(h + 1) * G] = (torch.exp(a - z[:, None]) @ v).view(T, G, d)
            lse[b, :, h * G:(h + 1) * G] = z.view(T, G)
    return {"out": out, "lse": lse}


def _exact_logp(case, s):
    """Row by row, in 64 bits; the order by the values first and the indices second."""
    B, T, n = case["B"], case["T"], case["top"]
    if B * T > 8192:
        return None
    logp, entropy = (torch.empty((B, T), dtype=torch.float64, device=DEV) for _ in range(2))
    rank = torch.empty((B, T), dtype=torch.int32, device=DEV)
    top_tok = torch.empty((B, T, n), dtype=torch.int32, device=DEV)
    top_logp = torch.empty((B, T, n), dtype=torch.float64, device=DEV)
    index = torch.arange(case["V"], device=DEV)
    for b in range(B):
        tok = s["tok"][b].tolist()
        for t in range(T):
            raw = s["x"][b, t]
            x = raw.double() / s["temp"][b]
            lp = x - torch.logsumexp(x, 0)
            logp[b, t] = lp[tok[t]]
            entropy[b, t] = -(torch.exp(lp) * lp).sum()
            rank[b, t] = ((raw > raw[tok[t]]) | ((raw == raw[tok[t]]) & (index < tok[t]))).sum()
            if n:
                least = torch.topk(raw, n).values[-1]                               # all that can be among the first n
                among = torch.nonzero(raw >= least)[:, 0]
                among = among[torch.argsort(raw[among].double(), descending=True, stable=True)][:n]
                top_tok[b, t], top_logp[b, t] = among.to(torch.int32), lp[among]
    got = {"logp": logp, "rank": rank, "entropy": entropy}
    return dict(got, top_tok=top_tok, top_logp=top_logp) if n else got
