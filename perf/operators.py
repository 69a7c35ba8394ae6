"""The 8-bit key/value cache, the attention over it, and sampling, as cases that can be timed and checked.

Three operators of a verifying target and its draft, each in a plain form (elementary torch operations) and as
the framework's calls:
  append   new K/V rows into a cache in e4m3 with one scale per block of tokens and KV head (kv8_append)
  attn     the T-query attention over that cache, T = 1 a single token's (verify_attn_kv8)
  sample   temperature, top-k, top-p and min-p over logits with given uniforms: tokens and, where the accept
           rule needs it, the filtered distribution (sample)
Inputs are synthetic and made on the GPU from the seed: N(0, 1) rows whose size changes from block to block and
with a few large channels, as keys have; logits of a body N(0, 2.2^2) under a Zipf-like head of 256 tokens.
"""
import math
import random

import torch

own = False
DEV = "cuda"
E4M3 = torch.float8_e4m3fn
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one sequence's new token goes into the middle of a block: the smallest write, latency alone
        dict(name="append_token", kind="append", B=1, n=1, ragged=False, Hkv=8, d=64, block=16, dtype="bf16", lo=8183, hi=8183, room=8),
        # the target's verify pass of a serving batch: gamma + 1 rows each, at ragged lengths
        dict(name="append_verify16", kind="append", B=16, n=5, ragged=False, Hkv=8, d=128, block=32, dtype="bf16", lo=600, hi=12000, room=64),
        # chunks of prompts of uneven length in fp32 (parity work), few heads
        dict(name="append_chunks_f32", kind="append", B=4, n=777, ragged=True, Hkv=4, d=64, block=64, dtype="f32", lo=0, hi=900, room=9),
        # two long prompts at once: the largest write
        dict(name="append_prompts", kind="append", B=2, n=16384, ragged=True, Hkv=8, d=128, block=128, dtype="bf16", lo=0, hi=0, room=128),
        # one token over a short context: the smallest read
        dict(name="attn_token_short", kind="attn", B=1, T=1, Hq=32, Hkv=8, d=64, block=16, dtype="bf16", lo=317, hi=317, pow2=True),
        # verification at a long prefix, 8 query heads per KV head, one sequence
        dict(name="attn_verify_32k", kind="attn", B=1, T=5, Hq=64, Hkv=8, d=128, block=128, dtype="bf16", lo=32773, hi=32773, pow2=True),
        # a serving batch in verification: ragged prefixes; scales as another writer leaves them (max / 448)
        dict(name="attn_ragged16", kind="attn", B=16, T=6, Hq=64, Hkv=8, d=128, block=32, dtype="bf16", lo=600, hi=12000, pow2=False),
        # the fp32 form (parity and numerics work)
        dict(name="attn_f32", kind="attn", B=4, T=3, Hq=32, Hkv=8, d=64, block=64, dtype="f32", lo=200, hi=6000, pow2=True),
        # the draft's next token: one row, the usual top-k with top-p
        dict(name="sample_draft", kind="sample", B=1, T=1, V=50257, dtype="bf16", mode="topk", probs=False),
        # a drafted block of 4 sequences to verify, a vocabulary without alignment: tokens and distributions
        dict(name="sample_block4", kind="sample", B=4, T=5, V=50257, dtype="f32", mode="topk", probs=True),
        # 64 sequences of a serving batch, each with settings of its own (greedy ones among them), tokens only
        dict(name="sample_mixed64", kind="sample", B=64, T=1, V=128256, dtype="bf16", mode="mixed", probs=False),
        # the target's distributions for 16 drafted blocks, nucleus sampling: the largest
        dict(name="sample_nucleus16", kind="sample", B=16, T=5, V=128256, dtype="f32", mode="topp", probs=True),
    ]


def _logu(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "attn", "attn", "sample", "sample"])
    if kind == "sample":
        V = rng.choice([50257, 128256, 32000, _logu(rng, 2000, 160000), _logu(rng, 100, 160000)])
        B, T = _logu(rng, 1, 64), rng.choice([1, 1, rng.randrange(2, 9)])
        B = max(1, min(B, 10_000_000 // (T * V)))
        return dict(kind=kind, B=B, T=T, V=V, dtype=rng.choice(["bf16", "f32"]), probs=rng.random() < 0.5,
                    mode=rng.choice(["topk", "topk", "topp", "topp", "minp", "plain", "mixed"]))
    Hkv, G = rng.choice([(8, 4), (8, 4), (8, 8), (8, 1), (2, 16), (4, 2), (3, 4)])
    d, block = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    c = dict(kind=kind, Hkv=Hkv, d=d, block=block, dtype=dtype)
    if kind == "append":
        n = _logu(rng, 1, 16384)
        B = _logu(rng, 1, max(1, min(64, 32768 // n)))
        hi = _logu(rng, 1, 8000)
        return dict(c, B=B, n=n, ragged=rng.random() < 0.5, lo=hi // rng.choice([1, 2, 8]), hi=hi, room=rng.randrange(0, 200))
    T = rng.randrange(1, min(8, 64 // G) + 1)
    B = _logu(rng, 1, 64)
    hi = _logu(rng, 64, max(64, min(65536, 100_000_000 // (B * Hkv * d))))
    return dict(c, Hq=Hkv * G, B=B, T=T, lo=max(16, hi // rng.choice([1, 2, 8])), hi=hi, pow2=rng.random() < 0.5)


# ---------------------------------------------------------------- inputs ----

def _lengths(case, rng):
    return [rng.randint(case["lo"], case["hi"]) for _ in range(case["B"])]


def _rows(g, shape, channels):
    """N(0, 1) values [..., d] with `channels` of the d eight times as large, each row scaled by its own factor."""
    x = torch.randn(shape, generator=g, device=DEV)
    x *= torch.exp(0.5 * torch.randn(shape[:-1] + (1,), generator=g, device=DEV))
    at = torch.randperm(shape[-1], generator=g, device=DEV)[:channels]
    x[..., at] *= 8
    return x


def _cache(g, B, Hkv, cap, d, block, pow2, channels):
    """A filled cache: e4m3 [B, Hkv, cap, d] and its scales [B, Hkv, blocks]; the scale of a block is the least power
    of two (pow2) or the very number that brings its largest value to 448."""
    nb = -(-cap // block)
    codes = torch.empty((B, Hkv, cap, d), dtype=E4M3, device=DEV)
    scale = torch.empty((B, Hkv, nb), device=DEV)
    for b in range(B):
        x = _rows(g, (Hkv, nb * block, d), channels).view(Hkv, nb, block, d)
        s = x.abs().amax((2, 3)) / 448
        if pow2:
            s = torch.exp2(torch.ceil(torch.log2(s)))
        codes[b] = (x / s[:, :, None, None]).clamp(-448, 448).view(Hkv, nb * block, d)[:, :cap].to(E4M3)
        scale[b] = s
    return codes, scale


def _settings(mode, B, rng):
    """(temperature, top_k, top_p, min_p), a list of B each."""
    def one(m):
        t = round(rng.uniform(0.6, 1.2), 2)
        if m == "topk":
            return t, rng.choice([20, 40, 50, 100]), rng.choice([0.8, 0.9, 0.95]), rng.choice([0.0, 0.05])
        if m == "topp":
            return t, 0, round(rng.uniform(0.8, 0.98), 3), 0.0
        if m == "minp":
            return t, 0, 1.0, rng.choice([0.02, 0.05, 0.1])
        return (0.0 if m == "greedy" else t), 0, 1.0, 0.0
    kinds = ["greedy", "topk", "topp", "minp", "plain"]
    got = [one(kinds[(b + rng.randrange(2)) % 5] if mode == "mixed" else mode) for b in range(B)]
    return [list(v) for v in zip(*got)]


def _inputs(case, seed):
    rng = random.Random("%s %d" % (case["kind"], seed))
    g = torch.Generator(device=DEV).manual_seed(seed)
    B, dt = case["B"], TYPES[case["dtype"]]
    if case["kind"] == "sample":
        T, V = case["T"], case["V"]
        x = 2.2 * torch.randn((B, T, V), generator=g, device=DEV)
        m = min(256, V)
        at = torch.rand((B, T, V), generator=g, device=DEV).topk(m).indices
        head = 15 - 2 * torch.log(torch.arange(1, m + 1, device=DEV).float()) + 0.7 * torch.randn((B, T, m), generator=g, device=DEV)
        x.scatter_(2, at, head)
        t, k, p, mp = _settings(case["mode"], B, rng)
        return dict(x=x.to(dt), u=torch.rand((B, T), generator=g, device=DEV), t=t, k=k, p=p, mp=mp)
    Hkv, d, block, lens = case["Hkv"], case["d"], case["block"], _lengths(case, rng)
    if case["kind"] == "append":
        n = [rng.randint(max(1, case["n"] // 3), case["n"]) if case["ragged"] else case["n"] for _ in range(B)]
        cap = case["hi"] + case["n"] + case["room"]
        kc, ks = _cache(g, B, Hkv, cap, d, block, True, 4)
        vc, vs = _cache(g, B, Hkv, cap, d, block, True, 0)
        return dict(lens=lens, n=n, kc=kc, ks=ks, vc=vc, vs=vs,
                    k=_rows(g, (B, case["n"], Hkv, d), 4).to(dt), v=_rows(g, (B, case["n"], Hkv, d), 0).to(dt))
    lens = [max(l, case["T"]) for l in lens]
    cap = max(lens) + 5
    kc, ks = _cache(g, B, Hkv, cap, d, block, case["pow2"], 4)
    vc, vs = _cache(g, B, Hkv, cap, d, block, case["pow2"], 0)
    q = 0.5 * torch.randn((B, case["T"], case["Hq"], d), generator=g, device=DEV)
    return dict(lens=lens, kc=kc, ks=ks, vc=vc, vs=vs, q=q.to(dt))


def prepare(case, seed):
    s = dict(case, **_inputs(case, seed))
    B = case["B"]
    if case["kind"] == "sample":
        # the settings on the device, for the plain form; the framework takes them from the host
        s["dev"] = [torch.tensor(v, dtype=torch.float64, device=DEV)[:, None, None] for v in (s["t"], s["p"], s["mp"])]
        s["dev_k"] = torch.tensor(s["k"], device=DEV)[:, None, None]
        s["tok"] = torch.empty((B, case["T"]), dtype=torch.int32, device=DEV)
        s["out"] = torch.empty((B, case["T"], case["V"]), device=DEV) if case["probs"] else None
        return s
    s["len_dev"] = torch.tensor(s["lens"], device=DEV)
    if case["kind"] == "append":
        s["n_dev"] = torch.tensor(s["n"], device=DEV)
    else:
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:3], device=DEV)
    if own:
        import paper_2608_30252_amd as mad
        s["kv"] = mad.KV8(s["kc"], s["vc"], s["ks"], s["vs"], s["lens"], case["block"])
    return s


# ------------------------------------------------------------------- run ----

def run(s):
    if own:
        import paper_2608_30252_amd as mad
        if s["kind"] == "append":
            mad.kv8_append(s["k"], s["v"], s["kv"], s["n"])
            return {"k": s["kc"], "k_scale": s["ks"], "v": s["vc"], "v_scale": s["vs"]}
        if s["kind"] == "attn":
            out, lse = mad.verify_attn_kv8(s["q"], s["kv"], s["out"], s["lse"])
            return {"out": out, "lse": lse}
        tok, probs = mad.sample(s["x"], s["u"], s["t"], s["k"], s["p"], s["mp"], tok=s["tok"], probs=s["out"])
        return {"tok": tok} if probs is None else {"tok": tok, "probs": probs}
    if s["kind"] == "append":
        _append_one(s, s["k"], s["kc"], s["ks"])
        _append_one(s, s["v"], s["vc"], s["vs"])
        return {"k": s["kc"], "k_scale": s["ks"], "v": s["vc"], "v_scale": s["vs"]}
    return _attn(s) if s["kind"] == "attn" else _sample(s)


def _append_one(s, new, codes, scale):
    """The blocks that the new rows touch are taken out, filled, scaled and put back."""
    B, Hkv, cap, d, block, n = s["B"], s["Hkv"], codes.shape[2], s["d"], s["block"], new.shape[1]
    ln, nn = s["len_dev"], s["n_dev"]
    nb = (n + block - 2) // block + 1
    blk = ln[:, None] // block + torch.arange(nb, device=DEV)                        # [B, nb] touched blocks
    rows = (blk[:, :, None] * block + torch.arange(block, device=DEV)).view(B, -1)   # [B, nb * block] their rows
    i = rows - ln[:, None]                                                           # the row's number among the new ones
    is_new, is_old = (i >= 0) & (i < nn[:, None]), i < 0
    hit = is_new.view(B, nb, block).any(2)                                           # blocks with a new row
    x = torch.gather(new, 1, i.clamp(0, n - 1)[:, :, None, None].expand(B, nb * block, Hkv, d)).float()
    x = x.permute(0, 2, 1, 3)                                                        # [B, Hkv, rows, d]
    fine = torch.isfinite(x)
    big = torch.where(fine & is_new[:, None, :, None], x.abs(), 0).reshape(B, Hkv, nb, -1).amax(3)
    m, e = torch.frexp(big)                                                          # big = m 2^e, m in [0.5, 1); 448 = 0.875 2^9
    e = torch.where(big > 0, e - 9 + (m > 0.875).to(e.dtype), -100).clamp_min(-100)
    need = ((e + 127) << 23).to(torch.int32).view(torch.float32)                     # 2^e, exactly
    at = blk.clamp_max(scale.shape[2] - 1)[:, None].expand(B, Hkv, nb)
    was = torch.gather(scale, 2, at)
    had = is_old.view(B, 1, nb, block).any(3)
    now = torch.where(had, torch.maximum(was, need), need)
    each = lambda t: t[:, :, :, None].expand(B, Hkv, nb, block).reshape(B, Hkv, nb * block, 1)   # noqa: E731
    src = rows.clamp_max(cap - 1)[:, None, :, None].expand(B, Hkv, nb * block, d)
    old = torch.gather(codes.view(torch.uint8), 2, src).view(E4M3).float() * each(was)
    val = torch.where(is_new[:, None, :, None], torch.where(fine, x, torch.nan), old) / each(now)
    # rows of blocks without a new row go back as they were; rows past the cache stand for the first one again
    raw = torch.gather(codes.view(torch.uint8), 2, src)
    mine = hit[:, :, None].expand(B, nb, block).reshape(B, -1) & (is_new | is_old)
    put = torch.where(mine[:, None, :, None], val.to(E4M3).view(torch.uint8), raw)
    turn = torch.where(rows < cap, torch.arange(nb * block, device=DEV), 0)
    to = torch.gather(rows, 1, turn)[:, None, :, None].expand(B, Hkv, nb * block, d)
    put = torch.gather(put, 2, turn[:, None, :, None].expand(B, Hkv, nb * block, d))
    codes.view(torch.uint8).scatter_(2, to, put)
    turn = torch.where(blk < scale.shape[2], torch.arange(nb, device=DEV), 0)
    to = torch.gather(blk, 1, turn)[:, None].expand(B, Hkv, nb)
    put = torch.where(hit[:, None], now, was)
    scale.scatter_(2, to, torch.gather(put, 2, turn[:, None].expand(B, Hkv, nb)))


def _attn(s):
    B, T, Hq, Hkv, d = s["B"], s["T"], s["Hq"], s["Hkv"], s["d"]
    L = max(s["lens"])
    key = torch.arange(L, device=DEV)
    k = s["kc"][:, :, :L].float() * s["ks"][:, :, key // s["block"], None]
    v = s["vc"][:, :, :L].float() * s["vs"][:, :, key // s["block"], None]
    q = s["q"].float().view(B, T, Hkv, Hq // Hkv, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, d)
    w = torch.matmul(q, k.transpose(2, 3).contiguous()) * d ** -0.5                      # [B, Hkv, T G, L]
    sees = key < (s["len_dev"][:, None] - T + 1 + torch.arange(T, device=DEV))[:, :, None]   # [B, T, L]
    sees = sees[:, None, :, None].expand(B, 1, T, Hq // Hkv, L).reshape(B, 1, -1, L)
    w = torch.where(sees, w, -torch.inf)
    top = w.amax(3, keepdim=True)
    w = torch.exp(w - top)
    z = w.sum(3, keepdim=True)
    back = lambda t: t.view(B, Hkv, T, Hq // Hkv, -1).permute(0, 2, 1, 3, 4).reshape(B, T, Hq, -1)   # noqa: E731
    return {"out": back(torch.matmul(w, v) / z).to(s["q"].dtype), "lse": back(top + torch.log(z))[..., 0]}


def _sample(s):
    t, p, mp = s["dev"]
    greedy = t == 0
    x, i = torch.sort(s["x"].double(), dim=2, descending=True, stable=True)       # ties: the lower index first
    w = torch.exp((x - x[:, :, :1]) / torch.where(greedy, 1.0, t))
    rank = torch.arange(x.shape[2], device=DEV)
    k = torch.where(greedy, 1, torch.where(s["dev_k"] > 0, s["dev_k"], x.shape[2]))
    w = torch.where(rank < k, w, 0)
    before = torch.cumsum(w, 2) - w
    w = torch.where((before < p * w.sum(2, keepdim=True)) | (p >= 1), w, 0)
    w = torch.where(w >= mp, w, 0)
    w = torch.zeros_like(w).scatter_(2, i, w)                                      # by index
    run_sum = torch.cumsum(w, 2)
    z = run_sum[:, :, -1:]
    last = torch.where(w > 0, rank, -1).amax(2)
    tok = torch.minimum((run_sum <= s["u"].double()[:, :, None] * z).sum(2), last).to(torch.int32)
    return {"tok": tok, "probs": (w / z).float()} if s["probs"] else {"tok": tok}


# ------------------------------------------------------------ floors, 64 bits ----

def work(case):
    B = case["B"]
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "sample":
        n = B * case["T"] * case["V"]
        return {"bytes": n * (e + (4 if case["probs"] else 0)) + 8 * B * case["T"], "flops": 2 * n}
    mean = (case["lo"] + case["hi"]) / 2
    if case["kind"] == "append":
        n = B * case["n"] * (2 / 3 if case["ragged"] else 1)
        return {"bytes": 2 * case["Hkv"] * n * (case["d"] * (e + 1) + 4 / case["block"]), "flops": 4 * n * case["Hkv"] * case["d"]}
    keys = B * max(mean, case["T"])
    rows = B * case["T"] * case["Hq"]
    return {"bytes": 2 * case["Hkv"] * keys * (case["d"] + 4 / case["block"]) + rows * (2 * e * case["d"] + 4),
            "flops": 4 * keys * case["T"] * case["Hq"] * case["d"]}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "append":
        return {"k": _exact_append(case, s, s["k"], s["kc"], s["ks"]), "k_scale": s["ks"],
                "v": _exact_append(case, s, s["v"], s["vc"], s["vs"]), "v_scale": s["vs"]}
    return _exact_attn(case, s) if case["kind"] == "attn" else _exact_sample(case, s)


def _exact_append(case, s, new, codes, scale):
    """Block by block, sequence by sequence; returns the codes' values, with `scale` brought up to date."""
    block = case["block"]
    got = codes.double()
    for b in range(case["B"]):
        first, end = s["lens"][b], s["lens"][b] + s["n"][b]
        x = new[b].double().transpose(0, 1)                                        # [Hkv, n, d]
        lo = first // block
        hi = (end - 1) // block
        # whole blocks between the first and the last are alike, and many: at once
        for j0, j1 in ((lo, lo + 1), (lo + 1, hi), (max(hi, lo + 1), hi + 1)):
            if j1 <= j0:
                continue
            r0, r1 = max(j0 * block, first), min(j1 * block, end)
            part = x[:, r0 - first:r1 - first]
            pad = torch.zeros((part.shape[0], (j1 - j0) * block, part.shape[2]), dtype=torch.float64, device=DEV)
            pad[:, r0 - j0 * block:r1 - j0 * block] = part
            most = pad.view(part.shape[0], j1 - j0, -1).abs().amax(2).clamp_min(448 * 2.0 ** -100)
            k = torch.ceil(torch.log2(most / 448))
            k += (most > 448 * _two_to(k)).double() - (most <= 448 * _two_to(k - 1)).double()   # log2 may round
            sc = _two_to(k)
            if r0 > j0 * block:                                                    # the block held rows before
                was = scale[b, :, j0:j1].double()
                sc = torch.maximum(sc, was)
                old = got[b, :, j0 * block:r0]
                got[b, :, j0 * block:r0] = _nearest(old * (was / sc)[:, :, None].expand(-1, -1, r0 - j0 * block).reshape(old.shape[0], -1, 1))
            scale[b, :, j0:j1] = sc.float()
            each = sc[:, :, None].expand(-1, -1, block).reshape(sc.shape[0], -1)[:, r0 - j0 * block:r1 - j0 * block, None]
            got[b, :, r0:r1] = _nearest(part / each)
    return got


def _two_to(k):
    """2^k in 64 bits without a rounding (pow and exp2 have one on some devices)."""
    return ((k.to(torch.int64) + 1023) << 52).view(torch.float64)


def _nearest(x):
    """The e4m3 value nearest x, ties to even: steps of 2^-3 of the leading power of two, of 2^-9 below 2^-6."""
    e = torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6)))
    e -= (x.abs() < _two_to(e)).double() * (e > -6)
    step = _two_to(e - 3)
    return torch.round(x / step) * step


def _exact_attn(case, s):
    B, T, Hq, Hkv, d, block = (case[n] for n in ("B", "T", "Hq", "Hkv", "d", "block"))
    G = Hq // Hkv
    out = torch.empty((B, T, Hq, d), dtype=torch.float64, device=DEV)
    lse = torch.empty((B, T, Hq), dtype=torch.float64, device=DEV)
    for b in range(B):
        n = s["lens"][b]
        for h in range(Hkv):
            k = s["kc"][b, h, :n].double() * s["ks"][b, h].double().repeat_interleave(block)[:n, None]
            v = s["vc"][b, h, :n].double() * s["vs"][b, h].double().repeat_interleave(block)[:n, None]
            q = s["q"][b, :, h * G:(h + 1) * G].double().reshape(T * G, d)
            a = (q @ k.t()) / math.sqrt(d)
            late = torch.arange(n, device=DEV)[None] > (n - T + torch.arange(T, device=DEV).repeat_interleave(G))[:, None]
            a.masked_fill_(late, -math.inf)
            z = torch.logsumexp(a, 1)
            out[b, :, h * G:(h + 1) * G] = (torch.exp(a - z[:, None]) @ v).view(T, G, d)
            lse[b, :, h * G:(h + 1) * G] = z.view(T, G)
    return {"out": out, "lse": lse}


def _exact_sample(case, s):
    """Row by row over the candidates in order, in 64 bits."""
    B, T, V = case["B"], case["T"], case["V"]
    tok = torch.zeros((B, T), dtype=torch.int32, device=DEV)
    probs = torch.zeros((B, T, V), dtype=torch.float64, device=DEV) if case["probs"] else None
    for b in range(B):
        temp, k, p, mp = s["t"][b], s["k"][b], s["p"][b], s["mp"][b]
        for t in range(T):
            x = s["x"][b, t].double()
            if temp == 0:
                keep, w = torch.nonzero(x == x.max())[:1, 0], torch.ones(1, dtype=torch.float64, device=DEV)
            else:
                order = torch.argsort(-x, stable=True)
                if k > 0:
                    order = order[:k]
                w = torch.exp(x[order] / temp - x.max() / temp)
                part = torch.cumsum(w, 0)
                n = int((part - w < p * part[-1]).sum()) if p < 1 else len(order)
                n = min(n, int((w >= mp).sum()))
                keep, at = torch.sort(order[:n])
                w = w[at]
            part = torch.cumsum(w, 0)
            i = min(int((part <= float(s["u"][b, t]) * part[-1]).sum()), len(keep) - 1)
            tok[b, t] = keep[i]
            if probs is not None:
                probs[b, t, keep] = w / part[-1]
    return {"tok": tok, "probs": probs} if case["probs"] else {"tok": tok}
