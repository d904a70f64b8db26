"""Timing cases of the operators around attention: rotary positions, and a cache of keys and values in 8 bits with what writes,
reads, weighs and trims it.

A case is a dict of plain values.  Its kind says which operator runs:
  rope    queries and keys rotated by their positions; grad: through autograd, with the gradients
  append  N new tokens of every sequence quantised into the cache
  attend  N queries a head against the cache, causal, aligned at the bottom right
  weigh   the attention weight that each cached token got from those queries, added to what it had
  evict   the cache cut down to `budget` tokens a head: the last `recent` and the heaviest of the rest
and the sizes are B sequences, H query heads, Hkv key/value heads, N new tokens, head size d, capacity cap; lengths are spread over
lo .. cap by `mix`; ragged: sequences bring fewer than N tokens (a padded batch).

The cache: K [B,Hkv,cap,d] and V [B,Hkv,cap/64,d,64] in E4M3, one scale (a power of two) for each 64 tokens of a head, K and V apart.

own: False, the operators in elementary torch operations; True, the framework's kernels.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
BLOCK = 64
LOWEST_EXPONENT = -100      # of a scale: blocks below 448 * 2^-100 lose their last bits
BASE = 10000.0


def listed():
    return [
        # one new token of 32 conversations, far beyond the trained length: latency, and angles of far positions
        dict(name="rope token", kind="rope", B=32, H=32, Hkv=8, N=1, d=128, rot=128, interleaved=False, scaling="yarn", factor=32.0,
             far=131072, grad=False, fused=True, mix=1),
        # a training step of 16384 tokens, q and k straight from the fused projection, half of each head rotated
        dict(name="rope train", kind="rope", B=4, H=32, Hkv=32, N=4096, d=128, rot=64, interleaved=True, scaling="none", factor=1.0,
             far=0, grad=True, fused=True, mix=2),
        # one new token of 32 conversations into their caches
        dict(name="append token", kind="append", B=32, Hkv=8, N=1, d=128, cap=2048, lo=1, ragged=False, mix=3),
        # two prompts of up to 8192 tokens, padded to the longer
        dict(name="append prompt", kind="append", B=2, Hkv=8, N=8192, d=128, cap=8192, lo=8192, ragged=True, mix=4),
        # one token of one sequence in a small model with 12 plain heads: the smallest answer, latency alone
        dict(name="attend one", kind="attend", B=1, H=12, Hkv=12, N=1, d=64, cap=1024, lo=700, ragged=False, mix=5),
        # one token of 64 conversations of all lengths up to 8192
        dict(name="attend batch", kind="attend", B=64, H=32, Hkv=8, N=1, d=128, cap=8192, lo=64, ragged=False, mix=6),
        # one token against one long document
        dict(name="attend long", kind="attend", B=1, H=32, Hkv=4, N=1, d=128, cap=262144, lo=262144, ragged=False, mix=7),
        # a chunk of a long prompt against what came before it
        dict(name="attend chunk", kind="attend", B=1, H=32, Hkv=8, N=2048, d=128, cap=16384, lo=16384, ragged=False, mix=8),
        # the weights that a token of 32 conversations gave, kept for the next eviction
        dict(name="weigh token", kind="weigh", B=32, H=32, Hkv=8, N=1, d=128, cap=4160, lo=2000, ragged=False, mix=9),
        # the weights that the last queries of a prompt gave
        dict(name="weigh chunk", kind="weigh", B=1, H=32, Hkv=8, N=500, d=128, cap=16384, lo=16384, ragged=False, mix=10),
        # caches that have run over their budget by a few hundred tokens
        dict(name="evict step", kind="evict", B=16, Hkv=8, d=128, cap=4416, lo=4200, budget=4096, recent=256, mix=11),
        # a long prompt cut down to what is kept of it
        dict(name="evict prompt", kind="evict", B=1, Hkv=8, d=128, cap=32768, lo=32700, budget=4096, recent=512, mix=12),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


_MOST_BYTES, _MOST_FLOPS = 1e9, 3e11        # of a drawn case


def draw(rng):
    while True:
        kind = rng.choice(("rope", "append", "attend", "attend", "weigh", "evict"))
        d = rng.choice((32, 64, 64, 96, 128, 128, 128, 256))
        Hkv = rng.choice((1, 2, 3, 4, 8, 12))
        B, mix = _log_int(rng, 1, 64), rng.randrange(1 << 20)
        if kind == "rope":
            scaling = rng.choice(("none", "linear", "ntk", "yarn"))
            c = dict(kind=kind, B=min(B, 16), H=Hkv * rng.choice((1, 1, 2, 4, 7)), Hkv=Hkv, N=rng.choice((1, _log_int(rng, 1, 8192))), d=d,
                     rot=rng.choice((d, d, d // 2, d // 4, 2 * rng.randint(2, d // 2))), interleaved=rng.random() < 0.5, scaling=scaling,
                     factor=1.0 if scaling == "none" else round(rng.uniform(1.5, 32.0), 2), far=rng.choice((0, _log_int(rng, 1000, 1000000))),
                     grad=rng.random() < 0.5, fused=rng.random() < 0.5, mix=mix)
        elif kind == "evict":
            cap = BLOCK * _log_int(rng, 2, 1024)
            budget = rng.randint(cap // 8, cap - 1)
            c = dict(kind=kind, B=min(B, 16), Hkv=Hkv, d=d, cap=cap, lo=rng.randint(0, cap), budget=budget, recent=rng.randint(0, budget), mix=mix)
        else:
            cap = BLOCK * _log_int(rng, 1, 2048)
            N = rng.choice((1, 1, rng.randint(1, 8), _log_int(rng, 1, min(cap, 4096))))
            ragged = N > 1 and rng.random() < 0.5
            c = dict(kind=kind, B=B, H=Hkv * rng.choice((1, 2, 4, 5, 8, 16)), Hkv=Hkv, N=N, d=d, cap=cap, lo=rng.randint(N, cap), ragged=ragged,
                     mix=mix)
            if kind == "append":
                del c["H"]
        w = work(c)
        slots = 2.0 * c["B"] * Hkv * c.get("cap", 0) * d          # what the caches hold, used or not
        if w["bytes"] <= _MOST_BYTES and w["flops"] <= _MOST_FLOPS and slots <= 2 * _MOST_BYTES:
            return c


def _lengths(c):
    """Tokens of each sequence in its cache, the new ones among them, and how many are new: part of the case, whatever the seed."""
    r = random.Random(c["mix"])
    lengths = [c["cap"]] + [r.randint(c["lo"], c["cap"]) for _ in range(c["B"] - 1)]
    if c["kind"] == "evict":
        return lengths, [0] * c["B"]
    if not c["ragged"]:
        return lengths, [c["N"]] * c["B"]
    return lengths, [c["N"]] + [r.randint(0, c["N"]) for _ in range(c["B"] - 1)]


def _visible(n, length):
    """Pairs of a query and a token it sees, for the last n of `length` tokens."""
    return n * length - n * (n - 1) // 2


def work(case):
    c, d, B, Hkv = case, case["d"], case["B"], case["Hkv"]
    if c["kind"] == "rope":
        elements = B * (c["H"] + Hkv) * c["N"] * d
        return {"bytes": 4.0 * elements * (2 if c["grad"] else 1), "flops": 3.0 * elements * c["rot"] / d * (2 if c["grad"] else 1)}
    lengths, counts = _lengths(c)
    if c["kind"] == "append":
        elements = 2.0 * Hkv * d * sum(counts)
        return {"bytes": 3.0 * elements, "flops": 2.0 * elements}
    if c["kind"] == "evict":
        kept = sum(min(n, c["budget"]) for n in lengths)
        return {"bytes": Hkv * (4.0 * sum(lengths) + kept * (4.0 * d + 8)), "flops": 2.0 * Hkv * sum(lengths)}
    pairs = c["H"] * sum(_visible(n, l) for n, l in zip(counts, lengths))
    rows = c["H"] * sum(counts)
    if c["kind"] == "attend":
        return {"bytes": 2.0 * Hkv * d * sum(lengths) + rows * (4.0 * d + 4), "flops": 4.0 * d * pairs}
    return {"bytes": Hkv * sum(lengths) * (d + 8.0) + rows * (2.0 * d + 4), "flops": 2.0 * d * pairs}


# ---- inputs

def _round_up_power(amax):
    """The power of two of a block whose largest magnitude is amax: the least 2^e, e >= -100, with amax <= 448 * 2^e."""
    m, e = torch.frexp(amax)                               # amax = m 2^e, m in [0.5, 1)
    e = torch.where(m <= 0.875, e - 9, e - 8)              # 448 = 0.875 * 2^9
    return torch.where(amax > 0, e, LOWEST_EXPONENT).clamp(min=LOWEST_EXPONENT)


def _power(e):
    """2^e in float32 by its bits; 2^-126 for less."""
    return ((e.int().clamp(min=-126) + 127) << 23).view(torch.float32)


def _cache(c, g, lengths):
    """A cache as appending left it: E4M3 codes, a power of two for each block, zeros behind the last token of a used block."""
    B, Hkv, d, cap = c["B"], c["Hkv"], c["d"], c["cap"]
    nb = cap // BLOCK
    K8 = torch.zeros((B, Hkv, cap, d), dtype=torch.float8_e4m3fn, device=DEV)
    V8 = torch.zeros((B, Hkv, nb, d, BLOCK), dtype=torch.float8_e4m3fn, device=DEV)
    scales = [torch.ones((B, Hkv, nb), device=DEV) for _ in range(2)]
    gain = torch.exp(0.5 * torch.randn((2, Hkv, 1, d), generator=g, device=DEV))     # channels of a head differ
    at = torch.arange(cap, device=DEV)
    for b in range(B):
        used = (at < lengths[b]).view(1, cap, 1)
        for which in range(2):
            x = torch.randn((Hkv, cap, d), generator=g, device=DEV) * gain[which] * used
            x = x.bfloat16().float().view(Hkv, nb, BLOCK, d)
            e = _round_up_power(x.abs().amax((2, 3)))
            codes = (x * _power(-e)[:, :, None, None]).to(torch.float8_e4m3fn)
            scales[which][b] = _power(e)
            if which == 0:
                K8[b] = codes.view(Hkv, cap, d)
            else:
                V8[b] = codes.view(torch.uint8).transpose(2, 3).contiguous().view(torch.float8_e4m3fn)
    return K8, V8, scales[0], scales[1]


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _frequencies(c):
    """Radians per position of each rotated pair, in 64 bits, and the factor on the rotated values."""
    rot, s = c["rot"], c["factor"]
    base = BASE * s ** (rot / (rot - 2)) if c["scaling"] == "ntk" else BASE
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    if c["scaling"] == "linear":
        return f / s, 1.0
    if c["scaling"] != "yarn":
        return f, 1.0
    turns = _TRAINED * f / (2 * math.pi)                   # over the trained length
    keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
    return f * keep + f / s * (1 - keep), 0.1 * math.log(s) + 1.0


_TRAINED = 4096


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, generator=g, device=DEV)
    B, Hkv, d = c["B"], c["Hkv"], c["d"]
    s = {"case": c}
    if c["kind"] == "rope":
        H, N = c["H"], c["N"]
        if c["fused"]:                                     # views into one projection [B,N,H+2Hkv,d]
            x = randn(B, N, H + 2 * Hkv, d).bfloat16()
            q, k = x[:, :, :H].permute(0, 2, 1, 3), x[:, :, H:H + Hkv].permute(0, 2, 1, 3)
        else:
            q, k = randn(B, H, N, d).bfloat16(), randn(B, Hkv, N, d).bfloat16()
        r = random.Random(c["mix"])
        start = torch.tensor([r.randint(0, c["far"]) for _ in range(B)], device=DEV)
        s["positions"] = (start[:, None] + torch.arange(N, device=DEV)).int()
        s["q"], s["k"] = q.detach().requires_grad_(c["grad"]), k.detach().requires_grad_(c["grad"])
        if c["grad"]:
            s["dq"], s["dk"] = randn(B, H, N, d).bfloat16(), randn(B, Hkv, N, d).bfloat16()
        if own:
            from paper_2510_04212_amd import binding
            s["frequencies"], s["magnitude"] = binding.rope_frequencies(c["rot"], BASE, scaling=c["scaling"], factor=c["factor"],
                                                                        original_length=_TRAINED, device=DEV)
        else:
            s["frequencies"], s["magnitude"] = _frequencies(c)
        return s
    lengths, counts = _lengths(c)
    s["host_lengths"], s["host_counts"] = lengths, counts
    s["lengths"], s["counts"] = _i32(lengths), _i32(counts) if c.get("ragged") else None
    if c["kind"] == "append":
        before = [l - n for l, n in zip(lengths, counts)]
        s["cache"] = _cache(c, g, before)
        gain = torch.exp(0.7 * randn(2, Hkv, 1, d))
        s["k"], s["v"] = ((randn(B, Hkv, c["N"], d) * gain[i]).bfloat16() for i in range(2))
        # the plain form's plan: the (sequence, block) pairs that get tokens
        pairs = [(b, j) for b in range(B) if counts[b] for j in range(before[b] // BLOCK, (lengths[b] - 1) // BLOCK + 1)]
        s["touched"] = torch.tensor(pairs, device=DEV).view(-1, 2)
        return s
    s["cache"] = _cache(c, g, lengths)
    if c["kind"] == "evict":
        nb = -(-c["budget"] // BLOCK)
        s["weights"] = (torch.exp(2.0 * randn(B, Hkv, c["cap"])) * 1e-3).bfloat16().float()       # with ties
        s["out"] = (torch.zeros((B, Hkv, nb * BLOCK, d), dtype=torch.float8_e4m3fn, device=DEV),
                    torch.zeros((B, Hkv, nb, d, BLOCK), dtype=torch.float8_e4m3fn, device=DEV),
                    torch.ones((B, Hkv, nb), device=DEV), torch.ones((B, Hkv, nb), device=DEV))
        return s
    s["q"] = randn(B, c["H"], c["N"], d).bfloat16()
    s["scale"] = d ** -0.5
    if c["kind"] == "weigh":
        s["lse"] = _attend(s, values=False)[1]
        s["weights"] = torch.exp(2.0 * randn(B, Hkv, c["cap"])) * 1e-3
    return s


# ---- one pass

def run(state):
    c = state["case"]
    if own:
        return _RUN_OWN[c["kind"]](state)
    return _RUN_PLAIN[c["kind"]](state)


def _own_rope(s):
    from paper_2510_04212_amd import autograd, binding
    c = s["case"]
    if not c["grad"]:
        return binding.attn_rope(s["q"], s["k"], s["frequencies"], positions=s["positions"], interleaved=c["interleaved"],
                                 magnitude=s["magnitude"])
    q, k = autograd.rope(s["q"], s["k"], s["frequencies"], positions=s["positions"], interleaved=c["interleaved"], magnitude=s["magnitude"])
    return (q, k) + torch.autograd.grad((q, k), (s["q"], s["k"]), (s["dq"], s["dk"]))


def _own_append(s):
    from paper_2510_04212_amd import binding
    cache = binding.Cache(*s["cache"])
    binding.attn_cache_append(cache, s["k"], s["v"], s["lengths"], counts=s["counts"])
    return tuple(cache)


def _own_attend(s):
    from paper_2510_04212_amd import binding
    return binding.attn_cache_fwd(s["q"], binding.Cache(*s["cache"]), s["lengths"], s["scale"], counts=s["counts"])


def _own_weigh(s):
    from paper_2510_04212_amd import binding
    return binding.attn_cache_weights(s["q"], binding.Cache(*s["cache"]), s["lse"], s["lengths"], s["scale"], counts=s["counts"],
                                      weights=s["weights"], out=torch.empty_like(s["weights"]))


def _own_evict(s):
    from paper_2510_04212_amd import binding
    c = s["case"]
    out, weights, kept = binding.attn_cache_evict(binding.Cache(*s["cache"]), s["weights"], s["lengths"], c["budget"], c["recent"],
                                                  out=binding.Cache(*s["out"]))
    return tuple(out) + (weights, kept)


_RUN_OWN = {"rope": _own_rope, "append": _own_append, "attend": _own_attend, "weigh": _own_weigh, "evict": _own_evict}


def _rotate(x, cos, sin, c, inverse):
    rot, m = c["rot"], x.float()
    a, b = (m[..., 0:rot:2], m[..., 1:rot:2]) if c["interleaved"] else (m[..., :rot // 2], m[..., rot // 2:rot])
    if inverse:
        sin = -sin
    u, v = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((u, v), -1).flatten(-2) if c["interleaved"] else torch.cat((u, v), -1)
    return torch.cat((turned, m[..., rot:]), -1).to(x.dtype)


def _plain_rope(s):
    c = s["case"]
    angle = s["positions"].double()[:, None, :, None] * s["frequencies"]
    cos, sin = ((f(angle) * s["magnitude"]).float() for f in (torch.cos, torch.sin))
    q, k = s["q"].detach(), s["k"].detach()
    out = (_rotate(q, cos, sin, c, False), _rotate(k, cos, sin, c, False))
    if c["grad"]:
        out += (_rotate(s["dq"], cos, sin, c, True), _rotate(s["dk"], cos, sin, c, True))
    return out


def _quantise(x, old, old_scale, new, kept, fresh):
    """Codes and scales of blocks [M,64,Hkv,d]: the new tokens of x, the old codes brought to the new scale, zeros elsewhere."""
    finite = torch.where(torch.isfinite(x) & new, x, 0.0)
    e = _round_up_power(finite.abs().amax((1, 3)))                                     # [M,Hkv]
    before = torch.where(fresh[:, None], LOWEST_EXPONENT, torch.frexp(old_scale)[1] - 1)
    e = torch.maximum(e, before)
    x = torch.where(new, x * _power(-e)[:, None, :, None], 0.0)
    x = torch.where(kept, old * _power(before - e)[:, None, :, None], x)
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn), _power(e)


def _plain_append(s):
    c = s["case"]
    K8, V8, Ks, Vs = s["cache"]
    b, j = s["touched"].unbind(1)
    counts = s["lengths"] * 0 + c["N"] if s["counts"] is None else s["counts"]
    first = (s["lengths"] - counts).long()[b]                                          # position of a sequence's first new token
    at = j[:, None] * BLOCK + torch.arange(BLOCK, device=DEV)                          # [M,64] positions
    i = at - first[:, None]
    new, kept = ((i >= 0) & (i < counts.long()[b, None])), i < 0
    new, kept, i = new[:, :, None, None], kept[:, :, None, None], i.clamp(0, c["N"] - 1)
    fresh = j * BLOCK >= first
    Hkv, d, nb = c["Hkv"], c["d"], c["cap"] // BLOCK
    for x, codes, scales, turned in ((s["k"], K8, Ks, False), (s["v"], V8, Vs, True)):
        bytes_ = codes.view(torch.uint8)
        blocks = bytes_ if turned else bytes_.view(c["B"], Hkv, nb, BLOCK, d)
        old = blocks[b, :, j].view(torch.float8_e4m3fn).float()                        # [M,Hkv,d,64] or [M,Hkv,64,d]
        old = old.permute(0, 3, 1, 2) if turned else old.permute(0, 2, 1, 3)
        y, sc = _quantise(x[b[:, None], :, i].float(), old, scales[b, :, j], new, kept, fresh)
        y = y.view(torch.uint8)
        blocks[b, :, j] = y.permute(0, 2, 3, 1) if turned else y.permute(0, 2, 1, 3)
        scales[b, :, j] = sc
    return s["cache"]


def _dequantised(s, b, length, values, dtype=torch.float32):
    """K and V of one sequence, [Hkv,length,d]."""
    K8, V8, Ks, Vs = s["cache"]
    nb = -(-length // BLOCK)
    Hkv, d = K8.shape[1], K8.shape[3]
    k = (K8[b, :, :nb * BLOCK].to(dtype).view(Hkv, nb, BLOCK, d) * Ks[b, :, :nb, None, None].to(dtype)).view(Hkv, nb * BLOCK, d)[:, :length]
    if not values:
        return k, None
    v = (V8[b, :, :nb].to(dtype) * Vs[b, :, :nb, None, None].to(dtype)).transpose(2, 3).reshape(Hkv, nb * BLOCK, d)[:, :length]
    return k, v


def _scores(s, k, b, n, length):
    """Masked scores of the n queries of sequence b, [Hkv,group,n,length]."""
    c = s["case"]
    Hkv, d = c["Hkv"], c["d"]
    q = s["q"][b, :, :n].float().reshape(Hkv, -1, d)
    x = (q @ k.transpose(1, 2)).view(Hkv, c["H"] // Hkv, n, length).mul_(s["scale"])
    if n > 1:
        i, t = torch.arange(n, device=DEV)[:, None], torch.arange(length, device=DEV)
        x.masked_fill_(t > i + (length - n), -math.inf)
    return x


def _attend(s, values=True):
    c = s["case"]
    O = torch.zeros_like(s["q"])
    lse = torch.full(s["q"].shape[:3], -math.inf, device=DEV)
    for b, (length, n) in enumerate(zip(s["host_lengths"], s["host_counts"])):
        if n == 0:
            continue
        k, v = _dequantised(s, b, length, values)
        x = _scores(s, k, b, n, length)
        m = x.amax(-1, keepdim=True)
        x = x.sub_(m).exp_()
        l = x.sum(-1, keepdim=True)
        lse[b, :, :n] = (m + l.log()).view(c["H"], n)
        if values:
            o = (x.view(c["Hkv"], -1, length) @ v).view(c["Hkv"], -1, n, c["d"]) / l
            O[b, :, :n] = o.view(c["H"], n, c["d"]).to(O.dtype)
    return O, lse


def _plain_attend(s):
    return _attend(s)


def _plain_weigh(s):
    c = s["case"]
    out = torch.zeros_like(s["weights"])
    for b, (length, n) in enumerate(zip(s["host_lengths"], s["host_counts"])):
        out[b, :, :length - n] = s["weights"][b, :, :length - n]
        if n:
            k, _ = _dequantised(s, b, length, False)
            lse = s["lse"][b, :, :n].reshape(c["Hkv"], -1, n, 1)
            out[b, :, :length] += _scores(s, k, b, n, length).sub_(lse).exp_().sum((1, 2))
    return out


def _plain_evict(s):
    c = s["case"]
    K8, V8, Ks, Vs = s["cache"]
    Ko, Vo, Kso, Vso = s["out"]
    B, Hkv, d, budget = c["B"], c["Hkv"], c["d"], c["budget"]
    weights = torch.zeros((B, Hkv, Ko.shape[2]), device=DEV)
    kept = torch.full((B, Hkv, budget), -1, dtype=torch.int32, device=DEV)
    bytes_ = [t.view(torch.uint8) for t in (K8, V8, Ko, Vo)]
    for b, length in enumerate(s["host_lengths"]):
        if length <= budget:
            at = torch.arange(length, device=DEV).expand(Hkv, length)
        else:
            old = length - c["recent"]
            heavy = torch.sort(s["weights"][b, :, :old], dim=-1, descending=True, stable=True)[1][:, :budget - c["recent"]]
            last = torch.arange(old, length, device=DEV).expand(Hkv, -1)
            at = torch.cat((heavy, last), 1).sort(1)[0]
        n = at.shape[1]
        nb = -(-n // BLOCK)
        if n == 0:
            continue
        kept[b, :, :n] = at.int()
        weights[b, :, :n] = s["weights"][b].gather(1, at)
        h = torch.arange(Hkv, device=DEV)[:, None]
        inside = torch.zeros((Hkv, nb * BLOCK), dtype=torch.bool, device=DEV)
        inside[:, :n] = True
        at = torch.nn.functional.pad(at, (0, nb * BLOCK - n))
        for which, (scales, scales_out) in enumerate(((Ks, Kso), (Vs, Vso))):
            e = torch.frexp(scales[b])[1].gather(1, at // BLOCK) - 1                   # [Hkv,n']
            new = torch.where(inside, e, -(1 << 20)).view(Hkv, nb, BLOCK).amax(2)
            scales_out[b, :, :nb] = _power(new)
            x = bytes_[0][b][h, at] if which == 0 else bytes_[1][b][h, at // BLOCK, :, at % BLOCK]
            x = x.view(torch.float8_e4m3fn).float() * _power(e - new.repeat_interleave(BLOCK, 1))[:, :, None]
            x = torch.where(inside[:, :, None], x, 0.0).to(torch.float8_e4m3fn).view(torch.uint8)
            if which == 0:
                bytes_[2][b, :, :nb * BLOCK] = x
            else:
                bytes_[3][b, :, :nb] = x.view(Hkv, nb, BLOCK, d).transpose(2, 3)
    return s["out"] + (weights, kept)


_RUN_PLAIN = {"rope": _plain_rope, "append": _plain_append, "attend": _plain_attend, "weigh": _plain_weigh, "evict": _plain_evict}


# ---- the definitions in 64 bits, written apart

def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return _EXACT[case["kind"]](s)


def _exact_rope(s):
    c = s["case"]
    rot, half = c["rot"], c["rot"] // 2
    first = [2 * i if c["interleaved"] else i for i in range(half)]
    second = [2 * i + 1 if c["interleaved"] else i + half for i in range(half)]
    phase = torch.exp(1j * s["positions"].double()[:, None, :, None] * s["frequencies"]) * s["magnitude"]

    def turn(x, by):
        y = x.detach().double().clone()
        z = torch.complex(y[..., first], y[..., second]) * by
        y[..., first], y[..., second] = z.real, z.imag
        return y

    out = (turn(s["q"], phase), turn(s["k"], phase))
    if c["grad"]:
        out += (turn(s["dq"], phase.conj()), turn(s["dk"], phase.conj()))
    return out


def _nearest_e4m3(x):
    """The nearest E4M3 number, ties to the even code: spacing 2^(floor(log2|x|) - 3), 2^-9 below 2^-6."""
    a = x.abs()
    step = torch.exp2((torch.floor(torch.log2(torch.where(a > 0, a, 1.0)))).clamp(min=-6.0) - 3.0)
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def _power_for(amax):
    """The least power of two p >= 2^-100 with amax <= 448 p, by looking on both sides of the logarithm."""
    e = torch.floor(torch.log2(torch.where(amax > 0, amax, 1.0) / 448.0))
    for _ in range(2):
        e = torch.where(448.0 * torch.exp2(e) < amax, e + 1, e)
    return torch.where(amax > 0, e, -100.0).clamp(min=-100.0)


def _exact_append(s):
    c = s["case"]
    d, cap, Hkv = c["d"], c["cap"], c["Hkv"]
    K8, V8, Ks, Vs = s["cache"]
    both = [(K8.double(), Ks.double(), s["k"].double()), (V8.double().transpose(3, 4).reshape(K8.shape), Vs.double(), s["v"].double())]
    for codes, scales, x in both:
        for b, (length, n) in enumerate(zip(s["host_lengths"], s["host_counts"])):
            at = length - n
            while at < length:                                                         # one piece of a block after the other
                j, to = at // BLOCK, min(length, (at // BLOCK + 1) * BLOCK)
                piece = x[b, :, at - (length - n):to - (length - n)]
                e = _power_for(piece.abs().amax((1, 2)))
                lo, hi = j * BLOCK, (j + 1) * BLOCK
                if at > lo:
                    e = torch.maximum(e, torch.log2(scales[b, :, j]))
                    codes[b, :, lo:at] = _nearest_e4m3(codes[b, :, lo:at] * (scales[b, :, j] / torch.exp2(e))[:, None, None])
                codes[b, :, at:to] = _nearest_e4m3(piece / torch.exp2(e)[:, None, None])
                codes[b, :, to:hi] = 0.0
                scales[b, :, j] = torch.exp2(e)
                at = to
    (k, ks, _), (v, vs, _) = both
    return k, v.view(c["B"], Hkv, cap // BLOCK, BLOCK, d).transpose(3, 4).contiguous(), ks, vs


def _exact_rows(s, b, h, n, length, want_values):
    """Scores in 64 bits of the query heads of key/value head h, [group,n,length], and V."""
    c = s["case"]
    K8, V8, Ks, Vs = s["cache"]
    group = c["H"] // c["Hkv"]
    block = torch.arange(length, device=DEV) // BLOCK
    k = K8[b, h, :length].double() * Ks[b, h].double()[block][:, None]
    x = torch.matmul(s["q"][b, h * group:(h + 1) * group, :n].double(), k.t()) * s["scale"]
    hidden = torch.ones((n, length), dtype=torch.bool, device=DEV).triu(length - n + 1)
    v = None
    if want_values:
        v = V8[b, h].double().transpose(1, 2).reshape(-1, c["d"])[:length] * Vs[b, h].double()[block][:, None]
    return x.masked_fill(hidden, -math.inf), v


def _exact_attend(s):
    c = s["case"]
    group = c["H"] // c["Hkv"]
    O, lse = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV), torch.full(s["q"].shape[:3], -math.inf, dtype=torch.float64, device=DEV)
    for b, (length, n) in enumerate(zip(s["host_lengths"], s["host_counts"])):
        for h in range(c["Hkv"]) if n else ():
            x, v = _exact_rows(s, b, h, n, length, True)
            rows = slice(h * group, (h + 1) * group)
            lse[b, rows, :n] = torch.logsumexp(x, -1)
            O[b, rows, :n] = torch.softmax(x, -1) @ v
    return O, lse


def _exact_weigh(s):
    c = s["case"]
    group = c["H"] // c["Hkv"]
    out = s["weights"].double()
    for b, (length, n) in enumerate(zip(s["host_lengths"], s["host_counts"])):
        out[b, :, length - n:] = 0.0
        for h in range(c["Hkv"]) if n else ():
            x, _ = _exact_rows(s, b, h, n, length, False)
            out[b, h, :length] += torch.exp(x - s["lse"][b, h * group:(h + 1) * group, :n].double()[..., None]).sum((0, 1))
    return out


def _exact_evict(s):
    c = s["case"]
    K8, V8, Ks, Vs = s["cache"]
    out = [t.double() for t in s["out"]]
    kept = torch.full((c["B"], c["Hkv"], c["budget"]), -1, dtype=torch.int64)
    weights = torch.zeros((c["B"], c["Hkv"], s["out"][0].shape[2]), dtype=torch.float64, device=DEV)
    host = s["weights"].cpu()
    for b, length in enumerate(s["host_lengths"]):
        for h in range(c["Hkv"]):
            old = max(0, length - c["recent"])
            w = host[b, h, :old].double().numpy()
            heaviest = (-w).argsort(kind="stable")[:max(0, min(length, c["budget"]) - (length - old))]
            at = torch.tensor(sorted(heaviest.tolist()) + list(range(old, length)), dtype=torch.int64)[-c["budget"]:]
            n = len(at)
            kept[b, h, :n] = at
            if n == 0:
                continue
            at = at.to(DEV)
            weights[b, h, :n] = s["weights"][b, h].double()[at]
            block, blocks = at // BLOCK, -(-n // BLOCK)
            k, v = K8[b, h].double()[at], V8[b, h].double()[block, :, at % BLOCK]
            for x, scales, o in ((k, Ks, 0), (v, Vs, 1)):
                whole = torch.zeros((blocks * BLOCK, c["d"]), dtype=torch.float64, device=DEV)
                power = torch.zeros(blocks * BLOCK, dtype=torch.float64, device=DEV)
                power[:n] = scales[b, h].double()[block]
                whole[:n] = x * power[:n, None]
                p = power.view(blocks, BLOCK).amax(1)
                y = _nearest_e4m3(whole.view(blocks, BLOCK, -1) / p[:, None, None])
                out[2 + o][b, h, :blocks] = p
                if o == 0:
                    out[0][b, h, :blocks * BLOCK] = y.view(blocks * BLOCK, -1)
                else:
                    out[1][b, h, :blocks] = y.transpose(1, 2)
    return tuple(out) + (weights, kept.to(DEV))


_EXACT = {"rope": _exact_rope, "append": _exact_append, "attend": _exact_attend, "weigh": _exact_weigh, "evict": _exact_evict}
