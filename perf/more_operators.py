"""Timing cases of what continues one prompt several times: attention over a cache whose prefix several sequences share, copies of
cached sequences, and the choice among beams.

A case is a dict of plain values.  Its kind says which operator runs:
  attend   N queries a head of each of P * S sequences against their prefix's cache (sequence b continues prefix b // S) and against their own,
           causal in their own, aligned at the bottom right
  fork     a cache whose sequences are copies of another's: sequence i of sources[i]
  reorder  the sequences of a cache replaced by others of their group of S, in place
  select   the n best continuations of each of B prompts, of `beams` beams and V tokens
and the sizes are H query heads, Hkv key/value heads, head size d, capacity cap (pcap of the prefixes); lengths are spread over lo .. cap
(plo .. pcap) by `mix`; ragged: sequences bring fewer than N tokens (a padded batch).

Caches: K [B,Hkv,cap,d] and V [B,Hkv,cap/64,d,64] in E4M3, one scale (a power of two) for each 64 tokens of a head, K and V apart.

own: False, the operators in elementary torch operations; True, the framework's kernels.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
BLOCK = 64
LOWEST_EXPONENT = -100      # of a scale
END = 2                     # the token that ends a sequence


def listed():
    return [
        # four beams of one short prompt in a small model with 12 plain heads: the smallest answer, latency alone
        dict(name="attend one", kind="attend", P=1, S=4, H=12, Hkv=12, N=1, d=64, pcap=1024, plo=700, cap=128, lo=16, ragged=False, mix=1),
        # a token of eight beams each of sixteen prompts
        dict(name="attend beams", kind="attend", P=16, S=8, H=32, Hkv=8, N=1, d=128, pcap=4096, plo=1000, cap=512, lo=32, ragged=False, mix=2),
        # a token of 64 conversations that begin with the same instructions
        dict(name="attend batch", kind="attend", P=1, S=64, H=32, Hkv=8, N=1, d=128, pcap=8192, plo=8000, cap=2048, lo=64, ragged=False, mix=3),
        # a token of 16 answers about one long document
        dict(name="attend long", kind="attend", P=1, S=16, H=32, Hkv=4, N=1, d=128, pcap=131072, plo=130000, cap=1024, lo=100, ragged=False, mix=4),
        # eight short questions each about two documents, padded to the longest
        dict(name="attend chunk", kind="attend", P=2, S=8, H=32, Hkv=8, N=64, d=128, pcap=8192, plo=6000, cap=1024, lo=64, ragged=True, mix=5),
        # a prompt's cache for each of eight answers
        dict(name="fork prompt", kind="fork", B=1, out=8, Hkv=8, d=128, cap=2048, lo=1500, cap_out=2304, mix=6),
        # a batch in which 16 of 64 conversations have ended, moved together
        dict(name="fork batch", kind="fork", B=64, out=48, Hkv=8, d=128, cap=4096, lo=64, cap_out=4096, mix=7),
        # the young beams of four prompts in a small model
        dict(name="reorder young", kind="reorder", P=4, S=4, Hkv=12, d=64, cap=256, lo=16, mix=8),
        # the long beams of sixteen prompts
        dict(name="reorder long", kind="reorder", P=16, S=8, Hkv=8, d=128, cap=2048, lo=300, mix=9),
        # four beams of one prompt: latency
        dict(name="select one", kind="select", B=1, beams=4, V=32000, n=8, wide=True, pad=0, ended=False, first=False, mix=10),
        # a vocabulary of odd size in 16 bits; some beams have ended
        dict(name="select odd", kind="select", B=6, beams=5, V=50257, n=5, wide=False, pad=0, ended=True, first=False, mix=11),
        # eight beams each of 32 prompts, twice as many continuations as beams, a large vocabulary
        dict(name="select batch", kind="select", B=32, beams=8, V=131072, n=16, wide=True, pad=0, ended=False, first=False, mix=12),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


_MOST_BYTES, _MOST_FLOPS, _MOST_SCORES = 4e8, 1.2e11, 2.5e8        # of a drawn case


def draw(rng):
    while True:
        kind = rng.choice(("attend", "attend", "attend", "fork", "reorder", "select", "select"))
        d = rng.choice((32, 64, 64, 96, 128, 128, 128, 256))
        Hkv = rng.choice((1, 2, 3, 4, 8, 12))
        mix = rng.randrange(1 << 20)
        if kind == "select":
            beams = _log_int(rng, 1, 32)
            V = _log_int(rng, 100, 200000)
            c = dict(kind=kind, B=_log_int(rng, 1, 64), beams=beams, V=V, n=min(V, rng.choice((beams, 2 * beams, rng.randint(1, 64)))), wide=rng.random() < 0.5,
                     pad=rng.choice((0, 0, -V % 64)), ended=rng.random() < 0.5, first=rng.random() < 0.2, mix=mix)
        elif kind == "fork":
            cap = BLOCK * _log_int(rng, 1, 512)
            c = dict(kind=kind, B=_log_int(rng, 1, 64), out=_log_int(rng, 1, 64), Hkv=Hkv, d=d, cap=cap, lo=rng.randint(0, cap),
                     cap_out=BLOCK * rng.randint(-(-cap // (2 * BLOCK)), 2 * cap // BLOCK), mix=mix)
        elif kind == "reorder":
            cap = BLOCK * _log_int(rng, 1, 512)
            c = dict(kind=kind, P=_log_int(rng, 1, 32), S=_log_int(rng, 2, 32), Hkv=Hkv, d=d, cap=cap, lo=rng.randint(0, cap), mix=mix)
        else:
            pcap, cap = BLOCK * _log_int(rng, 1, 2048), BLOCK * _log_int(rng, 1, 64)
            N = rng.choice((1, 1, 1, rng.randint(1, 8), _log_int(rng, 1, min(cap, 256))))
            c = dict(kind=kind, P=rng.choice((1, 1, _log_int(rng, 1, 16))), S=_log_int(rng, 1, 64), H=Hkv * rng.choice((1, 2, 4, 5, 8)), Hkv=Hkv, N=N, d=d,
                     pcap=pcap, plo=rng.randint(0, pcap), cap=cap, lo=rng.randint(N, cap), ragged=N > 1 and rng.random() < 0.5, mix=mix)
        w = work(c)
        slots = 2.0 * Hkv * d * (c.get("P", 0) * c.get("pcap", 0) + c.get("P", 1) * c.get("S", c.get("B", 0)) * c.get("cap", 0)
                                 + c.get("out", 0) * c.get("cap_out", 0))                  # what the caches hold, used or not
        scores = c["P"] * c["S"] * c["H"] * c["N"] * float(c["pcap"] + c["cap"]) if kind == "attend" else 0.0
        if w["bytes"] <= _MOST_BYTES and w["flops"] <= _MOST_FLOPS and slots <= 2 * _MOST_BYTES and scores <= _MOST_SCORES:
            return c


# ---- what a case says beyond its sizes, whatever the seed

def _lengths(c):
    """Tokens of each sequence in its own cache, the new ones among them, how many are new, and tokens of each prefix."""
    r = random.Random(c["mix"])
    B = c["B"] if c["kind"] == "fork" else c["P"] * c["S"]
    lengths = [r.randint(c["lo"], c["cap"]) for _ in range(B)]
    if c["kind"] != "attend":
        return lengths, None, None
    counts = [c["N"]] * B
    if c["ragged"]:
        counts = [c["N"]] + [r.randint(0, c["N"]) for _ in range(B - 1)]
    return lengths, counts, [r.randint(c["plo"], c["pcap"]) for _ in range(c["P"])]


def _sources(c):
    """fork: copies of one sequence, or of some of them in their order; otherwise of any."""
    r = random.Random(c["mix"] + 1)
    if c["out"] <= c["B"]:
        return sorted(r.sample(range(c["B"]), c["out"]))
    return [r.randrange(c["B"]) for _ in range(c["out"])]


def _parents(c):
    """reorder: beams that go on keep their place, and the places of the others go to copies of them."""
    r = random.Random(c["mix"] + 1)
    groups = []
    for _ in range(c["P"]):
        stay = sorted(r.sample(range(c["S"]), r.randint(1, c["S"] - 1)))
        groups.append([s if s in stay else r.choice(stay) for s in range(c["S"])])
    return groups


def _blocks(n):
    return -(-n // BLOCK)


def work(case):
    c = case
    if c["kind"] == "select":
        logits = float(c["B"]) * c["beams"] * c["V"]
        return {"bytes": logits * (4 if c["wide"] else 2) + c["B"] * (5.0 * c["beams"] + 13.0 * c["n"]), "flops": 4.0 * logits}
    per_block = c["Hkv"] * (2.0 * BLOCK * c["d"] + 8)
    lengths, counts, prefixes = _lengths(c)
    if c["kind"] == "fork":
        sources = _sources(c)
        size = [_blocks(min(n, c["cap_out"])) for n in lengths]
        return {"bytes": per_block * (sum(size[s] for s in set(sources)) + sum(size[s] for s in sources)), "flops": 0.0}
    if c["kind"] == "reorder":
        moved = read = 0
        for p, parents in enumerate(_parents(c)):
            goes = [s for s, parent in enumerate(parents) if s != parent]
            moved += sum(_blocks(lengths[p * c["S"] + parents[s]]) for s in goes)
            read += sum(_blocks(lengths[p * c["S"] + s]) for s in {parents[s] for s in goes})
        return {"bytes": max(per_block * (moved + read), 8.0 * len(lengths)), "flops": 0.0}
    S, d = c["S"], c["d"]
    pairs = sum(n * (prefixes[b // S] + l) - n * (n - 1) // 2 for b, (n, l) in enumerate(zip(counts, lengths)))
    tokens = sum(prefixes) + sum(l for l, n in zip(lengths, counts) if n)
    return {"bytes": 2.0 * c["Hkv"] * d * tokens + c["H"] * sum(counts) * (4.0 * d + 4), "flops": 4.0 * d * c["H"] * pairs}


# ---- inputs

def _power(e):
    """2^e in float32 by its bits; 2^-126 for less."""
    return ((e.int().clamp(min=-126) + 127) << 23).view(torch.float32)


def _cache(g, B, Hkv, cap, d, lengths):
    """A cache as appending left it: E4M3 codes, for each block the least power of two that reaches its values, zeros behind the last token."""
    nb = cap // BLOCK
    K8 = torch.zeros((B, Hkv, cap, d), dtype=torch.float8_e4m3fn, device=DEV)
    V8 = torch.zeros((B, Hkv, nb, d, BLOCK), dtype=torch.float8_e4m3fn, device=DEV)
    scales = [torch.ones((B, Hkv, nb), device=DEV) for _ in range(2)]
    gain = torch.exp(0.5 * torch.randn((2, Hkv, 1, d), generator=g, device=DEV))           # channels of a head differ
    for b in range(B):
        n = _blocks(lengths[b])
        used = (torch.arange(n * BLOCK, device=DEV) < lengths[b]).view(n * BLOCK, 1)
        for which in range(2 if n else 0):
            x = torch.randn((Hkv, n * BLOCK, d), generator=g, device=DEV) * gain[which] * used
            x = x.bfloat16().float().view(Hkv, n, BLOCK, d)
            m, e = torch.frexp(x.abs().amax((2, 3)))                                       # amax = m 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
            e = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=LOWEST_EXPONENT)
            codes = (x * _power(-e)[:, :, None, None]).to(torch.float8_e4m3fn)
            scales[which][b, :, :n] = _power(e)
            if which == 0:
                K8[b, :, :n * BLOCK] = codes.view(Hkv, n * BLOCK, d)
            else:
                V8[b, :, :n] = codes.view(torch.uint8).transpose(2, 3).contiguous().view(torch.float8_e4m3fn)
    return K8, V8, scales[0], scales[1]


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, generator=g, device=DEV)
    rand = lambda *shape: torch.rand(shape, generator=g, device=DEV)
    s = {"case": c}
    if c["kind"] == "select":
        B, beams, V = c["B"], c["beams"], c["V"]
        x = randn(B, beams, V + c["pad"]) * 2.5 + 1.5 * randn(V + c["pad"])                # tokens that all beams find likely
        x[rand(B, beams, V + c["pad"]) < 0.01] = -math.inf                                 # and forbidden ones
        s["logits"] = (x if c["wide"] else x.bfloat16())[:, :, :V]
        s["scores"] = -(rand(B, beams) * 6.0 + 4.0)
        s["ended"] = None
        if c["first"]:                                     # the first step: all beams are the same, one counts
            s["scores"][:, 1:] = -math.inf
        elif c["ended"]:
            s["ended"] = rand(B, beams) < 0.25
        return s
    d, Hkv = c["d"], c["Hkv"]
    lengths, counts, prefixes = _lengths(c)
    s["host_lengths"], s["lengths"] = lengths, _i32(lengths)
    s["cache"] = _cache(g, len(lengths), Hkv, c["cap"], d, lengths)
    if c["kind"] == "fork":
        nb = c["cap_out"] // BLOCK
        s["sources"] = _i32(_sources(c))
        s["out"] = (torch.zeros((c["out"], Hkv, nb * BLOCK, d), dtype=torch.float8_e4m3fn, device=DEV),
                    torch.zeros((c["out"], Hkv, nb, d, BLOCK), dtype=torch.float8_e4m3fn, device=DEV),
                    torch.ones((c["out"], Hkv, nb), device=DEV), torch.ones((c["out"], Hkv, nb), device=DEV))
    elif c["kind"] == "reorder":
        s["parents"] = _i32(_parents(c))
    else:
        s["host_counts"], s["host_prefixes"] = counts, prefixes
        s["counts"] = _i32(counts) if c["ragged"] else None
        s["prefix_lengths"] = _i32(prefixes)
        s["prefix"] = _cache(g, c["P"], Hkv, c["pcap"], d, prefixes)
        s["q"] = randn(len(lengths), c["H"], c["N"], d).bfloat16()
        s["scale"] = d ** -0.5
    return s


# ---- one pass

def run(state):
    c = state["case"]
    if own:
        return _RUN_OWN[c["kind"]](state)
    return _RUN_PLAIN[c["kind"]](state)


def _own_attend(s):
    from paper_2510_04212_amd import binding
    return binding.attn_cache_fwd_shared(s["q"], binding.Cache(*s["prefix"]), s["prefix_lengths"], binding.Cache(*s["cache"]), s["lengths"], s["scale"],
                                         counts=s["counts"])


def _own_fork(s):
    from paper_2510_04212_amd import binding
    out, lengths = binding.attn_cache_fork(binding.Cache(*s["cache"]), s["sources"], s["lengths"], out=binding.Cache(*s["out"]))
    return tuple(out) + (lengths,)


def _own_reorder(s):
    from paper_2510_04212_amd import binding
    lengths = binding.attn_cache_reorder(binding.Cache(*s["cache"]), s["parents"], s["lengths"])
    return s["cache"] + (lengths,)


def _own_select(s):
    from paper_2510_04212_amd import binding
    return binding.attn_beam_select(s["logits"], s["scores"], s["case"]["n"], finished=s["ended"], end_token=END)


_RUN_OWN = {"attend": _own_attend, "fork": _own_fork, "reorder": _own_reorder, "select": _own_select}


def _values(cache):
    """K and V in float32, [B,Hkv,cap,d]."""
    K8, V8, Ks, Vs = cache
    B, Hkv, cap, d = K8.shape
    k = (K8.float().view(B, Hkv, -1, BLOCK, d) * Ks[..., None, None]).view(K8.shape)
    v = (V8.float() * Vs[..., None, None]).transpose(3, 4).reshape(K8.shape)
    return k, v


def _plain_attend(s):
    c = s["case"]
    P, S, H, Hkv, N, d = (c[k] for k in ("P", "S", "H", "Hkv", "N", "d"))
    B, group = P * S, H // Hkv
    kp, vp = _values(s["prefix"])
    ko, vo = _values(s["cache"])
    counts = torch.full_like(s["lengths"], N) if s["counts"] is None else s["counts"]
    i = torch.arange(N, device=DEV)
    # the prefix: all rows of its sequences against it; [P,Hkv,S,group,N,pcap]
    q = s["q"].float().reshape(P, S, Hkv, group, N, d)
    xp = (q.transpose(1, 2).reshape(P, Hkv, -1, d) @ kp.transpose(2, 3)).mul_(s["scale"])
    xp.masked_fill_(torch.arange(c["pcap"], device=DEV) >= s["prefix_lengths"][:, None, None, None], -math.inf)
    # their own: [B,Hkv,group,N,cap]
    xo = (q.reshape(B, Hkv, -1, d) @ ko.transpose(2, 3)).mul_(s["scale"]).reshape(B, Hkv, group, N, c["cap"])
    last = (s["lengths"] - counts)[:, None] + i                                            # [B,N]
    xo.masked_fill_(torch.arange(c["cap"], device=DEV) > last[:, None, None, :, None], -math.inf)
    back = lambda x: x.reshape(P, Hkv, S, group, N, -1).transpose(1, 2).reshape(B, Hkv, group, N, -1)
    m = torch.maximum(back(xp.amax(-1, keepdim=True)), xo.amax(-1, keepdim=True))
    safe = torch.where(m == -math.inf, 0.0, m)
    xp.sub_(safe.reshape(P, S, Hkv, group * N, 1).transpose(1, 2).reshape(P, Hkv, -1, 1)).exp_()
    xo.sub_(safe).exp_()
    l = back(xp.sum(-1, keepdim=True)) + xo.sum(-1, keepdim=True)
    o = back(xp @ vp) + (xo.reshape(B, Hkv, -1, c["cap"]) @ vo).reshape(B, Hkv, group, N, d)
    there = (i < counts[:, None])[:, None, None, :, None] & (l > 0)
    O = torch.where(there, o / torch.where(there, l, 1.0), 0.0).reshape(B, H, N, d).to(s["q"].dtype)
    return O, torch.where(there, safe + l.log(), -math.inf).reshape(B, H, N)


def _gather(cache, into, sources, lengths):
    """Blocks of the sequences `sources` of a cache into another (or the same): those with tokens."""
    nb = min(cache[2].shape[2], into[2].shape[2])
    blocks = torch.arange(nb, device=DEV) < ((lengths + BLOCK - 1) // BLOCK)[:, None]     # [B,nb]
    for x, y in zip(cache, into):
        if x.dtype == torch.float32:
            x, y, has = x[:, :, :nb], y[:, :, :nb], blocks[:, None]
        else:
            flat = lambda t: t.view(torch.uint8).view(t.shape[0], t.shape[1], -1, BLOCK * cache[0].shape[3])[:, :, :nb]
            x, y, has = flat(x), flat(y), blocks[:, None, :, None]
        y.copy_(torch.where(has, x[sources], y))


def _plain_fork(s):
    at = s["sources"].long()
    lengths = s["lengths"][at].clamp(min=0, max=min(s["case"]["cap"], s["case"]["cap_out"]))
    _gather(s["cache"], s["out"], at, lengths)
    return s["out"] + (lengths,)


def _plain_reorder(s):
    S = s["case"]["S"]
    at = (s["parents"] + S * torch.arange(s["case"]["P"], device=DEV)[:, None]).view(-1)
    lengths = s["lengths"][at]
    _gather(s["cache"], s["cache"], at, lengths)
    return s["cache"] + (lengths,)


def _plain_select(s):
    """In 64 bits: candidates of different beams can be next to one another."""
    c = s["case"]
    x = s["logits"].double()
    m = x.amax(-1, keepdim=True)
    x = s["scores"].double()[..., None] + x.sub_(m).sub_(torch.exp(x).sum(-1, keepdim=True).log())
    if s["ended"] is not None:
        x.masked_fill_(s["ended"][..., None], -math.inf)
        x[:, :, END] = torch.where(s["ended"], s["scores"].double(), x[:, :, END])
    total, at = torch.sort(x.view(c["B"], -1), dim=-1, descending=True, stable=True)
    total, at = total[:, :c["n"]], at[:, :c["n"]]
    there = total > -math.inf
    parents, tokens = torch.where(there, at // c["V"], -1), torch.where(there, at % c["V"], -1)
    ended = there & (tokens == END)
    if s["ended"] is not None:
        ended |= there & s["ended"].gather(1, parents.clamp(min=0))
    return parents.int(), tokens.int(), total.float(), ended


_RUN_PLAIN = {"attend": _plain_attend, "fork": _plain_fork, "reorder": _plain_reorder, "select": _plain_select}


# ---- the definitions in 64 bits, written apart

def exact(case, seed):
    return _EXACT[case["kind"]](prepare(case, seed))


def _tokens_of(cache, b, h, length):
    """K and V of a head's first `length` tokens in 64 bits."""
    K8, V8, Ks, Vs = cache
    block = torch.arange(length, device=DEV) // BLOCK
    v = V8[b, h, :_blocks(length)].double().transpose(1, 2).reshape(-1, K8.shape[3])[:length]
    return K8[b, h, :length].double() * Ks[b, h].double()[block, None], v * Vs[b, h].double()[block, None]


def _exact_attend(s):
    c = s["case"]
    group = c["H"] // c["Hkv"]
    O, lse = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV), torch.full(s["q"].shape[:3], -math.inf, dtype=torch.float64, device=DEV)
    for h in range(c["Hkv"]):
        rows = slice(h * group, (h + 1) * group)
        for p in range(c["P"]):
            before = _tokens_of(s["prefix"], p, h, s["host_prefixes"][p])
            for b in range(p * c["S"], (p + 1) * c["S"]):
                n, length = s["host_counts"][b], s["host_lengths"][b]
                if n == 0:
                    continue
                k, v = (torch.cat(x) for x in zip(before, _tokens_of(s["cache"], b, h, length)))
                hidden = torch.ones((n, len(k)), dtype=torch.bool, device=DEV).triu(len(k) - n + 1)
                x = torch.matmul(s["q"][b, rows, :n].double(), k.t()).mul(s["scale"]).masked_fill(hidden, -math.inf)
                lse[b, rows, :n] = torch.logsumexp(x, -1)
                O[b, rows, :n] = torch.softmax(x, -1) @ v
    return O, lse


def _copied(cache, into, pairs, lengths, most):
    """[into with the blocks of the sequences (from, to)] in 64 bits, and the lengths."""
    out, left = [t.double() for t in into], torch.zeros(len(into[0]), dtype=torch.int32)
    for a, b in pairs:
        n = min(lengths[a], most)
        left[b] = n
        blocks = _blocks(n)
        out[0][b, :, :blocks * BLOCK] = cache[0][a, :, :blocks * BLOCK].double()
        for i in (1, 2, 3):
            out[i][b, :, :blocks] = cache[i][a, :, :blocks].double()
    return tuple(out) + (left,)


def _exact_fork(s):
    c = s["case"]
    return _copied(s["cache"], s["out"], [(a, i) for i, a in enumerate(_sources(c))], s["host_lengths"], min(c["cap"], c["cap_out"]))


def _exact_reorder(s):
    c = s["case"]
    pairs = [(p * c["S"] + a, p * c["S"] + i) for p, parents in enumerate(_parents(c)) for i, a in enumerate(parents)]
    return _copied(s["cache"], s["cache"], pairs, s["host_lengths"], c["cap"])


def _exact_select(s):
    c = s["case"]
    B, n, V = c["B"], c["n"], c["V"]
    parents, tokens = (torch.full((B, n), -1, dtype=torch.int32) for _ in range(2))
    total, ended = torch.full((B, n), -math.inf, dtype=torch.float64), torch.zeros((B, n), dtype=torch.bool)
    for b in range(B):
        candidates = []
        for k in range(c["beams"]):
            score = s["scores"][b, k].item()
            if s["ended"] is not None and s["ended"][b, k]:
                candidates.append((-score, k, END, True))
                continue
            x = s["logits"][b, k].double()
            x = score + (x - torch.logsumexp(x, 0))
            least = torch.topk(x, min(n, V))[0][-1]
            at = torch.nonzero((x >= least) & (x > -math.inf))[:, 0]
            candidates += [(-y, k, t, t == END) for y, t in zip(x[at].tolist(), at.tolist())]
        for j, (y, k, t, e) in enumerate(sorted(candidates)[:n]):
            if y < math.inf:
                parents[b, j], tokens[b, j], total[b, j], ended[b, j] = k, t, -y, e
    return parents, tokens, total, ended


_EXACT = {"attend": _exact_attend, "fork": _exact_fork, "reorder": _exact_reorder, "select": _exact_select}
