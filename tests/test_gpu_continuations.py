"""One prompt, many continuations (attn_cache_fwd_shared, attn_cache_fork, attn_cache_reorder, attn_beam_select) against the 64-bit oracle.

Copies and choices have to be the oracle's.  Tolerances of attention: those of test_gpu_cache.py, whose arithmetic this is:
  scores   within e = 2 (d + 4) 2^-24 alpha sum |q k| + 2^-22 |S|;  LSE  e + 2^-16;
  O        (2^-8 + e + 2^-16) (sum P |v| + |O|) and one bf16 rounding.
Sums of the choice among beams: float32 exponentials of x - m, each within (|x - m| + 2) 2^-23 of itself, so that with |x - m| e^(x - m) <= 1/e the
logarithm of their sum is within 4 * 2^-23 (the |x - m|-weighted mean is below log V + 1 <= 20: 22 * 2^-23); a thread's sum of 32 adds 32 * 2^-24; the
result is rounded to float32: 2^-24 of itself.  Together: 40 * 2^-23 + 2^-23 |sum|.  Candidates of different beams are further apart than these sums are off,
or exactly equal: an order that they leave open would show as a difference."""
import numpy as np
import pytest
import torch

from oracle import beams as oracle
from paper_2510_04212_amd import binding
from test_gpu_cache import DEV, DIMS, _bf16, _dequantised, _filled, _garbage, _gen, _i32

pytestmark = pytest.mark.gpu


# ---- attention

def _check(q, prefix, prefix_lengths, cache, lengths, counts, alpha, causal, O, lse, label=""):
    B, H, N, d = q.shape
    (Kp, Vp), (K, V) = _dequantised(prefix), _dequantised(cache)
    S, group = B // Kp.shape[0], H // K.shape[1]
    q, O, L = q.double().cpu().numpy(), O.double().cpu().numpy(), lse.double().cpu().numpy()
    for b in range(B):
        n, length, before = counts[b], lengths[b], prefix_lengths[b // S]
        for h in range(H):
            at = h // group
            of_prefix, own = (Kp[b // S, at, :before], Vp[b // S, at, :before]), (K[b, at, :length], V[b, at, :length])
            o, l, size = oracle.attend(q[b, h], of_prefix, own, n, alpha, causal)
            none = np.isneginf(l)
            assert np.array_equal(none, np.isneginf(L[b, h])) and (O[b, h][none] == 0).all(), (label, b, h)
            if none.all():
                continue
            x, k = q[b, h], np.concatenate((of_prefix[0], own[0]))
            e = 2 * (d + 4) * 2.0 ** -24 * alpha * (np.abs(x) @ np.abs(k.T)).max(1) + 2.0 ** -22 * np.abs(alpha * x @ k.T).max(1) + 2.0 ** -16
            off = np.abs(L[b, h][~none] - l[~none]) - e[~none]
            assert off.max() <= 0, (label, "LSE", b, h, off.max())
            off = np.abs(O[b, h] - o) - (2.0 ** -8 * np.abs(o) + (2.0 ** -8 + e[:, None]) * 1.01 * (size + np.abs(o)))
            assert off[~none].max() <= 0, (label, "O", b, h, off.max())


def _problem(seed, P, S, group, Hkv, N, d, pcap, prefix_lengths, cap, lengths):
    g = _gen(seed)
    prefix, cache = _filled(g, P, Hkv, pcap, d, prefix_lengths), _filled(g, P * S, Hkv, cap, d, lengths)
    return _bf16(g, P * S, group * Hkv, N, d).to(DEV), prefix, cache


def _run(q, prefix, prefix_lengths, cache, lengths, counts=None, alpha=None, causal=True, label="", **kw):
    alpha = q.shape[3] ** -0.5 if alpha is None else alpha
    O, lse = binding.attn_cache_fwd_shared(q, prefix, _i32(prefix_lengths), cache, _i32(lengths), alpha, causal, None if counts is None else _i32(counts), **kw)
    _check(q, prefix, prefix_lengths, cache, lengths, [q.shape[2]] * q.shape[0] if counts is None else counts, alpha, causal, O, lse, label)
    return O, lse


def _some(seed, n, lo, hi):
    g = np.random.default_rng(seed)
    return [int(x) for x in g.integers(lo, hi + 1, n)]


@pytest.mark.parametrize("d", DIMS)
@pytest.mark.parametrize("P,S", [(1, 1), (1, 5), (3, 2), (2, 17), (1, 40)])
def test_single_tokens(lib, d, P, S):
    for group, Hkv, pcap, cap in ((1, 2, 64, 64), (4, 1, 1088, 128), (3, 2, 320, 192), (1, 3, 192, 64), (2, 9, 128, 128), (4, 4, 640, 192)):
        prefix_lengths = [pcap, 1, 65][:P] if P > 1 else [pcap - 1]
        lengths = [1, 64, cap, 63][:P * S] + _some(d + S, max(0, P * S - 4), 1, cap)
        q, prefix, cache = _problem(S + group, P, S, group, Hkv, 1, d, pcap, prefix_lengths, cap, lengths)
        _run(q, prefix, prefix_lengths, cache, lengths, label=f"group {group}")


@pytest.mark.parametrize("d", DIMS)
@pytest.mark.parametrize("causal", (True, False))
def test_chunks(lib, d, causal):
    for N, P, S, group, Hkv, pcap, cap in ((2, 2, 3, 4, 1, 192, 128), (9, 1, 4, 2, 2, 448, 64), (40, 2, 2, 1, 2, 1024, 192), (70, 1, 3, 3, 1, 128, 128)):
        prefix_lengths = [pcap - 5, 64][:P]
        lengths = [min(cap, N + x) for x in _some(N, P * S, 0, cap)]
        counts = [N] + _some(N + d, P * S - 1, 0, N)
        q, prefix, cache = _problem(N, P, S, group, Hkv, N, d, pcap, prefix_lengths, cap, lengths)
        _run(q, prefix, prefix_lengths, cache, lengths, counts, 1.5 * d ** -0.5, causal, f"N {N} ragged")
        _run(q, prefix, prefix_lengths, cache, lengths, None, d ** -0.5, causal, f"N {N}")


def _values_on_gpu(c):
    """K and V of a cache in 64 bits, [B,Hkv,cap,d]."""
    B, Hkv, cap, d = c.K.shape
    k = c.K.double().view(B, Hkv, -1, 64, d) * c.K_scale.double()[..., None, None]
    v = (c.V.double() * c.V_scale.double()[..., None, None]).transpose(3, 4)
    return k.reshape(B, Hkv, cap, d), v.reshape(B, Hkv, cap, d)


def _check_on_gpu(q, prefix, prefix_lengths, cache, lengths, counts, alpha, causal, O, lse, label=""):
    """As _check, for sizes that numpy is slow for: the same definition in 64 bits in torch, a sequence and key/value head at a time."""
    B, H, N, d = q.shape
    (Kp, Vp), (K, V) = _values_on_gpu(prefix), _values_on_gpu(cache)
    S, Hkv = B // Kp.shape[0], K.shape[1]
    group = H // Hkv
    for b in range(B) if B <= 24 else sorted({0, 1, S - 1, B - S, B - 2, B - 1, *range(0, B, 7)}):
        n, length, before = counts[b], lengths[b], prefix_lengths[b // S]
        assert (O[b, :, n:] == 0).all() and torch.isneginf(lse[b, :, n:]).all(), (label, b)
        for h in range(Hkv if n and before + length else 0):
            k, v = torch.cat((Kp[b // S, h, :before], K[b, h, :length])), torch.cat((Vp[b // S, h, :before], V[b, h, :length]))
            x = q[b, h * group:(h + 1) * group, :n].double().reshape(-1, d)
            s = alpha * (x @ k.t())
            own = length - n + 1 + torch.arange(n, device=DEV) if causal else torch.full((n,), length, device=DEV)
            hidden = torch.arange(before + length, device=DEV) >= before + own.clamp(0, length)[:, None]
            s = s.view(group, n, -1).masked_fill(hidden, -float("inf")).view(group * n, -1)
            l, p = torch.logsumexp(s, 1), torch.softmax(s, 1)
            e = 2 * (d + 4) * 2.0 ** -24 * alpha * (x.abs() @ k.abs().t()).amax(1) + 2.0 ** -22 * (alpha * (x @ k.t())).abs().amax(1) + 2.0 ** -16
            rows = slice(h * group, (h + 1) * group)
            off = ((lse[b, rows, :n].double().reshape(-1) - l).abs() - e).max().item()
            assert off <= 0, (label, "LSE", b, h, off)
            o = p @ v
            tol = 2.0 ** -8 * o.abs() + (2.0 ** -8 + e[:, None]) * 1.01 * (p @ v.abs() + o.abs())
            off = ((O[b, rows, :n].double().reshape(-1, d) - o).abs() - tol).max().item()
            assert off <= 0, (label, "O", b, h, off)


def _fill_on_gpu(seed, B, Hkv, cap, d, lengths):
    g = torch.Generator(device=DEV).manual_seed(seed)
    c, n = _garbage(B, Hkv, cap, d), max(lengths)
    k, v = (torch.randn((B, Hkv, n, d), generator=g, device=DEV) * torch.exp2(torch.randint(-2, 3, (B, Hkv, n, 1), generator=g, device=DEV).float()) for _ in range(2))
    binding.attn_cache_append(c, (0.5 * k).bfloat16(), v.bfloat16(), _i32(lengths), _i32(lengths))
    return c


@pytest.mark.parametrize("d", DIMS)
@pytest.mark.parametrize("P,S,Hkv,group,N,pcap,cap", [
    (1, 3, 2, 2, 1, 8192, 128),             # up to 16 rows a prefix; own heads one to a work-group
    (2, 2, 5, 3, 1, 8192, 192),             # own heads four to a work-group, the last one alone
    (1, 40, 4, 1, 1, 9600, 64),             # up to 64 rows
    (1, 40, 3, 1, 1, 9600, 448),            # with own segments of a work-group each
    (2, 3, 3, 2, 2, 4096, 3200),            # and with long ones, shared out
    (1, 30, 2, 5, 1, 9600, 64),             # several tiles of 64
    (2, 64, 8, 4, 1, 10240, 128),           # of 128, own heads four to a work-group
    (2, 64, 8, 4, 1, 10240, 320),           # or one
    (1, 5, 2, 4, 7, 4096, 128),             # 28 rows of a sequence
    (1, 12, 8, 3, 16, 8192, 64),            # 48, and tiles of 128 of the prefix
    (2, 3, 1, 3, 45, 3200, 640),            # 135
    (1, 33, 4, 2, 1, 9600, 128),            # one query a sequence, of some that have ended
])
def test_prefixes_that_are_read_once(lib, d, P, S, Hkv, group, N, pcap, cap):
    """Every pair of forms of the two lists, with padded batches and without."""
    assert binding.cache_fwd_shared_workspace_bytes(P, S, group * Hkv, Hkv, N, d, pcap, cap) > 0
    prefix_lengths = [pcap - 5, pcap // 2 + 64][:P]
    lengths = [cap, N] + [min(cap, N + x) for x in _some(N + S, P * S - 2, 0, cap)]
    counts = [0, N] + _some(d + S, P * S - 2, 0, N)
    prefix, cache = _fill_on_gpu(S, P, Hkv, pcap, d, prefix_lengths), _fill_on_gpu(N, P * S, Hkv, cap, d, lengths)
    g = torch.Generator(device=DEV).manual_seed(d)
    q = torch.randn((P * S, group * Hkv, N, d), generator=g, device=DEV).bfloat16()
    for c, causal in ((None, True), (counts, True), (counts, False)):
        O, lse = binding.attn_cache_fwd_shared(q, prefix, _i32(prefix_lengths), cache, _i32(lengths), d ** -0.5, causal, None if c is None else _i32(c))
        _check_on_gpu(q, prefix, prefix_lengths, cache, lengths, [N] * (P * S) if c is None else c, d ** -0.5, causal, O, lse, f"{c is None} {causal}")
    # ends of lengths: an empty prefix, empty caches, nobody real
    zero = [0] * (P * S)
    for pl, l, c in ((([0] * P), lengths, counts), (prefix_lengths, zero, None), ([0] * P, zero, None), (prefix_lengths, lengths, zero)):
        O, lse = binding.attn_cache_fwd_shared(q, prefix, _i32(pl), cache, _i32(l), d ** -0.5, True, None if c is None else _i32(c))
        _check_on_gpu(q, prefix, pl, cache, l, [N] * (P * S) if c is None else c, d ** -0.5, True, O, lse, "ends")
        if not any(pl) and not any(l):
            assert (O == 0).all() and torch.isneginf(lse).all()
    # lengths and counts that no cache has: full, empty, all, none
    wild = [[2 ** 31 - 1, -7, cap, -2 ** 31][i % 4] for i in range(P * S)]
    full = _fill_on_gpu(3, P * S, Hkv, cap, d, [cap] * (P * S))
    O, lse = binding.attn_cache_fwd_shared(q, prefix, _i32([-1, 2 ** 31 - 1][:P]), full, _i32(wild), d ** -0.5, False, _i32([[N + 9, 2 ** 31 - 1, -1][i % 3] for i in range(P * S)]))
    if P == 1:
        _check_on_gpu(q, prefix, [0], full, [min(max(w, 0), cap) for w in wild], [[N, N, 0][i % 3] for i in range(P * S)], d ** -0.5, False, O, lse, "wild")


@pytest.mark.parametrize("d", (64, 128, 256))
@pytest.mark.parametrize("P,S,Hkv,group,N,pcap,cap", [
    (4, 2, 5, 3, 1, 8192, 192),             # own heads four to a work-group
    (4, 40, 3, 1, 1, 4096, 448),            # segments of a work-group each
    (4, 3, 3, 2, 2, 4096, 3200),            # shared out
    (4, 12, 8, 3, 16, 8192, 64),            # 48 rows of a sequence
    (4, 3, 1, 3, 45, 3200, 640),            # 135
])
def test_lengths_that_no_prefix_has(lib, d, P, S, Hkv, group, N, pcap, cap):
    """Lengths beyond a prefix's cache are the cache's, negative ones none, for prefixes that are read once."""
    assert binding.cache_fwd_shared_workspace_bytes(P, S, group * Hkv, Hkv, N, d, pcap, cap) > 0
    prefix, cache = _fill_on_gpu(S, P, Hkv, pcap, d, [pcap] * P), _fill_on_gpu(N, P * S, Hkv, cap, d, [cap] * (P * S))
    q = torch.randn((P * S, group * Hkv, N, d), generator=torch.Generator(device=DEV).manual_seed(d), device=DEV).bfloat16()
    wild = [(2 ** 31 - 1, -7, cap, cap + 1, -2 ** 31)[i % 5] for i in range(P * S)]
    counts = [(N + 9, 2 ** 31 - 1, -1, N)[i % 4] for i in range(P * S)]
    (Kp, Vp), (K, V) = _values_on_gpu(prefix), _values_on_gpu(cache)
    alpha = d ** -0.5
    for prefix_lengths in ([2 ** 31 - 1, -1, pcap + 1, pcap - 70], [-2 ** 31, pcap + 64, 0, 2 ** 31 - 1]):
        for c, causal in ((None, False), (counts, False), (counts, True)):
            O, lse = binding.attn_cache_fwd_shared(q, prefix, _i32(prefix_lengths), cache, _i32(wild), alpha, causal, None if c is None else _i32(c))
            for b in range(P * S) if P * S <= 24 else (0, 1, 2, 3, 4, S, S + 1, 2 * S - 1, 3 * S, P * S - 1):
                n = min(max(c[b], 0), N) if c else N
                before, own = min(max(prefix_lengths[b // S], 0), pcap), min(max(wild[b], 0), cap)
                # query i sees positions up to length - n + i, whatever the length, of those that the cache has
                seen = torch.tensor([min(own, max(0, wild[b] - n + i + 1)) if causal else own for i in range(n)], device=DEV)
                for h in range(Hkv):
                    rows = slice(h * group, (h + 1) * group)
                    assert (O[b, rows, n:] == 0).all() and torch.isneginf(lse[b, rows, n:]).all(), (b, h)
                    none = (before + seen == 0).expand(group, n) if n else seen.expand(group, 0) > 0
                    o_got, l_got = O[b, rows, :n].double(), lse[b, rows, :n].double()
                    assert (o_got[none] == 0).all() and torch.isneginf(l_got[none]).all(), (b, h)
                    if none.all():
                        continue
                    k, v = torch.cat((Kp[b // S, h, :before], K[b, h, :own])), torch.cat((Vp[b // S, h, :before], V[b, h, :own]))
                    x = q[b, rows, :n].double().reshape(-1, d)
                    s = alpha * (x @ k.t())
                    e = 2 * (d + 4) * 2.0 ** -24 * alpha * (x.abs() @ k.abs().t()).amax(1) + 2.0 ** -22 * s.abs().amax(1) + 2.0 ** -16
                    s = s.view(group, n, -1).masked_fill(torch.arange(before + own, device=DEV) >= before + seen[:, None], -float("inf")).view(group * n, -1)
                    l, p = torch.logsumexp(s, 1), torch.softmax(s, 1)
                    real = ~none.reshape(-1)
                    assert ((l_got.reshape(-1) - l).abs() <= e)[real].all(), (b, h, prefix_lengths, causal)
                    o = p @ v
                    tol = 2.0 ** -8 * o.abs() + (2.0 ** -8 + e[:, None]) * 1.01 * (p @ v.abs() + o.abs())
                    assert ((o_got.reshape(-1, d) - o).abs() <= tol)[real].all(), (b, h, prefix_lengths, causal)


@pytest.mark.parametrize("P,S,group,Hkv,N,d,pcap", [(16, 1, 4, 2, 1, 128, 32768), (6, 2, 1, 3, 1, 64, 65536), (5, 1, 2, 2, 9, 96, 16384), (9, 1, 3, 1, 30, 32, 32768)])
def test_one_long_prefix_among_short_ones(lib, P, S, group, Hkv, N, d, pcap):
    """Hardly any sequence shares its prefix, and one prefix is long: it is read in parts."""
    assert binding.cache_fwd_shared_workspace_bytes(P, S, group * Hkv, Hkv, N, d, pcap, 128) > 0
    prefix_lengths = _some(P, P, 1, 300)
    prefix_lengths[P // 2] = pcap - 3
    lengths = [min(128, N + x) for x in _some(N, P * S, 0, 128)]
    prefix, cache = _fill_on_gpu(S, P, Hkv, pcap, d, prefix_lengths), _fill_on_gpu(N, P * S, Hkv, 128, d, lengths)
    q = torch.randn((P * S, group * Hkv, N, d), generator=torch.Generator(device=DEV).manual_seed(d), device=DEV).bfloat16()
    for counts in (None, [N - i % (N + 1) for i in range(P * S)]):
        O, lse = binding.attn_cache_fwd_shared(q, prefix, _i32(prefix_lengths), cache, _i32(lengths), d ** -0.5, True, None if counts is None else _i32(counts))
        _check_on_gpu(q, prefix, prefix_lengths, cache, lengths, [N] * (P * S) if counts is None else counts, d ** -0.5, True, O, lse, f"{counts is None}")


@pytest.mark.parametrize("N", (1, 7, 30))
def test_lengths_at_their_ends(lib, N):
    """Empty prefixes, empty caches, queries without tokens of their own, padded sequences, all together; and lengths that no cache has."""
    d, Hkv, group, pcap, cap = 64, 2, 2, 128, 64
    prefix_lengths = [0, 128, 64]
    lengths = [0, 64, N, 0, 1, 64, 0, 30, 64]
    counts = [0, N, N, N, N, 0, N, N, 1]
    q, prefix, cache = _problem(N, 3, 3, group, Hkv, N, d, pcap, prefix_lengths, cap, lengths)
    _run(q, prefix, prefix_lengths, cache, lengths, counts)
    _run(q, prefix, prefix_lengths, cache, lengths, counts, causal=False)
    _run(q, prefix, prefix_lengths, cache, lengths)
    # beyond the caches: as full ones, or none; what is past a cache's end does not exist
    g = _gen(4)
    prefix, cache = _filled(g, 3, Hkv, pcap, d, [pcap] * 3), _filled(g, 9, Hkv, cap, d, [cap] * 9)
    wild = [2 ** 31 - 1, -5, -2 ** 31, cap + 40, cap, 2 ** 31 - 1, 10, 1, 0]
    O, lse = binding.attn_cache_fwd_shared(q, prefix, _i32([2 ** 31 - 1, -1, -2 ** 31]), cache, _i32(wild), 0.125, causal=False, counts=_i32([N] * 8 + [-3]))
    _check(q, prefix, [pcap, 0, 0], cache, [min(max(w, 0), cap) for w in wild], [N] * 8 + [0], 0.125, False, O, lse)


def test_nan_and_infinities_stay_where_they_are_seen(lib):
    """NaN in what a masked place holds, behind the ends of prefix and cache, and in a later query's token, reaches nobody who does not see it."""
    d, Hkv, N = 64, 1, 4
    for S, group, pcap in ((3, 2, 128), (20, 4, 128), (20, 4, 8192)):
        prefix_lengths, lengths = [pcap - 28], [5 + s for s in range(S)]
        q, prefix, cache = _problem(S, 1, S, group, Hkv, N, d, pcap, prefix_lengths, 64, lengths)
        want = binding.attn_cache_fwd_shared(q, prefix, _i32(prefix_lengths), cache, _i32(lengths), 0.125)
        for c, n in ((prefix, prefix_lengths), (cache, lengths)):
            for b, l in enumerate(n):
                c.K[b].view(torch.uint8)[:, l:] = 0x7f
                c.V[b].view(torch.uint8)[:, l // 64, :, l % 64:] = 0xff
                c.V_scale[b, :, l // 64].neg_()                # a NaN in the block
        got = binding.attn_cache_fwd_shared(q, prefix, _i32(prefix_lengths), cache, _i32(lengths), 0.125)
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        # the last token's V: NaN for the last query alone
        for b, l in enumerate(lengths):
            cache.V[b].view(torch.uint8)[:, 0, 7, l - 1] = 0x7f
        O, lse = binding.attn_cache_fwd_shared(q, prefix, _i32(prefix_lengths), cache, _i32(lengths), 0.125)
        assert torch.isnan(O[:, :, -1, 7]).all() and not torch.isnan(O[:, :, :-1]).any() and torch.equal(lse, want[1])
        # a NaN in the prefix: for all
        prefix.V.view(torch.uint8)[0, :, 0, 3, 10] = 0x7f
        prefix.V_scale[0, :, 0] = -prefix.V_scale[0, :, 0].abs()
        O, _ = binding.attn_cache_fwd_shared(q, prefix, _i32(prefix_lengths), cache, _i32(lengths), 0.125)
        assert torch.isnan(O[..., 3]).all() and not torch.isnan(O[..., 4]).any()


@pytest.mark.parametrize("pcap", (1600, 6400))              # read for each sequence; read once
def test_strides_outputs_workspaces_and_streams(lib, pcap):
    P, S, Hkv, group, N, d, cap = 2, 9, 2, 4, 3, 96, 192
    prefix_lengths, lengths = [pcap, 700], _some(1, P * S, N, cap)
    q, prefix, cache = _problem(5, P, S, group, Hkv, N, d, pcap, prefix_lengths, cap, lengths)
    H = group * Hkv
    want = _run(q, prefix, prefix_lengths, cache, lengths)
    qkv = torch.full((P * S, N, H + 4, d), float("nan"), dtype=torch.bfloat16, device=DEV)
    qkv[:, :, :H] = q.permute(0, 2, 1, 3)
    out = torch.zeros((P * S, N, H, d), dtype=torch.bfloat16, device=DEV)
    args = (qkv[:, :, :H].permute(0, 2, 1, 3), prefix, _i32(prefix_lengths), cache, _i32(lengths), d ** -0.5)
    O, lse = binding.attn_cache_fwd_shared(*args, O=out.permute(0, 2, 1, 3))
    assert torch.equal(out.permute(0, 2, 1, 3), want[0]) and torch.equal(lse, want[1])
    # a workspace of the caller's with whatever in it, a stream of its own, several times the same bits
    need = binding.cache_fwd_shared_workspace_bytes(P, S, H, Hkv, N, d, pcap, cap)
    for fill in (0, 0xff):
        ws = torch.full((max(need, 16),), fill, dtype=torch.uint8, device=DEV)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        O, lse = binding.attn_cache_fwd_shared(*args, workspace=ws, stream=side)
        side.synchronize()
        assert torch.equal(O, want[0]) and torch.equal(lse, want[1])
    # one query for all heads: an expanded head dimension
    one = q[:, :1].expand(-1, H, -1, -1)
    a = binding.attn_cache_fwd_shared(one, *args[1:])
    b = binding.attn_cache_fwd_shared(one.contiguous(), *args[1:])
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_a_prefix_beyond_32_bits(lib):
    """A second head that begins 2^32 bytes behind the first, and tokens in the last blocks of a cache."""
    d, cap, length = 128, 1 << 25, 130
    small, big = _fill_on_gpu(1, 1, 2, 192, d, [length]), binding.cache_empty(1, 2, cap, d, DEV)
    for t, u in zip(_blocks(small), _blocks(big)):
        u[:, :, :3] = t
    cache = _fill_on_gpu(2, 5, 2, 64, d, [9, 8, 7, 64, 1])
    q = torch.randn((5, 6, 1, d), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV).bfloat16()
    args = (cache, _i32([9, 8, 7, 64, 1]), d ** -0.5)
    O, lse = binding.attn_cache_fwd_shared(q, big, _i32([length]), *args)
    _check_on_gpu(q, small, [length], cache, [9, 8, 7, 64, 1], [1] * 5, d ** -0.5, True, O, lse)
    # all of it: weights of one huge key's block near the end decide
    for t in big[:2]:
        t.view(torch.uint8).zero_()
    big.K_scale.fill_(1.0), big.V_scale.fill_(1.0)
    big.K.view(torch.uint8)[0, :, cap - 70] = 0x7e          # 448
    big.V.view(torch.uint8)[0, :, (cap - 70) // 64, :, (cap - 70) % 64] = 0x38          # 1
    O, lse = binding.attn_cache_fwd_shared(q.abs(), big, _i32([cap]), *args)
    assert (O == 1).all()


def test_caches_without_heads_are_refused(lib):
    c = binding.cache_empty(2, 0, 64, 64, DEV)
    for call in (lambda: binding.attn_cache_fork(c, _i32([0]), _i32([1, 1])), lambda: binding.attn_cache_reorder(c, _i32([[1, 0]]), _i32([1, 1]))):
        with pytest.raises(ValueError):
            call()


def test_two_calls_at_once(lib):
    """On two streams, with workspaces of their own, and replays of two graphs in turn: each call's results are its own."""
    calls = []
    for seed, (P, S, N) in enumerate(((2, 24, 1), (1, 6, 9))):
        prefix, cache = _fill_on_gpu(seed, P, 4, 8192, 64, [8000 - seed] * P), _fill_on_gpu(seed + 5, P * S, 4, 128, 64, [100 + seed] * (P * S))
        q = torch.randn((P * S, 16, N, 64), generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).bfloat16()
        assert binding.cache_fwd_shared_workspace_bytes(P, S, 16, 4, N, 64, 8192, 128) > 0
        calls.append((q, prefix, _i32([8000 - seed] * P), cache, _i32([100 + seed] * (P * S)), 0.125))
    want = [binding.attn_cache_fwd_shared(*c) for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(20):
        got = []
        for c, st in zip(calls, streams):
            with torch.cuda.stream(st):
                got.append(binding.attn_cache_fwd_shared(*c))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(want, got) for a, b in zip(x, y))
    graphs, outs = [], []
    for c in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(binding.attn_cache_fwd_shared(*c))
    for _ in range(4):
        for g, out, w, c in zip(graphs, outs, want, calls):
            out[0].zero_(), out[1].zero_()
            g.replay()
            again = binding.attn_cache_fwd_shared(*c)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(w, out)) and all(torch.equal(a, b) for a, b in zip(w, again))


def test_sharing_is_what_copies_would_give(lib):
    """Against attn_cache_fwd over caches that hold prefix and own tokens (the prefix whole blocks, so that no code differs)."""
    P, S, Hkv, group, d = 2, 6, 2, 4, 128
    g = _gen(9)
    prefix_lengths, lengths = [1024, 576], _some(2, P * S, 1, 128)
    prefix, cache = _filled(g, P, Hkv, 1024, d, prefix_lengths), _filled(g, P * S, Hkv, 128, d, lengths)
    both = binding.cache_empty(P * S, Hkv, 1152, d, DEV)
    binding.attn_cache_fork(prefix, _i32([b // S for b in range(P * S)]), _i32(prefix_lengths), out=both)
    for b in range(P * S):
        first = prefix_lengths[b // S] // 64
        both.K.view(torch.uint8)[b, :, first * 64:first * 64 + 128] = cache.K.view(torch.uint8)[b]
        both.V.view(torch.uint8)[b, :, first:first + 2] = cache.V.view(torch.uint8)[b]
        both.K_scale[b, :, first:first + 2], both.V_scale[b, :, first:first + 2] = cache.K_scale[b], cache.V_scale[b]
    for N in (1, 5):
        q = _bf16(g, P * S, Hkv * group, N, d).to(DEV)
        _run(q, prefix, prefix_lengths, cache, lengths)
        O, lse = binding.attn_cache_fwd_shared(q, prefix, _i32(prefix_lengths), cache, _i32(lengths), d ** -0.5, causal=False)
        O2, lse2 = binding.attn_cache_fwd(q, both, _i32([prefix_lengths[b // S] + l for b, l in enumerate(lengths)]), d ** -0.5, causal=False)
        assert (lse - lse2).abs().max() < 2.0 ** -15 and (O.float() - O2.float()).abs().max() < 2.0 ** -6 * O2.float().abs().max()


# ---- copies

def _bytes(cache):
    return [t.clone().view(torch.uint8) for t in cache]


def _blocks(cache):
    """A cache's codes and scales as [B,Hkv,nb,bytes of a block] tensors."""
    B, Hkv, cap, d = cache.K.shape
    nb = cap // 64
    return [cache.K.view(torch.uint8).view(B, Hkv, nb, 64 * d), cache.V.view(torch.uint8).view(B, Hkv, nb, 64 * d),
            cache.K_scale.view(torch.uint8).view(B, Hkv, nb, 4), cache.V_scale.view(torch.uint8).view(B, Hkv, nb, 4)]


def _noise(g, B, Hkv, cap, d):
    """Any bytes, scales too: copies do not interpret them."""
    c = binding.cache_empty(B, Hkv, cap, d, DEV)
    for t in c:
        t.view(torch.uint8).copy_(torch.randint(0, 256, t.view(torch.uint8).shape, generator=g, dtype=torch.uint8))
    return c


def _expect(before, source, pairs, lengths):
    """`before` (blocks) with the first blocks of sequences (from, to) of `source`, as many as lengths[from] tokens have."""
    want = [t.clone() for t in before]
    for a, b in pairs:
        n = -(-lengths[a] // 64)
        for w, s in zip(want, source):
            w[b, :, :n] = s[a, :, :n]
    return want


@pytest.mark.parametrize("d", DIMS)
def test_fork(lib, d):
    for B, sources, cap, cap_out, lengths in ((1, [0] * 5, 320, 448, [257]), (4, [3, 0, 0, 2, 1], 192, 128, [192, 64, 0, 65]), (3, [2], 64, 64, [1, 1, 63]),
                                              (3, [-1, 5, 1, 3, -2 ** 31, 2 ** 31 - 1], 128, 192, [128, 100, 7]), (2, [1, 0], 128, 192, [-4, 2 ** 31 - 1])):
        g = _gen(d + cap)
        c, out = _noise(g, B, 3, cap, d), _noise(g, len(sources), 3, cap_out, d)
        left = [min(max(lengths[s], 0), cap, cap_out) if 0 <= s < B else 0 for s in sources]
        want = [t.clone() for t in _blocks(out)]
        for i, s in enumerate(sources):
            n = -(-left[i] // 64)
            for w, x in zip(want, _blocks(c)):
                if n:
                    w[i, :, :n] = x[s, :, :n]
        before = _bytes(c)
        got, lengths_out = binding.attn_cache_fork(c, _i32(sources), _i32(lengths), out=out)
        assert got is out and lengths_out.tolist() == left
        assert all(torch.equal(a, b) for a, b in zip(want, _blocks(out))) and all(torch.equal(a, b) for a, b in zip(before, _bytes(c)))
    new, lengths_out = binding.attn_cache_fork(c, _i32([1]), _i32([128, 77]))
    assert new.K.shape == (1, 3, 128, d) and lengths_out.tolist() == [77] and torch.equal(_blocks(new)[0][0, :, :2], _blocks(c)[0][1, :, :2])
    none, lengths_out = binding.attn_cache_fork(c, _i32([]), _i32([128, 77]))
    assert none.K.shape[0] == 0 and lengths_out.shape == (0,)


@pytest.mark.parametrize("d", DIMS)
@pytest.mark.parametrize("S", (1, 2, 3, 4, 5, 8, 13, 16, 30, 32, 33, 64))
def test_reorder(lib, d, S):
    rng = np.random.default_rng(S + d)
    for P, cap in ((1, 192), (3, 64)):
        kinds = [np.roll(np.arange(S), 1), np.arange(S)[::-1], rng.integers(0, S, S), np.zeros(S, int), rng.permutation(S), rng.integers(-2, S + 2, S)]
        for parents in (kinds[:3], kinds[3:]):
            parents = np.array(parents)[:P] if P > 1 else np.array(parents)[S % 3:][:1]
            g = _gen(S)
            c = _noise(g, P * S, 2, cap, d)
            lengths = [int(x) for x in rng.choice([0, 1, 63, 64, 65, cap - 1, cap, cap + 9, -3], P * S)]
            at = [p * S + s for p in range(P) for s in oracle.origin(parents[p].tolist())]
            source = [t.clone() for t in _blocks(c)]
            want = [t.clone() for t in source]
            for i, s in enumerate(at):
                n = -(-min(max(lengths[s], 0), cap) // 64)
                for w, x in zip(want, source):
                    w[i, :, :n] = x[s, :, :n]
            out = binding.attn_cache_reorder(c, torch.tensor(parents, dtype=torch.int32, device=DEV), _i32(lengths))
            assert out.tolist() == [lengths[s] for s in at]
            assert all(torch.equal(a, b) for a, b in zip(want, _blocks(c))), (parents, lengths)


def test_copies_of_long_sequences(lib):
    """More than one round of a work-group, on a stream of its own; sequences that begin beyond 2^32 bytes."""
    g = _gen(1)
    d, Hkv, cap = 32, 1, 64 * 1200
    c = binding.cache_empty(4, Hkv, cap, d, DEV)
    lengths = [cap, 70000, 65, cap - 1]
    rnd = torch.Generator(device=DEV).manual_seed(1)
    for t in c:
        t.view(torch.uint8).copy_(torch.randint(0, 256, t.view(torch.uint8).shape, generator=rnd, dtype=torch.uint8, device=DEV))
    before = [t.clone() for t in _blocks(c)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, _ = binding.attn_cache_fork(c, _i32([3, 0]), _i32(lengths), stream=side)
    side.synchronize()
    for x, y in zip(_blocks(out), before):
        assert torch.equal(x[0], y[3]) and torch.equal(x[1], y[0])
    binding.attn_cache_reorder(c, _i32([[1, 2, 3, 0]]), _i32(lengths))
    for x, y in zip(_blocks(c), before):
        n = [-(-lengths[s] // 64) for s in (1, 2, 3, 0)]
        assert torch.equal(x[0, :, :n[0]], y[1, :, :n[0]]) and torch.equal(x[0, :, n[0]:], y[0, :, n[0]:])
        assert torch.equal(x[1, :, :2], y[2, :, :2]) and torch.equal(x[1, :, 2:], y[1, :, 2:])
        assert torch.equal(x[2], y[3]) and torch.equal(x[3], y[0])
    del c, out, before
    big = binding.cache_empty(5, 1, 1 << 23, 256, DEV)      # 2 GiB a sequence, keys and values each
    for t in big[:2]:
        t.view(torch.uint8)[2:].zero_()
    mark = torch.arange(64 * 256, device=DEV).remainder(251).to(torch.uint8).view(64, 256)
    big.K.view(torch.uint8)[4, 0, -64:], big.V.view(torch.uint8)[4, 0, -1] = mark, mark.t()
    big.K_scale.fill_(1.0), big.V_scale.fill_(2.0)
    big.K_scale[4, 0, -1] = 8.0
    binding.attn_cache_reorder(big, _i32([[0, 1, 4, 3, 4]]), _i32([1 << 23] * 5))
    assert torch.equal(big.K.view(torch.uint8)[2, 0, -64:], mark) and torch.equal(big.V.view(torch.uint8)[2, 0, -1], mark.t()) and big.K_scale[2, 0, -1] == 8.0
    assert (big.K.view(torch.uint8)[3] == 0).all()
    small = binding.cache_empty(1, 1, 1 << 23, 256, DEV)
    binding.attn_cache_fork(big, _i32([4]), _i32([1 << 23] * 5), out=small)
    assert torch.equal(small.K.view(torch.uint8)[0, 0, -64:], mark) and torch.equal(small.V.view(torch.uint8)[0, 0, -1], mark.t())


# ---- the choice among beams

def _select(logits, scores, n, finished=None, end=None, label=""):
    got = binding.attn_beam_select(logits, scores, n, finished, end)
    x, s = logits.double().cpu().numpy(), scores.double().cpu().numpy()
    f = None if finished is None else finished.cpu().numpy()
    for b in range(logits.shape[0]):
        p, t, sums, e = oracle.select(x[b], s[b], n, None if f is None else f[b], -1 if end is None else end)
        assert got[0][b].tolist() == p and got[1][b].tolist() == t, (label, b, got[0][b].tolist(), p, got[1][b].tolist(), t)
        assert got[3][b].tolist() == e, (label, b)
        have, sums = got[2][b].double().cpu().numpy(), np.array(sums)
        none = np.isneginf(sums)
        assert np.array_equal(none, np.isneginf(have))
        have, sums = have[~none], sums[~none]
        assert (np.abs(have - sums) <= 40 * 2.0 ** -23 + 2.0 ** -23 * np.abs(sums)).all(), (label, b, have - sums)
    return got


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("V", (1, 2, 63, 500, 2047, 2048, 2049, 8185, 50257))
def test_select(lib, dtype, V):
    for B, beams, n in ((1, 1, 1), (2, 3, 6), (3, 4, 4), (1, 64, 128), (5, 7, 33)):
        g = _gen(V + n)
        logits = (3.0 * torch.randn((B, beams, V), generator=g)).to(dtype).to(DEV)
        scores = (-10 * torch.rand((B, beams), generator=g)).to(DEV)
        _select(logits, scores, n, label=f"{B} {beams} {n}")
        if V > 2:
            logits[torch.rand(logits.shape, generator=g) < 0.3] = -float("inf")
            _select(logits, scores, n, (torch.rand((B, beams), generator=g) < 0.4).to(DEV), V // 2, label=f"{B} {beams} {n} ended")


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_select_from_long_rows(lib, dtype):
    """More than one chunk a row in both sizes of chunks."""
    for B, beams, V, n in ((2, 2, 200000, 4), (4, 8, 40000, 16), (1, 3, 300001, 100), (30, 2, 30011, 1)):
        g = torch.Generator(device=DEV).manual_seed(V)
        logits = (2.5 * torch.randn((B, beams, V), generator=g, device=DEV)).to(dtype)
        _select(logits, -5 * torch.rand((B, beams), generator=g, device=DEV), n, label=f"{V}")


def test_select_ties(lib):
    """All equal; few values; -0 and 0; the last chunk's alone; equal beams."""
    for V, n in ((5000, 128), (70, 128), (20001, 40)):
        x = torch.zeros((3, 2, V), device=DEV)
        x[1] = -0.0
        x[1, :, ::3] = 0.0
        x[2] = (torch.arange(V, device=DEV) % 5).float()
        _select(x, torch.tensor([[-1.0, -1.0], [-2.0, -1.0], [0.0, 0.0]], device=DEV), n, label=f"{V}")
        x = torch.full((1, 3, V), -30.0, device=DEV)
        x[:, :, -7:] = 4.0
        _select(x, torch.tensor([[0.0, -float("inf"), 0.0]], device=DEV), min(n, 20), label=f"{V} last")
    x = (2 * torch.randn((1, 1, 3000), generator=_gen(3))).to(DEV).expand(2, 4, 3000)      # an expanded tensor: all beams the same
    _select(x, torch.tensor([[0.0, 0.0, 0.0, 0.0], [-float("inf"), 0.0, -float("inf"), 0.0]], device=DEV), 9, label="equal beams")


def test_select_without_candidates(lib):
    inf, nan = float("inf"), float("nan")
    g = _gen(8)
    x = torch.randn((2, 7, 3000), generator=g).to(DEV)
    x[0, 1, 2999], x[0, 2, 5], x[0, 3], x[1, 4, :2998] = nan, inf, -inf, -inf
    scores = torch.tensor([[0.0, 5.0, 5.0, 5.0, nan, inf, -inf], [-inf, nan, -inf, inf, 3.0, -inf, -inf]], device=DEV)
    _select(x, scores, 10)
    ended = torch.tensor([[False, True, True, False, True, True, False], [True, True, False, False, False, True, False]], device=DEV)
    _select(x, scores, 10, ended, 2999)
    _select(torch.full((1, 2, 100), -inf, device=DEV), torch.zeros((1, 2), device=DEV), 3)
    _select(torch.full((1, 2, 100), 3e38, device=DEV), torch.tensor([[3e38, -3e38]], device=DEV), 3)
    # numbers at the ends of their range
    x = torch.tensor([3.4e38, -3.4e38, 1e-45, -1e-45, 0.0, 1.0], device=DEV).repeat(50).view(1, 3, 100)
    _select(x, torch.zeros((1, 3), device=DEV), 30)
    got = binding.attn_beam_select(x, torch.zeros((1, 3), device=DEV), 0)
    assert all(t.shape == (1, 0) for t in got)


def test_select_strides_and_alignment(lib):
    """Rows that begin at any element, of padded vocabularies, views and slices; nothing around them is looked at."""
    g = _gen(11)
    for dtype in (torch.float32, torch.bfloat16):
        whole = torch.full((3, 6, 4111), float("nan"), dtype=dtype, device=DEV)
        for first in range(9):
            x = whole[:, 1:5, first:first + 4099]
            x.copy_((3 * torch.randn(x.shape, generator=g)).to(dtype))
            _select(x, torch.zeros((3, 4), device=DEV), 8, label=f"{first}")
            _select(x.transpose(0, 1), torch.zeros((4, 3), device=DEV), 8, label=f"{first} transposed")
            x.fill_(float("nan"))


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_select_does_not_depend_on_where_rows_lie(lib, dtype):
    """Equal beams of ordinary logits in rows that begin anywhere between two 16-byte boundaries: their sums are the same bits, so the lower beam goes first, and the
    same values at another address or distance give the same bits."""
    size = dtype.itemsize
    for V, beams, n in ((4099, 8, 5), (4099, 8, 60), (50257, 8, 12), (33001, 5, 128), (200003, 8, 6)):
        for seed in range(3):
            row = 2.5 * torch.randn(V, generator=_gen(V + seed)).to(DEV)
            x = row.to(dtype).repeat(1, beams, 1)
            assert len({x[0, k].data_ptr() % 16 for k in range(beams)}) == min(beams, 16 // size)
            scores = torch.full((1, beams), -3.7, device=DEV)
            want = _select(x, scores, n, label=f"{V} {n} {seed}")
            for first, pitch in ((0, -(-V // 64) * 64), (1, V), (3, V + 2), (7, V + 13)):
                room = torch.full((first + beams * pitch,), float("nan"), dtype=dtype, device=DEV)
                y = room[first:].view(1, beams, pitch)[:, :, :V]
                y.copy_(x)
                got = binding.attn_beam_select(y, scores, n)
                assert all(torch.equal(a, b) for a, b in zip(want, got)), (V, n, seed, first, pitch)


def test_select_on_a_stream_with_a_workspace(lib):
    g = _gen(12)
    x, s = torch.randn((4, 4, 9000), generator=g).to(DEV), torch.zeros((4, 4), device=DEV)
    want = _select(x, s, 8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = torch.full((binding.beam_select_workspace_bytes(4, 4, 9000, 8),), 0xff, dtype=torch.uint8, device=DEV)
    got = binding.attn_beam_select(x, s, 8, workspace=ws, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


# ---- together

def test_beam_search(lib):
    """Three prompts, four beams: append, attend, choose, reorder, for 70 tokens (into the second block), against the same search with a cache of
    its own for every beam, prompt and all, gathered by torch; then the ended prompt's beams leave the batch."""
    P, S, Hkv, group, d, V, steps = 3, 4, 2, 2, 64, 300, 70
    g = _gen(21)
    H, B = Hkv * group, P * S
    prompt = [130, 64, 200]
    embed_q, embed_k, embed_v = (_bf16(g, V, h, d).to(DEV) for h in (H, Hkv, Hkv))
    head = (0.3 * torch.randn((H * d, V), generator=g)).to(DEV)
    prefix = _filled(g, P, Hkv, 256, d, prompt)
    own, whole = _garbage(B, Hkv, 128, d), binding.cache_empty(B, Hkv, 384, d, DEV)
    whole, at = binding.attn_cache_fork(prefix, _i32([b // S for b in range(B)]), _i32(prompt), out=whole)
    prefix_lengths, lengths = _i32(prompt), _i32([0] * B)
    scores = torch.tensor([[0.0] + [-float("inf")] * (S - 1)] * P, device=DEV)
    tokens, ended = torch.full((P, S), 7, dtype=torch.int32, device=DEV), torch.zeros((P, S), dtype=torch.bool, device=DEV)
    for step in range(steps):
        lengths, at = lengths + 1, at + 1
        t = tokens.view(-1).long()
        q, k, v = embed_q[t][:, :, None], embed_k[t][:, :, None], embed_v[t][:, :, None]
        binding.attn_cache_append(own, k, v, lengths)
        binding.attn_cache_append(whole, k, v, at)
        O, lse = binding.attn_cache_fwd_shared(q, prefix, prefix_lengths, own, lengths, 0.3)
        O2, lse2 = binding.attn_cache_fwd(q, whole, at, 0.3)
        # the two hold the same tokens in blocks that begin elsewhere: their codes differ where scales do, by half a step of E4M3 of the largest
        assert (lse - lse2).abs().max() < 0.05
        logits = (O.float().view(P, S, -1) @ head).contiguous()
        parents, tokens, scores, ended = _select(logits, scores, S, ended, 3, label=f"step {step}")
        origin = (parents + S * torch.arange(P, device=DEV)[:, None]).view(-1).long()
        want = [x[origin] for x in _blocks(own)]
        lengths2 = binding.attn_cache_reorder(own, parents, lengths)
        n = -(-(step + 1) // 64)
        assert torch.equal(lengths2, lengths[origin]) and all(torch.equal(x[:, :, :n], y[:, :, :n]) for x, y in zip(want, _blocks(own)))
        lengths = lengths2
        for x in _blocks(whole):
            x.copy_(x[origin])
        at = at[origin]
    keep = _i32([b for b in range(B) if b // S != 1])
    left, lengths_left = binding.attn_cache_fork(own, keep, lengths)
    assert lengths_left.tolist() == [steps] * (B - S)
    assert all(torch.equal(x[:, :, :2], y[keep.long()][:, :, :2]) for x, y in zip(_blocks(left), _blocks(own)))


@pytest.mark.parametrize("pcap", (2048, 8192))
def test_a_captured_step(lib, pcap):
    """Append, attend, choose and reorder in one graph, replayed between eager steps of another search that uses the same kernels."""
    P, S, Hkv, group, d, V = 2, 4, 2, 4, 64, 3000
    g = _gen(31)
    H, B = Hkv * group, P * S
    prefix = _filled(g, P, Hkv, pcap, d, [pcap - 48, 1500])
    prefix_lengths = _i32([pcap - 48, 1500])
    head = (0.1 * torch.randn((H * d, V), generator=g)).to(DEV)
    embed = [_bf16(g, V, h, d).to(DEV) for h in (H, Hkv, Hkv)]

    class Search:
        def __init__(self):
            self.own = binding.cache_empty(B, Hkv, 128, d, DEV)
            for t in self.own:
                t.view(torch.uint8).zero_()
            self.lengths, self.tokens = _i32([0] * B), torch.arange(B, dtype=torch.int32, device=DEV).view(P, S)
            self.scores, self.ended = torch.zeros((P, S), device=DEV), torch.zeros((P, S), dtype=torch.bool, device=DEV)

        def step(self):
            self.lengths.add_(1)
            t = self.tokens.view(-1).long()
            q, k, v = (e[t][:, :, None] for e in embed)
            binding.attn_cache_append(self.own, k, v, self.lengths)
            O, _ = binding.attn_cache_fwd_shared(q, prefix, prefix_lengths, self.own, self.lengths, 0.2)
            parents, tokens, scores, ended = binding.attn_beam_select(torch.mm(O.float().view(B, -1), head).view(P, S, V), self.scores, S, self.ended, 5)
            self.lengths.copy_(binding.attn_cache_reorder(self.own, parents, self.lengths))
            self.tokens.copy_(tokens), self.scores.copy_(scores), self.ended.copy_(ended)

        def state(self):
            return [x.clone() for x in (self.lengths, self.tokens, self.scores, self.ended)] + [x[:, :, :1].clone() for x in _blocks(self.own)]

    eager, captured = Search(), Search()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        captured.step()                                    # (a step on the side, so that the library's first calls are not captured)
    torch.cuda.current_stream().wait_stream(side)
    eager.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.step()
    for i in range(6):
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager.state(), captured.state())), i
