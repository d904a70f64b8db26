"""The 8-bit cache (attn_cache_append, attn_cache_fwd, attn_cache_weights, attn_cache_evict) against the 64-bit oracle.

Codes, scales and kept positions have to be the oracle's.  Tolerances of what is computed in float32:
  scores   a product of d bf16 values summed in float32: within e = 2 (d + 4) 2^-24 alpha sum |q k| + 2^-22 |S| (the factor log2(e) and the
           subtraction of the maximum);
  LSE      e + 2^-16 (a hardware exponential, 2^-22, and a sum of at most 2^8 terms a lane after the other);
  O        probabilities off by 2^-8 (bf16) + e + 2^-16 each, so the quotient by that times (sum P |v| + |O|), and one bf16 rounding;
  weights  e + 2^-16 of the sum, which all terms share, + 2^-22 |LSE|."""
import numpy as np
import pytest
import torch

from oracle import cache as oracle
from oracle import positions
from paper_2510_04212_amd import autograd, binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DIMS = (32, 64, 96, 128, 256)


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _bf16(g, *shape, gain=1.0):
    return (gain * torch.randn(shape, generator=g)).to(torch.bfloat16)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _garbage(B, Hkv, cap, d):
    """A cache as an allocator may hand it over: NaN codes, NaN and infinite scales."""
    c = binding.cache_empty(B, Hkv, cap, d, DEV)
    c.K.view(torch.uint8).fill_(0x7f)
    c.V.view(torch.uint8).fill_(0xff)
    c.K_scale.fill_(float("nan"))
    c.V_scale.fill_(float("inf"))
    return c


def _values(c):
    """Codes as float64, V's blocks turned to rows, and the exponents: numpy [B,Hkv,cap,d] and [B,Hkv,nb], K and V."""
    B, Hkv, cap, d = c.K.shape
    k = c.K.double().cpu().numpy()
    v = c.V.double().cpu().transpose(3, 4).reshape(B, Hkv, cap, d).numpy()
    with np.errstate(divide="ignore", invalid="ignore"):
        e = [np.round(np.log2(np.abs(s.double().cpu().numpy()))) for s in (c.K_scale, c.V_scale)]
    return (k, v), e


class Pair:
    """The library's cache and the oracle's, filled alike."""

    def __init__(self, B, Hkv, cap, d):
        self.dev = _garbage(B, Hkv, cap, d)
        self.ref = [[oracle.Cache(cap, d) for _ in range(Hkv)] for _ in range(B)]
        self.lengths = [0] * B

    def append(self, k, v, counts=None):
        B, Hkv, N, d = k.shape
        n = [N] * B if counts is None else counts
        self.lengths = [l + c for l, c in zip(self.lengths, n)]
        binding.attn_cache_append(self.dev, k.to(DEV), v.to(DEV), _i32(self.lengths), None if counts is None else _i32(counts))
        for b in range(B):
            for h in range(Hkv):
                self.ref[b][h].append(self.lengths[b], k[b, h, :n[b]].double().numpy(), v[b, h, :n[b]].double().numpy())

    def check(self):
        values, exponents = _values(self.dev)
        for b, length in enumerate(self.lengths):
            blocks = -(-length // 64)
            for h, ref in enumerate(self.ref[b]):
                for w in range(2):
                    assert np.array_equal(exponents[w][b, h, :blocks], ref.exponents[w][:blocks]), (b, h, w)
                    assert np.array_equal(values[w][b, h, :length], ref.values[w][:length], equal_nan=True), (b, h, w)
                # the sign of V's scale: NaN in the block (or among tokens it held when they were appended)
                marked = (self.dev.V_scale[b, h, :blocks] < 0).cpu().numpy()
                nan = np.array([np.isnan(ref.values[1][64 * j:min(length, 64 * j + 64)]).any() for j in range(blocks)], dtype=bool)
                assert np.array_equal(marked, nan) and (self.dev.K_scale[b, h, :blocks] > 0).all()


# ---- append

@pytest.mark.parametrize("d", DIMS)
def test_append(lib, d):
    g = _gen(d)
    p = Pair(3, 2, 320, d)
    # blocks begun, filled and crossed; scales that grow (x1000), stay and would shrink; padded batches, a sequence without new tokens
    for N, counts, gain in ((1, None, 1.0), (1, None, 1000.0), (61, None, 1.0), (2, None, 3.0), (70, [70, 0, 33], 1e-3), (130, [1, 130, 64], 50.0), (1, None, 1e5),
                            (5, [0, 0, 0], 1.0)):
        p.append(_bf16(g, 3, 2, N, d, gain=gain), _bf16(g, 3, 2, N, d, gain=1.0 / gain), counts)
        p.check()
    # a sequence starts again in memory that held others: nothing of them is left
    p.lengths = [0, 0, 0]
    p.append(_bf16(g, 3, 2, 3, d, gain=1e-6), _bf16(g, 3, 2, 3, d, gain=1e-6))
    p.check()
    values, _ = _values(p.dev)
    assert all((v[:, :, 3:64] == 0).all() for v in values)


def test_append_takes_every_bf16_number(lib):
    """All 65536 bit patterns, 256 to a token: subnormals, the largest, infinities, NaN, with zeros (whole blocks of them) between."""
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(1, 1, 256, 256)
    x = torch.cat((x, torch.zeros(1, 1, 64, 256, dtype=torch.bfloat16), -x[:, :, :60]), 2)
    p = Pair(1, 1, 384, 256)
    p.append(x, x.flip(2))
    p.check()


def test_append_strides_streams_and_what_it_leaves_alone(lib):
    g = _gen(3)
    B, Hkv, N, d = 2, 3, 50, 96
    qkv = _bf16(g, B, N, 4 + 2 * Hkv, d).to(DEV)
    k, v = qkv[:, :, 4:4 + Hkv].permute(0, 2, 1, 3), qkv[:, :, 4 + Hkv:].permute(0, 2, 1, 3)
    lengths = _i32([90, 130])
    one, two = _garbage(B, Hkv, 256, d), _garbage(B, Hkv, 256, d)
    for c in (one, two):                                   # older tokens, and a scale for them
        c.K_scale.fill_(2.0 ** -6)
        c.V_scale.fill_(2.0 ** -6)
    binding.attn_cache_append(one, k, v, lengths)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    binding.attn_cache_append(two, k.contiguous(), v.contiguous(), lengths, stream=side)
    side.synchronize()
    for a, b in zip(one, two):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    # sequence 0: positions 40 .. 89; 1: 80 .. 129.  Blocks without a new token keep their bytes
    assert (one.K.view(torch.uint8)[0, :, 128:] == 0x7f).all() and (one.V.view(torch.uint8)[0, :, 2:] == 0xff).all()
    assert (one.K.view(torch.uint8)[1, :, :64] == 0x7f).all() and (one.K.view(torch.uint8)[1, :, 192:] == 0x7f).all()
    assert (one.K_scale[0, :, 2:] == 2.0 ** -6).all() and (one.V_scale[1, :, 0] == 2.0 ** -6).all()
    # lengths that no cache has: tokens outside [0, capacity) do not exist, memory around them stays
    three = _garbage(B, Hkv, 256, d)
    binding.attn_cache_append(three, k, v, _i32([20, 280]))
    values, _ = _values(three)
    ref = oracle.Cache(256, d)
    x = [t[0, 1].double().cpu().numpy() for t in (k, v)]
    ref.append(20, x[0][30:], x[1][30:])                   # the first 30 of 50 tokens would stand before the beginning
    for w in range(2):
        assert np.array_equal(values[w][0, 1, :20], ref.values[w][:20])
    assert (three.K.view(torch.uint8)[1, :, :192] == 0x7f).all() and torch.isfinite(three.K[1, :, 230:].float()).all()
    before = [t.clone() for t in three]
    for lengths, counts in (([-5, 0], None), ([2 ** 31 - 1, 1000], None), ([100, 100], [0, -7])):
        binding.attn_cache_append(three, k, v, _i32(lengths), None if counts is None else _i32(counts))
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, three))


# ---- attention and weights

def _filled(g, B, Hkv, cap, d, lengths, gain=1.0, mixed=True):
    """A cache whose blocks have scales of their own."""
    c = _garbage(B, Hkv, cap, d)
    N = max(max(lengths), 1)
    per_block = torch.exp2(torch.randint(-3, 4, (B, Hkv, -(-N // 64), 1), generator=g).float()).repeat_interleave(64, 2)[:, :, :N] if mixed else 1.0
    k, v = (_bf16(g, B, Hkv, N, d, gain=gain), (_bf16(g, B, Hkv, N, d).float() * per_block).to(torch.bfloat16))
    binding.attn_cache_append(c, k.to(DEV), v.to(DEV), _i32(lengths), _i32(lengths))
    return c


def _dequantised(c):
    (k, v), (ek, ev) = _values(c)
    times = lambda x, e: x * np.repeat(2.0 ** e, 64, axis=2)[..., None]
    with np.errstate(invalid="ignore", over="ignore"):
        return times(k, ek), times(v, ev)


def _check_attention(q, c, lengths, counts, alpha, causal, O, lse, w=None, w_in=None, label=""):
    B, H, N, d = q.shape
    K, V = _dequantised(c)
    Hkv, cap = K.shape[1], K.shape[2]
    group = H // Hkv
    q, O, L = q.double().cpu().numpy(), O.double().cpu().numpy(), lse.double().cpu().numpy()
    for b in range(B):
        n, length = counts[b], lengths[b]
        for h in range(H):
            k, v, x = K[b, h // group, :length], V[b, h // group, :length], q[b, h, :n]
            o, l, size = oracle.attend(x, k, v, alpha, causal)
            assert (O[b, h, n:] == 0).all() and np.isneginf(L[b, h, n:]).all(), (label, b, h)
            none = np.isneginf(l)
            assert np.array_equal(none, np.isneginf(L[b, h, :n])) and (O[b, h, :n][none] == 0).all(), (label, b, h)
            if none.all():
                continue
            e = 2 * (d + 4) * 2.0 ** -24 * alpha * (np.abs(x) @ np.abs(k.T)).max(1) + 2.0 ** -22 * np.abs(alpha * x @ k.T).max(1) + 2.0 ** -16
            off = np.abs(L[b, h, :n][~none] - l[~none]) - e[~none]
            assert off.max() <= 0, (label, "LSE", b, h, off.max())
            tol = 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + e[:, None]) * 1.01 * (size + np.abs(o))
            off = np.abs(O[b, h, :n] - o) - tol
            assert off.max() <= 0, (label, "O", b, h, off.max(), np.unravel_index(off.argmax(), off.shape))
        if w is None:
            continue
        for hk in range(Hkv):
            # a single probability below 2^-126, which float32 holds as a subnormal number only, is 0 (the hardware exponential)
            want, tol = np.zeros(cap), np.full(cap, n * group * 2.0 ** -126)
            want[:length - n] = 0.0 if w_in is None else w_in[b, hk, :length - n]
            for h in range(hk * group, (hk + 1) * group):
                k, x = K[b, hk, :length], q[b, h, :n]
                got = oracle.weights(x, k, L[b, h, :n], alpha, causal)
                want[:length] += got
                if n and length:
                    e = 2 * (d + 4) * 2.0 ** -24 * alpha * (np.abs(x) @ np.abs(k.T)).max() + 2.0 ** -22 * np.abs(alpha * x @ k.T).max() + 2.0 ** -15
                    finite = L[b, h, :n][np.isfinite(L[b, h, :n])]
                    tol[:length] += got * (e + 2.0 ** -21 * (np.abs(finite).max() if finite.size else 0))
            off = np.abs(w[b, hk].double().cpu().numpy() - want) - (tol + 2.0 ** -23 * np.abs(want))
            assert off.max() <= 0, (label, "weights", b, hk, off.max(), off.argmax())


def _run(q, c, lengths, counts, alpha, causal, label="", w_in=None):
    cts = None if counts is None else _i32(counts)
    O, lse = binding.attn_cache_fwd(q, c, _i32(lengths), alpha, causal, cts)
    w = binding.attn_cache_weights(q, c, lse, _i32(lengths), alpha, causal, cts, weights=w_in)
    B, _, N, _ = q.shape
    _check_attention(q, c, lengths, [N] * B if counts is None else counts, alpha, causal, O, lse, w, None if w_in is None else w_in.double().cpu().numpy(), label)
    return O, lse, w


@pytest.mark.parametrize("d", DIMS)
@pytest.mark.parametrize("cap", (64, 1024, 1280))          # one block; the longest that one work-group reads; shared out
def test_single_tokens(lib, d, cap):
    for group, Hkv in ((1, 3), (4, 2), (16, 1), (5, 2), (24, 1), (48, 1)):
        lengths = [min(cap, l) for l in (cap, 1, 64, 65, cap - 1, 2)]
        g = _gen(cap + group)
        c = _filled(g, len(lengths), Hkv, cap, d, lengths)
        q = _bf16(g, len(lengths), group * Hkv, 1, d).to(DEV)
        _run(q, c, lengths, None, d ** -0.5, True, f"group {group}")


@pytest.mark.parametrize("d", DIMS)
@pytest.mark.parametrize("causal", (True, False))
@pytest.mark.parametrize("cap", (192, 1600))
def test_chunks(lib, d, causal, cap):
    for N, group, lengths, counts in ((2, 1, [cap, 2, 70], None), (7, 4, [cap - 3, 7, 129], [7, 3, 0]), (40, 2, [cap, 100, 40], [40, 40, 1]),
                                      (33, 3, [0, 1, 66], [0, 1, 33]), (150, 1, [cap, 160, 151], [150, 20, 150])):
        g = _gen(N)
        c = _filled(g, 3, 2, cap, d, lengths)
        q = _bf16(g, 3, 2 * group, N, d).to(DEV)
        w_in = torch.rand((3, 2, cap), generator=g).to(DEV)
        w_in[:, :, -1] = float("nan")                      # a token of the call's, or behind the end: not read
        for b, (l, n) in enumerate(zip(lengths, counts or [N] * 3)):
            w_in[b, :, l - n:] = float("nan")
        _run(q, c, lengths, counts, 1.5 * d ** -0.5, causal, f"N {N}", w_in)


@pytest.mark.parametrize("d", DIMS)
@pytest.mark.parametrize("causal", (True, False))
def test_many_rows(lib, d, causal):
    """More rows than 3 d at any head size, and an odd number of blocks."""
    N, group, cap, lengths, counts = 210, 4, 448, [448, 215, 130], [210, 200, 130]
    g = _gen(d)
    c = _filled(g, 3, 2, cap, d, lengths)
    w_in = torch.rand((3, 2, cap), generator=g).to(DEV)
    _run(_bf16(g, 3, 2 * group, N, d).to(DEV), c, lengths, counts, d ** -0.5, causal, w_in=w_in)


@pytest.mark.parametrize("N,cap", [(1, 2112), (20, 1088)])
def test_a_work_group_for_each_of_many_segments(lib, N, cap):
    """Segments that fill the chip by themselves are not shared out up to twice the length."""
    B, Hkv, d = 33, 16, 32
    g = _gen(N)
    lengths = [cap if b % 4 == 0 else (b * 977) % cap for b in range(B)]
    c = _filled(g, B, Hkv, cap, d, lengths)
    assert binding.cache_fwd_workspace_bytes(B, Hkv, Hkv, N, d, cap) == 0 < binding.cache_fwd_workspace_bytes(B, Hkv, Hkv, N, d, 4 * cap)
    _run(_bf16(g, B, Hkv, N, d).to(DEV), c, lengths, [min(N, l) for l in lengths], d ** -0.5, True)


def test_sizes_beyond_int_are_refused(lib):
    """Views of any size cost no memory."""
    x = torch.ones(64, dtype=torch.bfloat16, device=DEV).expand(1, 1, 2 ** 31, 64)
    c, out = binding.cache_empty(1, 1, 64, 64, DEV), binding.cache_empty(1, 1, 64, 64, DEV)
    f, _ = binding.rope_frequencies(64, device=DEV)
    weights = torch.zeros(1, 1, 64, device=DEV)
    for call in (lambda: binding.attn_rope(x, None, f), lambda: binding.attn_cache_append(c, x, x, _i32([64])), lambda: binding.attn_cache_fwd(x, c, _i32([64]), 0.1),
                 lambda: binding.attn_cache_evict(c, weights, _i32([0]), 2 ** 32 + 64, 0, out=out), lambda: binding.cache_fwd_workspace_bytes(1, 1, 1, 1, 64, 2 ** 32 + 64)):
        with pytest.raises(ValueError):
            call()


def test_more_queries_than_tokens(lib):
    """The first queries of a chunk that is longer than its cache see nothing."""
    g = _gen(11)
    c = _filled(g, 2, 1, 128, 64, [5, 128])
    q = _bf16(g, 2, 4, 20, 64).to(DEV)
    O, lse, w = _run(q, c, [5, 0], None, 0.125, True)
    assert torch.isneginf(lse[0, :, :15]).all() and torch.isneginf(lse[1]).all() and (w[1] == 0).all()
    # lengths that no cache has are taken as far as it goes (sequence 1's is full; 0's memory holds NaN behind its 5 tokens)
    for bad in ([-3, -1], [2 ** 31 - 1, 200]):
        O, lse = binding.attn_cache_fwd(q, c, _i32(bad), 0.125)
        assert torch.isfinite(O[1].float()).all()
        assert (torch.isneginf(lse) if bad[0] < 0 else torch.isfinite(lse[1])).all()
        w = binding.attn_cache_weights(q, c, lse, _i32(bad), 0.125)
        assert torch.isfinite(w[1]).all() and (bad[0] > 0 or (w == 0).all())


@pytest.mark.parametrize("N,group", [(1, 4), (9, 4), (64, 2)])
@pytest.mark.parametrize("length", (50, 1500))
def test_nan_and_infinities_reach_only_who_sees_them(lib, N, group, length):
    d, cap = 128, 1536
    g = _gen(N)
    k, v = _bf16(g, 1, 1, length, d), _bf16(g, 1, 1, length, d)
    q = _bf16(g, 1, group, N, d).to(DEV)
    c = _garbage(1, 1, cap, d)
    where = length - max(1, N // 2)                        # seen by the last N // 2 queries alone (by the only one)
    v[0, 0, where, 7] = float("nan")
    v[0, 0, where, 9] = float("inf")                       # becomes the block's largest number
    binding.attn_cache_append(c, k.to(DEV), v.to(DEV), _i32([length]))
    O, lse = binding.attn_cache_fwd(q, c, _i32([length]), d ** -0.5)
    clean = v.clone()
    clean[0, 0, where, 7] = 0.0
    c2 = _garbage(1, 1, cap, d)
    binding.attn_cache_append(c2, k.to(DEV), clean.to(DEV), _i32([length]))
    O2, lse2 = binding.attn_cache_fwd(q, c2, _i32([length]), d ** -0.5)
    first = N - max(1, N // 2)
    assert torch.equal(O[:, :, :first], O2[:, :, :first]) and torch.equal(lse, lse2) and torch.isfinite(O2.float()).all()
    assert torch.isnan(O[:, :, first:, 7]).all()
    keep = [i for i in range(d) if i != 7]
    assert torch.equal(O[:, :, first:, keep], O2[:, :, first:, keep])
    # a NaN key: the rows that see it are NaN, the others and their weights are not
    k[0, 0, where, 3] = float("nan")
    binding.attn_cache_append(c, k.to(DEV), clean.to(DEV), _i32([length]))
    O3, lse3 = binding.attn_cache_fwd(q, c, _i32([length]), d ** -0.5)
    assert torch.equal(O3[:, :, :first], O2[:, :, :first]) and torch.equal(lse3[:, :, :first], lse2[:, :, :first])
    assert torch.isnan(O3[:, :, first:]).all() and torch.isnan(lse3[:, :, first:]).all()
    # tokens behind the end, rolled back, bring nothing
    back = where
    binding.attn_cache_append(c, k.to(DEV), v.to(DEV), _i32([length]))
    if back > N:
        O4, lse4 = binding.attn_cache_fwd(q, c, _i32([back]), d ** -0.5)
        assert torch.isfinite(O4.float()).all() and torch.isfinite(lse4).all()


def test_every_code_and_scale(lib):
    """One token, one query: O is the token's value, LSE its score, exactly."""
    codes = torch.arange(256, dtype=torch.uint8)
    value = codes.view(torch.float8_e4m3fn).double()
    for e in (-100, -20, 0, 13, 100, 119):
        c = _garbage(1, 1, 64, 256)
        c.K.view(torch.uint8)[0, 0, 0] = codes.to(DEV)
        c.V.view(torch.uint8)[0, 0, 0, :, 0] = codes.to(DEV)
        c.K_scale.fill_(2.0 ** e)
        c.V_scale.fill_(-(2.0 ** e))                       # there is NaN, among the codes and behind the token
        q = torch.zeros(1, 1, 1, 256, dtype=torch.bfloat16, device=DEV)
        c.K.view(torch.uint8)[0, 0, 0, 127] = c.K.view(torch.uint8)[0, 0, 0, 255] = 0
        O, lse = binding.attn_cache_fwd(q, c, _i32([1]), 1.0)
        assert lse.item() == 0.0
        assert np.array_equal(O[0, 0, 0].double().cpu().numpy(), (value * 2.0 ** e).numpy(), equal_nan=True)
        if abs(e) <= 20:
            eye = torch.eye(256, dtype=torch.bfloat16, device=DEV).view(1, 256, 1, 256)
            _, lse = binding.attn_cache_fwd(eye, c, _i32([1]), 1.0)
            want = (value * 2.0 ** e).clone()
            want[[127, 255]] = 0.0
            got = lse[0, :, 0].double().cpu()
            assert torch.allclose(got, want, rtol=3 * 2.0 ** -23, atol=0)


def test_sharp_scores_and_masked_rows_of_large_values(lib):
    """Scores of hundreds, a maximum that grows block after block, and one that stands first."""
    d, cap = 64, 2048
    for order, ends in (("growing", (0.1, 30.0)), ("falling", (30.0, 0.1))):
        g = _gen(5)
        k = _bf16(g, 1, 2, cap, d)
        ramp = torch.linspace(*ends, cap).view(1, 1, cap, 1)
        k = (k.float() * ramp).to(torch.bfloat16)
        v = _bf16(g, 1, 2, cap, d)
        c = _garbage(1, 2, cap, d)
        binding.attn_cache_append(c, k.to(DEV), v.to(DEV), _i32([cap]))
        for N in (1, 100):
            _run(_bf16(g, 1, 4, N, d, gain=2.0).to(DEV), c, [cap], None, 0.125, True, f"{order} {N}")


def test_strides_outputs_streams_workspaces(lib):
    g = _gen(6)
    B, H, Hkv, N, d, cap = 3, 8, 2, 5, 128, 2048
    lengths = _i32([2000, 7, 1111])
    c = _filled(g, B, Hkv, cap, d, [2000, 7, 1111])
    x = _bf16(g, B, N, H + 4, d).to(DEV)
    q = x[:, :, :H].permute(0, 2, 1, 3)
    O, lse = binding.attn_cache_fwd(q.contiguous(), c, lengths, 0.09)
    out = torch.full((B, N, H, d), float("nan"), dtype=torch.bfloat16, device=DEV).permute(0, 2, 1, 3)
    ws = torch.empty(binding.cache_fwd_workspace_bytes(B, H, Hkv, N, d, cap), dtype=torch.uint8, device=DEV).fill_(0xff)
    O2, lse2 = binding.attn_cache_fwd(q, c, lengths, 0.09, O=out, workspace=ws)
    assert O2 is out and torch.equal(O2, O) and torch.equal(lse2, lse)
    w, w2 = (binding.attn_cache_weights(t, c, lse, lengths, 0.09) for t in (q, q.contiguous()))
    assert torch.equal(w, w2)
    w3 = torch.rand_like(w)
    keep = w3.clone()
    assert binding.attn_cache_weights(q, c, lse, lengths, 0.09, weights=w3, out=w3) is w3
    assert torch.equal(w3, binding.attn_cache_weights(q, c, lse, lengths, 0.09, weights=keep))
    assert (w3[1, :, 7:] == 0).all() and torch.equal(w3[1, :, 2:7], w[1, :, 2:7])
    # several streams at once, each call with a workspace of its own
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        got.append(binding.attn_cache_fwd(q, c, lengths, 0.09, stream=s))
    torch.cuda.synchronize()
    assert all(torch.equal(a, O) and torch.equal(b, lse) for a, b in got)
    with pytest.raises(ValueError):
        binding.attn_cache_fwd(q, c, lengths.long(), 0.09)
    with pytest.raises(ValueError):
        binding.attn_cache_fwd(q[:2], c, lengths, 0.09)
    with pytest.raises(binding.AttnError) as e:
        binding.attn_cache_fwd(q, c, lengths, 0.09, workspace=ws[:-1])
    assert e.value.status == 4


def test_offsets_past_32_bits(lib):
    """A cache of more than 4 GiB of keys: the last head of the last sequence, against torch in float64."""
    B, Hkv, cap, d, group = 2, 3, 6 << 20, 128, 4
    c = binding.cache_empty(B, Hkv, cap, d, DEV)
    assert c.K.numel() > 1 << 32
    length = cap - 5
    pattern = torch.randint(0, 0x58, (1 << 20,), dtype=torch.uint8, generator=_gen(1)).to(DEV)          # finite codes up to 16
    pattern |= (torch.rand(1 << 20, generator=_gen(2)) < 0.5).to(torch.uint8).to(DEV) << 7
    for t in (c.K, c.V):
        t.view(torch.uint8).view(-1, 1 << 20)[:] = pattern
    g = _gen(3)
    c.K_scale.copy_(torch.exp2(torch.randint(-8, -4, c.K_scale.shape, generator=g).float()))
    c.V_scale.copy_(torch.exp2(torch.randint(-3, 3, c.V_scale.shape, generator=g).float()))
    q = _bf16(g, B, Hkv * group, 1, d).to(DEV)
    lengths = _i32([70, length])
    O, lse = binding.attn_cache_fwd(q, c, lengths, d ** -0.5)
    w = binding.attn_cache_weights(q, c, lse, lengths, d ** -0.5)
    total, most, parts = 0.0, [], []
    x = q[1, -group:, 0].double()
    s = torch.cat([(x @ (c.K[1, -1, i:i + (1 << 20)].double() * c.K_scale[1, -1, i // 64:(i >> 6) + (1 << 14)].double().repeat_interleave(64)[:, None]).t())
                   for i in range(0, cap, 1 << 20)], 1)[:, :length] * d ** -0.5
    want = torch.logsumexp(s, 1)
    # a sum of 6 << 20 terms, 2^14 after one another at most in one lane: 2^-24 * 2^14 in the worst case, 2^-13 with room
    assert (lse[1, -group:, 0].double() - want).abs().max() < 2.0 ** -10
    p = torch.softmax(s, 1)
    o = torch.zeros(group, d, dtype=torch.float64, device=DEV)
    size = torch.zeros_like(o)
    for i in range(0, length, 1 << 20):
        v = (c.V[1, -1, i // 64:(i >> 6) + (1 << 14)].double() * c.V_scale[1, -1, i // 64:(i >> 6) + (1 << 14)].double()[:, None, None]).transpose(1, 2).reshape(-1, d)
        v = v[:min(1 << 20, length - i)]
        o += p[:, i:i + len(v)] @ v
        size += p[:, i:i + len(v)] @ v.abs()
    assert ((O[1, -group:, 0].double() - o).abs() <= 2.0 ** -8 * o.abs() + (2.0 ** -8 + 2.0 ** -10) * (size + o.abs())).all()
    got = w[1, -1].double()
    mass = torch.exp(s - lse[1, -group:, 0].double()[:, None]).sum(0)
    assert (got[length:] == 0).all() and ((got[:length] - mass).abs() <= 2.0 ** -14 * mass).all()
    # a token into the last block of the last head
    k, v = _bf16(g, B, Hkv, 1, d).to(DEV), _bf16(g, B, Hkv, 1, d).to(DEV)
    c.K_scale[1, -1, -1] = c.V_scale[1, -1, -1] = 2.0 ** -6
    before = [t.view(torch.uint8)[1, -1, -1:].clone() for t in (c.K, c.V)]
    binding.attn_cache_append(c, k, v, _i32([71, cap]))
    assert not torch.equal(c.K.view(torch.uint8)[1, -1, -1:], before[0]) and not torch.equal(c.V.view(torch.uint8)[1, -1, -1:], before[1])
    near = c.K[1, -1, -1].double() * c.K_scale[1, -1, -1].double()
    assert ((near - k[1, -1, 0].double()).abs() <= 2.0 ** -4 * k[1, -1, 0].double().abs() + 2.0 ** -10 * c.K_scale[1, -1, -1].double()).all()


# ---- evict

def _check_evict(c, weights, lengths, budget, recent, out=None):
    got, w, kept = binding.attn_cache_evict(c, weights, _i32(lengths), budget, recent, out=out)
    B, Hkv, cap, d = c.K.shape
    (k, v), (ek, ev) = _values(c)
    (ko, vo), (eko, evo) = _values(got)
    host = weights.cpu()
    for b, length in enumerate(lengths):
        for h in range(Hkv):
            want = oracle.kept(host[b, h].tolist(), length, budget, recent)
            n = len(want)
            assert kept[b, h, :n].tolist() == want and (kept[b, h, n:] == -1).all(), (b, h)
            assert torch.equal(w[b, h, :n].cpu(), host[b, h, want]) or n == 0 or host[b, h, want].isnan().any()
            assert (w[b, h, n:] == 0).all()
            ref = oracle.Cache(cap, d)
            ref.values, ref.exponents = [k[b, h], v[b, h]], [np.nan_to_num(e, posinf=0, neginf=0).astype(int) for e in (ek[b, h], ev[b, h])]
            for which, (values, exps) in enumerate(((ko, eko), (vo, evo))):
                if n == 0:
                    continue
                x, e = oracle.gathered(ref, which, want)
                assert exps[b, h, :len(e)].tolist() == e
                if which == 1:
                    marked = [any(c.V_scale[b, h, t // 64] < 0 for t in want[lo:lo + 64]) for lo in range(0, n, 64)]
                    assert (got.V_scale[b, h, :len(e)] < 0).tolist() == marked
                assert np.array_equal(values[b, h, :n], x, equal_nan=True)
                assert (values[b, h, n:-(-n // 64) * 64] == 0).all()
    return got, w, kept


@pytest.mark.parametrize("d", DIMS)
def test_evict(lib, d):
    g = _gen(d)
    B, Hkv, cap = 4, 2, 448
    lengths = [448, 300, 100, 0]
    c = _filled(g, B, Hkv, cap, d, lengths)
    c.V.view(torch.uint8)[0, 1, 2, 5, 7] = 0x7f            # a NaN in token 135
    c.V_scale[0, 1, 2] *= -1
    for budget, recent in ((100, 20), (300, 300), (65, 0), (1, 1), (1, 0), (447, 63), (448, 5)):
        w = torch.exp(2 * torch.randn((B, Hkv, cap), generator=g)).to(DEV)
        out = None
        if budget == 65:                                   # room for more: what stands behind stays
            out = _garbage(B, Hkv, 256, d)
        got, _, _ = _check_evict(c, w, lengths, budget, recent, out)
        if out is not None:
            assert (got.K.view(torch.uint8)[:, :, 128:] == 0x7f).all() and (got.V.view(torch.uint8)[:, :, 2:] == 0xff).all()
            assert got.K_scale[:3, :, 2:].isnan().all() and got.K_scale[3].isnan().all()


def test_evict_ties_and_odd_weights(lib):
    g = _gen(1)
    c = _filled(g, 3, 1, 16384, 32, [16384, 9000, 5000])
    w = torch.randint(0, 4, (3, 1, 16384), generator=g).float() * 0.25          # thousands of ties
    w[1, 0, :3000] = -0.0
    w[1, 0, 3000:6000] = 0.0
    w[1, 0, 6000:] = -1.0
    w[2, 0, ::7] = float("nan")
    w[2, 0, 1::7] = float("inf")
    w[2, 0, 2::7] = float("-inf")
    w[2, 0, 3::7] = 1e-42
    for budget, recent in ((4096, 100), (1000, 0), (8200, 8000), (4999, 1)):
        _check_evict(c, w.to(DEV), [16384, 9000, 5000], budget, recent)
    # weights that differ in their last bits alone
    w = (1.0 + torch.randperm(16384, generator=g).float() * 2.0 ** -23).repeat(3, 1).view(3, 1, 16384).to(DEV)
    _check_evict(c, w, [16384, 9000, 5000], 3001, 7)


# ---- together

def test_answering_step_by_step_in_a_graph(lib):
    """A prompt, then tokens one by one through a captured graph (rotate, append, attend, weigh; lengths and positions move on the device),
    cut down once and carried on: every step against the oracle, every replay against an eager call."""
    B, H, Hkv, d, cap, budget, recent = 2, 8, 2, 64, 1280, 200, 32
    g = _gen(21)
    freq, m = lib.rope_frequencies(d, scaling="yarn", factor=8.0, original_length=256, device=DEV)
    alpha = d ** -0.5
    prompt = [250, 131]
    N = max(prompt)
    q, k, v = (_bf16(g, B, h, N, d).to(DEV) for h in (H, Hkv, Hkv))
    lengths, counts = _i32(prompt), _i32(prompt)
    big = _garbage(B, Hkv, 256, d)
    q, k = lib.attn_rope(q, k, freq, magnitude=m)
    binding.attn_cache_append(big, k, v, lengths, counts)
    O, lse = binding.attn_cache_fwd(q, big, lengths, alpha, counts=counts)
    w = binding.attn_cache_weights(q, big, lse, lengths, alpha, counts=counts)
    _check_attention(q, big, prompt, prompt, alpha, True, O, lse, w)
    # the prompt's cache, cut down into the one that answers
    cache = _garbage(B, Hkv, cap, d)
    cache, weights, kept = binding.attn_cache_evict(big, w, lengths, budget, recent, out=cache)
    lengths.clamp_(max=budget)
    position = _i32(prompt).view(B, 1)
    new = {n: torch.zeros(B, h, 1, d, dtype=torch.bfloat16, device=DEV) for n, h in (("q", H), ("k", Hkv), ("v", Hkv))}
    ws = torch.empty(binding.cache_fwd_workspace_bytes(B, H, Hkv, 1, d, cap), dtype=torch.uint8, device=DEV)

    def step():
        lengths.add_(1)
        a, b = lib.attn_rope(new["q"], new["k"], freq, positions=position, magnitude=m)
        binding.attn_cache_append(cache, b, new["v"], lengths)
        o, l = binding.attn_cache_fwd(a, cache, lengths, alpha, workspace=ws)
        binding.attn_cache_weights(a, cache, l, lengths, alpha, weights=weights, out=weights)
        position.add_(1)
        return a, b, o, l

    at, pos = lengths.clone(), position.clone()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                          # once outside, as torch wants it, and undone
        step()
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        a, b, o, l = step()
    lengths.copy_(at)
    position.copy_(pos)
    weights.copy_(_kept_weights(w, kept, cap))
    for i in range(70):                                    # over a block's end
        for n in new:
            new[n].copy_(_bf16(g, *new[n].shape))
        before = weights.clone()
        graph.replay()
        torch.cuda.synchronize()
        now = lengths.tolist()
        assert now == [x + i + 1 for x in at.tolist()] and position.view(-1).tolist() == [x + i + 1 for x in prompt]
        if i in (0, 1, 55, 56, 63, 69):
            o2, l2 = binding.attn_cache_fwd(a, cache, lengths, alpha)
            assert torch.equal(o, o2) and torch.equal(l, l2)
            _check_attention(a, cache, now, [1, 1], alpha, True, o, l, weights, before.double().cpu().numpy(), f"step {i}")
            want = positions.rotate(new["q"].double().cpu().numpy(), (position.cpu() - 1).numpy(), freq.cpu().numpy(), False, m)
            assert np.abs(a.double().cpu().numpy() - want).max() <= 2.0 ** -8 * np.abs(want).max() + 1e-5
            K, _ = _dequantised(cache)
            for s in range(B):                             # the newest key stands where it belongs
                e = np.round(np.log2(cache.K_scale[s, :, (now[s] - 1) // 64].double().cpu().numpy()))
                x = b[s, :, 0].double().cpu().numpy()
                assert (np.abs(K[s, :, now[s] - 1] - x) <= 2.0 ** -4 * np.abs(x) + 2.0 ** (e[:, None] - 10)).all()
    # and down again, between two caches
    _check_evict(cache, weights, lengths.tolist(), budget, recent)


def _kept_weights(w, kept, cap):
    out = torch.zeros((*w.shape[:2], cap), device=w.device)
    n = kept.shape[2]
    out[:, :, :n] = torch.where(kept >= 0, w.gather(2, kept.long().clamp(min=0)), 0.0)
    return out


def test_training_with_positions(lib):
    """rope, then attention, forward and backward: gradients against float64 automatic differentiation of the definition."""
    B, H, N, d = 1, 2, 96, 64
    g = _gen(31)
    q, k, v, do = (_bf16(g, B, H, N, d).to(DEV) for _ in range(4))
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    freq, m = lib.rope_frequencies(d // 2, device=DEV)
    a, b = autograd.rope(leaves[0], leaves[1], freq, interleaved=True)
    o = autograd.attention(a, b, leaves[2], causal=True, variant=binding.STANDARD)
    o.backward(do)

    def rotate(x):
        angle = torch.arange(N, dtype=torch.float64)[:, None] * freq.cpu()
        x1, x2 = x[..., 0:d // 2:2], x[..., 1:d // 2:2]
        y = torch.stack((x1 * angle.cos() - x2 * angle.sin(), x1 * angle.sin() + x2 * angle.cos()), -1).flatten(-2)
        return torch.cat((y, x[..., d // 2:]), -1)

    ref = [t.double().cpu().requires_grad_() for t in (q, k, v)]
    s = rotate(ref[0]) @ rotate(ref[1]).transpose(2, 3) * d ** -0.5
    s = s.masked_fill(torch.ones(N, N, dtype=torch.bool).triu(1), float("-inf"))
    want = torch.softmax(s, -1) @ ref[2]
    want.backward(do.double().cpu())
    # the attention's own tolerance (max-abs 2e-2, relative L2 1e-2) holds with rotated inputs rounded to bf16: relative 2^-8 each way more
    for got, w in [(o, want)] + [(x.grad, y.grad) for x, y in zip(leaves, ref)]:
        w, got = w.detach(), got.detach().double().cpu()
        assert (got - w).norm() <= 2e-2 * w.norm() and (got - w).abs().max() <= 5e-2 * max(1.0, w.abs().max().item())


def test_answering_goes_on_after_an_eviction(lib):
    """The cache that attn_cache_evict makes by itself has room for the tokens that follow."""
    g = _gen(51)
    B, H, Hkv, d, cap, budget = 2, 4, 2, 64, 256, 128
    lengths = [250, 90]
    c = _filled(g, B, Hkv, cap, d, lengths)
    w = torch.rand((B, Hkv, cap), generator=g).to(DEV)
    c, w, _ = _check_evict(c, w, lengths, budget, 16)
    assert c.K.shape[2] == cap and w.shape == (B, Hkv, cap)
    lengths = [min(n, budget) for n in lengths]
    for _ in range(3):
        lengths = [n + 1 for n in lengths]
        q, k, v = (_bf16(g, B, h, 1, d) for h in (H, Hkv, Hkv))
        binding.attn_cache_append(c, k.to(DEV), v.to(DEV), _i32(lengths))
        (K, V), (ek, ev) = _dequantised(c), _values(c)[1]
        for b, n in enumerate(lengths):                    # an E4M3 code: half a step, 2^-4 of the value or 2^-10 of the scale
            for x, got, e in ((k, K, ek), (v, V, ev)):
                want = x[b, :, 0].double().numpy()
                assert (np.abs(got[b, :, n - 1] - want) <= 2.0 ** -4 * np.abs(want) + 2.0 ** (e[b, :, (n - 1) // 64, None] - 10)).all()
        _, _, w = _run(q.to(DEV), c, lengths, None, d ** -0.5, True, w_in=w)
    # a budget beyond the old cache's capacity has its room
    more, w2, _ = binding.attn_cache_evict(c, w, _i32(lengths), 300, 0)
    assert more.K.shape[2] == 320 and w2.shape == (B, Hkv, 320)


def test_weights_of_no_queries_are_refused(lib):
    c = binding.cache_empty(2, 3, 64, 64, DEV)
    q = torch.empty(2, 0, 5, 64, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError):
        binding.attn_cache_weights(q, c, torch.empty(2, 0, 5, device=DEV), _i32([5, 9]), 0.125)


def test_append_more_tokens_than_there_is_room_for(lib):
    """2^31 - 1 new tokens (a view of one): those that would stand before the beginning do not exist."""
    x = _bf16(_gen(61), 1, 1, 1, 32).to(DEV)
    N = 2 ** 31 - 1
    for cap, length in ((64, 64), (192, 130)):
        many, few = _garbage(1, 1, cap, 32), _garbage(1, 1, cap, 32)
        binding.attn_cache_append(many, x.expand(1, 1, N, 32), x.expand(1, 1, N, 32), _i32([length]))
        binding.attn_cache_append(few, x.expand(1, 1, length, 32), x.expand(1, 1, length, 32), _i32([length]))
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(many, few))


# ---- forms that only longer caches, more segments and more rows reach

def _filled_on_gpu(seed, B, Hkv, cap, d, lengths):
    """As _filled, with keys whose blocks have scales of their own, too."""
    g = torch.Generator(DEV).manual_seed(seed)

    def rows(lo, hi):
        gain = torch.exp2(torch.randint(lo, hi, (B, Hkv, cap // 64, 1, 1), generator=g, device=DEV).float())
        x = torch.randn((B, Hkv, cap // 64, 64, d), generator=g, device=DEV)
        return x.mul_(gain).to(torch.bfloat16).view(B, Hkv, cap, d)

    c = _garbage(B, Hkv, cap, d)
    binding.attn_cache_append(c, rows(-2, 1), rows(-3, 4), _i32(lengths), _i32(lengths))
    return c


def _check_rows(q, c, lengths, counts, alpha, O, lse, pairs, terms):
    """Single queries of (sequence, key/value head) pairs against the oracle, causal.  terms: additions one after the other in a row's sum of
    probabilities, 2^-24 each; 64 more for the joins (parts and waves) and the hardware exponential's 2^-22."""
    H, N, d = q.shape[1:]
    group = H // c.K.shape[1]
    assert all((O[b, :, n:] == 0).all() and torch.isneginf(lse[b, :, n:]).all() for b, n in enumerate(counts))
    for b, hk in pairs:
        n, length = counts[b], lengths[b]
        (K, V), (ek, ev) = _values(binding.Cache(*(t[b:b + 1, hk:hk + 1] for t in c)))
        with np.errstate(invalid="ignore"):
            K, V = ((x[0, 0] * np.repeat(2.0 ** e[0, 0], 64)[:, None])[:length] for x, e in ((K, ek), (V, ev)))
        for i in sorted({*range(0, n, 13), n - 1} if n else ()):
            seen = length - n + i + 1
            for h in range(hk * group, (hk + 1) * group):
                x = q[b, h, i:i + 1].double().cpu().numpy()
                if seen <= 0:
                    assert (O[b, h, i] == 0).all() and torch.isneginf(lse[b, h, i])
                    continue
                k, v = K[:seen], V[:seen]
                o, l, size = oracle.attend(x, k, v, alpha, True)
                e = (2 * (d + 4) * alpha * (np.abs(x) @ np.abs(k.T)).max() + terms + 64) * 2.0 ** -24 + 2.0 ** -22 * np.abs(alpha * x @ k.T).max()
                assert abs(lse[b, h, i].item() - l[0]) <= e, (b, h, i)
                off = np.abs(O[b, h, i].double().cpu().numpy() - o[0]) - (2.0 ** -8 * np.abs(o[0]) + (2.0 ** -8 + e) * 1.01 * (size[0] + np.abs(o[0])))
                assert off.max() <= 0, (b, h, i, off.max(), off.argmax())


@pytest.mark.parametrize("d", DIMS)
@pytest.mark.parametrize("B,Hkv,group,N,cap", [
    (17, 8, 2, 1, 4160),           # a wave's own blocks: segments in a few parts, as many shares as run at once
    (41, 16, 1, 1, 4160),          # more segments than shares
    (6, 8, 2, 20, 1280),           # blocks shared through LDS, one row tile a wave
    (2, 8, 4, 300, 1280)])         # two, and ten tiles a sequence and head
def test_parts_joined_by_two_waves(lib, d, B, Hkv, group, N, cap):
    """Every segment is shared out (the call has a workspace), and in fewer than four parts on average."""
    lengths = [cap if b % 5 == 0 else max(N, b * 977 % cap) for b in range(B)]
    counts = [N if b % 2 == 0 else N - N // 3 for b in range(B)]
    if B > 3:
        lengths[3] = counts[3] = 0
    c = _filled_on_gpu(d + N, B, Hkv, cap, d, lengths)
    assert binding.cache_fwd_workspace_bytes(B, group * Hkv, Hkv, N, d, cap) > 0
    q = _bf16(_gen(B), B, group * Hkv, N, d).to(DEV)
    O, lse = binding.attn_cache_fwd(q, c, _i32(lengths), d ** -0.5, counts=_i32(counts))
    # a lane adds 16 probabilities a block; a segment's blocks lie in one lane at most
    _check_rows(q, c, lengths, counts, d ** -0.5, O, lse, [(b, h) for b in range(B) for h in (0, Hkv // 2 + 1)], cap // 4)


@pytest.mark.parametrize("d", DIMS)
@pytest.mark.parametrize("N", (20, 40))                    # 40 rows: one row tile a wave; 80: two
def test_more_than_64_staged_blocks_of_a_segment(lib, d, N):
    """72 full segments of 512 blocks on 512 work-groups (256 at d = 256): 72 blocks or more each, whose scales come 64 at a time."""
    B, Hkv, group, cap = 9, 8, 2, 32768
    c = _filled_on_gpu(d + N, B, Hkv, cap, d, [cap] * B)
    q = _bf16(_gen(N), B, group * Hkv, N, d).to(DEV)
    O, lse = binding.attn_cache_fwd(q, c, _i32([cap] * B), d ** -0.5)
    _check_rows(q, c, [cap] * B, [N] * B, d ** -0.5, O, lse, [(0, 0), (0, 1), (4, 3), (8, 7)], 16 * 512)


def test_evict_more_weights_than_fit_into_lds(lib):
    """32768 weights in front of the recent ones stay in LDS, one more does not; ends inside a thread's four."""
    g = _gen(41)
    lengths, cap = [32868, 32869, 39999], 40000
    c = _filled(g, 3, 1, cap, 32, lengths)
    spread = torch.exp(2 * torch.randn((3, 1, cap), generator=g))
    tied = torch.randint(0, 4, (3, 1, cap), generator=g).float() * 0.25
    tied[1, 0, ::3] = -0.0
    for w in (spread, tied):
        for budget, recent in ((5000, 100), (33000, 0), (1, 0)):
            _check_evict(c, w.to(DEV), lengths, budget, recent)
