"""CPU-only checks of the entry points for continuations of a prompt: what they refuse before anything is launched."""
import ctypes
import math

import pytest
import torch

OK, NULL, BAD, UNSUP, WS = 0, 1, 2, 3, 4


@pytest.fixture(scope="module")
def binding():
    from paper_2510_04212_amd import binding as b
    return b


def _p(n):
    return ctypes.c_void_p(0x100000 * n)          # aligned, never dereferenced


MIS = ctypes.c_void_p(0x1004)
INT_MIS = ctypes.c_void_p(0x1002)


def _strides(*s):
    return (ctypes.c_longlong * len(s))(*s)


def test_shared_attention_refusals(binding):
    lib = binding.raw()
    names = ["Q", "strides", "Kp", "Vp", "Kps", "Vps", "plen", "K", "V", "Ks", "Vs", "len", "counts", "O", "L", "ws"]

    def fwd(P=2, S=3, H=4, Hkv=2, N=3, d=64, pcap=2048, cap=128, scale=0.125, wb=1 << 50, **kw):
        a = [kw.get(n, None if n in ("strides", "counts") else _p(i + 1)) for i, n in enumerate(names)]
        return lib.attn_cache_fwd_shared(*a, wb, P, S, H, Hkv, N, d, pcap, cap, 1, scale, None)

    assert fwd(P=0, Q=None, O=None) == OK and fwd(S=0) == OK and fwd(H=0, Hkv=0) == OK
    for n in names:
        if n in ("strides", "counts", "ws"):
            continue
        assert fwd(**{n: None}) == NULL, n
        assert fwd(**{n: INT_MIS if n in ("plen", "len") else MIS}) == BAD, n
    assert fwd(counts=INT_MIS) == BAD
    assert fwd(P=-1) == BAD and fwd(S=-1) == BAD and fwd(N=-1) == BAD and fwd(H=3) == BAD and fwd(Hkv=0) == BAD and fwd(H=2, Hkv=4) == BAD
    assert fwd(scale=0.0) == BAD and fwd(scale=math.nan) == BAD and fwd(scale=math.inf) == BAD
    assert fwd(cap=100) == BAD and fwd(pcap=100) == BAD and fwd(pcap=0) == BAD and fwd(N=0) == UNSUP and fwd(d=48) == UNSUP
    assert fwd(P=256, S=256) == UNSUP and fwd(P=1 << 16, S=1 << 16) == UNSUP and fwd(pcap=(1 << 30) + 64) == UNSUP
    assert fwd(P=1, S=1 << 12, N=1 << 16) == UNSUP                               # rows of a prefix are counted in int
    assert fwd(P=1, S=16384, H=64, Hkv=64, pcap=1 << 20, N=1) == UNSUP           # and so is the work
    for out in ("O", "L"):
        for n in ("Q", "Kp", "Vp", "Kps", "Vps", "K", "V", "Ks", "Vs"):
            assert fwd(**{out: _p(names.index(n) + 1)}) == BAD, (out, n)
    assert fwd(O=_p(15)) == BAD
    assert fwd(strides=_strides(768, 192, 64, 768, 192, 0)) == BAD and fwd(strides=_strides(768, 192, 4, 768, 192, 64)) == BAD
    for size in ((1, 4, 12, 12, 1, 64, 1024, 128), (16, 8, 32, 8, 1, 128, 4096, 512), (2, 8, 32, 8, 64, 128, 8192, 1024)):
        need = binding.cache_fwd_shared_workspace_bytes(*size)
        P, S, H, Hkv, N, d, pcap, cap = size
        if need:
            kw = dict(P=P, S=S, H=H, Hkv=Hkv, N=N, d=d, pcap=pcap, cap=cap)
            assert fwd(ws=None, **kw) == NULL and fwd(wb=need - 1, **kw) == WS and fwd(ws=MIS, **kw) == WS
    assert binding.cache_fwd_shared_workspace_bytes(0, 4, 4, 2, 1, 64, 64, 64) == 0 == binding.cache_fwd_shared_workspace_bytes(1, 4, 3, 2, 1, 64, 64, 64)


def test_long_prefixes_are_shared_out(binding):
    """A work-group that walks a long prefix alone ends long after the others where these are short: such calls have parts, and so a workspace, however little the
    sequences share."""
    for P in (1, 4, 16, 64):
        for S in (1, 2, 3):
            for H, Hkv, d, N in ((32, 8, 128, 1), (12, 12, 64, 1), (16, 8, 32, 1), (8, 4, 256, 1), (32, 8, 128, 16), (16, 8, 32, 16), (32, 8, 128, 64), (8, 1, 128, 2)):
                for pcap in (1 << 15, 1 << 17, 1 << 20):
                    assert binding.cache_fwd_shared_workspace_bytes(P, S, H, Hkv, N, d, pcap, 512) > 0, (P, S, H, Hkv, N, d, pcap)


def test_more_row_tiles_than_a_grid_has_are_refused(binding):
    """Tiles of 128 rows are the grid's second dimension in the form without parts; the other form is not asked for more either."""
    null = [None] * 4
    for P, S in ((1, 1), (1, 2), (2, 1)):
        for pcap in (64, 8192):
            size = lambda N: (P, S, 1, 1, N, 64, pcap, 64)
            refused = lambda N: binding.raw().attn_cache_fwd_shared(None, None, *null, None, *null, None, None, None, None, None, 0, *size(N), 1, 0.125, None)
            assert refused(65535 * 128) == NULL and refused(65535 * 128 + 1) == UNSUP
            assert binding.cache_fwd_shared_workspace_bytes(*size(65535 * 128 + 1)) == 0


def test_fork_refusals(binding):
    lib = binding.raw()
    names = ["K", "V", "Ks", "Vs", "sources", "lengths", "Ko", "Vo", "Kso", "Vso", "lo"]

    def fork(B=2, Bo=3, H=2, d=64, cap=128, cap_out=256, **kw):
        return lib.attn_cache_fork(*[kw.get(n, _p(i + 1)) for i, n in enumerate(names)], B, Bo, H, d, cap, cap_out, None)

    assert fork(Bo=0, K=None) == OK and fork(H=0) == OK
    for n in names:
        assert fork(**{n: None}) == NULL, n
        assert fork(**{n: INT_MIS if n in ("sources", "lengths", "lo") else MIS}) == BAD, n
    assert fork(B=0) == BAD and fork(B=-1) == BAD and fork(Bo=-1) == BAD and fork(cap=100) == BAD and fork(cap_out=0) == BAD
    assert fork(d=48) == UNSUP and fork(B=1 << 16) == UNSUP and fork(Bo=1 << 16) == UNSUP and fork(Bo=4096, H=64, cap_out=1 << 20) == UNSUP
    for i, out in enumerate(names[6:]):
        for n in names[:6 + i]:
            assert fork(**{out: _p(names.index(n) + 1)}) == BAD, (out, n)


def test_reorder_refusals(binding):
    lib = binding.raw()
    names = ["K", "V", "Ks", "Vs", "parents", "lengths", "lo"]

    def reorder(P=2, S=3, H=2, d=64, cap=128, **kw):
        return lib.attn_cache_reorder(*[kw.get(n, _p(i + 1)) for i, n in enumerate(names)], P, S, H, d, cap, None)

    assert reorder(P=0, K=None) == OK and reorder(S=0) == OK and reorder(H=0) == OK
    for n in names:
        assert reorder(**{n: None}) == NULL, n
        assert reorder(**{n: INT_MIS if n in ("parents", "lengths", "lo") else MIS}) == BAD, n
    assert reorder(P=-1) == BAD and reorder(S=-1) == BAD and reorder(cap=32) == BAD and reorder(H=-1) == BAD
    assert reorder(S=65) == UNSUP and reorder(P=1 << 16) == UNSUP and reorder(P=1025, S=64) == UNSUP and reorder(d=80) == UNSUP
    for i, a in enumerate(names):
        for b in names[:i]:
            if {a, b} != {"parents", "lengths"}:
                assert reorder(**{a: _p(names.index(b) + 1)}) == BAD, (a, b)


def test_select_refusals(binding):
    lib = binding.raw()
    names = ["logits", "scores", "finished", "parents", "tokens", "sums", "ended", "ws"]

    def select(type=1, sb=4000, sk=1000, end=2, wb=1 << 50, B=2, beams=4, V=1000, n=8, **kw):
        p = {m: kw.get(m, _p(i + 1)) for i, m in enumerate(names)}
        return lib.attn_beam_select(p["logits"], type, sb, sk, p["scores"], p["finished"], end, p["parents"], p["tokens"], p["sums"], p["ended"], p["ws"], wb,
                                    B, beams, V, n, None)

    assert select(B=0, logits=None) == OK and select(n=0, logits=None) == OK
    for n in ("logits", "scores", "parents", "tokens", "sums", "ws"):
        assert select(**{n: None}) == NULL, n
        assert select(**{n: MIS if n == "ws" else INT_MIS}) == (WS if n == "ws" else BAD), n
    assert select(type=0, logits=ctypes.c_void_p(0x1001)) == BAD and select(type=2) == BAD and select(type=-1) == BAD
    assert select(B=-1) == BAD and select(n=-1) == BAD and select(beams=0) == BAD and select(V=0) == BAD and select(sb=-1) == BAD and select(sk=-1) == BAD
    assert select(end=1000) == BAD and select(end=-1) == BAD                      # ended beams need their token
    assert select(beams=65) == UNSUP and select(n=129) == UNSUP and select(V=(1 << 24) + 1) == UNSUP and select(B=(1 << 20) + 1) == UNSUP
    assert select(B=1 << 20, beams=64, V=1 << 20) == UNSUP                        # a grid beyond the runtime's limit
    need = binding.beam_select_workspace_bytes(2, 4, 1000, 8)
    assert need > 0 and select(wb=need - 1) == WS
    for i, a in enumerate(names[3:7]):
        for b in names[:3 + i]:
            assert select(**{a: _p(names.index(b) + 1)}) == BAD, (a, b)
    assert binding.beam_select_workspace_bytes(2, 65, 1000, 8) == 0


def test_binding_refuses_what_does_not_fit_together(binding):
    cache = binding.cache_empty(2, 2, 64, 64, device="cpu")
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)
    q = torch.zeros((2, 2, 1, 64), dtype=torch.bfloat16)
    x = torch.zeros((1, 2, 10))
    for call in (lambda: binding.attn_cache_fwd_shared(q, cache, i32(1, 1), cache, i32(1, 1), 0.1), lambda: binding.attn_cache_fork(cache, i32(0), i32(1, 1)),
                 lambda: binding.attn_cache_reorder(cache, i32(0, 1).view(1, 2), i32(1, 1)), lambda: binding.attn_beam_select(x, x[:, :, 0], 2)):
        with pytest.raises(ValueError):
            call()
    for sizes in ((2 ** 31, 1, 1, 1), (1, 1, 2 ** 32 + 5, 1)):
        with pytest.raises(ValueError):
            binding.beam_select_workspace_bytes(*sizes)
    with pytest.raises(ValueError):
        binding.cache_fwd_shared_workspace_bytes(1, 1, 1, 1, 1, 64, 2 ** 32 + 64, 64)
