"""CPU-only checks of the rotary positions' and the 8-bit cache's entry points: what they refuse before anything is launched."""
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


def test_rope_refusals(binding):
    lib = binding.raw()

    def rope(Q=_p(1), K=_p(2), Qo=_p(3), Ko=_p(4), strides=None, pos=None, ps=0, f=_p(5), B=1, H=4, Hkv=2, N=8, d=64, rot=64, m=1.0):
        return lib.attn_rope(Q, K, Qo, Ko, strides, pos, ps, f, B, H, Hkv, N, d, rot, 0, m, 0, None)

    assert rope(B=0, Q=None, Qo=None, K=None, Ko=None, f=None) == OK and rope(H=0, Q=None, Qo=None, K=None, Ko=None, f=None) == OK
    assert rope(Q=None) == NULL and rope(Qo=None) == NULL and rope(f=None) == NULL
    assert rope(Ko=None) == NULL and rope(K=None) == NULL                       # keys without a place for them, and the reverse
    assert rope(Q=MIS) == BAD and rope(K=MIS) == BAD and rope(f=MIS) == BAD and rope(pos=INT_MIS) == BAD
    assert rope(rot=0) == BAD and rope(rot=3) == BAD and rope(rot=66) == BAD and rope(rot=-2) == BAD
    assert rope(d=80, rot=16) == UNSUP and rope(N=0) == UNSUP and rope(N=-1) == BAD and rope(Hkv=-1) == BAD
    assert rope(m=math.inf) == BAD and rope(m=math.nan) == BAD
    assert rope(H=65000, Hkv=1000) == UNSUP and rope(B=1 << 16, H=1, Hkv=1, N=1 << 16, d=32, rot=32) == UNSUP
    assert rope(pos=_p(6), ps=-8) == BAD
    good = (2048, 512, 64)
    bad = lambda i, s: rope(strides=_strides(*[x for j in range(4) for x in (s if j == i else good)]))
    for i in range(4):
        assert bad(i, (2048, 512, 60)) == BAD and bad(i, (2048, -512, 64)) == BAD
    assert bad(2, (0, 512, 64)) == BAD and bad(3, (2048, 512, 0)) == BAD         # expanded outputs
    assert rope(Ko=_p(3)) == BAD and rope(Qo=_p(2)) == BAD and rope(Ko=_p(1)) == BAD
    assert rope(Qo=_p(1), strides=_strides(*good, *good, 4096, 1024, 64, *good)) == BAD      # in place with other strides


def test_rope_frequencies_refusals(binding):
    for kw in (dict(rot=0), dict(rot=3), dict(rot=258), dict(base=0.0), dict(base=math.inf), dict(base=math.nan), dict(scaling="linear", factor=0.5),
               dict(scaling="ntk", rot=2, factor=2.0), dict(scaling="yarn", factor=2.0), dict(scaling="yarn", factor=2.0, original_length=math.inf),
               dict(scaling="yarn", factor=2.0, original_length=10, beta_fast=1.0, beta_slow=1.0), dict(scaling="linear", factor=math.nan),
               dict(scaling="yarn", factor=2.0, original_length=10, beta_slow=-1.0)):
        with pytest.raises(binding.AttnError) as e:
            binding.rope_frequencies(**{"rot": 64, **kw}, device="cpu")
        assert e.value.status == BAD, kw
    with pytest.raises(ValueError):
        binding.rope_frequencies(64, scaling="other", device="cpu")
    f, m = binding.rope_frequencies(4, 100.0, device="cpu")
    assert f.tolist() == [1.0, 0.1] and m == 1.0
    assert binding.raw().attn_rope_frequencies(None, None, 64, 1e4, 0, 1.0, 0.0, 0.0, 0.0) == NULL


def test_append_refusals(binding):
    lib = binding.raw()

    def append(K=_p(1), V=_p(2), strides=None, Kc=_p(3), Vc=_p(4), Ks=_p(5), Vs=_p(6), lengths=_p(7), counts=None, B=2, H=2, N=3, d=64, cap=128):
        return lib.attn_cache_append(K, V, strides, Kc, Vc, Ks, Vs, lengths, counts, B, H, N, d, cap, None)

    assert append(B=0, K=None, V=None, Kc=None, Vc=None, Ks=None, Vs=None, lengths=None) == OK and append(H=0) == OK
    for name in ("K", "V", "Kc", "Vc", "Ks", "Vs", "lengths"):
        assert append(**{name: None}) == NULL, name
        assert append(**{name: INT_MIS if name == "lengths" else MIS}) == BAD, name
    assert append(counts=INT_MIS) == BAD
    assert append(cap=0) == BAD and append(cap=100) == BAD and append(cap=-64) == BAD and append(cap=(1 << 30) + 64) == UNSUP
    assert append(d=80) == UNSUP and append(N=0) == UNSUP and append(N=-1) == BAD and append(B=-1) == BAD
    assert append(B=1 << 16) == UNSUP and append(H=1 << 16) == UNSUP and append(B=4096, H=64, cap=1 << 20) == UNSUP
    assert append(Kc=_p(1)) == BAD and append(Vc=_p(3)) == BAD and append(Vs=_p(5)) == BAD
    assert append(strides=_strides(512, 64, 60, 512, 64, 64)) == BAD and append(strides=_strides(512, 64, 64, 512, -64, 64)) == BAD


def test_attention_and_weights_refusals(binding):
    lib = binding.raw()
    big = 1 << 40

    def fwd(Q=_p(1), strides=None, Kc=_p(2), Vc=_p(3), Ks=_p(4), Vs=_p(5), lengths=_p(6), counts=None, O=_p(7), L=_p(8), ws=_p(9), wb=big, B=2, H=4,
            Hkv=2, N=3, d=64, cap=2048, scale=0.125):
        return lib.attn_cache_fwd(Q, strides, Kc, Vc, Ks, Vs, lengths, counts, O, L, ws, wb, B, H, Hkv, N, d, cap, 1, scale, None)

    assert fwd(B=0, Q=None, O=None) == OK and fwd(H=0, Hkv=0) == OK
    for name in ("Q", "Kc", "Vc", "Ks", "Vs", "lengths", "O", "L"):
        assert fwd(**{name: None}) == NULL, name
        assert fwd(**{name: INT_MIS if name == "lengths" else MIS}) == BAD, name
    need = binding.cache_fwd_workspace_bytes(2, 4, 2, 3, 64, 2048)
    assert need > 0 and fwd(ws=None) == NULL and fwd(wb=need - 1) == WS and fwd(ws=MIS) == WS
    assert fwd(H=3) == BAD and fwd(Hkv=0) == BAD and fwd(Hkv=-1) == BAD and fwd(H=2, Hkv=4) == BAD
    assert fwd(scale=0.0) == BAD and fwd(scale=math.nan) == BAD and fwd(scale=math.inf) == BAD
    assert fwd(cap=100) == BAD and fwd(N=0) == UNSUP and fwd(d=48) == UNSUP
    assert fwd(O=_p(1)) == BAD and fwd(O=_p(3)) == BAD and fwd(L=_p(4)) == BAD
    assert fwd(strides=_strides(768, 192, 64, 768, 192, 0)) == BAD and fwd(strides=_strides(768, 192, 4, 768, 192, 64)) == BAD
    assert fwd(N=1 << 28) == UNSUP                                               # rows of a sequence are counted in int
    assert binding.cache_fwd_workspace_bytes(2, 3, 2, 3, 64, 2048) == 0 == binding.cache_fwd_workspace_bytes(0, 4, 2, 3, 64, 2048)

    def weigh(Q=_p(1), strides=None, Kc=_p(2), Ks=_p(3), L=_p(4), lengths=_p(5), counts=None, win=_p(6), out=_p(7), H=4, cap=2048, scale=0.125):
        return lib.attn_cache_weights(Q, strides, Kc, Ks, L, lengths, counts, win, out, 2, H, 2, 3, 64, cap, 1, scale, None)

    for name in ("Q", "Kc", "Ks", "L", "lengths", "out"):
        assert weigh(**{name: None}) == NULL, name
        assert weigh(**{name: INT_MIS if name == "lengths" else MIS}) == BAD, name
    assert weigh(win=MIS) == BAD and weigh(out=_p(2)) == BAD and weigh(out=_p(4)) == BAD and weigh(H=3) == BAD and weigh(cap=32) == BAD
    assert weigh(scale=-1.0) == BAD and weigh(strides=_strides(768, 192, 63)) == BAD


def test_evict_refusals(binding):
    lib = binding.raw()
    names = ["K", "V", "Ks", "Vs", "w", "lengths", "Ko", "Vo", "Kso", "Vso", "wo", "kept"]

    def evict(B=2, H=2, d=64, cap=256, cap_out=128, budget=100, recent=10, **kw):
        ptrs = [kw.get(n, _p(i + 1)) for i, n in enumerate(names)]
        return lib.attn_cache_evict(*ptrs, B, H, d, cap, cap_out, budget, recent, None)

    assert evict(B=0, K=None) == OK
    for n in names:
        if n != "wo":
            assert evict(**{n: None}) == NULL, n
        assert evict(**{n: INT_MIS if n in ("lengths", "kept") else MIS}) == BAD, n
    assert evict(budget=0) == BAD and evict(budget=129) == BAD and evict(recent=-1) == BAD and evict(recent=101) == BAD
    assert evict(cap=100) == BAD and evict(cap_out=100) == BAD and evict(d=48) == UNSUP and evict(B=-1) == BAD
    assert evict(Ko=_p(1)) == BAD and evict(wo=_p(5)) == BAD and evict(Vo=_p(7)) == BAD and evict(kept=_p(6)) == BAD


def test_binding_refuses_tensors_that_are_not_the_gpus(binding):
    cpu = torch.zeros((1, 2, 3, 64), dtype=torch.bfloat16)
    cache = binding.cache_empty(1, 2, 64, 64, device="cpu")
    lengths = torch.ones(1, dtype=torch.int32)
    assert cache.V.shape == (1, 2, 1, 64, 64) and cache.K.dtype == torch.float8_e4m3fn
    with pytest.raises(ValueError):
        binding.cache_empty(1, 2, 100, 64, device="cpu")
    for call in (lambda: binding.attn_rope(cpu, cpu, torch.ones(32, dtype=torch.float64)), lambda: binding.attn_cache_append(cache, cpu, cpu, lengths),
                 lambda: binding.attn_cache_fwd(cpu, cache, lengths, 0.1), lambda: binding.attn_cache_evict(cache, lengths, lengths, 10, 1)):
        with pytest.raises((ValueError, RuntimeError)):
            call()


def test_rope_of_keys_alone_is_checked_like_any(binding):
    lib = binding.raw()

    def rope(K=_p(2), Ko=_p(4), strides=None, f=_p(5), B=1, Hkv=2, N=8, d=64, rot=64):
        return lib.attn_rope(None, K, None, Ko, strides, None, 0, f, B, 0, Hkv, N, d, rot, 0, 1.0, 0, None)

    assert rope(B=0) == OK and rope(Hkv=0) == OK
    assert rope(K=MIS) == BAD and rope(f=None) == NULL and rope(Ko=None) == NULL and rope(rot=3) == BAD and rope(d=80, rot=16) == UNSUP
    good, other = (1024, 512, 64), (4096, 2048, 64)
    assert rope(strides=_strides(*good, 1024, 512, 60, *good, *good)) == BAD and rope(strides=_strides(*good, *good, *good, 1024, 0, 64)) == BAD
    assert rope(Ko=_p(2), strides=_strides(*good, *good, *good, *other)) == BAD          # in place with other strides


def test_rope_grids_beyond_the_limit(binding):
    """Refused before they are launched: 2^32 threads along a dimension."""
    lib = binding.raw()

    def rope(N, d, rot, interleaved, B=1):
        return lib.attn_rope(_p(1), None, _p(3), None, None, None, 0, _p(5), B, 1, 0, N, d, rot, interleaved, 1.0, 0, None)

    assert rope(1 << 24, 256, 2, 0) == UNSUP and rope(1 << 12, 256, 2, 0, B=1 << 12) == UNSUP          # 255 threads a token
    assert rope(1 << 24, 256, 250, 0) == UNSUP and rope(1 << 28, 96, 96, 1) == UNSUP                   # 131; 24: ten tokens a work-group
    assert rope((1 << 30) - 63, 32, 32, 0) == UNSUP and rope(1 << 29, 32, 32, 1) == UNSUP              # 4: 64; 8: 32


def test_append_grids_beyond_the_limit(binding):
    lib = binding.raw()
    for N in (1 << 30, (1 << 30) - 126, (1 << 31) - 1):
        assert lib.attn_cache_append(_p(1), _p(2), None, _p(3), _p(4), _p(5), _p(6), _p(7), None, 1, 1, N, 32, 1 << 30, None) == UNSUP


def test_evict_grids_beyond_the_limit(binding):
    """Before the first of its kernels has written anything."""
    lib = binding.raw()
    assert lib.attn_cache_evict(*[_p(i + 1) for i in range(12)], 1, 1, 32, 1 << 20, 1 << 30, 100, 10, None) == UNSUP


def test_weights_grids_beyond_the_limit(binding):
    lib = binding.raw()
    assert lib.attn_cache_weights(_p(1), None, _p(2), _p(3), _p(4), _p(5), None, _p(6), _p(7), 1, 1, 1, 769, 256, 1 << 30, 1, 0.125, None) == UNSUP


def test_attention_does_without_the_marshalling_of_plain_calls():
    """The binding imports where _operators does not (built for another torch, say); the calls that need it say so."""
    import os
    import subprocess
    import sys
    code = """
import sys
sys.modules['paper_2510_04212_amd._operators'] = None
from paper_2510_04212_amd import binding
assert binding.attn_fwd and binding.bwd_workspace_bytes(1, 2, 128, 64) > 0
x = binding.torch.zeros((1, 1, 1, 64), dtype=binding.torch.bfloat16)
c = binding.cache_empty(1, 1, 64, 64, device='cpu')
f, _ = binding.rope_frequencies(64, device='cpu')
for call in (lambda: binding.attn_rope(x, None, f), lambda: binding.attn_cache_append(c, x, x, None), lambda: binding.attn_cache_fwd(x, c, None, 1.0),
             lambda: binding.attn_cache_weights(x, c, x, None, 1.0), lambda: binding.attn_cache_evict(c, x, x, 1, 0, out=c)):
    try:
        call()
    except ImportError as e:
        assert 'build' in str(e) and e.__cause__ is not None
    else:
        raise SystemExit('nothing raised')
print('fine')
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "fine", r.stderr


def test_frequencies_of_sizes_beyond_int_are_refused(binding):
    for rot in (2 ** 32 + 64, -2 ** 32 + 64):
        with pytest.raises(ValueError):
            binding.rope_frequencies(rot, device="cpu")
    with pytest.raises(binding.AttnError):
        binding.rope_frequencies(2 ** 31 - 2, device="cpu")
