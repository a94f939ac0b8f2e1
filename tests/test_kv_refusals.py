"""What the entry points of the quantised cache and of rotary positions refuse, before any HIP call (no GPU needed)."""
import ctypes
import math
import os
import re

import numpy as np
import pytest

from paper_2604_18616_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x1000                                       # an aligned address, never followed: the checks come before any HIP call
L3 = ctypes.c_longlong * 3
GOOD = L3(8 * 64 * 128, 64 * 128, 128)


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def cache(k=A, v=A, ke=A, ve=A, pages=10, Hkv=2, page=16, D=128):
    return ctypes.byref(binding._CacheStruct(k, v, ke, ve, pages, Hkv, page, D))


BAD_CACHES = [(dict(k=None), -1), (dict(v=None), -1), (dict(ke=None), -1), (dict(ve=None), -1), (dict(pages=0), -2), (dict(Hkv=0), -2),
              (dict(Hkv=-1), -2), (dict(page=0), -2), (dict(D=0), -2), (dict(page=8), -3), (dict(page=48), -3), (dict(page=256), -3),
              (dict(D=96), -3), (dict(D=256), -3), (dict(k=A + 8), -4), (dict(v=A + 1), -4), (dict(pages=1 << 30, Hkv=2), -2)]


def test_headers_declare_what_the_library_exports(lib):
    names = {}
    for header in ("kv_cache.h", "rope.h"):
        src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
        names[header] = set(re.findall(r"\b([a-z_][a-z0-9_]*)\s*\([^;{]*\)\s*;", src))
        for name in names[header]:
            assert hasattr(lib, name), name
    assert names == {"kv_cache.h": {"kv_fp8_write", "kv_fp8_read", "attn_kv_fp8", "attn_kv_fp8_workspace_bytes"}, "rope.h": {"rope_bf16", "rope_frequencies"}}


def test_headers_are_plain_c(tmp_path):
    import subprocess
    c = tmp_path / "use.c"
    c.write_text('#include "kv_cache.h"\n#include "rope.h"\nint main(void) { KvFp8Cache c = {0, 0, 0, 0, 1, 1, 16, 64}; return c.page == 16 && (void *)attn_kv_fp8 != (void *)rope_bf16 ? 0 : 1; }\n')
    exe = str(tmp_path / "use")
    binding.load_library()
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(c), "-o", exe, binding.LIB_PATH,
                           "-Wl,-rpath," + os.path.dirname(binding.LIB_PATH), "-Wl,-rpath,/opt/rocm/lib"])
    assert subprocess.call([exe]) == 0


def test_write_refuses(lib):
    def w(c=None, k=A, v=A, ks=GOOD, vs=GOOD, table=A, pitch=8, width=8, start=A, count=A, B=1, S=4, **kw):
        return lib.kv_fp8_write(c or cache(**kw), k, v, ks, vs, table, pitch, width, start, count, B, S, None)

    for kw, code in BAD_CACHES:
        assert w(**kw) == code, kw
    assert lib.kv_fp8_write(None, A, A, GOOD, GOOD, A, 8, 8, A, A, 1, 4, None) == -1
    for kw in (dict(table=None), dict(start=None), dict(ks=None), dict(vs=None)):
        assert w(**kw) == -1, kw
    assert lib.kv_fp8_write(cache(), None, A, GOOD, GOOD, A, 8, 8, A, A, 1, 4, None) == -1
    for kw in (dict(B=0), dict(S=0), dict(S=1 << 30), dict(width=0), dict(width=1 << 26), dict(pitch=-1), dict(ks=L3(0, 0, 64)), dict(vs=L3(-8, 0, 128)),
               dict(ks=L3(0, 0, 1 << 28)), dict(B=1 << 20, S=1 << 20)):
        assert w(**kw) == -2, kw
    for kw in (dict(table=A + 2), dict(start=A + 1), dict(count=A + 2), dict(ks=L3(0, 0, 132))):
        assert w(**kw) == -4, kw


def test_read_refuses(lib):
    def r(c=None, k=A, v=A, ks=GOOD, vs=GOOD, table=A, pitch=8, width=8, lens=A, B=1, S=4, first=0, **kw):
        return lib.kv_fp8_read(c or cache(**kw), table, pitch, width, lens, k, v, ks, vs, B, S, first, None)

    for kw, code in BAD_CACHES:
        assert r(**kw) == code, kw
    for kw in (dict(table=None), dict(lens=None), dict(ks=None), dict(vs=None)):
        assert r(**kw) == -1, kw
    for kw in (dict(B=0), dict(S=0), dict(first=-1), dict(S=1 << 30), dict(width=0), dict(B=1 << 20, S=1 << 20), dict(vs=L3(0, 0, 64))):
        assert r(**kw) == -2, kw
    for kw in (dict(table=A + 2), dict(lens=A + 1), dict(vs=L3(4, 0, 128))):
        assert r(**kw) == -4, kw


def test_attention_refuses(lib):
    def a(q=A, c=None, table=A, pitch=8, width=8, lens=A, q_lens=None, o=A, lse=A, B=1, Hq=4, Sq=2, qs=GOOD, os_=GOOD, causal=1, window=0, sinks=0,
          scale=0.1, max_len=0, ws=None, wsb=0, splits=0, wg_rows=0, **kw):
        return lib.attn_kv_fp8(q, c or cache(**kw), table, pitch, width, lens, q_lens, o, lse, B, Hq, Sq, qs, os_, causal, window, sinks, scale, max_len,
                               ws, wsb, splits, wg_rows, None)

    for kw, code in BAD_CACHES:
        assert a(**kw) == code, kw
    for kw in (dict(q=None), dict(o=None), dict(table=None), dict(lens=None), dict(qs=None), dict(os_=None)):
        assert a(**kw) == -1, kw
    for kw in (dict(B=0), dict(Hq=0), dict(Hq=5), dict(Sq=0), dict(window=-1), dict(sinks=-1), dict(max_len=-1), dict(Sq=1 << 28), dict(B=1 << 20, Sq=1 << 20),
               dict(width=-1), dict(qs=L3(0, 0, 64)), dict(os_=L3(0, -8, 128))):
        assert a(**kw) == -2, kw
    for kw in (dict(splits=-1), dict(splits=257), dict(wg_rows=32), dict(wg_rows=-16)):
        assert a(**kw) == -3, kw
    for kw in (dict(q=A + 2), dict(o=A + 8), dict(lse=A + 2), dict(lens=A + 1), dict(q_lens=A + 2), dict(ws=A + 8, wsb=1 << 20), dict(qs=L3(0, 4, 128))):
        assert a(**kw) == -4, kw
    for scale in (0.0, -1.0, math.nan, math.inf, 2e38):
        assert a(scale=scale) == -5


def test_workspace_sizes(lib):
    need = lib.attn_kv_fp8_workspace_bytes
    for kw in ((0, 8, 2, 1, 100, 128, 0, 0), (1, 8, 3, 1, 100, 128, 0, 0), (1, 8, 2, 0, 100, 128, 0, 0), (1, 8, 2, 1, 0, 128, 0, 0), (1, 8, 2, 1, 100, 96, 0, 0),
               (1, 8, 2, 1, 100, 128, -1, 0), (1, 8, 2, 1, 100, 128, 0, -1), (1, 8, 2, 1, 1 << 30, 128, 0, 0)):
        assert need(*kw) == 0, kw
    assert need(1, 8, 2, 1, 64, 128, 0, 0) == 0                     # one tile: nothing to cut
    long = need(1, 8, 2, 1, 100000, 128, 0, 0)
    assert long > 0 and long % (4 * 8 * 130) == 0
    assert need(1, 8, 2, 1, 100000, 128, 64, 4) < long              # a window: few keys to cut


def test_rope_refuses(lib):
    freq = A
    g = L3(4 * 8 * 128, 8 * 128, 128)

    def r(q=A, qo=A, k=A, ko=A, B=1, Hq=4, Hk=2, S=8, D=128, R=64, qs=g, qos=g, ks=g, kos=g, pos=A, pitch=8, inv=freq, scale=1.0):
        return lib.rope_bf16(q, qo, k, ko, B, Hq, Hk, S, D, R, qs, qos, ks, kos, pos, pitch, inv, 0, 0, scale, None)

    for kw in (dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(qs=None), dict(qos=None), dict(ks=None), dict(kos=None), dict(pos=None), dict(inv=None), dict(Hk=0)):
        assert r(**kw) == -1, kw
    for kw in (dict(B=0), dict(Hq=0), dict(S=-1), dict(Hk=-1, k=None, ko=None), dict(D=0), dict(pitch=-1), dict(Hq=65535), dict(B=1 << 14, S=1 << 14),
               dict(qs=L3(0, 0, 64)), dict(kos=L3(-8, 0, 128)), dict(qos=L3(1 << 40, 0, 128))):
        assert r(**kw) == -2, kw
    for kw in (dict(D=124), dict(D=1032, qs=L3(0, 0, 2048)), dict(R=0), dict(R=63), dict(R=130)):
        assert r(**kw) == -3, kw
    for kw in (dict(q=A + 2), dict(ko=A + 8), dict(pos=A + 2), dict(inv=A + 4), dict(qs=L3(4, 0, 128)), dict(ks=L3(0, 0, 132))):
        assert r(**kw) == -4, kw
    for scale in (math.nan, math.inf, -math.inf):
        assert r(scale=scale) == -5


def test_frequencies_refuse_and_answer(lib):
    out = (ctypes.c_double * 4)()
    f = lambda R=8, base=10000.0, factor=1.0, length=0, slow=1.0, fast=32.0, to=out: lib.rope_frequencies(R, base, factor, length, slow, fast, to)
    assert f(to=None) == -1 and f(R=7) == -2 and f(R=0) == -2 and f(length=-1) == -2
    for kw in (dict(base=1.0), dict(base=math.nan), dict(base=math.inf), dict(factor=0.5), dict(factor=math.inf), dict(length=10, slow=-1.0), dict(length=10, fast=1.0),
               dict(length=10, fast=math.inf)):
        assert f(**kw) == -5, kw
    assert f() == 0 and np.allclose(list(out), 10000.0 ** (-np.arange(4) / 4), rtol=1e-15)
    assert f(factor=4.0) == 0 and np.allclose(list(out), 10000.0 ** (-np.arange(4) / 4) / 4, rtol=1e-15)


def test_python_refuses_what_is_not_a_cache_on_the_gpu():
    torch = pytest.importorskip("torch")
    c = binding.kv_fp8_cache(4, 2, 16, 64, device="cpu")
    table, lens = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    x = torch.zeros(1, 2, 1, 64, dtype=torch.bfloat16)
    for call in (lambda: binding.kv_fp8_write(c, x, x, table, lens), lambda: binding.kv_fp8_read(c, table, lens, 4), lambda: binding.attn_kv_fp8(x, c, table, lens),
                 lambda: binding.rope_bf16(x, lens, torch.ones(32, dtype=torch.float64))):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    with pytest.raises(ValueError):
        binding.rope_frequencies(7, device="cpu")
    with pytest.raises(binding.AttnError):
        binding.rope_frequencies(8, factor=0.5, device="cpu")
    assert binding.rope_frequencies(8, device="cpu").shape == (4,)
