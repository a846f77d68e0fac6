"""The operators around decoding as far as they can be checked without a GPU: refusals, the sizes of workspaces, frequencies, and arguments
of the binding.  The entry points' host code is built by the host compiler with launchers that only count."""
import ctypes
import math
import os
import shutil
import subprocess
import tempfile

import numpy as np
import pytest
import torch

from paper_2209_06979_amd import binding as mc

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2209_06979_amd", "csrc")
STUBS = r"""
#include "decode.h"
static int launches = 0;
extern "C" int host_launches() { const int n = launches; launches = 0; return n; }
extern "C" hipError_t hipGetDevice(int *d) { return *d = 0, hipSuccess; }
bool hip_ok(hipError_t e, const char *) { return e == hipSuccess; }
void note_detail(const char *, ...) {}
hipError_t launch_rope(const RopeArgs &, mc_type, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_cache_write(const CacheArgs &, mc_type, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_cache_read(const CacheArgs &, mc_type, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_cache_attention(const CacheAttnArgs &, mc_type, int, int, hipStream_t) { return ++launches, hipSuccess; }
"""
NAMES = ("mc_rope", "mc_cache_write", "mc_cache_read", "mc_cache_attention", "mc_cache_attention_workspace")


@pytest.fixture(scope="module")
def lib():
    cxx = shutil.which("clang++") or "/opt/rocm/lib/llvm/bin/clang++"
    with tempfile.TemporaryDirectory() as d:
        with open(os.path.join(d, "stubs.cpp"), "w") as f:
            f.write(STUBS)
        out = os.path.join(d, "libdecode.so")
        subprocess.run([cxx, "-std=c++17", "-O1", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", f"-I{CSRC}", "-x", "c++",
                        os.path.join(CSRC, "decode_api.hip"), os.path.join(d, "stubs.cpp"), "-o", out], check=True)
        L = ctypes.CDLL(out)
        for n in NAMES:
            getattr(L, n).argtypes = getattr(mc.lib, n).argtypes
        L.mc_cache_attention_workspace.restype = ctypes.c_size_t
        yield L


AT = 1 << 20                                    # an aligned address that nobody reads


def _cache(**kw):
    return mc.CacheDescription(**{**dict(k_codes=AT, v_codes=AT, k_scales=AT, v_scales=AT, pages=10, page_size=16, kv_heads=2, dk=64, bits=8, device=0), **kw})


def _rope(L, type=0, tokens=5, heads=2, dim=64, rot=64, magnitude=1.0, x=AT, y=AT, positions=AT, freq=AT):
    return L.mc_rope(x, type, tokens, heads, dim, heads * dim, dim, positions, freq, rot, 0, magnitude, 0, y, heads * dim, dim, None)


def _write(L, cache=None, type=0, tokens=5, ts=128, hs=64, k=AT, v=AT, slots=AT, rope=None):
    return L.mc_cache_write(cache or _cache(), k, v, type, tokens, ts, hs, ts, hs, slots, rope, None)


def _read(L, cache=None, type=0, tokens=5, ts=128, hs=64, k=AT, v=AT, slots=AT):
    return L.mc_cache_read(cache or _cache(), slots, tokens, type, k, v, ts, hs, ts, hs, None)


def _attend(L, cache=None, type=0, total=3, heads=4, qts=256, qhs=64, q=AT, starts=AT, batch=3, max_new=1, lengths=AT, table=AT, stride=4, pages=4,
            tree=None, scale=0.1, o=AT, ws=None, ws_bytes=0):
    return L.mc_cache_attention(cache or _cache(), q, type, total, heads, qts, qhs, starts, batch, max_new, lengths, table, stride, pages, tree, scale, o, qts, qhs,
                                ws, ws_bytes, None)


REFUSED = [
    (_rope, dict(type=3), mc.MC_EUNSUPPORTED), (_rope, dict(tokens=-1), mc.MC_EINVAL), (_rope, dict(heads=0), mc.MC_EINVAL), (_rope, dict(rot=65), mc.MC_EINVAL),
    (_rope, dict(rot=66), mc.MC_EINVAL), (_rope, dict(rot=-2), mc.MC_EINVAL), (_rope, dict(dim=0, rot=0), mc.MC_EINVAL), (_rope, dict(magnitude=math.inf), mc.MC_EINVAL),
    (_rope, dict(magnitude=math.nan), mc.MC_EINVAL), (_rope, dict(x=None), mc.MC_EINVAL), (_rope, dict(y=None), mc.MC_EINVAL), (_rope, dict(positions=None), mc.MC_EINVAL),
    (_rope, dict(freq=None), mc.MC_EINVAL), (_rope, dict(tokens=1 << 30, heads=1000), mc.MC_EINVAL),
    (_write, dict(type=-1), mc.MC_EUNSUPPORTED), (_write, dict(tokens=-1), mc.MC_EINVAL), (_write, dict(k=None), mc.MC_EINVAL), (_write, dict(v=None), mc.MC_EINVAL),
    (_write, dict(slots=None), mc.MC_EINVAL), (_write, dict(k=AT + 8), mc.MC_EALIGN), (_write, dict(v=AT + 2), mc.MC_EALIGN), (_write, dict(type=1, hs=66), mc.MC_EALIGN),
    (_write, dict(type=2, ts=132), mc.MC_EALIGN), (_write, dict(tokens=1 << 30), mc.MC_EINVAL),
    (_write, dict(rope=mc.RopeKeys(AT, AT, 66, 0, 1.0)), mc.MC_EINVAL), (_write, dict(rope=mc.RopeKeys(AT, AT, 7, 0, 1.0)), mc.MC_EINVAL),
    (_write, dict(rope=mc.RopeKeys(None, AT, 8, 0, 1.0)), mc.MC_EINVAL), (_write, dict(rope=mc.RopeKeys(AT, None, 8, 0, 1.0)), mc.MC_EINVAL),
    (_write, dict(rope=mc.RopeKeys(AT, AT, 8, 0, math.inf)), mc.MC_EINVAL),
    (_read, dict(type=5), mc.MC_EUNSUPPORTED), (_read, dict(tokens=-1), mc.MC_EINVAL), (_read, dict(slots=None), mc.MC_EINVAL), (_read, dict(k=None), mc.MC_EINVAL),
    (_read, dict(k=AT + 4), mc.MC_EALIGN), (_read, dict(ts=130), mc.MC_EALIGN), (_read, dict(tokens=1 << 30), mc.MC_EINVAL),
    (_attend, dict(type=9), mc.MC_EUNSUPPORTED), (_attend, dict(heads=3), mc.MC_EINVAL), (_attend, dict(heads=0), mc.MC_EINVAL), (_attend, dict(batch=-1), mc.MC_EINVAL),
    (_attend, dict(batch=65536), mc.MC_EINVAL), (_attend, dict(max_new=-1), mc.MC_EINVAL), (_attend, dict(pages=-1), mc.MC_EINVAL), (_attend, dict(stride=3), mc.MC_EINVAL),
    (_attend, dict(max_new=65, tree=AT), mc.MC_EINVAL), (_attend, dict(scale=math.inf), mc.MC_EINVAL), (_attend, dict(scale=math.nan), mc.MC_EINVAL),
    (_attend, dict(starts=None, total=4), mc.MC_EINVAL), (_attend, dict(q=None), mc.MC_EINVAL), (_attend, dict(o=None), mc.MC_EINVAL), (_attend, dict(lengths=None), mc.MC_EINVAL),
    (_attend, dict(table=None), mc.MC_EINVAL), (_attend, dict(q=AT + 8), mc.MC_EALIGN), (_attend, dict(o=AT + 4), mc.MC_EALIGN), (_attend, dict(type=1, qhs=68), mc.MC_EALIGN),
    (_attend, dict(max_new=1 << 20, heads=1000), mc.MC_EINVAL), (_attend, dict(pages=1 << 27, stride=1 << 27), mc.MC_EINVAL),
    (_attend, dict(pages=1 << 20, stride=1 << 20, batch=65535), mc.MC_EINVAL), (_attend, dict(pages=(1 << 26) + 1, stride=1 << 27), mc.MC_EINVAL),
    (_attend, dict(cache=_cache(kv_heads=65535), heads=65535, batch=500), mc.MC_EINVAL), (_attend, dict(batch=65535, max_new=65535, total=65535), mc.MC_EINVAL),
    (_attend, dict(pages=4000, stride=4000), mc.MC_ENOMEM), (_attend, dict(pages=4000, stride=4000, ws=AT, ws_bytes=1024), mc.MC_ENOMEM),
    (_attend, dict(pages=4000, stride=4000, ws=AT + 16, ws_bytes=1 << 40), mc.MC_EALIGN),
]
BAD_CACHES = [
    (dict(k_codes=None), mc.MC_EINVAL), (dict(v_scales=None), mc.MC_EINVAL), (dict(bits=16), mc.MC_EUNSUPPORTED), (dict(pages=0), mc.MC_EINVAL), (dict(page_size=8), mc.MC_EINVAL),
    (dict(page_size=48), mc.MC_EINVAL), (dict(page_size=8192), mc.MC_EINVAL), (dict(kv_heads=0), mc.MC_EINVAL), (dict(dk=0), mc.MC_EINVAL), (dict(dk=72), mc.MC_EINVAL),
    (dict(dk=272), mc.MC_EINVAL), (dict(dk=48, bits=4), mc.MC_EINVAL), (dict(v_codes=AT + 8), mc.MC_EALIGN), (dict(k_scales=AT + 4), mc.MC_EALIGN), (dict(device=1), mc.MC_EINVAL),
]


@pytest.mark.parametrize("call,kw,status", REFUSED)
def test_refusals(lib, call, kw, status):
    assert call(lib, **kw) == status
    assert lib.host_launches() == 0


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_caches_that_are_refused(lib, kw, status):
    for call in (_write, _read, _attend):
        assert call(lib, cache=_cache(**kw)) == status
    assert lib.host_launches() == 0


def test_calls_that_launch_and_calls_that_have_nothing_to_do(lib):
    for call in (_rope, _write, _read, _attend):
        assert call(lib) == 0
        assert lib.host_launches() == 1
    for call, kw in ((_rope, dict(tokens=0, x=None, y=None)), (_write, dict(tokens=0, k=None)), (_read, dict(tokens=0, k=None)), (_attend, dict(total=0, q=None)),
                     (_attend, dict(batch=0, total=0, starts=None, lengths=None)), (_attend, dict(max_new=0, total=0, q=None))):
        assert call(lib, **kw) == 0
        assert lib.host_launches() == 0
    assert _attend(lib, starts=None) == 0 and _attend(lib, pages=0, table=None) == 0 and _attend(lib, tree=AT, max_new=64, total=70) == 0


def test_workspace(lib):
    """None where no sequence can be cut; else it grows with what can be, and not beyond twice the pieces asked for."""
    ask = lambda **kw: lib.mc_cache_attention_workspace(_cache(**{k: kw.pop(k) for k in ("dk", "kv_heads", "page_size") if k in kw}), kw.get("heads", 4), kw.get("batch", 8),
                                                        kw.get("max_new", 1), kw.get("pages", 4000))
    assert ask(pages=16) == 0 and ask(pages=0) == 0 and ask(batch=0) == 0 and ask(max_new=0) == 0 and ask(heads=3) == 0
    assert ask() > 0 and ask() % 4 == 0 and ask(batch=60000) >= ask() and ask(batch=60000) <= 2 * 1024 * 16 * (64 + 2) * 4
    assert ask(kv_heads=65535, heads=65535, batch=500) == 0 and ask(pages=(1 << 26) + 1) == 0 and ask(pages=1 << 26) > 0   # (sizes that are refused; the longest)
    need = ask(dk=64)
    assert _attend(lib, batch=8, total=8, pages=4000, stride=4000, ws=AT, ws_bytes=need) == 0
    assert _attend(lib, batch=8, total=8, pages=4000, stride=4000, ws=AT, ws_bytes=need - 4) == mc.MC_ENOMEM


@pytest.mark.parametrize("rot", [2, 8, 64, 128, 34])
def test_frequencies(rot):
    j = np.arange(0, rot, 2)
    f = 10000.0 ** (-j / rot)
    close = lambda a, b: np.allclose(a, b, rtol=1e-14, atol=0)
    assert close(mc.rope_frequencies(rot)[0], f) and mc.rope_frequencies(rot)[1] == 1
    assert close(mc.rope_frequencies(rot, 500000.0)[0], 500000.0 ** (-j / rot))
    assert close(mc.rope_frequencies(rot, scaling="linear", factor=4.0)[0], f / 4)
    if rot >= 4:
        g = mc.rope_frequencies(rot, scaling="base", factor=8.0)[0]
        assert g[0] == 1 and math.isclose(g[-1], f[-1] / 8, rel_tol=1e-13)
    g, m = mc.rope_frequencies(rot, scaling="parts", factor=16.0, original=8192)
    turns = 8192 * f / (2 * math.pi)
    assert close(g[turns >= 32], f[turns >= 32]) and close(g[turns <= 1], f[turns <= 1] / 16) and math.isclose(m, 0.1 * math.log(16) + 1)
    assert (g <= f * (1 + 1e-15)).all() and (g >= f / 16 * (1 - 1e-15)).all()


@pytest.mark.parametrize("kw", [dict(rot=0), dict(rot=7), dict(rot=-4), dict(rot=8, base=0.0), dict(rot=8, base=math.inf), dict(rot=8, scaling="linear", factor=0.5),
                                dict(rot=2, scaling="base", factor=2.0), dict(rot=8, scaling="parts", original=0.0), dict(rot=8, scaling="parts", low=4.0, high=4.0),
                                dict(rot=8, scaling="parts", low=-1.0)])
def test_frequencies_that_are_refused(kw):
    with pytest.raises(mc.MagicubeError) as e:
        mc.rope_frequencies(**kw)
    assert e.value.status == mc.MC_EINVAL


cpu = torch.zeros((4, 2, 64))


@pytest.mark.parametrize("call", [mc.rope, mc.cache_write, mc.cache_read, mc.cache_attention])
def test_missing_surplus_and_unknown_arguments(call):
    with pytest.raises(TypeError):
        call()
    with pytest.raises(TypeError):
        call(*([None] * 20))
    with pytest.raises(TypeError):
        call(cpu, cpu, cpu, cpu, nothing=1)


def test_wrong_kinds_of_arguments():
    with pytest.raises(AssertionError):
        mc.rope(cpu, cpu, cpu)                               # not on the device
    with pytest.raises(TypeError):
        mc.rope(cpu, "positions", cpu)
    with pytest.raises(TypeError):
        mc.cache_read(cpu, cpu)
    with pytest.raises(TypeError):
        mc.cache_attention(cpu, cpu, cpu, cpu)
    with pytest.raises(AssertionError):
        mc.KVCache(cpu, cpu, cpu, cpu)
    with pytest.raises(mc.MagicubeError):
        mc.KVCache(cpu, cpu, cpu, cpu, bits=2)
    with pytest.raises(KeyError):
        mc.rope_frequencies(8, scaling="other")
