"""Norms, feed-forward block and log probabilities as far as they can be checked without a GPU: refusals, the sizes of workspaces, how products are
cut, and arguments of the binding.  The entry points' host code is built by the host compiler with launchers that only count."""
import ctypes
import math
import os
import shutil
import subprocess
import tempfile

import pytest
import torch

from paper_2209_06979_amd import binding as mc

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2209_06979_amd", "csrc")
STUBS = r"""
#include "layer.h"
static int launches = 0;
extern "C" int host_launches() { const int n = launches; launches = 0; return n; }
bool hip_ok(hipError_t e, const char *) { return e == hipSuccess; }
void note_detail(const char *, ...) {}
hipError_t launch_block_norm(const NormArgs &, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_block_norm_backward(NormArgs, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_token_logprobs(const LogprobArgs &, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_token_logprobs_backward(const LogprobArgs &, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_gated_product(const ProductArgs &, mc_type, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_product(const ProductArgs &, ProductPlan, bool, mc_type, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_few_rows(const FewRowsArgs &, mc_type, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_gated_grad(const GatedGradArgs &, mc_type, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_pad_rows(const PadRowsArgs &, mc_type, hipStream_t) { return ++launches, hipSuccess; }
extern "C" void host_plan(int64_t m, int64_t n, int64_t k, int batch, int type, int gated, int *out)
{
    const ProductPlan p = product_plan(m, n, k, batch, (mc_type)type, gated != 0);
    out[0] = p.tile;
    out[1] = p.splits;
}
extern "C" void host_pieces(int64_t rows, int vocab, int type, int *out)
{
    const LogprobPlan p = logprob_plan(rows, vocab, type);
    out[0] = p.pieces;
    out[1] = p.piece_vectors;
}
extern "C" int host_norm_workgroups(int64_t rows, int dim) { return norm_workgroups(rows, dim); }
"""
NAMES = ("mc_block_norm", "mc_block_norm_backward", "mc_block_norm_backward_workspace", "mc_gated_ffn", "mc_gated_ffn_workspace", "mc_gated_ffn_backward",
         "mc_gated_ffn_backward_workspace", "mc_token_logprobs", "mc_token_logprobs_workspace", "mc_token_logprobs_backward")


@pytest.fixture(scope="module")
def lib():
    cxx = shutil.which("clang++") or "/opt/rocm/lib/llvm/bin/clang++"
    with tempfile.TemporaryDirectory() as d:
        with open(os.path.join(d, "stubs.cpp"), "w") as f:
            f.write(STUBS)
        out = os.path.join(d, "liblayer.so")
        subprocess.run([cxx, "-std=c++17", "-O1", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", f"-I{CSRC}", "-x", "c++",
                        os.path.join(CSRC, "layer_api.hip"), os.path.join(d, "stubs.cpp"), "-o", out], check=True)
        L = ctypes.CDLL(out)
        for n in NAMES:
            getattr(L, n).argtypes, getattr(L, n).restype = getattr(mc.lib, n).argtypes, getattr(mc.lib, n).restype
        L.host_plan.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int] * 3 + [ctypes.POINTER(ctypes.c_int)]
        L.host_pieces.argtypes = [ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_int)]
        L.host_norm_workgroups.argtypes = [ctypes.c_int64, ctypes.c_int]
        yield L


AT = 1 << 20                                    # an aligned address that nobody reads
PLENTY = 1 << 40


def _norm_args(**kw):
    a = dict(rows=6, dim=64, type=1, residual_type=1, param_type=1, pre=1, post=1, x_dev=AT, x_stride=64, residual_dev=AT, residual_stride=64, weight_dev=AT, bias_dev=AT,
             post_weight_dev=AT, post_bias_dev=AT, gate_dev=AT, gate_groups=3, gate_stride=64, branch_scale=1.0, residual_scale=1.0, eps=1e-6)
    return mc.BlockNormArgs(**{**a, **kw})


def _norm(L, y=AT, ys=64, n=AT, ns=64, **kw):
    return L.mc_block_norm(_norm_args(**kw), y, ys, n, ns, None)


def _norm_back(L, dy=AT, dys=64, dn=AT, dns=64, ws=AT, bytes=PLENTY, grads=None, **kw):
    g = mc.BlockNormGrads(**{**dict(dx_dev=AT, dx_stride=64, dresidual_dev=AT, dresidual_stride=64, dgate_dev=AT, dgate_stride=64, dweight_dev=AT, dbias_dev=AT,
                                    dpost_weight_dev=AT, dpost_bias_dev=AT), **(grads or {})})
    return L.mc_block_norm_backward(_norm_args(**kw), dy, dys, dn, dns, g, ws, bytes, None)


def _ffn_args(**kw):
    a = dict(rows=100, dim=64, hidden=48, type=1, activation=0, x_dev=AT, x_stride=64, gate_dev=AT, gate_stride=64, up_dev=AT, up_stride=64)
    return mc.GatedFfnArgs(**{**a, **kw})


def _ffn(L, h=AT, hs=48, g=None, u=None, ss=48, ws=None, bytes=0, **kw):
    return L.mc_gated_ffn(_ffn_args(**kw), h, hs, g, u, ss, ws, bytes, None)


def _ffn_back(L, dh=AT, dhs=48, g=AT, u=AT, ss=48, dx=AT, dxs=64, dg=AT, dgs=64, du=AT, dus=64, ws=AT, bytes=PLENTY, **kw):
    return L.mc_gated_ffn_backward(_ffn_args(**kw), dh, dhs, g, u, ss, dx, dxs, dg, dgs, du, dus, ws, bytes, None)


def _logp(L, x=AT, type=1, rows=4, vocab=100, stride=100, tokens=AT, scale=1.0, top=2, lp=AT, h=AT, tl=AT, tt=AT, sums=None, ws=None, bytes=0):
    return L.mc_token_logprobs(x, type, rows, vocab, stride, tokens, scale, top, lp, h, tl, tt, sums, ws, bytes, None)


def _logp_back(L, x=AT, type=1, rows=4, vocab=100, stride=100, tokens=AT, scale=1.0, top=2, tt=AT, sums=AT, h=AT, dl=AT, dh=AT, dt=AT, d=AT, ds=100):
    return L.mc_token_logprobs_backward(x, type, rows, vocab, stride, tokens, scale, top, tt, sums, h, dl, dh, dt, d, ds, None)


E, U, A, M = mc.MC_EINVAL, mc.MC_EUNSUPPORTED, mc.MC_EALIGN, mc.MC_ENOMEM
BOTH_NORMS = [
    (dict(type=3), U), (dict(type=1, residual_type=2), U), (dict(type=2, param_type=1), U), (dict(type=0, param_type=1), U), (dict(pre=3), U), (dict(post=-1), U), (dict(rows=-1), E),
    (dict(rows=1 << 31), E), (dict(dim=0), E), (dict(dim=16385, x_stride=20000, residual_stride=20000, gate_stride=20000), E), (dict(eps=-1.0), E), (dict(eps=math.nan), E),
    (dict(eps=math.inf), E), (dict(branch_scale=math.inf), E), (dict(residual_scale=math.nan), E), (dict(post=0), E), (dict(gate_groups=4), E), (dict(gate_groups=0), E),
    (dict(gate_dev=None), E), (dict(x_dev=None), E), (dict(x_dev=AT + 1), E), (dict(x_stride=63), E), (dict(residual_stride=0), E), (dict(gate_stride=32), E), (dict(weight_dev=AT + 1), E),
    (dict(rows=0, gate_groups=65533), E),
]
REFUSED = [(c, kw, s) for kw, s in BOTH_NORMS for c in (_norm, _norm_back)] + [
    (_norm, dict(pre=0, weight_dev=None, bias_dev=None), E), (_norm, dict(n=None), E), (_norm, dict(y=None, n=None, pre=0, weight_dev=None, bias_dev=None), E), (_norm, dict(ys=63), E),
    (_norm, dict(ns=10), E), (_norm, dict(y=AT + 1), E), (_norm, dict(pre=0, weight_dev=None, bias_dev=AT), E),
    (_norm_back, dict(pre=0, weight_dev=None, bias_dev=None, grads=dict(dweight_dev=None, dbias_dev=None)), E), (_norm_back, dict(weight_dev=None), E),
    (_norm_back, dict(residual_dev=None), E), (_norm_back, dict(gate_dev=None, gate_groups=0), E), (_norm_back, dict(post_bias_dev=None), E), (_norm_back, dict(dys=1), E),
    (_norm_back, dict(dn=AT + 1), E), (_norm_back, dict(grads=dict(dx_stride=2)), E), (_norm_back, dict(grads=dict(dgate_dev=AT + 1)), E),
    (_norm_back, dict(ws=None), M), (_norm_back, dict(bytes=6 * 6 * 64 * 4 - 1), M), (_norm_back, dict(ws=AT + 16), A),
] + [(c, kw, s) for c in (_ffn, _ffn_back) for kw, s in [
    (dict(type=7), U), (dict(activation=5), U), (dict(activation=-1), U), (dict(rows=-1), E), (dict(rows=(1 << 21) + 1), E), (dict(dim=0), E), (dict(hidden=0), E),
    (dict(hidden=(1 << 20) + 1), E), (dict(rows=1 << 21, hidden=1 << 14, hs=1 << 14) if c is _ffn else dict(rows=1 << 21, hidden=1 << 14), E),
    (dict(dim=1 << 17, hidden=1 << 18, x_stride=1 << 17, gate_stride=1 << 17, up_stride=1 << 17), E), (dict(x_dev=None), E), (dict(gate_dev=None), E), (dict(up_dev=AT + 1), E),
    (dict(x_stride=63), E), (dict(gate_stride=0), E), (dict(up_stride=1 << 23), E)]] + [
    (_ffn, dict(h=None), E), (_ffn, dict(hs=47), E), (_ffn, dict(g=AT), E), (_ffn, dict(u=AT), E), (_ffn, dict(g=AT, u=AT + 2), E), (_ffn, dict(g=AT, u=AT, ss=40), E),
    (_ffn, dict(x_dev=AT + 8), M), (_ffn, dict(dim=63), M), (_ffn, dict(gate_stride=65, ws=AT, bytes=48 * 128 - 1), M), (_ffn, dict(gate_stride=65, ws=AT + 128, bytes=PLENTY), A),
    (_ffn_back, dict(dh=None), E), (_ffn_back, dict(g=None), E), (_ffn_back, dict(u=AT + 2), E), (_ffn_back, dict(ss=47), E), (_ffn_back, dict(dxs=63), E), (_ffn_back, dict(du=AT + 1), E),
    (_ffn_back, dict(ws=None), M), (_ffn_back, dict(bytes=100), M), (_ffn_back, dict(ws=AT + 64), A),
] + [(c, kw, s) for c in (_logp, _logp_back) for kw, s in [
    (dict(type=-1), U), (dict(rows=-1), E), (dict(vocab=0), E), (dict(vocab=(1 << 30) + 1, stride=1 << 31), E), (dict(stride=99), E), (dict(scale=0.0), E), (dict(scale=-1.0), E),
    (dict(scale=math.nan), E), (dict(scale=math.inf), E), (dict(scale=3e38), E), (dict(top=-1), E), (dict(top=65), E), (dict(vocab=1, top=2), E), (dict(x=None), E), (dict(x=AT + 1), E),
    (dict(tokens=None), E), (dict(rows=1 << 23, vocab=5000, stride=5000), E), (dict(h=None), E), (dict(tt=None), E)]] + [
    (_logp, dict(lp=None), E), (_logp, dict(tl=None), E), (_logp, dict(vocab=100000, stride=100000), M), (_logp, dict(vocab=100000, stride=100000, ws=AT + 8, bytes=PLENTY), A),
    (_logp_back, dict(sums=None), E), (_logp_back, dict(d=None), E), (_logp_back, dict(ds=99), E),
]


@pytest.mark.parametrize("call,kw,status", REFUSED)
def test_refusals(lib, call, kw, status):
    assert call(lib, **kw) == status
    assert lib.host_launches() == 0


def test_calls_that_launch_and_calls_that_have_nothing_to_do(lib):
    for call, launches in ((_norm, 1), (_norm_back, 1), (_ffn, 1), (_ffn_back, 3), (_logp, 1), (_logp_back, 1)):
        assert call(lib) == 0 and lib.host_launches() == launches, call
    assert _norm(lib, rows=0, x_dev=None, y=None, n=None, gate_groups=1) == 0 and lib.host_launches() == 0
    assert _norm(lib, y=None) == 0 and lib.host_launches() == 1
    assert _norm_back(lib, dy=None, dn=None, grads=dict(dx_dev=None)) == 0 and lib.host_launches() == 1
    assert _norm_back(lib, rows=0, x_dev=None, ws=None, bytes=0) == 0 and lib.host_launches() == 1          # sums over no rows
    assert _ffn(lib, rows=0, x_dev=None, h=None) == 0 and lib.host_launches() == 0
    assert _ffn(lib, rows=3, dim=63, gate_stride=65) == 0 and lib.host_launches() == 1                    # a few rows: no copies
    assert _ffn(lib, rows=200, dim=63, ws=AT, bytes=PLENTY) == 0 and lib.host_launches() == 2              # copies, in one launch
    assert _ffn_back(lib, dg=None, du=None) == 0 and lib.host_launches() == 2
    assert _ffn_back(lib, dx=None, dg=None) == 0 and lib.host_launches() == 2
    assert _ffn_back(lib, rows=0, x_dev=None, dh=None, g=None, u=None) == 0 and lib.host_launches() == 1    # weights' gradients of no rows
    assert _ffn_back(lib, dim=63, dxs=63, dgs=63, dus=63, x_stride=63, gate_stride=63, up_stride=63) == 0 and lib.host_launches() == 4
    assert _logp(lib, rows=0, x=None, tokens=None) == 0 and lib.host_launches() == 0
    assert _logp(lib, top=0, tl=None, tt=None) == 0 and lib.host_launches() == 1
    assert _logp_back(lib, dl=None, dh=None, dt=None, tt=None) == 0 and lib.host_launches() == 1


def test_workspaces(lib):
    """No workspace where none is used; enough for what is."""
    assert lib.mc_gated_ffn_workspace(_ffn_args()) == 0
    assert lib.mc_gated_ffn_workspace(_ffn_args(rows=0)) == 0
    assert lib.mc_gated_ffn_workspace(_ffn_args(type=9)) == 0
    assert lib.mc_gated_ffn_workspace(_ffn_args(rows=200, dim=63)) >= (200 + 2 * 48) * 64 * 2
    assert lib.mc_gated_ffn_workspace(_ffn_args(rows=64, dim=63)) == 0
    for rows in (1, 50, 3000):
        assert lib.mc_gated_ffn_backward_workspace(_ffn_args(rows=rows)) >= 2 * rows * 48 * 2
    assert lib.mc_block_norm_backward_workspace(0, 64) == 0
    for rows, dim in ((1, 1), (100, 512), (5000, 1000), (5000, 2048), (5000, 4096), (5000, 4097), (5000, 16384)):
        groups = lib.host_norm_workgroups(rows, dim)
        assert 1 <= groups <= rows
        assert lib.mc_block_norm_backward_workspace(rows, dim) >= 4 * (groups * 6 * dim + (8 * rows if dim > 4096 else 0))
    assert lib.mc_token_logprobs_workspace(2000, 100000, 1, 20) == 0
    assert lib.mc_token_logprobs_workspace(1, 100, 1, 101) == 0


def test_pieces_of_logits_cover_a_row_once(lib):
    out = (ctypes.c_int * 2)()
    for rows in (1, 2, 16, 100, 1000, 1024, 5000):
        for vocab in (1, 7, 8, 100, 8191, 8192, 8193, 32000, 50257, 131072, 262145, 1 << 30):
            for type in (0, 1, 2):
                lib.host_pieces(rows, vocab, type, out)
                vectors = -(-vocab // (4 if type == 0 else 8))
                assert 1 <= out[0] <= 64 and out[0] * out[1] >= vectors > (out[0] - 1) * out[1]
                size = lib.mc_token_logprobs_workspace(rows, vocab, type, 1)
                assert size == (0 if out[0] == 1 or rows > 8388607 // -(-vocab // 4096) else rows * out[0] * (4 + 2) * 4)


def test_products_are_cut_within_their_steps(lib):
    """Every piece along k has steps of its own, and no launch has more threads than a grid counts."""
    out = (ctypes.c_int * 2)()
    tiles = {256: (256, 256), 128: (128, 128), 96: (128, 64), 64: (64, 64), 32: (32, 64)}
    for m in (1, 65, 777, 8192, 1 << 21):
        for n in (1, 48, 1001, 4096, 8192):
            for k in (0, 1, 64, 5462, 22016, 1 << 20):
                for type in (0, 2):
                    for gated, batch in ((1, 1), (0, 1), (0, 2)):
                        lib.host_plan(m, n, k, batch, type, gated, out)
                        tile, splits = out
                        steps = -(-k * (4 if type == 0 else 2) // 128)
                        assert tile in tiles and 1 <= splits <= max(1, steps) and (not gated or splits == 1)
                        count = -(-m // tiles[tile][0]) * -(-n * (2 if gated else 1) // tiles[tile][1]) * batch * splits
                        assert count * 512 < 1 << 32


def test_arguments_of_the_binding():
    x, tokens = torch.zeros((4, 8)), torch.zeros(4, dtype=torch.long)
    for call in (mc.block_norm, mc.gated_ffn, mc.token_logprobs):
        with pytest.raises(TypeError):
            call()
        with pytest.raises(TypeError):
            call(*([None] * 20))
        with pytest.raises(TypeError):
            call(x, nothing=1)
        with pytest.raises(TypeError):
            call("x", "y", "z")
    for call in (lambda: mc.block_norm(x), lambda: mc.gated_ffn(x, x, x), lambda: mc.token_logprobs(x, tokens)):     # not on the device
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: mc.block_norm(x, pre="batch"), lambda: mc.block_norm(x, post=1), lambda: mc.gated_ffn(x, x, x, "swish"), lambda: mc.gated_ffn(x, x, x, activation=None)):
        with pytest.raises(KeyError):
            call()
