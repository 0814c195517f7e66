"""The entry points of the dense half in 8-bit integers on a host without a GPU: they refuse bad arguments before any
launch, and their checks run under the sanitizers.  No call here reaches a kernel."""
import os
import shutil
import subprocess

import pytest
import torch

import paper_2606_21712_amd as moe

INVALID, UNSUPPORTED, WS_SMALL = 1, 2, 3
P = 0x10000          # a 16-byte aligned address that is never dereferenced
S = None
NAN, INF = float("nan"), float("inf")
HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2606_21712_amd", "csrc")


@pytest.fixture(scope="module")
def L():
    return moe.lib()


@pytest.fixture
def cus():
    moe.set_cu_budget(256)
    yield
    moe.set_cu_budget(0)


def join(L, x=P, xs=256, dt=1, y=P, ys=256, post=1, wpost=P, gate=P, gs=256, kind=3, sig=0, alpha=1.0, wpre=P, off=0.0,
         eps=1e-6, T=3, H=256, out=P, os_=256, codes=1, z=P, zs=P):
    return L.moe_norm_join(x, xs, dt, y, ys, post, wpost, gate, gs, kind, sig, alpha, wpre, off, eps, T, H, out, os_, codes,
                           z, zs, S)


def quantize(L, src=P, stride=256, rows=4, K=256, codes=P, scales=P):
    return L.moe_quantize_int8(src, stride, rows, K, codes, scales, S)


def pack(L, codes=P, rows=4, K=256, out=P):
    return L.moe_pack_int8(codes, rows, K, out, S)


def matmul(L, x=P, xs=P, w=P, ws_=P, bias=None, T=3, N=16, K=256, y=P, ws=P, n=1 << 40):
    return L.moe_matmul_int8(x, xs, w, ws_, bias, T, N, K, y, ws, n, S)


def gated(L, x=P, xs=P, wg=P, sg=P, wu=P, su=P, T=3, N=16, K=256, h=P, ws=P, n=1 << 40):
    return L.moe_gated_int8(x, xs, wg, sg, wu, su, T, N, K, h, ws, n, S)


def test_norm_join(L):
    for bad in (dict(H=0), dict(H=-8), dict(H=12), dict(T=-1), dict(post=2), dict(sig=-1), dict(codes=2), dict(kind=4),
                dict(kind=-1), dict(eps=-1e-9), dict(eps=NAN), dict(eps=INF), dict(alpha=NAN), dict(alpha=INF),
                dict(off=NAN), dict(off=-INF), dict(x=None), dict(x=P + 8), dict(xs=255), dict(xs=252), dict(xs=260),
                dict(y=P + 2), dict(ys=250), dict(out=None), dict(out=P + 4), dict(os_=248), dict(wpost=P + 8),
                dict(post=0), dict(gate=None), dict(kind=0), dict(gate=P + 2), dict(gs=0), dict(kind=2, gs=0),
                dict(kind=2, gs=-1), dict(wpre=P + 4), dict(z=P + 8), dict(zs=None), dict(zs=P + 4), dict(codes=0),
                dict(z=None), dict(z=None, wpre=None), dict(z=None, wpre=None, codes=0), dict(dt=0, xs=258),
                dict(dt=0, os_=257),
                # without y: nothing that belongs to it
                dict(y=None), dict(y=None, post=0, wpost=None, gate=None, kind=0),
                dict(y=None, post=0, wpost=None, out=None), dict(y=None, wpost=None, gate=None, kind=0, out=None),
                dict(y=None, post=0, wpost=None, gate=None, kind=0, out=None, z=None, zs=None, wpre=None, codes=0)):
        assert join(L, **bad) == INVALID, bad
        assert b"moe_norm_join" in L.moe_last_error()
    # in place only with the same rows; a column of gates anywhere, but at a whole element
    for bad in (dict(out=P, os_=512), dict(out=P, xs=512, os_=256), dict(kind=2, gate=P + 1)):
        assert join(L, **bad) == INVALID, bad
    for bad in (dict(H=32776, xs=1 << 16), dict(dt=7), dict(T=(1 << 31) + 1)):
        assert join(L, **bad) == UNSUPPORTED, bad
    assert join(L, T=0, x=None, y=None, out=None, z=None, zs=None) == 0


def test_quantize_and_pack(L):
    for bad in (dict(rows=-1), dict(K=0), dict(K=-16), dict(K=24), dict(src=None), dict(src=P + 2), dict(stride=255),
                dict(stride=260), dict(stride=128), dict(codes=None), dict(scales=P + 4)):
        assert quantize(L, **bad) == INVALID, bad
    for bad in (dict(K=131072, stride=1 << 18), dict(rows=(1 << 31) + 1)):
        assert quantize(L, **bad) == UNSUPPORTED, bad
    assert quantize(L, rows=0, src=None, codes=None, scales=None) == 0
    for bad in (dict(rows=-1), dict(K=8), dict(codes=None), dict(out=P + 8)):
        assert pack(L, **bad) == INVALID, bad
    for bad in (dict(rows=(1 << 24) + 1), dict(rows=1 << 24, K=131056)):
        assert pack(L, **bad) == UNSUPPORTED, bad
    assert pack(L, rows=0, codes=None, out=None) == 0


@pytest.mark.parametrize("rows,K,n", [(16, 64, 2048), (1, 16, 2048), (17, 144, 32 * 256), (28672, 4096, 28672 * 4096),
                                      (0, 64, 0), (-1, 64, 0), (16, 0, 0), (1 << 62, 64, 0)])
def test_code_bytes(rows, K, n):
    assert moe.moe_int8_code_bytes(rows, K) == n


@pytest.mark.parametrize("call", [matmul, gated])
def test_products(L, cus, call):
    for bad in (dict(T=-1), dict(N=0), dict(N=-4), dict(K=0), dict(K=72), dict(x=None), dict(x=P + 8), dict(xs=None),
                dict(xs=P + 4)):
        assert call(L, **bad) == INVALID, bad
    for bad in (dict(T=(1 << 20) + 1), dict(N=(1 << 24) + 1), dict(K=131072), dict(T=1 << 20, N=1 << 18)):
        assert call(L, **bad) == UNSUPPORTED, bad
    assert call(L, T=0, x=None, xs=None, ws=None, n=0) == 0
    own = (dict(w=None), dict(w=P + 8), dict(ws_=None), dict(bias=P + 2), dict(y=None)) if call is matmul else (
        dict(wg=None), dict(sg=P + 4), dict(wu=None), dict(wu=P + 1), dict(su=None), dict(h=P + 2))
    for bad in own:
        assert call(L, **bad) == INVALID, bad


@pytest.mark.parametrize("call,size", [(matmul, moe.moe_matmul_int8_workspace_bytes), (gated, moe.moe_gated_int8_workspace_bytes)])
def test_workspace(L, cus, call, size):
    """None where tiles are whole; where they are cut along k, the sums of every part, and no less is taken."""
    assert size(16384, 4096, 14336) == 0 and size(1, 4096, 4096) == 0
    for bad in ((0, 16, 64), (-1, 16, 64), (1, 0, 64), (1, 16, 8), (1, 16, 1 << 20), (1 << 21, 16, 64)):
        assert size(*bad) == 0
    need = size(128, 4096, 14336)
    assert need > 0 and need % (128 * 4096 * 4) == 0
    sizes = dict(T=128, N=4096, K=14336)
    assert call(L, **sizes, n=need - 1) == WS_SMALL
    assert call(L, **sizes, ws=None) == INVALID and call(L, **sizes, ws=P + 8) == INVALID


def test_binding_refusals():
    """Tensors of wrong types and shapes, and tensors on the host."""
    bf = torch.bfloat16
    x, y, w = torch.zeros(2, 64, dtype=bf), torch.zeros(2, 64, dtype=bf), torch.ones(64, dtype=bf)
    q, s = torch.zeros(2, 64, dtype=torch.int8), torch.ones(2)
    for call in (lambda: moe.moe_norm_join(x, y, pre=w), lambda: moe.moe_quantize_int8(x), lambda: moe.moe_pack_int8(q, s),
                 lambda: moe.Int8(torch.zeros(4096, dtype=torch.int8), torch.ones(16), (16, 64))):
        with pytest.raises(ValueError):
            call()                                                                          # on the host
    for call in (lambda: moe.moe_norm_join(x.half(), y, pre=w), lambda: moe.moe_quantize_int8(x.float()),
                 lambda: moe.moe_pack_int8(x, s), lambda: moe.Int8(torch.zeros(4096, dtype=torch.uint8), torch.ones(16), (16, 64))):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        moe.Int8(torch.zeros(100, dtype=torch.int8), torch.ones(16), (16, 64))              # too few codes
    with pytest.raises(ValueError):
        moe.Int8(torch.zeros(4096, dtype=torch.int8), torch.ones(15), (16, 64))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_checks_under_sanitizers(tmp_path):
    exe = str(tmp_path / "int8_validate_fuzz")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-I", CSRC, os.path.join(HERE, "native", "int8_validate_fuzz.cpp"), os.path.join(CSRC, "moe_validate.cpp"),
           "-o", exe]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0", UBSAN_OPTIONS="halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "no failures" in r.stdout
