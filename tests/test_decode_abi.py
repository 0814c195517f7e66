"""The entry points for few sequences on a host without a GPU: they refuse bad arguments before any launch, report
their workspaces, and their checks run under the sanitizers.  No call here reaches a kernel."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import paper_2606_21712_amd as moe

INVALID, UNSUPPORTED, WS_SMALL = 1, 2, 3
P = 0x10000          # a 16-byte aligned address that is never dereferenced
S = None
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


# ---------------------------------------------------------------- 4-bit weights
@pytest.mark.parametrize("rows,K,g,codes,scales,with_zeros", [
    (16, 128, 128, 1024, 32, 64), (1, 32, 32, 1024, 128, 256), (17, 160, 32, 4096, 512, 1024),
    (28672, 4096, 64, 28672 * 2048, 28672 * 128, 28672 * 256), (0, 128, 64, 0, 0, 0), (16, 128, 48, 1024, 0, 0)])
def test_int4_bytes(rows, K, g, codes, scales, with_zeros):
    assert moe.moe_int4_code_bytes(rows, K) == codes
    assert moe.moe_int4_scale_bytes(rows, K, g) == scales
    assert moe.moe_int4_scale_bytes(rows, K, g, True) == with_zeros


def quantize(L, src=P, rows=4, K=128, g=64, codes=P, scales=P, zeros=None):
    return L.moe_quantize_int4(src, rows, K, g, codes, scales, zeros, S)


def pack(L, codes=P, scales=P, zeros=None, mats=1, rows=4, K=128, g=64, oc=P, os_=P):
    return L.moe_pack_int4(codes, scales, zeros, mats, rows, K, g, oc, os_, S)


def matvec(L, x=P, codes=P, scales=P, zeros=0, T=1, N=16, K=128, g=64, y=P):
    return L.moe_matvec_int4(x, codes, scales, zeros, T, N, K, g, y, S)


@pytest.mark.parametrize("call", [quantize, pack, matvec])
def test_int4_sizes(L, call):
    for bad in (dict(g=16), dict(g=0), dict(g=-64), dict(K=96), dict(K=0), dict(K=-64)):
        assert call(L, **bad) == INVALID, bad
    assert call(L, K=1 << 24) == UNSUPPORTED
    assert b"K=" in L.moe_last_error()


def test_quantize_and_pack(L):
    assert quantize(L, rows=-1) == INVALID
    assert quantize(L, rows=1 << 40) == UNSUPPORTED
    for bad in (dict(src=None), dict(codes=P + 1), dict(scales=None), dict(zeros=P + 8)):
        assert quantize(L, **bad) == INVALID, bad
    assert quantize(L, rows=0, src=None, codes=None, scales=None) == 0
    assert pack(L, mats=-1) == INVALID and pack(L, rows=-1) == INVALID
    assert pack(L, mats=1 << 40) == UNSUPPORTED and pack(L, rows=1 << 40) == UNSUPPORTED
    for bad in (dict(codes=None), dict(scales=P + 2), dict(zeros=P + 4), dict(oc=None), dict(os_=P + 8)):
        assert pack(L, **bad) == INVALID, bad
    assert pack(L, mats=0, codes=None) == 0 and pack(L, rows=0, codes=None) == 0


def test_matvec(L):
    for bad in (dict(T=-1), dict(N=0), dict(N=-5), dict(zeros=2), dict(zeros=-1), dict(x=None), dict(codes=P + 4),
                dict(scales=None), dict(y=P + 2)):
        assert matvec(L, **bad) == INVALID, bad
    assert matvec(L, T=(1 << 20) + 1) == UNSUPPORTED
    assert matvec(L, N=1 << 20, K=4096) == UNSUPPORTED                    # 2 GiB of codes
    assert matvec(L, T=0, x=None, codes=None, scales=None, y=None) == 0


# ---------------------------------------------------------------- the layer for few tokens
def few(L, x=P, logits=P, T=8, H=256, E=8, k=2, F=512, Fs=0, renorm=1, w=(P,) * 6, ids=P, wts=P, y=P, ws=P,
        n=1 << 30):
    return L.moe_few_tokens(x, logits, T, H, E, k, F, Fs, renorm, *w, ids, wts, y, ws, n, S)


def few4(L, x=P, logits=P, T=8, H=256, E=8, k=2, F=512, Fs=0, renorm=1, w=(P,) * 6, ids=P, wts=P, y=P, ws=P,
         n=1 << 30, g=64, zeros=0):
    refs = (moe._Int4Ref * 6)(*[(p, p) for p in w]) if w else None
    return L.moe_few_tokens_int4(x, logits, T, H, E, k, F, Fs, renorm, g, zeros, refs, ids, wts, y, ws, n, S)


@pytest.mark.parametrize("call", [few, few4])
def test_few(L, call):
    for bad in (dict(T=-1), dict(k=0), dict(k=9), dict(E=0), dict(H=100), dict(H=0), dict(F=32), dict(F=-64), dict(Fs=-64),
                dict(Fs=32), dict(renorm=2), dict(x=None), dict(logits=P + 4), dict(ids=None), dict(wts=P + 8),
                dict(y=None), dict(ws=None), dict(w=(P, P, None, P, P, P)), dict(w=(P,) * 5 + (None,), Fs=64),
                dict(w=(P + 2,) + (P,) * 5)):
        assert call(L, **bad) == INVALID, bad
    for bad in (dict(T=17), dict(E=300), dict(E=64, k=17), dict(H=(1 << 20) + 64), dict(F=1 << 20, H=1 << 12)):
        assert call(L, **bad) == UNSUPPORTED, bad
    need = moe.moe_few_tokens_workspace_bytes(8, 256, 2, 512)
    assert need > 0 and call(L, n=need - 1) == WS_SMALL
    assert call(L, T=0, x=None, logits=None, w=(None,) * 6, ids=None, wts=None, y=None, ws=None, n=0) == 0


def test_few_int4(L):
    for bad in (dict(w=None), dict(g=48), dict(zeros=2), dict(g=128, H=192), dict(g=128, F=192), dict(g=128, Fs=64)):
        assert few4(L, **bad) == INVALID, bad


@pytest.mark.parametrize("bad", [(0, 64, 1, 64), (17, 64, 1, 64), (1, 0, 1, 64), (1, 64, 0, 64), (1, 64, 1, 0), (1, 64, 17, 64),
                                 (1, 64, 1, 64, -1)])
def test_few_workspace(bad):
    assert moe.moe_few_tokens_workspace_bytes(*bad) == 0
    sizes = [moe.moe_few_tokens_workspace_bytes(T, 4096, 2, 14336) for T in range(1, 17)]
    assert sizes == sorted(sizes) and sizes[0] >= 2 * 14336 * 4


# ---------------------------------------------------------------- the paged 8-bit cache
def cache(k=P, v=P, ke=P, ve=P, pages=8, page=64, heads=2, dim=128):
    return ctypes.byref(moe._Kv8Cache(k, v, ke, ve, pages, page, heads, dim))


def append(L, q=P, qs=512, k=P, ks=256, v=P, vs=256, T=3, Hq=4, cs=P, positions=100, rot=128, inter=0, c="", table=P,
           cols=4, lens=P, cu=P, B=2, out=P):
    return L.moe_kv8_append(q, qs, k, ks, v, vs, T, Hq, cs, positions, rot, inter, cache() if c == "" else c, table, cols,
                            lens, cu, B, out, S)


def attend(L, q=P, T=3, Hq=4, c="", table=P, cols=4, lens=P, cu=P, B=2, new=2, length=200, window=0, scale=0.1, out=P,
           ws=P, n=1 << 40):
    return L.moe_kv8_attention(q, T, Hq, cache() if c == "" else c, table, cols, lens, cu, B, new, length, window, scale,
                               out, ws, n, S)


@pytest.mark.parametrize("call", [append, attend])
def test_kv8_common(L, cus, call):
    for bad in (dict(c=None), dict(c=cache(page=40)), dict(c=cache(page=0)), dict(c=cache(heads=0)), dict(c=cache(heads=3)),
                dict(c=cache(pages=0)), dict(c=cache(k=None)), dict(c=cache(v=P + 8)), dict(c=cache(ke=None)),
                dict(c=cache(ve=P + 1)), dict(Hq=0), dict(Hq=3), dict(T=-1), dict(B=-1), dict(B=0), dict(cols=0), dict(table=None),
                dict(lens=P + 4), dict(cu=None), dict(q=None), dict(out=P + 2)):
        assert call(L, **bad) == INVALID, bad
    for bad in (dict(c=cache(dim=96)), dict(c=cache(dim=512)), dict(c=cache(heads=70000), Hq=70000), dict(T=1 << 24),
                dict(B=1 << 23), dict(c=cache(pages=1 << 40)), dict(cols=1 << 30)):
        assert call(L, **bad) == UNSUPPORTED, bad
    assert call(L, T=0, q=None, table=None, lens=None, cu=None, out=None) == 0


def test_append(L):
    for bad in (dict(rot=8), dict(rot=144), dict(rot=-16), dict(inter=2), dict(positions=0), dict(cs=None), dict(qs=511),
                dict(qs=508), dict(ks=128), dict(vs=260), dict(k=None), dict(v=P + 4)):
        assert append(L, **bad) == INVALID, bad
    assert b"moe_kv8_append" in L.moe_last_error()


def test_attention(L, cus):
    nan, inf = float("nan"), float("inf")
    for bad in (dict(new=0), dict(length=-1), dict(window=-1), dict(scale=0.0), dict(scale=-0.1), dict(scale=nan),
                dict(scale=inf)):
        assert attend(L, **bad) == INVALID, bad
    assert attend(L, new=1 << 24) == UNSUPPORTED
    need = moe.moe_kv8_attention_workspace_bytes(3, 2, 4, 2, 128, 2, 100000)
    assert need > 0 and attend(L, length=100000, n=need - 1) == WS_SMALL
    assert attend(L, length=100000, ws=None) == INVALID


def test_attention_workspace(cus):
    ws = moe.moe_kv8_attention_workspace_bytes
    assert ws(2, 2, 4, 2, 128, 1, 64) == 0                                # short: nothing is cut
    assert ws(4096, 64, 32, 8, 128, 64, 4096) == 0                        # enough tiles
    for bad in ((0, 1, 1, 1, 64, 1, 1), (1, 0, 1, 1, 64, 1, 1), (1, 1, 3, 2, 64, 1, 1), (1, 1, 1, 1, 80, 1, 1),
                (1, 1, 1, 1, 64, 0, 1), (1, 1, 1, 1, 64, 1, -1), (1, 1, 1, 1, 64, 1, 1, -1)):
        assert ws(*bad) == 0
    # rows' descriptions, and parts of 16 rows of 128 sums and more: at least the tiles', at most four a compute
    # unit besides
    rows, part = 8 * 32 * 2 * 4, 16 * 130 * 4
    assert rows + 64 * part <= ws(8, 8, 32, 8, 128, 1, 40960) <= rows + (64 + 1024) * (part + 16 * 8)


# ---------------------------------------------------------------- the binding
def test_binding_refusals():
    """Tensors of wrong types and shapes, and tensors on the host."""
    bf, u8 = torch.bfloat16, torch.uint8
    x = torch.zeros(2, 64, dtype=bf)
    with pytest.raises(ValueError):
        moe.Int4(torch.zeros(1024, dtype=u8), torch.zeros(16, dtype=u8), False, (16, 64), 64)      # scales too small
    with pytest.raises(TypeError):
        moe.Int4(torch.zeros(1024, dtype=bf), torch.zeros(64, dtype=u8), False, (16, 64), 64)
    with pytest.raises(ValueError):
        moe.Int4(torch.zeros(1024, dtype=u8), torch.zeros(64, dtype=u8), False, (16, 64), 64)      # on the host
    with pytest.raises(TypeError):
        moe.moe_few_tokens(x.float(), torch.zeros(2, 4), 1, *(torch.zeros(4, 64, 64, dtype=bf),) * 3,
                           ws=torch.zeros(1 << 20, dtype=u8))
    with pytest.raises(ValueError):
        moe.moe_few_tokens(x, torch.zeros(2, 4), 1, *(torch.zeros(4, 64, 64, dtype=bf),) * 3)      # on the host
    with pytest.raises(ValueError):
        moe.MoELayerFew(17, 64, 4, 1, 64, device="cpu")
    with pytest.raises(TypeError):
        moe.KVCache8(*(torch.zeros(s, dtype=bf) for s in ((1, 1, 16, 64), (1, 1, 1, 64, 16), (1, 1, 1), (1, 1, 1))))
    with pytest.raises(ValueError):
        moe.KVCache8(*(torch.zeros(s, dtype=u8) for s in ((1, 1, 16, 64), (1, 1, 1, 16, 64), (1, 1, 1), (1, 1, 1))))
    with pytest.raises(ValueError):
        moe.KVCache8.empty(1, 1, 64, 16, device="cpu")


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_checks_under_sanitizers(tmp_path):
    exe = str(tmp_path / "decode_validate_fuzz")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-I", CSRC, os.path.join(HERE, "native", "decode_validate_fuzz.cpp"), os.path.join(CSRC, "moe_validate.cpp"),
           "-o", exe]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0", UBSAN_OPTIONS="halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "no failures" in r.stdout
