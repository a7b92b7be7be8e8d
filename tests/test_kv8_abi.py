"""Host-side validation of the cache, attention and matrix-vector entry points: refused before any launch.  CPU only."""
import ctypes
import os

import pytest
import torch

import paper_2605_20315_amd as mq

OK, NULL, SHAPE, ALIGN, ARG, SCRATCH = 0, 1, 2, 3, 4, 6
FAKE = 1 << 20  # an address that is never read: every call here is refused first


@pytest.fixture(scope="module")
def lib():
    from paper_2605_20315_amd import _lib, build
    if not os.path.exists(_lib.LIB_PATH):
        build.build_library()
    return _lib.load()


def matvec(lib, **kw):
    a = dict(x=FAKE, ldx=64, c=FAKE, s=FAKE, al=FAKE, M=1, N=8, K=64, y=FAKE, ldy=8, out=0, layout=0, ws=None, bytes=0)
    a.update(kw)
    return lib.nvfp4_matvec(*a.values(), None)


def test_matvec(lib):
    assert matvec(lib, M=0) == OK and matvec(lib, N=0, ldy=0) == OK
    for bad in (dict(M=-1), dict(N=-1), dict(K=0), dict(K=24), dict(ldx=56), dict(ldy=7), dict(K=48, ldx=48, layout=1), dict(bytes=-1), dict(M=65536),
                dict(N=1 << 31, ldy=1 << 31), dict(K=1 << 31, ldx=1 << 31)):
        assert matvec(lib, **bad) == SHAPE, bad
    assert matvec(lib, out=2) == ARG and matvec(lib, layout=2) == ARG
    for name in ("x", "c", "s", "al", "y"):
        assert matvec(lib, **{name: None}) == NULL
    for bad in (dict(x=FAKE + 8), dict(ldx=68), dict(c=FAKE + 8), dict(s=FAKE + 2), dict(al=FAKE + 2), dict(y=FAKE + 1), dict(y=FAKE + 2, out=1),
                dict(M=9, ws=FAKE + 8, bytes=1 << 20)):
        assert matvec(lib, **bad) == ALIGN, bad
    need = lib.mq_nvfp4_matvec_workspace_bytes(9, 8, 64)
    assert need > 0 and matvec(lib, M=9, ws=FAKE, bytes=need - 1) == SCRATCH and matvec(lib, M=9) == SCRATCH


def test_matvec_workspace(lib):
    w = lib.mq_nvfp4_matvec_workspace_bytes
    assert w(1, 4096, 4096) == w(4, 4096, 8192) == w(100, 4096, 48) == w(0, 1, 64) == w(1, 1, 24) == 0
    assert w(5, 4096, 4096) > 0 and w(4, 4096, 8256) > 0 and w(1, 4096, 32832) > 0
    assert w(64, 28672, 4096) >= 64 * 4096 * 2 and w(40, 5120, 25600) >= 3 * 40 * 5120 * 4


def append(lib, **kw):
    a = dict(q=FAKE, ldq=256, k=FAKE, ldk=128, v=FAKE, ldv=128, o=FAKE, kc=FAKE, ks=FAKE, vc=FAKE, vs=FAKE, pages=4, P=16, Hq=4, Hkv=2, D=64, pt=FAKE,
             pt_ld=2, W=2, cu=FAKE, lens=FAKE, B=1, T=3, table=FAKE, max_pos=32, rot=64, pos=None, inter=0)
    a.update(kw)
    return lib.kv8_append(*a.values(), None)


def attend(lib, **kw):
    a = dict(q=FAKE, ldq=256, kc=FAKE, ks=FAKE, vc=FAKE, vs=FAKE, pages=4, P=16, Hq=4, Hkv=2, D=64, pt=FAKE, pt_ld=2, W=2, cu=FAKE, lens=FAKE, B=1, T=3,
             scale=0.125, window=0, y=FAKE, ldy=256, ws=None, bytes=0)
    a.update(kw)
    return lib.kv8_attention(*a.values(), None)


CACHE_SHAPES = (dict(pages=-1), dict(P=8), dict(P=256), dict(P=48), dict(D=32), dict(D=96), dict(Hkv=0), dict(Hq=0), dict(Hq=5), dict(Hkv=-2), dict(W=-1),
                dict(pt_ld=1), dict(B=-1), dict(T=-1), dict(W=1 << 27, pt_ld=1 << 27), dict(T=1 << 30), dict(ldq=248))


def test_append(lib):
    assert append(lib, T=0) == OK and append(lib, B=0) == OK
    for bad in CACHE_SHAPES + (dict(rot=8), dict(rot=80), dict(rot=-16), dict(max_pos=-1), dict(max_pos=0), dict(ldk=64), dict(ldv=120)):
        assert append(lib, **bad) == SHAPE, bad
    for name in ("q", "k", "v", "o", "kc", "ks", "vc", "vs", "pt", "cu", "lens", "table"):
        assert append(lib, **{name: None}) == NULL, name
    for bad in (dict(q=FAKE + 8), dict(k=FAKE + 8), dict(v=FAKE + 2), dict(o=FAKE + 8), dict(kc=FAKE + 8), dict(vc=FAKE + 1), dict(pt=FAKE + 2),
                dict(cu=FAKE + 1), dict(lens=FAKE + 2), dict(table=FAKE + 8), dict(pos=FAKE + 2), dict(ldq=260), dict(ldk=132), dict(ldv=129)):
        assert append(lib, **bad) == ALIGN, bad


def test_attention(lib):
    assert attend(lib, T=0) == OK and attend(lib, B=0) == OK
    for bad in CACHE_SHAPES + (dict(ldy=128), dict(bytes=-1)):
        assert attend(lib, **bad) == SHAPE, bad
    for bad in (0.0, -1.0, float("inf"), float("nan")):
        assert attend(lib, scale=bad) == ARG
    for name in ("q", "y", "kc", "ks", "vc", "vs", "pt", "cu", "lens"):
        assert attend(lib, **{name: None}) == NULL, name
    for bad in (dict(q=FAKE + 8), dict(y=FAKE + 8), dict(kc=FAKE + 8), dict(vc=FAKE + 8), dict(pt=FAKE + 2), dict(cu=FAKE + 1), dict(lens=FAKE + 2),
                dict(ldq=260), dict(ldy=258), dict(ws=FAKE + 8, bytes=64)):
        assert attend(lib, **bad) == ALIGN, bad
    w = lib.mq_kv8_attention_workspace_bytes
    assert 0 < w(1, 1, 4, 2, 64) <= 64 << 20 and w(0, 1, 4, 2, 64) == w(1, 1, 5, 2, 64) == w(1, 1, 4, 2, 96) == 0


def test_rope_table(lib):
    def table(**kw):
        a = dict(t=FAKE, n=16, rot=64, base=1e4, kind=0, factor=4.0, orig=4096, fast=32.0, slow=1.0, gain=1.0)
        a.update(kw)
        return lib.mq_rope_table(*a.values(), None)

    assert table(n=0) == OK
    for bad in (dict(n=-1), dict(n=1 << 31), dict(rot=0), dict(rot=8), dict(rot=272), dict(rot=40), dict(kind=2, orig=0)):
        assert table(**bad) == SHAPE, bad
    nan, inf = float("nan"), float("inf")
    for bad in (dict(kind=3), dict(kind=-1), dict(base=1.0), dict(base=nan), dict(base=inf), dict(kind=1, factor=0.5), dict(kind=2, factor=nan), dict(gain=nan),
                dict(kind=2, fast=0.5), dict(kind=2, slow=0.0), dict(kind=2, fast=inf)):
        assert table(**bad) == ARG, bad
    assert table(t=None) == NULL and table(t=FAKE + 4) == ALIGN


def test_tensors_on_the_cpu_are_refused():
    x, u8, f, i = torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(8, 32, dtype=torch.uint8), torch.zeros(1), torch.zeros(2, dtype=torch.int32)
    h, codes, scales = torch.zeros(2, 2, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 16, 64, dtype=torch.uint8), torch.zeros(3, 2, dtype=torch.uint8)
    with pytest.raises(mq.MixQuantError, match="GPU"):
        mq.nvfp4_matvec(x, u8, torch.zeros(8, 4, dtype=torch.uint8), f)
    with pytest.raises(mq.MixQuantError, match="GPU"):
        mq.kv8_append(h, h, h, codes, scales, codes, scales, i.view(1, 2), i, i[:1])
    with pytest.raises(mq.MixQuantError, match="GPU"):
        mq.kv8_attention(h, codes, scales, codes, scales, i.view(1, 2), i, i[:1], 0.125)
    with pytest.raises(mq.MixQuantError, match="GPU"):
        mq.mq_rope_table(16, 64, device="cpu")


def test_matvec_workspace_of_wide_layers(lib):
    # where many workgroups would each bring the activations into their LDS, a launch in front does it once
    w = lib.mq_nvfp4_matvec_workspace_bytes
    assert w(2, 28672, 4096) == 0 and w(3, 28672, 4096) > 0 and w(4, 8191, 4096) == 0
