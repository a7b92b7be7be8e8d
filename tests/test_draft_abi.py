"""Host-side validation of the entry points for drafted tokens: refused before any launch.  CPU only."""
import os

import pytest
import torch

import paper_2605_20315_amd as mq
from paper_2605_20315_amd import ops

OK, NULL, SHAPE, ALIGN, ARG, SCRATCH = 0, 1, 2, 3, 4, 6
FAKE = 1 << 20  # an address that is never read: every call here is refused first


@pytest.fixture(scope="module")
def lib():
    from paper_2605_20315_amd import _lib, build
    if not os.path.exists(_lib.LIB_PATH):
        build.build_library()
    return _lib.load()


def with_defaults(fn, defaults):
    def call(**kw):
        a = dict(defaults)
        a.update(kw)
        return fn(*a.values(), None)
    return call


def test_tree(lib):
    call = with_defaults(lib.mq_draft_tree, dict(parents=FAKE, cu=FAKE, lens=FAKE, B=2, T=5, words=1, window=0, tree=FAKE, pos=FAKE))
    assert call(T=0) == OK and call(B=0) == OK
    for bad in (dict(B=-1), dict(T=-1), dict(words=0), dict(words=33), dict(words=-1), dict(T=1 << 31), dict(B=1 << 31)):
        assert call(**bad) == SHAPE, bad
    for name in ("parents", "cu", "lens", "tree", "pos"):
        assert call(**{name: None}) == NULL and call(**{name: FAKE + 2}) == ALIGN, name


def test_accept(lib):
    pointers = ("parents", "tokens", "sampled", "cu", "lens", "path", "counts", "next", "out")
    call = with_defaults(lib.mq_draft_accept, dict(parents=FAKE, tokens=FAKE, sampled=FAKE, cu=FAKE, lens=FAKE, B=2, T=5, path=FAKE, counts=FAKE,
                                                   next=FAKE, out=FAKE))
    assert call(B=0) == OK
    for bad in (dict(B=-1), dict(T=-1), dict(T=1 << 31), dict(B=1 << 31)):
        assert call(**bad) == SHAPE, bad
    for name in pointers:
        assert call(**{name: None}) == NULL and call(**{name: FAKE + 1}) == ALIGN, name


def test_compact(lib):
    call = with_defaults(lib.kv8_compact, dict(kc=FAKE, ks=FAKE, vc=FAKE, vs=FAKE, pages=4, P=16, Hkv=2, D=64, pt=FAKE, pt_ld=2, W=2, cu=FAKE, lens=FAKE,
                                               B=1, T=3, path=FAKE, counts=FAKE))
    assert call(T=0) == OK and call(B=0) == OK
    for bad in (dict(pages=-1), dict(P=8), dict(P=48), dict(D=96), dict(Hkv=0), dict(W=-1), dict(pt_ld=1), dict(B=-1), dict(T=-1), dict(W=1 << 27, pt_ld=1 << 27),
                dict(B=1 << 30, Hkv=1)):
        assert call(**bad) == SHAPE, bad
    for name in ("kc", "ks", "vc", "vs", "pt", "cu", "lens", "path", "counts"):
        assert call(**{name: None}) == NULL, name
    for bad in (dict(kc=FAKE + 8), dict(vc=FAKE + 1), dict(pt=FAKE + 2), dict(cu=FAKE + 1), dict(lens=FAKE + 2), dict(path=FAKE + 2), dict(counts=FAKE + 1)):
        assert call(**bad) == ALIGN, bad


def test_tree_attention(lib):
    call = with_defaults(lib.kv8_tree_attention, dict(q=FAKE, ldq=256, kc=FAKE, ks=FAKE, vc=FAKE, vs=FAKE, pages=4, P=16, Hq=4, Hkv=2, D=64, pt=FAKE, pt_ld=2,
                                                      W=2, cu=FAKE, lens=FAKE, B=1, T=3, tree=FAKE, words=1, pos=None, scale=0.125, window=0, y=FAKE,
                                                      ldy=256, ws=None, bytes=0))
    assert call(T=0) == OK and call(B=0) == OK
    for bad in (dict(pages=-1), dict(P=8), dict(P=256), dict(D=32), dict(Hkv=0), dict(Hq=5), dict(W=-1), dict(pt_ld=1), dict(B=-1), dict(T=-1),
                dict(W=1 << 27, pt_ld=1 << 27), dict(T=1 << 30), dict(ldq=248), dict(ldy=128), dict(bytes=-1), dict(words=0), dict(words=33)):
        assert call(**bad) == SHAPE, bad
    for bad in (0.0, -1.0, float("inf"), float("nan")):
        assert call(scale=bad) == ARG
    for name in ("q", "y", "kc", "ks", "vc", "vs", "pt", "cu", "lens", "tree"):
        assert call(**{name: None}) == NULL, name
    for bad in (dict(q=FAKE + 8), dict(y=FAKE + 8), dict(kc=FAKE + 8), dict(vc=FAKE + 8), dict(pt=FAKE + 2), dict(cu=FAKE + 1), dict(lens=FAKE + 2),
                dict(ldq=260), dict(ldy=258), dict(ws=FAKE + 8, bytes=64), dict(tree=FAKE + 2), dict(pos=FAKE + 1)):
        assert call(**bad) == ALIGN, bad


def test_sample(lib):
    call = with_defaults(lib.mq_sample, dict(x=FAKE, rows=2, V=100, ld=100, type=0, u=FAKE, t=FAKE, k=FAKE, p=FAKE, mp=FAKE, tokens=FAKE, ws=FAKE,
                                             bytes=1 << 40))
    assert call(rows=0) == OK
    for bad in (dict(rows=-1), dict(V=0), dict(V=-5), dict(ld=99), dict(V=(1 << 20) + 1, ld=1 << 21), dict(rows=(1 << 20) + 1), dict(bytes=-1)):
        assert call(**bad) == SHAPE, bad
    assert call(type=2) == ARG and call(type=-1) == ARG
    for name in ("x", "u", "tokens"):
        assert call(**{name: None}) == NULL, name
    for bad in (dict(x=FAKE + 1), dict(x=FAKE + 2, type=1), dict(u=FAKE + 2), dict(t=FAKE + 1), dict(k=FAKE + 2), dict(p=FAKE + 2), dict(mp=FAKE + 3),
                dict(tokens=FAKE + 2), dict(ws=FAKE + 8)):
        assert call(**bad) == ALIGN, bad
    need = lib.mq_sample_workspace_bytes
    assert need(0, 100) == need(-1, 100) == need(5, 0) == need(1, (1 << 20) + 1) == need((1 << 20) + 1, 5) == 0
    if need(2, 100):
        assert call(bytes=need(2, 100) - 1) == SCRATCH and call(ws=None, bytes=0) == SCRATCH and call(ws=None) == SCRATCH


def test_tensors_on_the_cpu_are_refused():
    i, f, u8 = torch.zeros(2, dtype=torch.int32), torch.zeros(2), torch.zeros(3, 2, dtype=torch.uint8)
    h, codes = torch.zeros(2, 2, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 16, 64, dtype=torch.uint8)
    for call in (lambda: mq.mq_draft_tree(i, i, i[:1], 1), lambda: mq.mq_draft_accept(i, i, i, i, i[:1]), lambda: mq.mq_sample(torch.zeros(2, 9), f),
                 lambda: mq.kv8_tree_attention(h, codes, u8, codes, u8, i.view(1, 2), i, i[:1], i.view(2, 1), 0.125),
                 lambda: mq.kv8_compact(codes, u8, codes, u8, i.view(1, 2), i, i[:1], i, i[:1])):
        with pytest.raises(mq.MixQuantError, match="GPU"):
            call()


def test_tensors_of_another_device_are_refused(monkeypatch):
    class There:
        is_cuda, device = True, torch.device("cuda", 1)

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(mq.MixQuantError, match="cuda:1.*current device is cuda:0"):
        ops._here(There())
