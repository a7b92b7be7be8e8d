"""The kernels' forms of kv8_tree_attention that short calls do not reach: two tiles of rows from one expansion, which a wide page table brings,
both joins of partial sums, and caches of more than 4 GiB."""
import numpy as np
import pytest
import torch

import _kv8_ref as ref
import paper_2605_20315_amd as mq
from test_gpu_kv8_attention import dev
from test_gpu_kv8_compact import ints
from test_gpu_kv8_tree_attention import Problem

pytestmark = pytest.mark.gpu


def wide(p):
    """Room in the page table for so long histories that a call counts as one of much arithmetic."""
    T, Hq, _ = p.q.shape
    pages = (49 << 20) // (T * Hq * p.kc.shape[2]) + 1
    more = np.full((len(p.lens), pages - p.pt.shape[1]), -1, np.int32)
    p.pt = np.concatenate([p.pt, more], 1)
    return p


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_trees_of_many_sizes(D, P):
    wide(Problem(D + P, [1, 2, 5, 8, 9, 17, 31, 32], [0, 1, 33, 64, 127, 200, 31, 500], 8, 2, D, P)).check()
    wide(Problem(D + P + 1, [33, 64, 65, 100, 0, 40], [200, 0, 77, 1300, 9, 31], 8, 2, D, P)).check()


@pytest.mark.parametrize("Hq,Hkv", [(7, 7), (28, 4), (36, 3), (40, 2)])
def test_groups_of_heads(Hq, Hkv):
    wide(Problem(Hq, [17, 20, 40], [770, 130, 3], Hq, Hkv, 128, 32)).check()


@pytest.mark.parametrize("window", [1, 16, 33, 100, 1000])
@pytest.mark.parametrize("D", [64, 128])
def test_windows(D, window):
    wide(Problem(window, [24, 25, 10, 41, 3], [300, 2000, 0, 3, 63], 4, 2, D, 16, window)).check()
    wide(Problem(window + 2, [70, 6], [70, 400], 8, 2, D, 64, window, positions=False)).check()


def test_masks_lengths_and_pages_of_all_kinds():
    p = wide(Problem(2, [100, 33], [40, 0], 4, 2, 64, 16, words=4))
    p.tree = p.r.integers(-(2 ** 31), 2 ** 31, p.tree.shape).astype(np.int32)
    p.check()
    p.tree[:50], p.tree[100:] = 0, 0
    p.check()
    p = wide(Problem(11, [30, 20, 50, 70], [0, 4, 0, 0], 4, 2, 128, 16))
    p.lens[0], p.lens[2], p.lens[3] = 1, 0, 30
    p.pt[1, 0] = -1
    p.check()
    p = wide(Problem(12, [10, 20, 80], [200, 100, 40], 4, 2, 64, 16))
    p.pt[0, 3], p.pt[0, 12], p.pt[1, 0], p.pt[2, 2] = -1, 2 ** 31 - 1, len(p.kc), -(2 ** 31)
    p.check()


@pytest.mark.parametrize("D,P", [(64, 16), (128, 64)])
def test_nan_reaches_the_rows_that_see_it_and_no_others(D, P):
    for seed, (n, past) in enumerate((([40], [300]), ([12, 70], [64, 10]))):
        p = wide(Problem(seed, n, past, 8, 2, D, P, window=40))
        r = np.random.default_rng(seed)
        for codes in (p.kc, p.vc):
            for page in p.pt[0][p.pt[0] >= 0][:4]:
                codes[page, r.integers(2), r.integers(P), r.integers(D)] = 0x7F
            codes[p.pt[0, (past[0] + 3) // P], 0, (past[0] + 3) % P, 5] = 0xFF
        p.check()


def test_long_histories_are_cut_and_joined():
    # with few rows a join's workgroup takes a row's chunks, from 2048 rows (tokens times heads) on four to sixteen rows
    wide(Problem(5, [9, 30, 20], [9000, 20, 3001], 4, 2, 64, 64)).check()
    wide(Problem(6, [60], [5000], 8, 2, 128, 16)).check()
    wide(Problem(7, [12] * 40, [int(x) for x in np.random.default_rng(1).integers(0, 700, 40)], 8, 4, 64, 32)).check("full")
    wide(Problem(8, [130, 140], [3000, 10], 8, 1, 128, 64)).check("full")
    Problem(9, [130, 140], [3000, 10], 8, 1, 256, 64).check("full")


@pytest.mark.parametrize("D,window", [(64, 0), (128, 90), (256, 0)])
def test_more_items_than_places_begin_with_the_longest(D, window):
    r = np.random.default_rng(D)
    for B, Hq, Hkv in ((256, 4, 4), (200, 8, 4), (2, 64, 8), (97, 8, 8)):
        n = [int(x) for x in r.integers(0, 6, B)] if B > 2 else [130, 131]
        past = [int(x) for x in r.integers(0, 300, B)] if B > 97 else [200] * B  # lengths of all kinds, and all alike
        p = Problem(B, n, past, Hq, Hkv, D, 64, window)
        p.lens[B // 2] = 0 if n[B // 2] > 5 else p.lens[B // 2]
        p.check()
        wide(p).check()


def test_scores_that_grow_along_the_history():
    """The maximum is followed only where it is outgrown by 2^8: scores that rise by less, by more, and by much, and that fall."""
    for seed, by in enumerate((1.0, 30.0, 3000.0, -30.0)):
        p = Problem(seed, [20], [700], 8, 2, 64, 16)
        p.q[:] = np.abs(p.q)
        at = np.repeat(np.arange(len(p.pt[0])), p.kc.shape[2])[:720]
        for j in range(720):  # a key's codes all of one size, its page's scale as it is
            page = p.pt[0, j // 16]
            x = by * (j / 720 if by > 0 else (j / 720 - 1)) / 64 / 2.0 ** (p.ks[page].astype(int) - 127.0)
            p.kc[page, :, j % 16] = ref.e4m3_code(np.broadcast_to(x[:, None], (2, 64)))
        p.check()
        wide(p).check()


def far(p, pages):
    """The problem's caches at the end of device arrays of so many pages, and the table there."""
    first, out = pages - len(p.kc), []
    for x in (p.kc, p.ks, p.vc, p.vs):
        t = torch.empty((pages,) + x.shape[1:], dtype=torch.uint8, device="cuda")
        t[first:] = dev(x)
        out.append(t)
    return out, dev(np.where(p.pt >= 0, p.pt + first, p.pt).astype(np.int32))


@pytest.mark.parametrize("D", [128, 256])
def test_caches_beyond_4_gib(D):
    p = Problem(D, [30, 9], [300, 1000], 8, 2, D, 128)
    pages = (1 << 32) // (2 * 128 * D) + 40
    (kc, ks, vc, vs), pt = far(p, pages)
    assert kc.numel() > 1 << 32 and int(pt.max()) * 2 * 128 * D > 1 << 32
    args = p.device()
    near = mq.kv8_tree_attention(*args, p.scale, 0, dev(p.positions))
    got = mq.kv8_tree_attention(args[0], kc, ks, vc, vs, pt, *args[6:], p.scale, 0, dev(p.positions))
    assert torch.equal(near.view(torch.int16), got.view(torch.int16))
    path, counts = ints([0, 2, 5] + [-1] * 27 + [0, 3, 8] + [-1] * 6), ints([3, 3])
    cache = [dev(x) for x in (p.kc, p.ks, p.vc, p.vs)]
    mq.kv8_compact(*cache, args[5], *args[6:8], path, counts)
    mq.kv8_compact(kc, ks, vc, vs, pt, *args[6:8], path, counts)
    assert not torch.equal(cache[0], dev(p.kc))
    for a, b in zip(cache, (kc, ks, vc, vs)):
        assert torch.equal(a, b[pages - len(p.kc):])
