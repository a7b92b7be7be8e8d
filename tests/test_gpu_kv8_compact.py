"""kv8_compact against its definition: codes and scales equal bit for bit, all other places left as they were."""
import numpy as np
import pytest
import torch

import _draft_ref as draft
import _kv8_ref as ref
import paper_2605_20315_amd as mq

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


class Problem:
    def __init__(self, seed, n, past, Hkv=2, D=64, P=16, jumps=True):
        r = self.r = np.random.default_rng(seed)
        total = [a + b for a, b in zip(n, past)]
        held = [-(-m // P) for m in total]
        pages = sum(held) + 2
        order = r.permutation(pages)
        self.pt = np.full((len(n), max(max(held), 1)), -1, np.int32)
        at = 0
        for b, m in enumerate(held):
            self.pt[b, :m] = order[at : at + m]
            at += m
        self.cu, self.lens = np.cumsum([0] + list(n)).astype(np.int32), np.array(total, np.int32)
        self.codes = [r.integers(0, 256, (pages, Hkv, P, D)).astype(np.uint8) for _ in "kv"]
        self.scales = [r.integers(127 - 6, 127 + 7, (pages, Hkv)).astype(np.uint8) for _ in "kv"] if jumps else [np.full((pages, Hkv), 120, np.uint8) for _ in "kv"]
        self.path, self.counts = np.full(sum(n), -1, np.int32), np.zeros(len(n), np.int32)
        for b, m in enumerate(n):
            c = self.counts[b] = int(r.integers(1, m + 1)) if m else 0
            self.path[self.cu[b] : self.cu[b] + c] = [0] + sorted(r.choice(np.arange(1, m), c - 1, replace=False)) if c else []

    def check(self):
        want = [x.copy() for x in (self.codes[0], self.scales[0], self.codes[1], self.scales[1])]
        draft.compact(*want, self.pt, self.cu, self.lens, self.path, self.counts)
        got = [torch.from_numpy(x.copy()).cuda() for x in (self.codes[0], self.scales[0], self.codes[1], self.scales[1])]
        assert mq.kv8_compact(*got, ints(self.pt), ints(self.cu), ints(self.lens), ints(self.path), ints(self.counts)) is None
        for name, g, w in zip(("k_codes", "k_scales", "v_codes", "v_scales"), got, want):
            g = g.cpu().numpy()
            if "codes" in name:  # a NaN brought to another scale keeps no more than being one
                g, w = (np.where((x & 0x7F) == 0x7F, 0x7F, x) for x in (g, w))
            assert np.array_equal(g, w), (name, np.argwhere(g != w)[:4])
        return want


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_paths_of_many_lengths(D, P):
    n = [1, 2, 3, 8, 9, 17, 40, 64, 65, 0, 130]
    for seed in range(2):
        r = np.random.default_rng(seed)
        Problem(seed, n, [int(x) for x in r.integers(0, 3 * P, len(n))], D=D, P=P).check()


def test_the_first_page_holds_earlier_tokens():
    changed = 0
    for seed in range(6):
        p = Problem(seed, [30, 30], [9, 14], P=16)
        for s in p.scales:
            s[p.pt[:, 0]] = 121  # below the others: it has to grow, and its tokens with it
            s[p.pt[:, 1:3]] = 125
        want = p.check()
        changed += sum(int((want[i][p.pt[:, 0], :, :9] != p.codes[i // 2][p.pt[:, 0], :, :9]).sum()) for i in (0, 2))
    assert changed > 100


def test_nothing_to_do():
    p = Problem(1, [20, 5, 0, 7], [3, 40, 9, 0])
    for b, m in enumerate((20, 5, 0, 7)):
        p.path[p.cu[b] : p.cu[b] + m], p.counts[b] = np.arange(m), m
    want = p.check()
    assert all(np.array_equal(w, x) for w, x in zip(want, (p.codes[0], p.scales[0], p.codes[1], p.scales[1])))
    p.counts[:] = 0
    p.check()


def test_scales_at_their_bounds():
    for seed in range(4):
        p = Problem(seed, [40, 60], [5, 0], P=16)
        for s in p.scales:
            s[:] = p.r.choice([127 - 112, 127 - 111, 127, 127 + 118, 127 + 119], s.shape)
        p.check()


def test_small_numbers_are_rounded_once():
    p = Problem(3, [50], [7], P=16)
    for c, s in zip(p.codes, p.scales):
        c[:] = p.r.integers(0, 24, c.shape)  # subnormal codes, and small ones above them
        s[:] = p.r.integers(120, 130, s.shape)
    p.check()


def test_places_without_a_page_and_tables_with_a_stride():
    p = Problem(4, [40, 40, 40], [10, 10, 10], P=16)
    p.pt[0, 0], p.pt[1, 1], p.pt[2, 2] = -1, 2 ** 31 - 1, len(p.codes[0])
    p.check()
    p = Problem(5, [40, 20], [10, 0], P=16)
    want = [x.copy() for x in (p.codes[0], p.scales[0], p.codes[1], p.scales[1])]
    draft.compact(*want, p.pt, p.cu, p.lens, p.path, p.counts)
    wide = torch.full((2, p.pt.shape[1] + 3), 1 << 30, dtype=torch.int32, device="cuda")
    wide[:, : p.pt.shape[1]] = ints(p.pt)
    got = [torch.from_numpy(x.copy()).cuda() for x in (p.codes[0], p.scales[0], p.codes[1], p.scales[1])]
    mq.kv8_compact(*got, wide[:, : p.pt.shape[1]], ints(p.cu), ints(p.lens), ints(p.path), ints(p.counts))
    assert np.array_equal(got[1].cpu().numpy(), want[1]) and np.array_equal(got[3].cpu().numpy(), want[3])


def test_lengths_that_do_not_fit():
    p = Problem(6, [30, 30, 12], [0, 0, 8], P=16)
    p.lens[:] = [20, 0, 20]      # ten tokens, and all of them, lie before the first place
    p.counts[:] = [25, 30, 1000]  # and a path is no longer than the new tokens
    p.path[:] = np.concatenate([np.arange(30) + np.minimum(np.arange(30) // 5, 4), np.arange(30), np.arange(12)])
    p.path[25:30] = -1
    p.check()
    p = Problem(7, [30], [0], P=16)
    p.lens[:] = 2 ** 30  # beyond the table
    p.check()


def test_an_empty_pool():
    from paper_2605_20315_amd import _lib
    codes, scales = torch.full((1, 2, 16, 64), 9, dtype=torch.uint8, device="cuda"), torch.full((1, 2), 120, dtype=torch.uint8, device="cuda")
    args = [ints([[0, 0]]), ints([0, 9]), ints([20]), ints([0, 2, 3, 4, 5, 6, 7, 8, -1]), ints([8])]
    c, s, (pt, cu, lens, path, counts) = codes.data_ptr(), scales.data_ptr(), (x.data_ptr() for x in args)
    rc = _lib.load().kv8_compact(c, s, c, s, 0, 16, 2, 64, pt, 2, 2, cu, lens, 1, 9, path, counts, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert rc == 0 and (codes == 9).all() and (scales == 120).all()
    with pytest.raises(mq.MixQuantError, match="MQ_ERR_NULL"):  # (a tensor of no elements has no address)
        mq.kv8_compact(codes[:0], scales[:0], codes[:0], scales[:0], *args)


def test_refusals():
    p = Problem(8, [5], [3])
    cache = [torch.from_numpy(x).cuda() for x in (p.codes[0], p.scales[0], p.codes[1], p.scales[1])]
    args = [ints(p.pt), ints(p.cu), ints(p.lens)]
    with pytest.raises(mq.MixQuantError, match="path"):
        mq.kv8_compact(*cache, *args, ints(p.path).long(), ints(p.counts))
    with pytest.raises(mq.MixQuantError, match="counts"):
        mq.kv8_compact(*cache, *args, ints(p.path), ints([1, 1]))
    with pytest.raises(AssertionError):
        mq.kv8_compact(cache[0][..., :32], *cache[1:], *args, ints(p.path), ints(p.counts))
