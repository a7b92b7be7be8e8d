"""kv8_tree_attention against its definition in binary64, within the tolerance that kv8_attention's roundings give."""
import numpy as np
import pytest
import torch

import _draft_ref as draft
import _kv8_ref as ref
import paper_2605_20315_amd as mq
from test_gpu_kv8_attention import Problem as Causal, dev

pytestmark = pytest.mark.gpu


class Problem(Causal):
    def __init__(self, seed, n, past, Hq, Hkv, D, P, window=0, words=None, spread=9, positions=True):
        super().__init__(seed, n, past, Hq, Hkv, D, P, window)
        parents = [p for m in n for p in draft.random_parents(self.r, m, spread)]
        self.words = words or max(1, -(-max(n) // 32))
        self.tree, depth = draft.tree(parents, self.cu, self.lens, self.words)
        self.positions = depth if positions else None

    def device(self):
        return super().device() + [dev(self.tree)]

    def reference(self):
        return draft.tree_attention(self.q, self.kc, self.ks, self.vc, self.vs, self.pt, self.cu, self.lens, self.tree, self.scale, self.window, self.positions)

    def check(self, workspace="both"):
        y, a, s = self.reference()
        tol = ref.attention_tolerance(y, a, s, self.D)
        args, positions = self.device(), None if self.positions is None else dev(self.positions)
        T, Hq, D = self.q.shape
        owned = int(self.cu[-1])
        for ws in (None, "full") if workspace == "both" else (workspace,):
            if ws:
                n = mq.mq_kv8_attention_workspace_bytes(T, len(self.lens), Hq, self.kc.shape[1], D)
                ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN: nothing of it may be read before it is written
            out = torch.full((T, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
            assert mq.kv8_tree_attention(*args, self.scale, self.window, positions, out, ws) is out
            torch.cuda.synchronize()
            got = out.float().cpu().numpy().astype(np.float64)[:owned]
            assert np.array_equal(np.isnan(got), np.isnan(y[:owned]))
            off = np.abs(got - y[:owned])
            bad = ~np.isnan(got) & ~(off <= tol[:owned])
            assert not bad.any(), (ws is not None, np.argwhere(bad)[:4], off[bad][:4], tol[:owned][bad][:4])
            again = mq.kv8_tree_attention(*args, self.scale, self.window, positions, workspace=ws)
            assert torch.equal(again[:owned].view(torch.int16), out[:owned].view(torch.int16))


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_trees_of_many_sizes_after_histories_of_many_lengths(D, P):
    Problem(D + P, [1, 2, 5, 8, 9, 17, 31, 32], [0, 1, 33, 64, 127, 200, 31, 500], 8, 2, D, P).check()   # tiles of 16 and 32 rows
    Problem(D + P + 1, [33, 64, 65, 100, 0, 40], [200, 0, 77, 130, 9, 31], 8, 2, D, P).check()             # of 128 rows


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 1), (7, 7), (28, 4), (36, 3), (40, 2)])
def test_groups_of_heads(Hq, Hkv):
    Problem(Hq, [1, 12, 40], [77, 130, 3], Hq, Hkv, 128, 32).check()


@pytest.mark.parametrize("window", [1, 2, 16, 33, 64, 100, 1000])
@pytest.mark.parametrize("D", [64, 128])
def test_windows(D, window):
    Problem(window, [4, 5, 10, 1, 3], [300, 200, 0, 3, 63], 4, 2, D, 16, window).check()
    Problem(window + 1, [70, 90], [70, 400], 8, 2, D, 64, window).check()
    Problem(window + 2, [70, 6], [70, 400], 8, 2, D, 64, window, positions=False).check()


def test_positions_of_all_kinds():
    p = Problem(1, [9, 80], [50, 60], 4, 2, 64, 16, window=20)
    p.positions = p.r.integers(-100, 200, p.positions.shape).astype(np.int32)
    p.positions[3], p.positions[20] = 2 ** 31 - 1, -(2 ** 31)
    p.check()


@pytest.mark.parametrize("n", [[6, 30], [100, 33]])
def test_masks_of_all_kinds(n):
    p = Problem(2, n, [40, 0], 4, 2, 64, 16, words=4)
    p.tree = p.r.integers(-(2 ** 31), 2 ** 31, p.tree.shape).astype(np.int32)  # any sets, and bits of tokens that are not there
    p.check()
    p.tree[: n[0] // 2], p.tree[n[0] :] = 0, 0  # rows that see the history alone, and rows that see nothing
    p.check()
    assert not p.reference()[0][n[0] :].any()


def test_tokens_beyond_the_masks():
    p = Problem(3, [50, 140], [40, 20], 4, 2, 128, 32, words=1)
    p.check()


def test_a_chain_is_causal_attention():
    """To the tolerance that either has of its definition: the kernels may leave a row's maximum up to 2^8 behind at other places, which
    changes which numbers are rounded but not how far a rounding goes, 2^-8 of a probability and 2^-24 of a sum."""
    for n, past in (([5, 1, 7], [300, 20, 0]), ([100, 64], [900, 0])):
        p = Problem(4, n, past, 8, 2, 128, 64, spread=1)
        args = p.device()
        y, a, s = p.reference()
        assert np.array_equal(y, ref.attention(p.q, p.kc, p.ks, p.vc, p.vs, p.pt, p.cu, p.lens, p.scale)[0])
        for got in (mq.kv8_tree_attention(*args, p.scale), mq.kv8_attention(*args[:-1], p.scale)):
            assert (np.abs(got.float().cpu().numpy() - y) <= ref.attention_tolerance(y, a, s, 128)).all()


def test_long_histories_are_cut_and_joined():
    Problem(5, [1, 7, 4], [9000, 20, 3001], 4, 2, 64, 64).check()
    Problem(6, [60], [5000], 8, 2, 128, 16).check()
    Problem(7, [12] * 3 + [40] + [6] * 4, [4000, 0, 100, 2600, 64, 128, 3999, 1], 2, 1, 128, 16).check()
    Problem(8, [30], [6000], 8, 1, 256, 128, window=3000).check()


def test_uneven_batch_of_many_sequences():
    r = np.random.default_rng(3)
    Problem(9, [int(x) for x in r.integers(0, 9, 300)], [int(x) for x in r.integers(0, 60, 300)], 2, 1, 64, 16).check()
    Problem(10, [4] * 150 + [90] + [3] * 30, [int(x) for x in r.integers(0, 200, 181)], 4, 2, 64, 32).check()


def test_rows_that_see_nothing_are_zero():
    p = Problem(11, [3, 2, 5, 70], [0, 4, 0, 0], 4, 2, 128, 16)
    p.lens[0] = 1    # two of three tokens lie before the first place
    p.lens[2] = 0    # all of them
    p.lens[3] = 30
    p.pt[1, 0] = -1  # the only page is none
    p.check()


def test_pages_that_are_none_and_lengths_beyond_the_table():
    p = Problem(12, [1, 20, 80], [200, 100, 40], 4, 2, 64, 16)
    p.pt[0, 3], p.pt[0, 12], p.pt[1, 0], p.pt[2, 2] = -1, 2 ** 31 - 1, len(p.kc), -(2 ** 31)
    p.check()
    p = Problem(13, [2, 100], [30, 0], 4, 2, 64, 16)
    p.lens[:] = [2 ** 30, 130]
    p.check()


def test_tokens_of_no_sequence():
    p = Problem(14, [3, 4, 90], [30, 9, 0], 4, 2, 64, 16)
    p.cu[3], p.lens[2] = 50, 43
    p.check()


def test_an_empty_pool():
    from paper_2605_20315_amd import _lib
    for n in ([3, 4], [3, 90]):
        p = Problem(15, n, [30, 9], 4, 2, 64, 16)
        q, kc, ks, vc, vs, pt, cu, lens, tree = p.device()
        y, W = torch.full(q.shape, 3.0, dtype=torch.bfloat16, device="cuda"), pt.shape[1]
        rc = _lib.load().kv8_tree_attention(q.data_ptr(), 256, kc.data_ptr(), ks.data_ptr(), vc.data_ptr(), vs.data_ptr(), 0, 16, 4, 2, 64, pt.data_ptr(), W, W,
                                            cu.data_ptr(), lens.data_ptr(), 2, len(q), tree.data_ptr(), tree.shape[1], None, 0.125, 0, y.data_ptr(), 256,
                                            None, 0, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert rc == 0 and not y.any()


@pytest.mark.parametrize("D,P", [(64, 16), (128, 64), (256, 32)])
def test_nan_reaches_the_rows_that_see_it_and_no_others(D, P):
    for n, past, window in (([5, 30], [40, 70], 0), ([7, 100], [90, 3], 33), ([64], [100], 64)):
        p = Problem(D, n, past, 4, 2, D, P, window)
        for b, (m, start) in enumerate(zip(n, past)):
            for place, h, d in ((start - 1, 0, 1), (start + m // 2, 1, D - 1), (start + m - 1, 0, D // 2), (start + m // 3, 1, 7)):
                p.vc[p.pt[b, place // P], h, place % P, d] = 0x7F if d % 2 else 0xFF
            place = start + m - 2
            p.kc[p.pt[b, place // P], 1, place % P, 3] = 0x7F
        assert np.isnan(p.reference()[0]).any() and not np.isnan(p.reference()[0]).all()
        with np.errstate(invalid="ignore"):
            p.check()


def test_scores_of_minus_infinity_alone():
    p = Problem(15, [2, 40], [30, 20], 4, 2, 64, 16)
    p.q[:] = np.where(np.arange(64) == 0, np.float32(3e38), 0.0)
    p.ks[:] = 127 + 100
    p.kc[..., 0] = 0xFE  # -448
    got = mq.kv8_tree_attention(*p.device(), p.scale)
    assert got.isnan().all()


def test_strided_queries_outputs_and_tables():
    p = Problem(16, [1, 13, 100], [40, 7, 0], 4, 2, 64, 16)
    y, a, s = p.reference()
    q, kc, ks, vc, vs, pt, cu, lens, tree = p.device()
    wide = torch.full((len(q), 11, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 2:6] = q
    table = torch.full((3, pt.shape[1] + 5), 1 << 30, dtype=torch.int32, device="cuda")
    table[:, : pt.shape[1]] = pt
    out = torch.full((len(q), 9, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    mq.kv8_tree_attention(wide[:, 2:6], kc, ks, vc, vs, table[:, : pt.shape[1]], cu, lens, tree, p.scale, y=out[:, 3:7])
    assert (out[:, :3] == 5).all() and (out[:, 7:] == 5).all()
    assert (np.abs(out[:, 3:7].float().cpu().numpy() - y) <= ref.attention_tolerance(y, a, s, 64)).all()


def test_two_streams_with_a_workspace_each():
    p = Problem(17, [20, 6], [2000, 900], 8, 2, 128, 16)
    args = p.device()
    want = mq.kv8_tree_attention(*args, p.scale, workspace=torch.empty(64 << 20, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    got = []
    for _ in range(2):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            got += [mq.kv8_tree_attention(*args, p.scale, workspace=torch.empty(64 << 20, dtype=torch.uint8, device="cuda")) for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(g.view(torch.int16), want.view(torch.int16)) for g in got)


def test_refusals():
    p = Problem(18, [3, 4], [10, 10], 4, 2, 64, 16)
    *args, tree = p.device()
    for bad in (tree.long(), tree[:-1], tree.view(-1), tree.expand(7, 1).t()):
        with pytest.raises(mq.MixQuantError, match="tree"):
            mq.kv8_tree_attention(*args, bad, p.scale)
    with pytest.raises(mq.MixQuantError, match="positions"):
        mq.kv8_tree_attention(*args, tree, p.scale, positions=dev(p.positions)[:-1])
    with pytest.raises(mq.MixQuantError, match="MQ_ERR_ARG"):
        mq.kv8_tree_attention(*args, tree, 0.0)
    with pytest.raises(mq.MixQuantError, match="MQ_ERR_SHAPE"):
        mq.kv8_tree_attention(*args, torch.zeros(7, 33, dtype=torch.int32, device="cuda"), p.scale)
    with pytest.raises(mq.MixQuantError, match="shape"):
        mq.kv8_tree_attention(*args, tree, p.scale, y=torch.empty(7, 2, 64, dtype=torch.bfloat16, device="cuda"))
