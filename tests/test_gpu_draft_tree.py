"""mq_draft_tree and mq_draft_accept against their definitions: whole numbers, equal in every place."""
import numpy as np
import pytest
import torch

import _draft_ref as draft
import paper_2605_20315_amd as mq

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def sequences(seed, n, spread=9, roots=0.0):
    r = np.random.default_rng(seed)
    parents = np.array([p for m in n for p in draft.random_parents(r, m, spread, roots)], np.int32)
    cu = np.cumsum([0] + list(n)).astype(np.int32)
    return r, parents, cu, (np.array(n) + r.integers(0, 5000, len(n))).astype(np.int32)


SIZES = [[1], [60], [0, 1, 2, 31, 32, 33, 63, 64, 65, 0], [127, 5, 128, 129, 200, 255, 256, 257], [1000, 1024], [20] * 300]


@pytest.mark.parametrize("n", SIZES, ids=lambda n: f"{len(n)}x{max(n)}")
@pytest.mark.parametrize("spread,roots", [(1, 0.0), (9, 0.0), (1000, 0.1)])
@pytest.mark.parametrize("window", [0, 1, 7])
def test_tree(n, spread, roots, window):
    _, parents, cu, lens = sequences(len(n), n, spread, roots)
    for words in {-(-max(n) // 32), min(32, max(n) // 32 + 3)}:
        want = draft.tree(parents, cu, lens, words, window)
        got = mq.mq_draft_tree(ints(parents), ints(cu), ints(lens), words, window)
        for g, w in zip(got, want):
            assert np.array_equal(g.cpu().numpy(), w)


def test_tree_of_more_tokens_than_bits():
    _, parents, cu, lens = sequences(1, [100, 40, 1500])
    for words in (1, 2, 32):
        for g, w in zip(mq.mq_draft_tree(ints(parents), ints(cu), ints(lens), words), draft.tree(parents, cu, lens, words)):
            assert np.array_equal(g.cpu().numpy(), w)


def test_parents_that_are_none():
    parents = np.array([-1, 1, 0, 7, -(2 ** 31), 2 ** 31 - 1, 3, 0, 0, 2], np.int32)
    cu, lens = np.array([0, 4, 10], np.int32), np.array([4, 2], np.int32)
    for g, w in zip(mq.mq_draft_tree(ints(parents), ints(cu), ints(lens), 1), draft.tree(parents, cu, lens, 1)):
        assert np.array_equal(g.cpu().numpy(), w)


def test_rows_of_no_sequence_are_left():
    _, parents, cu, lens = sequences(2, [5, 9])
    parents = np.concatenate([parents, [0, 0, 0]]).astype(np.int32)
    tree, positions = torch.full((17, 2), 77, dtype=torch.int32, device="cuda"), torch.full((17,), 78, dtype=torch.int32, device="cuda")
    got = mq.mq_draft_tree(ints(parents), ints(cu), ints(lens), 2, tree=tree, positions=positions)
    assert got[0] is tree and got[1] is positions
    want = draft.tree(parents[:14], cu, lens, 2)
    assert np.array_equal(tree[:14].cpu().numpy(), want[0]) and np.array_equal(positions[:14].cpu().numpy(), want[1])
    assert (tree[14:] == 77).all() and (positions[14:] == 78).all()


@pytest.mark.parametrize("n", SIZES, ids=lambda n: f"{len(n)}x{max(n)}")
@pytest.mark.parametrize("kinds", [2, 5, 100000])
def test_accept(n, kinds):
    for seed in range(3):
        r, parents, cu, lens = sequences(seed, n)
        T = len(parents)
        tokens, sampled = (r.integers(0, kinds, T).astype(np.int32) for _ in "ab")
        for b, m in enumerate(n):  # most parents want one of their children
            for i in range(1, m):
                if r.random() < 0.7:
                    sampled[cu[b] + parents[cu[b] + i]] = tokens[cu[b] + i]
        got = mq.mq_draft_accept(*(ints(x) for x in (parents, tokens, sampled, cu, lens)))
        for name, g, w in zip(("path", "counts", "next", "lens"), got, draft.accept(parents, tokens, sampled, cu, lens)):
            assert np.array_equal(g.cpu().numpy(), w), name


def test_accept_a_whole_chain_and_nothing():
    n = 300
    parents, cu, lens = np.arange(-1, n - 1), [0, n], [n + 7]
    tokens = np.arange(n)
    for sampled, count in ((tokens + 1, n), (tokens + 2, 1), (np.where(tokens == 150, -5, tokens + 1), 151)):
        path, counts, following, out = mq.mq_draft_accept(*(ints(x) for x in (parents, tokens, sampled, cu, lens)))
        assert counts.tolist() == [count] and out.tolist() == [7 + count] and following.tolist() == [int(sampled[count - 1])]
        assert path.tolist() == list(range(count)) + [-1] * (n - count)


def test_accept_without_tokens_and_rows_of_no_sequence():
    path = torch.full((5,), 9, dtype=torch.int32, device="cuda")
    z = ints([0, 0, 0, 0, 0])
    got = mq.mq_draft_accept(ints([-1, 0, 0, 0, 0]), z, z, ints([0, 0, 2, 2]), ints([12, 1, 0]), path=path)
    assert got[0] is path and path.tolist() == [0, 1, 9, 9, 9]
    assert [g.tolist() for g in got[1:]] == [[0, 2, 0], [-1, 0, -1], [12, 1, 0]]
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert [g.tolist() for g in mq.mq_draft_accept(none, none, none, ints([0, 0]), ints([3]))] == [[], [0], [-1], [3]]


def test_refusals():
    i = ints([0, 1, 2])
    with pytest.raises(mq.MixQuantError, match="words"):
        mq.mq_draft_tree(i, ints([0, 3]), i[:1], 2, tree=torch.zeros(3, 3, dtype=torch.int32, device="cuda"))
    with pytest.raises(mq.MixQuantError, match="MQ_ERR_SHAPE"):
        mq.mq_draft_tree(i, ints([0, 3]), i[:1], 33)
    for bad in (i.long(), i[::2], i[:2], i.view(1, 3)):
        with pytest.raises(mq.MixQuantError, match="tokens"):
            mq.mq_draft_accept(i, bad, i, ints([0, 3]), i[:1])
    with pytest.raises(mq.MixQuantError, match="cu_q"):
        mq.mq_draft_accept(i, i, i, i, i[:1])
