"""What attention over the cache launches, asked on the host."""
import pytest

import paper_2605_20315_amd as mq

FULL = 64 << 20


@pytest.mark.parametrize("T", [1, 3, 90, 5000])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_a_pool_without_pages_has_no_places(T, D):
    """Else a kernel would look into the page that it takes for a number that is none."""
    for B in (1, 40):
        for ws in (0, FULL):
            none, some = (mq.mq_kv8_attention_launches(pages, 64, 8, 2, D, 1000, B, T, ws) for pages in (0, 1))
            assert none and {p["places"] for p in none} == {0} and not any(p["cut"] for p in none)
            assert {p["places"] for p in some} == {64000}


def test_sizes_that_are_refused():
    assert mq.mq_kv8_attention_launches(4, 16, 4, 2, 64, 8, 0, 5) == mq.mq_kv8_attention_launches(4, 16, 4, 2, 64, 8, 5, 0) == []
    for bad in ((-1, 16, 4, 2, 64, 8, 1, 1), (4, 8, 4, 2, 64, 8, 1, 1), (4, 16, 5, 2, 64, 8, 1, 1), (4, 16, 4, 2, 96, 8, 1, 1), (4, 16, 4, 2, 64, -8, 1, 1),
                (4, 16, 4, 2, 64, 8, 1, 1, -1)):
        with pytest.raises(mq.MixQuantError):
            mq.mq_kv8_attention_launches(*bad)


def _by_kernel(*a):
    return {p["kernel"]: p for p in mq.mq_kv8_attention_launches(*a)}


@pytest.mark.parametrize("D", [64, 128, 256])
def test_deep_histories_beside_a_prompt_are_cut(D):
    """A prompt's tokens count for the kernel that takes them, not for the one that takes the single tokens beside it."""
    for T, B in ((2048 + 8, 9), (2048 + 30, 31), (8192 + 20, 21), (300 + 9, 10)):
        p = _by_kernel(10 ** 6, 64, 32, 8, D, 2048, B, T, FULL)
        assert p["few"]["cut"], (T, B)
        assert p["few"]["workgroups"] <= B * 4 * 8 + 2 * 768
    # and the single tokens do not count for the prompt's
    assert _by_kernel(10 ** 6, 64, 32, 8, D, 2048, 200, 1000, FULL)["many"]["cut"]


def test_large_batches_of_single_tokens_are_not_cut():
    for B in (1, 64, 150, 153):
        assert _by_kernel(10 ** 6, 64, 32, 8, 128, 2048, B, B, FULL)["few"]["cut"]
    for B in (154, 170, 191, 300):  # timed: 3 to 10 us more with the join, which finds nothing to do where lengths are alike
        assert not _by_kernel(10 ** 6, 64, 32, 8, 128, 2048, B, B, FULL)["few"]["cut"]


def test_two_tiles_of_rows_where_the_average_sequence_has_more_than_one():
    # timed: 64 sequences of 4 tokens with four query heads a key head 121 us with one tile, of 5 tokens 150 with two
    for tokens, rows in ((1, 16), (4, 16), (5, 32), (13, 32)):
        assert _by_kernel(10 ** 5, 64, 32, 8, 128, 200, 64, 64 * tokens, FULL)["few"]["rows"] == rows
        assert _by_kernel(10 ** 5, 64, 32, 8, 256, 200, 64, 64 * tokens, FULL)["few"]["rows"] == 16


def test_every_tile_of_rows_has_a_workgroup():
    import random
    r = random.Random(0)
    for _ in range(3000):
        B, Hkv, G, D = r.randint(1, 40), r.choice([1, 2, 8]), r.choice([1, 2, 3, 4, 7, 16, 17, 33, 40, 64, 65, 100, 130]), r.choice([64, 128, 256])
        edge = r.choice([1, 4, 64 // G, 64 // G + 1, 128 // G + 1, 300])
        q = [r.choice([0, 1, 1, edge, r.randint(0, edge)]) for _ in range(B)]
        T = sum(q) + r.choice([0, 0, 5])
        plan = _by_kernel(100, 16, G * Hkv, Hkv, D, 100, B, T, r.choice([0, FULL]))
        for n in q:
            assert n == 0 or plan, (B, T)
        for kernel, p in plan.items():
            if len(plan) == 2:
                own = [n for n in q if 0 < n * G <= 64] if kernel == "few" else [n for n in q if n * G > 64]
            else:
                own = [n for n in q if n]
            assert p["workgroups"] >= sum(-(-n * G // p["rows"]) for n in own) * Hkv, (q, T, G, p)
