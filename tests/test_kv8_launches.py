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
