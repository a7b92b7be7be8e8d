"""kv8_attention of chunks of prompts whose histories are cut into parts: which kernel runs, and that it cuts, is asked on the host first."""
import numpy as np
import pytest

import paper_2605_20315_amd as mq
import test_gpu_kv8_attention as base

pytestmark = pytest.mark.gpu

FEW_ROWS, MANY_ROWS = ([40, 5, 1], [1500, 2100, 1700]), ([150, 120, 90, 200], [1500, 1800, 0, 2000])  # joined by rows, or each row by its chunks


def problem(seed, lengths, Hq, Hkv, D, P, window):
    q_lens, past = lengths
    p = base.Problem(seed, q_lens, past, Hq, Hkv, D, P, window)
    plan, = mq.mq_kv8_attention_launches(len(p.kc), P, Hq, Hkv, D, p.pt.shape[1], len(q_lens), sum(q_lens), 64 << 20)
    assert plan["kernel"] == "many" and plan["cut"]
    assert (sum(q_lens) * Hq >= 2048) == (lengths is MANY_ROWS)
    return p


@pytest.mark.parametrize("window", [0, 300, 1600])
@pytest.mark.parametrize("lengths", [FEW_ROWS, MANY_ROWS], ids=["few rows", "many rows"])
@pytest.mark.parametrize("Hq,Hkv,D,P", [(4, 2, 64, 16), (4, 1, 64, 128), (4, 1, 128, 64), (6, 3, 128, 32), (4, 2, 256, 32), (4, 1, 256, 16)])
def test_chunks_after_long_histories(Hq, Hkv, D, P, lengths, window):
    problem(D + P + window, lengths, Hq, Hkv, D, P, window).check()


@pytest.mark.parametrize("window", [0, 300])
@pytest.mark.parametrize("lengths", [FEW_ROWS, MANY_ROWS], ids=["few rows", "many rows"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_nan_values_and_pages_that_are_none_in_parts(D, lengths, window):
    p = problem(D + window, lengths, 4, 2, D, 16, window)
    for b, (n, start) in enumerate(zip(*lengths)):
        for place, h, d in ((start, 0, 1), (start + n // 2, 1, D - 1), (start // 2, 0, D // 2), (max(start - 250, 0), 1, 7)):
            p.vc[p.pt[b, place // 16], h, place % 16, d] = 0x7F if d % 2 else 0xFF
        if start:
            p.pt[b, start // 16 - 2], p.pt[b, start // 32 + 5] = -1, len(p.kc)
    assert np.isnan(p.reference()[0]).any()
    with np.errstate(invalid="ignore"):
        p.check()


@pytest.mark.parametrize("D", [64, 128, 256])
def test_rows_that_see_nothing_in_parts(D):
    p = problem(D, FEW_ROWS, 4, 2, D, 16, 0)
    p.pt[0] = -1                    # no page of the first sequence is one
    p.pt[1, :-40] = -1              # of the second, the last ones are
    p.check()
