"""mq_sample where a border or a draw falls exactly between two tokens.

With weights w = exp of different algebraic numbers, sums of which are equal only where every weight occurs equally often in both, that is so
where all tokens that count have the same logit, or where what lies in front of the draw is a like share of every logit's tokens.
"""
import numpy as np
import pytest
import torch

import _draft_ref as draft
import paper_2605_20315_amd as mq
from test_gpu_sample import check

pytestmark = pytest.mark.gpu

TYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
EIGHTHS = np.arange(256) / 8  # exact in BF16


def dev(x, dtype=torch.float32):
    return torch.from_numpy(np.array(x, np.float32)).to(dtype).cuda()


def sampled(x, u, dtype, **have):
    """Tokens of rows that all have the same settings."""
    rows = len(x)
    more = {k: torch.full((rows,), v, dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda") for k, v in have.items()}
    return mq.mq_sample(dev(x, dtype), dev(np.broadcast_to(np.float32(u), (rows,))), **more).cpu().numpy()


# ------------------------------------------------------------------------------------------------ the border of top_p

@TYPES
@pytest.mark.parametrize("n", [2, 4, 8, 1000])
@pytest.mark.parametrize("p", [0.25, 0.5, 0.75])
def test_top_p_keeps_a_whole_number_of_equal_logits(p, n, dtype):
    """before < top_p * mass is not so for the token with before = top_p * mass."""
    want = int(np.ceil(p * n)) - 1
    for temperature in (1.0, 0.7):
        got = sampled(np.repeat(EIGHTHS[:, None], n, 1), 1 - 2 ** -24, dtype, top_p=p, temperature=temperature)
        assert (got == want).all(), np.flatnonzero(got != want)[:8]


@TYPES
@pytest.mark.parametrize("V", [8192, 8193, 40000])
@pytest.mark.parametrize("rest", [-np.inf, -1e4, -60.0])
def test_top_p_among_few_equal_candidates(rest, V, dtype):
    """All other tokens masked, or of no weight."""
    r = np.random.default_rng(V)
    for n, p in ((2, 0.5), (4, 0.25), (4, 0.75), (8, 0.5), (200, 0.5)):
        x = EIGHTHS[::8, None] + np.full((1, V), rest)
        at = np.sort(r.choice(V, n, replace=False))
        x[:, at] = EIGHTHS[::8, None]
        got = sampled(x, 1 - 2 ** -24, dtype, top_p=p)
        assert (got == at[int(p * n) - 1]).all(), (n, p)


@TYPES
@pytest.mark.parametrize("V", [30, 8192, 20000])
def test_top_p_of_the_first_k_where_those_are_equal(V, dtype):
    x = np.repeat(EIGHTHS[::4, None], V, 1)
    x[:, 7::2] -= 1.0
    for k, p in ((2, 0.5), (4, 0.25), (8, 0.75)):
        even = [i for i in range(V) if i < 7 or i % 2 == 0]  # those of the largest logit
        got = sampled(x, 1 - 2 ** -24, dtype, top_k=k, top_p=p)
        assert (got == even[int(k * p) - 1]).all(), (k, p)


@TYPES
def test_top_p_of_rows_of_equal_logits_is_a_number_of_them(dtype):
    """For any top_p, the smallest number of tokens that is no less than top_p times all of them."""
    r = np.random.default_rng(1)
    for V in (300, 5000, 8191, 8193, 70001, 1 << 17):
        rows = 24
        p = np.concatenate([r.random(rows - 4), [2 ** -24, 1 - 2 ** -24, 0.5, 1 / 3]]).astype(np.float32)
        x = np.repeat(r.choice(EIGHTHS, (rows, 1)), V, 1)
        u = np.full(rows, 1 - 2 ** -24, np.float32)
        got = mq.mq_sample(dev(x, dtype), dev(u), top_p=dev(p)).cpu().numpy()
        kept = np.ceil(p.astype(np.float64) * V)  # 24 bits times 20: exact
        assert (got == np.floor(u.astype(np.float64) * kept)).all()


@TYPES
def test_top_p_of_nearly_equal_logits(dtype):
    """The largest bin of logits holds others than the largest: no number of equal ones."""
    r = np.random.default_rng(2)
    for V in (6, 400, 9000):
        x = np.full((32, V), 2.0)
        x[:, 1::2] = 2.0 - 2.0 ** -6
        x[:, 3 : 3 + V // 4] = -3.0
        for have in ({}, {"top_k": np.full(32, 3, np.int32)}, {"top_k": r.integers(2, V, 32).astype(np.int32)}):
            check(dev(x, dtype), r.random(32).astype(np.float32), {"top_p": r.uniform(0.1, 0.9, 32).astype(np.float32), **have})


# ------------------------------------------------------------------------------------------------ the draw

@TYPES
@pytest.mark.parametrize("V,parts", [(8190, 2), (6144, 2048), (8192, 8192), (7168, 1024)])
def test_draws_between_equal_logits_of_a_short_row(V, parts, dtype):
    """The lowest index with more than u of the mass up to it: with u = i / parts the token number u * V."""
    i = np.arange(256) * parts // 256
    for temperature in (1.0, 0.7):
        got = sampled(np.repeat(EIGHTHS[:, None], V, 1), i / parts, dtype, temperature=temperature)
        assert (got == i * V // parts).all(), np.flatnonzero(got != i * V // parts)[:8]
