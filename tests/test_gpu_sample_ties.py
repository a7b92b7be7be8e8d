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


@TYPES
@pytest.mark.parametrize("V,parts", [(16384, 16384), (12288, 4096), (1 << 17, 1 << 17), (8194, 2), (100352, 2048)])
def test_draws_between_equal_logits_of_a_long_row(V, parts, dtype):
    r = np.random.default_rng(V)
    rows = 64
    for have in ({}, {"temperature": 0.7}, {"top_k": V}, {"top_k": V // 2}, {"temperature": 0.7, "min_p": 0.5}, {"top_p": 0.5}):
        i = r.integers(0, parts, rows)
        i[:3] = 0, 1, parts - 1
        kept = V // 2 if have.get("top_k") == V // 2 or "top_p" in have else V
        got = sampled(np.repeat(r.choice(EIGHTHS, (rows, 1)), V, 1), i / parts, dtype, **have)
        assert (got == i * kept // parts).all(), (have, got[got != i * kept // parts][:4])


@TYPES
@pytest.mark.parametrize("V", [100, 8192, 16384, 24576, 32768, 50000])
def test_half_of_a_mirrored_row(V, dtype):
    """A row and its mirror image behind it: the draw of a half falls between them, whatever the logits."""
    r = np.random.default_rng(V)
    half = r.normal(size=(32, V // 2)) * 2.5
    half[8:16, : V // 3] -= 12.0   # the parts of the row lie far apart
    half[16:24, V // 3 :] -= 25.0
    half[:, -1] = 3.0
    x = dev(np.concatenate([half, half[:, ::-1]], 1), dtype)
    values = x.float().cpu().numpy()
    u = np.full(32, 0.5, np.float32)
    assert (mq.mq_sample(x, dev(u)).cpu().numpy() == V // 2).all()
    assert (mq.mq_sample(x, dev(u), dev(np.full(32, 1.7))).cpu().numpy() == V // 2).all()
    got = mq.mq_sample(x, dev(u), min_p=dev(np.full(32, 0.01))).cpu().numpy()
    top = values.max(1, keepdims=True).astype(np.float64)
    kept = np.exp(values - top) >= np.float32(0.01)
    assert (got == [V // 2 + int(np.argmax(row[V // 2 :])) for row in kept]).all()


@TYPES
def test_draws_of_zero_take_the_first_token_that_is_kept(dtype):
    r = np.random.default_rng(4)
    for V in (500, 20000, 60000):
        x = r.normal(size=(16, V)) * 3
        u = np.zeros(16, np.float32)
        for have in ({}, {"top_k": np.full(16, 5, np.int32)}, {"min_p": np.full(16, 0.2, np.float32)}, {"top_p": np.full(16, 0.8, np.float32)}):
            check(dev(x, dtype), u, have)


@TYPES
def test_the_first_of_the_kept_tokens_weighs_next_to_nothing(dtype):
    """2^-40 of the largest, in a part of the row by itself: a draw of zero takes it, as its weight is above the 2^-43 that may count as none."""
    x = np.full((4, 30000), -np.inf)
    x[:, 100], x[:, 25000] = 0.0, 28.0  # e^-28 = 2^-40.4
    for have in ({}, {"top_k": np.full(4, 5, np.int32)}, {"min_p": np.full(4, 1e-13, np.float32)}):
        assert check(dev(x, dtype), np.zeros(4, np.float32), have).tolist() == [100] * 4
        assert check(dev(x, dtype), np.full(4, 2.0 ** -20, np.float32), have).tolist() == [25000] * 4


# ------------------------------------------------------------------------------------------------ weights of one from different logits

@TYPES
@pytest.mark.parametrize("V", [8, 512, 8192, 16384])
def test_an_endless_temperature_makes_all_weights_one(V, dtype):
    """Kept are the first of the order, top_p of all of them; the draw counts tokens."""
    r = np.random.default_rng(V)
    x = dev(r.normal(size=(24, V)) * 3, dtype)
    order = np.argsort(-x.double().cpu().numpy(), axis=1, kind="stable")
    for t in (np.inf, 3e38):
        for p in (0.25, 0.5, 0.75, 1.0):
            u = r.integers(0, 8, 24) / 8
            got = mq.mq_sample(x, dev(u), temperature=dev(np.full(24, t)), top_p=dev(np.full(24, p))).cpu().numpy()
            kept = np.sort(order[:, : int(p * V)], 1)
            assert (got == kept[np.arange(24), (u * kept.shape[1]).astype(int)]).all(), (t, p)


@TYPES
def test_logits_that_are_nearly_the_same(dtype):
    """Differences of 2^-90 make weights that are one in binary64."""
    r = np.random.default_rng(6)
    for V in (8, 40, 8192, 16384):
        x = dev(2.0 ** -90 * r.normal(size=(24, V)), dtype)
        order = np.argsort(-x.double().cpu().numpy(), axis=1, kind="stable")
        for p in (0.25, 0.5, 0.75):
            u = np.full(24, 1 - 2 ** -24)
            got = mq.mq_sample(x, dev(u), top_p=dev(np.full(24, p))).cpu().numpy()
            assert (got == np.sort(order[:, : int(p * V)], 1)[:, -1]).all(), (V, p)
