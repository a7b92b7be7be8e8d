"""mq_sample against its definition in binary64: the very tokens."""
import numpy as np
import pytest
import torch

import _draft_ref as draft
import paper_2605_20315_amd as mq

pytestmark = pytest.mark.gpu

OFF = {"temperature": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0}


def logits_of(r, rows, V, dtype, kind="mixed"):
    x = 2.5 * r.normal(size=(rows, V))
    if kind == "mixed" and V > 20:
        for row in x:
            row[r.integers(0, V, 10)] += r.uniform(3, 14)
    if kind == "steps":  # few different values: many equal ones
        x = np.round(x)
    if kind == "equal":
        x[:] = 1.5
    return torch.from_numpy(x).float().to(dtype).cuda()


def settings(r, rows):
    return {"temperature": r.choice([0.0, 0.4, 0.8, 1.0, 1.7], rows).astype(np.float32), "top_k": r.choice([0, 1, 2, 7, 50, 700, 10 ** 6], rows).astype(np.int32),
            "top_p": r.choice([1.0, 0.3, 0.8, 0.95, 0.999], rows).astype(np.float32), "min_p": r.choice([0.0, 0.0, 0.01, 0.2], rows).astype(np.float32)}


def check(x, u, have, workspace=None, tokens=None):
    dev = {k: torch.from_numpy(v).cuda() for k, v in have.items()}
    got = mq.mq_sample(x, torch.from_numpy(u).cuda(), **dev, workspace=workspace, tokens=tokens)
    assert got.dtype == torch.int32
    rows = x.float().cpu().numpy()
    want = [draft.sample(row, u[i], *(have[k][i] if k in have else v for k, v in OFF.items())) for i, row in enumerate(rows)]
    bad = np.flatnonzero(got.cpu().numpy() != want)
    assert not len(bad), [(int(i), got[int(i)].item(), want[i], float(u[i]), {k: v[i] for k, v in have.items()}) for i in bad[:4]]
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("V", [1, 2, 63, 64, 65, 500, 1000, 2049, 4096, 8191, 20001, 32000, 50257, 131073])
def test_sizes(V, dtype):
    r = np.random.default_rng(V)
    rows = 40 if V < 10000 else 12
    x, u = logits_of(r, rows, V, dtype), r.random(rows).astype(np.float32)
    check(x, u, {})
    have = settings(r, rows)
    check(x, u, have)
    for name in have:
        check(x, u, {name: have[name]})
    check(x, u, {k: have[k] for k in ("temperature", "top_p")})
    check(x, u, {k: have[k] for k in ("top_k", "min_p")})


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["steps", "equal", "flat"])
def test_equal_logits_go_by_index(kind, dtype):
    for V in (7, 300, 5000, 70000):
        r = np.random.default_rng(V)
        x, u = logits_of(r, 16, V, dtype, kind), r.random(16).astype(np.float32)
        have = settings(r, 16)
        check(x, u, have)
        have["top_k"][:] = r.integers(2, V + 2, 16)
        check(x, u, {"top_k": have["top_k"]})
        check(x, u, {"top_p": np.linspace(0.01, 0.99, 16).astype(np.float32)})
        have["min_p"][:] = 0.0
        check(x, u, have)


def test_many_rows():
    r = np.random.default_rng(1)
    for rows, V in ((513, 1200), (2000, 300), (300, 9000)):
        check(logits_of(r, rows, V, torch.bfloat16), r.random(rows).astype(np.float32), settings(r, rows))


def test_the_largest_row():
    r = np.random.default_rng(2)
    for dtype in (torch.bfloat16, torch.float32):
        x = logits_of(r, 3, 1 << 20, dtype)
        check(x, r.random(3).astype(np.float32), {})
        check(x, r.random(3).astype(np.float32), {"top_p": np.float32([0.9, 0.99, 0.5]), "top_k": np.int32([0, 600000, 5])})
    check(logits_of(r, 2, 1 << 20, torch.bfloat16, "equal"), np.float32([0.25, 1 - 2 ** -24]), {"top_p": np.float32([0.5, 1.0])})


def test_draws_at_the_ends():
    r = np.random.default_rng(3)
    for V in (10, 3000):
        x = logits_of(r, 8, V, torch.float32, "flat")
        u = np.float32([0.0, -0.0, 2 ** -30, 1 - 2 ** -24, 1.0, 5.0, -3.0, np.nan])
        check(x, u, {})
        check(x, u, {"top_k": np.full(8, 4, np.int32)})
        check(x, u, {"top_p": np.full(8, 0.6, np.float32)})


def test_settings_at_the_ends():
    r = np.random.default_rng(4)
    inf, nan = np.inf, np.nan
    for V in (9, 5000, 30000):
        for name, values in (("temperature", [0.0, -0.0, -1.0, nan, inf, -inf, 1e-30, 1e-45, 1e30, 3e38, 1e-3, 100.0]),
                             ("top_k", [0, -1, -(2 ** 31), 1, 2, V - 1, V, V + 1, 2 ** 31 - 1, 3, 4, 5]),
                             ("top_p", [0.0, -1.0, nan, 1.0, 2.0, inf, 1e-30, 1 - 2 ** -24, 2 ** -20, 0.5, -inf, 1e-45]),
                             ("min_p", [0.0, -1.0, nan, 1.0, 1.5, inf, 1e-30, 1e-10, 0.9999, -inf, 1 - 2 ** -24, 0.5])):
            x, u = logits_of(r, 12, V, torch.bfloat16), r.random(12).astype(np.float32)
            check(x, u, {name: np.array(values, np.int32 if name == "top_k" else np.float32)})


def test_logits_that_are_no_numbers():
    r = np.random.default_rng(5)
    inf, nan = np.inf, np.nan
    for dtype in (torch.bfloat16, torch.float32):
        for V in (6, 700, 9001):
            x = logits_of(r, 10, V, dtype)
            x[0, :] = -inf
            x[1, :] = nan
            x[2, V // 2] = inf
            x[3, ::2] = inf
            x[4, ::3], x[4, 1] = nan, inf
            x[5, 1:] = -inf
            x[6, :-1] = nan
            x[7, ::2] = -inf
            x[8, ::2], x[8, 1::2] = 0.0, -0.0
            x[9, 0] = nan
            u = r.random(10).astype(np.float32)
            got = check(x, u, {})
            assert got[:2].tolist() == [-1, -1]
            check(x, u, {"temperature": np.zeros(10, np.float32)})
            check(x, u, {"top_k": np.full(10, 3, np.int32), "top_p": np.full(10, 0.7, np.float32)})
            check(x, u, {"min_p": np.full(10, 0.1, np.float32)})


def test_wide_ranges_of_logits():
    r = np.random.default_rng(6)
    x = torch.from_numpy((10.0 ** r.uniform(-40, 38, (8, 4000)) * r.choice([-1, 1], (8, 4000))).astype(np.float32)).cuda()
    for t in (1.0, 1e30, 1e37):
        check(x, r.random(8).astype(np.float32), {"temperature": np.full(8, t, np.float32)})
        check(x, r.random(8).astype(np.float32), {"temperature": np.full(8, t, np.float32), "top_k": np.full(8, 900, np.int32), "top_p": np.full(8, 0.9, np.float32)})


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("V", [17, 4097, 8192, 8193, 16384])
def test_rows_about_one_workgroups_size(V, dtype):
    """Rows of at most 8192 logits take one launch, longer ones three."""
    r = np.random.default_rng(V)
    for kind in ("mixed", "steps", "equal", "flat"):
        x = logits_of(r, 24, V, dtype, kind)
        x[1] = float("-inf")
        x[2] = float("nan")
        x[3, : V // 2] = float("nan")
        x[4, V // 3] = x[4, V - 1] = float("inf")
        x[5, 1:] = float("-inf")
        x[6, : V - 1] = float("-inf")
        x[7] = torch.finfo(dtype).min
        for have in ({}, settings(r, 24), {"top_p": np.full(24, 0.9, np.float32)}, {"top_k": np.full(24, 300, np.int32)},
                     {"min_p": np.full(24, 0.05, np.float32)}, {"temperature": np.zeros(24, np.float32)}):
            check(x, r.random(24).astype(np.float32), have)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_signalling_nans_are_nans(dtype):
    r = np.random.default_rng(12)
    x = logits_of(r, 12, 20001, dtype)
    small = torch.int16 if dtype == torch.bfloat16 else torch.int32
    codes = [0x7F81, 0x7FA3 - 0x10000 + 0x8000, 0x7FC1] if dtype == torch.bfloat16 else [0x7F800001, 0x7FA00000 - 2 ** 31, 0x7FC00001]
    at = torch.from_numpy(r.random((12, 20001)) < 0.3).cuda()
    at[:, 8192:16384] = True  # a part that holds nothing else
    x.view(small)[at] = torch.tensor(codes, dtype=small, device="cuda")[torch.arange(int(at.sum()), device="cuda") % 3]
    have = settings(r, 12)
    check(x, r.random(12).astype(np.float32), {})
    check(x, r.random(12).astype(np.float32), have)
    check(x, r.random(12).astype(np.float32), {"temperature": np.zeros(12, np.float32)})


def test_the_lowest_logits_at_the_border_of_a_bin():
    """Temperatures with which the lowest finite number lies just below a whole number of eighths of a power of two, and the next just above:
    the first belongs to another bin than the second, which is the last that is kept."""
    low = np.float32(np.finfo(np.float32).min)
    following = np.nextafter(low, np.float32(0))
    cases = []
    for n in range(-3000, -600, 37):
        t = np.float32(8 * np.log2(np.e) / (n / float(following)))
        for t in (t, np.nextafter(t, np.float32(0)), np.nextafter(t, np.float32(np.inf))):
            scale = 8.0 * 1.4426950408889634074 / float(t)
            if np.floor(float(low) * scale) == n - 1 and np.floor(float(following) * scale) == n:
                cases.append((t, n, scale))
    assert len(cases) > 20
    x = np.full((len(cases), 300), -np.inf, np.float32)
    for row, (_, n, scale) in zip(x, cases):
        row[7], row[10:13], row[20:25] = (n + 2.5) / scale, following, low
    have = {"temperature": np.array([t for t, _, _ in cases], np.float32), "top_k": np.full(len(cases), 4, np.int32)}
    got = check(torch.from_numpy(x).cuda(), np.full(len(cases), 0.99, np.float32), have)
    assert set(got.tolist()) == {12}
    # and 511 bins below the largest, the last that is counted
    for row, (_, n, scale) in zip(x, cases):
        row[7] = (n + 511.5) / scale
    got = check(torch.from_numpy(x).cuda(), np.full(len(cases), 0.99, np.float32), {"temperature": have["temperature"], "top_p": np.full(len(cases), 0.9, np.float32)})
    assert set(got.tolist()) == {7}


@pytest.mark.parametrize("below", [448, 503, 504, 505, 510, 511, 512, 520])
def test_parts_of_a_row_that_lie_far_below_its_largest(below):
    """A part of 8192 logits so many eighths of a power of two below the largest: its mass, next to nothing, is not to move the border of top_p."""
    eighth = np.log(2.0) / 8
    rows = []
    for first in range(8):
        x = np.full(16384, -np.inf)
        x[0], x[1:51] = (32 + first + 0.5) * eighth, (32 + first + 0.5) * eighth - np.log(1000.0)
        x[8192:] = (32 + first - below + 0.5) * eighth
        rows.append(x)
    x = torch.tensor(np.array(rows), dtype=torch.float32, device="cuda")
    for p in (0.9, 0.9999, 1.0):
        got = check(x, np.full(8, 0.99, np.float32), {"top_p": np.full(8, p, np.float32)})
        assert p > 0.9 or got.tolist() == [0] * 8


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_rows_of_any_stride_and_alignment(dtype):
    r = np.random.default_rng(7)
    for V, ld, skip in ((1001, 1001, 1), (1001, 1007, 3), (5000, 5001, 5), (20000, 20003, 7), (9, 9, 1), (40001, 40001, 2)):
        whole = torch.full((12 * ld + 16,), 1000.0, dtype=dtype, device="cuda")
        x = whole[skip:].as_strided((12, V), (ld, 1))
        x.copy_(logits_of(r, 12, V, dtype))
        check(x, r.random(12).astype(np.float32), settings(r, 12))
        check(x, r.random(12).astype(np.float32), {})


def test_the_workspace_is_written_before_it_is_read_and_outputs_are_the_callers():
    r = np.random.default_rng(8)
    for rows, V in ((1, 131072), (30, 20000), (70, 700)):
        ws = torch.full((max(16, mq.mq_sample_workspace_bytes(rows, V)),), 0xFF, dtype=torch.uint8, device="cuda")
        x, u, tokens = logits_of(r, rows, V, torch.bfloat16), r.random(rows).astype(np.float32), torch.full((rows,), -7, dtype=torch.int32, device="cuda")
        assert check(x, u, settings(r, rows), ws, tokens) is tokens


def test_shares_of_draws_follow_the_weights():
    """100 000 draws of one row: each share within six standard deviations of its probability."""
    n, x = 100000, np.float32([1.0, 3.0, -2.0, 2.5, 0.0, 2.0, -9.0])
    got = mq.mq_sample(torch.from_numpy(x).cuda().expand(n, 7).contiguous(), torch.rand(n, device="cuda", generator=torch.Generator("cuda").manual_seed(1)),
                       torch.full((n,), 0.7, device="cuda"), torch.full((n,), 5, dtype=torch.int32, device="cuda"))
    p = np.exp(x.astype(np.float64) / 0.7)
    p[[2, 6]] = 0.0
    p /= p.sum()
    share = np.bincount(got.cpu().numpy(), minlength=7) / n
    assert (np.abs(share - p) <= 6 * np.sqrt(p * (1 - p) / n)).all(), (share, p)


def test_refusals():
    x, u = torch.zeros(3, 50, device="cuda"), torch.zeros(3, device="cuda")
    with pytest.raises(mq.MixQuantError, match="BF16 or FP32"):
        mq.mq_sample(x.half(), u)
    for bad in (x.t(), x[0], x[:, ::2]):
        with pytest.raises(mq.MixQuantError):
            mq.mq_sample(bad, u)
    for name, bad in (("uniform", u[:2]), ("uniform", u.double())):
        with pytest.raises(mq.MixQuantError, match=name):
            mq.mq_sample(x, bad)
    for name in ("temperature", "top_p", "min_p"):
        with pytest.raises(mq.MixQuantError, match=name):
            mq.mq_sample(x, u, **{name: u.int()})
    with pytest.raises(mq.MixQuantError, match="top_k"):
        mq.mq_sample(x, u, top_k=u)
    with pytest.raises(mq.MixQuantError, match="MQ_ERR_SHAPE"):
        mq.mq_sample(torch.zeros(1, (1 << 20) + 1, device="cuda"), u[:1])
    if mq.mq_sample_workspace_bytes(3, 50):
        with pytest.raises(mq.MixQuantError, match="MQ_ERR_SCRATCH"):
            mq.mq_sample(x, u, workspace=torch.empty(mq.mq_sample_workspace_bytes(3, 50) - 1, dtype=torch.uint8, device="cuda"))
    assert mq.mq_sample(x[:0], u[:0]).shape == (0,)
