"""mq_sample with a workspace of just the size asked for: refusals, both call paths, and more rows than it holds at a time."""
import numpy as np
import pytest
import torch

import paper_2605_20315_amd as mq
from test_gpu_draft_binding import check as same_by_both_paths
from test_gpu_sample import check, logits_of, settings

pytestmark = pytest.mark.gpu


def workspace(rows, V):
    """One of that size, all ones, with 4 KiB behind it that are not part of it."""
    n = mq.mq_sample_workspace_bytes(rows, V)
    whole = torch.full((n + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    return whole[:n], whole[n:]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_too_little_is_refused(dtype):
    x, u = torch.zeros(2, 9000, dtype=dtype, device="cuda"), torch.zeros(2, device="cuda")
    n = mq.mq_sample_workspace_bytes(2, 9000)
    assert n > 0
    for ws in (torch.empty(n - 1, dtype=torch.uint8, device="cuda"), torch.empty(0, device="cuda")):
        for more in ({}, {"top_p": u + 0.5}):
            with pytest.raises(mq.MixQuantError, match="MQ_ERR_SCRATCH"):
                mq.mq_sample(x, u, workspace=ws, **more)


def test_both_call_paths_with_a_workspace_and_without(monkeypatch):
    for dtype in (torch.bfloat16, torch.float32):
        x = torch.randn(5, 20003, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(dtype)
        u, f = torch.rand(5, device="cuda", generator=torch.Generator("cuda").manual_seed(2)), torch.full((5,), 0.7, device="cuda")
        k = torch.tensor([1, 2, 30, 0, 5], dtype=torch.int32, device="cuda")
        ws, behind = workspace(5, 20003)
        for more in ({}, {"temperature": f}, {"top_k": k}, {"top_p": f, "min_p": f * 0.1}):
            same_by_both_paths(monkeypatch, lambda: mq.mq_sample(x, u, **more))
            same_by_both_paths(monkeypatch, lambda: mq.mq_sample(x, u, **more, workspace=ws))
            same_by_both_paths(monkeypatch, lambda: mq.mq_sample(x[:, 1:20002], u, **more, workspace=ws))
        assert (behind == 0xFF).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_more_rows_than_one_launch_holds(dtype):
    """Rows of two parts, 64 MiB hold 1421 of them with filters: a second launch of 79."""
    r = np.random.default_rng(11)
    rows, V = 1500, 8193
    ws, behind = workspace(rows, V)
    assert len(ws) == mq.mq_sample_workspace_bytes(rows - 1, V) < rows * mq.mq_sample_workspace_bytes(1, V)
    x, u = logits_of(r, rows, V, dtype), r.random(rows).astype(np.float32)
    x[1421], x[1430, ::2], x[1440, 17] = float("-inf"), float("nan"), float("inf")
    check(x, u, settings(r, rows), ws)
    assert (behind == 0xFF).all()


def test_more_long_rows_than_one_launch_holds():
    """130 rows near the longest, 118 to a launch: the same tokens as from calls of one launch each."""
    g = torch.Generator("cuda").manual_seed(5)
    rows, V = 130, (1 << 20) - 3
    x = (2.5 * torch.randn(rows, V, device="cuda", generator=g)).to(torch.bfloat16)
    u = torch.rand(rows, device="cuda", generator=g)
    have = {"temperature": 0.5 + torch.rand(rows, device="cuda", generator=g), "top_k": torch.randint(0, 3000, (rows,), device="cuda", generator=g).int(),
            "top_p": 0.6 + 0.39 * torch.rand(rows, device="cuda", generator=g), "min_p": 0.01 * torch.rand(rows, device="cuda", generator=g)}
    ws, behind = workspace(rows, V)
    assert len(ws) < rows * mq.mq_sample_workspace_bytes(1, V)
    got = mq.mq_sample(x, u, **have, workspace=ws)
    assert (behind == 0xFF).all()
    for a, b in ((0, 65), (65, 130), (117, 119)):
        assert torch.equal(got[a:b], mq.mq_sample(x[a:b], u[a:b], **{k: v[a:b] for k, v in have.items()}))
    at = [0, 64, 117, 118, 129]
    check(x[at], u[at].cpu().numpy(), {k: v[at].cpu().numpy() for k, v in have.items()})
