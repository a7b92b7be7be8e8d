"""mq_sample with a workspace of just the size asked for: refusals, and both call paths."""
import pytest
import torch

import paper_2605_20315_amd as mq
from test_gpu_draft_binding import check as same_by_both_paths

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
