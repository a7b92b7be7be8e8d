"""The native call forms of the operators on drafted tokens against the general path: the same tensors, and the same refusals."""
import pytest
import torch

import paper_2605_20315_amd as mq
from test_gpu_kv8_binding import both, cache, heads, sequences

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def check(monkeypatch, call, native=True):
    one, two = both(monkeypatch, call, native)
    one, two = (x if isinstance(x, tuple) else (x,) for x in (one, two))
    assert len(one) == len(two) and all(torch.equal(a, b) and a.dtype == b.dtype for a, b in zip(one, two))


def test_tree(monkeypatch):
    args = ints([-1, -1, 0, 1]), ints([0, 1, 4]), ints([20, 30])
    check(monkeypatch, lambda: mq.mq_draft_tree(*args, 1))
    check(monkeypatch, lambda: mq.mq_draft_tree(*args, 2, window=1))
    tree, positions = torch.empty(4, 2, dtype=torch.int32, device="cuda"), torch.empty(4, dtype=torch.int32, device="cuda")
    check(monkeypatch, lambda: mq.mq_draft_tree(*args, 2, tree=tree, positions=positions))
    assert mq.mq_draft_tree(*args, 2, tree=tree, positions=positions)[0] is tree


def test_accept(monkeypatch):
    args = ints([-1, -1, 0, 1]), ints([5, 6, 7, 8]), ints([1, 7, 8, 9]), ints([0, 1, 4]), ints([20, 30])
    check(monkeypatch, lambda: mq.mq_draft_accept(*args))
    outs = [ints([0] * n) for n in (4, 2, 2, 2)]
    check(monkeypatch, lambda: mq.mq_draft_accept(*args, *outs))
    got = mq.mq_draft_accept(*args, *outs)
    assert all(a is b for a, b in zip(got, outs)) and got[0].tolist() == [0, 0, 1, 2]


def test_attention(monkeypatch):
    q, tree = heads(4), ints([[1], [1], [3], [7]])
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    for more in ({}, {"window": 5}, {"positions": ints([19, 27, 28, 28])}, {"workspace": ws}, {"y": torch.empty_like(q)}):
        check(monkeypatch, lambda: mq.kv8_tree_attention(q, *cache(), *sequences(), tree, 0.125, **more))
    check(monkeypatch, lambda: mq.kv8_tree_attention(q, *cache(), *sequences(), tree, 0.125, window=2 ** 40), native=False)


def test_compact(monkeypatch):
    def call():
        c = cache()
        assert mq.kv8_compact(*c, *sequences(), ints([0, 0, 2, -1]), ints([1, 2])) is None
        return tuple(c)
    check(monkeypatch, call)
    assert any(not torch.equal(a, b) for a, b in zip(call(), cache()))


def test_sample(monkeypatch):
    for dtype in (torch.bfloat16, torch.float32):
        x = torch.randn(5, 901, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(dtype)
        u, f = torch.rand(5, device="cuda", generator=torch.Generator("cuda").manual_seed(2)), torch.full((5,), 0.7, device="cuda")
        ws = torch.empty(mq.mq_sample_workspace_bytes(5, 901), dtype=torch.uint8, device="cuda")
        for more in ({}, {"temperature": f}, {"top_k": ints([1, 2, 30, 0, 5])}, {"top_p": f, "min_p": f * 0.1, "workspace": ws}, {"tokens": ints([0] * 5)}):
            check(monkeypatch, lambda: mq.mq_sample(x, u, **more))
        check(monkeypatch, lambda: mq.mq_sample(x[:, 1:900], u))


def test_what_the_native_forms_leave_to_the_general_path(monkeypatch):
    def refused(call):
        def outcome():
            try:
                call()
            except (mq.MixQuantError, AssertionError) as e:
                return str(e)
            raise AssertionError("not refused")
        one, two = both(monkeypatch, outcome, native=False)
        assert one == two

    i, q = ints([0, 1, 2, 3]), heads(4)
    refused(lambda: mq.mq_draft_tree(i.long(), ints([0, 1, 4]), ints([20, 30]), 1))
    refused(lambda: mq.mq_draft_tree(i, ints([0, 4]), ints([20, 30]), 1))
    refused(lambda: mq.mq_draft_accept(i, i[:3], i, ints([0, 1, 4]), ints([20, 30])))
    refused(lambda: mq.kv8_tree_attention(q, *cache(), *sequences(), i, 0.125))
    refused(lambda: mq.kv8_compact(*cache(), *sequences(), i.float(), ints([1, 1])))
    refused(lambda: mq.mq_sample(torch.zeros(4, 9, device="cuda").half(), torch.zeros(4, device="cuda")))
    refused(lambda: mq.mq_sample(torch.zeros(4, 9, device="cuda"), torch.zeros(4, device="cuda"), top_k=i.float()))
