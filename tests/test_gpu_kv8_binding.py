"""The native call forms of append, attention and matvec against the general path: the same tensors, and the same refusals."""
import pytest
import torch

import paper_2605_20315_amd as mq
from paper_2605_20315_amd import _lib, ops

pytestmark = pytest.mark.gpu


class _General:
    def __getattr__(self, name):
        return lambda *args: None


class _Recorder:
    def __init__(self):
        self.module, self.taken = _lib.load_binding(), []

    def __getattr__(self, name):
        def call(*args):
            result = getattr(self.module, name)(*args)
            self.taken.append(result is not None)
            return result
        return call


def both(monkeypatch, call, native=True):
    """What `call` gives through the native forms and through the general path."""
    recorder = _Recorder()
    monkeypatch.setattr(ops, "_fast", recorder)
    one = call()
    assert recorder.taken and all(recorder.taken) == native
    monkeypatch.setattr(ops, "_fast", _General())
    two = call()
    return one, two


def cache(seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = [torch.randint(0, 120, (6, 2, 16, 64), dtype=torch.uint8, device="cuda", generator=g) for _ in "kv"]
    scales = [torch.full((6, 2), 118, dtype=torch.uint8, device="cuda") for _ in "kv"]
    return [codes[0], scales[0], codes[1], scales[1]]


def sequences():
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return [ints([[5, 0], [3, 1]]), ints([0, 1, 4]), ints([20, 30])]


def heads(n, seed=1):
    return torch.randn(4, n, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(torch.bfloat16)


def test_append(monkeypatch):
    qkv = heads(8)
    q, k, v = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]
    table = mq.mq_rope_table(64, 32)
    for more in ({}, {"interleaved": True}, {"positions": torch.arange(4, dtype=torch.int32, device="cuda")}, {"q_out": torch.empty(4, 4, 64, dtype=torch.bfloat16, device="cuda")}):
        def call():
            c = cache()
            return [mq.kv8_append(q, k, v, *c, *sequences(), table, **more)] + c
        one, two = both(monkeypatch, call)
        assert all(torch.equal(a, b) for a, b in zip(one, two))
    one, two = both(monkeypatch, lambda: mq.kv8_append(q, k, v, *cache(), *sequences()))
    assert torch.equal(one, q) and torch.equal(two, q)


def test_attention(monkeypatch):
    q, c = heads(4), cache()
    for more in ({}, {"window": 5}, {"workspace": torch.empty(64 << 20, dtype=torch.uint8, device="cuda")}, {"y": torch.empty(4, 9, 64, dtype=torch.bfloat16, device="cuda")[:, 2:6]}):
        one, two = both(monkeypatch, lambda: mq.kv8_attention(q, *c, *sequences(), 0.125, **more).clone())
        assert torch.equal(one, two)
    both(monkeypatch, lambda: mq.kv8_attention(q, *c, *sequences(), 1))  # an integer is a number


def test_matvec(monkeypatch):
    w, s, alpha = torch.randint(0, 256, (48, 64), dtype=torch.uint8, device="cuda"), torch.randint(0, 100, (48, 8), dtype=torch.uint8, device="cuda"), torch.ones(1, device="cuda")
    for M in (1, 3, 20):
        x = torch.randn(M, 128, device="cuda").to(torch.bfloat16)
        for more in ({}, {"layout": mq.MQ_LAYOUT_KTILE}, {"out": mq.MQ_OUT_FP32}, {"workspace": torch.empty(1 << 20, dtype=torch.uint8, device="cuda")},
                     {"y": torch.empty(M, 50, dtype=torch.bfloat16, device="cuda")[:, 1:49]}):
            one, two = both(monkeypatch, lambda: mq.nvfp4_matvec(x, w, s, alpha, **more).clone())
            assert torch.equal(one, two)


@pytest.mark.parametrize("path", ["native", "general"])
def test_refusals(monkeypatch, path):
    if path == "general":
        monkeypatch.setattr(ops, "_fast", _General())
    q, c, s = heads(4), cache(), sequences()
    k = heads(2)
    bad = (AssertionError, mq.MixQuantError)
    for call in (
        lambda: mq.kv8_attention(q.float(), *c, *s, 0.125),                                    # types
        lambda: mq.kv8_attention(q, *c, s[0].long(), s[1], s[2], 0.125),
        lambda: mq.kv8_attention(q, *c, s[0], s[1][:-1], s[2], 0.125),                          # sizes
        lambda: mq.kv8_attention(q[..., :32], *c, *s, 0.125),
        lambda: mq.kv8_attention(heads(3), *c, *s, 0.125),                                      # three query heads on two key heads
        lambda: mq.kv8_attention(heads(8)[:, ::2], *c, *s, 0.125),                              # heads that are not adjacent
        lambda: mq.kv8_attention(q, *c, *s, 0.0),
        lambda: mq.kv8_attention(q, *c, *s, 0.125, y=torch.empty(4, 4, 64, device="cuda")),
        lambda: mq.kv8_attention(q, *c, *s, 0.125, workspace=torch.empty(8, 8, device="cuda").t()),
        lambda: mq.kv8_attention(q.cpu(), *c, *s, 0.125),
        lambda: mq.kv8_append(q, k, heads(3), *c, *s),
        lambda: mq.kv8_append(q, k, k[:3], *c, *s),
        lambda: mq.kv8_append(q, k, k, c[0], c[1][:5], c[2], c[3], *s),
        lambda: mq.kv8_append(q, k, k, *c, *s, torch.zeros(8, 24, device="cuda")),              # 24 rotated elements
        lambda: mq.kv8_append(q, k, k, *c, *s, torch.zeros(8, 128, device="cuda")),             # more than the head has
        lambda: mq.kv8_append(q, k, k, *c, *s, torch.zeros(8, 64, device="cuda", dtype=torch.float64)),
        lambda: mq.kv8_append(q, k, k, *c, *s, torch.zeros(8, 64, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")),
        lambda: mq.kv8_append(q, k, k, *c, *s, q_out=torch.empty(4, 5, 64, dtype=torch.bfloat16, device="cuda")),
        lambda: mq.nvfp4_matvec(torch.zeros(1, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(8, 64, dtype=torch.uint8, device="cuda"),
                                torch.zeros(8, 7, dtype=torch.uint8, device="cuda"), torch.ones(1, device="cuda")),
        lambda: mq.nvfp4_matvec(torch.zeros(1, 48, dtype=torch.bfloat16, device="cuda"), torch.zeros(8, 24, dtype=torch.uint8, device="cuda"),
                                torch.zeros(8, 3, dtype=torch.uint8, device="cuda"), torch.ones(1, device="cuda"), layout=mq.MQ_LAYOUT_KTILE),
        lambda: mq.nvfp4_matvec(torch.zeros(1, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(8, 32, dtype=torch.uint8, device="cuda"),
                                torch.zeros(8, 4, dtype=torch.uint8, device="cuda"), torch.ones(1, device="cuda"), out=7),
        lambda: mq.nvfp4_matvec(torch.zeros(9, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(8, 32, dtype=torch.uint8, device="cuda"),
                                torch.zeros(8, 4, dtype=torch.uint8, device="cuda"), torch.ones(1, device="cuda"),
                                workspace=torch.empty(64, dtype=torch.uint8, device="cuda")),
    ):
        with pytest.raises(bad):
            call()


def test_a_small_call_costs_little_host_time():
    """About 5 us with its output given; through the general path about 15."""
    import time
    q, c, s = heads(4), cache(), sequences()
    y = torch.empty_like(q)
    best = float("inf")
    for _ in range(20):
        torch.cuda.synchronize()
        start = time.perf_counter()
        for _ in range(50):
            mq.kv8_attention(q, *c, *s, 0.125, 0, y)
        best = min(best, (time.perf_counter() - start) / 50 * 1e6)
    assert best < 25, f"{best:.1f} us"
