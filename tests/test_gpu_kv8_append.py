"""kv8_append and mq_rope_table against their definitions, bit for bit (the table: against binary64)."""
import numpy as np
import pytest
import torch

import _kv8_ref as ref

pytestmark = pytest.mark.gpu


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x))
    return (t.to(dtype) if dtype else t).cuda()


def host(t):
    return t.float().cpu().numpy() if t.dtype == torch.bfloat16 else t.cpu().numpy()


def same_bits(got, want, what):
    """BF16 values or bytes, NaN equal to NaN."""
    if want.dtype == np.uint8:
        if what.endswith("codes"):  # a NaN code keeps a sign
            got, want = (np.where((x & 127) == 127, 127, x) for x in (got, want))
        assert np.array_equal(got, want), (what, np.argwhere(got != want)[:5])
    else:
        assert np.array_equal(np.isnan(got), np.isnan(want)), what
        ok = ~np.isnan(want)
        assert np.array_equal(got[ok].view(np.uint32), want[ok].view(np.uint32)), what


class Problem:
    def __init__(self, seed, q_lens, past, Hq, Hkv, D, P, rot, interleaved=False, extra_pages=2, width=None, max_pos=None):
        r = self.r = np.random.default_rng(seed)
        self.interleaved = interleaved
        T, B = sum(q_lens), len(q_lens)
        total = [a + b for a, b in zip(q_lens, past)]
        held = [max(-(-n // P), 0) for n in total]
        self.W = width or max(max(held), 1)
        pages = sum(held) + extra_pages
        order = r.permutation(pages)
        self.pt = np.full((B, self.W), -7, np.int32)
        at = 0
        for b, n in enumerate(held):
            n = min(n, self.W)
            self.pt[b, :n] = order[at : at + n]
            at += n
        self.cu = np.cumsum([0] + list(q_lens)).astype(np.int32)
        self.lens = np.array(total, np.int32)
        scale = np.exp(r.normal(0, 1.5, (T, 1, 1)))
        self.qkv = ref.bf16((r.normal(size=(T, Hq + 2 * Hkv, D)) * scale).astype(np.float32))
        self.Hq, self.Hkv = Hq, Hkv
        # what the pool holds before: any code, NaN among them, under small scales, so that some pages have to grow
        self.kc, self.vc = (r.integers(0, 256, (pages, Hkv, P, D)).astype(np.uint8) for _ in "kv")
        self.ks, self.vs = (r.integers(112, 128, (pages, Hkv)).astype(np.uint8) for _ in "kv")
        ang = np.arange(max_pos or max(max(total), 1))[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / rot) if rot else None
        self.table = np.concatenate([np.cos(ang), np.sin(ang)], 1).astype(np.float32) if rot else None
        self.positions = None

    def check(self, stream=None):
        import paper_2605_20315_amd as mq
        Hq, Hkv = self.Hq, self.Hkv
        qkv = dev(self.qkv, torch.bfloat16)
        q, k, v = qkv[:, :Hq], qkv[:, Hq : Hq + Hkv], qkv[:, Hq + Hkv :]
        cache = [dev(x) for x in (self.kc, self.ks, self.vc, self.vs)]
        args = [dev(x) for x in (self.pt, self.cu, self.lens)]
        table = dev(self.table) if self.table is not None else None
        pos = dev(self.positions) if self.positions is not None else None
        torch.cuda.synchronize()
        out = mq.kv8_append(q, k, v, *cache, *args, table, pos, self.interleaved)
        torch.cuda.synchronize()
        want_cache = [x.copy() for x in (self.kc, self.ks, self.vc, self.vs)]
        want = ref.append(self.qkv[:, :Hq], self.qkv[:, Hq : Hq + Hkv], self.qkv[:, Hq + Hkv :], *want_cache, self.pt, self.cu, self.lens,
                          self.table, self.positions, self.interleaved)
        owned = slice(0, int(self.cu[-1]))
        same_bits(host(out)[owned], want[owned], "queries")
        for name, got, w in zip(("k codes", "k scales", "v codes", "v scales"), cache, want_cache):
            same_bits(host(got), w, name)
        return out, cache


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_tokens_into_pages_of_every_size(D, P):
    # one token a sequence: into an empty page, behind others, the last place, the first place of the next page
    Problem(D + P, [1, 1, 1, 1, 1], [0, 5, P - 1, P, 3 * P + 7], 4, 2, D, P, D).check()
    # prompts: shorter than a page, exactly one, ending inside one, starting inside one
    Problem(D * P, [P - 1, P, 2 * P + 3, 3 * P + 1], [0, 0, 0, P // 2], 4, 2, D, P, D).check()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(64, 16), (64, 48), (128, 32), (128, 64), (128, 0), (256, 128), (256, 112)])
def test_part_of_the_head_rotated(D, rot, interleaved):
    Problem(D + rot, [1, 70, 3], [9, 40, 0], 6, 2, D, 32, rot, interleaved).check()


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (7, 1), (5, 5), (33, 11), (64, 2)])
def test_numbers_of_heads(Hq, Hkv):
    Problem(Hq, [2, 19], [3, 0], Hq, Hkv, 128, 16, 128).check()


def test_uneven_batch_with_empty_sequences():
    r = np.random.default_rng(5)
    q = [0, 1, 0, 130, 1, 1, 17, 0] + list(r.integers(0, 4, 200))
    past = [0, 0, 50, 31, 64, 63, 1, 7] + list(r.integers(0, 90, 200))
    Problem(6, q, past, 2, 1, 64, 32, 32).check()
    # as many sequences again without any token: more than a wave looks at in one step
    Problem(7, [0] * 300 + [2] + [0] * 100 + [1], [3] * 402, 2, 1, 64, 16, 64).check()


def test_a_page_filled_token_by_token_equals_its_definition():
    # (the scale grows on the way: the codes are brought along each time)
    p = Problem(8, [1], [0], 2, 2, 128, 16, 128, max_pos=40)
    p.W, p.pt = 3, np.array([[2, 0, 1]], np.int32)
    pages = 3
    p.kc, p.vc, p.ks, p.vs = p.kc[:pages], p.vc[:pages], p.ks[:pages], p.vs[:pages]
    for n in range(36):
        p.qkv = ref.bf16((p.r.normal(size=(1, 6, 128)) * 1.3 ** n).astype(np.float32))
        p.lens = np.array([n + 1], np.int32)
        _, cache = p.check()
        p.kc, p.ks, p.vc, p.vs = (host(t) for t in cache)


def test_special_values():
    p = Problem(9, [40], [24], 2, 2, 64, 16, 0)
    tiny, huge = 2.0 ** -133, 3.38e38
    for i, x in enumerate([np.inf, -np.inf, np.nan, huge, -huge, tiny, -tiny, 0.0, -0.0, 448.0, 464.0, 1.75, 1.7578125]):
        p.qkv[i * 3, 2:, i % 64] = ref.bf16(np.float32(x))
    p.qkv[24:40, 2:] = 0.0  # a page of zeros
    p.qkv[3:8, 4:] = ref.bf16((p.r.normal(size=(5, 2, 64)) * 1e-37).astype(np.float32))
    p.check()
    # borders of the scale's exponent, values on ties of E4M3
    p = Problem(10, [64], [0], 2, 2, 64, 16, 0)
    p.qkv[:, 2:] = ref.bf16(p.r.choice([448, 450, 447, 224, 0.001953125, 0.0029296875, 17, 19, 25, 416, 432], size=(64, 4, 64)).astype(np.float32))
    p.check()


def test_positions_of_their_own_and_outside_the_table():
    p = Problem(11, [5, 3], [2, 0], 4, 2, 128, 16, 64, max_pos=10)
    p.positions = np.array([9, 0, 3, 3, 10, -1, 2 ** 31 - 1, 5], np.int32)
    p.check()


def test_pages_that_are_none_take_nothing():
    p = Problem(12, [40, 1, 20], [0, 16, 90], 2, 1, 64, 16, 64)
    p.pt[0, 1], p.pt[1, 1], p.pt[2, 6] = -1, len(p.kc), 2 ** 31 - 1
    p.check()
    # places beyond the table's width, and a stated length below the number of new tokens
    p = Problem(13, [40, 9], [0, 0], 2, 1, 64, 16, 64, width=2)
    p.lens[1] = 4
    p.table = np.concatenate([np.ones((64, 32), np.float32), np.zeros((64, 32), np.float32)], 1)
    p.check()


def test_rows_of_no_sequence_and_many_tokens_per_wave():
    p = Problem(14, [200], [3], 2, 1, 64, 128, 64)  # four waves a page of 128
    p.check()
    q = [300] + [0] * 99  # few tokens a sequence on the whole, many in one: the same wave takes a page's tokens in turns
    Problem(15, q, [77] * 100, 2, 1, 256, 128, 256).check()
    p = Problem(16, [3, 2], [0, 1], 2, 1, 64, 16, 64, max_pos=64)
    p.cu = np.array([0, 3, 4], np.int32)
    p.lens = np.array([3, 2], np.int32)
    p.check()


def test_other_stream_and_graph_replays():
    import paper_2605_20315_amd as mq
    p = Problem(17, [1] * 6, [3, 15, 16, 17, 0, 40], 4, 2, 128, 16, 128)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        p.check()
    qkv = dev(p.qkv, torch.bfloat16)
    q, k, v = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]
    state = [dev(x) for x in (p.kc, p.ks, p.vc, p.vs)]
    first = [t.clone() for t in state]
    args = [dev(x) for x in (p.pt, p.cu, p.lens)]
    table, out = dev(p.table), torch.empty(6, 4, 128, dtype=torch.bfloat16, device="cuda")
    mq.mq_init()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mq.kv8_append(q, k, v, *state, *args, table, q_out=out)
    for i in range(3):
        qkv.copy_(torch.randn_like(qkv) * (i + 1))
        for t, f in zip(state, first):
            t.copy_(f)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in state] + [out.clone()]
        for t, f in zip(state, first):
            t.copy_(f)
        eager = mq.kv8_append(q, k, v, *state, *args, table)
        assert all(torch.equal(x, y) for x, y in zip(got, state + [eager]))


@pytest.mark.parametrize("R", [16, 64, 128, 256])
def test_rope_table_against_binary64(R):
    import paper_2605_20315_amd as mq
    n = 5000

    def close(t, freq, gain=1.0):
        ang = np.arange(n)[:, None] * freq
        want = np.concatenate([np.cos(ang), np.sin(ang)], 1) * gain
        # one rounding of the function and one of the product; angles up to 5000 are off by 5000 * 2^-52 in binary64
        assert np.abs(host(t) - want).max() <= 2.0 ** -23 * gain + 1e-11

    i = np.arange(R // 2)
    f = 500000.0 ** (-2.0 * i / R)
    close(mq.mq_rope_table(n, R, 500000.0), f)
    close(mq.mq_rope_table(n, R, 500000.0, mq.MQ_ROPE_LINEAR, 4.0), f / 4)
    lo = np.floor(R * np.log(4096 / (32 * 2 * np.pi)) / (2 * np.log(500000.0)))
    hi = np.ceil(R * np.log(4096 / (2 * np.pi)) / (2 * np.log(500000.0)))
    lo, hi = np.clip([lo, hi], 0, R - 1)
    w = np.clip((i - lo) / (hi - lo if hi > lo else 0.001), 0, 1)
    close(mq.mq_rope_table(n, R, 500000.0, mq.MQ_ROPE_YARN, 4.0, 4096), f / 4 * w + f * (1 - w), 0.1 * np.log(4.0) + 1)
    close(mq.mq_rope_table(n, R, 500000.0, mq.MQ_ROPE_YARN, 4.0, 4096, gain=1.0), f / 4 * w + f * (1 - w))


def test_rope_table_of_far_positions():
    import paper_2605_20315_amd as mq
    t = host(mq.mq_rope_table(131072, 64, 10000.0))[-7:]
    ang = np.arange(131065, 131072)[:, None] * 10000.0 ** (-np.arange(32) / 32)
    assert np.abs(t - np.concatenate([np.cos(ang), np.sin(ang)], 1)).max() <= 2.0 ** -24 + 1e-9
