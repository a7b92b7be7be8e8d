"""kv8_attention against its definition in binary64, within a tolerance derived from its roundings."""
import numpy as np
import pytest
import torch

import _kv8_ref as ref

pytestmark = pytest.mark.gpu


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x))
    return (t.to(dtype) if dtype else t).cuda()


class Problem:
    def __init__(self, seed, q_lens, past, Hq, Hkv, D, P, window=0):
        r = self.r = np.random.default_rng(seed)
        self.window, self.scale, self.D = window, D ** -0.5, D
        T, B = sum(q_lens), len(q_lens)
        total = [a + b for a, b in zip(q_lens, past)]
        held = [-(-n // P) for n in total]
        pages = sum(held) + 2
        order = r.permutation(pages)
        self.pt = np.full((B, max(max(held), 1)), -1, np.int32)
        at = 0
        for b, n in enumerate(held):
            self.pt[b, :n] = order[at : at + n]
            at += n
        self.cu = np.cumsum([0] + list(q_lens)).astype(np.int32)
        self.lens = np.array(total, np.int32)
        self.q = ref.bf16(r.normal(size=(T, Hq, D)).astype(np.float32) * 2)
        # every place, also those that hold no token, gets codes; NaN codes go where no query looks
        self.kc, self.vc = (ref.e4m3_code(r.normal(size=(pages, Hkv, P, D)) * 100) for _ in "kv")
        self.ks, self.vs = (r.integers(119, 123, (pages, Hkv)).astype(np.uint8) for _ in "kv")
        for b, n in enumerate(total):
            if n % P:
                last = self.pt[b, n // P]
                self.kc[last, :, n % P :], self.vc[last, :, n % P :] = 0x7F, 0xFF
        for page in order[at:]:
            self.kc[page], self.vc[page] = 0xFF, 0x7F

    def device(self):
        return [dev(self.q, torch.bfloat16)] + [dev(x) for x in (self.kc, self.ks, self.vc, self.vs, self.pt, self.cu, self.lens)]

    def reference(self):
        return ref.attention(self.q, self.kc, self.ks, self.vc, self.vs, self.pt, self.cu, self.lens, self.scale, self.window)

    def check(self, workspace="both"):
        import paper_2605_20315_amd as mq
        y, a, s = self.reference()
        tol = ref.attention_tolerance(y, a, s, self.D)
        args = self.device()
        T, Hq, D = self.q.shape
        owned = int(self.cu[-1])
        for ws in ([None, "full"] if workspace == "both" else [workspace]):
            if ws:
                n = mq.mq_kv8_attention_workspace_bytes(T, len(self.lens), Hq, self.kc.shape[1], D)
                assert 0 < n <= 64 << 20
                ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN: nothing of it may be read before it is written
            out = torch.full((T, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
            assert mq.kv8_attention(*args, self.scale, self.window, out, ws) is out
            torch.cuda.synchronize()
            got = out.float().cpu().numpy().astype(np.float64)[:owned]
            assert np.array_equal(np.isnan(got), np.isnan(y[:owned]))  # NaN where the definition says so, and nowhere else
            off = np.abs(got - y[:owned])
            bad = ~np.isnan(got) & ~(off <= tol[:owned])
            assert not bad.any(), (ws is not None, np.argwhere(bad)[:4], off[bad][:4], tol[:owned][bad][:4])
            again = mq.kv8_attention(*args, self.scale, self.window, workspace=ws)
            assert torch.equal(again[:owned].view(torch.int16), out[:owned].view(torch.int16))  # the same sums in the same order


LENGTHS = [0, 1, 2, 14, 15, 16, 30, 31, 32, 33, 62, 63, 64, 65, 127, 128, 200, 511]


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_one_token_after_histories_of_many_lengths(D, P):
    Problem(D + P, [1] * len(LENGTHS), LENGTHS, 8, 2, D, P).check()


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 1), (7, 7), (28, 4), (36, 3), (40, 2)])
def test_groups_of_heads(Hq, Hkv):
    Problem(Hq, [1, 2, 9], [77, 130, 0], Hq, Hkv, 128, 32).check()


@pytest.mark.parametrize("window", [1, 2, 16, 33, 64, 100, 1000])
@pytest.mark.parametrize("D", [64, 128])
def test_windows(D, window):
    Problem(window, [1, 5, 40, 1, 3], [300, 200, 0, 0, 63], 4, 2, D, 16, window).check()
    Problem(window + 1, [130, 90], [70, 0], 8, 2, D, 64, window).check()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (8, 2), (6, 1)])
def test_prompts(Hq, Hkv, D):
    Problem(D + Hq, [1, 63, 200, 17, 0, 129], [0, 0, 0, 300, 5, 64], Hq, Hkv, D, 32).check()


@pytest.mark.parametrize("P", [16, 64, 128])
def test_one_long_prompt_and_one_long_chunk(P):
    Problem(P, [700], [0], 4, 2, 128, P).check()
    Problem(P + 1, [150], [1500], 4, 1, 128, P).check()


def test_long_histories_are_cut_and_joined():
    Problem(1, [1, 1, 4], [9000, 20, 3001], 4, 2, 64, 64).check()
    Problem(2, [1] * 3 + [40] + [1] * 4, [5000, 0, 100, 2600, 64, 128, 4999, 1], 2, 1, 128, 16).check()
    Problem(3, [2], [7000], 8, 1, 256, 128).check()


def test_uneven_batch_of_many_sequences():
    r = np.random.default_rng(3)
    Problem(4, [int(n) for n in r.integers(0, 3, 700)], [int(n) for n in r.integers(0, 60, 700)], 2, 1, 64, 16).check()
    Problem(5, [1] * 300 + [90] + [1] * 30, [int(n) for n in r.integers(0, 200, 331)], 4, 2, 64, 32).check()


def test_rows_that_see_nothing_are_zero():
    p = Problem(6, [3, 2, 5, 70], [0, 4, 0, 0], 4, 2, 128, 16)
    p.lens[0] = 1   # two of three tokens lie before the first place
    p.lens[2] = 0   # all of them
    p.lens[3] = 30
    p.pt[1, 0] = -1  # the only page is none
    p.check()


def test_pages_that_are_none_are_not_seen():
    p = Problem(7, [1, 20, 80], [200, 100, 40], 4, 2, 64, 16)
    p.pt[0, 3], p.pt[0, 12], p.pt[1, 0], p.pt[2, 2] = -1, 2 ** 31 - 1, len(p.kc), -(2 ** 31)
    p.check()


def test_a_length_beyond_the_table_ends_there():
    p = Problem(8, [2, 100], [30, 0], 4, 2, 64, 16)
    p.lens[:] = [2 ** 30, 130]
    p.check()


def test_tokens_of_no_sequence():
    p = Problem(9, [3, 4, 90], [30, 9, 0], 4, 2, 64, 16)
    p.cu[3] = 50
    p.lens[2] = 43
    p.check()


def test_extreme_scores_and_scales():
    p = Problem(10, [1, 40], [90, 200], 4, 2, 128, 16)
    p.ks[:] = 127  # scores of tens of thousands: one place takes all
    p.check()
    p = Problem(11, [1, 40], [90, 200], 4, 2, 128, 16)
    p.ks[:] = 127 - 60   # all the same
    p.vs[:] = p.r.integers(127 - 100, 127 + 100, p.vs.shape)
    p.check()
    p = Problem(12, [1, 40], [90, 200], 4, 2, 128, 16)
    p.q[:] = 0.0
    p.kc[:] = np.where(p.kc == 0x7F, 0x7F, 0)
    p.check()


def test_nan_and_infinity_reach_only_who_sees_them():
    import paper_2605_20315_amd as mq
    p = Problem(13, [1, 1, 3], [40, 40, 50], 4, 2, 64, 16)
    clean = mq.kv8_attention(*p.device(), p.scale).float().cpu().numpy()
    p.kc[p.pt[0, 1], 0, 3, 5] = 0x7F  # of sequence 0, key head 0
    p.q[1, 3] = np.inf                # of sequence 1, query head 3 alone
    p.kc[p.pt[2, 3], 1, 4, 0] = 0x7F  # place 52, the last token's own: the two before it do not see it
    got = mq.kv8_attention(*p.device(), p.scale).float().cpu().numpy()
    assert np.isnan(got[0, :2]).all() and np.array_equal(got[0, 2:], clean[0, 2:])
    assert np.isnan(got[1, 3]).all() and np.array_equal(got[1, :3], clean[1, :3])
    assert np.isnan(got[4, 2:]).all() and np.array_equal(got[4, :2], clean[4, :2]) and np.array_equal(got[2:4], clean[2:4])


@pytest.mark.parametrize("D,P", [(64, 16), (128, 64), (256, 32)])
def test_a_nan_value_reaches_the_rows_and_elements_that_see_it(D, P):
    for q_lens, past, window in (([5, 90], [40, 70], 0), ([7, 130], [90, 3], 33), ([300], [100], 64)):
        p = Problem(D, q_lens, past, 4, 2, D, P, window)
        for b, (n, start) in enumerate(zip(q_lens, past)):
            for place, h, d in ((start, 0, 1), (start + n // 2, 1, D - 1), (start + n - 1, 0, D // 2), (start + n // 3, 1, 7)):
                p.vc[p.pt[b, place // P], h, place % P, d] = 0x7F if d % 2 else 0xFF
        assert np.isnan(p.reference()[0]).any()
        with np.errstate(invalid="ignore"):
            p.check()


def test_strided_queries_outputs_and_tables():
    import paper_2605_20315_amd as mq
    p = Problem(14, [1, 33, 100], [40, 7, 0], 4, 2, 64, 16)
    y, a, s = p.reference()
    q, kc, ks, vc, vs, pt, cu, lens = p.device()
    wide = torch.full((len(q), 11, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 2:6] = q
    table = torch.full((3, pt.shape[1] + 5), 1 << 30, dtype=torch.int32, device="cuda")
    table[:, : pt.shape[1]] = pt
    out = torch.full((len(q), 9, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    mq.kv8_attention(wide[:, 2:6], kc, ks, vc, vs, table[:, : pt.shape[1]], cu, lens, p.scale, y=out[:, 3:7])
    assert (out[:, :3] == 5).all() and (out[:, 7:] == 5).all()
    assert (np.abs(out[:, 3:7].float().cpu().numpy() - y) <= ref.attention_tolerance(y, a, s, 64)).all()


def test_a_cache_beyond_4_gib():
    import paper_2605_20315_amd as mq
    p = Problem(15, [1, 20, 120], [500, 60, 100], 4, 2, 128, 64)
    pages = (5 << 30) // (2 * 64 * 128)
    shift = pages - len(p.kc)
    want = mq.kv8_attention(*p.device(), p.scale)
    q, kc, ks, vc, vs, pt, cu, lens = p.device()
    big = []
    for codes, scales in ((kc, ks), (vc, vs)):
        c = torch.empty((pages, 2, 64, 128), dtype=torch.uint8, device="cuda")
        c[shift:] = codes
        sc = torch.empty((pages, 2), dtype=torch.uint8, device="cuda")
        sc[shift:] = scales
        big += [c, sc]
    far = torch.where(pt >= 0, pt + shift, pt)
    assert torch.equal(mq.kv8_attention(q, *big, far, cu, lens, p.scale), want)
    # and the append writes there
    k = torch.randn(121 + 20, 2, 128, device="cuda").to(torch.bfloat16)
    small = [t.clone() for t in (kc, ks, vc, vs)]
    mq.kv8_append(q, k, k, *small, pt, cu, lens)
    mq.kv8_append(q, k, k, *big, far, cu, lens)
    assert all(torch.equal(b[shift:], t) for b, t in zip(big, small))


def test_other_stream_and_graph_replays():
    import paper_2605_20315_amd as mq
    p = Problem(16, [1, 2, 1, 70], [2000, 3, 100, 30], 8, 2, 128, 16)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        p.check()
    args = p.device()
    ws = torch.empty(mq.mq_kv8_attention_workspace_bytes(74, 4, 8, 2, 128), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(args[0])
    mq.mq_init()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mq.kv8_attention(*args, p.scale, 0, out, ws)
    for i in range(4):
        args[0].copy_(torch.randn_like(args[0]))
        args[7].copy_(dev(p.lens - i))  # other lengths in the same graph
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, mq.kv8_attention(*args, p.scale, 0, None, ws))


@pytest.mark.parametrize("window", [0, 1, 5, 17, 64, 200])
@pytest.mark.parametrize("Hq,Hkv,D,P", [(4, 2, 64, 16), (8, 1, 128, 64), (24, 2, 128, 16), (20, 1, 64, 128), (6, 1, 256, 32), (32, 4, 256, 16)])
def test_a_batch_of_drafted_tokens(Hq, Hkv, D, P, window):
    """One to four tokens a sequence: rows of one, two and more tiles, masks that end inside them, cut and whole histories."""
    Problem(window + D, [1, 4, 2, 3] * 3, [0, 1, 14, 29, 31, 62, 65, 127, 190, 333, 1500, 700], Hq, Hkv, D, P, window).check()


@pytest.mark.parametrize("Hq,D", [(2, 64), (5, 128), (12, 128), (9, 256)])
def test_a_nan_value_among_drafted_tokens(Hq, D):
    for window in (0, 3):
        p = Problem(D + Hq, [4, 1, 3, 4, 4], [30, 0, 61, 300, 15], Hq, 1, D, 16, window)
        for b, (n, start) in enumerate(zip([4, 1, 3, 4, 4], [30, 0, 61, 300, 15])):
            for place, d in ((start + n - 1, 1), (start + n // 2, D - 1), (start, 6)):
                p.vc[p.pt[b, place // 16], 0, place % 16, d] = 0x7F if place % 2 else 0xFF
        assert np.isnan(p.reference()[0]).any()
        with np.errstate(invalid="ignore"):
            p.check()


def test_drafted_tokens_that_see_nothing_and_pages_that_are_none():
    p = Problem(20, [4, 3, 2, 4, 1], [0, 60, 9, 40, 5], 8, 1, 128, 16)
    p.lens[0] = 2             # two of four lie before the first place
    p.lens[2] = 0
    p.pt[1, 1], p.pt[3, 2] = -1, 10 ** 6
    p.pt[4, 0] = len(p.kc)
    p.check()


def test_one_long_prompt_among_single_tokens():
    # few tokens a sequence on the whole: the prompt goes the same way as the others
    Problem(21, [1] * 60 + [170] + [1] * 20, [int(n) for n in np.random.default_rng(1).integers(0, 90, 81)], 4, 2, 64, 32).check()


@pytest.mark.parametrize("D", [64, 128, 256])
def test_a_pool_without_pages(D):
    """Every page number is none: zeros, and nothing to append to.  (An empty tensor has no address: the cache's pointers are those of another.)"""
    from paper_2605_20315_amd import _lib
    lib = _lib.load()
    codes, scales = (torch.full((4 * 128 * 256,), x, dtype=torch.uint8, device="cuda") for x in (0x38, 127))
    ws = torch.full((64 << 20,), 0xFF, dtype=torch.uint8, device="cuda")
    for q_lens in ([1], [40], [1] * 12, [300] + [2] * 11):
        B, T, W = len(q_lens), sum(q_lens), 300
        q, kv = torch.randn(T, 4, D, device="cuda").to(torch.bfloat16), torch.randn(T, 2, D, device="cuda").to(torch.bfloat16)
        pt, cu = torch.zeros(B, W, dtype=torch.int32, device="cuda"), dev(np.cumsum([0] + q_lens).astype(np.int32))
        lens = torch.full((B,), 9000, dtype=torch.int32, device="cuda")
        out = torch.empty_like(q)
        cache = [t.data_ptr() for t in (codes, scales, codes, scales)]
        assert lib.kv8_append(q.data_ptr(), 4 * D, kv.data_ptr(), 2 * D, kv.data_ptr(), 2 * D, out.data_ptr(), *cache, 0, 32, 4, 2, D, pt.data_ptr(), W, W,
                              cu.data_ptr(), lens.data_ptr(), B, T, None, 0, 0, None, 0, torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(out, q)
        for bytes_ in (0, ws.numel()):
            y = torch.full((T, 4, D), float("nan"), dtype=torch.bfloat16, device="cuda")
            assert lib.kv8_attention(q.data_ptr(), 4 * D, *cache, 0, 32, 4, 2, D, pt.data_ptr(), W, W, cu.data_ptr(), lens.data_ptr(), B, T, 0.125, 0,
                                     y.data_ptr(), 4 * D, ws.data_ptr() if bytes_ else None, bytes_, torch.cuda.current_stream().cuda_stream) == 0
            assert (y == 0).all()
    assert (codes == 0x38).all() and (scales == 127).all()


@pytest.mark.parametrize("D", [64, 128])
def test_windows_of_lengths_beyond_the_table(D):
    """The places of the tokens count on past the table's W * P, so that a window of that many still leaves some out."""
    for q_lens, past, lens in (([1, 3], [60, 61], [100, 64]), ([1] * 9 + [90], [63] * 10, [64 + 8 * b for b in range(9)] + [2 ** 20]),
                               ([70], [0], [120]), ([2], [3000], [3500])):
        places = (max(a + b for a, b in zip(q_lens, past)) + 15) // 16 * 16
        for window in (1, places // 2, places - 1, places, places + 1, 2 * places):
            p = Problem(D + window, q_lens, past, 4, 2, D, 16, window)
            assert p.pt.shape[1] * 16 == places
            p.pt[:] = p.r.permutation(len(p.kc))[: p.pt.size].reshape(p.pt.shape) if p.pt.size <= len(p.kc) else p.r.integers(0, len(p.kc), p.pt.shape)
            p.kc[:], p.vc[:] = (ref.e4m3_code(p.r.normal(size=p.kc.shape) * 100) for _ in "kv")
            p.lens[:] = lens
            p.check()


def test_windows_larger_than_any_place():
    import paper_2605_20315_amd as mq
    p = Problem(30, [1, 40, 5, 90], [30, 0, 200, 70], 4, 2, 64, 16)
    p.lens[1] = 11  # rows before the first place
    args = p.device()
    want = mq.kv8_attention(*args, p.scale)
    for window in (2 ** 31 - 2, 2 ** 31 - 1, 2 ** 31, 2 ** 40, -1, -(2 ** 40)):
        assert torch.equal(mq.kv8_attention(*args, p.scale, window).view(torch.int16), want.view(torch.int16)), window


@pytest.mark.parametrize("D", [64, 128, 256])
def test_rows_whose_scores_are_all_minus_infinity_are_nan(D):
    """As their softmax is; rows that see no place stay zero, and all others are what they are."""
    for q_lens, past, window in (([1, 1, 4], [0, 200, 40], 0), ([1, 2, 1], [5000, 3, 300], 0), ([40, 90, 5], [2600, 10, 0], 0), ([3, 70], [90, 100], 20),
                                 ([1] * 9 + [130], list(range(0, 900, 100)) + [2600], 0)):
        p = Problem(D + len(q_lens), q_lens, past, 4, 2, D, 16, window)
        p.kc[..., 5] = np.where((p.kc[..., 5] & 127) == 127, p.kc[..., 5], p.kc[..., 5] & 127 | 8)  # positive, and zero nowhere
        p.q[::2, 1, 5] = p.q[1::3, 2, 5] = -np.inf
        p.lens[1] = min(p.lens[1], q_lens[1] - 1) if q_lens[1] > 1 else p.lens[1]  # its first row sees nothing
        with np.errstate(invalid="ignore"):
            assert np.isnan(p.reference()[0]).any()
            p.check()


@pytest.mark.parametrize("Hq,Hkv,D", [(4, 2, 64), (8, 2, 128), (2, 1, 256), (20, 1, 128)])
def test_deep_histories_beside_a_prompt(Hq, Hkv, D):
    """More than eight sequences: two kernels, both of which cut histories."""
    import paper_2605_20315_amd as mq
    q_lens, past = [150] + [1, 2, 1, 3, 1, 1, 1, 1, 1, 0, 1], [2000, 3000, 1700, 0, 2600, 1, 90, 64, 2048, 31, 5, 1000]
    p = Problem(D, q_lens, past, Hq, Hkv, D, 16)
    plan = mq.mq_kv8_attention_launches(len(p.kc), 16, Hq, Hkv, D, p.pt.shape[1], len(q_lens), sum(q_lens), 64 << 20)
    assert [x["kernel"] for x in plan] == ["few", "many"] and all(x["cut"] for x in plan)
    p.check()
