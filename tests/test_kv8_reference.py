"""The plain definitions that the GPU tests compare with, against torch's own E4M3, hand-worked values and differences.  CPU only."""
import numpy as np
import torch

import _kv8_ref as ref


def test_e4m3_against_torch():
    r = np.random.default_rng(0)
    x = (r.normal(size=200000) * np.exp(4 * r.normal(size=200000))).astype(np.float32)
    x = np.concatenate([x, ((ref.E4M3[:126] + ref.E4M3[1:127]) / 2).astype(np.float32), np.float32([0.0, -0.0, np.inf, -np.inf])])
    want = torch.from_numpy(x).clamp(-448, 448).to(torch.float8_e4m3fn)
    assert np.array_equal(ref.e4m3_code(x), want.view(torch.uint8).numpy())
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(ref.E4M3[~np.isnan(ref.E4M3)], every[~np.isnan(every)]) and np.isnan(ref.E4M3[[127, 255]]).all()
    assert np.array_equal(ref.bf16(x[:-2]), torch.from_numpy(x[:-2]).to(torch.bfloat16).float().numpy())


def test_exponent_by_hand():
    for x, e in ((448.0, 0), (449.0, 1), (896.0, 1), (1.0, -8), (1.75, -8), (1.76, -7), (0.0, -112), (1e-37, -112), (3.3e38, 119), (2.0, -7)):
        assert ref.exponent(np.array([0.0, -x, x / 2])) == e, x
    assert ref.exponent(np.array([np.inf, np.nan, 3.0])) == -7


def test_rotation_keeps_lengths_and_relative_positions():
    r = np.random.default_rng(1)
    q, k = r.normal(size=(2, 1, 64)).astype(np.float32)
    ang = np.arange(50)[:, None] * 100.0 ** (-np.arange(16) / 16)
    t = np.concatenate([np.cos(ang), np.sin(ang)], 1).astype(np.float32)
    for inter in (False, True):
        at = lambda x, p: ref.rotate(x, t[p], inter).astype(np.float64)  # noqa: E731
        assert np.allclose((at(q, 7) ** 2).sum(), (q.astype(np.float64) ** 2).sum(), rtol=2 ** -7)
        assert abs((at(q, 9) * at(k, 4)).sum() - (at(q, 45) * at(k, 40)).sum()) < 64 * 2 ** -7
        assert np.array_equal(at(q, 7)[:, 32:], q[:, 32:].astype(np.float64).astype(np.float32).astype(np.float64))
    # one pair by hand: 90 degrees take (a, b) to (-b, a)
    x = np.zeros((1, 32), np.float32)
    x[0, 0], x[0, 1], x[0, 8] = 3.0, 5.0, 7.0
    turn = np.concatenate([np.ones(8), np.zeros(8)]).astype(np.float32)
    turn[0], turn[8] = 0.0, 1.0
    half, inter = ref.rotate(x, turn, False), ref.rotate(x, turn, True)
    assert (half[0, 0], half[0, 8], half[0, 1]) == (-7.0, 3.0, 5.0) and (inter[0, 0], inter[0, 1], inter[0, 8]) == (-5.0, 3.0, 7.0)


def test_a_page_grows_by_whole_binades():
    pages = [np.zeros((1, 1, 16, 64), np.uint8), np.zeros((1, 1), np.uint8), np.zeros((1, 1, 16, 64), np.uint8), np.zeros((1, 1), np.uint8)]
    pt, x = np.zeros((1, 1), np.int32), np.zeros((1, 1, 64), np.float32)
    x[0, 0, :3] = 1.0, 0.40625, 2.0 ** -9
    ref.append(x, x, x, *pages, pt, [0, 1], [1])
    assert pages[1][0, 0] == 127 - 8 and ref.E4M3[pages[0][0, 0, 0, :3]].tolist() == [256.0, 104.0, 0.5]
    y = np.zeros_like(x)
    y[0, 0, 0] = 1000.0
    ref.append(y, y, y, *pages, pt, [0, 1], [2])
    # 2^-8 -> 2^2: 1 and 0.40625 are the same values still, 2^-9 underflows to nothing
    assert pages[1][0, 0] == 127 + 2 and (ref.E4M3[pages[0][0, 0, 0, :3]] * 4).tolist() == [1.0, 0.40625, 0.0]
    assert ref.E4M3[pages[0][0, 0, 1, 0]] * 4 == 1024.0  # 250 lies between 240 and 256


def test_attention_of_equal_keys_is_a_mean():
    r = np.random.default_rng(2)
    kc, vc = np.full((3, 1, 16, 64), ref.e4m3_code(1.0)), ref.e4m3_code(r.normal(size=(3, 1, 16, 64)))
    s = np.full((3, 1), 127, np.uint8)
    pt = np.array([[2, 0]], np.int32)
    q = r.normal(size=(2, 1, 64)).astype(np.float32)
    y, a, _ = ref.attention(q, kc, s, vc, s, pt, [0, 2], [20], 0.125)
    v = ref.E4M3[np.concatenate([vc[2, 0], vc[0, 0]])]
    assert np.allclose(y[1, 0], v[:20].mean(0)) and np.allclose(y[0, 0], v[:19].mean(0)) and np.allclose(a[1, 0], np.abs(v[:20]).mean(0))
    y = ref.attention(q, kc, s, vc, s, pt, [0, 2], [20], 0.125, 3)[0]
    assert np.allclose(y[1, 0], v[17:20].mean(0)) and np.allclose(y[0, 0], v[16:19].mean(0))


def test_the_tolerance_sees_a_mistake_of_one_place():
    # planted in the definition: a mask that is off by one place is far outside what roundings explain
    r = np.random.default_rng(3)
    kc, vc = (ref.e4m3_code(r.normal(size=(4, 1, 16, 64)) * 100) for _ in "kv")
    s = np.full((4, 1), 121, np.uint8)
    q, pt = r.normal(size=(1, 1, 64)).astype(np.float32), np.array([[0, 1, 2, 3]], np.int32)
    y, a, sc = ref.attention(q, kc, s, vc, s, pt, [0, 1], [40], 0.125)
    wrong = ref.attention(q, kc, s, vc, s, pt, [0, 1], [39], 0.125)[0]
    assert (np.abs(wrong - y) > ref.attention_tolerance(y, a, sc, 64)).any()
