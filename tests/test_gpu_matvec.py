"""nvfp4_matvec against binary64, within a tolerance derived from its roundings: products are exact, a binary32 sum of K terms is
off by at most K * 2^-24 of the sum of their magnitudes, the factor alpha and a BF16 result round once more."""
import numpy as np
import pytest
import torch

import _kv8_ref as ref

pytestmark = pytest.mark.gpu


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x))
    return (t.to(dtype) if dtype else t).cuda()


def problem(seed, M, N, K):
    r = np.random.default_rng(seed)
    x = ref.bf16((r.normal(size=(M, K)) * np.exp(r.normal(size=(M, 1)))).astype(np.float32))
    codes, scales = r.integers(0, 256, (N, K // 2)).astype(np.uint8), r.integers(0, 127, (N, K // 16)).astype(np.uint8)
    alpha = np.array([0.0123], np.float32)
    w = ref.dequantize(codes, scales)
    return x, codes, scales, alpha, w


def to_ktile(codes, scales):
    N, K = codes.shape[0], codes.shape[1] * 2
    return (codes.reshape(N, K // 64, 32).transpose(1, 0, 2).reshape(N, K // 2), scales.reshape(N, K // 64, 4).transpose(1, 0, 2).reshape(N, K // 16))


def close(y, x, w, alpha, out):
    want, size = x.astype(np.float64) @ w.T * float(alpha[0]), np.abs(x).astype(np.float64) @ np.abs(w).T * float(alpha[0])
    tol = (x.shape[1] + 2) * 2.0 ** -24 * size + (2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -8) if out == 0 else 0.0)
    off = np.abs(y.float().cpu().numpy().astype(np.float64) - want)
    assert (off <= tol).all(), (np.argwhere(~(off <= tol))[:4], off.max())


def check(seed, M, N, K, layouts=(0, 1), outs=(0, 1)):
    import paper_2605_20315_amd as mq
    x, codes, scales, alpha, w = problem(seed, M, N, K)
    xd, ad = dev(x, torch.bfloat16), dev(alpha)
    seen = {}
    for layout in layouts:
        if layout == 1 and K % 64:
            continue
        c, s = to_ktile(codes, scales) if layout else (codes, scales)
        for out in outs:
            y = mq.nvfp4_matvec(xd, dev(c), dev(s), ad, out, layout=layout)
            assert y.shape == (M, N) and y.dtype == (torch.float32 if out else torch.bfloat16)
            close(y, x, w, alpha, out)
            seen[layout, out] = y
    for out in outs:  # the order of the bytes changes no sum
        if (0, out) in seen and (1, out) in seen:
            assert torch.equal(seen[0, out], seen[1, out])
    if (0, 0) in seen and (0, 1) in seen:
        assert torch.equal(seen[0, 1].to(torch.bfloat16), seen[0, 0])


@pytest.mark.parametrize("K", [64, 128, 192, 448, 1024, 4160])
@pytest.mark.parametrize("N", [1, 15, 16, 17, 100, 513])
def test_shapes(N, K):
    check(N + K, 1, N, K)
    check(N + K + 1, 5, N, K)


@pytest.mark.parametrize("M", [2, 3, 4, 7, 8, 9, 15, 16, 17, 31, 32, 33, 48, 49, 64, 65, 130])
def test_numbers_of_tokens(M):
    check(M, M, 130, 640)
    check(M + 1, M, 33, 2048)


@pytest.mark.parametrize("K", [16, 48, 80, 1008, 2064])
def test_k_of_no_whole_steps(K):
    check(K, 3, 37, K)


def test_many_rows_and_a_long_k():
    check(1, 1, 20000, 256)
    check(2, 20, 9001, 128)
    check(3, 6, 40, 25600)
    check(4, 40, 24, 25600)


def test_strides_and_padding():
    import paper_2605_20315_amd as mq
    for M in (1, 3, 20):
        x, codes, scales, alpha, w = problem(M, M, 70, 256)
        wide = torch.full((M, 320), float("nan"), dtype=torch.bfloat16, device="cuda")
        wide[:, 32:288] = dev(x, torch.bfloat16)
        for out in (0, 1):
            y = torch.full((M, 77), 3.0, dtype=torch.float32 if out else torch.bfloat16, device="cuda")
            mq.nvfp4_matvec(wide[:, 32:288], dev(codes), dev(scales), dev(alpha), out, y[:, 1:71])
            close(y[:, 1:71], x, w, alpha, out)
            assert (y[:, 0] == 3).all() and (y[:, 71:] == 3).all()


def test_quantized_weights_and_values_at_the_ends():
    """What nvfp4_quantize makes of a weight matrix, and activations that FP16 would not hold."""
    import paper_2605_20315_amd as mq
    r = np.random.default_rng(0)
    wd = torch.from_numpy(r.normal(size=(96, 512)).astype(np.float32)).cuda().to(torch.bfloat16)
    alpha = mq.nvfp4_global_scale(wd)
    x = ref.bf16((r.normal(size=(4, 512)) * np.array([[1e30], [1e-30], [1.0], [0.0]])).astype(np.float32))
    for layout in (0, 1):
        codes, scales = mq.nvfp4_quantize(wd, alpha, layout=layout)
        if layout == 0:
            w = ref.dequantize(codes.cpu().numpy(), scales.cpu().numpy())
        close(mq.nvfp4_matvec(dev(x, torch.bfloat16), codes, scales, alpha, 1, layout=layout), x, w, alpha.cpu().numpy(), 1)
    x[2, 7] = np.inf
    x[0, 9] = np.nan
    y = mq.nvfp4_matvec(dev(x, torch.bfloat16), codes, scales, alpha, layout=1).float().cpu().numpy()
    assert not np.isfinite(y[0]).any() and not np.isfinite(y[2]).any() and np.isfinite(y[[1, 3]]).all()


def test_empty_and_repeated():
    import paper_2605_20315_amd as mq
    x, codes, scales, alpha, w = problem(5, 3, 40, 320)
    args = dev(codes), dev(scales), dev(alpha)
    assert mq.nvfp4_matvec(dev(x[:0], torch.bfloat16), *args).shape == (0, 40)
    xd = dev(x, torch.bfloat16)
    first = mq.nvfp4_matvec(xd, *args)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        assert torch.equal(mq.nvfp4_matvec(xd, *args), first)
    mq.mq_init()
    out = torch.empty_like(first)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mq.nvfp4_matvec(xd, *args, y=out)
    for _ in range(3):
        xd.copy_(torch.randn_like(xd))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, mq.nvfp4_matvec(xd, *args))


def test_k_in_two_slabs():
    check(5, 20, 4090, 10240)
    check(6, 5, 40, 6144)


def test_four_strips_and_slabs():
    check(7, 18, 5100, 12800)
    check(8, 70, 8200, 128)
