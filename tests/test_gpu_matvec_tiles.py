"""nvfp4_matvec in each of its tiles (16 to 64 tokens by 32 or 64 rows of W), with and without slabs of K, and with activations brought into
LDS for wide layers: which one runs is asked on the host first."""
import pytest

import paper_2605_20315_amd as mq
import test_gpu_matvec as base

pytestmark = pytest.mark.gpu


def check(M, N, K, kernel, tile, slabs):
    plan, = mq.mq_nvfp4_matvec_launches(M, N, K)
    assert plan["kernel"] == kernel and plan["tile"] == tile and min(plan["slabs"], 2) == slabs, plan
    base.check(M + N + K, M, N, K)


@pytest.mark.parametrize("M", [5, 16, 17, 32, 33, 48, 49, 64])
def test_four_strips(M):
    check(M, 8300, 2112, "matvec", (-(-M // 16) * 16, 64), 1)


@pytest.mark.parametrize("M", [9, 20, 40, 60])
def test_four_strips_with_slabs(M):
    check(M, 2944, 10368, "matvec", (-(-M // 16) * 16, 64), 2)


@pytest.mark.parametrize("M", [16, 30, 48, 64])
def test_two_strips_with_slabs(M):
    check(M, 70, 7232, "matvec", (-(-M // 16) * 16, 32), 2)


@pytest.mark.parametrize("M", [70, 100, 129])
def test_more_than_64_tokens(M):
    check(M, 4200, 2112, "matvec", (64, 64), 1)
    check(M, 50, 9472 if M <= 128 else 14336, "matvec", (64, 32), 2)


@pytest.mark.parametrize("M,N,K", [(1, 8192, 4096), (2, 8200, 4160), (1, 8255, 6144), (2, 8193, 1088)])
def test_wide_layers_with_activations_in_lds(M, N, K):
    check(M, N, K, "matvec_lds", (16, 64), 1)


@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (4, 4000, 4160), (3, 100, 8192), (4, 8191, 1088)])
def test_narrow_layers_with_activations_in_lds(M, N, K):
    check(M, N, K, "matvec_lds", (16, 16), 1)
