"""kv8_tree_attention where every score that a row sees is a very low number: the softmax goes by differences."""
import numpy as np
import pytest
import torch

import _kv8_ref as ref
import paper_2605_20315_amd as mq
from test_gpu_kv8_tree_attention import Problem, dev
from test_gpu_kv8_tree_tiles import wide

pytestmark = pytest.mark.gpu


def lowered(p, exponents):
    """Scores of -2^(60 + e) at the places of page i, e = exponents[i]: of the queries' and keys' elements only the first is not zero."""
    p.q[:], p.kc[:] = 0.0, 0
    p.q[..., 0], p.kc[..., 0] = 2.0 ** 60, 0xB8  # -1
    p.scale = 1.0
    for b in range(len(p.lens)):
        for i, page in enumerate(p.pt[b]):
            if 0 <= page < len(p.ks):
                p.ks[page] = 127 + exponents[min(i, len(exponents) - 1)]
    return p


def check(p):
    """Probabilities are 0 or the same for all of the highest scores, which are exact: what is left to round are the sums, the probabilities' sum and y."""
    y, a, _ = p.reference()
    tol = ref.attention_tolerance(y, a, np.zeros(y.shape[:2] + (1,)), p.D)
    positions = None if p.positions is None else dev(p.positions)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    for workspace in (None, ws):
        got = mq.kv8_tree_attention(*p.device(), p.scale, p.window, positions, workspace=workspace).float().cpu().numpy()
        assert np.isfinite(got).all()
        assert (np.abs(got - y) <= tol).all(), np.argwhere(np.abs(got - y) > tol)[:4]


@pytest.mark.parametrize("exponents", [[62], [64], [66, 62], [62, 66], [64, 64, 62, 66], [60], [61, 59], [59, 60, 61, 20]], ids=str)
@pytest.mark.parametrize("D,P", [(64, 16), (128, 64), (256, 32)])
def test_scores_about_the_lowest(D, P, exponents):
    check(lowered(Problem(D + P, [9, 40], [300, 77], 8, 2, D, P), exponents))
    check(lowered(Problem(D + P, [1, 3], [0, 5], 8, 2, D, P), exponents))
    check(lowered(wide(Problem(D + P, [30, 20], [90, 500], 8, 2, D, P)), exponents))


def test_rows_that_see_one_place():
    p = lowered(Problem(3, [20], [0], 4, 2, 128, 16), [62])
    p.tree[:] = 0
    for i in range(20):
        p.tree[i, 0] = 1 << (i * 7 % 20)
    check(p)


def test_long_histories_in_parts():
    check(lowered(Problem(5, [12, 3], [5000, 900], 8, 2, 128, 64), [62, 62, 61, 63, 62]))
