"""Attention of trees: what lies in slots behind a request's last row changes neither its results nor the way they are computed."""
import pytest
import torch

import test_gpu_tree_attention as trees
from gpu_utils import announce
from plain_attention import slots

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def fsr():
    import paper_2604_20503_amd as f
    f.load_library()
    return f


@pytest.mark.parametrize("token_major", [False, True])
@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("D,P", [(128, 16), (128, 5), (64, 64)])
def test_free_slots(fsr, D, P, dtype, out_dtype, token_major):
    """Zeros, NaN or infinities there: the results are the same bit for bit, since sums are added in the same order."""
    announce(f"tree attention, free slots: {D} {P} {dtype} {out_dtype} token_major={token_major}")
    b = trees.Batch(61, [(300, 20), (0, 9), (63, 1), (64, 65), (777, 12), (15, 1), (130, 62)], 8, 2, D, P, dtype, token_major)
    kf, vf = b.k.flatten(0, 1), b.v.flatten(0, 1)
    free = torch.ones(kf.shape[0], dtype=torch.bool)
    for i, (c, n) in enumerate(b.reqs):
        free[slots(b.bt[i], c + n, P)] = False
    first = None
    for x in (0.0, float("nan"), float("inf"), -float("inf"), 3e38):
        kf[free], vf[free] = x, x
        got = b.run(fsr, out_dtype)
        first = first or got
        assert torch.equal(got[0], first[0]) and torch.equal(got[1], first[1]), x
    b.compare("free slots", first)
