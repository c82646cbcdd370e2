"""Attention of trees: values that are not finite among those of the context, which all rows see, and of a leaf, which its own row sees;
wherever the line of tiles is cut, with weights in one or two parts, with a weight that counts and with one that is nothing in fp32."""
import pytest
import torch

import test_gpu_tree_attention as trees
from gpu_utils import announce
from plain_attention import slots
from test_gpu_infinite_values import TYPES, compare, fsr, plant  # noqa: F401

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("workgroups", [1, 0])
@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("counts", [True, False])
@pytest.mark.parametrize("D,P", [(128, 16), (64, 5)])
@pytest.mark.parametrize("context,at", [(64, 3), (66, 62), (128, 3), (150, 130), (777, 3), (777, 330)])
def test_context(fsr, context, at, D, P, counts, dtype, out_dtype, workgroups):  # noqa: F811
    """The planted keys at `at` and behind it are seen by all rows."""
    announce(f"tree attention, infinite values: {context} {at} {D} {P} {counts} {dtype} {out_dtype} {workgroups}")
    b = trees.Batch(51, [(context, 12), (context, 3)], 4, 2, D, P, dtype)
    k, v = b.k.flatten(0, 1), b.v.flatten(0, 1)
    of = [slots(b.bt[i], c + n, P) for i, (c, n) in enumerate(b.reqs)]
    if not counts:  # a score 200 below
        b.q[..., 0], k[:, :, 0] = 16.0, 0.0
        for s in of:
            k[s[at:at + 2], :, 0] = -200.0 / (16.0 * b.scale)
    want = b.reference()
    sees_late = torch.zeros(b.N, dtype=torch.bool)
    for i, s in enumerate(of):
        x = v[s]
        plant(x, at, at + 1, len(s) - 1)  # (a request's last row is a leaf)
        v[s] = x
        sees_late[int(b.cu[i + 1]) - 1] = True
    compare("tree", *b.run(fsr, out_dtype, max_workgroups=workgroups), want, sees_late, counts, dtype)


@pytest.mark.parametrize("workgroups", [1, 0])
@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("context", [64, 128, 777])
def test_context_alone(fsr, context, sign, dtype, out_dtype, workgroups):  # noqa: F811
    """One infinite value of the context, none in the tree: no tile is looked at before its products."""
    announce(f"tree attention, one infinite value: {context} {sign} {dtype} {out_dtype} {workgroups}")
    b = trees.Batch(52, [(context, 12)], 32, 8, 128, 16, dtype)
    o, lse, A, e = b.reference()
    s = slots(b.bt[0], context + 12, 16)
    b.v.flatten(0, 1)[s[7], :, 11] = sign * float("inf")
    out, got = b.run(fsr, out_dtype, max_workgroups=workgroups)
    assert out[..., 11].eq(sign * float("inf")).all()
    rest = torch.arange(128) != 11
    trees.check("others", out[..., rest.cuda()].reshape(-1, 127), got.reshape(-1), o[..., rest].reshape(-1, 127), lse.view(-1), A[..., rest].reshape(-1, 127), e.view(-1), dtype)
