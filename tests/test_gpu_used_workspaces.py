"""The attention over latent caches and behind shared prefixes takes nothing from what a workspace held before: bytes of every kind in it
leave the results as they are, bit for bit."""
import pytest
import torch

import test_gpu_latent as latent
import test_gpu_latent_expanded as expanded
import test_gpu_shared_prefix as shared
from gpu_utils import announce

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
BYTES = [0x00, 0xFF, 0x01, 0x41, 0x7F]  # numbers: zeros, NaN and -1, small ones with every fourth bit, ordinary, the largest


@pytest.fixture(scope="module")
def fsr():
    import paper_2604_20503_amd as f
    f.load_library()
    return f


def same_for_all(need, run):
    first = None
    for byte in BYTES:
        ws = torch.full((need,), byte, dtype=torch.uint8, device="cuda")
        got = run(ws)
        first = first or got
        assert all(torch.equal(x, y) for x, y in zip(got, first)), f"workspace of bytes {byte:#x}"
    return first


@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("case", shared.CASES, ids=[c[0] for c in shared.CASES])
def test_shared(fsr, case, dtype, out_dtype):
    announce(f"shared prefix, used workspace: {case} {dtype} {out_dtype}")
    b = shared.Batch(1, *case[1:], dtype)
    need = fsr.shared_workspace_bytes(N_cap=b.N + 2, H_q=b.H_q, H_kv=b.H_kv, D=b.D, dtype=dtype, out_dtype=out_dtype)
    b.compare(case[0], same_for_all(need, lambda ws: b.run(fsr, out_dtype, workspace=ws)))


@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (F32, F32)])
@pytest.mark.parametrize("ctx,rows", [([9000], [2]), ([777], [1]), ([10, 600, 40, 8], [1, 3, 2, 1]), ([300, 20], [19, 30])])
def test_latent(fsr, ctx, rows, dtype, out_dtype):
    announce(f"latent attention, used workspace: {ctx} {rows} {dtype}")
    b = latent.Batch(1, ctx, rows, 16, 512, 64, 16, dtype)
    need = fsr.latent_workspace_bytes(N_cap=b.N, H=16, D_latent=512, D_rope=64, dtype=dtype, out_dtype=out_dtype)
    latent.compare("used workspace", b, same_for_all(need, lambda ws: latent.run(fsr, b, out_dtype, workspace=ws)))


@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (F32, F32)])
@pytest.mark.parametrize("rows,keys", [([40], [2500]), ([3, 0, 200], [70, 5, 900])])
def test_expanded(fsr, rows, keys, dtype, out_dtype):
    announce(f"latent expanded, used workspace: {rows} {keys} {dtype}")
    b = expanded.Batch(1, rows, keys, 2, expanded.BIG, dtype)
    need = fsr.expanded_workspace_bytes(N_cap=b.q.shape[0], H=2, D_nope=128, D_rope=64, D_v=128, dtype=dtype, out_dtype=out_dtype)
    b.compare("used workspace", same_for_all(need, lambda ws: b.run(fsr, out_dtype, workspace=ws)))


@pytest.mark.parametrize("rows,ctx", [([8, 7, 8, 8, 6, 8, 8, 7, 8, 8, 8, 8, 8, 5, 8, 8, 8, 8, 1, 8], range(5, 405, 20)), ([200], [70]), ([1] * 250 + [9], [3] * 250 + [300])])
def test_more_row_tiles_than_workgroups(fsr, rows, ctx):
    """Pieces in several rounds, a request of many row tiles, more requests than fit one round."""
    announce(f"latent attention, row tiles in rounds: {rows} {list(ctx)}")
    b = latent.Batch(2, list(ctx), rows, 128, 512, 64, 16, BF)
    need = fsr.latent_workspace_bytes(N_cap=b.N, H=128, D_latent=512, D_rope=64, dtype=BF, out_dtype=BF)
    latent.compare("rounds", b, same_for_all(need, lambda ws: latent.run(fsr, b, BF, workspace=ws)))
