"""Appends whose offsets are a piece of a longer list: rows in front of the first offset belong to no request and change nothing."""
import pytest
import torch

from gpu_utils import announce
from plain_attention import offsets, pages, slots

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def fsr():
    import paper_2604_20503_amd as f
    f.load_library()
    return f


def batch(dtype, kv8):
    """Six requests' rows, of which the last three are appended; tokens in front of each request's context have a place."""
    gen = torch.Generator().manual_seed(3)
    ctx, rows, H_q, H_kv, D, P = torch.tensor([40, 9, 70, 33, 90, 50], dtype=torch.int32), [5, 20, 3, 7, 1, 12], 4, 2, 64, 16
    bt, n_pages = pages([int(c) + n for c, n in zip(ctx, rows)], P, gen)
    normal = lambda *s: torch.randn(s, generator=gen).to(dtype)  # noqa: E731
    q, k, v = normal(sum(rows), H_q, D), normal(sum(rows), H_kv, D), normal(sum(rows), H_kv, D)
    caches = [torch.randint(0, 120, (n_pages, H_kv, P, D), generator=gen, dtype=torch.uint8) if kv8 else normal(n_pages, H_kv, P, D) for _ in "kv"]
    scales = [(0.01 + 0.02 * torch.rand(H_kv, generator=gen)).cuda() for _ in "kv"]
    used = [slots(bt[i], int(ctx[i]) + rows[i], P)[int(ctx[i]):] for i in (3, 4, 5)]
    return dict(q=q.cuda(), k=k.cuda(), v=v.cuda(), caches=[c.cuda() for c in caches], scales=scales, bt=bt[3:].contiguous().cuda(), ctx=ctx[3:].contiguous().cuda(),
                cu=offsets(rows)[3:].contiguous().cuda(), first=sum(rows[:3]), used=torch.cat(used))


def same_elsewhere(before, after, used):
    rest = torch.ones(before.shape[0] * before.shape[2], dtype=torch.bool)
    rest[used] = False
    flat = [x.cpu().transpose(1, 2).flatten(0, 1) for x in (before, after)]
    assert torch.equal(flat[0][rest], flat[1][rest])
    return flat[1][used]


@pytest.mark.parametrize("dtype,kv8", [(BF, False), (F32, False), (BF, True)])
def test_append_with_rotation(fsr, dtype, kv8):
    announce(f"append with rotation, first offset {dtype} {kv8}")
    b = batch(dtype, kv8)
    table = torch.randn(120, 64, generator=torch.Generator().manual_seed(1)).cuda()
    scales = dict(k_scale=b["scales"][0], v_scale=b["scales"][1]) if kv8 else {}
    results = []
    for skip in (0, b["first"]):  # the piece as it is; its rows alone
        k, v = (c.clone() for c in b["caches"])
        out = torch.full_like(b["q"], 7.0)[skip:]
        fsr.kv_append_rope(b["q"][skip:], b["k"][skip:], b["v"][skip:], table, k, v, b["bt"], b["ctx"], b["cu"] - skip, q_out=out, **scales)
        torch.cuda.synchronize()
        results.append((out, *(same_elsewhere(x, y, b["used"]) for x, y in zip(b["caches"], (k, v)))))
    (out, *caches), (out_alone, *caches_alone) = results
    assert (out[:b["first"]] == 7).all() and torch.equal(out[b["first"]:], out_alone)
    assert all(torch.equal(x, y) for x, y in zip(caches, caches_alone))


@pytest.mark.parametrize("dtype,kv8", [(BF, False), (F32, False), (BF, True)])
def test_append(fsr, dtype, kv8):
    announce(f"append, first offset {dtype} {kv8}")
    b = batch(dtype, kv8)
    results = []
    for skip in (0, b["first"]):
        k, v = (c.clone() for c in b["caches"])
        if kv8:
            fsr.kv_append_kv8(b["k"][skip:], b["v"][skip:], k, v, *b["scales"], b["bt"], b["ctx"], b["cu"] - skip)
        else:
            fsr.kv_append(b["k"][skip:], b["v"][skip:], k, v, b["bt"], b["ctx"], b["cu"] - skip)
        torch.cuda.synchronize()
        results.append([same_elsewhere(x, y, b["used"]) for x, y in zip(b["caches"], (k, v))])
    assert all(torch.equal(x, y) for x, y in zip(*results))
