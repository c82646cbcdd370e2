"""Values that are not finite among those that rows see, wherever the line of tiles is cut: in tiles that all rows see whole, behind a piece's
first one, as well as in those with masked keys; with weights in one or two parts; with a weight that counts, and with one that is nothing in fp32."""
import pytest
import torch

import test_gpu_latent as latent
import test_gpu_latent_expanded as expanded
import test_gpu_shared_prefix as shared
from gpu_utils import announce
from plain_attention import attend, check, slots

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")
TYPES = [(BF, BF), (BF, F32), (F32, F32)]
UP, DOWN, BOTH, ODD, LATE = 5, 6, 9, 33, 11  # columns


@pytest.fixture(scope="module")
def fsr():
    import paper_2604_20503_amd as f
    f.load_library()
    return f


def plant(v, a, b, late):
    """v [keys, heads, columns]: keys a and b are seen by all rows, `late` by some."""
    v[a, :, UP], v[a, :, DOWN], v[a, :, BOTH], v[b, :, BOTH], v[a, :, ODD], v[late, :, LATE] = INF, -INF, INF, -INF, NAN, INF


def compare(name, out, lse, want, sees_late, counts, dtype):
    """out [N, H, D]; counts: the weights of what has been planted do."""
    o, want_lse, A, e = want
    fine = torch.ones(out.shape[2], dtype=torch.bool)
    fine[[UP, DOWN, BOTH, ODD, LATE]] = False
    D = int(fine.sum())
    check(name, out[:, :, fine.cuda()].reshape(-1, D), lse.reshape(-1), o[:, :, fine].reshape(-1, D), want_lse.reshape(-1), A[:, :, fine].reshape(-1, D), e.reshape(-1), dtype)
    got = out.float().cpu()
    if counts:
        assert got[..., UP].eq(INF).all() and got[..., DOWN].eq(-INF).all()
    assert not got[..., UP].isfinite().any() and not got[..., DOWN].isfinite().any()
    assert not got[..., BOTH].isfinite().any() and got[..., ODD].isnan().all()
    assert got[sees_late][..., LATE].eq(INF).all()
    assert got[~sees_late][..., LATE].isfinite().all()


@pytest.mark.parametrize("workgroups", [1, 0])
@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("counts", [True, False])
@pytest.mark.parametrize("dims", [expanded.BIG, expanded.SMALL])
@pytest.mark.parametrize("at", [3, 130, 383])
def test_expanded(fsr, at, dims, counts, dtype, out_dtype, workgroups):
    announce(f"latent expanded, infinite values: {at} {dims} {counts} {dtype} {out_dtype} {workgroups}")
    n, L = 40, 7 * 64 + 60
    b = expanded.Batch(41, [n], [L], 2, dims, dtype)
    late = L - n + 10
    if not counts:  # a score 200 below
        b.q[..., b.Dn], b.rope[:, 0] = 16.0, 0.0
        b.rope[[at, at + 1], 0] = -200.0 / (16.0 * b.scale)
    want = b.reference()
    plant(b.kv[..., b.Dn:], at, at + 1, late)
    compare("expanded", *b.run(fsr, out_dtype, max_workgroups=workgroups), want, torch.arange(n) >= 10, counts, dtype)


@pytest.mark.parametrize("workgroups", [1, 0])
@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("counts", [True, False])
@pytest.mark.parametrize("D,P", [(128, 16), (64, 5)])
@pytest.mark.parametrize("at", [130, 5 * 64 + 7 + 100])
def test_shared(fsr, at, D, P, counts, dtype, out_dtype, workgroups):
    announce(f"shared prefix, infinite values: {at} {D} {P} {counts} {dtype} {out_dtype} {workgroups}")
    prefix, own = 5 * 64 + 7, 4 * 64
    b = shared.Batch(42, [(prefix, [(own, 3), (own, 2)])], 4, 2, D, P, dtype)
    k, v = b.k.flatten(0, 1), b.v.flatten(0, 1)
    of = [slots(b.bt[i], c + n, P) for i, (_, c, n) in enumerate(b.reqs)]
    if not counts:
        b.q[..., 0], k[:, :, 0] = 16.0, 0.0
        for s in of:
            k[s[at:at + 2], :, 0] = -200.0 / (16.0 * b.scale)
    want = b.reference()
    for s in of:
        x = v[s]
        plant(x, at, at + 1, prefix + own + 1)
        v[s] = x
    compare("shared", *b.run(fsr, out_dtype, max_workgroups=workgroups), want, torch.tensor([0, 1, 1, 0, 1]).bool(), counts, dtype)


@pytest.mark.parametrize("workgroups", [1, 0])
@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("P", [16, 7])
@pytest.mark.parametrize("at", [3, 130, 383])
def test_latent_value_of_a_key_without_weight(fsr, at, P, dtype, out_dtype, workgroups):
    """An infinite element where all queries are -1 makes a key's scores -inf: it has no weight, and still is a value that all rows see (0 times
    infinity by the definition)."""
    announce(f"latent attention, infinite value: {at} {P} {dtype} {out_dtype} {workgroups}")
    b = latent.Batch(43, [7 * 64 + 20], [3], 16, 512, 64, P, dtype)
    b.q[..., UP] = -1.0
    x = b.keys(0).clone()
    rest = torch.arange(len(x)) != at
    want = attend(b.q[:b.N].flatten(0, 1), x[rest], x[rest][:, :512], b.scale, (7 * 64 + 19 + torch.arange(3)).repeat_interleave(16))
    b.cache.view(-1, 576)[slots(b.bt[0], len(x), P)[at], UP] = INF
    out, lse = latent.run(fsr, b, out_dtype, max_workgroups=workgroups)
    fine = torch.arange(512) != UP
    o, want_lse, A, e = want
    check("latent", out.reshape(-1, 512)[:, fine.cuda()], lse.reshape(-1), o[:, fine], want_lse, A[:, fine], e, dtype)
    assert not out[..., UP].isfinite().any()


@pytest.mark.parametrize("out_dtype", [BF, F32])
@pytest.mark.parametrize("D_latent,D_rope,P", [(512, 64, 16), (512, 64, 7), (256, 32, 16), (256, 64, 5)])
def test_latent_values_behind_the_rows(fsr, D_latent, D_rope, P, out_dtype):
    """Slots behind the last token hold NaN, the last token infinities and NaN: the rows before it do not see them, the last row does."""
    announce(f"latent attention, not finite behind: {D_latent} {D_rope} {P} {out_dtype}")
    b = latent.Batch(44, [70, 126, 5, 300], [3, 2, 4, 5], 16, D_latent, D_rope, P, BF)
    want = b.reference()
    flat = b.cache.view(-1, b.cache.shape[2])
    used = torch.zeros(flat.shape[0], dtype=torch.bool)
    for i in range(4):
        s = slots(b.bt[i], b.ctx[i] + b.rows[i], P)
        used[s] = True
        flat[s[-1], 3:6] = torch.tensor([INF, -INF, NAN]).to(BF)
    flat[~used] = NAN
    out, lse = latent.run(fsr, b, out_dtype)
    last = torch.zeros(b.N, dtype=torch.bool)
    last[b.cu[1:].long() - 1] = True
    pick = lambda x: x[~last.to(x.device)].reshape(-1, x.shape[-1]) if x.dim() == 3 else x[~last.to(x.device)].reshape(-1)  # noqa: E731
    check("rows before", pick(out), pick(lse), *(pick(x) for x in want), BF)
    assert torch.isnan(out[last.cuda()]).all()


@pytest.mark.parametrize("dtype,out_dtype", TYPES)
def test_latent_value_at_the_end_of_the_type(fsr, dtype, out_dtype):
    """An element of 3e38 whose queries are 0 takes no part in scores: it reaches the row that sees it, in its column, and no other row."""
    announce(f"latent attention, large value {dtype} {out_dtype}")
    b = latent.Batch(45, [20], [3], 4, 512, 64, 16, dtype)
    b.q[:, :, 9] = 0.0
    b.cache.view(-1, 576)[slots(b.bt[0], 23, 16)[-1], 9] = 3.0e38
    latent.compare("large value", b, latent.run(fsr, b, out_dtype))
