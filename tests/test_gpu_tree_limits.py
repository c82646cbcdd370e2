"""The calls on trees and log probabilities at their limits: hundreds of requests, a thousand rows of one, caches and logits beyond 2^32
bytes, scores that keep growing, workspaces with any bytes in them or in use elsewhere, nothing to do."""
import pytest
import torch

import test_gpu_token_logprobs as logprobs
import test_gpu_tree_attention as trees
from gpu_utils import announce
from plain_attention import check, offsets
from plain_tree import attend_masked, rotate

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def fsr():
    import paper_2604_20503_amd as f
    f.load_library()
    return f


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B", [64, 65, 257, 1000])
def test_many_requests(fsr, B, dtype):
    announce(f"tree attention, {B} requests {dtype}")
    reqs = [(13 * k % 90, k * 7 % 5) for k in range(B)]
    b = trees.Batch(1, reqs, 4, 2, 64, 16, dtype)
    b.compare("many", b.run(fsr, dtype))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_thousand_rows(fsr, dtype):
    announce(f"tree attention, 1024 rows {dtype}")
    b = trees.Batch(2, [(100, 1024), (3, 2)], 4, 1, 64, 16, dtype)
    assert b.words == 16
    b.compare("rows", b.run(fsr, dtype))


@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32)])
def test_scores_that_keep_growing(fsr, dtype, out_dtype):
    """Every 64 keys the scores of some rows are far above all before: their references move again and again, also in whole tiles; those of other
    rows fall."""
    announce(f"tree attention, growing scores {dtype} {out_dtype}")
    b = trees.Batch(3, [(1500, 9), (700, 40)], 4, 1, 64, 16, dtype)
    way = torch.randn(64, generator=torch.Generator().manual_seed(5))
    for i, (c, n) in enumerate(b.reqs):
        s = trees.slots(b.bt[i], c + n, 16)
        b.k.flatten(0, 1)[s] = (way * torch.linspace(0, 1, c + n)[:, None, None] + 0.01 * b.k.flatten(0, 1)[s].float()).to(dtype)
    b.q[:b.N] = ((torch.arange(b.N) % 3 - 1)[:, None, None] * 20 * way + 0.1 * b.q[:b.N].float()).to(dtype)
    b.compare("growing", b.run(fsr, out_dtype))


@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("case", [trees.CASES[3], trees.CASES[5], trees.CASES[10], trees.CASES[11]], ids=lambda c: c[0])
def test_used_workspaces(fsr, case, dtype, out_dtype):
    """Bytes of every kind in a workspace leave the results as they are, bit for bit; lse or not, out or not."""
    announce(f"tree attention, used workspace: {case[0]} {dtype} {out_dtype}")
    b = trees.Batch(1, *case[1:], dtype)
    need = fsr.tree_workspace_bytes(N_cap=b.N + 2, H_q=b.H_q, H_kv=b.H_kv, D=b.D, dtype=dtype, out_dtype=out_dtype)
    first = None
    for byte in (0x00, 0xFF, 0x01, 0x41, 0x7F):
        got = b.run(fsr, out_dtype, workspace=torch.full((need,), byte, dtype=torch.uint8, device="cuda"))
        first = first or got
        assert torch.equal(got[0], first[0]) and torch.equal(got[1], first[1])
    b.compare(case[0], first)
    out, lse = fsr.verify_attention_tree(**b.dev(), scale=b.scale, out_dtype=out_dtype, kv_layout=fsr.binding.KV_HEAD_MAJOR)
    assert lse is None and torch.equal(out[:b.N], first[0])


@pytest.mark.parametrize("N,V,K", [(2, 128256, 20), (40, 30000, 64), (1, 9000, 1)])
def test_used_workspaces_of_logprobs(fsr, N, V, K):
    announce(f"log probabilities, used workspace {N} x {V} K={K}")
    z = logprobs.logits(N, V, BF)
    need = fsr.logprob_workspace_bytes(N_cap=N, V=V, M=2, K=K, dtype=BF)
    first = None
    for byte in (0x00, 0xFF, 0x01, 0x41, 0x7F):
        ws = torch.full((need,), byte, dtype=torch.uint8, device="cuda")
        for _ in range(2):
            got = logprobs.compare(fsr, z, 2, K, 1.0, workspace=ws)
            first = first or [x.clone() for x in got]
            assert all(torch.equal(x, y) for x, y in zip(got, first))


def test_a_workspace_in_use_elsewhere_is_refused(fsr):
    announce("trees, workspaces on two streams")
    b, z = trees.Batch(4, [(6000, 60)] * 8, 32, 8, 128, 16, BF), logprobs.logits(300, 128256, BF)
    d = b.dev()
    tree_ws = torch.empty(fsr.tree_workspace_bytes(N_cap=b.N + 2, H_q=32, H_kv=8, D=128, dtype=BF, out_dtype=BF), dtype=torch.uint8, device="cuda")
    lp_ws = torch.empty(fsr.logprob_workspace_bytes(N_cap=300, V=128256, M=0, K=20, dtype=BF), dtype=torch.uint8, device="cuda")
    for call in (lambda: fsr.verify_attention_tree(**d, scale=b.scale, workspace=tree_ws), lambda: fsr.token_logprobs(z, top_k=20, workspace=lp_ws)):
        other, a = torch.cuda.Stream(), torch.ones(8192, 8192, device="cuda")
        call()
        torch.cuda.synchronize()
        for _ in range(8):  # tens of milliseconds of work before the call: the calls alone end as fast as they are made
            a @ a
        call()
        with torch.cuda.stream(other):
            with pytest.raises(fsr.FsrError) as e:
                call()
            assert e.value.code == -4
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            call()
        torch.cuda.synchronize()


def test_caches_beyond_32_bits(fsr):
    """Pages more than 2^32 bytes into the caches: append with rotation, attention and commit."""
    announce("trees, large caches")
    H_q, H_kv, D, P, n_pages = 8, 8, 128, 16, 150000
    k, v = (torch.zeros((n_pages, H_kv, P, D), dtype=BF, device="cuda") for _ in "kv")  # 4.9 GB each
    gen = torch.Generator().manual_seed(1)
    c, n = 75, 12
    bt = torch.tensor([[149999, 3, 140000, 132000, 149000, 7]], dtype=torch.int32)
    q, kn, vn = (torch.randn((n + c, h, D), generator=gen).to(BF) for h in (H_q, H_kv, H_kv))
    turn = torch.arange(128, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    table = torch.cat([turn.cos(), turn.sin()], 1).float()
    args = (table.cuda(), k, v, bt.cuda(), torch.tensor([0], dtype=torch.int32).cuda(), torch.tensor([0, c + n], dtype=torch.int32).cuda())
    turned = fsr.kv_append_rope(q.cuda(), kn.cuda(), vn.cuda(), *args)
    torch.cuda.synchronize()
    key, _ = rotate(kn, table[:c + n], D, False)
    s = trees.slots(bt[0], c + n, P)
    got = k[s // P, :, s % P].cpu()
    assert (got.double() - key).abs().max() <= 2.0 ** -8 * key.abs().max() and torch.equal(v[s // P, :, s % P].cpu(), vn)
    sees = torch.ones(n, n, dtype=torch.bool).tril()
    mask = trees.words_of(sees, 1).cuda()
    ctx, cu = torch.tensor([c], dtype=torch.int32).cuda(), torch.tensor([0, n], dtype=torch.int32).cuda()
    lse = torch.empty((n, H_q), device="cuda")
    out, _ = fsr.verify_attention_tree(turned[c:].contiguous(), k, v, bt.cuda(), ctx, cu, mask, scale=D ** -0.5, lse=lse)
    seen = torch.cat([torch.ones(n, c, dtype=torch.bool), sees], 1)
    for h in range(H_q):
        o, l, A, e = attend_masked(turned[c:, h].cpu(), got[:, h], vn[:, h], D ** -0.5, seen)
        check(f"head {h}", out[:, h], lse[:, h], o, l, A, e, BF)
    path = torch.tensor([[0, 2, 5, 11]], dtype=torch.int32).cuda()
    fsr.kv_commit(k, v, bt.cuda(), ctx, torch.tensor([3], dtype=torch.int32).cuda(), path)
    torch.cuda.synchronize()
    for j, p in ((1, 2), (2, 5), (3, 11)):
        t = c + j
        assert torch.equal(k[bt[0, t // P].item(), :, t % P].cpu(), got[c + p]) and torch.equal(v[bt[0, t // P].item(), :, t % P].cpu(), vn[c + p])


def test_logits_beyond_32_bits(fsr):
    announce("log probabilities, 5 GB of logits")
    N, V = 20000, 128256
    z = torch.empty((N, V), dtype=BF, device="cuda")
    z.copy_(logprobs.logits(1, V, BF).expand(N, V))
    z[N - 1] = logprobs.logits(1, V, BF, seed=3)[0]
    got = fsr.token_logprobs(z, torch.full((N,), 5, dtype=torch.int32, device="cuda"), top_k=4)
    for r in (0, N // 2, 16800, N - 1):
        lp, H, ids, top, off, H_off = logprobs.plain(z[r:r + 1], torch.tensor([[5]], dtype=torch.int32, device="cuda"), 4, 1.0)
        logprobs.near(got[0][r:r + 1, None], lp, off[:, None])
        logprobs.near(got[1][r:r + 1], H, H_off)
        assert torch.equal(got[2][r:r + 1], ids)
    assert (got[2][:-1] == got[2][0]).all()


def test_nothing_to_do(fsr):
    announce("trees, empty batches")
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    q, cache, table = torch.zeros(0, 4, 64, device="cuda"), torch.zeros(3, 2, 16, 64, device="cuda"), torch.ones(9, 64, device="cuda")
    mask = torch.zeros(0, 1, dtype=torch.int64, device="cuda")
    for B in (0, 2):
        bt, ctx, cu = i32(B, 4), i32(B), i32(B + 1)
        assert fsr.kv_append_rope(q, q[:, :2], q[:, :2], table, cache, cache, bt, ctx, cu, tree_mask=mask).shape == (0, 4, 64)
        assert fsr.verify_attention_tree(q, cache, cache, bt, ctx, cu, mask, scale=1.0)[0].shape == (0, 4, 64)
        acc, nem, em, path = fsr.tree_accept(i32(0), i32(0), mask, cu, S_max=3)
        assert acc.tolist() == [-1] * B and nem.tolist() == [0] * B and (em == -1).all() and (path == -1).all()
        fsr.kv_commit(cache, cache, bt, ctx, acc, path)
    assert [None if x is None else tuple(x.shape) for x in fsr.token_logprobs(torch.zeros(0, 50, device="cuda"), i32(0), top_k=2)] == [(0,), (0,), (0, 2), (0, 2)]
    # rows allocated, none in use
    q = torch.full((5, 4, 64), 3.0, device="cuda")
    out = torch.full_like(q, 7.0)
    fsr.verify_attention_tree(q, cache, cache, i32(2, 4), i32(2), i32(3), torch.zeros(5, 1, dtype=torch.int64, device="cuda"), scale=1.0, out=out)
    torch.cuda.synchronize()
    assert (out == 7).all() and not cache.any()


def test_offsets_that_do_not_hold_together_stay_inside_the_tensors(fsr):
    """Offsets out of order or beyond the rows, negative lengths, lengths behind the table: nothing is written but rows of the tensors."""
    announce("trees, bad offsets")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    guard = torch.full((30, 4, 64), 7.0, device="cuda")
    out = guard[10:20]  # 10 rows between others
    q, cache, table = torch.randn(10, 4, 64, device="cuda"), torch.randn(6, 2, 16, 64, device="cuda"), torch.ones(9, 64, device="cuda")
    mask = torch.full((10, 1), -1, dtype=torch.int64, device="cuda")
    before = cache.clone()
    for cu in ([0, 5, 1 << 30], [0, 8, 3], [-7, 4, 10], [12, 13, 14], [5, 5, 5]):
        for ctx in ([-9, 1 << 30], [40, 0], [0, 1 << 20]):
            bt = i32([[0, 1, 2], [3, -5, 1 << 30]])
            fsr.verify_attention_tree(q, cache, cache, bt, i32(ctx), i32(cu), mask, scale=0.1, out=out)
            fsr.tree_accept(i32([1] * 10), i32([1] * 10), mask, i32(cu), S_max=3)
            fsr.kv_append_rope(q, q[:, :2].contiguous(), q[:, 2:].contiguous(), table, cache.clone(), cache.clone(), bt, i32(ctx), i32(cu), tree_mask=mask, q_out=out)
            fsr.kv_commit(cache.clone(), cache.clone(), bt, i32(ctx), i32([3, 90]), i32([[0, 5, 1 << 30, 9], [0, -4, 7, 1 << 20]]))
    torch.cuda.synchronize()
    assert (guard[:10] == 7).all() and (guard[20:] == 7).all() and torch.equal(cache, before)


def test_two_calls_at_once(fsr):
    """Log probabilities of two batches on two streams, many times: each call has its own workspace."""
    announce("log probabilities, two streams")
    z = [logprobs.logits(5, 60000, BF, seed=1), logprobs.logits(3, 128256, F32, seed=2)]
    want = [[x.clone() for x in fsr.token_logprobs(x, top_k=9)[1:]] for x in z]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in z]
    for _ in range(20):
        got = []
        for x, s in zip(z, streams):
            with torch.cuda.stream(s):
                got.append(fsr.token_logprobs(x, top_k=9)[1:])
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(g, w))
