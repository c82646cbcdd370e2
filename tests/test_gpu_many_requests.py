"""More requests than a workgroup has threads: several sequences a thread where the line is added up, and no even pieces; results without lse;
two calls at once."""
import pytest
import torch

import test_gpu_latent as latent
import test_gpu_latent_expanded as expanded
import test_gpu_shared_prefix as shared
from gpu_utils import announce

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
TYPES = [(BF, BF), (BF, F32), (F32, F32)]


@pytest.fixture(scope="module")
def fsr():
    import paper_2604_20503_amd as f
    f.load_library()
    return f


def some(seed, n, lo, hi):
    return torch.randint(lo, hi + 1, (n,), generator=torch.Generator().manual_seed(seed)).tolist()


@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("B", [256, 257, 700])
def test_latent(fsr, B, dtype, out_dtype):
    announce(f"latent attention, {B} requests {dtype} {out_dtype}")
    ctx = some(1, B, 0, 40)
    ctx[B // 2], ctx[B - 1] = 900, 300
    b = latent.Batch(61, ctx, some(2, B, 0, 2), 4, 512, 64, 16, dtype)
    latent.compare(f"{B} requests", b, latent.run(fsr, b, out_dtype))


@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("B", [257, 900])
def test_expanded(fsr, B, dtype, out_dtype):
    announce(f"latent expanded, {B} requests {dtype} {out_dtype}")
    rows, keys = some(3, B, 0, 4), some(4, B, 0, 90)
    rows[B // 3], keys[B // 3] = 150, 700
    b = expanded.Batch(62, rows, keys, 2, expanded.SMALL, dtype)
    b.compare(f"{B} requests", b.run(fsr, out_dtype))


@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("B,groups", [(200, 57), (400, 3), (350, 350)])
def test_shared(fsr, B, groups, dtype, out_dtype):
    announce(f"shared prefix, {B} requests in {groups} groups {dtype} {out_dtype}")
    own, rows, prefix = some(5, B, 0, 30), some(6, B, 0, 2), some(7, groups, 0, 60)
    prefix[groups // 2] = 700
    of = torch.linspace(0, groups - 1e-3, B).long().tolist()
    b = shared.Batch(63, [(prefix[g], [(own[i], rows[i]) for i in range(B) if of[i] == g]) for g in range(groups)], 4, 2, 64, 16, dtype)
    b.compare(f"{B} requests", b.run(fsr, out_dtype))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_results_without_lse(fsr, dtype):
    announce(f"no lse {dtype}")
    a = latent.Batch(64, [700, 3], [2, 1], 16, 512, 64, 16, dtype)
    q, cache, bt, ctx, cu = a.dev()
    out, lse = fsr.latent_attention(q, cache, bt, ctx, cu, scale=a.scale, D_latent=512)
    assert lse is None and torch.equal(out, latent.run(fsr, a, dtype)[0])
    b = expanded.Batch(65, [150], [700], 1, expanded.BIG, dtype)
    from plain_attention import offsets
    out, _ = fsr.latent_attention_expanded(b.q.cuda(), b.kv.cuda(), b.rope.cuda(), offsets(b.rows).cuda(), offsets(b.keys).cuda(), scale=b.scale)
    assert torch.equal(out[:b.N], b.run(fsr, dtype)[0])
    c = shared.Batch(66, [(400, [(5, 2), (90, 1)])], 8, 2, 128, 16, dtype)
    out, _ = fsr.verify_attention_shared(**c.dev(), scale=c.scale)
    assert torch.equal(out[:c.N], c.run(fsr, dtype)[0])


def test_two_streams_at_once(fsr):
    """Calls on two streams, each with a workspace of its own, in flight together; and two graphs of them replayed side by side."""
    announce("two streams, two graphs")
    a = [latent.Batch(67 + k, [900 - 300 * k, 40], [3, 2], 16, 512, 64, 16, BF) for k in range(2)]
    want = [latent.run(fsr, x, BF) for x in a]
    need = [fsr.latent_workspace_bytes(N_cap=x.N, H=16, D_latent=512, D_rope=64, dtype=BF, out_dtype=BF) for x in a]
    dev, ws = [x.dev() for x in a], [torch.empty(n, dtype=torch.uint8, device="cuda") for n in need]
    outs, lses = [torch.zeros_like(w[0]) for w in want], [torch.zeros_like(w[1]) for w in want]
    streams = [torch.cuda.Stream() for _ in a]
    call = lambda k: fsr.latent_attention(*dev[k], scale=a[k].scale, D_latent=512, out=outs[k], lse=lses[k], workspace=ws[k])  # noqa: E731
    torch.cuda.synchronize()
    for _ in range(5):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                outs[k].zero_()
                call(k)
    torch.cuda.synchronize()
    assert all(torch.equal(outs[k], want[k][0]) and torch.equal(lses[k], want[k][1]) for k in range(2))
    graphs = [torch.cuda.CUDAGraph() for _ in a]
    for k, g in enumerate(graphs):
        with torch.cuda.graph(g):
            call(k)
    for _ in range(4):
        for x in outs + lses:
            x.zero_()
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(outs[k], want[k][0]) and torch.equal(lses[k], want[k][1]) for k in range(2))
