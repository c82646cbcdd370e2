"""fsr_token_logprobs against the definition in 64 bits.

How far fp32 sums may be off, with u = 2^-24 (half a step): x = (z - m) / T has three roundings, so a weight exp x is off by 3 u |x| + 2 u
relative (2 u: the exponential itself); a sum of V weights is taken by 256 threads at least, one after the other, so by chains of V / 256
and a few sums more.  With t = sum p |x| and t2 = sum p x^2 that makes log S off by 3 u t + (chain + 2) u, and sum p x by
3 u t2 + (chain + 4) u t and t times the former."""
import pytest
import torch

from gpu_utils import announce

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def fsr():
    import paper_2604_20503_amd as f
    f.load_library()
    return f


def plain(z, tokens, K, T):
    """On the GPU, in 64 bits: everything and how far it may be off."""
    V = z.shape[1]
    z = torch.where(z.isnan(), -INF, z.double())
    m = z.amax(1, keepdim=True)
    bad = ~torch.isfinite(m[:, 0])
    x = (z - m) / T
    w = torch.where(x == -INF, 0.0, x.exp())
    S = w.sum(1, keepdim=True)
    p, y = w / S, torch.where(w > 0, x, 0.0)
    t, t2, chain = (p * y.abs()).sum(1), (p * y * y).sum(1), V / 256 + 40
    log_s = S.log()[:, 0]
    off = 3 * U * t + (chain + 2) * U
    H = log_s + t
    H_off = off + 3 * U * t2 + (chain + 4) * U * t + t * off + 2 * U * H.abs()
    # descending, the lowest id first among equals
    order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :K]
    logp = lambda at: torch.gather(x, 1, at) - log_s[:, None]  # noqa: E731
    lp = None
    if tokens is not None:
        inside = (tokens >= 0) & (tokens < V)
        lp = torch.where(inside, logp(tokens.clamp(0, V - 1).long()), -INF)
        lp[bad] = NAN
    top = logp(order)
    H, top = H.clone(), top.clone()
    H[bad], top[bad] = NAN, NAN
    return lp, H, order.int(), top, off, H_off


def near(got, want, off):
    got = got.double()
    same = (got == want) | (got.isnan() & want.isnan())
    close = (got - want).abs() <= off + U * want.abs() + 1e-300
    assert (same | close).all(), f"{(got - want)[~(same | close)][:5]} where {off.flatten()[:5]} is allowed"


def compare(fsr, z, M, K, T, seed=0, **kw):
    N, V = z.shape
    gen = torch.Generator(device="cuda").manual_seed(seed)
    tokens = torch.randint(-2, V + 2, (N, M), generator=gen, device="cuda", dtype=torch.int32) if M else None
    out = [torch.full(s, 7, dtype=d, device="cuda") for s, d in (((N, M), F32), ((N,), F32), ((N, max(K, 1)), torch.int32), ((N, max(K, 1)), F32))]
    kw = {**dict(logprobs=out[0] if M else None, entropy=out[1], top_ids=out[2] if K else None, top_logprobs=out[3] if K else None), **kw}
    got = fsr.token_logprobs(z, tokens, top_k=K, temperature=T, **kw)
    torch.cuda.synchronize()
    n = int(kw["n_rows"]) if kw.get("n_rows") is not None else N
    n = max(min(n, N), 0)
    for x in got:
        assert x is None or (x[n:] == 7).all()
    lp, H, ids, top, off, H_off = plain(z[:n], None if tokens is None else tokens[:n], K, T)
    if M:
        near(got[0][:n], lp, off[:, None])
    near(got[1][:n], H, H_off)
    if K:
        assert torch.equal(got[2][:n], ids)
        near(got[3][:n], top, off[:, None])
    return got


def logits(N, V, dtype, sigma=2.5, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((N, V), generator=gen, device="cuda") * sigma).to(dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("N,V,M,K,T", [(1, 1, 1, 1, 1.0), (1, 2, 3, 2, 0.5), (3, 17, 1, 5, 1.0), (2, 64, 2, 64, 1.0), (5, 1000, 1, 20, 0.7), (1, 4096, 4, 32, 1.0), (7, 4097, 1, 10, 1.3),
                                       (2, 32000, 3, 0, 1.0), (1, 128256, 1, 5, 1.0), (33, 50257, 2, 64, 0.9), (300, 5000, 1, 20, 1.0), (4, 152064, 0, 20, 1.0), (9, 200001, 1, 33, 2.0)])
def test_logprobs(fsr, N, V, M, K, T, dtype):
    announce(f"log probabilities {N} x {V} M={M} K={K} T={T} {dtype}")
    compare(fsr, logits(N, V, dtype), M, K, T)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("K", [1, 20, 64])
def test_orders_of_logits(fsr, K, dtype):
    """Equal logits, ascending and descending ones, all large ones at one place, few that are allowed, steps that repeat."""
    announce(f"log probabilities, orders, K={K} {dtype}")
    V = 70001
    rows = [torch.zeros(V), torch.full((V,), -3e38), torch.linspace(-9, 9, V), torch.linspace(9, -9, V), torch.linspace(5, 6, V), (torch.arange(V) % 7).float(),
            (torch.arange(V) % 4096).float() / 400, (torch.arange(V) // 4096).float(), (torch.arange(V) % 256 == 3).float() * 5, -(torch.arange(V) % 2048).float() / 100]
    few = torch.full((3, V), -INF)
    few[0, [5, 60000]] = torch.tensor([1.0, 2.0])
    few[1, 4000:4030] = 1.0
    few[2, V - 1] = -50.0
    masked = torch.full((2, V), torch.finfo(dtype).min)
    masked[0, [9, 40000]] = torch.tensor([3.0, 3.0])
    late = torch.zeros(2, V)
    late[0, -3000:] = torch.linspace(1, 2, 3000)
    late[1, ::251] = 1.0
    compare(fsr, torch.cat([torch.stack(rows), few, masked, late]).to(dtype).cuda(), 2, K, 1.0)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_values_that_are_not_finite(fsr, dtype):
    announce(f"log probabilities, not finite {dtype}")
    z = logits(8, 9001, dtype)
    z[0, ::3] = NAN
    z[1, :] = -INF
    z[2, :] = NAN
    z[3, [7, 8000]] = INF
    z[4, 100:] = -INF
    z[5, 0], z[5, 1] = NAN, -INF
    z[6, :] = 0.0
    z[6, ::2] = -0.0  # equal to 0: the order is by id
    bits = z.view(torch.int16 if dtype == BF else torch.int32)
    bits[7, 5:9000:2] = 0x7f81 if dtype == BF else 0x7f800001  # signalling
    compare(fsr, z, 3, 20, 1.0)


@pytest.mark.parametrize("size", [1e-6, 1e4, 1e30, 3e38])
@pytest.mark.parametrize("T", [1e-6, 1.0, 1e6])
def test_logits_and_temperatures_of_any_size(fsr, size, T):
    announce(f"log probabilities, size {size} T={T}")
    z = (torch.rand((3, 3001), generator=torch.Generator().manual_seed(1)) * 2 - 1) * size
    z = z.float().cuda()
    if size > 1e38 or T < 1e-3 or size / T > 1e5:  # weights beyond fp32: the largest takes all, and differences may be beyond fp32 too
        got = fsr.token_logprobs(z, top_k=3, temperature=T)
        order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :3].int()
        assert torch.equal(got[2], order) and not got[3].isnan().any() and (got[1] >= 0).all()
        gap = (z.double().gather(1, order.long()) - z.double().amax(1, keepdim=True)) / T
        clear = gap[:, 1] < -200
        assert (got[3][clear, 0].abs() < 1e-6).all()
    else:
        compare(fsr, z, 2, 20, T)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_slices_of_wider_rows_and_rows_behind_the_last(fsr, dtype):
    announce(f"log probabilities, strides {dtype}")
    z = logits(11, 5003, dtype)
    compare(fsr, z[:, :5000], 2, 9, 1.0)
    compare(fsr, z[:, 1:4098], 2, 9, 1.0)  # rows that begin anywhere
    for n in (0, 1, 7, 11, 12, -3):
        compare(fsr, z, 1, 4, 1.0, n_rows=torch.tensor([n], dtype=torch.int32, device="cuda"))


def test_one_token_a_row(fsr):
    z = logits(6, 999, F32)
    tokens = torch.arange(6, dtype=torch.int32, device="cuda")
    one, two = fsr.token_logprobs(z, tokens), fsr.token_logprobs(z, tokens[:, None].contiguous())
    assert one[0].shape == (6,) and torch.equal(one[0], two[0][:, 0]) and one[2] is None and one[3] is None


@pytest.mark.parametrize("N,V", [(3, 128256), (200, 6000)])
def test_replays(fsr, N, V):
    announce(f"log probabilities, graph {N} x {V}")
    z, other = logits(N, V, BF, seed=1), logits(N, V, BF, seed=2)
    tokens = torch.randint(0, V, (N, 2), device="cuda", dtype=torch.int32)
    want = [[x.clone() for x in fsr.token_logprobs(y, tokens, top_k=7)] for y in (z, other)]
    out = [torch.zeros_like(x) for x in want[0]]
    ws = torch.randint(0, 255, (fsr.logprob_workspace_bytes(N_cap=N, V=V, M=2, K=7, dtype=BF),), dtype=torch.uint8, device="cuda")
    room = z.clone()
    call = lambda: fsr.token_logprobs(room, tokens, top_k=7, logprobs=out[0], entropy=out[1], top_ids=out[2], top_logprobs=out[3], workspace=ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(4):
        room.copy_((z, other)[k % 2])
        for x in out:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[k % 2]))
        compare(fsr, other, 1, 3, 1.0)
