"""Log probabilities and entropies of rows in which one token has nearly all the mass: both are about the mass of the others and keep its
digits.

u = 2^-24.  A weight is off by 3 u |x| + 2 u relative (x = (z - m) / T in three roundings, the exponential), a thread adds up the weights of
its share of a row, V / 256 at most, and a few sums more are added: so far the mass of the others, relative to itself.  Sums of 1 and more are
kept in 53 bits: 2^-47 absolute after the handful of additions that follow."""
import pytest
import torch

from gpu_utils import announce

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


@pytest.fixture(scope="module")
def fsr():
    import paper_2604_20503_amd as f
    f.load_library()
    return f


def near(got, want, off):
    assert ((got.double() - want).abs() <= off * want.abs() + 2.0 ** -47).all(), ((got.double() - want) / want).abs().max()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [1.0, 0.7])
@pytest.mark.parametrize("N,V", [(4, 2), (3, 17), (5, 5000), (5, 128256), (3, 200001), (1200, 9000), (530, 32000)])
def test_near_certain_rows(fsr, N, V, T, dtype):
    announce(f"log probabilities, near-certain rows {N} x {V} T={T} {dtype}")
    gen = torch.Generator(device="cuda").manual_seed(V)
    z = (torch.randn((N, V), generator=gen, device="cuda") * 2.0).to(dtype)
    at = torch.randint(0, V, (N, 1), generator=gen, device="cuda")
    at[0], at[-1] = 0, V - 1
    gap = torch.linspace(16, 34, N, device="cuda")[:, None].to(dtype)  # the others' mass: from a tenth down to 1e-9
    z.scatter_(1, at, gap)
    x = (z.double() - gap.double()) / T
    x.scatter_(1, at, -float("inf"))
    rest, lost = x.exp().sum(1), -(x.exp() * x.clamp(min=-1e3)).sum(1)
    lp, entropy, ids, top = fsr.token_logprobs(z, at.int(), top_k=1, temperature=T)
    torch.cuda.synchronize()
    off = (3 * float(-x[x > -float("inf")].min()) + 2 + V / 256 + 60) * U
    want = -torch.log1p(rest)
    assert torch.equal(ids, at.int())
    near(lp[:, 0], want, off)
    near(top[:, 0], want, off)
    near(entropy, torch.log1p(rest) + lost / (1 + rest), 3 * off)
    # without alternatives, and out of wider rows that begin anywhere: the same sums
    wide = torch.full((N, V + 9), 50.0, dtype=dtype, device="cuda")
    wide[:, 1:V + 1] = z
    for x in (z, wide[:, 1:V + 1]):
        lp_only, entropy_only, _, _ = fsr.token_logprobs(x, at.int(), temperature=T)
        assert torch.equal(lp_only, lp) and torch.equal(entropy_only, entropy)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_nearly_a_half(fsr, dtype):
    """Around the place where the largest token has as much as all others; two of it."""
    announce(f"log probabilities, nearly a half {dtype}")
    V = 30000
    gap = torch.linspace(11.5, 13.5, 41, device="cuda")
    z = torch.randn((42, V), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda") * 2.0
    z[:41, 777] = gap
    z[41, [5, 29000]] = 25.0
    z = z.to(dtype)
    lp, entropy, ids, _ = fsr.token_logprobs(z, ids_of := z.argmax(1).int(), top_k=2)
    exact = torch.log_softmax(z.double(), 1)
    torch.cuda.synchronize()
    off = (3 * 45 + 2 + V / 256 + 60) * U
    assert torch.equal(ids[:, 0], ids_of) and ids[41].tolist() == [5, 29000]
    near(lp, exact.gather(1, ids_of.long()[:, None])[:, 0], off)
    near(entropy, torch.special.entr(exact.exp()).sum(1), 3 * off)


def test_replays(fsr):
    """Near-certain and other rows in turn through one captured call."""
    announce("log probabilities, near-certain rows, graph")
    gen = torch.Generator(device="cuda").manual_seed(9)
    z = [torch.randn((3, 60000), generator=gen, device="cuda") for _ in range(2)]
    z[0][:, 1234] = 28.0
    want = [[x.clone() for x in fsr.token_logprobs(x, top_k=3)[1:]] for x in z]
    room, ws = z[0].clone(), torch.empty(fsr.logprob_workspace_bytes(N_cap=3, V=60000, M=0, K=3, dtype=F32), dtype=torch.uint8, device="cuda")
    out = [torch.zeros_like(x) for x in want[0]]
    call = lambda: fsr.token_logprobs(room, top_k=3, entropy=out[0], top_ids=out[1], top_logprobs=out[2], workspace=ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(4):
        room.copy_(z[k % 2])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[k % 2]))
