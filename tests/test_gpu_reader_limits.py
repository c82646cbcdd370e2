"""The attention over latent caches and behind shared prefixes at the ends of what its arguments may be."""
import pytest
import torch

import test_gpu_latent as latent
import test_gpu_latent_expanded as expanded
import test_gpu_shared_prefix as shared
from gpu_utils import announce

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def fsr():
    import paper_2604_20503_amd as f
    f.load_library()
    return f


@pytest.mark.parametrize("most", [2 ** 31 - 1, 2 ** 30, 2 ** 30 + 1])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_any_number_of_workgroups_is_a_bound(fsr, dtype, most):
    """A bound beyond the device's units is none, up to the largest number."""
    announce(f"bounds on workgroups: {dtype} {most}")
    a = latent.Batch(51, [70, 3], [2, 1], 16, 512, 64, 16, dtype)
    assert all(torch.equal(x, y) for x, y in zip(latent.run(fsr, a, dtype, max_workgroups=most), latent.run(fsr, a, dtype)))
    b = expanded.Batch(52, [30], [200], 2, expanded.BIG, dtype)
    assert all(torch.equal(x, y) for x, y in zip(b.run(fsr, dtype, max_workgroups=most), b.run(fsr, dtype)))
    c = shared.Batch(53, [(100, [(5, 2), (9, 1)])], 8, 2, 128, 16, dtype)
    assert all(torch.equal(x, y) for x, y in zip(c.run(fsr, dtype, max_workgroups=most), c.run(fsr, dtype)))


def room(gib):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB")


def test_rows_allocated_by_the_hundred_million(fsr):
    """Buffers of 2^29 + 5 rows, of which the last three are the call's: more than one launch holds."""
    room(24)
    n = 2 ** 29 + 5
    announce(f"latent append and gather, {n} rows allocated")
    rows, rope = (torch.empty(n, 8, dtype=BF, device="cuda") for _ in range(2))
    rows[-3:], rope[-3:] = torch.arange(24, device="cuda").view(3, 8).to(BF), -torch.arange(24, device="cuda").view(3, 8).to(BF)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cache, bt, cu = torch.zeros(3, 4, 16, dtype=BF, device="cuda"), i32(2, 0).view(2, 1), i32(n - 3, n - 1, n)
    fsr.latent_append(rows, rope, cache, bt, i32(1, 3), cu)
    want = torch.zeros_like(cache)
    want[2, 1:3], want[0, 3] = torch.cat([rows[-3:-1], rope[-3:-1]], 1), torch.cat([rows[-1], rope[-1]])
    assert torch.equal(cache, want)
    cache.copy_(torch.arange(cache.numel(), device="cuda").view_as(cache).to(BF))
    rows[-4:], rope[-4:] = 7.0, 7.0
    fsr.latent_gather(cache, bt, cu, T_cap=n, D_latent=8, latent=rows, rope=rope)
    got = torch.cat([rows[-4:], rope[-4:]], 1)
    assert torch.equal(got[1:3], cache[2, :2]) and torch.equal(got[3], cache[0, 0]) and got[0].eq(7).all()
    del rows, rope
    torch.cuda.empty_cache()


def test_joins_of_rows_by_the_ten_million(fsr):
    """2^26 + 128 rows and heads allocated, the last 80 of them the call's."""
    room(64)
    announce("shared prefix, 2^26 rows and heads allocated")
    b = shared.Batch(54, [(200, [(5, 2), (90, 3)])], 16, 1, 64, 16, BF)
    d, N = b.dev(), 2 ** 22 + 8
    q, out = (torch.empty(N, 16, 64, dtype=BF, device="cuda") for _ in range(2))
    lse = torch.empty(N, 16, device="cuda")
    q[N - b.N:], out[N - b.N - 1], lse[N - b.N - 1] = d["q"][:b.N], 7.0, 7.0
    d.update(q=q, cu_q=d["cu_q"] + (N - b.N))
    fsr.verify_attention_shared(**d, scale=b.scale, out=out, lse=lse)
    b.compare("far rows", (out[N - b.N:], lse[N - b.N:]))
    assert out[N - b.N - 1].eq(7).all() and lse[N - b.N - 1].eq(7).all()
    del d, q, out, lse
    torch.cuda.empty_cache()
