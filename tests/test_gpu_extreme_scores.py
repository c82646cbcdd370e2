"""Scores far beyond what exponents of two hold: a row's result is the softmax of its products whatever their size, in every form, in one piece
or joined of many, and where the sizes change along the keys.

A score is the sum of two products with a query of ones, both exact in bf16 and with an exact sum in fp32, so that what is compared is the
softmax alone.  (Where all keys' scores are alike, the rows' queries are 1, 1 + 1/128, 1 + 2/128 ..: products of 16 bits, exact as well.)

Its error, in units of u = 2^-24 and relative for every weight: the distance d of a score from the largest times scale * log2(e), rounded, 3 u d,
then minus at most 40 + 12, rounded, u (d + 52), the exponential 2 u; from d = 127 on a weight is less than any rounding: 4 * 127 + 54 in all.
Sums over L keys (L + 16) u.  The denominators carry the same, hence twice; parts put together, once more.
"""
import pytest
import torch

import test_gpu_latent as latent
import test_gpu_latent_expanded as expanded
import test_gpu_shared_prefix as shared
from gpu_utils import announce
from plain_attention import U, check

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
TYPES = [(BF, BF), (BF, F32), (F32, F32)]
M26, M31 = 2.0 ** 26, 2.0 ** 31
# name: (scale, products by tile of 64 keys (again from the first behind the last), size of the small steps between keys of a tile)
PROFILES = {
    "ordinary": (1.0, [0.0, 5.0], 1.0),
    "2^20 and steps of one": (1.0, [2.0 ** 20], 1.0),
    "-2^20 and steps of one": (1.0, [-(2.0 ** 20)], 1.0),
    "2^27, scale 1/16": (0.0625, [2.0 ** 27], 16.0),
    "below the border": (1.0, [1.25 * M26], 8.0),
    "behind the border": (1.0, [1.5 * M26], 8.0),
    "below and behind the border": (1.0, [1.25 * M26, 1.5 * M26, 1.25 * M26], 8.0),
    "the border from below zero": (1.0, [-1.25 * M26, -1.5 * M26, -1.25 * M26], 8.0),
    "alike, 2^31": (1.0, [M31], 0.0),
    "alike, -2^34": (1.0, [-8 * M31], 0.0),
    "alike, 2^40 and a third": (0.3333, [2.0 ** 40], 0.0),
    "beyond fp32 with the scale": (16.0, [2.0 ** 126], 0.0),
    "below fp32 with the scale": (16.0, [-(2.0 ** 126)], 0.0),
    "climbing": (1.0, [-(2.0 ** 127), -M31, -128.0, 0.0, M31, 2.0 ** 60, 2.0 ** 127, -5.0], 0.0),
    "falling": (1.0, [2.0 ** 127, 2.0 ** 60, M31, 0.0, -128.0, -M31, -(2.0 ** 127)], 0.0),
    "one step below zero": (1.0, [-(2.0 ** 100), -(2.0 ** 40), -(2.0 ** 33), -(2.0 ** 30), -(2.0 ** 35)], 0.0),
}


@pytest.fixture(scope="module")
def fsr():
    import paper_2604_20503_amd as f
    f.load_library()
    return f


def products(profile, n, gen):
    """Both products of the scores of n keys."""
    _, bases, step = PROFILES[profile]
    base = torch.tensor(bases, dtype=torch.float64)[torch.arange(n) // 64 % len(bases)]
    small = step * torch.randint(0, 4, (n,), generator=gen).double()
    assert torch.equal((base + small).float().double(), base + small) and torch.equal(base.bfloat16().double(), base)
    return torch.stack([base, small], 1)


def queries(profile, n):
    return 1.0 + torch.arange(n).double() % 128 / 128 if profile.startswith("alike") else torch.ones(n).double()


def attend(q, z, v, scale, last):
    """Rows that see keys 0 .. last: result, lse (infinite where fp32 does not hold it), weighted magnitudes, error."""
    n, L = len(last), z.shape[0]
    seen = torch.arange(L)[None] <= last[:, None]
    s = torch.where(seen, q[:, None] * z.sum(1) * scale, float("-inf"))
    w, v = torch.softmax(s, 1), v.double()
    e = 2 * (4 * 127 + 54 + L + 16) * U
    return w @ v, torch.logsumexp(s, 1).float().double(), w @ v.abs(), torch.full((n,), e, dtype=torch.float64)


def same(name, got, parts, dtype, times=1):
    """parts: by request and head."""
    o, lse, A, e = (torch.cat(p) for p in zip(*parts))
    check(name, got[0].reshape(-1, o.shape[1]), got[1].reshape(-1), o, lse, A, times * e, dtype)


@pytest.mark.parametrize("workgroups", [1, 0])
@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("Dl,Dr,P", [(512, 64, 16), (256, 32, 7)])
@pytest.mark.parametrize("profile", PROFILES)
def test_latent(fsr, profile, Dl, Dr, P, dtype, out_dtype, workgroups):
    announce(f"latent attention, extreme scores: {profile} {Dl} {Dr} {P} {dtype} {out_dtype} {workgroups}")
    gen = torch.Generator().manual_seed(1)
    b = latent.Batch(31, [7 * 64 + 20, 200], [3, 2], 12, Dl, Dr, P, dtype)
    b.scale = PROFILES[profile][0]
    b.q.zero_()
    q = queries(profile, b.N * b.H)
    b.q[..., Dl:Dl + 2] = q.view(b.N, b.H, 1).to(dtype)
    parts = []
    for i, n in enumerate(b.rows):
        s = latent.slots(b.bt[i], b.ctx[i] + n, P)
        z = products(profile, len(s), gen)
        b.cache.view(-1, Dl + Dr)[s, Dl:Dl + 2] = z.to(dtype)
        parts.append(attend(q[int(b.cu[i]) * b.H:int(b.cu[i + 1]) * b.H], z, b.keys(i)[:, :Dl], b.scale, (b.ctx[i] + torch.arange(n)).repeat_interleave(b.H)))
    same(profile, latent.run(fsr, b, out_dtype, max_workgroups=workgroups), parts, dtype)


@pytest.mark.parametrize("workgroups", [1, 0])
@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("dims", [expanded.BIG, expanded.SMALL])
@pytest.mark.parametrize("profile", PROFILES)
def test_expanded(fsr, profile, dims, dtype, out_dtype, workgroups):
    announce(f"latent expanded, extreme scores: {profile} {dims} {dtype} {out_dtype} {workgroups}")
    gen = torch.Generator().manual_seed(2)
    b = expanded.Batch(32, [40, 5], [7 * 64 + 60, 150], 1, dims, dtype)
    b.scale = PROFILES[profile][0]
    b.q.zero_()
    q = queries(profile, b.N)
    b.q[:b.N, :, b.Dn:b.Dn + 2] = q[:, None, None].to(dtype)
    parts, at, row = [], 0, 0
    for n, L in zip(b.rows, b.keys):
        z = products(profile, L, gen)
        b.rope[at:at + L, :2] = z.to(dtype)
        parts.append(attend(q[row:row + n], z, b.kv[at:at + L, 0, b.Dn:], b.scale, L - n + torch.arange(n)))
        at, row = at + L, row + n
    same(profile, b.run(fsr, out_dtype, max_workgroups=workgroups), parts, dtype)


@pytest.mark.parametrize("workgroups", [1, 0])
@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("prefix,own,D,P", [(7 * 64 + 10, 30, 128, 16), (4 * 64, 4 * 64 + 9, 64, 5)])
@pytest.mark.parametrize("profile", PROFILES)
def test_shared(fsr, profile, prefix, own, D, P, dtype, out_dtype, workgroups):
    announce(f"shared prefix, extreme scores: {profile} {prefix} {own} {D} {P} {dtype} {out_dtype} {workgroups}")
    gen = torch.Generator().manual_seed(3)
    b = shared.Batch(33, [(prefix, [(own, 3), (own + 9, 2)])], 1, 1, D, P, dtype)
    b.scale = PROFILES[profile][0]
    b.q.zero_()
    q = queries(profile, b.N)
    b.q[:b.N, :, :2] = q[:, None, None].to(dtype)
    z = products(profile, prefix + own + 9 + 2, gen)  # (by position, the same for both requests)
    parts = []
    for i, (_, c, n) in enumerate(b.reqs):
        s = shared.slots(b.bt[i], c + n, P)
        b.k.flatten(0, 1)[s, 0, :2] = z[:c + n].to(dtype)
        parts.append(attend(q[int(b.cu[i]):int(b.cu[i + 1])], z[:c + n], b.v.flatten(0, 1)[s, 0], b.scale, c + torch.arange(n)))
    same(profile, b.run(fsr, out_dtype, max_workgroups=workgroups), parts, dtype, times=2)
