"""Rows whose largest score grows along the keys by more than an exponent reference is kept ahead of it (40 powers of two): the bf16 kernels
give up a tile in their loop over whole tiles, move the reference and take the loop up again.

Scores climb by CLIMB powers of two from chosen tiles of 64 keys on, by one column of the keys, in all rows or in some.  What is left behind
weighs 2^-CLIMB a step; half of the value columns are the larger by as much in earlier tiles, so that the sums in front of a step count in the
results as much as those behind it: a sum that is not rescaled, or twice, is off by its whole size.
"""
import math

import pytest
import torch

import test_gpu_latent as latent
import test_gpu_latent_expanded as expanded
import test_gpu_shared_prefix as shared
from gpu_utils import announce

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
CLIMB, QUERY = 45, 16.0
MOVES = {"second tile": [1], "third tile": [2], "last whole tile": [6], "second and third": [1, 2], "every tile": [1, 2, 3, 4, 5, 6]}
WHO = ["all rows", "some rows"]
TYPES = [(BF, BF), (BF, F32)]  # (the fp32 kernel keeps its references at the largest score: every test moves them)


@pytest.fixture(scope="module")
def fsr():
    import paper_2604_20503_amd as f
    f.load_library()
    return f


def climbed(moves, n):
    """Steps that the scores have climbed, by key."""
    tile = torch.arange(n) // 64
    return sum((tile >= m).long() for m in moves)


def key_element(steps, scale):
    """A key's element that adds CLIMB powers of two a step where the query's is QUERY."""
    return steps * (CLIMB * math.log(2) / (scale * QUERY))


def bigger(steps):
    """By how much values are larger: two steps' worth at most, which bf16 holds."""
    return 2.0 ** (CLIMB * (steps.max() - steps).clamp(max=2)).double()


def every_other(n):
    """A query's element: QUERY in some rows, 0 in the others."""
    return torch.where(torch.arange(n) // 3 % 2 == 1, QUERY, 0.0)


def query_element(who, n):
    return torch.full((n,), QUERY) if who == "all rows" else every_other(n)


@pytest.mark.parametrize("workgroups", [1, 0])
@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("shape", [(512, 64, 16), (512, 64, 7), (256, 32, 16)])
@pytest.mark.parametrize("who", WHO + ["the second 32 rows of a tile"])
@pytest.mark.parametrize("moves", MOVES.values(), ids=MOVES.keys())
def test_latent(fsr, moves, who, shape, dtype, out_dtype, workgroups):
    announce(f"latent attention, moving references: {moves} {who} {shape} {dtype} {out_dtype} {workgroups}")
    Dl, Dr, P = shape
    b = latent.Batch(21, [7 * 64 + 20, 7 * 64 + 3], [4, 1], 16, Dl, Dr, P, dtype)
    n = b.N * b.H
    element = torch.where(torch.arange(n) % 64 >= 32, QUERY, 0.0) if who.startswith("the second") else query_element(who, n)
    b.q[..., Dl] = element.view(b.N, b.H).to(dtype)
    b.q[..., :Dl // 2] = 0.0  # (columns of values that are large: not part of the scores)
    rows = b.cache.view(-1, Dl + Dr)
    for i in range(2):
        s = latent.slots(b.bt[i], b.ctx[i] + b.rows[i], P)
        steps = climbed(moves, len(s))
        rows[s, Dl] = key_element(steps, b.scale).to(dtype)
        rows[s, :Dl // 2] = (rows[s, :Dl // 2].double() * bigger(steps)[:, None]).to(dtype)
    latent.compare("moving references", b, latent.run(fsr, b, out_dtype, max_workgroups=workgroups))


@pytest.mark.parametrize("workgroups", [1, 0])
@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("dims", [expanded.BIG, expanded.SMALL])
@pytest.mark.parametrize("who", WHO)
@pytest.mark.parametrize("moves", MOVES.values(), ids=MOVES.keys())
def test_expanded(fsr, moves, who, dims, dtype, out_dtype, workgroups):
    announce(f"latent expanded, moving references: {moves} {who} {dims} {dtype} {out_dtype} {workgroups}")
    b = expanded.Batch(22, [40, 130], [7 * 64 + 60, 7 * 64 + 140], 1, dims, dtype)
    b.q[..., b.Dn] = query_element(who, b.q.shape[0])[:, None].to(dtype)
    at = 0
    for L in b.keys:
        steps = climbed(moves, L)
        b.rope[at:at + L, 0] = key_element(steps, b.scale).to(dtype)
        values = b.kv[at:at + L, :, b.Dn:b.Dn + b.Dv // 2]
        values.copy_((values.double() * bigger(steps)[:, None, None]).to(dtype))
        at += L
    b.compare("moving references", b.run(fsr, out_dtype, max_workgroups=workgroups))


@pytest.mark.parametrize("workgroups", [1, 0])
@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("shape", [(128, 16), (64, 5)])
@pytest.mark.parametrize("who", WHO)
@pytest.mark.parametrize("where", ["prefix", "own", "both"])
@pytest.mark.parametrize("moves", MOVES.values(), ids=MOVES.keys())
def test_shared(fsr, moves, where, who, shape, dtype, out_dtype, workgroups):
    announce(f"shared prefix, moving references: {moves} {where} {who} {shape} {dtype} {out_dtype} {workgroups}")
    D, P = shape
    prefix, own = {"prefix": (7 * 64 + 10, 30), "own": (32, 7 * 64 + 10), "both": (7 * 32 + 3, 7 * 32 + 10)}[where]
    b = shared.Batch(23, [(prefix, [(own, 3), (own + 9, 2)])], 4, 1, D, P, dtype)
    b.q[..., 0] = query_element(who, b.q.shape[0] * 4).view(-1, 4).to(dtype)
    # (the copies of a prefix's last page are different rows for different requests, and are to hold the same: values are scaled from a copy)
    v, k = b.v.flatten(0, 1), b.k.flatten(0, 1)
    old = v.clone()
    for i, (_, c, n) in enumerate(b.reqs):
        s = shared.slots(b.bt[i], c + n, P)
        steps = climbed(moves, prefix + own)  # (the requests' numbers of steps are the same, whatever their lengths)
        steps = torch.cat([steps, steps.max().expand(len(s) - len(steps))])
        k[s, :, 0] = key_element(steps, b.scale)[:, None].to(dtype)
        v[s, :, :D // 2] = (old[s, :, :D // 2].double() * bigger(steps)[:, None, None]).to(dtype)
    b.compare("moving references", b.run(fsr, out_dtype, max_workgroups=workgroups))
