"""Attention in 64 bits, row by row, for the tests of the calls over caches with several readers; and how far a kernel may be off.

A row's result is o = sum_t w_t v_t with w = softmax(z).  With A = sum_t w_t |v_t| (elementwise) an error of relative size e in
every weight moves o by at most e A, whatever the signs.  What makes such errors, in units of the value u = 2^-24 (half a step of
fp32, relative):
  scores: a sum of D products in fp32, any order: (D + 2) u S with S = scale * sum |q||k|; times scale * log2(e), rounded: 4 u |z|
  exponential: 2 u, its argument's own rounding: 4 u |z - m| <= 8 u max|z|;     sums over L keys: (L + 16) u, of weights and of products
The denominators carry the same, hence the factor 2.  Weights that enter the second product in bf16: 2^-8 (half a step); as a pair of
bf16: 2^-16.  A bf16 result: 2^-8 |o|.
"""
import torch

U = 2.0 ** -24


def attend(q, k, v, scale, last):
    """q [n, D], k [L, D], v [L, Dv] in any type, last [n]: last key that each row sees.  Returns o, lse, A and the relative error
    of fp32 arithmetic (per row)."""
    q, k, v = q.double(), k.double(), v.double()
    n, L = q.shape[0], k.shape[0]
    o, A = torch.zeros(n, v.shape[1], dtype=torch.float64), torch.zeros(n, v.shape[1], dtype=torch.float64)
    lse, e = torch.full((n,), float("-inf"), dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
    for r in range(n):
        m = min(int(last[r]) + 1, L)
        if m <= 0:
            continue
        z = (k[:m] @ q[r]) * scale
        lse[r] = torch.logsumexp(z, 0)
        w = torch.softmax(z, 0)
        o[r], A[r] = w @ v[:m], w @ v[:m].abs()
        S = float(((k[:m].abs() @ q[r].abs()) * scale).max())
        e[r] = 2 * ((q.shape[1] + 2) * S + 12 * float(z.abs().max()) + m + 18) * U
    return o, lse, A, e


def check(name, got, got_lse, o, lse, A, e, in_dtype):
    got, dtype = got.double().cpu(), got.dtype
    weights = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -16 if in_dtype == torch.bfloat16 else 0.0
    bound = (e[:, None] + weights) * A * 1.001 + 1e-37
    if dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (o.abs() + bound)
    assert not torch.isnan(got).any(), name
    off = (got - o).abs()
    worst = (off / bound).max().item() if off.numel() else 0.0
    assert worst <= 1.0, f"{name}: out is {worst:.3g} times what it may be off"
    if got_lse is not None:
        got_lse = got_lse.double().cpu()
        none = torch.isinf(lse)
        assert torch.equal(got_lse[none], lse[none]), name
        off = (got_lse - lse).abs()[~none]
        assert (off <= (e[~none] + 8 * U * (1 + lse[~none].abs()))).all(), f"{name}: lse is {off.max():.3g} off"


def pages(lens, P, gen, spare=2):
    """Block tables over a permuted pool: [B, max_pages] int32, pages in the pool."""
    need = [-(-int(x) // P) for x in lens]
    n_pages = sum(need) + spare
    perm = torch.randperm(n_pages, generator=gen).to(torch.int32)
    bt = torch.full((len(need), max(need + [1])), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        bt[i, :n] = perm[at:at + n]
        at += n
    return bt, n_pages


def offsets(lens):
    return torch.tensor([0] + list(torch.tensor(list(lens), dtype=torch.int64).cumsum(0)) if len(lens) else [0], dtype=torch.int32)


def slots(bt_row, L, P):
    """Slots of positions 0 .. L-1."""
    t = torch.arange(L)
    return bt_row[t // P].long() * P + t % P
