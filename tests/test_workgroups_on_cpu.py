"""Kernels whose waves hand each other data through LDS, on the CPU with the waves in orders of our choice: no result may depend on it."""
import ctypes
import os

import pytest
import torch

import workgroup_on_cpu
from plain_attention import offsets
from plain_tree import sees_of, tree, walk, words_of

BF, F32 = torch.bfloat16, torch.float32
ORDERS = [0, 1, 2, 3]  # of waves: ascending, descending, two shuffles
U = 2.0 ** -24

pytestmark = pytest.mark.skipif(not os.path.exists(workgroup_on_cpu.CLANG), reason="no clang for the host")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    lib = workgroup_on_cpu.build(str(tmp_path_factory.mktemp("kernels")), ["library.hip", "token_logprobs.hip", "tree_accept.hip"])
    lib.fsr_last_error.restype = ctypes.c_char_p
    return lib


def pointer(x):
    return None if x is None else ctypes.c_void_p(x.data_ptr())


def aligned(n):
    """n bytes of a workspace."""
    room = torch.randint(0, 255, (n + 256,), dtype=torch.uint8)
    return room[-room.data_ptr() % 256:][:n]


def token_logprobs(lib, z, tokens, K, T=1.0, N_cap=None):
    """The first rows' results; N_cap: rows allocated, of which a call's cut depends."""
    from paper_2604_20503_amd.binding import LogprobParams

    (N, V), N_cap = z.shape, N_cap or len(z)
    p = LogprobParams(N_cap=N_cap, V=V, M=tokens.shape[1], K=K, dtype=int(z.dtype == BF), reserved=0, stride=V, temperature=T)
    need = ctypes.c_size_t()
    assert lib.fsr_logprob_workspace_bytes(ctypes.byref(p), ctypes.byref(need)) == 0
    ws, n_rows = aligned(need.value), torch.tensor([N], dtype=torch.int32)
    lp, entropy, ids, top = torch.empty(tokens.shape), torch.empty(N), torch.full((N, K), -7, dtype=torch.int32), torch.empty(N, K)
    rc = lib.fsr_token_logprobs(pointer(z), pointer(n_rows), pointer(tokens), pointer(lp), pointer(entropy), pointer(ids), pointer(top), ctypes.byref(p), pointer(ws),
                                ctypes.c_size_t(need.value), None)
    assert rc == 0, lib.fsr_last_error()
    return lp, entropy, ids, top


def rows(kind, V):
    gen = torch.Generator().manual_seed(V)
    if kind == "normal":
        return torch.randn(1, V, generator=gen) * 2.5
    if kind == "equal":  # every group has the largest logit: more groups than are listed
        return torch.zeros(1, V)
    z = torch.full((1, V), -float("inf"))  # a few that are allowed
    z[0, torch.randperm(V, generator=gen)[:9]] = torch.randn(9, generator=gen)
    return z


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("kind,V,K", [("normal", 5000, 5), ("normal", 700, 20), ("normal", 20000, 64), ("equal", 14000, 3), ("few", 6000, 20), ("normal", 3, 2)])
def test_alternatives_do_not_depend_on_the_order_of_waves(lib, kind, V, K, dtype, order):
    lib.set_wave_order(order)
    N_cap = 1024 if kind == "equal" else 1  # (a row in one chunk, of more groups than are listed; or in as many as it has tiles)
    z = rows(kind, V).to(dtype)
    tokens = torch.tensor([[0, V - 1]], dtype=torch.int32)
    lp, entropy, ids, top = token_logprobs(lib, z, tokens, K, N_cap=N_cap)
    x = z.double()
    want = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :K]
    assert torch.equal(ids, want.int())
    logp = torch.log_softmax(x, 1)
    # a sum of V weights, each off by 2 u and 3 u |x|, |x| < 40 where a weight counts; added up in any order: V u
    off = (V + 130) * U
    for got, exact in ((lp, logp.gather(1, tokens.long())), (top, logp.gather(1, want))):
        same = got.double() == exact
        assert (same | ((got.double() - exact).abs() <= off + U * exact.abs())).all()


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V,at,N_cap", [(3, 1, 1), (5000, 4999, 1), (20000, 0, 1), (14000, 7000, 1024)])
def test_digits_of_a_near_certain_token(lib, V, at, N_cap, dtype, order):
    """log p of a token that has nearly all the mass is about minus the mass of all others, and keeps its digits."""
    lib.set_wave_order(order)
    z = rows("normal", V)
    z[0, at] = 30.0
    z = z.to(dtype)
    lp, entropy, ids, _ = token_logprobs(lib, z, torch.tensor([[at]], dtype=torch.int32), 1, N_cap=N_cap)
    x = z.double() - 30.0
    x[0, at] = -float("inf")
    rest, much = x.exp().sum(), (x.exp() * x.clamp(min=-99)).sum()
    want, H = -torch.log1p(rest), torch.log1p(rest) - much / (1 + rest)
    # a weight is off by 3 u |x| + 2 u, |x| < 45; a thread adds V / 256 of them (or all of its tiles'), a few sums more; sums of 1 and more are
    # kept in 53 bits
    off = (137 + V / 256 + 60) * U
    assert ids[0, 0] == at and abs(lp[0, 0].double() - want) <= off * want.abs() + 2.0 ** -47
    assert abs(entropy[0].double() - H) <= 3 * off * H + 2.0 ** -47


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("at", [0, 700, 2999])
def test_one_logit_at_the_end_of_the_type(lib, at, order):
    """The lowest finite logit is the only one: it has all the mass."""
    lib.set_wave_order(order)
    z = torch.full((1, 3000), -float("inf"))
    z[0, at] = torch.finfo(F32).min
    lp, entropy, ids, top = token_logprobs(lib, z, torch.tensor([[at, (at + 1) % 3000]], dtype=torch.int32), 1)
    assert lp.tolist() == [[0.0, -float("inf")]] and entropy.tolist() == [0.0] and ids.tolist() == [[at]] and top.tolist() == [[0.0]]


@pytest.mark.parametrize("S_max", [0, 2, 40])
@pytest.mark.parametrize("sizes", [[12, 0, 1, 30], [64, 65, 130]], ids=str)
def test_acceptance_of_trees(lib, sizes, S_max):
    """Lanes one behind the other between the places where they wait for each other."""
    from paper_2604_20503_amd.binding import TreeParams

    lib.set_wave_order(0)
    gen = torch.Generator().manual_seed(4)
    B, N, cu, words = len(sizes), sum(sizes), offsets(sizes), 3
    parents = [tree(n, gen, 0.6) if n else [] for n in sizes]
    mask = torch.cat([words_of(sees_of(p), words) for p in parents if p])
    draft, target = (torch.randint(0, 2, (N,), generator=gen, dtype=torch.int32) for _ in "dt")
    accepted, emitted, path = (torch.full(s, -7, dtype=torch.int32) for s in ((2, B), (B, S_max + 1), (B, S_max + 1)))
    keep = torch.full((N,), 9, dtype=torch.uint8)
    p = TreeParams(B=B, N_cap=N, tree_words=words, S_max=S_max, reserved=0)
    rc = lib.fsr_tree_accept(*(pointer(x) for x in (target, draft, mask, cu, accepted[0], accepted[1], emitted, path, keep)), ctypes.byref(p), None)
    assert rc == 0, lib.fsr_last_error()
    for i, parent in enumerate(parents):
        a, b = int(cu[i]), int(cu[i + 1])
        rows, tokens = walk(parent, draft[a:b].tolist(), target[a:b].tolist(), S_max)
        pad = [-1] * (S_max + 1 - len(rows))
        assert path[i].tolist() == rows + pad and emitted[i].tolist() == tokens + pad
        assert accepted[:, i].tolist() == [len(rows) - 1, len(rows)] and keep[a:b].nonzero()[:, 0].tolist() == rows
