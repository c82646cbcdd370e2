"""The calls that verify trees of drafted tokens, and that report log probabilities, as measurable cases.

A request may bring a tree of drafts instead of a chain: its rows are rotated to the position of their depth on their way into
the paged cache (``kv_append_rope``), attend to the context and to their ancestors (``verify_attention_tree``), the path that
the target agrees with is found (``tree_accept``) and its keys and values move together (``kv_commit``); ``token_logprobs``
gives what a server reports of the answer.  With ``own`` false ``run`` computes them by elementary torch operations in 32
bits, with ``own`` true through the package.

``listed()`` gives the fixed cases, ``draw(rng)`` one more case of the same ranges, ``prepare(case, seed)`` what the program
holds on the GPU before the call, ``run(state)`` one pass, ``work(case)`` the bytes and operations a pass cannot do without
and ``exact(case, seed)`` the result in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
INF = float("inf")


# ---------------------------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one user's small tree enters the cache: the smallest call there is
        dict(name="rope_b1", kind="rope", dtype="bf16", cache="same", B=1, H_q=32, H_kv=8, D=128, R=128, pairs=False, P=16, layout="head",
             ctx_lo=900, ctx_hi=900, rows_lo=8, rows_hi=8, tree=True, lengths=1),
        # chunks of prompts enter 8-bit caches, wide query groups, the token-major layout
        dict(name="rope_kv8_b5", kind="rope", dtype="bf16", cache="kv8", B=5, H_q=64, H_kv=8, D=128, R=128, pairs=False, P=16, layout="token",
             ctx_lo=0, ctx_hi=700, rows_lo=300, rows_hi=1024, tree=False, lengths=2),
        # one user's tree behind a short context: latency
        dict(name="tree_b1", kind="tree", dtype="bf16", B=1, H_q=32, H_kv=8, D=128, P=16, layout="head", ctx_lo=777, ctx_hi=777, rows_lo=12,
             rows_hi=12, lengths=3),
        # the ordinary batch, trees of 24 to 64 tokens: the caches are read at memory speed
        dict(name="tree_b16", kind="tree", dtype="bf16", B=16, H_q=32, H_kv=8, D=128, P=16, layout="head", ctx_lo=1024, ctx_hi=4096, rows_lo=24,
             rows_hi=64, lengths=4),
        # large trees, wide query groups, long contexts, pages of 64 tokens: bound by the matrix cores
        dict(name="tree_wide_b12", kind="tree", dtype="bf16", B=12, H_q=64, H_kv=8, D=128, P=64, layout="token", ctx_lo=2048, ctx_hi=16384,
             rows_lo=33, rows_hi=150, lengths=5),
        # heads of 64 at full precision, the package's debugging workload
        dict(name="tree_f32_b8", kind="tree", dtype="f32", B=8, H_q=8, H_kv=2, D=64, P=16, layout="head", ctx_lo=0, ctx_hi=600, rows_lo=1,
             rows_hi=16, lengths=6),
        # the rows of one user's answer, five alternatives each: few rows, latency
        dict(name="logprob_b5", kind="logprob", dtype="bf16", N=5, V=128256, M=1, K=5, temperature=1.0, masked=False),
        # the rows of a loaded server's step at full precision, some of them under a grammar that masks most tokens
        dict(name="logprob_f32_b400", kind="logprob", dtype="f32", N=400, V=152064, M=3, K=20, temperature=0.7, masked=True),
        # one user's tree
        dict(name="accept_b1", kind="accept", B=1, rows_lo=12, rows_hi=12, S_max=6, lengths=9),
        # a loaded server's trees, some beyond 64 rows
        dict(name="accept_b256", kind="accept", B=256, rows_lo=8, rows_hi=160, S_max=12, lengths=10),
        # the accepted paths of a handful of users in 16-bit caches
        dict(name="commit_b4", kind="commit", cache="bf16", B=4, H_kv=8, D=128, P=16, layout="head", ctx_lo=100, ctx_hi=600, rows_lo=24, rows_hi=64,
             S_max=8, lengths=11),
        # a loaded server's, in 8-bit caches
        dict(name="commit_kv8_b256", kind="commit", cache="kv8", B=256, H_kv=8, D=128, P=16, layout="token", ctx_lo=16, ctx_hi=300, rows_lo=16,
             rows_hi=64, S_max=8, lengths=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn(rng):
    kind = rng.choice(["rope", "rope", "tree", "tree", "tree", "logprob", "logprob", "accept", "commit"])
    if kind == "logprob":
        return dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]), N=_log_int(rng, 1, 600), V=rng.choice([128256, 152064, 32000, 5000, _log_int(rng, 100, 200000)]),
                    M=rng.randint(1, 8), K=rng.choice([1, 5, 20, rng.randint(2, 32)]), temperature=rng.choice([1.0, 1.0, 0.7, 1.3]), masked=rng.random() < 0.4)
    lengths = rng.randrange(1 << 30)
    rows_lo = _log_int(rng, 1, 64)
    rows = dict(rows_lo=rows_lo, rows_hi=max(rows_lo, _log_int(rng, 4, 220)), lengths=lengths)
    if kind == "accept":
        return dict(kind=kind, B=_log_int(rng, 1, 500), S_max=rng.randint(1, 16), **rows)
    ctx_lo = rng.choice([0, _log_int(rng, 1, 1024)])
    P, layout = rng.choice([16, 16, 64, 32, rng.randint(1, 60)]), rng.choice(["head", "token"])
    if kind == "commit":
        return dict(kind=kind, cache=rng.choice(["bf16", "f32", "kv8"]), B=_log_int(rng, 1, 300), H_kv=rng.choice([1, 2, 4, 8]), D=rng.choice([64, 128, 128]),
                    P=P, layout=layout, ctx_lo=ctx_lo % 200, ctx_hi=ctx_lo % 200 + rng.randint(0, 300), S_max=rng.randint(1, 12), **rows)
    H_q, H_kv = rng.choice([(32, 8), (8, 2), (28, 4), (16, 16), (64, 8), (20, 4)])
    if kind == "rope":
        kv8 = rng.random() < 0.3
        D = rng.choice([64, 128, 128])
        tree = rng.random() < 0.6
        if not tree and rng.random() < 0.5:
            rows.update(rows_hi=rows_lo + _log_int(rng, 8, 900))
        return dict(kind=kind, dtype="bf16" if kv8 else rng.choice(["bf16", "bf16", "f32"]), cache="kv8" if kv8 else "same", B=_log_int(rng, 1, 64), H_q=H_q, H_kv=H_kv,
                    D=D, R=rng.choice([D, D, D // 2]), pairs=rng.random() < 0.3, P=P, layout=layout, ctx_lo=ctx_lo, ctx_hi=ctx_lo + rng.randint(0, 600), tree=tree, **rows)
    f32 = rng.random() < 0.2
    return dict(kind=kind, dtype="f32" if f32 else "bf16", B=_log_int(rng, 1, 8 if f32 else 48), H_q=H_q, H_kv=H_kv, D=rng.choice([64, 128, 128]), P=P, layout=layout,
                ctx_lo=ctx_lo, ctx_hi=max(ctx_lo, _log_int(rng, 64, 2048 if f32 else 16384)), **rows)


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        case = _drawn(rng)
        if _cost(case) <= most and _padded_scores(case) <= 3 << 30:
            return case


def _padded_scores(case):
    """Scores that the plain form of attention holds at once."""
    if case["kind"] != "tree":
        return 0
    ctx, rows = _lengths(case)
    return case["B"] * int(rows.max()) * case["H_q"] * int((ctx + rows).max())


# ---------------------------------------------------------------------------------------------------------------
# lengths, offsets, trees and page tables: a function of the case alone, so that its work is known without its data
# ---------------------------------------------------------------------------------------------------------------
def _lengths(case):
    """(tokens in front of the call's rows, rows) of every request."""
    rng = np.random.Generator(np.random.PCG64(case["lengths"]))
    rows = rng.integers(case["rows_lo"], case["rows_hi"] + 1, size=case["B"])
    ctx = rng.integers(case["ctx_lo"], case["ctx_hi"] + 1, size=case["B"]) if "ctx_lo" in case else np.zeros(case["B"], np.int64)
    return ctx, rows


def _offsets(lens):
    cu = np.zeros(len(lens) + 1, np.int32)
    np.cumsum(lens, out=cu[1:])
    return cu


def _trees(case, rows):
    """Parent of every row within its request (-1: the first row) and the rows that it sees, [N, W] int64.  Rows are in the order in
    which a drafter that extends its best leaves finds them: parents lie in front, near the root rather than far from it."""
    rng = np.random.Generator(np.random.PCG64(case["lengths"] + 1))
    B, most = len(rows), int(rows.max())
    W = -(-most // 64)
    parent = np.full((B, most), -1, np.int64)
    mask = np.zeros((B, most, W), np.uint64)
    every = np.arange(B)
    for j in range(most):
        if j:
            parent[:, j] = np.minimum((j * rng.random(B) ** 1.6).astype(np.int64), j - 1)
            mask[:, j] = mask[every, parent[:, j]]
        mask[:, j, j // 64] |= np.uint64(1 << (j % 64))
    there = np.arange(most)[None, :] < rows[:, None]
    return parent[there], mask[there].view(np.int64)


def _depths(mask):
    return np.unpackbits(mask.view(np.uint8), axis=1).sum(1).astype(np.int64) - 1


def _elem(case):
    return {"bf16": 2, "f32": 4, "kv8": 1}[case["dtype"] if case.get("cache", "same") == "same" else case["cache"]]


def work(case):
    if case["kind"] == "logprob":
        N, e = case["N"], 2 if case["dtype"] == "bf16" else 4
        return dict(bytes=N * (case["V"] * e + 4 * (2 * case["M"] + 2 * case["K"] + 1)), flops=0)
    ctx, rows = _lengths(case)
    N, B, words = int(rows.sum()), case["B"], -(-int(rows.max()) // 64)
    if case["kind"] == "accept":
        return dict(bytes=N * (8 + 8 * words) + B * 4 * (3 + 2 * (case["S_max"] + 1)), flops=0)
    row = case["H_kv"] * case["D"]
    if case["kind"] == "commit":
        moved = int(np.minimum(rows - 1, case["S_max"]).sum()) // 2  # about half of the longest paths
        return dict(bytes=max(4 * row * moved * _elem(case), 64) + 4 * B * (case["S_max"] + 3), flops=0)
    if case["kind"] == "rope":
        e = 2 if case["dtype"] == "bf16" else 4
        return dict(bytes=N * (2 * case["H_q"] * case["D"] * e + 2 * row * (e + _elem(case)) + 4 * case["R"] + (8 * words if case["tree"] else 0)), flops=0)
    _, mask = _trees(case, rows)
    seen = float((rows * ctx).sum() + (_depths(mask) + 1).sum())  # (row, key) pairs that are not masked
    e = _elem(case)
    return dict(bytes=int((ctx + rows).sum()) * 2 * row * e + N * (case["H_q"] * (2 * case["D"] * e + 4) + 8 * words), flops=4 * seen * case["H_q"] * case["D"])


# ---------------------------------------------------------------------------------------------------------------
# what the program holds before the call
# ---------------------------------------------------------------------------------------------------------------
def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _normal(gen, shape, dtype, sigma=1.0):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for a in range(0, flat.numel(), 1 << 28):
        n = min(1 << 28, flat.numel() - a)
        flat[a:a + n] = (torch.randn(n, generator=gen, device="cuda", dtype=torch.float32) * sigma).to(dtype)
    return out


def _tables(case, ctx, rows, seed):
    """Block tables over a permuted pool."""
    rng = np.random.Generator(np.random.PCG64(seed))
    pages = -(-(ctx + rows) // case["P"])
    n_pages = int(pages.sum()) + 3
    perm = rng.permutation(n_pages).astype(np.int32)
    bt = np.full((case["B"], int(pages.max())), -1, np.int32)
    bt[np.arange(bt.shape[1])[None, :] < pages[:, None]] = perm[:int(pages.sum())]
    return bt, n_pages


def _caches(case, gen, n_pages, dtype):
    shape = (n_pages, case["H_kv"], case["P"], case["D"]) if case["layout"] == "head" else (n_pages, case["P"], case["H_kv"], case["D"])
    if dtype == "kv8":  # finite codes: bytes of E4M3
        return tuple(_normal(gen, shape, torch.float32).to(torch.float8_e4m3fn).view(torch.uint8) for _ in "kv")
    return tuple(_normal(gen, shape, dtype) for _ in "kv")


def _tokens(case, seed, parent, cu, rows):
    """Drafted tokens of all rows, and the target's choice at each: a child's token at most of them."""
    rng = np.random.Generator(np.random.PCG64(seed))
    N = int(cu[-1])
    draft = rng.integers(0, 128256, size=N).astype(np.int32)
    target = rng.integers(0, 128256, size=N).astype(np.int32)
    child = np.flatnonzero(parent >= 0)
    child = rng.permutation(child)  # of several children one at random
    of = (parent + np.repeat(cu[:-1], rows))[child]
    agree = rng.random(N) < 0.75
    target[of[agree[of]]] = draft[child[agree[of]]]
    return draft, target


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["kind"] == "logprob":
        N, V, M = case["N"], case["V"], case["M"]
        z = _normal(gen, (N, V), DTYPES[case["dtype"]], 2.5)
        # a few likely tokens in every row, as a model that knows what it says has them
        likely = torch.randint(0, V, (N, 6), generator=gen, device="cuda")
        z.scatter_(1, likely, (6.0 + 8.0 * torch.rand((N, 6), generator=gen, device="cuda")).to(z.dtype))
        tokens = torch.randint(0, V, (N, M), generator=gen, device="cuda", dtype=torch.int32)
        tokens[:, 0] = likely[:, 0].int()
        if case["masked"]:  # a grammar allows a tenth of the tokens of every second row
            allowed = torch.rand((N, V), generator=gen, device="cuda") < 0.1
            allowed.scatter_(1, likely, True)
            allowed[1::2] = True
            z.masked_fill_(~allowed, -INF)
        return dict(case=case, z=z, tokens=tokens)
    ctx, rows = _lengths(case)
    parent, mask = _trees(case, rows)
    cu, N, B = _offsets(rows), int(rows.sum()), case["B"]
    s = dict(case=case, N=N, q_max=int(rows.max()), k_max=int((ctx + rows).max()), ctx=_dev(ctx.astype(np.int32)), cu_q=_dev(cu), mask=_dev(mask))
    if case["kind"] in ("accept", "commit"):
        draft, target = _tokens(case, seed, parent, cu, rows)
        s.update(draft=_dev(draft), target=_dev(target))
    if case["kind"] == "accept":
        return s
    bt, n_pages = _tables(case, ctx, rows, seed)
    dtype = DTYPES.get(case["dtype"] if "dtype" in case else case["cache"])
    k, v = _caches(case, gen, n_pages, "kv8" if case.get("cache") == "kv8" else dtype)
    s.update(bt=_dev(bt), n_pages=n_pages, k=k, v=v)
    if case["kind"] == "commit":
        s["accepted"], _, _, s["path"] = _plain_accept(s)
        return s
    s["q"] = _normal(gen, (N, case["H_q"], case["D"]), dtype)
    if case["kind"] == "tree":
        s["scale"] = case["D"] ** -0.5
        return s
    s.update(k_new=_normal(gen, (N, case["H_kv"], case["D"]), dtype), v_new=_normal(gen, (N, case["H_kv"], case["D"]), dtype))
    turn = torch.arange(s["k_max"], device="cuda", dtype=torch.float64)[:, None] * 500000.0 ** (-torch.arange(0, case["R"], 2, device="cuda", dtype=torch.float64) / case["R"])
    s["cos_sin"] = torch.cat([turn.cos(), turn.sin()], 1).float()
    if case["cache"] == "kv8":
        s.update(k_scale=0.01 + 0.02 * torch.rand(case["H_kv"], generator=gen, device="cuda"), v_scale=0.01 + 0.02 * torch.rand(case["H_kv"], generator=gen, device="cuda"))
    return s


# ---------------------------------------------------------------------------------------------------------------
# one pass, in plain form
# ---------------------------------------------------------------------------------------------------------------
def _owners(s):
    """Request of every row, and its place in it."""
    i = torch.repeat_interleave(torch.arange(s["case"]["B"], device="cuda"), s["cu_q"].diff().long(), output_size=s["N"])
    return i, torch.arange(s["N"], device="cuda") - s["cu_q"][i]


def _slots(s, i, pos):
    """Slot in the pool of positions `pos` of requests `i`."""
    P = s["case"]["P"]
    return s["bt"][i, pos // P].long() * P + pos % P


def _of_tokens(x, layout):
    """A cache as [pages, P, H, D] (a view)."""
    return x.transpose(1, 2) if layout == "head" else x


def _bits(s):
    """[N, 64 W]: whether a row sees a row of its request."""
    return ((s["mask"][:, :, None] >> torch.arange(64, device="cuda")) & 1).flatten(1).bool()


def _rotate(x, table, R, pairs):
    c, n = table[:, None, :R // 2], table[:, None, R // 2:]
    x = x.float()
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if pairs else (x[..., :R // 2], x[..., R // 2:R])
    y, z = a * c - b * n, b * c + a * n
    turned = torch.stack([y, z], -1).flatten(2) if pairs else torch.cat([y, z], 2)
    return torch.cat([turned, x[..., R:]], 2)


def _plain_rope(s):
    case = s["case"]
    i, j = _owners(s)
    pos = s["ctx"][i] + (_bits(s).sum(1) - 1 if case["tree"] else j)
    table = s["cos_sin"][pos]
    q, k = (_rotate(s[x], table, case["R"], case["pairs"]) for x in ("q", "k_new"))
    v, at = s["v_new"].float(), _slots(s, i, s["ctx"][i] + j)
    if case["cache"] == "kv8":
        k, v = ((x / sc[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for x, sc in ((k, s["k_scale"]), (v, s["v_scale"])))
    for cache, x in ((s["k"], k), (s["v"], v)):
        _of_tokens(cache, case["layout"])[at // case["P"], at % case["P"]] = x.to(cache.dtype)
    return q.to(s["q"].dtype), _values(s["k"]), _values(s["v"])


def _values(cache):
    return cache.view(torch.float8_e4m3fn) if cache.dtype == torch.uint8 else cache


def _plain_tree(s):
    case = s["case"]
    B, H_q, H_kv, D, q_max, k_max = case["B"], case["H_q"], case["H_kv"], case["D"], s["q_max"], s["k_max"]
    G = H_q // H_kv
    i, j = _owners(s)
    pos = torch.arange(k_max, device="cuda")
    at = _slots(s, torch.arange(B, device="cuda")[:, None], pos[None, :]).clamp(min=0)
    k, v = (_of_tokens(s[x], case["layout"])[at // case["P"], at % case["P"]].float() for x in "kv")
    rows = (s["cu_q"][:-1, None] + torch.arange(q_max, device="cuda")).clamp(max=s["N"] - 1)
    q = s["q"][rows].float().view(B, q_max, H_kv, G, D).permute(0, 2, 1, 3, 4).reshape(B, H_kv, q_max * G, D)
    z = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()).mul_(s["scale"])
    row_of = pos[None, :] - s["ctx"][:, None]  # of the request's rows, the one that a key belongs to
    bits = _bits(s)[rows]
    seen = torch.gather(bits, 2, row_of.clamp(0, bits.shape[2] - 1)[:, None, :].expand(-1, q_max, -1)) & (row_of < bits.shape[2])[:, None]
    seen = torch.where((row_of < 0)[:, None], True, seen)
    z.view(B, H_kv, q_max, G, k_max).masked_fill_(~seen[:, None, :, None, :], -INF)
    m = z.amax(-1, keepdim=True)
    e = z.sub_(m).exp_()
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e, v.transpose(1, 2).contiguous()) / total
    back = lambda x: x.view(B, H_kv, q_max, G, -1)[i, :, j]  # noqa: E731
    return back(o).reshape(-1, H_q, D).to(s["q"].dtype), back(m + torch.log(total)).reshape(-1, H_q)


def _plain_logprob(s):
    K, T = s["case"]["K"], s["case"]["temperature"]
    z = s["z"].float()
    m = z.amax(1, keepdim=True)
    x = (z - m) / T
    e = x.exp()
    total = e.sum(1, keepdim=True)
    logp = lambda at: torch.gather(x, 1, at) - total.log()  # noqa: E731
    entropy = total.log()[:, 0] - torch.where(e > 0, e * x, 0.0).sum(1) / total[:, 0]
    top = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :K]
    return logp(s["tokens"].long()), entropy, top.int(), logp(top)


def _plain_accept(s):
    N, S = s["N"], s["case"]["S_max"]
    i, j = _owners(s)
    bits = _bits(s)
    places = torch.arange(bits.shape[1], device="cuda")
    above = bits & (places < j[:, None])
    parent = torch.where(above, places, -1).amax(1)
    first = s["cu_q"][i].long()
    agrees = (parent >= 0) & (s["draft"] == s["target"][first + parent.clamp(min=0)])
    # of several children with the token, the first
    best = torch.full((N,), N, device="cuda").scatter_reduce(0, (first + parent.clamp(min=0))[agrees], torch.arange(N, device="cuda")[agrees], "amin")
    chosen = (agrees & (best[first + parent.clamp(min=0)] == torch.arange(N, device="cuda"))) | (j == 0)
    depth = bits.sum(1) - 1
    padded = chosen[(first[:, None] + places).clamp(max=N - 1)]
    on_path = (padded | ~bits).all(1) & (depth <= S)
    B = s["case"]["B"]
    path = torch.full((B, S + 1), -1, dtype=torch.int32, device="cuda")
    path[i[on_path], depth[on_path]] = j[on_path].int()
    emitted = torch.full((B, S + 1), -1, dtype=torch.int32, device="cuda")
    emitted[i[on_path], depth[on_path]] = s["target"][on_path]
    n = torch.zeros(B, dtype=torch.int32, device="cuda").index_add_(0, i, on_path.int())
    return n - 1, n, emitted, path


def _plain_commit(s):
    case = s["case"]
    S, P = case["S_max"], case["P"]
    step = torch.arange(1, S + 1, device="cuda")
    i, k = torch.nonzero(step[None, :] <= s["accepted"][:, None], as_tuple=True)
    k = k + 1
    source, to = _slots(s, i, s["ctx"][i] + s["path"][i, k]), _slots(s, i, s["ctx"][i] + k)
    for cache in (s["k"], s["v"]):
        x = _of_tokens(cache, case["layout"])
        x[to // P, to % P] = x[source // P, source % P]
    return _values(s["k"]), _values(s["v"])


PLAIN = dict(rope=_plain_rope, tree=_plain_tree, logprob=_plain_logprob, accept=_plain_accept, commit=_plain_commit)


# ---------------------------------------------------------------------------------------------------------------
# one pass, through the package
# ---------------------------------------------------------------------------------------------------------------
def _own(s):
    import paper_2604_20503_amd as fsr

    case = s["case"]
    kind = case["kind"]
    if kind == "logprob":
        return fsr.token_logprobs(s["z"], s["tokens"], top_k=case["K"], temperature=case["temperature"])
    if kind == "accept":
        return fsr.tree_accept(s["target"], s["draft"], s["mask"], s["cu_q"], S_max=case["S_max"])
    layout = fsr.binding.KV_HEAD_MAJOR if case["layout"] == "head" else fsr.binding.KV_TOKEN_MAJOR
    if kind == "commit":
        fsr.kv_commit(s["k"], s["v"], s["bt"], s["ctx"], s["accepted"], s["path"], kv_layout=layout)
        return _values(s["k"]), _values(s["v"])
    if kind == "rope":
        q = fsr.kv_append_rope(s["q"], s["k_new"], s["v_new"], s["cos_sin"], s["k"], s["v"], s["bt"], s["ctx"], s["cu_q"],
                               tree_mask=s["mask"] if case["tree"] else None, pairs=case["pairs"], k_scale=s.get("k_scale"), v_scale=s.get("v_scale"), kv_layout=layout)
        return q, _values(s["k"]), _values(s["v"])
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
    return fsr.verify_attention_tree(s["q"], s["k"], s["v"], s["bt"], s["ctx"], s["cu_q"], s["mask"], scale=s["scale"], lse=lse, max_q_len=s["q_max"],
                                     kv_layout=layout)


def run(state):
    return _own(state) if own else PLAIN[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _exact_logprob(s):
    case = s["case"]
    logp = torch.log_softmax(s["z"].double() / case["temperature"], 1)
    ranked = torch.sort(s["z"].double(), 1, descending=True).values[:, :case["K"]] / case["temperature"]
    return (torch.gather(logp, 1, s["tokens"].long()), torch.special.entr(logp.exp()).sum(1), None,
            ranked - torch.logsumexp(s["z"].double() / case["temperature"], 1, keepdim=True))


def _exact_rope(s):
    """Rows as complex numbers, turned; a row at a time into the pages."""
    case, R = s["case"], s["case"]["R"]
    ctx, rows = _lengths(case)
    _, mask = _trees(case, rows)
    cu, bt, depth = _offsets(rows), s["bt"].cpu().numpy(), _depths(mask)
    turned = []
    owner = np.repeat(np.arange(case["B"]), rows)
    place = np.arange(s["N"]) - cu[owner]
    table = s["cos_sin"][_dev(ctx[owner] + (depth if case["tree"] else place))].double()
    turn = torch.complex(table[:, :R // 2].contiguous(), table[:, R // 2:].contiguous())[:, None]
    for x in (s["q"].double(), s["k_new"].double()):
        pair = x[..., :R].reshape(*x.shape[:2], R // 2, 2) if case["pairs"] else x[..., :R].reshape(*x.shape[:2], 2, R // 2).transpose(2, 3)
        y = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
        x[..., :R] = y.reshape(*x.shape[:2], R) if case["pairs"] else y.transpose(2, 3).reshape(*x.shape[:2], R)
        turned.append(x)
    new = [turned[1], s["v_new"].double()]
    out = []
    for x, cache, scale in zip(new, (s["k"], s["v"]), (s.get("k_scale"), s.get("v_scale"))):
        if scale is not None:
            x = x / scale.double()[:, None]
        cache = _values(cache).double()
        page, slot = _dev(bt[owner, (ctx[owner] + place) // case["P"]].astype(np.int64)), _dev((ctx[owner] + place) % case["P"])
        if case["layout"] == "head":
            cache.permute(0, 2, 1, 3)[page, slot] = x
        else:
            cache[page, slot] = x
        out.append(cache)
    return turned[0], out[0], out[1]


def _exact_tree(s):
    case = s["case"]
    ctx, rows = _lengths(case)
    _, mask = _trees(case, rows)
    cu, G = _offsets(rows), case["H_q"] // case["H_kv"]
    outs, lses = [], []
    for i in range(case["B"]):
        n, c = int(rows[i]), int(ctx[i])
        pages = s["bt"][i, :-(-(c + n) // case["P"])].long()
        k, v = (s[x][pages].double() for x in "kv")
        if case["layout"] == "head":
            k, v = k.transpose(1, 2), v.transpose(1, 2)
        k, v = (x.reshape(-1, case["H_kv"], case["D"])[:c + n].permute(1, 0, 2).contiguous() for x in (k, v))
        seen = np.unpackbits(mask[cu[i]:cu[i + 1]].view(np.uint8), axis=1, bitorder="little")[:, :n].astype(bool)
        seen = torch.cat([torch.ones((n, c), dtype=torch.bool, device="cuda"), _dev(seen)], 1)
        q = s["q"][int(cu[i]):int(cu[i + 1])].double().view(n, case["H_kv"], G, case["D"])
        for g in range(G):
            z = torch.matmul(q[:, :, g].transpose(0, 1).contiguous(), k.transpose(1, 2).contiguous()) * s["scale"]
            z.masked_fill_(~seen, -INF)
            outs.append(torch.matmul(torch.softmax(z, -1), v).transpose(0, 1))
            lses.append(torch.logsumexp(z, -1).transpose(0, 1))
        outs[-G:] = [torch.stack(outs[-G:], 2).reshape(n, case["H_q"], -1)]
        lses[-G:] = [torch.stack(lses[-G:], 2).reshape(n, case["H_q"])]
    return torch.cat(outs), torch.cat(lses)


def _exact_commit(s):
    """Row by row, from the last committed one on."""
    case = s["case"]
    bt, ctx, n, path = (s[x].cpu().numpy() for x in ("bt", "ctx", "accepted", "path"))
    out = []
    for cache in (s["k"], s["v"]):
        x = _values(cache).double()
        y = x.permute(0, 2, 1, 3) if case["layout"] == "head" else x
        for i in range(case["B"]):
            for k in range(1, int(n[i]) + 1):
                a, b = int(ctx[i]) + int(path[i, k]), int(ctx[i]) + k
                y[int(bt[i, b // case["P"]]), b % case["P"]] = y[int(bt[i, a // case["P"]]), a % case["P"]]
        out.append(x)
    return out


EXACT = dict(rope=_exact_rope, tree=_exact_tree, logprob=_exact_logprob, commit=_exact_commit)


def exact(case, seed):
    if case["kind"] not in EXACT or work(case)["flops"] > 2e12:
        return None
    return EXACT[case["kind"]](prepare(case, seed))
