"""The attention calls over caches that several readers share, as measurable cases.

A target model whose attention reads one shared latent vector per token (``latent_append``, ``latent_gather``,
``latent_attention``, ``latent_attention_expanded``), and a batch whose requests share a long prefix
(``verify_attention_shared``).  With ``own`` false ``run`` computes them by elementary torch operations in 32 bits,
with ``own`` true through the package.

``listed()`` gives the fixed cases, ``draw(rng)`` one more case of the same ranges, ``prepare(case, seed)`` what the
program holds on the GPU before the call, ``run(state)`` one pass, ``work(case)`` the bytes and operations a pass
cannot do without and ``exact(case, seed)`` the result in 64 bits.
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
        # one user's decode step, the smallest call there is: four rows of one layer enter the latent cache
        dict(name="append_b1", kind="append", dtype="bf16", B=1, D_latent=512, D_rope=64, P=16, ctx_lo=257, ctx_hi=257,
             spec_lo=3, spec_hi=3, lengths=1),
        # prompts of a debugging run at full precision enter the cache, hundreds of rows a request
        dict(name="append_f32_b24", kind="append", dtype="f32", B=24, D_latent=512, D_rope=64, P=16, ctx_lo=0,
             ctx_hi=600, spec_lo=100, spec_hi=700, lengths=2),
        # contexts of a handful of requests are read back for the expanded form
        dict(name="gather_b8", kind="gather", dtype="bf16", B=8, D_latent=512, D_rope=64, P=16, ctx_lo=300, ctx_hi=2500,
             spec_lo=0, spec_hi=8, lengths=3),
        # a loaded server's contexts, small latent, pages of 64
        dict(name="gather_b96", kind="gather", dtype="bf16", B=96, D_latent=256, D_rope=32, P=64, ctx_lo=512,
             ctx_hi=8192, spec_lo=0, spec_hi=8, lengths=4),
        # single token of one user, a tensor-parallel share of the heads: latency
        dict(name="latent_b1", kind="latent", dtype="bf16", B=1, H=16, D_latent=512, D_rope=64, P=16, ctx_lo=777,
             ctx_hi=777, spec_lo=0, spec_hi=0, lengths=5),
        # an ordinary verification batch on a share of the heads: the cache is read at memory speed
        dict(name="latent_b32", kind="latent", dtype="bf16", B=32, H=16, D_latent=512, D_rope=64, P=16, ctx_lo=1024,
             ctx_hi=8192, spec_lo=1, spec_hi=8, lengths=6),
        # all heads on one GPU, requests with up to three drafts: bound by the matrix cores
        dict(name="latent_h128_b64", kind="latent", dtype="bf16", B=64, H=128, D_latent=512, D_rope=64, P=64,
             ctx_lo=512, ctx_hi=4096, spec_lo=0, spec_hi=3, lengths=7),
        # prompts that join a running batch, some behind a cached context
        dict(name="expanded_b4", kind="expanded", dtype="bf16", B=4, H=16, D_nope=128, D_rope=64, D_v=128, ctx_lo=0,
             ctx_hi=2048, spec_lo=200, spec_hi=700, lengths=8),
        # one chunk of a long prompt behind 6000 tokens of it
        dict(name="expanded_long", kind="expanded", dtype="bf16", B=1, H=32, D_nope=128, D_rope=64, D_v=128,
             ctx_lo=6000, ctx_hi=6000, spec_lo=2047, spec_hi=2047, lengths=9),
        # heads of 64 at full precision (the package's debugging workload) behind a short common instruction
        dict(name="shared_f32_b8", kind="shared", dtype="f32", B=8, H_q=8, H_kv=2, D=64, P=16, layout="head", groups=1,
             prefix_lo=437, prefix_hi=437, ctx_lo=0, ctx_hi=200, spec_lo=0, spec_hi=4, lengths=10),
        # one long system prompt in front of a batch of conversations
        dict(name="shared_b64", kind="shared", dtype="bf16", B=64, H_q=32, H_kv=8, D=128, P=16, layout="head",
             groups=1, prefix_lo=8192, prefix_hi=8192, ctx_lo=64, ctx_hi=1024, spec_lo=1, spec_hi=8, lengths=11),
        # several long documents, each with many questions, wide query groups, the token-major layout
        dict(name="shared_wide_b192", kind="shared", dtype="bf16", B=192, H_q=64, H_kv=8, D=128, P=16, layout="token",
             groups=4, prefix_lo=2000, prefix_hi=16000, ctx_lo=16, ctx_hi=512, spec_lo=0, spec_hi=7, lengths=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn(rng):
    kind = rng.choice(["append", "gather", "latent", "latent", "expanded", "expanded", "shared", "shared"])
    lengths = rng.randrange(1 << 30)
    spec_lo = rng.randint(0, 3)
    spec = dict(spec_lo=spec_lo, spec_hi=spec_lo + rng.randint(0, 7), lengths=lengths)
    ctx_lo = _log_int(rng, 1, 1024)
    ctx = dict(ctx_lo=ctx_lo, ctx_hi=max(ctx_lo, _log_int(rng, 128, 8192)))
    D_latent, D_rope = rng.choice([(512, 64), (512, 64), (512, 64), (256, 32), (256, 64), (512, 32)])
    P = rng.choice([16, 16, 64, 32, rng.randint(1, 100)])
    latent = dict(D_latent=D_latent, D_rope=D_rope, P=P)
    if kind in ("append", "gather"):
        case = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]), B=_log_int(rng, 1, 256), **latent, **ctx, **spec)
        if rng.random() < 0.5:
            case.update(spec_hi=spec_lo + _log_int(rng, 8, 600))
        return case
    if kind == "latent":
        f32 = rng.random() < 0.15
        return dict(kind=kind, dtype="f32" if f32 else "bf16", B=_log_int(rng, 1, 8 if f32 else 96),
                    H=rng.choice([8, 16, 16, 32, 64, 128, rng.randint(1, 128)]), **latent, **ctx, **spec)
    if kind == "expanded":
        D_nope, D_rope, D_v = rng.choice([(128, 64, 128), (128, 64, 128), (64, 32, 64)])
        B = _log_int(rng, 1, 16)
        rows_lo = _log_int(rng, 1, 500)
        return dict(kind=kind, dtype="f32" if rng.random() < 0.15 else "bf16", B=B, H=rng.choice([4, 16, 16, 32, 64, rng.randint(1, 64)]),
                    D_nope=D_nope, D_rope=D_rope, D_v=D_v, ctx_lo=rng.choice([0, 0, _log_int(rng, 1, 2048)]),
                    ctx_hi=_log_int(rng, 2048, 8192) if B < 4 else 2048, spec_lo=rows_lo,
                    spec_hi=max(rows_lo, _log_int(rng, 16, 2048)), lengths=lengths)
    f32 = rng.random() < 0.15
    H_q, H_kv = rng.choice([(32, 8), (8, 2), (28, 4), (16, 16), (64, 8), (24, 8)])
    B = _log_int(rng, 2, 12 if f32 else 192)
    prefix_lo = _log_int(rng, 32, 4096)
    return dict(kind="shared", dtype="f32" if f32 else "bf16", B=B, H_q=H_q, H_kv=H_kv, D=rng.choice([64, 128, 128]), P=rng.choice([16, 16, 64, rng.randint(1, 40)]),
                layout=rng.choice(["head", "token"]), groups=rng.randint(1, min(B, 6)), prefix_lo=prefix_lo,
                prefix_hi=max(prefix_lo, _log_int(rng, 256, 16384)), ctx_lo=rng.randint(0, 64), ctx_hi=_log_int(rng, 64, 1024), **spec)


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        case = _drawn(rng)
        if _cost(case) <= most:
            return case


# ---------------------------------------------------------------------------------------------------------------
# lengths, offsets and page tables: a function of the case alone, so that its work is known without its data
# ---------------------------------------------------------------------------------------------------------------
def _lengths(case):
    """(tokens in front of the call's rows, rows) of every request, and the groups' prefixes and bounds."""
    rng = np.random.Generator(np.random.PCG64(case["lengths"]))
    B = case["B"]
    rows = rng.integers(case["spec_lo"], case["spec_hi"] + 1, size=B) + 1
    ctx = rng.integers(case["ctx_lo"], case["ctx_hi"] + 1, size=B)
    if case["kind"] != "shared":
        return ctx, rows, None, None
    prefix = rng.integers(case["prefix_lo"], case["prefix_hi"] + 1, size=case["groups"])
    cuts = np.sort(rng.choice(np.arange(1, B), size=case["groups"] - 1, replace=False)) if case["groups"] > 1 else []
    bounds = np.concatenate([[0], cuts, [B]]).astype(np.int64)
    return ctx + np.repeat(prefix, np.diff(bounds)), rows, prefix, bounds


def _offsets(lens):
    cu = np.zeros(len(lens) + 1, np.int32)
    np.cumsum(lens, out=cu[1:])
    return cu


def _elem(case):
    return 2 if case["dtype"] == "bf16" else 4


def work(case):
    ctx, rows, prefix, bounds = _lengths(case)
    e, N, L = _elem(case), int(rows.sum()), ctx + rows
    seen = float((rows * ctx + rows * (rows + 1) / 2).sum())  # (row, key) pairs that are not masked
    if case["kind"] == "append":
        return dict(bytes=2 * N * (case["D_latent"] + case["D_rope"]) * e, flops=0)
    if case["kind"] == "gather":
        return dict(bytes=2 * int(L.sum()) * (case["D_latent"] + case["D_rope"]) * e + 4 * int((-(-L // case["P"])).sum()), flops=0)
    if case["kind"] == "latent":
        D_k, D_v, H = case["D_latent"] + case["D_rope"], case["D_latent"], case["H"]
        return dict(bytes=int(L.sum()) * D_k * e + N * H * ((D_k + D_v) * e + 4) + 4 * int((-(-L // case["P"])).sum()),
                    flops=2 * seen * H * (D_k + D_v))
    if case["kind"] == "expanded":
        D_k, D_v, H = case["D_nope"] + case["D_rope"], case["D_v"], case["H"]
        return dict(bytes=int(L.sum()) * (H * (case["D_nope"] + D_v) + case["D_rope"]) * e + N * H * ((D_k + D_v) * e + 4),
                    flops=2 * seen * H * (D_k + D_v))
    H_q, H_kv, D = case["H_q"], case["H_kv"], case["D"]
    tokens = int(prefix.sum() + (L - np.repeat(prefix, np.diff(bounds))).sum())
    return dict(bytes=2 * tokens * H_kv * D * e + N * H_q * (2 * D * e + 4) + 4 * (tokens // case["P"]), flops=4 * seen * H_q * D)


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


def _tables(case, seed):
    """Block tables over a permuted pool; the requests of a group hold the pages of its prefix in common."""
    ctx, rows, prefix, bounds = _lengths(case)
    rng = np.random.Generator(np.random.PCG64(seed))
    P, L = case["P"], ctx + rows
    pages = -(-L // P)
    whole = np.zeros_like(pages) if prefix is None else np.repeat(prefix // P, np.diff(bounds))
    n_pages = int((pages - whole).sum()) + (0 if prefix is None else int((prefix // P).sum())) + 3
    perm = rng.permutation(n_pages).astype(np.int32)
    bt = np.full((case["B"], int(pages.max())), -1, np.int32)
    at = 0
    for g in range(0 if prefix is None else len(prefix)):
        n = int(prefix[g] // P)
        bt[bounds[g]:bounds[g + 1], :n] = perm[at:at + n]
        at += n
    for i in range(case["B"]):
        n = int(pages[i] - whole[i])
        bt[i, whole[i]:pages[i]] = perm[at:at + n]
        at += n
    return bt, n_pages


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    ctx, rows, prefix, bounds = _lengths(case)
    N, B, dtype, kind = int(rows.sum()), case["B"], DTYPES[case["dtype"]], case["kind"]
    s = dict(case=case, N=N, T=int((ctx + rows).sum()), q_max=int(rows.max()), k_max=int((ctx + rows).max()), ctx=_dev(ctx.astype(np.int32)), cu_q=_dev(_offsets(rows)))
    if kind == "expanded":
        H, T = case["H"], s["T"]
        s.update(cu_k=_dev(_offsets(ctx + rows)), q=_normal(gen, (N, H, case["D_nope"] + case["D_rope"]), dtype),
                 kv=_normal(gen, (T, H, case["D_nope"] + case["D_v"]), dtype), k_rope=_normal(gen, (T, case["D_rope"]), dtype),
                 scale=(case["D_nope"] + case["D_rope"]) ** -0.5)
        return s
    bt, n_pages = _tables(case, seed)
    s.update(bt=_dev(bt), n_pages=n_pages)
    if kind == "shared":
        H_q, H_kv, D, P = case["H_q"], case["H_kv"], case["D"], case["P"]
        shape = (n_pages, H_kv, P, D) if case["layout"] == "head" else (n_pages, P, H_kv, D)
        group_rows = np.add.reduceat(rows, bounds[:-1])
        s.update(k=_normal(gen, shape, dtype), v=_normal(gen, shape, dtype), q=_normal(gen, (N, H_q, D), dtype), scale=D ** -0.5,
                 cu_groups=_dev(bounds.astype(np.int32)), prefix=_dev(prefix.astype(np.int32)), r_max=int(group_rows.max()),
                 p_max=int(prefix.max()), o_max=int((ctx + rows - np.repeat(prefix, np.diff(bounds))).max()))
        return s
    D_k = case["D_latent"] + case["D_rope"]
    s["cache"] = _normal(gen, (n_pages, case["P"], D_k), dtype)
    if kind == "append":
        s.update(latent=_normal(gen, (N, case["D_latent"]), dtype), rope=_normal(gen, (N, case["D_rope"]), dtype))
    elif kind == "gather":
        s.update(cu_k=_dev(_offsets(ctx + rows)))
    else:  # queries that have been taken into the latent's space
        s.update(q=_normal(gen, (N, case["H"], D_k), dtype), scale=D_k ** -0.5)
    return s


# ---------------------------------------------------------------------------------------------------------------
# one pass, in plain form
# ---------------------------------------------------------------------------------------------------------------
def _owners(cu, n, B):
    """Request of every row, and its place in it."""
    i = torch.repeat_interleave(torch.arange(B, device="cuda"), cu.diff().long(), output_size=n)
    return i, torch.arange(n, device="cuda") - cu[i]


def _slots(s, i, pos):
    """Slot in the pool of positions `pos` of requests `i`."""
    P = s["case"]["P"]
    return s["bt"][i, pos // P].long() * P + pos % P


def _padded(x, cu, most):
    """[B, most, ...] in 32 bits out of ragged rows (places behind a request's last row hold some other row)."""
    at = (cu[:-1, None] + torch.arange(most, device="cuda")).clamp(max=x.shape[0] - 1)
    return x[at].float()


def _joined(*parts):
    """Softmax over the keys of several (scores, values): weighted values and log of the sum of exponentials."""
    m = torch.stack([p[0].amax(-1) for p in parts]).amax(0)
    e = [torch.exp(p[0] - m[..., None]) for p in parts]
    total = sum(x.sum(-1) for x in e)
    return sum(torch.matmul(x, p[1]) for x, p in zip(e, parts)) / total[..., None], m + torch.log(total)


def _plain_append(s):
    i, j = _owners(s["cu_q"], s["N"], s["case"]["B"])
    s["cache"].view(-1, s["cache"].shape[2])[_slots(s, i, s["ctx"][i] + j)] = torch.cat([s["latent"], s["rope"]], 1)
    return s["cache"]


def _plain_gather(s):
    i, j = _owners(s["cu_k"], s["T"], s["case"]["B"])
    x = s["cache"].view(-1, s["cache"].shape[2])[_slots(s, i, j)]
    D = s["case"]["D_latent"]
    return x[:, :D].contiguous(), x[:, D:].contiguous()


def _plain_latent(s):
    case = s["case"]
    B, H, D_v, q_max, k_max = case["B"], case["H"], case["D_latent"], s["q_max"], s["k_max"]
    pos = torch.arange(k_max, device="cuda")
    slots = _slots(s, torch.arange(B, device="cuda")[:, None], pos[None, :]).clamp(min=0)
    keys = s["cache"].view(-1, s["cache"].shape[2])[slots].float()
    q = _padded(s["q"], s["cu_q"], q_max).reshape(B, q_max * H, -1)
    z = torch.matmul(q, keys.transpose(1, 2).contiguous()).mul_(s["scale"]).view(B, q_max, H, k_max)
    last = s["ctx"][:, None] + torch.arange(q_max, device="cuda")
    z.masked_fill_((pos > last[..., None])[:, :, None, :], -INF)
    o, lse = _joined((z.view(B, q_max * H, k_max), keys[..., :D_v].contiguous()))
    i, j = _owners(s["cu_q"], s["N"], B)
    return o.view(B, q_max, H, D_v)[i, j].to(s["q"].dtype), lse.view(B, q_max, H)[i, j]


def _plain_expanded(s):
    case = s["case"]
    B, H, D, q_max, k_max = case["B"], case["H"], case["D_nope"], s["q_max"], s["k_max"]
    q = _padded(s["q"], s["cu_q"], q_max).transpose(1, 2).contiguous()
    kv = _padded(s["kv"], s["cu_k"], k_max)
    rope = _padded(s["k_rope"], s["cu_k"], k_max)
    z = torch.matmul(q[..., :D].contiguous(), kv[..., :D].permute(0, 2, 3, 1).contiguous())
    z += torch.matmul(q[..., D:].reshape(B, H * q_max, -1), rope.transpose(1, 2).contiguous()).view(B, H, q_max, k_max)
    z *= s["scale"]
    pos, last = torch.arange(k_max, device="cuda"), s["ctx"][:, None] + torch.arange(q_max, device="cuda")
    z.masked_fill_((pos > last[..., None])[:, None], -INF)
    o, lse = _joined((z, kv[..., D:].transpose(1, 2).contiguous()))
    i, j = _owners(s["cu_q"], s["N"], B)
    return o[i, :, j].to(s["q"].dtype), lse[i, :, j]


def _heads_first(x, layout):
    """[pages, P, H, D] of a cache, as slots of all heads."""
    x = x.transpose(1, 2) if layout == "head" else x
    return x.reshape(-1, x.shape[2], x.shape[3])


def _plain_shared(s):
    case = s["case"]
    B, H_q, H_kv, D, q_max = case["B"], case["H_q"], case["H_kv"], case["D"], s["q_max"]
    G, n_g, first = H_q // H_kv, case["groups"], s["cu_groups"][:-1].long()
    group = torch.repeat_interleave(torch.arange(n_g, device="cuda"), s["cu_groups"].diff().long(), output_size=B)
    i, j = _owners(s["cu_q"], s["N"], B)
    k, v = (_heads_first(s[x], case["layout"]) for x in "kv")
    # the prefix: all rows of a group in one product per KV head
    pos = torch.arange(s["p_max"], device="cuda")
    at = _slots(s, first[:, None], pos[None, :].expand(n_g, -1)).clamp(min=0)
    cu_r = s["cu_q"][s["cu_groups"].long()]
    q1 = _padded(s["q"], cu_r, s["r_max"]).view(n_g, s["r_max"], H_kv, G, D).permute(0, 2, 1, 3, 4).reshape(n_g, H_kv, s["r_max"] * G, D)
    z1 = torch.matmul(q1, k[at].float().permute(0, 2, 3, 1).contiguous()) * s["scale"]
    z1.masked_fill_((pos >= s["prefix"][:, None])[:, None, None, :], -INF)
    v1 = v[at].float().transpose(1, 2).contiguous()
    m1 = z1.amax(-1)
    e1 = torch.exp_(z1 - m1[..., None])
    place = torch.arange(s["N"], device="cuda") - cu_r[group[i]]
    rows = lambda x: x.view(n_g, H_kv, s["r_max"], G, -1)[group[i], :, place]  # noqa: E731  [N, H_kv, G, .]
    o1, l1, m1 = rows(torch.matmul(e1, v1)), rows(e1.sum(-1)), rows(m1)
    # what is a request's own
    base = s["prefix"][group]
    own_pos = base[:, None] + torch.arange(s["o_max"], device="cuda")
    at = _slots(s, torch.arange(B, device="cuda")[:, None], own_pos.clamp(max=s["bt"].shape[1] * case["P"] - 1)).clamp(min=0)
    q2 = _padded(s["q"], s["cu_q"], q_max).view(B, q_max, H_kv, G, D).permute(0, 2, 1, 3, 4).reshape(B, H_kv, q_max * G, D)
    z2 = (torch.matmul(q2, k[at].float().permute(0, 2, 3, 1).contiguous()) * s["scale"]).view(B, H_kv, q_max, G, -1)
    last = s["ctx"][:, None] + torch.arange(q_max, device="cuda")
    z2 = z2.masked_fill((own_pos[:, None, :] > last[..., None])[:, None, :, None, :], -INF).view(B, H_kv, q_max * G, -1)
    m2 = z2.amax(-1)
    e2 = torch.exp(z2 - m2[..., None])
    rows = lambda x: x.view(B, H_kv, q_max, G, -1)[i, :, j]  # noqa: E731
    o2, l2, m2 = rows(torch.matmul(e2, v[at].float().transpose(1, 2).contiguous())), rows(e2.sum(-1)), rows(m2)
    m = torch.maximum(m1, m2)
    w1, w2 = torch.exp(m1 - m), torch.exp(m2 - m)
    total = w1 * l1 + w2 * l2
    return ((w1 * o1 + w2 * o2) / total).view(-1, H_q, D).to(s["q"].dtype), (m + torch.log(total)).view(-1, H_q)


PLAIN = dict(append=_plain_append, gather=_plain_gather, latent=_plain_latent, expanded=_plain_expanded, shared=_plain_shared)


# ---------------------------------------------------------------------------------------------------------------
# one pass, through the package
# ---------------------------------------------------------------------------------------------------------------
def _own(s):
    import paper_2604_20503_amd as fsr

    case = s["case"]
    kind = case["kind"]
    if kind == "append":
        fsr.latent_append(s["latent"], s["rope"], s["cache"], s["bt"], s["ctx"], s["cu_q"])
        return s["cache"]
    if kind == "gather":
        return fsr.latent_gather(s["cache"], s["bt"], s["cu_k"], T_cap=s["T"], D_latent=case["D_latent"])
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
    if kind == "latent":
        return fsr.latent_attention(s["q"], s["cache"], s["bt"], s["ctx"], s["cu_q"], scale=s["scale"], D_latent=case["D_latent"],
                                    lse=lse, max_q_len=s["q_max"])
    if kind == "expanded":
        return fsr.latent_attention_expanded(s["q"], s["kv"], s["k_rope"], s["cu_q"], s["cu_k"], scale=s["scale"], lse=lse, max_q_len=s["q_max"])
    layout = fsr.binding.KV_HEAD_MAJOR if case["layout"] == "head" else fsr.binding.KV_TOKEN_MAJOR
    return fsr.verify_attention_shared(s["q"], s["k"], s["v"], s["bt"], s["ctx"], s["cu_q"], s["cu_groups"], s["prefix"],
                                       scale=s["scale"], lse=lse, max_q_len=s["q_max"], kv_layout=layout)


def run(state):
    return _own(state) if own else PLAIN[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------------------------------------------
# the definition in 64 bits, request by request
# ---------------------------------------------------------------------------------------------------------------
def _attend(q, k, v, scale, ctx):
    """q [n, heads, D], k / v [L, heads, .] in 64 bits; row j sees the keys up to position ctx + j."""
    z = torch.matmul(q.transpose(0, 1), k.permute(1, 2, 0)) * scale
    z.masked_fill_(torch.arange(k.shape[0], device="cuda") > (ctx + torch.arange(q.shape[0], device="cuda"))[:, None], -INF)
    return torch.matmul(torch.softmax(z, -1), v.transpose(0, 1)).transpose(0, 1), torch.logsumexp(z, -1).transpose(0, 1)


def exact(case, seed):
    if work(case)["flops"] > 2e12:
        return None
    s = prepare(case, seed)
    ctx, rows, prefix, bounds = _lengths(case)
    cu, kind, H = _offsets(rows), case["kind"], case.get("H", 0)
    if kind == "append":
        cache = s["cache"].double()
        for r in range(s["N"]):
            i = int(np.searchsorted(cu, r, side="right")) - 1
            t = int(ctx[i]) + r - int(cu[i])
            page = int(s["bt"][i, t // case["P"]])
            cache[page, t % case["P"], :case["D_latent"]] = s["latent"][r].double()
            cache[page, t % case["P"], case["D_latent"]:] = s["rope"][r].double()
        return cache
    outs, lses = [], []
    for i in range(case["B"]):
        n, L = int(rows[i]), int(ctx[i] + rows[i])
        if kind == "expanded":
            a = int((ctx + rows)[:i].sum())
            kv, rope = s["kv"][a:a + L].double(), s["k_rope"][a:a + L].double()
            k = torch.cat([kv[..., :case["D_nope"]], rope[:, None].expand(-1, H, -1)], 2)
            v = kv[..., case["D_nope"]:]
        else:
            pages = s["bt"][i, :-(-L // case["P"])].long()
            if kind == "shared":
                k, v = (s[x][pages].double() for x in "kv")
                if case["layout"] == "head":
                    k, v = k.transpose(1, 2), v.transpose(1, 2)
                k, v = (x.reshape(-1, case["H_kv"], case["D"])[:L] for x in (k, v))
                # the prefix is the one in the pages of the group's first request
                g = int(np.searchsorted(bounds, i, side="right")) - 1
                p = int(prefix[g])
                head = s["bt"][int(bounds[g]), :-(-p // case["P"])].long()
                kp, vp = (s[x][head].double() for x in "kv")
                if case["layout"] == "head":
                    kp, vp = kp.transpose(1, 2), vp.transpose(1, 2)
                k = torch.cat([kp.reshape(-1, case["H_kv"], case["D"])[:p], k[p:]])
                v = torch.cat([vp.reshape(-1, case["H_kv"], case["D"])[:p], v[p:]])
                G = case["H_q"] // case["H_kv"]
                k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
            else:
                x = s["cache"][pages].double().reshape(-1, s["cache"].shape[2])[:L]
                if kind == "gather":
                    outs.append(x[:, :case["D_latent"]])
                    lses.append(x[:, case["D_latent"]:])
                    continue
                q = s["q"][int(cu[i]):int(cu[i + 1])].double().reshape(1, n * H, -1)
                z = torch.matmul(q, x.t().contiguous()).view(n, H, L) * s["scale"]
                z.masked_fill_((torch.arange(L, device="cuda") > (int(ctx[i]) + torch.arange(n, device="cuda"))[:, None])[:, None], -INF)
                outs.append(torch.matmul(torch.softmax(z, -1).view(n * H, L), x[:, :case["D_latent"]].contiguous()).view(n, H, -1))
                lses.append(torch.logsumexp(z, -1))
                continue
        o, lse = _attend(s["q"][int(cu[i]):int(cu[i + 1])].double(), k.contiguous(), v.contiguous(), s["scale"], int(ctx[i]))
        outs.append(o)
        lses.append(lse)
    return torch.cat(outs), torch.cat(lses)
