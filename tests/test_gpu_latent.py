"""fsr_latent_append, fsr_latent_gather and fsr_latent_attention against the definition in 64 bits."""
import pytest
import torch

from gpu_utils import announce
from plain_attention import attend, check, offsets, pages, slots

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def fsr():
    import paper_2604_20503_amd as f
    f.load_library()
    return f


def normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen).to(dtype)


class Batch:
    def __init__(self, seed, ctx, rows, H, D_latent, D_rope, P, dtype, extra_rows=0):
        gen = torch.Generator().manual_seed(seed)
        self.ctx, self.rows, self.H, self.Dl, self.P, self.dtype = list(ctx), list(rows), H, D_latent, P, dtype
        D = D_latent + D_rope
        self.bt, self.n_pages = pages([c + n for c, n in zip(ctx, rows)], P, gen)
        self.cache = normal(gen, (self.n_pages, P, D), dtype)
        self.cu = offsets(rows)
        self.N = int(self.cu[-1])
        self.q = normal(gen, (self.N + extra_rows, H, D), dtype)
        self.scale = D ** -0.5

    def dev(self):
        return [x.cuda() for x in (self.q, self.cache, self.bt, torch.tensor(self.ctx, dtype=torch.int32), self.cu)]

    def keys(self, i):
        return self.cache.view(-1, self.cache.shape[2])[slots(self.bt[i], self.ctx[i] + self.rows[i], self.P)]

    def reference(self):
        parts = []
        for i, n in enumerate(self.rows):
            x = self.keys(i)
            q = self.q[int(self.cu[i]):int(self.cu[i]) + n].flatten(0, 1)
            last = (self.ctx[i] + torch.arange(n)).repeat_interleave(self.H)
            parts.append(attend(q, x, x[:, :self.Dl], self.scale, last))
        o, lse, A, e = (torch.cat(p) for p in zip(*parts))
        return o.view(self.N, self.H, -1), lse.view(self.N, self.H), A.view(self.N, self.H, -1), e.view(self.N, self.H)


def run(fsr, b, out_dtype, **kw):
    q, cache, bt, ctx, cu = b.dev()
    out = torch.full((q.shape[0], b.H, b.Dl), 7.0, dtype=out_dtype, device="cuda")
    lse = torch.full((q.shape[0], b.H), 7.0, dtype=F32, device="cuda")
    fsr.latent_attention(q, cache, bt, ctx, cu, scale=b.scale, D_latent=b.Dl, out=out, lse=lse, **kw)
    torch.cuda.synchronize()
    assert (out[b.N:] == 7).all() and (lse[b.N:] == 7).all()  # rows behind the last request stay
    return out[:b.N], lse[:b.N]


def compare(name, b, got):
    o, lse, A, e = b.reference()
    flat = lambda x: x.reshape(-1, x.shape[-1]) if x.dim() == 3 else x.reshape(-1)  # noqa: E731
    check(name, flat(got[0]), flat(got[1]), flat(o), flat(lse), flat(A), flat(e), b.dtype)


CASES = [
    ("one token, empty context", [0], [1], 16, 512, 64, 16),
    ("one token", [777], [1], 16, 512, 64, 16),
    ("lengths around pages and tiles", [0, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129], [1, 2, 1, 3, 1, 1, 2, 1, 1, 1, 1, 1, 1], 8, 512, 64, 16),
    ("requests without rows", [5, 70, 200, 9, 33], [0, 2, 0, 3, 0], 16, 512, 64, 16),
    ("all heads, several drafts", [130, 300], [4, 2], 128, 512, 64, 64),
    ("odd heads and pages", [40, 250, 3], [3, 7, 5], 5, 512, 64, 7),
    ("one head, pages of one token", [50, 90], [2, 33], 1, 512, 64, 1),
    ("more rows than a tile, ragged", [300, 20], [19, 30], 12, 512, 64, 16),
    ("small latent", [100, 513], [9, 1], 16, 256, 32, 16),
    ("small latent, wide position", [64, 1, 200], [2, 1, 6], 24, 256, 64, 32),
    ("narrow position", [97, 161], [5, 2], 16, 512, 32, 48),
    ("a long context", [9000], [2], 16, 512, 64, 16),
    ("a long one among short ones", [10, 6000, 40, 8], [1, 3, 2, 1], 16, 512, 64, 16),
]


@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_attention(fsr, case, dtype, out_dtype):
    announce(f"latent attention: {case} {dtype} {out_dtype}")
    b = Batch(1, *case[1:], dtype, extra_rows=3)
    compare(case[0], b, run(fsr, b, out_dtype, max_q_len=max(b.rows)))


@pytest.mark.parametrize("workgroups", [1, 2, 7, 100])
def test_attention_on_part_of_the_device(fsr, workgroups):
    announce(f"latent attention, {workgroups} workgroups")
    b = Batch(2, [500, 20, 1100, 64], [3, 1, 2, 12], 16, 512, 64, 16, BF)
    compare("workgroups", b, run(fsr, b, BF, max_workgroups=workgroups))


@pytest.mark.parametrize("seed", range(6))
def test_attention_random_shapes(fsr, seed):
    gen = torch.Generator().manual_seed(100 + seed)
    draw = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=gen))  # noqa: E731
    B = draw(1, 40)
    ctx, rows = [draw(0, 400) for _ in range(B)], [draw(0, 6) for _ in range(B)]
    shape = (draw(1, 40), [256, 512][draw(0, 1)], [32, 64][draw(0, 1)], draw(1, 80))
    announce(f"latent attention, random: {seed} {ctx} {rows} {shape}")
    b = Batch(seed, ctx, rows, *shape, [BF, F32][draw(0, 1)])
    compare(f"random {seed}", b, run(fsr, b, b.dtype))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_values_that_are_not_finite_stay_where_they_are_seen(fsr, dtype):
    """Slots behind a request's last token hold NaN; the last row's own token holds infinities and NaN: the rows before it do
    not see them, the last row does."""
    announce(f"latent attention, not finite {dtype}")
    b = Batch(3, [70, 126, 5], [3, 2, 4], 16, 512, 64, 16, dtype)
    want = b.reference()
    flat = b.cache.view(-1, b.cache.shape[2])
    used = torch.zeros(flat.shape[0], dtype=torch.bool)
    for i in range(3):
        s = slots(b.bt[i], b.ctx[i] + b.rows[i], b.P)
        used[s] = True
        flat[s[-1], 3:6] = torch.tensor([float("inf"), float("-inf"), float("nan")]).to(dtype)
        flat[s[-1], 40] = float("inf")
    flat[~used] = float("nan")
    out, lse = run(fsr, b, dtype)
    last = torch.zeros(b.N, dtype=torch.bool)
    last[b.cu[1:].long() - 1] = True
    pick = lambda x: x[~last].reshape(-1, x.shape[-1]) if x.dim() == 3 else x[~last].reshape(-1)  # noqa: E731
    check("rows before", pick(out), pick(lse), *(pick(x) for x in want), dtype)
    assert torch.isnan(out[last.cuda()]).all()  # their scores hold inf * q of both signs, or NaN


@pytest.mark.parametrize("dtype", [BF, F32])
def test_infinite_value_reaches_the_rows_that_see_it(fsr, dtype):
    """A value of inf whose key part is finite: only its column turns infinite, and only in rows that see it."""
    announce(f"latent attention, infinite value {dtype}")
    b = Batch(4, [20], [3], 4, 512, 64, 16, dtype)
    b.q[:, :, 9] = 0.0  # (0 * inf in the score would be NaN: the column is left out of the scores by being tiny instead)
    s = slots(b.bt[0], 23, 16)
    b.cache.view(-1, 576)[s[-1], 9] = 3.0e38
    b.q[:, :, 9] = 0.0
    out, _ = run(fsr, b, dtype)
    assert torch.isfinite(out[:2].float()).all() and out[2, :, 9].float().abs().min() > 1e30
    assert torch.isfinite(out[2, :, :9].float()).all()


def test_table_entries_outside_the_pool_are_clamped(fsr):
    announce("latent attention, bad pages")
    b = Batch(5, [40, 100], [2, 1], 16, 512, 64, 16, BF)
    bad = b.bt.clone()
    b.bt[0, 1], bad[0, 1] = b.n_pages - 1, b.n_pages + 1000
    b.bt[1, 2], bad[1, 2] = 0, -7
    o, lse, A, e = b.reference()
    b.bt = bad
    got = run(fsr, b, BF)
    check("clamped", got[0].reshape(-1, 512), got[1].reshape(-1), o.reshape(-1, 512), lse.reshape(-1), A.reshape(-1, 512), e.reshape(-1), BF)


def test_replays_and_streams(fsr):
    """One captured graph of two calls on one workspace, replayed between eager calls, gives the eager result each time; so does
    a call on another stream."""
    announce("latent attention, graph and stream")
    b = Batch(6, [700, 33, 250], [3, 1, 5], 16, 512, 64, 16, BF)
    q, cache, bt, ctx, cu = b.dev()
    need = fsr.latent_workspace_bytes(N_cap=b.N, H=16, D_latent=512, D_rope=64, dtype=BF, out_dtype=BF)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    want, want_lse = run(fsr, b, BF)
    outs = [torch.zeros_like(want) for _ in range(2)]
    lses = [torch.zeros_like(want_lse) for _ in range(2)]
    call = lambda k, w=ws: fsr.latent_attention(q, cache, bt, ctx, cu, scale=b.scale, D_latent=512, out=outs[k], lse=lses[k], workspace=w)  # noqa: E731
    call(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(0)
        call(1)
    for _ in range(4):
        for x in outs + lses:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, want) for x in outs) and all(torch.equal(x, want_lse) for x in lses)
        run(fsr, b, BF)
    side = torch.cuda.Stream()
    outs[0].zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(0, torch.empty_like(ws))
    side.synchronize()
    assert torch.equal(outs[0], want)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("ctx,rows,Dl,Dr,P", [([0], [1], 512, 64, 16), ([257], [4], 512, 64, 16), ([3, 0, 31, 500, 16], [5, 0, 2, 70, 1], 512, 64, 16),
                                              ([7, 90], [40, 3], 256, 32, 5), ([0] * 40, [9] * 40, 24, 8, 64)])
def test_append_and_gather_move_every_bit(fsr, ctx, rows, Dl, Dr, P, dtype):
    announce(f"latent append and gather {ctx} {rows} {Dl} {Dr} {P} {dtype}")
    gen = torch.Generator().manual_seed(9)
    lens = [c + n for c, n in zip(ctx, rows)]
    bt, n_pages = pages(lens, P, gen)
    bits, kind = (torch.int16, 1 << 15) if dtype == BF else (torch.int32, 1 << 31)
    some = lambda *shape: torch.randint(-kind, kind, shape, generator=gen, dtype=torch.int64).to(bits).view(dtype)  # noqa: E731
    cache, N = some(n_pages, P, Dl + Dr), sum(rows)
    latent, rope = some(N + 2, Dl), some(N + 2, Dr)  # (two rows behind the last request are not read)
    got = cache.cuda()
    bt_d, cu = bt.cuda(), offsets(rows).cuda()
    fsr.latent_append(latent.cuda(), rope.cuda(), got, bt_d, torch.tensor(ctx, dtype=torch.int32).cuda(), cu)
    want, flat = cache.clone(), None
    flat = want.view(bits).view(-1, Dl + Dr)
    new = torch.cat([latent.view(bits), rope.view(bits)], 1)
    at = 0
    for i, n in enumerate(rows):
        flat[slots(bt[i], lens[i], P)[ctx[i]:]] = new[at:at + n]
        at += n
    assert torch.equal(got.cpu().view(bits), want.view(bits))
    T = sum(lens)
    l_out, r_out = torch.zeros(T + 3, Dl, dtype=dtype, device="cuda"), torch.zeros(T + 3, Dr, dtype=dtype, device="cuda")
    fsr.latent_gather(got, bt_d, offsets(lens).cuda(), T_cap=T + 3, D_latent=Dl, latent=l_out, rope=r_out)
    back = torch.cat([flat[slots(bt[i], lens[i], P)] for i in range(len(lens))])
    assert torch.equal(l_out.cpu().view(bits)[:T], back[:, :Dl]) and torch.equal(r_out.cpu().view(bits)[:T], back[:, Dl:])
    assert not l_out.cpu().view(bits)[T:].any() and not r_out.cpu().view(bits)[T:].any()


def test_append_skips_and_gather_clamps(fsr):
    announce("latent append and gather, bad tables")
    cache = torch.zeros(4, 8, 24, device="cuda")
    bt = torch.tensor([[0, 9], [-1, 2], [1, 3]], dtype=torch.int32, device="cuda")
    rows = torch.ones(15, 16, device="cuda")
    rope = torch.ones(15, 8, device="cuda")
    # request 0: positions 6 .. 10 (page 9 is no page), request 1: 5 .. 9 (page -1), request 2: 14 .. 18 (no page behind 15)
    fsr.latent_append(rows, rope, cache, bt, torch.tensor([6, 5, 14], dtype=torch.int32, device="cuda"), offsets([5, 5, 5]).cuda())
    held = cache.sum(2).cpu() / 24
    want = torch.zeros(4, 8)
    want[0, 6:8] = 1
    want[2, 0:2] = 1
    want[3, 6:8] = 1
    assert torch.equal(held, want)
    cache[3] = 5.0
    cache[0] = 2.0
    latent, rope = fsr.latent_gather(cache, bt, offsets([16, 1, 18]).cuda(), T_cap=35, D_latent=16)
    got = latent[:, 0].cpu()
    assert got[:8].eq(2).all() and got[8:16].eq(5).all() and got[16] == 2  # page 9 reads the pool's last page, -1 its first
    assert got[17 + 8:17 + 16].eq(5).all() and got[33:].eq(0).all() and rope[33:].eq(0).all()


def test_run_of_all_forms(fsr):
    """A step as a program makes it: rows are appended, few rows attend in the latent's space, the contexts come back, an up-projection
    makes keys and values, and the expanded form gives the same attention."""
    from plain_attention import U
    announce("latent caches: append, attention, gather, expanded")
    gen = torch.Generator().manual_seed(11)
    H, Dl, Dr, Dn, Dv, P = 4, 512, 64, 128, 128, 16
    ctx, rows = [100, 37, 0], [3, 20, 2]
    lens = [c + n for c, n in zip(ctx, rows)]
    bt, n_pages = pages(lens, P, gen)
    cache = torch.randn(n_pages, P, Dl + Dr, generator=gen).cuda()
    N, cu, cu_k = sum(rows), offsets(rows).cuda(), offsets(lens).cuda()
    c_new, r_new = torch.randn(N, Dl, generator=gen).cuda(), torch.randn(N, Dr, generator=gen).cuda()
    ctx_d, bt_d = torch.tensor(ctx, dtype=torch.int32).cuda(), bt.cuda()
    fsr.latent_append(c_new, r_new, cache, bt_d, ctx_d, cu)
    w_k, w_v = torch.randn(H, Dl, Dn, generator=gen).cuda() * Dl ** -0.5, torch.randn(H, Dl, Dv, generator=gen).cuda() * Dl ** -0.5
    q = torch.randn(N, H, Dn + Dr, generator=gen).cuda()
    scale = (Dn + Dr) ** -0.5
    absorbed = torch.cat([torch.einsum("nhd,hcd->nhc", q[..., :Dn], w_k), q[..., Dn:]], 2).contiguous()
    o, lse = fsr.latent_attention(absorbed, cache, bt_d, ctx_d, cu, scale=scale, D_latent=Dl, lse=torch.empty(N, H, device="cuda"))
    o = torch.einsum("nhc,hcd->nhd", o, w_v)
    latent, rope = fsr.latent_gather(cache, bt_d, cu_k, T_cap=sum(lens), D_latent=Dl)
    kv = torch.cat([torch.einsum("tc,hcd->thd", latent, w_k), torch.einsum("tc,hcd->thd", latent, w_v)], 2).contiguous()
    e, e_lse = fsr.latent_attention_expanded(q, kv, rope, cu, cu_k, scale=scale, lse=torch.empty(N, H, device="cuda"))
    # products of 512 terms of size one in fp32, twice on each side: some 4 * 512 * U of the terms' sum of magnitudes (about 512 * 0.64)
    assert (o - e).abs().max() < 4 * 512 * U * 512 and (lse - e_lse).abs().max() < 4 * 512 * U * 512
