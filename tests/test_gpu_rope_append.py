"""fsr_kv_append_rope and fsr_kv_append_rope_kv8 against the definition in 64 bits."""
import pytest
import torch

from gpu_utils import announce
from plain_attention import offsets, pages, slots
from plain_tree import rotate, sees_of, tree, words_of

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def fsr():
    import paper_2604_20503_amd as f
    f.load_library()
    return f


class Rows:
    def __init__(self, seed, reqs, H_q, H_kv, D, R, P, dtype, kv8=False, token_major=False, spare=2):
        gen = torch.Generator().manual_seed(seed)
        self.reqs, self.H_q, self.H_kv, self.D, self.R, self.P, self.dtype, self.kv8, self.token_major = reqs, H_q, H_kv, D, R, P, dtype, kv8, token_major
        self.rows = [n for _, n in reqs]
        self.N, self.cu, self.spare = sum(self.rows), offsets(self.rows), spare
        self.bt, n_pages = pages([c + n for c, n in reqs], P, gen)
        normal = lambda *shape: torch.randn(shape, generator=gen).to(dtype)  # noqa: E731
        self.q, self.k, self.v = normal(self.N + spare, H_q, D), normal(self.N + spare, H_kv, D), normal(self.N + spare, H_kv, D)
        self.T = max([c + n for c, n in reqs] + [1]) + 1
        turn = torch.arange(self.T, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)
        self.table = torch.cat([turn.cos(), turn.sin()], 1).float()
        shape = (n_pages, P, H_kv, D) if token_major else (n_pages, H_kv, P, D)
        self.caches = [torch.randint(0, 120, shape, generator=gen, dtype=torch.uint8) if kv8 else normal(*shape) for _ in "kv"]
        self.scales = [0.005 + 0.02 * torch.rand(H_kv, generator=gen) for _ in "kv"] if kv8 else [None, None]
        self.parents = [tree(n, gen) for n in self.rows]
        self.owner = torch.repeat_interleave(torch.arange(len(reqs)), torch.tensor(self.rows, dtype=torch.int64))
        self.place = torch.arange(self.N) - self.cu[self.owner]
        self.ctx = torch.tensor([c for c, _ in reqs], dtype=torch.int64)

    def mask(self, words):
        rows = [words_of(sees_of(p), words) for p in self.parents if p]
        return torch.cat(rows + [torch.zeros(self.spare, words, dtype=torch.int64)])

    def depths(self):
        return torch.cat([sees_of(p).sum(1) - 1 for p in self.parents if p])

    def run(self, fsr, pairs=False, positions=None, words=None, in_place=False, **kw):
        lay = fsr.binding.KV_TOKEN_MAJOR if self.token_major else fsr.binding.KV_HEAD_MAJOR
        self.got = [x.cuda().clone() for x in self.caches]
        q = self.q.cuda()
        q_out = q if in_place else torch.full(q.shape, 7.0, dtype=self.dtype, device="cuda")
        args = dict(q=q, k_new=self.k.cuda(), v_new=self.v.cuda(), cos_sin=self.table.cuda(), k_cache=self.got[0], v_cache=self.got[1], block_tables=self.bt.cuda(),
                    ctx_lens=self.ctx.int().cuda(), cu_q=self.cu.cuda(), q_out=q_out, pairs=pairs, kv_layout=lay)
        if positions is not None:
            args["positions"] = torch.cat([positions, torch.zeros(self.spare)]).int().cuda()
        if words:
            args["tree_mask"] = self.mask(words).cuda()
        if self.kv8:
            args.update(k_scale=self.scales[0].cuda(), v_scale=self.scales[1].cuda())
        args.update(kw)
        out = fsr.kv_append_rope(**args)
        torch.cuda.synchronize()
        assert out is args["q_out"]
        want = self.q[self.N:].cuda() if in_place else torch.full_like(out[self.N:], 7.0)
        assert torch.equal(out[self.N:], want)
        return out[:self.N].cpu()

    def check(self, q_out, positions, pairs=False):
        t = self.table[positions.clamp(0, self.T - 1)]
        half = {BF: 2.0 ** -8, F32: 0.0}[self.dtype]
        y, err = rotate(self.q[:self.N], t, self.R, pairs)
        assert ((q_out.double() - y).abs() <= err + half * (y.abs() + err)).all()
        pos = self.ctx[self.owner] + self.place
        for name, x, cache, before, scale in zip("kv", (self.k, self.v), self.got, self.caches, self.scales):
            cache, before = ((c.cpu() if self.token_major else c.cpu().transpose(1, 2)) for c in (cache, before))
            flat, old = cache.reshape(-1, self.H_kv, self.D), before.reshape(-1, self.H_kv, self.D)
            at = torch.tensor([int(slots(self.bt[i], int(p) + 1, self.P)[-1]) for i, p in zip(self.owner, pos)], dtype=torch.int64)
            rest = torch.ones(flat.shape[0], dtype=torch.bool)
            rest[at] = False
            assert torch.equal(flat[rest], old[rest]), f"{name}: other slots changed"
            x = x[:self.N]
            if not self.kv8 and name == "v":
                assert torch.equal(flat[at], x)
                continue
            y, err = rotate(x, t, self.R, pairs) if name == "k" else (x.double(), torch.zeros(x.shape, dtype=torch.float64))
            if not self.kv8:
                assert ((flat[at].double() - y).abs() <= err + half * (y.abs() + err)).all()
                assert torch.equal(flat[at][..., self.R:], x[..., self.R:])  # what is not rotated keeps its bits
                continue
            # half a step of E4M3 (2^-4 relative, 2^-10 below the normal numbers) on top of the quotient's own rounding
            y, err = y / scale[:, None].double(), err / scale[:, None].double()
            err = err + 2.0 ** -24 * (y.abs() + err)
            code = flat[at].view(torch.float8_e4m3fn).double()
            far = y.abs() - err > 448
            assert (code[far].abs() == 448).all()
            assert (((code - y).abs() <= err + torch.maximum(2.0 ** -4 * (y.abs() + err), torch.tensor(2.0 ** -10, dtype=torch.float64))) | far).all()


CASES = [
    ("one row", [(0, 1)], 8, 2, 128, 128, 16),
    ("chains", [(40, 7), (100, 12), (3, 1), (129, 5)], 8, 2, 128, 128, 16),
    ("requests without rows", [(40, 0), (20, 9), (0, 0), (90, 4), (5, 0)], 8, 2, 128, 128, 16),
    ("part of a head", [(33, 17), (64, 3)], 6, 3, 128, 64, 16),
    ("small part of a wide head", [(9, 5)], 2, 1, 256, 32, 7),
    ("heads of 64, odd pages", [(77, 13), (5, 30)], 28, 4, 64, 64, 5),
    ("heads of 80", [(10, 6), (2, 2)], 5, 5, 80, 16, 16),
    ("wide", [(30, 40)], 64, 8, 128, 128, 64),
    ("many requests", [(11 * k % 60, 1 + 5 * k % 7) for k in range(150)], 4, 1, 64, 64, 16),
    ("more requests than a wave squared", [(k % 5, k % 2) for k in range(4200)], 1, 1, 64, 16, 4),
]


@pytest.mark.parametrize("token_major", [False, True])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dtype,kv8", [(BF, False), (F32, False), (BF, True)])
@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_rope(fsr, case, dtype, kv8, pairs, token_major):
    announce(f"append with rotation: {case[0]} {dtype} kv8={kv8} pairs={pairs} token_major={token_major}")
    r = Rows(1, *case[1:], dtype, kv8, token_major)
    pos = r.ctx[r.owner] + r.place
    r.check(r.run(fsr, pairs=pairs), pos, pairs)


@pytest.mark.parametrize("dtype,kv8", [(BF, False), (F32, False), (BF, True)])
def test_positions_of_trees(fsr, dtype, kv8):
    announce(f"append with rotation, trees {dtype} kv8={kv8}")
    r = Rows(2, [(30, 20), (0, 100), (64, 1), (7, 0), (9, 64)], 8, 2, 128, 128, 16, dtype, kv8)
    pos = r.ctx[r.owner] + r.depths()
    r.check(r.run(fsr, words=2), pos)
    r.check(r.run(fsr, positions=pos), pos)
    some = torch.randint(0, r.T, (r.N,), generator=torch.Generator().manual_seed(1))
    r.check(r.run(fsr, positions=some, pairs=True), some, True)
    r.check(r.run(fsr, positions=torch.full((r.N,), 1 << 30)), torch.full((r.N,), r.T - 1))  # clamped to the table
    r.check(r.run(fsr, positions=torch.full((r.N,), -5)), torch.zeros(r.N, dtype=torch.int64))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_in_place_and_slices_of_fused_rows(fsr, dtype):
    announce(f"append with rotation, in place and strided {dtype}")
    r = Rows(3, [(30, 9), (5, 14)], 8, 2, 128, 128, 16, dtype)
    pos = r.ctx[r.owner] + r.place
    want = r.run(fsr)
    caches = [x.clone() for x in r.got]
    assert torch.equal(r.run(fsr, in_place=True), want) and all(torch.equal(a, b) for a, b in zip(caches, r.got))
    fused = torch.cat([x.flatten(1) for x in (r.q, r.k, r.v)] + [torch.zeros(r.N + 2, 16, dtype=dtype)], 1).cuda()
    q, k, v = (fused[:, a:b].unflatten(1, (-1, 128)) for a, b in ((0, 1024), (1024, 1280), (1280, 1536)))
    assert torch.equal(r.run(fsr, q=q, k_new=k, v_new=v), want) and all(torch.equal(a, b) for a, b in zip(caches, r.got))
    r.check(want, pos)


def test_positions_without_a_page_are_skipped(fsr):
    announce("append with rotation, pages")
    r = Rows(4, [(30, 9), (5, 14)], 8, 2, 128, 128, 16, BF)
    want = r.run(fsr)
    for bad in (-1, 1 << 30, r.caches[0].shape[0]):
        bt = r.bt.clone()
        bt[0] = bad
        assert torch.equal(r.run(fsr, block_tables=bt.cuda()), want)  # queries are turned all the same
        for got, before in zip(r.got, r.caches):
            changed = (got.cpu() != before).flatten(1).any(1).nonzero()[:, 0].tolist()
            assert set(changed) <= set(r.bt[1, :2].tolist())
    assert torch.equal(r.run(fsr, block_tables=r.bt[:, :1].contiguous().cuda()), want)  # a table that ends before the rows do
    assert torch.equal(r.run(fsr, ctx_lens=torch.tensor([-50, -50], dtype=torch.int32).cuda(), positions=r.ctx[r.owner] + r.place), want)
    assert all(torch.equal(a.cpu(), b) for a, b in zip(r.got, r.caches))


def test_values_that_are_not_finite(fsr):
    announce("append with rotation, not finite")
    r = Rows(5, [(3, 4)], 2, 1, 64, 32, 16, BF)
    r.q[0, 0, 40], r.k[1, 0, 50], r.v[2, 0, 1] = float("nan"), float("inf"), float("-inf")
    out = r.run(fsr)
    assert out[0, 0].isnan().nonzero().tolist() == [[40]] and not out[1:].isnan().any()
    assert torch.isinf(r.got[0]).sum() == 1 and torch.isinf(r.got[1]).sum() == 1


def test_replays(fsr):
    announce("append with rotation, graph")
    r = Rows(6, [(30, 9), (5, 14)], 8, 2, 128, 128, 16, BF)
    want = r.run(fsr, words=1)
    caches = [x.clone() for x in r.got]
    k, v, out = (x.cuda() for x in (r.caches[0], r.caches[1], torch.zeros_like(r.q)))
    args = dict(q=r.q.cuda(), k_new=r.k.cuda(), v_new=r.v.cuda(), cos_sin=r.table.cuda(), k_cache=k, v_cache=v, block_tables=r.bt.cuda(), ctx_lens=r.ctx.int().cuda(),
                cu_q=r.cu.cuda(), q_out=out, tree_mask=r.mask(1).cuda())
    fsr.kv_append_rope(**args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fsr.kv_append_rope(**args)
    for _ in range(3):
        for x, y in ((k, r.caches[0]), (v, r.caches[1])):
            x.copy_(y)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:r.N].cpu(), want) and torch.equal(k, caches[0]) and torch.equal(v, caches[1])


def test_codes_are_those_of_kv_append_kv8(fsr):
    """Values, and keys by the cosine 1 and the sine 0, enter 8-bit caches as fsr_kv_append_kv8 stores them, whatever the scale: powers
    of two, fractions of all ones, tiny, huge and zero ones; values from the smallest to infinities and NaN."""
    announce("append with rotation, codes")
    scales = torch.tensor([1.0, 0.0123, 2.0 ** -9 * (2 - 2.0 ** -23), 3e-20, 1e-41, 7e33, 0.0, 1.7e-3])
    gen = torch.Generator().manual_seed(9)
    bits = torch.randint(-32768, 32768, (64, 8, 64), generator=gen).to(torch.int16)
    k, v = bits.view(BF).cuda(), (torch.randn(64, 8, 64, generator=gen) * scales[:, None] * 100).to(BF).cuda()
    v[:32] = (scales[:, None] * torch.arange(-16, 16)[:, None, None] / 16 * torch.linspace(0, 64, 64)).to(BF).cuda()  # on ties and beside them
    bt, ctx, cu = (torch.tensor(x, dtype=torch.int32).cuda() for x in ([[0, 1, 2, 3]], [0], [0, 64]))
    caches = [torch.zeros(4, 8, 16, 64, dtype=torch.uint8, device="cuda") for _ in range(4)]
    table = torch.cat([torch.ones(64, 32), torch.zeros(64, 32)], 1).cuda()
    fsr.kv_append_kv8(v, v, caches[0], caches[1], scales.cuda(), scales.cuda(), bt, ctx, cu)
    fsr.kv_append_rope(v, v, v, table, caches[2], caches[3], bt, ctx, cu, k_scale=scales.cuda(), v_scale=scales.cuda())
    value = lambda x: x.view(torch.float8_e4m3fn).float().nan_to_num(nan=1e3)  # noqa: E731
    assert [int((value(caches[0]) != value(caches[2]))[:, h].sum()) for h in range(8)] == [0] * 8 and torch.equal(caches[1], caches[3])  # (-0 - -0 * 0 = 0: the sign of a zero key may differ)
    # (what is not finite meets the sine 0, so of these only values are compared)
    fsr.kv_append_kv8(k, k, caches[0], caches[1], scales.cuda(), scales.cuda(), bt, ctx, cu)
    fsr.kv_append_rope(k, k, k, table, caches[2], caches[3], bt, ctx, cu, k_scale=scales.cuda(), v_scale=scales.cuda())
    assert torch.equal(caches[1], caches[3])
