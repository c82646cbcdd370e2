"""fsr_verify_attention_tree against the definition in 64 bits, and beside fsr_verify_attention."""
import pytest
import torch

from gpu_utils import announce
from plain_attention import check, offsets, pages, slots
from plain_tree import attend_masked, sees_of, tree, words_of

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def fsr():
    import paper_2604_20503_amd as f
    f.load_library()
    return f


class Batch:
    """reqs: [(context, rows), ...]; sees: one [rows, rows] mask each (trees by default)."""

    def __init__(self, seed, reqs, H_q, H_kv, D, P, dtype, token_major=False, words=None, sees=None):
        gen = torch.Generator().manual_seed(seed)
        self.reqs, self.H_q, self.H_kv, self.D, self.P, self.dtype, self.token_major = reqs, H_q, H_kv, D, P, dtype, token_major
        self.rows = [r for _, r in reqs]
        self.N, self.cu, self.scale = sum(self.rows), offsets(self.rows), D ** -0.5
        self.words = words or max(1, -(-max(self.rows + [1]) // 64))
        self.sees = sees or [sees_of(tree(n, gen)) if n else torch.zeros(0, 0, dtype=torch.bool) for n in self.rows]
        self.bt, n_pages = pages([c + n for c, n in reqs], P, gen)
        normal = lambda *shape: torch.randn(shape, generator=gen).to(dtype)  # noqa: E731
        self.k, self.v, self.q = normal(n_pages, P, H_kv, D), normal(n_pages, P, H_kv, D), normal(self.N + 2, H_q, D)
        self.mask = torch.cat([words_of(s, self.words) for s in self.sees] + [torch.full((2, self.words), -1)])

    def reference(self):
        G, shape = self.H_q // self.H_kv, (self.N, self.H_q)
        o, A = torch.zeros(*shape, self.D, dtype=torch.float64), torch.zeros(*shape, self.D, dtype=torch.float64)
        lse, e = torch.zeros(shape, dtype=torch.float64), torch.zeros(shape, dtype=torch.float64)
        for i, (c, n) in enumerate(self.reqs):
            a, s = int(self.cu[i]), slots(self.bt[i], c + n, self.P)
            tail = self.sees[i].clone()
            tail[:, 64 * self.words:] = False
            seen = torch.cat([torch.ones(n, c, dtype=torch.bool), tail], 1)
            for h in range(self.H_q):
                o[a:a + n, h], lse[a:a + n, h], A[a:a + n, h], e[a:a + n, h] = attend_masked(
                    self.q[a:a + n, h], self.k.flatten(0, 1)[s, h // G], self.v.flatten(0, 1)[s, h // G], self.scale, seen)
        return o, lse, A, e

    def dev(self):
        lay = (lambda x: x) if self.token_major else (lambda x: x.transpose(1, 2).contiguous())
        return dict(q=self.q.cuda(), k_cache=lay(self.k).cuda(), v_cache=lay(self.v).cuda(), block_tables=self.bt.cuda(),
                    ctx_lens=torch.tensor([c for c, _ in self.reqs], dtype=torch.int32).cuda(), cu_q=self.cu.cuda(), tree_mask=self.mask.cuda())

    def run(self, fsr, out_dtype, **kw):
        lay = fsr.binding.KV_TOKEN_MAJOR if self.token_major else fsr.binding.KV_HEAD_MAJOR
        out = torch.full((self.N + 2, self.H_q, self.D), 7.0, dtype=out_dtype, device="cuda")
        lse = torch.full((self.N + 2, self.H_q), 7.0, dtype=F32, device="cuda")
        fsr.verify_attention_tree(**{**self.dev(), **kw}, scale=self.scale, out=out, lse=lse, kv_layout=lay)
        torch.cuda.synchronize()
        assert (out[self.N:] == 7).all() and (lse[self.N:] == 7).all()
        return out[:self.N], lse[:self.N]

    def compare(self, name, got):
        o, lse, A, e = self.reference()
        check(name, got[0].reshape(-1, self.D), got[1].reshape(-1), o.view(-1, self.D), lse.view(-1), A.view(-1, self.D), e.view(-1), self.dtype)


CASES = [
    ("one row, no context", [(0, 1)], 8, 2, 128, 16),
    ("one row behind a context", [(70, 1)], 8, 2, 128, 16),
    ("a tree without context", [(0, 20)], 8, 2, 128, 16),
    ("small trees", [(40, 7), (100, 12), (3, 1), (129, 5)], 8, 2, 128, 16),
    ("trees that end and begin inside tiles", [(63, 2), (64, 3), (65, 31), (31, 33), (33, 64), (1, 63)], 8, 2, 128, 16),
    ("large trees", [(50, 65), (200, 130), (7, 200)], 4, 2, 128, 16),
    ("requests without rows", [(40, 0), (20, 9), (0, 0), (17, 0), (90, 4)], 8, 2, 128, 16),
    ("one head a group, odd pages", [(77, 13), (5, 30)], 3, 3, 128, 5),
    ("seven heads a group", [(128, 22), (30, 4)], 28, 4, 128, 32),
    ("wide groups", [(150, 40), (9, 3)], 32, 1, 128, 64),
    ("heads of 64", [(250, 20), (0, 5), (64, 64)], 8, 2, 64, 16),
    ("long contexts", [(3000, 17), (1700, 40)], 4, 1, 128, 16),
    ("many requests", [(11 * k % 150, 1 + 5 * k % 23) for k in range(40)], 8, 2, 128, 16),
]


@pytest.mark.parametrize("token_major", [False, True])
@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_tree(fsr, case, dtype, out_dtype, token_major):
    announce(f"tree attention: {case} {dtype} {out_dtype} token_major={token_major}")
    b = Batch(1, *case[1:], dtype, token_major)
    b.compare(case[0], b.run(fsr, out_dtype, max_q_len=max(b.rows)))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("words", [1, 2, 16])
def test_any_mask(fsr, words, dtype):
    """Masks that are no trees: rows that see nothing of the call, rows that see others than themselves, rows behind them, all rows; with
    and without a context in front; more rows than the mask has bits."""
    announce(f"tree attention, any mask, {words} words, {dtype}")
    gen = torch.Generator().manual_seed(5)
    reqs = [(0, 40), (30, 100), (64, 17), (0, 1), (5, 64)]
    sees = [torch.rand(n, n, generator=gen) < p for (_, n), p in zip(reqs, (0.3, 0.5, 0.0, 0.0, 1.1))]
    sees[0][3] = sees[0][11] = False  # no key at all: zeros and -inf
    b = Batch(6, reqs, 8, 2, 128, 16, dtype, words=words, sees=sees)
    out, lse = b.run(fsr, dtype)
    b.compare("any mask", (out, lse))
    for r in (3, 11, int(b.cu[3])):
        assert (out[r] == 0).all() and lse[r].eq(float("-inf")).all()


def test_a_chain_is_verify_attention(fsr):
    """Under the mask of a chain both calls have the same definition."""
    announce("tree attention beside verify_attention")
    reqs = [(40 * k + 3, 1 + k % 9) for k in range(12)]
    b = Batch(7, reqs, 32, 8, 128, 16, BF, sees=[torch.ones(n, n, dtype=torch.bool).tril() for _, n in reqs])
    out, lse = b.run(fsr, F32)
    d = b.dev()
    ref_lse = torch.empty(b.N + 2, 32, device="cuda")
    ref, _ = fsr.verify_attention(d["q"], d["k_cache"], d["v_cache"], d["block_tables"], d["ctx_lens"], None, d["cu_q"], scale=b.scale, out_dtype=F32, lse=ref_lse)
    _, _, A, e = b.reference()
    bound = ((2 * e[..., None] + 2.0 ** -15) * A).cuda()
    assert ((out - ref[:b.N]).abs() <= bound).all() and ((lse - ref_lse[:b.N]).abs() <= 2 * e.cuda() + 1e-6).all()


@pytest.mark.parametrize("workgroups", [1, 5, 60])
def test_part_of_the_device(fsr, workgroups):
    announce(f"tree attention, {workgroups} workgroups")
    b = Batch(2, [(400, 20), (130, 3), (700, 90), (0, 8), (20, 1)], 8, 2, 128, 16, BF)
    b.compare("workgroups", b.run(fsr, BF, max_workgroups=workgroups))


@pytest.mark.parametrize("seed", range(10))
def test_random_shapes(fsr, seed):
    gen = torch.Generator().manual_seed(700 + seed)
    draw = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=gen))  # noqa: E731
    reqs = [(draw(0, 900) * draw(0, 1) + draw(0, 70), draw(0, [6, 40, 150][draw(0, 2)])) for _ in range(draw(1, 10))]
    H_kv = draw(1, 3)
    args = (reqs, H_kv * draw(1, 9), H_kv, [64, 128][draw(0, 1)], draw(1, 70), [BF, F32][draw(0, 1)], bool(draw(0, 1)))
    announce(f"tree attention, random {seed}: {args}")
    b = Batch(seed, *args)
    b.compare(f"random {seed}", b.run(fsr, [b.dtype, F32][draw(0, 1)]))


@pytest.mark.parametrize("scale", [1e-3, 30.0, 1e6])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_scores_of_any_size(fsr, dtype, scale):
    announce(f"tree attention, scale {scale} {dtype}")
    b = Batch(9, [(200, 30), (0, 12)], 8, 2, 64, 16, dtype)
    b.scale = scale
    if scale < 1e5:
        b.compare("scale", b.run(fsr, dtype))
        return
    # scores so far apart that the largest one takes all: its value.  fp32: its weight is 1, all others are 0; where pieces of the keys
    # are joined it is multiplied by the piece's weight and by the inverse of that weight, three roundings of 2^-24.  bf16: its weight w
    # enters the product as bf16(w), off by 2^-8 at most, and the sum as it is; the quotient times the value is then rounded to bf16, which
    # makes |v| (1 + 2^-8) (1 + 2^-8) at most, and as much below.
    out, lse = b.run(fsr, dtype)
    for i, (c, n) in enumerate(b.reqs):
        a, s = int(b.cu[i]), slots(b.bt[i], c + n, 16)
        seen = torch.cat([torch.ones(n, c, dtype=torch.bool), b.sees[i]], 1)
        for h in range(8):
            z = (b.q[a:a + n, h].double() @ b.k.flatten(0, 1)[s, h // 4].double().T).masked_fill(~seen, float("-inf"))
            top = z.topk(2, 1) if z.shape[1] > 1 else None
            clear = torch.isinf(top.values[:, 1]) | (top.values[:, 0] - top.values[:, 1] > 1e-3)  # 1e-3 * 1e6: beyond any rounding of the scores
            want = b.v.flatten(0, 1)[s, h // 4][top.indices[:, 0]]
            off, size = (out[a:a + n, h].cpu()[clear].double() - want[clear].double()).abs(), want[clear].double().abs()
            assert (off <= (3.01 * 2.0 ** -24 if dtype == F32 else (1 + 2.0 ** -8) ** 2 - 1) * size).all()


@pytest.mark.parametrize("out_dtype", [BF, F32])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_values_that_are_not_finite_stay_where_they_are_seen(fsr, dtype, out_dtype):
    """NaN in every slot that no request uses; infinities and NaN in a leaf that its own row alone sees, with the lowest and infinite keys."""
    if dtype == F32 and out_dtype == BF:
        pytest.skip("fp32 inputs have fp32 results")
    announce(f"tree attention, not finite {dtype} {out_dtype}")
    b = Batch(8, [(90, 20), (0, 35), (64, 3)], 4, 2, 128, 16, dtype)
    o, lse, A, e = b.reference()
    kf, vf = b.k.flatten(0, 1), b.v.flatten(0, 1)
    used, odd = torch.zeros(kf.shape[0], dtype=torch.bool), torch.zeros(b.N, dtype=torch.bool)
    for i, (c, n) in enumerate(b.reqs):
        s = slots(b.bt[i], c + n, 16)
        used[s] = True
        vf[s[-1], :, 7], vf[s[-1], :, 8], vf[s[-1], :, 9] = float("inf"), float("nan"), float("-inf")
        odd[int(b.cu[i + 1]) - 1] = True  # (a request's last row is a leaf)
    kf[~used], vf[~used] = float("nan"), float("nan")
    out, got = b.run(fsr, out_dtype)
    check("other rows", out[~odd.cuda()].reshape(-1, 128), got[~odd.cuda()].reshape(-1), o[~odd].reshape(-1, 128), lse[~odd].reshape(-1), A[~odd].reshape(-1, 128),
          e[~odd].reshape(-1), dtype)
    late = out[odd.cuda()].float()
    assert late[..., 7].eq(float("inf")).all() and late[..., 8].isnan().all() and late[..., 9].eq(float("-inf")).all() and torch.isfinite(late[..., 10:]).all()
    # keys that are not finite, in the same leaves
    for i, (c, n) in enumerate(b.reqs):
        s = slots(b.bt[i], c + n, 16)
        kf[s[-1]], vf[s[-1]] = float("nan"), 1.0
    out, got = b.run(fsr, out_dtype)
    check("other rows", out[~odd.cuda()].reshape(-1, 128), got[~odd.cuda()].reshape(-1), o[~odd].reshape(-1, 128), lse[~odd].reshape(-1), A[~odd].reshape(-1, 128),
          e[~odd].reshape(-1), dtype)


def test_page_ids_outside_the_pool_are_clamped(fsr):
    """Entries behind a request's last page hold anything."""
    announce("tree attention, page ids")
    b = Batch(10, [(40, 10), (100, 3)], 8, 2, 128, 16, BF)
    want = b.run(fsr, BF)
    bt = torch.cat([b.bt, torch.full((2, 3), 1 << 30, dtype=torch.int32)], 1)
    bt[bt < 0] = -(1 << 30)
    got = b.run(fsr, BF, block_tables=bt.cuda())
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_replays(fsr):
    """A captured call follows lengths and masks that change between replays; a used workspace, and eager calls in between."""
    announce("tree attention, graph")
    first, second = (Batch(11 + k, [(500 - 300 * k, 20), (100, 4 + 7 * k), (3, 9 - 7 * k)], 8, 2, 128, 16, BF) for k in range(2))
    assert first.N == second.N
    want = [b.run(fsr, BF) for b in (first, second)]
    d, e = first.dev(), second.dev()
    n_pages = max(d["k_cache"].shape[0], e["k_cache"].shape[0])
    width = max(d["block_tables"].shape[1], e["block_tables"].shape[1])
    room = {k: torch.zeros((n_pages,) + tuple(v.shape[1:]), dtype=v.dtype, device="cuda") if k.endswith("cache") else v.clone() for k, v in d.items()}
    room["block_tables"] = torch.zeros(3, width, dtype=torch.int32, device="cuda")

    def load(x):
        for k, v in x.items():
            if k.endswith("cache"):
                room[k][:v.shape[0]] = v
            elif k == "block_tables":
                room[k][:, :v.shape[1]] = v
            else:
                room[k].copy_(v)
    out, lse = torch.zeros(first.N + 2, 8, 128, dtype=BF, device="cuda"), torch.zeros(first.N + 2, 8, device="cuda")
    ws = torch.randint(0, 255, (fsr.tree_workspace_bytes(N_cap=first.N + 2, H_q=8, H_kv=2, D=128, dtype=BF, out_dtype=BF),), dtype=torch.uint8, device="cuda")
    call = lambda: fsr.verify_attention_tree(**room, scale=first.scale, out=out, lse=lse, workspace=ws)  # noqa: E731
    load(d)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(4):
        load((d, e)[k % 2])
        out.zero_()
        lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:first.N], want[k % 2][0]) and torch.equal(lse[:first.N], want[k % 2][1])
        first.run(fsr, BF)


def test_two_streams(fsr):
    announce("tree attention, two streams")
    a, b = Batch(13, [(900, 30), (20, 4)], 8, 2, 128, 16, BF), Batch(14, [(300, 70), (50, 2)], 8, 2, 128, 16, BF)
    want = [x.run(fsr, BF) for x in (a, b)]
    args, streams = [x.dev() for x in (a, b)], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(5):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                lse = torch.empty(args[k]["q"].shape[:2], device="cuda")
                got[k] = fsr.verify_attention_tree(**args[k], scale=a.scale, lse=lse)
    torch.cuda.synchronize()
    for k, x in enumerate((a, b)):
        assert torch.equal(got[k][0][:x.N], want[k][0]) and torch.equal(got[k][1][:x.N], want[k][1])
