"""fsr_verify_attention_shared against the definition in 64 bits, and beside fsr_verify_attention."""
import pytest
import torch

from gpu_utils import announce
from plain_attention import attend, check, offsets, slots

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def fsr():
    import paper_2604_20503_amd as f
    f.load_library()
    return f


class Batch:
    """groups: [(prefix, [(own context, rows), ...]), ...]."""

    def __init__(self, seed, groups, H_q, H_kv, D, P, dtype, token_major=False):
        gen = torch.Generator().manual_seed(seed)
        self.H_q, self.H_kv, self.D, self.P, self.dtype, self.token_major = H_q, H_kv, D, P, dtype, token_major
        self.prefix = [g[0] for g in groups]
        self.cu_groups = offsets([len(g[1]) for g in groups])
        self.reqs = [(k, p + c, n) for k, (p, rs) in enumerate(groups) for c, n in rs]
        self.rows = [r[2] for r in self.reqs]
        self.N, self.cu = sum(self.rows), offsets(self.rows)
        need = [-(-(c + n) // P) for _, c, n in self.reqs]
        whole = [self.prefix[g] // P for g, _, _ in self.reqs]  # pages held in common
        n_pages = sum(p // P for p in self.prefix) + sum(max(0, a - b) for a, b in zip(need, whole)) + 2
        perm = torch.randperm(n_pages, generator=gen).to(torch.int32)
        self.bt = torch.full((len(need), max(need + whole + [1])), -1, dtype=torch.int32)
        at, common = 0, []
        for p in self.prefix:
            common.append(perm[at:at + p // P])
            at += p // P
        for i, (g, _, _) in enumerate(self.reqs):
            self.bt[i, :whole[i]] = common[g]
            n = max(0, need[i] - whole[i])
            self.bt[i, whole[i]:whole[i] + n] = perm[at:at + n]
            at += n
        normal = lambda *shape: torch.randn(shape, generator=gen).to(dtype)  # noqa: E731
        self.k, self.v = normal(n_pages, P, H_kv, D), normal(n_pages, P, H_kv, D)
        self.q, self.n_pages = normal(self.N + 2, H_q, D), n_pages
        for x in (self.k, self.v):  # where a prefix ends inside a page, every request's copy of that page holds the same values
            for i, (g, _, _) in enumerate(self.reqs):
                first, r = int(self.cu_groups[g]), self.prefix[g] % P
                if r and i != first:
                    x[self.bt[i, whole[i]].long(), :r] = x[self.bt[first, whole[i]].long(), :r]
        self.scale = D ** -0.5

    def reference(self):
        G = self.H_q // self.H_kv
        shape = (self.N, self.H_q)
        o, A = torch.zeros(*shape, self.D, dtype=torch.float64), torch.zeros(*shape, self.D, dtype=torch.float64)
        lse, e = torch.zeros(shape, dtype=torch.float64), torch.zeros(shape, dtype=torch.float64)
        for i, (_, c, n) in enumerate(self.reqs):
            a = int(self.cu[i])
            s = slots(self.bt[i], c + n, self.P)
            for h in range(self.H_q):
                o[a:a + n, h], lse[a:a + n, h], A[a:a + n, h], e[a:a + n, h] = attend(
                    self.q[a:a + n, h], self.k.flatten(0, 1)[s, h // G], self.v.flatten(0, 1)[s, h // G], self.scale, c + torch.arange(n))
        return o, lse, A, 2 * e  # (the weights of two parts are put together once more)

    def dev(self):
        lay = (lambda x: x) if self.token_major else (lambda x: x.transpose(1, 2).contiguous())
        i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
        return dict(q=self.q.cuda(), k_cache=lay(self.k).cuda(), v_cache=lay(self.v).cuda(), block_tables=self.bt.cuda(), ctx_lens=i32([r[1] for r in self.reqs]),
                    cu_q=self.cu.cuda(), cu_groups=self.cu_groups.cuda(), prefix_lens=i32(self.prefix))

    def run(self, fsr, out_dtype, **kw):
        lay = fsr.binding.KV_TOKEN_MAJOR if self.token_major else fsr.binding.KV_HEAD_MAJOR
        out = torch.full((self.N + 2, self.H_q, self.D), 7.0, dtype=out_dtype, device="cuda")
        lse = torch.full((self.N + 2, self.H_q), 7.0, dtype=F32, device="cuda")
        fsr.verify_attention_shared(**{**self.dev(), **kw}, scale=self.scale, out=out, lse=lse, kv_layout=lay)
        torch.cuda.synchronize()
        assert (out[self.N:] == 7).all() and (lse[self.N:] == 7).all()
        return out[:self.N], lse[:self.N]

    def compare(self, name, got):
        o, lse, A, e = self.reference()
        check(name, got[0].reshape(-1, self.D), got[1].reshape(-1), o.view(-1, self.D), lse.view(-1), A.view(-1, self.D), e.view(-1), self.dtype)


CASES = [
    ("one request, no prefix", [(0, [(40, 3)])], 8, 2, 128, 16),
    ("one request behind a prefix", [(64, [(10, 2)])], 8, 2, 128, 16),
    ("one group", [(100, [(5, 1), (0, 4), (60, 2), (17, 0), (33, 9)])], 8, 2, 128, 16),
    ("groups with and without prefix", [(200, [(3, 2), (9, 1)]), (0, [(50, 3), (0, 1)]), (65, [(1, 1)])], 16, 4, 128, 16),
    ("prefix longer than all else", [(1500, [(0, 1), (0, 1), (2, 1)])], 8, 2, 128, 16),
    ("many rows a group", [(300, [(7 * k % 40, 1 + k % 6) for k in range(30)])], 8, 1, 128, 16),
    ("one head a group, odd pages", [(77, [(5, 3), (8, 2)]), (13, [(2, 1), (0, 7)])], 3, 3, 128, 5),
    ("seven heads a group", [(128, [(30, 2), (1, 4)])], 28, 4, 128, 32),
    ("heads of 64", [(250, [(20, 2), (0, 1), (64, 5)]), (40, [(9, 3)])], 8, 2, 64, 16),
    ("long own context", [(32, [(2500, 2), (3, 1)])], 4, 1, 128, 16),
    ("empty groups", [(90, []), (50, [(4, 2)]), (70, [])], 8, 2, 128, 16),
]


@pytest.mark.parametrize("token_major", [False, True])
@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_shared(fsr, case, dtype, out_dtype, token_major):
    announce(f"shared prefix: {case} {dtype} {out_dtype} token_major={token_major}")
    b = Batch(1, *case[1:], dtype, token_major)
    b.compare(case[0], b.run(fsr, out_dtype, max_q_len=max(b.rows)))


@pytest.mark.parametrize("workgroups", [1, 5, 60])
def test_shared_on_part_of_the_device(fsr, workgroups):
    announce(f"shared prefix, {workgroups} workgroups")
    b = Batch(2, [(400, [(5 * k, 1 + k % 4) for k in range(9)]), (130, [(70, 6), (300, 1)])], 8, 2, 128, 16, BF)
    b.compare("workgroups", b.run(fsr, BF, max_workgroups=workgroups))


@pytest.mark.parametrize("seed", range(6))
def test_shared_random_shapes(fsr, seed):
    gen = torch.Generator().manual_seed(300 + seed)
    draw = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=gen))  # noqa: E731
    groups = [(draw(0, 500) * draw(0, 1) + draw(0, 40), [(draw(0, 90), draw(0, 5)) for _ in range(draw(1, 9))]) for _ in range(draw(1, 4))]
    H_kv = draw(1, 3)
    args = (groups, H_kv * draw(1, 9), H_kv, [64, 128][draw(0, 1)], draw(1, 70), [BF, F32][draw(0, 1)], bool(draw(0, 1)))
    announce(f"shared prefix, random {seed}: {args}")
    b = Batch(seed, *args)
    b.compare(f"random {seed}", b.run(fsr, b.dtype))


def test_beside_the_call_without_groups(fsr):
    """The same batch through verify_attention, which reads the prefix request by request."""
    announce("shared prefix beside verify_attention")
    b = Batch(4, [(600, [(9 * k, 1 + k % 5) for k in range(12)])], 32, 8, 128, 16, BF)
    out, lse = b.run(fsr, F32)
    d = b.dev()
    ref_lse = torch.empty(b.N + 2, 32, device="cuda")
    ref, _ = fsr.verify_attention(d["q"], d["k_cache"], d["v_cache"], d["block_tables"], d["ctx_lens"], None, d["cu_q"], scale=b.scale, out_dtype=F32, lse=ref_lse)
    _, _, A, e = b.reference()
    bound = ((2 * e[..., None] + 2.0 ** -15) * A).cuda()
    assert ((out - ref[:b.N]).abs() <= bound).all() and ((lse - ref_lse[:b.N]).abs() <= 2 * e.cuda() + 1e-6).all()


def test_context_below_the_prefix_counts_as_the_prefix(fsr):
    announce("shared prefix, short context")
    b = Batch(5, [(50, [(6, 2), (0, 3)])], 4, 2, 128, 16, BF)
    ctx = torch.tensor([56, 12], dtype=torch.int32).cuda()  # request 1 says 12 instead of 50
    b.compare("short context", b.run(fsr, BF, ctx_lens=ctx))


def test_requests_outside_the_groups_get_no_output(fsr):
    announce("shared prefix, requests outside")
    b = Batch(6, [(30, [(4, 2)]), (40, [(8, 1), (2, 3)]), (20, [(1, 2)])], 4, 2, 128, 16, BF)
    want, want_lse = b.run(fsr, BF)
    out, lse = b.run(fsr, BF, cu_groups=b.cu_groups[1:3].cuda(), prefix_lens=torch.tensor([40], dtype=torch.int32).cuda())
    assert (out[:2] == 7).all() and (out[6:] == 7).all() and (lse[:2] == 7).all() and (lse[6:] == 7).all()
    # (another cut of the line, so other orders of sums: same bounds as always)
    o, l, A, e = b.reference()
    check("inside", out[2:6].reshape(-1, 128), lse[2:6].reshape(-1), o[2:6].reshape(-1, 128), l[2:6].reshape(-1), A[2:6].reshape(-1, 128), e[2:6].reshape(-1), BF)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_values_that_are_not_finite_stay_where_they_are_seen(fsr, dtype):
    """NaN in every slot that no request uses, and infinite values in the last token of each request."""
    announce(f"shared prefix, not finite {dtype}")
    b = Batch(7, [(90, [(10, 3), (50, 2)]), (0, [(20, 2)])], 4, 2, 128, 16, dtype)
    o, lse, A, e = b.reference()
    kf, vf = b.k.flatten(0, 1), b.v.flatten(0, 1)
    used = torch.zeros(kf.shape[0], dtype=torch.bool)
    last = torch.zeros(b.N, dtype=torch.bool)
    for i, (_, c, n) in enumerate(b.reqs):
        s = slots(b.bt[i], c + n, 16)
        used[s] = True
        vf[s[-1], :, 7], vf[s[-1], :, 8] = float("inf"), float("nan")
        last[int(b.cu[i + 1]) - 1] = True
    kf[~used], vf[~used] = float("nan"), float("nan")
    out, got = b.run(fsr, dtype)
    check("rows before", out[~last.cuda()].reshape(-1, 128), got[~last.cuda()].reshape(-1), o[~last].reshape(-1, 128), lse[~last].reshape(-1),
          A[~last].reshape(-1, 128), e[~last].reshape(-1), dtype)
    late = out[last.cuda()].float()
    assert late[..., 7].eq(float("inf")).all() and late[..., 8].isnan().all() and torch.isfinite(late[..., 9:]).all()


def test_replays(fsr):
    announce("shared prefix, graph")
    b = Batch(8, [(500, [(9, 2), (100, 4)]), (31, [(0, 1)])], 8, 2, 128, 16, BF)
    want, want_lse = b.run(fsr, BF)
    d = b.dev()
    out, lse = torch.zeros(b.N + 2, 8, 128, dtype=BF, device="cuda"), torch.zeros(b.N + 2, 8, device="cuda")
    ws = torch.empty(fsr.shared_workspace_bytes(N_cap=b.N + 2, H_q=8, H_kv=2, D=128, dtype=BF, out_dtype=BF), dtype=torch.uint8, device="cuda")
    call = lambda: fsr.verify_attention_shared(**d, scale=b.scale, out=out, lse=lse, workspace=ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        out.zero_()
        lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:b.N], want) and torch.equal(lse[:b.N], want_lse)
        b.run(fsr, BF)
