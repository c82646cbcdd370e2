"""fsr_latent_attention_expanded against the definition in 64 bits."""
import pytest
import torch

from gpu_utils import announce
from plain_attention import attend, check, offsets

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def fsr():
    import paper_2604_20503_amd as f
    f.load_library()
    return f


class Batch:
    def __init__(self, seed, rows, keys, H, dims, dtype):
        gen = torch.Generator().manual_seed(seed)
        self.Dn, self.Dr, self.Dv = dims
        self.rows, self.keys, self.H, self.dtype = rows, keys, H, dtype
        self.N, self.T = sum(rows), sum(keys)
        normal = lambda *shape: torch.randn(shape, generator=gen).to(dtype)  # noqa: E731
        self.q = normal(self.N + 2, H, self.Dn + self.Dr)
        self.kv, self.rope = normal(self.T + 1, H, self.Dn + self.Dv), normal(self.T + 1, self.Dr)
        self.scale = (self.Dn + self.Dr) ** -0.5

    def reference(self):
        o, A = torch.zeros(self.N, self.H, self.Dv, dtype=torch.float64), torch.zeros(self.N, self.H, self.Dv, dtype=torch.float64)
        lse, e = torch.zeros(self.N, self.H, dtype=torch.float64), torch.zeros(self.N, self.H, dtype=torch.float64)
        a = b = 0
        for n, L in zip(self.rows, self.keys):
            for h in range(self.H):
                k = torch.cat([self.kv[b:b + L, h, :self.Dn], self.rope[b:b + L]], 1)
                o[a:a + n, h], lse[a:a + n, h], A[a:a + n, h], e[a:a + n, h] = attend(
                    self.q[a:a + n, h], k, self.kv[b:b + L, h, self.Dn:], self.scale, L - n + torch.arange(n))
            a, b = a + n, b + L
        return o, lse, A, e

    def run(self, fsr, out_dtype, **kw):
        out = torch.full((self.N + 2, self.H, self.Dv), 7.0, dtype=out_dtype, device="cuda")
        lse = torch.full((self.N + 2, self.H), 7.0, dtype=F32, device="cuda")
        fsr.latent_attention_expanded(self.q.cuda(), self.kv.cuda(), self.rope.cuda(), offsets(self.rows).cuda(), offsets(self.keys).cuda(),
                                      scale=self.scale, out=out, lse=lse, **kw)
        torch.cuda.synchronize()
        assert (out[self.N:] == 7).all() and (lse[self.N:] == 7).all()
        return out[:self.N], lse[:self.N]

    def compare(self, name, got):
        o, lse, A, e = self.reference()
        check(name, got[0].reshape(-1, self.Dv), got[1].reshape(-1), o.view(-1, self.Dv), lse.view(-1), A.view(-1, self.Dv), e.view(-1), self.dtype)


BIG, SMALL = (128, 64, 128), (64, 32, 64)
CASES = [
    ("one row, one key", [1], [1], 2, BIG),
    ("one row, many keys", [1, 1], [300, 65], 3, BIG),
    ("square", [64, 128, 33], [64, 128, 33], 2, BIG),
    ("around tiles", [1, 63, 65, 127, 129], [2, 64, 130, 127, 200], 1, BIG),
    ("behind a context", [70, 10], [500, 267], 4, BIG),
    ("more rows than keys", [40, 150, 5], [7, 100, 0], 2, BIG),
    ("no rows, no keys", [0, 3, 0, 0, 2], [10, 20, 0, 5, 2], 2, BIG),
    ("one long request", [300], [1500], 1, BIG),
    ("small heads", [100, 1, 31], [100, 90, 200], 5, SMALL),
    ("small heads, rows that see nothing", [130, 20], [10, 40], 2, SMALL),
]


@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_expanded(fsr, case, dtype, out_dtype):
    announce(f"latent expanded: {case} {dtype} {out_dtype}")
    b = Batch(1, *case[1:], dtype)
    b.compare(case[0], b.run(fsr, out_dtype, max_q_len=max(b.rows)))


@pytest.mark.parametrize("workgroups", [1, 3, 50])
def test_expanded_on_part_of_the_device(fsr, workgroups):
    announce(f"latent expanded, {workgroups} workgroups")
    b = Batch(2, [150, 40, 1], [400, 40, 700], 3, BIG, BF)
    b.compare("workgroups", b.run(fsr, BF, max_workgroups=workgroups))


@pytest.mark.parametrize("seed", range(6))
def test_expanded_random_shapes(fsr, seed):
    gen = torch.Generator().manual_seed(200 + seed)
    draw = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=gen))  # noqa: E731
    B = draw(1, 8)
    rows = [draw(0, 200) for _ in range(B)]
    keys = [max(0, n + draw(-20, 300)) for n in rows]
    args = (rows, keys, draw(1, 4), [BIG, SMALL][draw(0, 1)], [BF, F32][draw(0, 1)])
    announce(f"latent expanded, random {seed}: {args}")
    b = Batch(seed, *args)
    b.compare(f"random {seed}", b.run(fsr, b.dtype))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_values_that_are_not_finite_stay_where_they_are_seen(fsr, dtype):
    """Values of inf, -inf and NaN at key 70: the rows before position 70 are as without them, the others take them over column by
    column (their keys are finite)."""
    announce(f"latent expanded, not finite {dtype}")
    b = Batch(3, [100], [100], 2, BIG, dtype)
    o, lse, A, e = b.reference()
    b.kv[70, :, 128 + 5], b.kv[70, :, 128 + 6], b.kv[70, :, 128 + 77] = float("inf"), float("-inf"), float("nan")
    out, got_lse = b.run(fsr, dtype)
    check("rows before", out[:70].reshape(-1, 128), got_lse[:70].reshape(-1), o[:70].reshape(-1, 128), lse[:70].reshape(-1), A[:70].reshape(-1, 128),
          e[:70].reshape(-1), dtype)
    late = out[70:].float().cpu()
    assert late[..., 5].eq(float("inf")).all() and late[..., 6].eq(float("-inf")).all() and late[..., 77].isnan().all()
    fine = torch.ones(128, dtype=torch.bool)
    fine[[5, 6, 77]] = False
    check("other columns", out[70:, :, fine.cuda()].reshape(-1, 125), got_lse[70:].reshape(-1), o[70:, :, fine].reshape(-1, 125), lse[70:].reshape(-1),
          A[70:, :, fine].reshape(-1, 125), e[70:].reshape(-1), dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_keys_that_are_not_finite_and_masked(fsr, dtype):
    """Keys of NaN and inf: rows that do not see them are as without them; a key of large negative scores takes no weight."""
    announce(f"latent expanded, keys not finite {dtype}")
    b = Batch(4, [90], [90], 1, SMALL, dtype)
    o, lse, A, e = b.reference()
    b.kv[80, 0, 3], b.rope[85, 1] = float("nan"), float("inf")
    out, got_lse = b.run(fsr, dtype)
    check("rows before", out[:80].reshape(-1, 64), got_lse[:80].reshape(-1), o[:80].reshape(-1, 64), lse[:80].reshape(-1), A[:80].reshape(-1, 64),
          e[:80].reshape(-1), dtype)
    assert out[80:].isnan().all() and got_lse[80:].isnan().all()


def test_scores_of_the_types_extremes(fsr):
    """Scores up to 3e38 in size, of both signs: the largest takes all the weight."""
    announce("latent expanded, extreme scores")
    b = Batch(5, [3], [40], 1, SMALL, F32)
    b.q[:], b.kv[:, :, :64], b.rope[:] = 0.0, 0.0, 0.0
    b.q[:, :, 0] = 1.0
    b.kv[:, 0, 0] = -3.0e38
    b.kv[11, 0, 0] = 2.5e38
    b.scale = 1.0
    out, lse = b.run(fsr, F32)
    assert torch.equal(out.cpu()[:, 0], b.kv[11, 0, 64:].expand(3, -1)) and torch.isfinite(lse).all()


def test_replays(fsr):
    announce("latent expanded, graph")
    b = Batch(6, [200, 30], [900, 30], 4, BIG, BF)
    want, want_lse = b.run(fsr, BF)
    q, kv, rope, cu, cu_k = b.q.cuda(), b.kv.cuda(), b.rope.cuda(), offsets(b.rows).cuda(), offsets(b.keys).cuda()
    out, lse = torch.zeros(b.q.shape[0], 4, 128, dtype=BF, device="cuda"), torch.zeros(b.q.shape[0], 4, device="cuda")
    ws = torch.empty(fsr.expanded_workspace_bytes(N_cap=b.q.shape[0], H=4, D_nope=128, D_rope=64, D_v=128, dtype=BF, out_dtype=BF), dtype=torch.uint8, device="cuda")
    call = lambda: fsr.latent_attention_expanded(q, kv, rope, cu, cu_k, scale=b.scale, out=out, lse=lse, workspace=ws)  # noqa: E731
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
