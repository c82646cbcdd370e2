"""fsr_tree_accept against the walk row by row, fsr_kv_commit against moves one after the other, and a step of trees as it is used."""
import pytest
import torch

from gpu_utils import announce
from plain_attention import offsets, pages, slots
from plain_tree import sees_of, tree, walk, words_of

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def fsr():
    import paper_2604_20503_amd as f
    f.load_library()
    return f


class Trees:
    def __init__(self, seed, rows, words=None, tokens=3):
        """Few tokens: several children agree with the target, and paths are long."""
        gen = torch.Generator().manual_seed(seed)
        self.rows, self.cu, self.N = rows, offsets(rows), sum(rows)
        self.words = words or max(1, -(-max(rows + [1]) // 64))
        self.parents = [tree(n, gen, 0.6) if n else [] for n in rows]
        self.mask = torch.cat([words_of(sees_of(p), self.words) for p in self.parents if p] + [torch.full((3, self.words), -1)])
        self.draft, self.target = (torch.randint(0, tokens, (self.N + 3,), generator=gen, dtype=torch.int32) for _ in "dt")

    def want(self, S_max):
        acc, emitted, path = [], [], []
        for i, p in enumerate(self.parents):
            a, b = int(self.cu[i]), int(self.cu[i + 1])
            w, e = walk(p, self.draft[a:b].tolist(), self.target[a:b].tolist(), S_max)
            acc.append(len(w) - 1)
            path.append(w + [-1] * (S_max + 1 - len(w)))
            emitted.append(e + [-1] * (S_max + 1 - len(e)))
        return acc, emitted, path

    def run(self, fsr, S_max, **kw):
        keep = torch.full((self.N + 3,), 9, dtype=torch.uint8, device="cuda")
        got = fsr.tree_accept(self.target.cuda(), self.draft.cuda(), self.mask.cuda(), self.cu.cuda(), S_max=S_max, keep_mask=keep, **kw)
        torch.cuda.synchronize()
        return [x.cpu() for x in got] + [keep.cpu()]

    def compare(self, fsr, S_max):
        acc, emitted, path = self.want(S_max)
        got = self.run(fsr, S_max)
        assert got[0].tolist() == acc and got[1].tolist() == [a + 1 for a in acc]
        assert got[2].tolist() == emitted and got[3].tolist() == path
        keep = torch.zeros(self.N, dtype=torch.uint8)
        for i, p in enumerate(path):
            keep[[int(self.cu[i]) + j for j in p if j >= 0]] = 1
        assert torch.equal(got[4][:self.N], keep) and (got[4][self.N:] == 9).all()


@pytest.mark.parametrize("S_max", [0, 1, 5, 40])
@pytest.mark.parametrize("rows", [[1], [12], [64, 65, 1, 0, 63, 128], [0, 0], [7] * 300, [1000, 3], [1024]], ids=str)
def test_accept(fsr, rows, S_max):
    announce(f"tree accept {rows[:6]} S_max={S_max}")
    Trees(1, rows).compare(fsr, S_max)
    Trees(2, rows, tokens=1).compare(fsr, S_max)  # every child agrees
    Trees(3, rows, tokens=1 << 30).compare(fsr, S_max)  # none does


def test_rows_without_a_bit_are_no_children(fsr):
    announce("tree accept, few words")
    t = Trees(4, [100, 20, 200], words=1, tokens=1)
    t.mask.zero_()
    for i, n in enumerate(t.rows):  # a chain through the rows that have a bit
        for j in range(min(n, 64)):
            t.mask[int(t.cu[i]) + j, 0] = -1 if j == 63 else (1 << (j + 1)) - 1
    acc, nem, em, path, keep = t.run(fsr, 90)
    assert acc.tolist() == [63, 19, 63] and path[0, :64].tolist() == list(range(64)) and (path[0, 64:] == -1).all()
    assert keep[:100].tolist() == [1] * 64 + [0] * 36


def test_first_of_equal_children(fsr):
    announce("tree accept, equal children")
    t = Trees(5, [5], tokens=1)
    t.parents = [[-1, 0, 0, 1, 2]]
    t.mask = torch.cat([words_of(sees_of(t.parents[0]), 1), torch.zeros(3, 1, dtype=torch.int64)])
    assert t.run(fsr, 4)[3].tolist() == [[0, 1, 3, -1, -1]]


class Paths:
    def __init__(self, seed, reqs, H_kv, D, P, dtype, token_major, S_max):
        gen = torch.Generator().manual_seed(seed)
        self.reqs, self.P, self.token_major, self.S_max = reqs, P, token_major, S_max
        self.bt, n_pages = pages([c + n for c, n in reqs], P, gen)
        shape = (n_pages, P, H_kv, D) if token_major else (n_pages, H_kv, P, D)
        self.k, self.v = ((torch.randint(0, 256, shape, generator=gen, dtype=torch.uint8) if dtype == torch.uint8 else torch.randn(shape, generator=gen).to(dtype)) for _ in "kv")
        self.ctx = torch.tensor([c for c, _ in reqs], dtype=torch.int32)
        self.path = torch.full((len(reqs), S_max + 1), -1, dtype=torch.int32)
        self.acc = torch.full((len(reqs),), -1, dtype=torch.int32)
        for i, (c, n) in enumerate(reqs):
            if n:
                a = int(torch.randint(0, min(n - 1, S_max) + 1, (1,), generator=gen))
                self.acc[i] = a
                self.path[i, 0] = 0
                self.path[i, 1:a + 1] = (torch.randperm(n - 1, generator=gen)[:a] + 1).sort().values.int()

    def want(self):
        out = []
        for cache in (self.k, self.v):
            x = (cache if self.token_major else cache.transpose(1, 2)).clone()
            flat = x.reshape(-1, *x.shape[2:])
            for i, (c, n) in enumerate(self.reqs):
                s = slots(self.bt[i], c + n, self.P)
                for k in range(1, int(self.acc[i]) + 1):
                    flat[s[c + k]] = flat[s[c + int(self.path[i, k])]]
            out.append(flat.view(x.shape) if self.token_major else flat.view(x.shape).transpose(1, 2).contiguous())
        return out

    def run(self, fsr, **kw):
        lay = fsr.binding.KV_TOKEN_MAJOR if self.token_major else fsr.binding.KV_HEAD_MAJOR
        args = {**dict(k_cache=self.k.cuda(), v_cache=self.v.cuda(), block_tables=self.bt.cuda(), ctx_lens=self.ctx.cuda(), accepted_len=self.acc.cuda(), path=self.path.cuda()), **kw}
        fsr.kv_commit(**args, kv_layout=lay)
        torch.cuda.synchronize()
        return args["k_cache"].cpu(), args["v_cache"].cpu()


@pytest.mark.parametrize("token_major", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32, torch.uint8])
@pytest.mark.parametrize("reqs,H_kv,D,P,S_max", [([(0, 1)], 2, 64, 16, 3), ([(100, 20), (33, 64), (0, 7), (5, 0), (31, 40)], 2, 128, 16, 6),
                                                 ([(10, 60), (0, 33)], 3, 64, 5, 40), ([(7 * k % 50, 1 + 3 * k % 30) for k in range(130)], 1, 128, 64, 9),
                                                 ([(3, 30)], 4, 128, 1, 29)], ids=str)
def test_commit(fsr, reqs, H_kv, D, P, S_max, dtype, token_major):
    announce(f"commit {len(reqs)} requests, {H_kv} heads of {D}, pages of {P}, S_max={S_max}, {dtype} token_major={token_major}")
    p = Paths(1, reqs, H_kv, D, P, dtype, token_major, S_max)
    for got, want in zip(p.run(fsr), p.want()):
        assert torch.equal(got.view(torch.uint8), want.view(torch.uint8))


def test_commit_of_long_paths_keeps_the_order(fsr):
    """Every row of a path one place to the front: each place that is written is the next one's source."""
    announce("commit, long path")
    p = Paths(2, [(20, 60)], 2, 64, 16, BF, False, 55)
    p.acc[0], p.path[0, 1:] = 55, torch.arange(2, 57)
    for got, want in zip(p.run(fsr), p.want()):
        assert torch.equal(got, want)


def test_commit_skips_what_has_no_place(fsr):
    announce("commit, places")
    p = Paths(3, [(20, 30), (40, 30)], 2, 64, 16, BF, False, 4)
    p.acc[:], p.path[:] = 4, torch.tensor([0, 5, 9, 20, 29])
    full = p.run(fsr)
    bt = p.bt.clone()
    bt[0] = 1 << 30
    k, v = p.run(fsr, block_tables=bt.cuda())
    rest = [x for x in range(p.k.shape[0]) if x not in p.bt[1].tolist()]
    assert torch.equal(k[rest], p.k[rest]) and torch.equal(k[p.bt[1].long().clamp(min=0)], full[0][p.bt[1].long().clamp(min=0)])
    p.path[0] = torch.tensor([0, -1, 1, -(1 << 30), 1 << 30])  # lower than their place, or far behind the table
    k, v = p.run(fsr)
    own = p.bt[0][p.bt[0] >= 0].long()
    assert torch.equal(k[own], p.k[own]) and torch.equal(v[own], p.v[own])


@pytest.mark.parametrize("near_root,longest", [(1.6, 1), (0.4, 2)], ids=["wide", "deep"])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_step_of_trees(fsr, dtype, near_root, longest):
    """Append with rotation, attention, log probabilities, acceptance and commit of a model of one layer; the caches and results are those of
    verifying the accepted path as a chain, and the next chain's context holds what the tree left."""
    announce(f"a step of trees {dtype}")
    gen = torch.Generator().manual_seed(21)
    H_q, H_kv, D, P, V, S_max, reqs = 8, 2, 64, 16, 50, 6, [(30, 20), (5, 33), (64, 1), (100, 12)]
    rows = [n for _, n in reqs]
    N, cu = sum(rows), offsets(rows)
    bt, n_pages = pages([c + n for c, n in reqs], P, gen)
    bt, cu_d, ctx = bt.cuda(), cu.cuda(), torch.tensor([c for c, _ in reqs], dtype=torch.int32).cuda()
    parents = [tree(n, gen, near_root) for n in rows]
    mask = torch.cat([words_of(sees_of(p), 1) for p in parents]).cuda()
    normal = lambda *s: torch.randn(s, generator=gen).cuda()  # noqa: E731
    embed, head = normal(V, (H_q + 2 * H_kv) * D).to(dtype), normal(H_q * D, V)
    draft = torch.randint(0, V, (N,), generator=gen, dtype=torch.int32).cuda()
    turn = torch.arange(200, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    table = torch.cat([turn.cos(), turn.sin()], 1).float().cuda()
    k, v = (normal(n_pages, H_kv, P, D).to(dtype) for _ in "kv")
    k0, v0 = k.clone(), v.clone()

    def forward(tokens, k, v, ctx, cu, mask=None):
        x = embed[tokens.long()]
        q, kn, vn = (x[:, a * D:b * D].unflatten(1, (-1, D)) for a, b in ((0, H_q), (H_q, H_q + H_kv), (H_q + H_kv, H_q + 2 * H_kv)))
        q = fsr.kv_append_rope(q, kn, vn, table, k, v, bt, ctx, cu, tree_mask=mask)
        if mask is None:
            mask = torch.cat([words_of(torch.ones(n, n, dtype=torch.bool).tril(), 1) for n in cu.diff().tolist()]).cuda()
        out, _ = fsr.verify_attention_tree(q, k, v, bt, ctx, cu, mask, scale=D ** -0.5, out_dtype=F32)
        return out.flatten(1) @ head

    first = forward(draft, k, v, ctx, cu_d, mask)
    # the target agrees with some child at most rows: the logits are pushed towards it
    for i, p in enumerate(parents):
        for j, of in enumerate(p):
            if of >= 0 and j % 3:
                first[int(cu[i]) + of, draft[int(cu[i]) + j].long()] += 1000.0 + j
    logprobs, entropy, top, top_lp = fsr.token_logprobs(first, draft, top_k=3)
    exact = torch.log_softmax(first.double(), 1)
    assert torch.equal(top[:, 0].long(), first.argmax(1)) and (logprobs - exact.gather(1, draft.long()[:, None])[:, 0]).abs().max() < 1e-2
    target = top[:, 0].contiguous()
    keep = torch.empty(N, dtype=torch.uint8, device="cuda")
    acc, nem, emitted, path = fsr.tree_accept(target, draft, mask, cu_d, S_max=S_max, keep_mask=keep)
    assert acc.max() >= longest and int(keep.sum()) == int(nem.sum())
    packed = fsr.prune_compact(keep, cu_d, suffix_close=False, payload=first)
    fsr.kv_commit(k, v, bt, ctx, acc, path)
    torch.cuda.synchronize()

    # the path as a chain, from the caches as they were
    chain = torch.cat([draft[int(cu[i]) + path[i, :int(nem[i])].long()] for i in range(len(reqs))])
    assert torch.equal(packed["new_cu_q"].cpu(), offsets(nem.tolist()))
    plain = forward(chain, k0, v0, ctx, packed["new_cu_q"])
    torch.cuda.synchronize()
    for i, (c, _) in enumerate(reqs):
        s = slots(bt[i].cpu(), c + int(nem[i]), P).cuda()
        for a, b in ((k, k0), (v, v0)):
            assert torch.equal(a.transpose(1, 2).flatten(0, 1)[s], b.transpose(1, 2).flatten(0, 1)[s])
    # (the same keys in another order of sums, weights rounded as pairs: 2^-15 of values of about one through 512 products of about one)
    kept = packed["payload"][:len(chain)]
    assert (torch.where(kept > 500, kept.remainder(1.0) * 0, kept - plain).abs() < 512 * 6 * 2.0 ** -12).all()


def test_replays(fsr):
    announce("tree accept and commit, graph")
    t = Trees(7, [20, 33, 1, 64], tokens=2)
    p = Paths(4, [(9, n) for n in t.rows], 2, 64, 16, BF, False, 6)
    target, draft, mask, cu = t.target.cuda(), t.draft.cuda(), t.mask.cuda(), t.cu.cuda()
    k, v, bt, ctx = p.k.cuda(), p.v.cuda(), p.bt.cuda(), p.ctx.cuda()
    res = fsr.tree_accept(target, draft, mask, cu, S_max=6)

    def call():
        fsr.tree_accept(target, draft, mask, cu, S_max=6, accepted_len=res[0], n_emitted=res[1], emitted=res[2], path=res[3])
        fsr.kv_commit(k, v, bt, ctx, res[0], res[3])
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(3):
        new = torch.randint(0, 2, target.shape, generator=torch.Generator().manual_seed(seed), dtype=torch.int32)
        t.target = new
        target.copy_(new)
        k.copy_(p.k)
        v.copy_(p.v)
        graph.replay()
        torch.cuda.synchronize()
        acc, emitted, path = t.want(6)
        assert res[0].tolist() == acc and res[2].tolist() == emitted and res[3].tolist() == path
        p.acc, p.path = torch.tensor(acc, dtype=torch.int32), torch.tensor(path, dtype=torch.int32)
        want = p.want()
        assert torch.equal(k.cpu(), want[0]) and torch.equal(v.cpu(), want[1])
