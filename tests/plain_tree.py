"""Trees of drafted tokens in plain form, for the tests of the calls on them: masks out of parents, attention under any mask in 64 bits
(its error bound as in plain_attention), the walk of an acceptance, and the rotation of heads."""
import torch

from plain_attention import U, attend


def tree(n, gen, near_root=1.6):
    """Parents of n rows (row 0: -1), each in front of its children."""
    return [-1][:n] + [min(int(j * float(torch.rand((), generator=gen)) ** near_root), j - 1) for j in range(1, n)]


def sees_of(parents, n=None):
    """[n, n] bool: row j sees its ancestors and itself."""
    n = len(parents) if n is None else n
    sees = torch.zeros(n, n, dtype=torch.bool)
    for j, p in enumerate(parents):
        if p >= 0:
            sees[j] = sees[p]
        sees[j, j] = True
    return sees


def words_of(sees, words):
    """[n, words] int64 out of [n, n] bool; rows that have no bit are dropped."""
    n = sees.shape[0]
    bits = torch.zeros(n, 64 * words, dtype=torch.int64)
    m = min(sees.shape[1], 64 * words)
    bits[:, :m] = sees[:, :m].long()
    weight = torch.ones(64, dtype=torch.int64) << torch.arange(64)
    return (bits.view(n, words, 64) * weight).sum(2)


def attend_masked(q, k, v, scale, seen):
    """q [n, D], k [L, D], v [L, Dv], seen [n, L] bool -> o, lse, A, e as plain_attention.attend."""
    n = q.shape[0]
    o, A = torch.zeros(n, v.shape[1], dtype=torch.float64), torch.zeros(n, v.shape[1], dtype=torch.float64)
    lse, e = torch.full((n,), float("-inf"), dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
    for r in range(n):
        s = seen[r].nonzero()[:, 0]
        if len(s):
            x = attend(q[r:r + 1], k[s], v[s], scale, [len(s) - 1])
            o[r], lse[r], A[r], e[r] = (y[0] for y in x)
    return o, lse, A, e


def walk(parents, draft, target, S_max):
    """Path and emitted tokens of one request."""
    if not parents:
        return [], []
    path = [0]
    while len(path) <= S_max:
        child = [c for c in range(1, len(parents)) if parents[c] == path[-1] and draft[c] == target[path[-1]]]
        if not child:
            break
        path.append(child[0])
    return path, [target[j] for j in path]


def rotate(x, cos_sin, R, pairs):
    """x [n, H, D], cos_sin [n, R] in any type.  Returns the result in 64 bits and |a cos| + |b sin| (elementwise), of which fp32
    arithmetic is off by 3 u at most: two products and a sum, each rounded."""
    x, t = x.double(), cos_sin.double()
    c, s = t[:, None, :R // 2], t[:, None, R // 2:]
    y, size = x.clone(), torch.zeros_like(x)
    first = slice(0, R, 2) if pairs else slice(0, R // 2)
    second = slice(1, R, 2) if pairs else slice(R // 2, R)
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    size[..., first], size[..., second] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
    return y, 3 * U * size
