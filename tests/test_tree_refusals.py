"""What the calls on trees of drafts and log probabilities refuse, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2604_20503_amd import binding as b

ONE, ODD = ctypes.c_void_p(256), ctypes.c_void_p(264)  # never read: the checks come first
BIG, NO = ctypes.c_size_t(1 << 40), ctypes.c_size_t(0)


@pytest.fixture(scope="module")
def lib():
    return b.load_library()


def rope(**kw):
    return b.RopeParams(**{**dict(B=2, N_cap=8, H_q=32, H_kv=8, D=128, R=128, P=16, max_pages=4, n_pages=16, T=100, tree_words=1, pairs=0, dtype=1, kv_layout=0,
                                  q_stride=4096, k_stride=1024, v_stride=1024, reserved=0), **kw})


def attn(**kw):
    return b.AttnParams(**{**dict(B=2, N_cap=8, H_q=32, H_kv=8, D=128, P=16, max_pages=4, n_pages=16, dtype=1, out_dtype=1, scale=0.1, max_q_len=0,
                                  max_workgroups=0, kv_layout=0), **kw})


def accept(**kw):
    return b.TreeParams(**{**dict(B=2, N_cap=8, tree_words=1, S_max=4, reserved=0), **kw})


def commit(**kw):
    return b.CommitParams(**{**dict(B=2, H_kv=8, row_bytes=256, P=16, max_pages=4, n_pages=16, S_max=4, kv_layout=0), **kw})


def logprob(**kw):
    return b.LogprobParams(**{**dict(N_cap=8, V=1000, M=1, K=5, dtype=1, reserved=0, stride=1000, temperature=1.0), **kw})


def call(lib, kind, p, args=None, ws=(ONE, BIG)):
    r = ctypes.byref(p)
    n = dict(rope=12, rope8=14, tree=8, accept=9, commit=6, logprob=7)[kind]
    a = [ONE] * n if args is None else args
    if kind == "rope":
        return lib.fsr_kv_append_rope(*a, r, None)
    if kind == "rope8":
        return lib.fsr_kv_append_rope_kv8(*a, r, None)
    if kind == "tree":
        return lib.fsr_verify_attention_tree(*a[:7], 1, a[7], None, r, *ws, None)
    if kind == "accept":
        return lib.fsr_tree_accept(*a, r, None)
    if kind == "commit":
        return lib.fsr_kv_commit(*a, r, None)
    return lib.fsr_token_logprobs(*a, r, *ws, None)


ROPE = [ONE] * 4 + [None, None] + [ONE] * 6
ROPE8 = [ONE] * 4 + [None, None] + [ONE] * 8


def test_struct_sizes():
    assert ctypes.sizeof(b.RopeParams) == 14 * 4 + 4 * 8 and ctypes.sizeof(b.TreeParams) == 20 and ctypes.sizeof(b.CommitParams) == 32
    assert ctypes.sizeof(b.LogprobParams) == 40 and b.LogprobParams.stride.offset == 24


@pytest.mark.parametrize("change,code", [(dict(B=-1), -1), (dict(H_q=0), -1), (dict(T=0), -1), (dict(P=0), -1), (dict(n_pages=0), -1), (dict(dtype=2), -3), (dict(kv_layout=2), -1),
                                         (dict(pairs=2), -1), (dict(reserved=1), -1), (dict(R=0), -2), (dict(R=144), -2), (dict(R=8), -3), (dict(R=120), -3),
                                         (dict(D=132, R=64, q_stride=132 * 32, k_stride=132 * 8, v_stride=132 * 8), -3), (dict(q_stride=4095), -2), (dict(k_stride=1000), -2),
                                         (dict(v_stride=0), -2), (dict(q_stride=4097), -1), (dict(v_stride=1025), -1)])
def test_rope_shapes(lib, change, code):
    assert call(lib, "rope", rope(**change), ROPE) == code
    assert call(lib, "rope8", rope(**change), ROPE8) == code


def test_rope_pointers(lib):
    for k in range(12):
        if k not in (4, 5):
            assert call(lib, "rope", rope(), [None if i == k else x for i, x in enumerate(ROPE)]) == -1
        if k in (0, 1, 2, 3, 6, 7, 8):
            assert call(lib, "rope", rope(), [ODD if i == k else x for i, x in enumerate(ROPE)]) == -1
    for k in range(14):
        if k not in (4, 5):
            assert call(lib, "rope8", rope(), [None if i == k else x for i, x in enumerate(ROPE8)]) == -1
    assert call(lib, "rope", rope()) == -1 and b"exclude" in lib.fsr_last_error()  # positions and a mask
    for words in (0, 17):
        assert call(lib, "rope", rope(tree_words=words), [ONE] * 4 + [None, ONE] + [ONE] * 6) == -1
    assert call(lib, "rope", rope(q_stride=8192), ROPE) == -1 and b"the same" in lib.fsr_last_error()  # in place, but apart
    assert call(lib, "rope8", rope(dtype=0), ROPE8) == -3
    assert call(lib, "rope8", rope(D=72, R=16), ROPE8) == -3  # 8-bit rows of 72 bytes
    assert lib.fsr_kv_append_rope(*ROPE, None, None) == -1
    for empty in (dict(B=0), dict(N_cap=0)):
        assert call(lib, "rope", rope(**empty), [None] * 12) == 0 and call(lib, "rope8", rope(**empty), [None] * 14) == 0


@pytest.mark.parametrize("change,code", [(dict(H_kv=5), -2), (dict(D=96), -3), (dict(dtype=2), -3), (dict(dtype=0, out_dtype=1), -3), (dict(scale=0.0), -1), (dict(scale=float("inf")), -1),
                                         (dict(kv_layout=2), -1), (dict(P=0), -1), (dict(max_pages=1 << 28), -3), (dict(n_pages=1 << 27), -3), (dict(N_cap=1 << 26), -3),
                                         (dict(max_q_len=-1), -1), (dict(max_workgroups=-1), -1), (dict(B=70000), -3)])
def test_tree_shapes(lib, change, code):
    out = ctypes.c_size_t(0)
    assert lib.fsr_tree_workspace_bytes(ctypes.byref(attn(**change)), ctypes.byref(out)) == code
    assert call(lib, "tree", attn(**change)) == code


def test_tree_pointers(lib):
    for k in range(8):
        assert call(lib, "tree", attn(), [None if i == k else ONE for i in range(8)]) == -1
    for k in (0, 1, 2, 7):
        assert call(lib, "tree", attn(), [ODD if i == k else ONE for i in range(8)]) == -1
    for words in (0, -1, 17):
        assert lib.fsr_verify_attention_tree(*[ONE] * 7, words, ONE, None, ctypes.byref(attn()), ONE, BIG, None) == -1
    for ws in ((None, BIG), (ONE, NO), (ctypes.c_void_p(128), BIG)):
        assert call(lib, "tree", attn(), ws=ws) == -4
    assert call(lib, "tree", attn(B=0), [None] * 8, (None, NO)) == 0 and call(lib, "tree", attn(N_cap=0), [None] * 8, (None, NO)) == 0
    out, sizes = ctypes.c_size_t(0), []
    assert lib.fsr_tree_workspace_bytes(None, ctypes.byref(out)) == -1 and lib.fsr_tree_workspace_bytes(ctypes.byref(attn()), None) == -1
    for n in (1, 2, 7, 8, 100, 5000):
        assert lib.fsr_tree_workspace_bytes(ctypes.byref(attn(N_cap=n)), ctypes.byref(out)) == 0
        sizes.append(out.value)
    assert sizes == sorted(sizes) and sizes[0] > 0


def test_accept_and_commit(lib):
    for change, code in ((dict(B=-1), -1), (dict(N_cap=-1), -1), (dict(S_max=-1), -1), (dict(reserved=1), -1), (dict(tree_words=0), -1), (dict(tree_words=17), -1), (dict(B=1 << 26), -3)):
        assert call(lib, "accept", accept(**change)) == code
    for k in range(8):
        assert call(lib, "accept", accept(), [None if i == k else ONE for i in range(9)]) == -1
    assert call(lib, "accept", accept(B=0), [None] * 9) == 0 and lib.fsr_tree_accept(*[ONE] * 9, None, None) == -1
    for change, code in ((dict(B=-1), -1), (dict(H_kv=0), -1), (dict(row_bytes=0), -1), (dict(row_bytes=72), -3), (dict(P=0), -1), (dict(S_max=-1), -1), (dict(kv_layout=2), -1),
                         (dict(n_pages=0), -1), (dict(B=1 << 28), -3)):
        assert call(lib, "commit", commit(**change)) == code
    for k in range(6):
        assert call(lib, "commit", commit(), [None if i == k else ONE for i in range(6)]) == -1
    assert call(lib, "commit", commit(), [ODD] + [ONE] * 5) == -1 and lib.fsr_kv_commit(*[ONE] * 6, None, None) == -1
    for empty in (dict(B=0), dict(S_max=0)):
        assert call(lib, "commit", commit(**empty), [None] * 6) == 0


def test_logprobs(lib):
    out, nan = ctypes.c_size_t(0), float("nan")
    for change, code in ((dict(N_cap=-1), -1), (dict(V=0), -1), (dict(M=-1), -1), (dict(K=-1), -1), (dict(reserved=1), -1), (dict(dtype=2), -3), (dict(K=65), -3), (dict(V=4, K=5), -2),
                         (dict(stride=999), -2), (dict(temperature=0.0), -1), (dict(temperature=nan), -1), (dict(temperature=1e7), -1), (dict(temperature=-1.0), -1), (dict(N_cap=1 << 23), -3)):
        assert call(lib, "logprob", logprob(**change)) == code
        assert lib.fsr_logprob_workspace_bytes(ctypes.byref(logprob(**change)), ctypes.byref(out)) == code
    for k in (0, 2, 3, 5, 6):
        assert call(lib, "logprob", logprob(), [None if i == k else ONE for i in range(7)]) == -1
    assert call(lib, "logprob", logprob(), [ctypes.c_void_p(257)] + [ONE] * 6) == -1 and call(lib, "logprob", logprob(dtype=0), [ctypes.c_void_p(258)] + [ONE] * 6) == -1
    for ws in ((None, BIG), (ONE, NO), (ctypes.c_void_p(128), BIG)):
        assert call(lib, "logprob", logprob(), ws=ws) == -4
    assert call(lib, "logprob", logprob(N_cap=0), [None] * 7, (None, NO)) == 0
    assert lib.fsr_logprob_workspace_bytes(None, ctypes.byref(out)) == -1 and lib.fsr_logprob_workspace_bytes(ctypes.byref(logprob()), None) == -1
    for V in (100, 128256):
        sizes = []
        for n in (1, 2, 3, 10, 60, 200, 1000, 5000, 100000):  # a size covers every smaller call
            assert lib.fsr_logprob_workspace_bytes(ctypes.byref(logprob(N_cap=n, V=V, stride=V)), ctypes.byref(out)) == 0
            sizes.append(out.value)
        assert sizes == sorted(sizes) and sizes[0] > 0


def test_binding_refuses_what_does_not_fit():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    bt, ctx, cu, mask = i32(2, 3), i32(2), i32(3), torch.zeros(4, 1, dtype=torch.int64)
    q, kn, cache, table = torch.zeros(4, 8, 128), torch.zeros(4, 2, 128), torch.zeros(6, 2, 16, 128), torch.zeros(50, 128)
    for bad in (dict(q=q[:, :, :64]), dict(kn=kn[:3]), dict(cache=cache.bfloat16()), dict(table=table[0]), dict(bt=bt[:1]), dict(cu=cu[:2]), dict(positions=i32(3)), dict(tree_mask=mask[:3]),
                dict(tree_mask=torch.zeros(4, 17, dtype=torch.int64)), dict(q_out=q[:3]), dict(q_out=q.bfloat16()), dict(k_scale=torch.ones(2)),
                dict(k_scale=torch.ones(2), v_scale=torch.ones(2)), dict(q=torch.zeros(4, 128, 8).transpose(1, 2)), dict()):
        x = {**dict(q=q, kn=kn, cache=cache, table=table, bt=bt, cu=cu), **bad}
        rest = {k: v for k, v in x.items() if k in ("positions", "tree_mask", "q_out", "k_scale", "v_scale")}
        with pytest.raises(ValueError):  # the last one: everything fits, but lives on the CPU
            b.kv_append_rope(x["q"], x["kn"], x["kn"], x["table"], x["cache"], x["cache"], x["bt"], ctx, x["cu"], **rest)
    for bad in (dict(q=q.bfloat16()), dict(mask=mask[:3]), dict(cu=cu[:2]), dict(mask=torch.zeros(4, 0, dtype=torch.int64)), dict()):
        x = {**dict(q=q, mask=mask, cu=cu), **bad}
        with pytest.raises(ValueError):
            b.verify_attention_tree(x["q"], cache, cache, bt, ctx, x["cu"], x["mask"], scale=1.0)
    for bad in (dict(draft=i32(3)), dict(mask=mask[:3]), dict(S_max=-1), dict(path=i32(2, 4)), dict(keep_mask=torch.zeros(3, dtype=torch.uint8)), dict()):
        x = {**dict(draft=i32(4), mask=mask, S_max=4), **bad}
        with pytest.raises(ValueError):
            b.tree_accept(i32(4), x.pop("draft"), x.pop("mask"), cu, **x)
    for bad in (dict(v=cache.bfloat16()), dict(acc=i32(3)), dict(path=i32(3, 5)), dict(path=i32(2, 0)), dict(bt=bt[:1]), dict()):
        x = {**dict(v=cache, acc=i32(2), path=i32(2, 5), bt=bt), **bad}
        with pytest.raises(ValueError):
            b.kv_commit(cache, x["v"], x["bt"], ctx, x["acc"], x["path"])
    z = torch.zeros(4, 100)
    for bad in (dict(z=z[0]), dict(tokens=i32(3)), dict(n_rows=i32(2)), dict(top_ids=i32(4, 4)), dict(z=z.half()), dict(z=torch.zeros(100, 4).T), dict()):
        x = {**dict(z=z, tokens=i32(4)), **bad}
        with pytest.raises(ValueError):
            b.token_logprobs(x.pop("z"), x.pop("tokens"), top_k=5, **x)


def test_call_ids_are_no_bytes_of_other_tensors(lib):
    """What tells a call's arrivals from whatever a workspace held before (the word's upper 48 bits) is met by no bytes of masks, no indexes
    and no counts, from a process's first call on."""
    next_id = lib._ZN3fsr12next_call_idEv
    next_id.restype, next_id.argtypes = ctypes.c_ulonglong, []
    ids = [next_id() for _ in range(300)]
    assert len(set(ids)) == 300 and all(0 < i < 1 << 48 for i in ids)
    for i in ids:
        word = i << 16
        tail = word.to_bytes(8, "little")[2:]  # (the count is below)
        assert any(x > 1 for x in tail), "a mask's bytes"
        assert word >= 1 << 62, "64-bit indexes"
        assert abs(float(torch.tensor([(i >> 32) - (1 << 16)], dtype=torch.int16).view(torch.bfloat16))) > 1e30, "floats, bf16"
