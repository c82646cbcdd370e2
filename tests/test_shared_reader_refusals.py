"""What the calls over caches with several readers refuse, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2604_20503_amd import binding as b

ONE = ctypes.c_void_p(256)  # never read: the checks come first


@pytest.fixture(scope="module")
def lib():
    return b.load_library()


def latent(**kw):
    return b.LatentParams(**{**dict(B=2, N_cap=8, H=16, D_latent=512, D_rope=64, P=16, max_pages=4, n_pages=16, dtype=1, out_dtype=1, scale=0.1,
                                    max_q_len=0, max_workgroups=0, reserved=0), **kw})


def expanded(**kw):
    return b.ExpandedParams(**{**dict(B=2, N_cap=8, T_cap=64, H=16, D_nope=128, D_rope=64, D_v=128, dtype=1, out_dtype=1, scale=0.1, max_q_len=0,
                                      max_workgroups=0, reserved=0), **kw})


def shared(**kw):
    return b.AttnParams(**{**dict(B=2, N_cap=8, H_q=32, H_kv=8, D=128, P=16, max_pages=4, n_pages=16, dtype=1, out_dtype=1, scale=0.1, max_q_len=0,
                                  max_workgroups=0, kv_layout=0), **kw})


def test_struct_sizes():
    assert ctypes.sizeof(b.LatentParams) == 14 * 4 and ctypes.sizeof(b.ExpandedParams) == 13 * 4


@pytest.mark.parametrize("make,size_of", [(latent, "fsr_latent_workspace_bytes"), (expanded, "fsr_expanded_workspace_bytes"), (shared, "fsr_shared_workspace_bytes")])
def test_workspace_sizes(lib, make, size_of):
    out = ctypes.c_size_t(0)
    f = getattr(lib, size_of)
    assert f(None, ctypes.byref(out)) == -1 and f(ctypes.byref(make()), None) == -1
    sizes = []
    for n in (1, 2, 7, 8, 100, 1000, 5000):  # a size covers every smaller call
        assert f(ctypes.byref(make(N_cap=n)), ctypes.byref(out)) == 0
        sizes.append(out.value)
    assert sizes == sorted(sizes) and sizes[0] > 0


@pytest.mark.parametrize("change,code", [(dict(D_latent=384), -3), (dict(D_rope=48), -3), (dict(dtype=2), -3), (dict(dtype=0, out_dtype=1), -3), (dict(scale=0.0), -1),
                                         (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(H=0), -1), (dict(B=-1), -1), (dict(P=0), -1),
                                         (dict(n_pages=0), -1), (dict(max_q_len=-1), -1), (dict(max_workgroups=-1), -1), (dict(reserved=1), -1), (dict(B=70000), -3),
                                         (dict(max_pages=1 << 28), -3), (dict(n_pages=1 << 30), -3), (dict(D_latent=4), -3)])
def test_latent_shapes(lib, change, code):
    out = ctypes.c_size_t(0)
    assert lib.fsr_latent_workspace_bytes(ctypes.byref(latent(**change)), ctypes.byref(out)) == code
    assert lib.fsr_latent_attention(ONE, ONE, ONE, ONE, ONE, ONE, None, ctypes.byref(latent(**change)), ONE, ctypes.c_size_t(1 << 40), None) == code


def test_latent_pointers(lib):
    p, big = latent(), ctypes.c_size_t(1 << 40)
    for k in range(6):
        args = [ONE] * 6
        args[k] = None
        assert lib.fsr_latent_attention(*args, None, ctypes.byref(p), ONE, big, None) == -1
        args = [ONE] * 6
        args[k] = None
        assert lib.fsr_latent_append(*args, ctypes.byref(p), None) == -1
    for k in range(5):
        args = [ONE] * 5
        args[k] = None
        assert lib.fsr_latent_gather(*args, ctypes.byref(p), None) == -1
    assert lib.fsr_latent_attention(*[ONE] * 6, None, ctypes.byref(p), None, big, None) == -4
    assert lib.fsr_latent_attention(*[ONE] * 6, None, ctypes.byref(p), ONE, ctypes.c_size_t(64), None) == -4
    assert lib.fsr_latent_attention(*[ONE] * 6, None, ctypes.byref(p), ctypes.c_void_p(128), big, None) == -4
    odd = ctypes.c_void_p(264)
    assert lib.fsr_latent_attention(odd, *[ONE] * 5, None, ctypes.byref(p), ONE, big, None) == -1
    assert lib.fsr_latent_append(odd, *[ONE] * 5, ctypes.byref(p), None) == -1
    assert lib.fsr_latent_gather(odd, *[ONE] * 4, ctypes.byref(p), None) == -1
    assert lib.fsr_latent_append(*[ONE] * 6, ctypes.byref(latent(D_rope=4)), None) == -3  # 8 bytes: no whole piece
    assert lib.fsr_latent_append(*[ONE] * 6, None, None) == -1
    for empty in (dict(B=0), dict(N_cap=0)):  # nothing to do is no error, and looks at no pointer
        q = latent(**empty)
        assert lib.fsr_latent_attention(*[None] * 7, ctypes.byref(q), None, ctypes.c_size_t(0), None) == 0
        assert lib.fsr_latent_append(*[None] * 6, ctypes.byref(q), None) == 0
        assert lib.fsr_latent_gather(*[None] * 5, ctypes.byref(q), None) == 0


@pytest.mark.parametrize("change,code", [(dict(D_nope=96), -3), (dict(D_v=64), -3), (dict(dtype=2), -3), (dict(dtype=0, out_dtype=1), -3), (dict(scale=-1.0), -1), (dict(H=0), -1),
                                         (dict(T_cap=-1), -1), (dict(reserved=1), -1), (dict(N_cap=(1 << 30) + 1), -3), (dict(H=70000), -3)])
def test_expanded_shapes(lib, change, code):
    assert lib.fsr_latent_attention_expanded(*[ONE] * 6, None, ctypes.byref(expanded(**change)), ONE, ctypes.c_size_t(1 << 40), None) == code


def test_expanded_pointers(lib):
    p, big = expanded(), ctypes.c_size_t(1 << 40)
    for k in range(6):
        args = [ONE] * 6
        args[k] = None
        assert lib.fsr_latent_attention_expanded(*args, None, ctypes.byref(p), ONE, big, None) == -1
    assert lib.fsr_latent_attention_expanded(*[ONE] * 6, None, ctypes.byref(p), None, big, None) == -4
    assert lib.fsr_latent_attention_expanded(*[None] * 7, ctypes.byref(expanded(N_cap=0)), None, ctypes.c_size_t(0), None) == 0


@pytest.mark.parametrize("change,code", [(dict(H_kv=5), -2), (dict(D=96), -3), (dict(dtype=2), -3), (dict(dtype=0, out_dtype=1), -3), (dict(scale=0.0), -1), (dict(kv_layout=2), -1),
                                         (dict(P=0), -1), (dict(max_pages=1 << 28), -3), (dict(n_pages=1 << 27), -3), (dict(N_cap=1 << 26), -3)])
def test_shared_shapes(lib, change, code):
    args = [ONE] * 8 + [2, ONE, None, ctypes.byref(shared(**change)), ONE, ctypes.c_size_t(1 << 40), None]
    assert lib.fsr_verify_attention_shared(*args) == code


def test_shared_pointers(lib):
    p, big = shared(), ctypes.c_size_t(1 << 40)
    for k in range(9):
        args = [ONE] * 9
        args[k] = None
        assert lib.fsr_verify_attention_shared(*args[:8], 2, args[8], None, ctypes.byref(p), ONE, big, None) == -1
    assert lib.fsr_verify_attention_shared(*[ONE] * 8, 2, ONE, None, ctypes.byref(p), ONE, ctypes.c_size_t(0), None) == -4
    assert lib.fsr_verify_attention_shared(*[ONE] * 8, 70000, ONE, None, ctypes.byref(p), ONE, big, None) == -3
    assert lib.fsr_verify_attention_shared(*[ONE] * 8, -1, ONE, None, ctypes.byref(p), ONE, big, None) == -1
    assert lib.fsr_verify_attention_shared(*[None] * 8, 0, None, None, ctypes.byref(p), None, ctypes.c_size_t(0), None) == 0  # no group: no rows


def test_binding_refuses_what_does_not_fit():
    q, cache = torch.zeros(4, 8, 576, dtype=torch.bfloat16), torch.zeros(6, 16, 576, dtype=torch.bfloat16)
    bt, ctx, cu = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    ok = dict(scale=0.1, D_latent=512)
    for bad in (dict(q=q[:, :, :512]), dict(cache=cache.float()), dict(bt=bt[:1]), dict(cu=cu[:2]), dict(D_latent=576), dict(D_latent=0),
                dict(out=torch.zeros(4, 8, 576, dtype=torch.bfloat16)), dict(lse=torch.zeros(4, 9)), dict(workspace=torch.zeros(256, dtype=torch.uint8))):
        x = {**dict(q=q, cache=cache, bt=bt, ctx=ctx, cu=cu), **ok, **bad}
        with pytest.raises(ValueError):  # the last one: everything fits, but lives on the CPU
            b.latent_attention(x.pop("q"), x.pop("cache"), x.pop("bt"), x.pop("ctx"), x.pop("cu"), **x)
    with pytest.raises(ValueError):
        b.latent_append(q[:, 0, :512].contiguous(), q[:3, 0, 512:].contiguous(), cache, bt, ctx, cu)
    with pytest.raises(ValueError):
        b.latent_append(q[:, 0, :512].contiguous(), q[:, 0, 512:].float().contiguous(), cache, bt, ctx, cu)
    with pytest.raises(ValueError):
        b.latent_gather(cache, bt, cu, T_cap=8, D_latent=512, latent=torch.zeros(8, 511, dtype=torch.bfloat16))
    qe, kv, rope = torch.zeros(4, 2, 192), torch.zeros(9, 2, 256), torch.zeros(9, 64)
    for bad in (dict(kv=kv[:, :1]), dict(rope=rope[:5]), dict(kv=kv.bfloat16()), dict(rope=torch.zeros(9, 192)), dict(cu_k=cu[:2])):
        x = {**dict(q=qe, kv=kv, rope=rope, cu_q=cu, cu_k=cu), **bad}
        with pytest.raises(ValueError):
            b.latent_attention_expanded(x["q"], x["kv"], x["rope"], x["cu_q"], x["cu_k"], scale=1.0)
    qs, k = torch.zeros(4, 8, 128), torch.zeros(6, 2, 16, 128)
    for bad in (dict(k=k.bfloat16()), dict(groups=cu), dict(bt=bt[:1])):
        x = {**dict(k=k, groups=torch.zeros(2, dtype=torch.int32), bt=bt), **bad}
        with pytest.raises(ValueError):
            b.verify_attention_shared(qs, x["k"], k, x["bt"], ctx, cu, x["groups"], torch.zeros(1, dtype=torch.int32), scale=1.0)


def test_tensors_of_another_device_are_refused(monkeypatch):
    class Elsewhere:
        is_cuda, device = True, torch.device("cuda:1")
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    with pytest.raises(ValueError, match="current device"):
        b._on_current_device(q=Elsewhere())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    b._on_current_device(q=Elsewhere(), out=None)
