"""Host-side checks of the rotary and paged-cache entry points that need no GPU: refusals with the documented codes."""
import ctypes

import pytest

from paper_2409_09086_amd import binding as B

ONE = ctypes.c_void_p(256)


def rotary(d=128, dtype=B.BF16, positions=1000):
    h = ctypes.c_void_p()
    return B.lib().infmllm_rotary_create(d, dtype, positions, ctypes.byref(h)), h


def paged(pages=8, page=16, heads=4, kv=2, d=64, dtype=B.BF16):
    h = ctypes.c_void_p()
    return B.lib().infmllm_paged_create(pages, page, heads, kv, d, dtype, ctypes.byref(h)), h


@pytest.mark.parametrize("args", [dict(d=96), dict(d=0), dict(dtype=3), dict(positions=0), dict(positions=-1), dict(positions=(1 << 24) + 1)])
def test_rotary_create_refuses(args):
    rc, h = rotary(**args)
    assert rc == B.EINVAL and not h.value and B.last_error()


@pytest.mark.parametrize("args", [dict(pages=0), dict(pages=(1 << 30) + 1), dict(page=8), dict(page=24), dict(page=2048), dict(heads=3), dict(heads=0),
                                  dict(kv=0), dict(kv=-2), dict(d=96), dict(dtype=2), dict(heads=1 << 17),
                                  dict(heads=8192, kv=1), dict(heads=16384, kv=16384, page=1024, d=128)])
def test_paged_create_refuses(args):
    rc, h = paged(**args)
    assert rc == B.EINVAL and not h.value and B.last_error()


def test_parameters_and_states():
    L = B.lib()
    assert L.infmllm_rotary_create(64, 0, 10, None) == B.EINVAL and L.infmllm_paged_create(8, 16, 4, 2, 64, 0, None) == B.EINVAL
    rc, r = rotary()
    assert rc == B.OK
    full = L.infmllm_rotary_workspace_bytes(r)
    assert full >= 1000 * 64 * 8
    for which, bad, ok in [(B.ROTARY_BASE, (1.0, 0.5, -1.0), (0.0, 500000.0)), (B.ROTARY_DIMS, (0.0, 8.0, 24.0, 130.0, 144.0, 16.5), (16.0, 112.0, 128.0)),
                           (B.ROTARY_LAYOUT, (-1.0, 2.0, 0.5), (0.0, 1.0)), (B.ROTARY_FACTOR, (0.0, 0.5, -2.0), (1.0, 8.0)),
                           (B.ROTARY_TRAINED, (-1.0,), (0.0, 4096.0)), (B.ROTARY_LOW, (-1.0,), (0.0, 1.0)), (B.ROTARY_HIGH, (0.0, -1.0), (1.0, 4.0)),
                           (B.ROTARY_MAGNITUDE, (0.0, -1.0), (1.5,)), (B.ROTARY_EPS, (-1e-6,), (0.0, 1e-5))]:
        for v in bad + (float("nan"), float("inf")):
            assert L.infmllm_rotary_set_param(r, which, v) == B.EINVAL, (which, v)
        for v in ok:
            assert L.infmllm_rotary_set_param(r, which, v) == B.OK, (which, v)
    assert L.infmllm_rotary_set_param(r, 99, 1.0) == B.EINVAL and L.infmllm_rotary_set_param(None, 0, 2.0) == B.EINVAL
    assert L.infmllm_rotary_set_param(r, B.ROTARY_DIMS, 32.0) == B.OK and L.infmllm_rotary_workspace_bytes(r) < full
    assert L.infmllm_rotary_apply(r, ONE, 1, 4, 2, ONE, 512, ONE, 256, None, None, ONE, 512, ONE, 256) == B.ESTATE
    assert L.infmllm_rotary_apply(None, ONE, 1, 4, 2, ONE, 512, ONE, 256, None, None, ONE, 512, ONE, 256) == B.EINVAL
    assert L.infmllm_rotary_attach(r, None, 1 << 30, None) == B.EINVAL
    assert L.infmllm_rotary_attach(r, ctypes.c_void_p(16), 1 << 30, None) == B.EINVAL
    assert L.infmllm_rotary_attach(r, ONE, 16, None) == B.ENOMEM
    assert L.infmllm_rotary_set_param(r, B.ROTARY_LOW, 4.0) == B.OK                     # low = high
    assert L.infmllm_rotary_attach(r, ONE, 1 << 30, None) == B.EINVAL
    rc, p = paged()
    assert rc == B.OK
    for which, bad, ok in [(B.PAGED_SCALE, (0.0, -1.0), (0.1,)), (B.PAGED_WINDOW, (-1.0, 1.5, 2.0 ** 31), (0.0, 1.0, 4096.0)),
                           (B.PAGED_KERNEL, (-1.0, 4.0, 0.5), (1.0, 2.0, 3.0, 0.0))]:
        for v in bad + (float("nan"), float("inf")):
            assert L.infmllm_paged_set_param(p, which, v) == B.EINVAL, (which, v)
        for v in ok:
            assert L.infmllm_paged_set_param(p, which, v) == B.OK, (which, v)
    assert L.infmllm_paged_set_param(p, 99, 1.0) == B.EINVAL and L.infmllm_paged_set_param(None, 0, 2.0) == B.EINVAL
    b = B._Batch(1, 1, 1, 1, 256, 256, 256, 1)
    ref = ctypes.byref(b)
    assert L.infmllm_paged_append(p, None, ref, ONE, 128, ONE, 128, None, None, 0, None, None, 0, ONE, ONE) == B.ESTATE
    assert L.infmllm_paged_attend(p, ref, ONE, 256, ONE, ONE, ONE, None) == B.ESTATE
    assert L.infmllm_paged_attend(None, ref, ONE, 256, ONE, ONE, ONE, None) == B.EINVAL
    assert L.infmllm_paged_attach(p, None, 1 << 30, None) == B.EINVAL
    assert L.infmllm_paged_attach(p, ctypes.c_void_p(8), 1 << 30, None) == B.EINVAL
    assert L.infmllm_paged_attach(p, ONE, 16, None) == B.ENOMEM
    assert L.infmllm_rotary_workspace_bytes(None) == 0 and L.infmllm_paged_workspace_bytes(None) == 0
    for f, h in ((L.infmllm_rotary_destroy, r), (L.infmllm_paged_destroy, p)):
        f(h)
        f(None)


@pytest.mark.gpu
def test_calls_of_attached_objects_refuse():
    """Every call is refused on the host, before any launch."""
    import torch
    L = B.lib()
    cache = B.PagedCache(8, 16, 4, 2, 64)
    rot, other, short = B.Rotary(64, 100), B.Rotary(64, 100, dtype=torch.float32), B.Rotary(64, 10)
    apply = lambda **k: L.infmllm_rotary_apply(*[k.get(n, v) for n, v in dict(
        r=rot._h, pos=ONE, tokens=4, heads=4, kv=2, q=ONE, qs=256, k=ONE, ks=128, qw=None, kw=None, qo=ONE, qos=256, ko=ONE, kos=128).items()])
    odd = ctypes.c_void_p(264)
    for bad in [dict(r=None), dict(pos=None), dict(pos=ctypes.c_void_p(258)), dict(tokens=-1), dict(heads=-1), dict(heads=0, kv=0), dict(heads=16385), dict(kv=1 << 20), dict(q=None), dict(k=None),
                dict(qo=None), dict(ko=None), dict(q=odd), dict(k=odd), dict(qo=odd), dict(qs=255), dict(qs=248), dict(ks=132), dict(kos=0),
                dict(qw=odd), dict(kw=odd)]:
        assert apply(**bad) == B.EINVAL, bad
    assert apply(tokens=0) == B.OK
    assert L.infmllm_rotary_set_param(rot._h, B.ROTARY_EPS, 0.1) == B.ESTATE and L.infmllm_paged_set_param(cache._h, B.PAGED_WINDOW, 1.0) == B.ESTATE
    assert L.infmllm_rotary_attach(rot._h, ONE, 1 << 30, None) == B.ESTATE and L.infmllm_paged_attach(cache._h, ONE, 1 << 30, None) == B.ESTATE

    def batch(**k):
        return ctypes.byref(B._Batch(*[k.get(n, v) for n, v in dict(seqs=1, tokens=2, max_new=2, max_len=20, starts=256, lens=256, table=256, per=2).items()]))

    def append(b=None, **k):
        return L.infmllm_paged_append(*[k.get(n, v) for n, v in dict(
            p=cache._h, r=rot._h, b=b or batch(), k=ONE, ks=128, v=ONE, vs=128, kw=None, q=ONE, qs=256, qw=None, qo=ONE, qos=256, K=ONE, V=ONE).items()])

    def attend(b=None, **k):
        return L.infmllm_paged_attend(*[k.get(n, v) for n, v in dict(
            p=cache._h, b=b or batch(), q=ONE, qs=256, K=ONE, V=ONE, out=ONE, lse=None).items()])
    for bad in [dict(seqs=0), dict(seqs=65537), dict(tokens=-1), dict(max_new=-1), dict(max_len=-1), dict(starts=None), dict(lens=None), dict(table=None),
                dict(table=258), dict(per=0)]:
        assert append(batch(**bad)) == B.EINVAL and attend(batch(**bad)) == B.EINVAL, bad
    assert append(batch(tokens=0)) == B.OK and attend(batch(tokens=0)) == B.OK
    for bad in [dict(p=None), dict(k=None), dict(v=None), dict(k=odd), dict(v=odd), dict(ks=64), dict(vs=130), dict(q=odd), dict(qo=None), dict(qos=128),
                dict(K=None), dict(V=None), dict(K=odd), dict(kw=odd), dict(qw=odd), dict(r=None), dict(r=other._h)]:
        assert append(**bad) == B.EINVAL, bad
    assert append(r=None, q=None, kw=ONE) == B.EINVAL and append(q=None, qw=ONE) == B.EINVAL
    assert append(r=short._h) == B.ECAPACITY
    for bad in [dict(p=None), dict(q=None), dict(q=odd), dict(qs=128), dict(qs=260), dict(K=None), dict(V=odd), dict(out=None), dict(out=odd),
                dict(lse=ctypes.c_void_p(258))]:
        assert attend(**bad) == B.EINVAL, bad


@pytest.mark.gpu
def test_binding_refuses_what_it_cannot_pass_on():
    import torch
    dev = "cuda:0"
    cache, rot = B.PagedCache(8, 16, 4, 2, 64), B.Rotary(64, 100)
    K, V = cache.pools()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=dev)
    b = B.PagedBatch(i32(0, 2), i32(5), i32(1).reshape(1, 1), 2, 2, 5)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device=dev)
    for bad in (q.float(), q[:1], q.cpu(), q.transpose(1, 2).contiguous().transpose(1, 2), q[:, :2]):
        with pytest.raises(ValueError):
            cache.attend(b, bad, K, V)
    with pytest.raises(ValueError):
        cache.attend(b, q, K[:7], V)
    with pytest.raises(ValueError):
        cache.attend(b, q, K, V, lse=torch.zeros((2, 4), dtype=torch.bfloat16, device=dev))
    with pytest.raises(ValueError):
        rot.apply(i32(1, 2).long(), q)
    with pytest.raises(ValueError):
        rot.apply(i32(1, 2), q, q_weight=torch.ones(64, device=dev))
    with pytest.raises(ValueError):
        B.PagedBatch(i32(0, 2), i32(5, 6), i32(1).reshape(1, 1), 2, 2, 5)
    with pytest.raises(ValueError):
        B.PagedBatch(torch.tensor([0, 2], dtype=torch.int32), torch.tensor([5], dtype=torch.int32), torch.ones((1, 1), dtype=torch.int32), 2, 2, 5)
    with pytest.raises(ValueError):
        B.Rotary(64, 100, layout="other")
    k = q[:, :2].contiguous()
    rot.close()
    with pytest.raises(ValueError):                            # not a cache without rotation by accident
        cache.append(b, k, k, K, V, rotary=rot)
    with pytest.raises(B.InfMLLMError):
        rot.apply(i32(1, 2), q)
    assert B.PagedCache(8, 16, 4, 2, 64, device="cuda").device == torch.device("cuda:0")
