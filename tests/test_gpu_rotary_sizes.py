"""Rotary calls of many tokens and of few take different numbers of heads a thread (bf16): the same bits either way, and those of 64-bit arithmetic
within a rounding."""
import pytest
import torch

import _paged as R
from paper_2409_09086_amd import binding as B
from test_gpu_paged import DEV, gen, randn, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,layout,dims", [(128, "half", 128), (128, "interleaved", 96), (64, "half", 48), (64, "interleaved", 64)])
@pytest.mark.parametrize("norm", [False, True])
def test_many_tokens_as_few(dtype, d, layout, dims, norm):
    print("sizes", dtype, d, layout, dims, norm, flush=True)
    n, heads, kv, dt, g = 4133, 17, 3, R.DT[dtype], gen(d + dims)
    rot = B.Rotary(d, 8192, dtype=dt, dims=dims, layout=layout, norm_eps=1e-6)
    x = randn(g, n, heads + kv, d, dtype=dt)
    w = (torch.rand(d, generator=g) + 0.5).to(dt) if norm else None
    wd, xd = (None if w is None else w.to(DEV)), x.to(DEV)
    pos = torch.randint(0, 8192, (n,), generator=g).to(torch.int32)
    q, k = rot.apply(pos.to(DEV), xd[:, :heads], xd[:, heads:], q_weight=wd, k_weight=wd)
    for a, b in ((0, 1), (1, 100), (4000, 4133)):
        qs, ks = rot.apply(pos[a:b].to(DEV), xd[a:b, :heads], xd[a:b, heads:], q_weight=wd, k_weight=wd)
        assert torch.equal(qs, q[a:b]) and torch.equal(ks, k[a:b]), (a, b)
    rows = torch.arange(0, n, 37)
    want = R.rotate(x[rows], pos[rows], R.frequencies(dims, 10000.0), layout, w)
    within(torch.cat([q, k], 1)[rows.to(DEV)], want, R.rotate_bound(want, dt, norm) + 1e-10, "rows")
