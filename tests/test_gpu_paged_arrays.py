"""Batch arrays that do not describe sequences: calls with them touch nothing outside the pools and the outputs, and do the sequences beside
them as ever."""
import pytest
import torch

import _paged as R
from paper_2409_09086_amd import binding as B
from test_gpu_paged import DEV, TYPES, Case, within

pytestmark = pytest.mark.gpu
LOW, HIGH = -2 ** 31, 2 ** 31 - 1

STARTS = [
    [0, 40, 41, 200],              # an end past the tokens
    [0, 40, 41, HIGH],
    [0, 41, 40, 60],               # descending by one, the tokens of two sequences overlap
    [60, 40, 20, 0],
    [1, LOW, 41, 60],
    [5, LOW, LOW + 3, 60],
    [-9, 40, 41, 60],
    [HIGH, HIGH, 7, LOW],
    [61, 200, 1000, 1 << 24],
    [0, 0, 0, 0],
]


def guarded(shape, fill, dtype, pad):
    """A tensor of that shape in the middle of a larger one, and the larger one."""
    whole = torch.full((shape[0] + 2 * pad,) + tuple(shape[1:]), fill, dtype=dtype, device=DEV)
    return whole[pad:pad + shape[0]], whole


def rim(whole, pad, fill):
    return bool((whole[:pad] == fill).all()) and bool((whole[-pad:] == fill).all())


@pytest.mark.parametrize("dtype,kernel", TYPES)
@pytest.mark.parametrize("starts", STARTS)
def test_attend_stays_inside(dtype, kernel, starts):
    print("starts", dtype, kernel, starts, flush=True)
    c = Case(21, dtype, 8, 2, 64, 16, [(40, 150), (1, 60), (19, 333)])
    c.starts = torch.tensor(starts).to(torch.int32)
    pad = 64
    out, whole = guarded((60, 8, 64), 777.0, c.dtype, pad)
    lse, lwhole = guarded((60, 8), 777.0, torch.float32, pad)
    c.cache(kernel=kernel).attend(c.batch(), c.q.to(DEV).contiguous(), c.K.to(DEV), c.V.to(DEV), out=out, lse=lse)
    torch.cuda.synchronize()
    assert rim(whole, pad, 777) and rim(lwhole, pad, 777)
    lone = [s for s in range(3) if 0 <= starts[s] < starts[s + 1] and all(
        x == s or max(starts[x], starts[s], 0) >= min(starts[x + 1], starts[s + 1], 60) for x in range(3))]
    for s in lone:                                             # tokens that one sequence alone claims
        rows = slice(starts[s], min(starts[s + 1], 60))
        want, wlse, mass, absq = R.attend(c.q, c.K, c.V, c.starts[s:s + 2], c.lens[s:s + 1], c.table[s:s + 1])
        bo, bl = R.attend_bounds(want, wlse, mass, absq, c.dtype, c.d, dtype == "bf16")
        within(out[rows], want[rows], bo[rows], "out")
        within(lse[rows], wlse[rows], bl[rows], "lse")
    claimed = [t for t in range(60) if any(starts[s] <= t < starts[s + 1] for s in range(3))]
    free = [t for t in range(60) if t not in claimed]
    assert (out[free] == 777).all() and (lse[free] == 777).all()


@pytest.mark.parametrize("kernel", [0, 1, 2, 3])
def test_attend_stays_inside_with_many_sequences(kernel):
    """More sequences than lanes, every third with ends that do not ascend."""
    print("many", kernel, flush=True)
    seqs = 200
    c = Case(22, "bf16", 4, 2, 64, 16, [(1, 30)] * seqs)
    starts = list(range(seqs + 1))
    for s in range(1, seqs, 3):
        starts[s] = (LOW, HIGH, -5, seqs + 9)[s % 4]
    c.starts = torch.tensor(starts).to(torch.int32)
    out, whole = guarded((seqs, 4, 64), 777.0, c.dtype, 64)
    c.cache(kernel=kernel).attend(c.batch(), c.q.to(DEV).contiguous(), c.K.to(DEV), c.V.to(DEV), out=out)
    torch.cuda.synchronize()
    assert rim(whole, 64, 777)


@pytest.mark.parametrize("starts", STARTS)
@pytest.mark.parametrize("lens", [[150, 60, 333], [HIGH, LOW, -1], [39, HIGH - 5, 10 ** 6]])
def test_append_stays_inside(starts, lens):
    print("append", starts, lens, flush=True)
    c = Case(23, "bf16", 4, 2, 64, 16, [(40, 150), (1, 60), (19, 333)])
    c.starts, c.lens = torch.tensor(starts).to(torch.int32), torch.tensor(lens).to(torch.int32)
    (K, wk), (V, wv), (qo, wq) = (guarded(s, 777.0, c.dtype, 64) for s in (c.K.shape, c.V.shape, (60, 4, 64)))
    held = torch.unique(c.table[c.table >= 0])
    rot = B.Rotary(64, 500)
    c.cache().append(c.batch(max_len=400), c.k.to(DEV).contiguous(), c.v.to(DEV).contiguous(), K, V, rotary=rot, q=c.q.to(DEV).contiguous(), q_out=qo)
    torch.cuda.synchronize()
    assert rim(wk, 64, 777) and rim(wv, 64, 777) and rim(wq, 64, 777)
    others = [p for p in range(c.pages) if p not in held.tolist()]
    assert (K[others] == 777).all() and (V[others] == 777).all()   # pages of no sequence


@pytest.mark.parametrize("dtype,kernel", TYPES)
@pytest.mark.parametrize("window", [0, 24])
def test_logits_that_are_all_minus_infinity(dtype, kernel, window):
    """exp(-inf) for every key that a row sees: 0 / 0, not the 0 of a row that sees no key.  One finite logit, and it is an ordinary row."""
    print("minus infinity", dtype, kernel, window, flush=True)
    c = Case(24, dtype, 4, 2, 128, 16, [(40, 40), (1, 3000), (1, 70), (90, 600), (3, 2), (1, 33)], window)
    c.fused[:, :4, 3] = c.fused[:, :4, 3].abs() + 0.5          # every logit of a key with -inf there is -inf

    def lost(s, head, keys):
        for j in keys:
            c.K[int(c.table[s, j // 16]), head, j % 16, 3] = float("-inf")
    lost(0, 0, range(16))
    lost(1, 0, range(3000))
    lost(3, 1, range(530, 600))
    lost(5, 0, range(32))                                      # one key is left
    c.table[2, :] = -1
    out, lse = c.attend(c.cache(kernel=kernel))
    want, wlse, mass, absq = R.attend(c.q, c.K, c.V, c.starts, c.lens, c.table, window)
    # (the sums of the finite logits stay below 12)
    bo, bl = R.attend_bounds(want, wlse, mass, absq.clamp(max=16.0), c.dtype, c.d, dtype == "bf16")
    assert torch.isnan(want[:16, :2]).all() and torch.isnan(want[40, :2]).all() and (want[41] == 0).all()
    assert torch.isfinite(want[-1]).all() and torch.isnan(want).any(-1).sum() == (16 * 2 + 2 if not window else 16 * 2 + 2 + 2 * (600 - 553))
    within(out, want, bo, "out")
    within(lse, wlse, bl, "lse")
