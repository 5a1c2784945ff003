"""Softmax weights of the kernel for few rows enter the second product as two bf16 terms, good for 16 bits: tolerances that one term would
break.  Values are +-1 and logits small, so that outputs are small beside the mass that they cancel from, and so is their own rounding."""
import pytest
import torch

import _paged as R
from test_gpu_paged import Case, within

# [(new, len)], and the sequences of at most 16 rows (which both kernels side by side leave to that for few rows)
RUNS = [(4, 2, 128, 16, [(1, 60), (1, 250), (3, 200), (30, 90)], [0, 1, 2]),
        (4, 4, 64, 32, [(1, 33), (16, 150), (70, 300), (1, 400)], [0, 1, 3])]


def cancelling(heads, kv, d, page, seqs):
    c = Case(41, "bf16", heads, kv, d, page, seqs, garbage=0.0, sigma=0.5)
    c.V = torch.where(c.V < 0, -1.0, 1.0).to(torch.bfloat16)
    want, lse, mass, absq = R.attend(c.q, c.K, c.V, c.starts, c.lens, c.table)
    # a weight is rounded to 8 bits, off by at most 2^-8 of it, and that rest to 8 more, off by at most 2^-8 of the rest
    bound, _ = R.attend_bounds(want, lse, mass, absq, torch.bfloat16, d, False)
    return c, want, bound + 2.0 ** -16 * mass


def restated(c, terms):
    """The outputs with weights, relative to the largest, as `terms` bf16 terms under their own unrounded sum."""
    out = torch.empty(c.q.shape, dtype=torch.float64)
    G = c.heads // c.kv
    for s, (new, n) in enumerate(c.seqs):
        rows = [(int(c.table[s, j // c.page]), j % c.page) for j in range(n)]
        pg, rw = torch.tensor([r[0] for r in rows]), torch.tensor([r[1] for r in rows])
        for g in range(c.heads):
            K, V = c.K[pg, g // G, rw].double(), c.V[pg, g // G, rw].double()
            for i in range(new):
                t, seen = int(c.starts[s]) + i, n - new + i + 1
                x = K[:seen] @ c.q[t, g].double() / c.d ** 0.5
                w = torch.exp(x - x.max())
                first = w.bfloat16().double()
                used = first if terms == 1 else first + (w - first).bfloat16().double()
                out[t, g] = used @ V[:seen] / w.sum()
    return out


@pytest.mark.parametrize("heads,kv,d,page,seqs,few", RUNS)
def test_the_bound_tells_one_term_from_two(heads, kv, d, page, seqs, few):
    c, want, bound = cancelling(heads, kv, d, page, seqs)
    for s, (new, _) in enumerate(seqs):
        rows = slice(int(c.starts[s]), int(c.starts[s]) + new)
        two, one = ((restated(c, t)[rows] - want[rows]).abs() > bound[rows] for t in (2, 1))
        assert not two.any() and one.float().mean() > 0.01, (s, float(one.float().mean()))


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kv,d,page,seqs,few", RUNS)
@pytest.mark.parametrize("kernel", [0, 1, 3])
def test_weights_of_few_rows_keep_sixteen_bits(heads, kv, d, page, seqs, few, kernel):
    print("weights", heads, kv, d, page, seqs, kernel, flush=True)
    c, want, bound = cancelling(heads, kv, d, page, seqs)
    if kernel == 0:                                            # decoded tokens alone: its own choice
        c = Case(42, "bf16", heads, kv, d, page, [(1, n) for _, n in seqs], garbage=0.0, sigma=0.5)
        c.V = torch.where(c.V < 0, -1.0, 1.0).to(torch.bfloat16)
        want, lse, mass, absq = R.attend(c.q, c.K, c.V, c.starts, c.lens, c.table)
        bound = R.attend_bounds(want, lse, mass, absq, torch.bfloat16, d, False)[0] + 2.0 ** -16 * mass
    out, _ = c.attend(c.cache(kernel=kernel))
    for s in range(len(seqs)) if kernel != 3 else few:
        rows = slice(int(c.starts[s]), int(c.starts[s + 1]))
        within(out[rows], want[rows], bound[rows], "out of sequence %d" % s)
