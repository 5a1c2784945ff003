"""Rotary positions, head norms, append to and attention over paged caches through the public entry points, against plain
64-bit arithmetic on the CPU (tests/_paged.py), at the sizes and masks where they can go wrong."""
import math

import pytest
import torch

import _paged as R
from paper_2409_09086_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g).to(dtype)


def within(got, want, bound, what):
    got, off = got.double().cpu(), None
    off = (got - want).abs()
    same = (torch.isnan(want) & torch.isnan(got)) | (got == want)
    bad = ~(same | (off <= bound))
    assert not bad.any(), "%s: %d of %d off, first at %s: got %s, want %s, bound %s" % (
        what, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), got[bad][0].item(), want[bad][0].item(), torch.broadcast_to(bound, want.shape)[bad][0].item())


# ---- rotary -------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,d,heads,kv,n,layout,dims,scaling,norm", [
    ("bf16", 128, 32, 8, 1, "half", 128, {}, ""),
    ("bf16", 128, 5, 1, 37, "interleaved", 128, {}, "qk"),
    ("bf16", 64, 3, 3, 130, "half", 32, {"factor": 4.0}, "k"),
    ("bf16", 64, 1, 0, 65, "interleaved", 16, {}, ""),
    ("bf16", 128, 0, 7, 9, "half", 112, {"factor": 8.0, "trained": 2048, "low_turns": 1.0, "high_turns": 4.0, "magnitude": 1.25}, ""),
    ("fp32", 128, 6, 2, 33, "half", 128, {"factor": 8.0, "trained": 8192}, "q"),
    ("fp32", 64, 9, 4, 100, "interleaved", 48, {"magnitude": 0.5}, "qk"),
    ("bf16", 128, 32, 8, 700, "half", 128, {}, "qk"),
    ("fp32", 64, 17, 5, 1999, "half", 64, {}, ""),
    ("bf16", 64, 4, 2, 17, "half", 64, {"base": 0.0}, "qk"),
])
def test_rotary_apply(dtype, d, heads, kv, n, layout, dims, scaling, norm):
    print("rotary", dtype, d, heads, kv, n, layout, dims, scaling, norm, flush=True)
    g, dt, P = gen(n + d), R.DT[dtype], 100000
    base = scaling.pop("base", 500000.0)
    rot = B.Rotary(d, P, dtype=dt, base=base, dims=dims, layout=layout, norm_eps=1e-5, **scaling)
    pos = torch.randint(0, P, (n,), generator=g).to(torch.int32)
    pos[0], pos[-1] = P - 1, 0
    fused = randn(g, n, heads + 2 * kv + 1, d, dtype=dt)                 # strided: rows of a fused projection
    w = {c: (torch.rand(d, generator=g) + 0.5).to(dt) if c in norm else None for c in "qk"}
    dev = fused.to(DEV)
    q, k = (dev[:, :heads] if heads else None), (dev[:, heads:heads + kv] if kv else None)
    wd = {c: None if x is None else x.to(DEV) for c, x in w.items()}
    qo, ko = rot.apply(pos.to(DEV), q, k, q_weight=wd["q"], k_weight=wd["k"])
    f = None if not base else R.frequencies(dims, base, **{{"low_turns": "low", "high_turns": "high"}.get(a, a): b for a, b in scaling.items() if a != "magnitude"})
    for got, x, c in ((qo, fused[:, :heads], "q"), (ko, fused[:, heads:heads + kv], "k")):
        if got is None:
            assert x.shape[1] == 0
            continue
        want = R.rotate(x, pos, f, layout, w[c], 1e-5, scaling.get("magnitude", 1.0))
        # the angles' cosines: 100000 * f in 64 bits is exact to 2e-11
        within(got, want, R.rotate_bound(want, dt, w[c] is not None) + 1e-10, c)
    # in place on the fused rows: the same bits, and the rest of the rows as they were
    rot.apply(pos.to(DEV), q, k, q_weight=wd["q"], k_weight=wd["k"], q_out=q, k_out=k)
    if heads:
        assert torch.equal(dev[:, :heads], qo)
    if kv:
        assert torch.equal(dev[:, heads:heads + kv], ko)
    assert torch.equal(dev[:, heads + kv:].cpu(), fused[:, heads + kv:])


def test_rotary_positions_outside_the_table_are_nan():
    rot = B.Rotary(64, 100, dtype=torch.float32, dims=32)
    x = randn(gen(1), 4, 3, 64)
    out, _ = rot.apply(torch.tensor([0, 100, -1, 99], dtype=torch.int32, device=DEV), x.to(DEV))
    out = out.cpu()
    assert torch.isnan(out[1:3, :, :32]).all() and torch.equal(out[1:3, :, 32:], x[1:3, :, 32:])
    assert torch.isfinite(out[[0, 3]]).all() and torch.equal(out[0], x[0])


def test_rotary_zero_tokens():
    rot = B.Rotary(64, 100)
    q, k = rot.apply(torch.empty(0, dtype=torch.int32, device=DEV), torch.empty((0, 2, 64), dtype=torch.bfloat16, device=DEV))
    assert q.shape == (0, 2, 64) and k is None


# ---- batches ------------------------------------------------------------------------------------------------------------

class Case:
    """Pools and a batch of sequences [(new, len)]; pages in random order, rows that nobody holds NaN."""

    def __init__(self, seed, dtype, heads, kv, d, page, seqs, window=0, spare=2, tail=0, garbage=math.nan, scale=None, sigma=1.0):
        g = gen(seed)
        self.dtype, self.heads, self.kv, self.d, self.page, self.window, self.scale = R.DT[dtype], heads, kv, d, page, window, scale
        self.seqs = seqs
        need = [-(-max(n, 0) // page) for _, n in seqs]
        self.pages = sum(need) + spare
        order = torch.randperm(self.pages, generator=g)
        self.table = torch.full((len(seqs), max(max(need), 1) + 1), -1, dtype=torch.int32)
        at = 0
        self.K, self.V = (torch.full((self.pages, kv, page, d), garbage).to(self.dtype) for _ in range(2))
        for s, (_, n) in enumerate(seqs):
            for i in range(need[s]):
                p = int(order[at + i])
                self.table[s, i] = p
                rows = min(page, n - i * page)
                self.K[p, :, :rows] = (sigma * randn(g, kv, rows, d)).to(self.dtype)
                self.V[p, :, :rows] = randn(g, kv, rows, d).to(self.dtype)
            at += need[s]
        starts = [0]
        for new, _ in seqs:
            starts.append(starts[-1] + new)
        self.starts = torch.tensor(starts, dtype=torch.int32)
        self.lens = torch.tensor([n for _, n in seqs], dtype=torch.int32)
        self.tokens = starts[-1] + tail
        self.fused = (sigma * randn(g, self.tokens, heads + 2 * kv, d)).to(self.dtype)
        self.q, self.k, self.v = self.fused[:, :heads], self.fused[:, heads:heads + kv], self.fused[:, heads + kv:]

    def cache(self, **kw):
        return B.PagedCache(self.pages, self.page, self.heads, self.kv, self.d, dtype=self.dtype, window=self.window or None,
                            scale=self.scale, **kw)

    def batch(self, max_new=None, max_len=None):
        return B.PagedBatch(self.starts.to(DEV), self.lens.to(DEV), self.table.to(DEV), self.tokens,
                            max([n for n, _ in self.seqs]) if max_new is None else max_new,
                            max([n for _, n in self.seqs]) if max_len is None else max_len)

    def attend(self, cache=None, batch=None, q=None):
        lse = torch.full((self.tokens, self.heads), 777.0, dtype=torch.float32, device=DEV)
        out = torch.full((self.tokens, self.heads, self.d), 777.0, dtype=self.dtype, device=DEV)
        q = self.fused.to(DEV)[:, :self.heads] if q is None else q
        (cache or self.cache()).attend(batch or self.batch(), q, self.K.to(DEV), self.V.to(DEV), out=out, lse=lse)
        return out, lse

    def check(self, out, lse, what="attend"):
        want, wlse, mass, absq = R.attend(self.q, self.K, self.V, self.starts, self.lens, self.table, self.window, self.scale)
        used = int(self.starts[-1])
        assert (out[used:] == 777).all() and (lse[used:] == 777).all(), "rows behind the last sequence"
        bo, bl = R.attend_bounds(want, wlse, mass, absq, self.dtype, self.d, self.dtype == torch.bfloat16)
        within(out[:used], want[:used], bo[:used], what + " out")
        within(lse[:used], wlse[:used], bl[:used], what + " lse")


KERNELS = [0, 1, 2, 3]     # its own choice; that for few rows, that for chunks, both
TYPES = [("bf16", k) for k in KERNELS] + [("fp32", 0)]

ATTEND = [
    # dtype, heads, kv, d, page, window, [(new, len)]
    ("bf16", 4, 4, 128, 16, 0, [(1, 1)]),
    ("bf16", 8, 2, 128, 16, 0, [(1, 17), (1, 1), (1, 200), (1, 64), (1, 63)]),
    ("bf16", 5, 1, 64, 32, 0, [(1, 33), (3, 40), (0, 50), (0, 0), (1, 0), (4, 2), (17, 17)]),
    ("bf16", 14, 2, 128, 64, 0, [(33, 100), (1, 500), (70, 70)]),
    ("bf16", 2, 2, 128, 128, 0, [(300, 700)]),
    ("bf16", 8, 2, 128, 16, 0, [(150, 333), (1, 900), (2, 31)]),
    ("bf16", 8, 1, 64, 256, 0, [(90, 400), (5, 5)]),
    ("bf16", 2, 2, 64, 16, 0, [(260, 515)]),
    ("bf16", 4, 2, 128, 16, 50, [(100, 300), (1, 300), (1, 20), (60, 60)]),
    ("bf16", 4, 4, 64, 64, 1, [(130, 200), (1, 65)]),
    ("bf16", 40, 8, 128, 32, 700, [(64, 1500), (1, 1025)]),
    ("bf16", 32, 1, 128, 1024, 0, [(2, 1030), (1, 3)]),
    ("bf16", 3, 1, 128, 16, 0, [(1, 5000), (1, 2500)]),
    ("fp32", 4, 4, 128, 16, 0, [(1, 1), (1, 100)]),
    ("fp32", 10, 2, 64, 32, 0, [(33, 70), (1, 130), (0, 3), (2, 1)]),
    ("fp32", 8, 2, 128, 64, 0, [(100, 300), (1, 700)]),
    ("fp32", 2, 2, 64, 16, 40, [(90, 200), (1, 50)]),
    ("fp32", 14, 2, 128, 16, 0, [(1, 1200), (20, 900)]),
    ("fp32", 16, 4, 64, 16, 0, [(150, 400), (1, 300), (130, 131)]),        # 32 rows a unit
    ("fp32", 10, 2, 64, 32, 100, [(200, 500), (0, 9), (230, 300), (3, 1)]),
    ("fp32", 16, 8, 64, 16, 0, [(300, 350), (1, 90), (290, 290)]),           # a wavefront a team
]


@pytest.mark.parametrize("dtype,heads,kv,d,page,window,seqs,kernel", [c + (k,) for c in ATTEND for k in (KERNELS if c[0] == "bf16" else [0])])
def test_attend(dtype, heads, kv, d, page, window, seqs, kernel):
    print("attend", dtype, heads, kv, d, page, window, seqs, kernel, flush=True)
    c = Case(len(seqs) + heads, dtype, heads, kv, d, page, seqs, window, tail=3)
    cache = c.cache(kernel=kernel)
    out, lse = c.attend(cache)
    c.check(out, lse)
    again = c.attend(cache)                                   # the same bits again, with the same workspace
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    other = c.attend(cache, c.batch(max_new=0, max_len=0))    # wrong bounds: slower, not wrong
    c.check(*other, what="wrong bounds")
    other = c.attend(cache, c.batch(max_new=c.tokens, max_len=1 << 20))
    c.check(*other, what="wide bounds")


@pytest.mark.parametrize("seqs,share,chunk,window", [(65, 1.0, 0, 0), (200, 0.7, 90, 0), (640, 1.0, 0, 30), (1100, 0.4, 0, 0), (5000, 0.05, 33, 0)])
@pytest.mark.parametrize("kernel", KERNELS)
def test_many_sequences(seqs, share, chunk, window, kernel):
    """More sequences than a wavefront has lanes, some without new tokens, perhaps a chunk among them."""
    print("many", seqs, share, chunk, window, kernel, flush=True)
    g = gen(seqs)
    new = (torch.rand(seqs, generator=g) < share).long().tolist()
    lens = [int(x) + n for x, n in zip(torch.randint(0, 90, (seqs,), generator=g), new)]
    if chunk:
        new[seqs // 3], lens[seqs // 3] = chunk, chunk + 200
    c = Case(seqs, "bf16", 4, 2, 64, 16, list(zip(new, lens)), window)
    out, lse = c.attend(c.cache(kernel=kernel))
    c.check(out, lse)


@pytest.mark.parametrize("dtype,kernel", TYPES)
@pytest.mark.parametrize("what", ["value", "key"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_hidden_rows_reach_no_result(dtype, what, bad, kernel):
    """A new token whose key or value is not finite: only the rows that see it may show it."""
    print("hidden", dtype, what, bad, kernel, flush=True)
    c = Case(5, dtype, 4, 2, 128, 16, [(90, 150), (2, 40), (1, 70)])
    pool = c.V if what == "value" else c.K
    for s, at in ((0, 110), (1, 39)):
        pool[int(c.table[s, at // 16]), 0, at % 16, 3] = bad
    out, lse = c.attend(c.cache(kernel=kernel))
    if what == "value":
        c.check(out, lse)
    else:
        rows = [r for r in range(93) if r < 110 - 60 or r in (90, 92)]
        want, wlse, mass, absq = R.attend(c.q, c.K, c.V, c.starts, c.lens, c.table)
        bo, bl = R.attend_bounds(want, wlse, mass, absq, c.dtype, c.d, dtype == "bf16")
        within(out[rows], want[rows], bo[rows], "rows that do not see the key")
        within(out[:, 2:], want[:, 2:], bo[:, 2:], "heads that do not see the key")
        within(lse[rows], wlse[rows], bl[rows], "lse")


@pytest.mark.parametrize("dtype,kernel", TYPES)
def test_bad_pages_are_hidden(dtype, kernel):
    c = Case(6, dtype, 4, 2, 128, 16, [(40, 150), (1, 60), (1, 20), (1, 500)])
    c.table[0, 2], c.table[0, 7] = -5, c.pages                # inside and in the causal part
    c.table[1, 0] = 1 << 30
    c.table[2, :] = -1                                        # nothing is left: 0
    c.table = c.table[:, :12].contiguous()                    # and a length beyond the table
    out, lse = c.attend(c.cache(kernel=kernel))
    c.check(out, lse)
    assert (out[41] == 0).all() and torch.isneginf(lse[41]).all()


@pytest.mark.parametrize("dtype,kernel", TYPES)
@pytest.mark.parametrize("window", [0, 150])
def test_lengths_beyond_the_table(dtype, kernel, window):
    """Tables that end inside a run of keys (176 = 5.5 * 32 = 2.75 * 64) ahead of the lengths."""
    print("beyond", dtype, kernel, window, flush=True)
    c = Case(12, dtype, 4, 2, 128, 16, [(100, 230), (1, 300), (3, 178), (1, 176), (1, 400), (130, 500)], window)
    c.table = c.table[:, :11].contiguous()
    out, lse = c.attend(c.cache(kernel=kernel))
    c.check(out, lse)


@pytest.mark.parametrize("dtype,kernel", TYPES)
@pytest.mark.parametrize("new", [1, 80])
def test_large_logits(dtype, new, kernel):
    """Logits of thousands, of both signs, whose references move from tile to tile."""
    c = Case(7, dtype, 4, 2, 128, 32, [(new, 300)], sigma=8.0, scale=1.0)
    out, lse = c.attend(c.cache(kernel=kernel))
    c.check(out, lse)


@pytest.mark.parametrize("dtype,kernel", TYPES)
def test_shared_pages_and_queries_that_are_not_finite(dtype, kernel):
    """Three sequences over the pages of a common prefix; one token's query of one head is NaN: its row alone shows it."""
    print("shared", dtype, kernel, flush=True)
    c = Case(17, dtype, 4, 2, 128, 16, [(60, 300), (1, 280), (1, 305)])
    c.table[1, :16], c.table[2, :16] = c.table[0, :16], c.table[0, :16]
    want, wlse, mass, absq = R.attend(c.q, c.K, c.V, c.starts, c.lens, c.table)
    bo, bl = R.attend_bounds(want, wlse, mass, absq, c.dtype, c.d, dtype == "bf16")
    c.fused[33, 1, 5] = math.nan
    out, lse = c.attend(c.cache(kernel=kernel))
    assert torch.isnan(out[33, 1]).all() and torch.isnan(lse[33, 1])
    others = torch.ones(c.tokens, 4, dtype=torch.bool)
    others[33, 1] = False
    on = others.to(DEV)
    within(out[on], want[others], bo[others], "out")
    within(lse[on], wlse[others], bl[others], "lse")


def test_one_token_has_no_stride():
    """A single token's row of a wider tensor, whatever the distance to a next one would be."""
    c = Case(18, "bf16", 8, 2, 128, 16, [(1, 77)])
    wide = torch.zeros(1, 8 * 128 + 3, dtype=torch.bfloat16, device=DEV)
    q = wide[:, :8 * 128].view(1, 8, 128)
    q.copy_(c.q)
    out, lse = c.attend(q=q)
    want = c.attend()
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    rot = B.Rotary(128, 100)
    pos = torch.tensor([76], dtype=torch.int32, device=DEV)
    assert torch.equal(rot.apply(pos, q)[0], rot.apply(pos, q.contiguous().clone())[0])


def test_attend_in_place_and_dense_queries():
    for dtype, new, kernel in (("bf16", 1, 0), ("bf16", 130, 1), ("bf16", 130, 2), ("bf16", 130, 3), ("fp32", 40, 0)):
        c = Case(8, dtype, 8, 2, 128, 16, [(new, 400), (1, 350)])
        want, _ = c.attend(c.cache(kernel=kernel))
        q = c.q.to(DEV).contiguous()
        got = c.cache(kernel=kernel).attend(c.batch(), q, c.K.to(DEV), c.V.to(DEV), out=q)
        assert got is q and torch.equal(q, want)


def test_pools_beyond_32_bit_offsets():
    """Pages whose rows lie more than 2^32 bytes (and 2^31 elements) into the pools."""
    page, kv, d = 256, 8, 128
    pages = (1 << 32) // (page * kv * d * 2) + 9
    g = gen(9)
    cache = B.PagedCache(pages, page, 16, kv, d)
    K, V = cache.pools()
    table = torch.tensor([[pages - 1, pages - 3], [pages - 2, 0]], dtype=torch.int32)
    rot = B.Rotary(d, 1000)
    starts, lens = torch.tensor([0, 300, 301], dtype=torch.int32), torch.tensor([300, 1], dtype=torch.int32)
    k, v, q = (randn(g, 301, h, d, dtype=torch.bfloat16) for h in (kv, kv, 16))
    b = B.PagedBatch(starts.to(DEV), lens.to(DEV), table.to(DEV), 301, 300, 300)
    qr = cache.append(b, k.to(DEV), v.to(DEV), K, V, rotary=rot, q=q.to(DEV))
    out = cache.attend(b, qr, K, V)
    used = [pages - 1, pages - 3, pages - 2]
    for kernel in KERNELS[1:]:
        got = B.PagedCache(pages, page, 16, kv, d, kernel=kernel).attend(b, qr, K, V).float()
        assert (got - out.float()).abs().max() < 0.02, kernel          # the weights' rounding: 2^-8 of values around 1
    small = B.PagedCache(3, page, 16, kv, d)
    Ks, Vs = K[used].contiguous(), V[used].contiguous()
    b2 = B.PagedBatch(starts.to(DEV), lens.to(DEV), torch.tensor([[0, 1], [2, 0]], dtype=torch.int32, device=DEV), 301, 300, 300)
    assert torch.equal(out, small.attend(b2, qr, Ks, Vs))
    assert torch.equal(Vs[0].transpose(0, 1).cpu(), v[:256])


# ---- append -------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,heads,kv,d,page,seqs,layout,dims,norm,with_q", [
    ("bf16", 8, 2, 128, 16, [(1, 1), (1, 17), (1, 16), (0, 40), (1, 33)], "half", 128, True, True),
    ("bf16", 6, 3, 64, 32, [(40, 70), (0, 0), (33, 33), (4, 2), (1, 0)], "interleaved", 32, False, True),
    ("fp32", 4, 4, 128, 64, [(100, 200), (1, 64)], "half", 64, True, True),
    ("fp32", 5, 1, 64, 16, [(7, 30)] * 70, "interleaved", 64, False, False),
    ("bf16", 32, 8, 128, 128, [(600, 700), (211, 300)], "half", 128, False, True),
    ("bf16", 4, 2, 128, 16, [(20, 90)], None, 0, False, False),
])
def test_append(dtype, heads, kv, d, page, seqs, layout, dims, norm, with_q):
    print("append", dtype, heads, kv, d, page, len(seqs), layout, dims, norm, with_q, flush=True)
    c = Case(len(seqs) + d, dtype, heads, kv, d, page, seqs, tail=2, garbage=5.0)
    g = gen(3)
    w = [(torch.rand(d, generator=g) + 0.5).to(c.dtype) if norm else None for _ in range(2)]
    wd = [None if x is None else x.to(DEV) for x in w]
    rot = B.Rotary(d, 4096, dtype=c.dtype, dims=dims, layout=layout) if layout else None
    f = R.frequencies(dims, 10000.0) if layout else None
    K, V, fused = c.K.to(DEV), c.V.to(DEV), c.fused.to(DEV)
    qo = torch.full((c.tokens, heads, d), 777.0, dtype=c.dtype, device=DEV) if with_q else None
    got = c.cache().append(c.batch(), fused[:, heads:heads + kv], fused[:, heads + kv:], K, V, rotary=rot, k_weight=wd[1],
                           q=fused[:, :heads] if with_q else None, q_weight=wd[0] if with_q else None, q_out=qo)
    pos = torch.cat([torch.arange(n - new, n) for new, n in seqs] + [torch.full((2,), -1)])
    k = R.rotate(c.k, pos, f, layout, w[1])
    bk = R.rotate_bound(k, c.dtype, norm) + 1e-10 if layout else torch.zeros_like(k)
    wantK, boundK, wantV = c.K.double(), torch.zeros(c.K.shape, dtype=torch.float64), c.V.clone()
    t = 0
    for s, (new, n) in enumerate(seqs):
        for r in range(new):
            p = n - new + r
            if p >= 0:
                at = (int(c.table[s, p // page]), slice(None), p % page)
                wantK[at], boundK[at], wantV[at] = k[t], bk[t], c.v[t]
            t += 1
    within(K, wantK, boundK, "K")
    assert torch.equal(V.cpu(), wantV)
    if with_q:
        assert got is qo
        q = R.rotate(c.q, pos, f, layout, w[0])
        there = pos >= 0
        within(qo[there.to(DEV)], q[there], R.rotate_bound(q[there], c.dtype, norm) + 1e-10, "q")
        assert (qo[(~there).to(DEV)] == 777).all()


def test_append_leaves_other_pages_alone():
    """Bad page numbers, lengths beyond the table: nothing is written for them."""
    c = Case(11, "bf16", 4, 2, 64, 16, [(20, 40), (1, 10), (3, 90)], garbage=5.0)
    c.table[0, 1] = c.pages
    c.table[1, 0] = -7
    c.table = c.table[:, :5].contiguous()                     # positions 80.. have no page
    K, V = c.K.to(DEV), c.V.to(DEV)
    c.cache().append(c.batch(), c.k.to(DEV), c.v.to(DEV), K, V)
    wantK, wantV = c.K.clone(), c.V.clone()
    for r, p in enumerate(range(20, 40)):
        if p >= 32:
            wantK[int(c.table[0, 2]), :, p % 16], wantV[int(c.table[0, 2]), :, p % 16] = c.k[r], c.v[r]
    assert torch.equal(K.cpu(), wantK) and torch.equal(V.cpu(), wantV)


# ---- together -----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_serving_run(dtype):
    """Two layers over a prompt, a second prompt beside decoded tokens, and decoded tokens: append and attend as a serving program uses
    them, against attention over the whole rotated history."""
    dt, heads, kv, d, page, pages = R.DT[dtype], 8, 2, 128, 16, 40
    g = gen(12)
    rot = B.Rotary(d, 512, dtype=dt, norm_eps=1e-6)
    w = [(torch.rand(d, generator=g) + 0.5).to(dt) for _ in range(2)]
    wd = [x.to(DEV) for x in w]
    cache = B.PagedCache(pages, page, heads, kv, d, dtype=dt)
    layers = [cache.pools() for _ in range(2)]
    for K, V in layers:
        K.fill_(math.nan), V.fill_(math.nan)
    table = torch.randperm(pages, generator=g)[:36].reshape(3, 12).to(torch.int32)
    lens = [0, 0, 0]
    pools = [(torch.full((pages, kv, page, d), math.nan).to(dt), torch.full((pages, kv, page, d), math.nan).to(dt)) for _ in layers]
    for step, new in enumerate([(70, 0, 0), (1, 33, 1), (1, 1, 40), (1, 1, 1), (1, 0, 1), (2, 5, 100)]):
        print("serving", dtype, step, new, flush=True)
        lens = [a + b for a, b in zip(lens, new)]
        starts = torch.tensor([0, new[0], new[0] + new[1], sum(new)], dtype=torch.int32)
        ln = torch.tensor(lens, dtype=torch.int32)
        b = B.PagedBatch(starts.to(DEV), ln.to(DEV), table.to(DEV), sum(new), max(new), max(lens))
        for (K, V), (hk, hv) in zip(layers, pools):
            fused = randn(g, sum(new), heads + 2 * kv, d, dtype=dt)
            dev = fused.to(DEV)
            q = cache.append(b, dev[:, heads:heads + kv], dev[:, heads + kv:], K, V, rotary=rot, k_weight=wd[1], q=dev[:, :heads], q_weight=wd[0])
            out = cache.attend(b, q, K, V)
            # the history as the library holds it (appends are tested above), attention in 64 bits
            hk.copy_(K.cpu()), hv.copy_(V.cpu())
            want, wlse, mass, absq = R.attend(q.cpu(), hk, hv, starts, ln, table)
            bo, _ = R.attend_bounds(want, wlse, mass, absq, dt, d, dtype == "bf16")
            within(out, want, bo, "layer")


@pytest.mark.parametrize("kernel", KERNELS)
def test_graph_follows_the_batch_arrays(kernel):
    """append + attend captured once (the attention on every kernel); replays with other lengths, between eager work, give what eager calls give."""
    c = Case(13, "bf16", 8, 2, 128, 16, [(1, 100), (1, 30), (1, 190)], garbage=0.0)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        cache, rot = c.cache(kernel=kernel), B.Rotary(128, 1024)
        b, K, V, fused = c.batch(max_len=200), c.K.to(DEV), c.V.to(DEV), c.fused.to(DEV)
        q, k, v = fused[:, :8], fused[:, 8:10], fused[:, 10:]
        qo, out = torch.empty_like(q.contiguous()), torch.empty((3, 8, 128), dtype=torch.bfloat16, device=DEV)
        work = lambda: (cache.append(b, k, v, K, V, rotary=rot, q=q, q_out=qo), cache.attend(b, qo, K, V, out=out))
        work()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            work()
        for lens in ([100, 30, 190], [101, 31, 1], [64, 16, 200], [5, 1, 17]):
            b.lens.copy_(torch.tensor(lens, dtype=torch.int32))
            K.copy_(c.K), V.copy_(c.V)
            out.zero_()
            graph.replay()
            side.synchronize()
            got, gK = out.clone(), K.clone()
            K.copy_(c.K), V.copy_(c.V)
            work()
            side.synchronize()
            assert torch.equal(got, out) and torch.equal(gK, K), lens


@pytest.mark.parametrize("kernel", KERNELS)
def test_graph_of_units_in_pieces(kernel):
    """Replays whose lengths and tables differ, with units cut over many teams: what one leaves for its merges the next one finds clear."""
    c = Case(16, "bf16", 8, 2, 128, 32, [(150, 2500), (1, 3000), (1, 700), (3, 1200)])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        cache, b = c.cache(kernel=kernel), c.batch()
        K, V, q = c.K.to(DEV), c.V.to(DEV), c.q.to(DEV).contiguous()
        out, lse = torch.empty_like(q), torch.empty((c.tokens, 8), device=DEV)
        cache.attend(b, q, K, V, out=out, lse=lse)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            cache.attend(b, q, K, V, out=out, lse=lse)
        for lens, rows in (([2500, 3000, 700, 1200], None), ([150, 1, 1, 3], None), ([1300, 2999, 64, 1150], [1, 0, 3, 2]), ([2500, 0, 650, 1], None)):
            c.lens = torch.tensor(lens, dtype=torch.int32)
            if rows:
                c.table, c.lens = c.table[rows].contiguous(), torch.minimum(c.lens, torch.tensor([2500, 3000, 700, 1200])[rows]).to(torch.int32)
            b.lens.copy_(c.lens), b.table.copy_(c.table)
            for _ in range(2):
                out.fill_(777), lse.fill_(777)
                graph.replay()
                side.synchronize()
                got = out.clone(), lse.clone()
                out.fill_(777), lse.fill_(777)
                cache.attend(b, q, K, V, out=out, lse=lse)
                side.synchronize()
                assert torch.equal(got[0], out) and torch.equal(got[1], lse), lens
            c.check(out, lse)


def test_two_objects_on_two_streams():
    a, b = Case(14, "bf16", 8, 2, 128, 16, [(200, 900), (1, 800)]), Case(15, "bf16", 4, 4, 64, 32, [(1, 2000), (1, 1000)])
    want = [x.attend(x.cache(kernel=3))[0] for x in (a, b)]
    torch.cuda.synchronize()
    runs = []
    for x in (a, b):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            runs.append((x.cache(kernel=3), x.batch(), x.q.to(DEV).contiguous(), x.K.to(DEV), x.V.to(DEV)))
        s.synchronize()
    outs = [[cache.attend(bt, q, K, V) for _ in range(4)] for cache, bt, q, K, V in runs]
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert all(torch.equal(w, y) for y in o)
