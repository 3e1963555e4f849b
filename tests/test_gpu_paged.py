"""The paged key/value cache on the GPU against its float64 oracle.

Tolerances.  With A = sum_j p_j |v_j| of a row and channel (at least |out|): weights are rounded to
bf16 before they meet the values, each off by at most half a step, 2^-8 relative, and so is the
output, together 2 * 2^-8 A to first order.  A score is a sum of up to 128 float32 products, off by
at most 128 * 2^-24 of big = sum_d |q_d k_d| / sqrt(hd), which moves weights by the same absolute
amount relative to themselves, numerator and denominator both: 2 * 2^-17 big; the second-order
terms, the scaling and the exponentials (a few units of 2^-23 of a score's size) stay below
another 2^-17 (1 + big).  Log sums carry the scores' error and a few units of 2^-23 of their own
size.  Kept pieces and groups change the order of float32 sums only.
"""
import numpy as np
import pytest
import torch

from oracle import paged as op
from paper_2607_14647_amd import lib as L
from paper_2607_14647_amd import workload as wl
from tests.gpu_common import need_gpu, note

pytestmark = pytest.mark.gpu

THETA = 500000.0


def bf(x):
    """Nearest bf16 values, as float64 numpy."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).bfloat16().double().numpy()


def dev(x, dtype=torch.bfloat16):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype).cuda()


class Batch:
    """A paged cache with its requests: host float64 copies and device tensors.  `d`, `ctx`: new rows and earlier keys of
    each request; `prefix`: per group (first request, one past the last, keys), whose whole pages are shared."""

    def __init__(self, n_q, n_kv, hd, page, d, ctx, seed=0, prefix=(), extra_rows=3, slack=0, qpad=0, stale=None):
        rng = np.random.default_rng(seed)
        self.n_q, self.n_kv, self.hd, self.page = n_q, n_kv, hd, page
        self.d, self.ctx, self.B = np.array(d), np.array(ctx), len(d)
        self.cu = np.concatenate([[0], np.cumsum(self.d)]).astype(np.int32)
        self.M = int(self.cu[-1])
        self.rows = self.M + extra_rows
        need = -(-(self.ctx + self.d) // page)
        total = int(need.sum()) + 2
        ids = rng.permutation(total)
        self.table = np.full((self.B, int(max(need.max(), 1)) + slack), -1, dtype=np.int32)
        at = 0
        for i in range(self.B):
            self.table[i, : need[i]] = ids[at: at + need[i]]
            at += need[i]
        self.k, self.v = bf(rng.standard_normal((total, n_kv, page, hd))), bf(rng.standard_normal((total, n_kv, page, hd)))
        for a, b, P in prefix:
            full = P // page
            for i in range(a + 1, b):
                self.table[i, :full] = self.table[a, :full]
                if P % page:                       # the partly shared page: a copy of its first keys
                    src, dst = self.table[a, full], self.table[i, full]
                    self.k[dst, :, : P % page], self.v[dst, :, : P % page] = self.k[src, :, : P % page], self.v[src, :, : P % page]
        self.q = bf(1.5 * rng.standard_normal((self.rows, n_q, hd)))
        if stale is not None:                      # everything that no row sees
            kept = np.zeros((total, page), dtype=bool)
            for i in range(self.B):
                for j in range(int(self.ctx[i] + self.d[i])):
                    kept[self.table[i, j // page], j % page] = True
            for x in (self.k, self.v):
                x[np.broadcast_to(~kept[:, None, :, None], x.shape)] = stale
            self.q[self.M:] = stale
        self.max_ctx, self.max_block = int((self.ctx + self.d).max()), int(self.d.max())
        qbuf = torch.zeros(self.rows, n_q * hd + qpad, dtype=torch.bfloat16, device="cuda")
        qbuf[:, : n_q * hd] = dev(self.q.reshape(self.rows, -1))
        self.dq = qbuf[:, : n_q * hd]
        self.dk, self.dv = dev(self.k), dev(self.v)
        self.dtable, self.dcu, self.dctx = dev(self.table, torch.int32), dev(self.cu, torch.int32), dev(self.ctx, torch.int32)
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.dkmin = self.dkmax = None

    def bounds(self):
        self.kmin, self.kmax = self.k.min(2), self.k.max(2)
        self.dkmin, self.dkmax = dev(self.kmin), dev(self.kmax)

    def cfg(self, **kw):
        d = dict(n_q=self.n_q, n_kv=self.n_kv, head_dim=self.hd, page=self.page, max_ctx=self.max_ctx,
                 max_block=self.max_block, max_rows=self.rows)
        d.update(kw)
        return L.paged_cfg(**d)

    def pages(self):
        return L.pages_desc(self.dk, self.dv, self.dtable, self.dkmin, self.dkmax)

    def outputs(self):
        out = torch.full((self.rows, self.n_q, self.hd), 7.0, dtype=torch.bfloat16, device="cuda")
        return out, torch.full((self.rows, self.n_q), 7.0, device="cuda")

    def run(self, call="attn", cfg=None, groups=None, sel=None, blocks=None, ws=None, lse=True, stream=None):
        cfg = self.cfg() if cfg is None else cfg
        out, ls = self.outputs()
        if ws is None:
            n = L.paged_workspace_bytes(call, cfg, self.B, sel[0] if sel else 0)
            ws = torch.full((max(n, 256),), 0x7f, dtype=torch.uint8, device="cuda")      # NaN-like rubbish
        a = (cfg, self.pages(), self.B, self.dq, self.dcu, self.dctx, out, ws)
        kw = dict(lse=ls if lse else None, dev_err=self.err, stream=stream)
        if call == "attn":
            L.paged_attn(*a, **kw)
        elif call == "shared":
            L.paged_attn_shared(*a, *groups, **kw)
        else:
            L.paged_attn_sparse(*a, *sel, blocks=blocks, **kw)
        return out, ls

    def check(self, out, ls, ref, rows=None, what=""):
        torch.cuda.synchronize()
        o, l = out.double().cpu().numpy(), ls.double().cpu().numpy()
        rows = np.arange(self.M) if rows is None else rows
        big = ref["big"][rows]
        tol = ref["mag"][rows] * (2 * 2.0 ** -8 * 1.01 + (3 * 2.0 ** -17) * (1 + big[:, :, None]))
        bad = np.abs(o[rows] - ref["out"][rows]) - tol
        ltol = 2.0 ** -17 * (1 + big) + 2.0 ** -20 * np.abs(ref["lse"][rows])
        lbad = np.abs(l[rows] - ref["lse"][rows]) - ltol
        note(f"{what}: {len(rows)} rows, out excess {bad.max(initial=-1):.2e}, lse excess {lbad.max(initial=-1):.2e}, "
             f"err {int(self.err.item())}")
        assert (bad <= 0).all() and (lbad <= 0).all(), what
        assert (o[self.M:] == 7.0).all() and (l[self.M:] == 7.0).all(), "rows past the last request's"

    def oracle(self):
        return op.paged_attn(self.q[: self.M], self.k, self.v, self.table, self.cu, self.ctx, self.page)


EDGE = [0, 1, 14, 15, 16, 17, 30, 31, 32, 33, 62, 63, 64, 65, 126, 127, 128, 129, 130, 255, 256, 257, 511, 700, 1300]
ATTN = {
    # one new row a request: contexts at the edges of tiles, pages, pieces; the empty context
    "decode": dict(n_q=8, n_kv=2, hd=128, page=16, d=[1] * len(EDGE), ctx=EDGE),
    "decode64": dict(n_q=14, n_kv=2, hd=64, page=32, d=[1] * len(EDGE), ctx=EDGE),
    "decode1": dict(n_q=4, n_kv=4, hd=128, page=64, d=[1], ctx=[0]),
    "single_long": dict(n_q=8, n_kv=1, hd=128, page=16, d=[1], ctx=[5000]),
    "big_page": dict(n_q=4, n_kv=2, hd=64, page=256, d=[1, 3, 2], ctx=[255, 254, 700]),
    # blocks, requests without rows, groups of 3 and 5 heads
    "verify": dict(n_q=9, n_kv=3, hd=64, page=16, d=[0, 4, 1, 0, 7, 16, 2, 5, 0], ctx=[50, 0, 1, 0, 300, 33, 16, 129, 700]),
    "verify5": dict(n_q=10, n_kv=2, hd=128, page=128, d=[3, 0, 13, 1], ctx=[200, 5, 127, 0]),
    # 65 to 128 pairs a request, in one tile and in several
    "wide": dict(n_q=16, n_kv=2, hd=128, page=16, d=[16, 9, 1], ctx=[100, 0, 40]),
    "group64": dict(n_q=64, n_kv=1, hd=64, page=16, d=[1, 3, 0, 2], ctx=[20, 400, 3, 0]),
    # prompts: many tiles a request, ragged, with and without context
    "prompt": dict(n_q=4, n_kv=1, hd=128, page=16, d=[150, 0, 1, 97, 33], ctx=[0, 3, 500, 63, 0]),
    "prompt64": dict(n_q=6, n_kv=2, hd=64, page=64, d=[1, 260, 128], ctx=[10, 200, 0]),
    "mha": dict(n_q=3, n_kv=3, hd=64, page=16, d=[5, 130], ctx=[77, 1]),
}


@pytest.mark.parametrize("name", list(ATTN))
def test_attn(name):
    need_gpu()
    b = Batch(seed=1, qpad=8 * (len(name) % 3), slack=len(name) % 2, **ATTN[name])
    out, ls = b.run()
    b.check(out, ls, b.oracle(), what=name)
    assert int(b.err.item()) == 0
    again, ls2 = b.run()
    assert torch.equal(out, again) and torch.equal(ls, ls2)
    none, _ = b.run(lse=False)
    assert torch.equal(out, none)


@pytest.mark.parametrize("stale", [np.nan, np.inf])
@pytest.mark.parametrize("name", ["decode", "verify", "wide", "prompt"])
def test_unseen_slots_may_hold_anything(name, stale):
    """Free pages, tails of last pages and rows past the last hold NaN or infinities."""
    need_gpu()
    b = Batch(seed=2, stale=stale, **ATTN[name])
    out, ls = b.run()
    b.check(out, ls, b.oracle(), what=f"{name} stale {stale}")


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("name", ["verify", "prompt"])
def test_later_rows_never_reach_earlier_ones(name, value):
    """The last row of every block has a key and a value of NaN or infinities: earlier rows are bitwise what they were."""
    need_gpu()
    b = Batch(seed=3, **ATTN[name])
    out, ls = b.run()
    rows = []
    for i in range(b.B):
        if b.d[i]:
            p = int(b.ctx[i] + b.d[i] - 1)
            for x in (b.dk, b.dv):
                x[int(b.table[i, p // b.page]), :, p % b.page, ::3] = value
            rows += list(range(b.cu[i], b.cu[i + 1] - 1))
    got, gls = b.run()
    torch.cuda.synchronize()
    rows = torch.tensor(rows, device="cuda")
    assert torch.equal(out[rows], got[rows]) and torch.equal(ls[rows], gls[rows])
    last = torch.tensor([b.cu[i + 1] - 1 for i in range(b.B) if b.d[i]], device="cuda")
    assert not torch.isfinite(got[last].float()).all(-1).any()


def test_seen_infinite_values():
    """Values of a block's first key infinite in some channels, its later rows see it: the same infinities and NaN."""
    need_gpu()
    b = Batch(n_q=4, n_kv=2, hd=64, page=16, d=[4, 6], ctx=[5, 40], seed=4)
    ref = b.oracle()
    for i in range(2):
        p = int(b.ctx[i])
        pg, s = int(b.table[i, p // 16]), p % 16
        b.dv[pg, :, s, 3], b.dv[pg, :, s, 5], b.dv[pg, :, s, 9] = np.inf, -np.inf, np.nan
        p2 = p + 2
        b.dv[int(b.table[i, p2 // 16]), :, p2 % 16, 3] = -np.inf       # and from row 2 on, both signs in channel 3
    out, _ = b.run()
    o = out.double().cpu().numpy()
    for i in range(2):
        for r in range(int(b.d[i])):
            t = b.cu[i] + r
            assert (np.isposinf(o[t, :, 3]) if r < 2 else np.isnan(o[t, :, 3])).all()
            assert np.isneginf(o[t, :, 5]).all() and np.isnan(o[t, :, 9]).all()
            assert np.abs(o[t, :, 10:] - ref["out"][t, :, 10:]).max() < 0.1


def test_rows_do_not_depend_on_the_rest_of_the_batch():
    need_gpu()
    b = Batch(seed=5, **ATTN["verify"])
    out, ls = b.run()
    # fewer kept rows of request 5, none of request 4, another context for request 6
    d2 = b.d.copy()
    d2[5], d2[4] = 3, 0
    rows_old = np.concatenate([np.arange(b.cu[i], b.cu[i] + d2[i]) for i in range(b.B) if i != 6])
    cu2 = np.concatenate([[0], np.cumsum(d2)]).astype(np.int32)
    rows_new = np.concatenate([np.arange(cu2[i], cu2[i + 1]) for i in range(b.B) if i != 6])
    src = np.concatenate([np.arange(b.cu[i], b.cu[i] + d2[i]) for i in range(b.B)])
    q2 = b.dq.clone()
    q2[: len(src)] = b.dq[torch.from_numpy(src).cuda()]
    b.dq = q2
    b.dcu.copy_(torch.from_numpy(cu2))
    b.dctx[6] = 11
    out2, ls2 = b.run()
    torch.cuda.synchronize()
    i, j = torch.from_numpy(rows_old).cuda(), torch.from_numpy(rows_new).cuda()
    assert torch.equal(out[i], out2[j]) and torch.equal(ls[i], ls2[j])


def test_scores_past_two_to_the_31():
    need_gpu()
    b = Batch(n_q=4, n_kv=2, hd=128, page=16, d=[2, 1], ctx=[100, 300], seed=6)
    b.q, b.k = b.q * 2.0 ** 22, b.k * 2.0 ** 22
    b.dq.mul_(2.0 ** 22)
    b.dk.mul_(2.0 ** 22)
    out, ls = b.run()
    ref = b.oracle()                          # one key's value, wherever the next score is not within rounding
    o = out.double().cpu().numpy()[: b.M]
    assert np.isfinite(o).all() and torch.isfinite(ls[: b.M]).all()
    assert (np.abs(o - ref["out"]) <= 2.0 ** -7 * np.abs(ref["out"]) + 1e-6).mean() > 0.99


@pytest.mark.parametrize("hd", [64, 128])
def test_scores_past_two_to_the_31_in_wide_tiles(hd):
    """As above, where a tile of rows is wider, as a request's own rows and through a shared prefix."""
    need_gpu()
    groups = [(0, 2, 96), (2, 3, 64)]
    b = Batch(n_q=4, n_kv=2, hd=hd, page=16, d=[50, 40, 1], ctx=[100, 300, 130], seed=11, prefix=groups)
    b.q, b.k = b.q * 2.0 ** 22, b.k * 2.0 ** 22
    b.dq.mul_(2.0 ** 22)
    b.dk.mul_(2.0 ** 22)
    for call in ("attn", "shared"):
        out, ls = b.run(call, groups=_groups(b, groups) if call == "shared" else None)
        ref = b.oracle()
        o = out.double().cpu().numpy()[: b.M]
        assert np.isfinite(o).all() and torch.isfinite(ls[: b.M]).all()
        assert (np.abs(o - ref["out"]) <= 2.0 ** -7 * np.abs(ref["out"]) + 1e-6).mean() > 0.99


BAD = {
    "page_minus_one": (L.DERR_PAGE, lambda b: b.dtable.__setitem__((4, 3), -1)),
    "page_past_pool": (L.DERR_PAGE, lambda b: b.dtable.__setitem__((4, 0), b.k.shape[0])),
    "negative_context": (L.DERR_CAPACITY, lambda b: b.dctx.__setitem__(4, -1)),
    "context_past_bound": (L.DERR_CAPACITY, lambda b: b.dctx.__setitem__(4, b.max_ctx - 1)),
    "huge_context": (L.DERR_CAPACITY, lambda b: b.dctx.__setitem__(4, 2 ** 31 - 1)),
}


@pytest.mark.parametrize("name", list(BAD))
def test_bad_device_data(name):
    """A fault of one request sets its bit and leaves the other requests' rows bitwise unchanged."""
    need_gpu()
    b = Batch(seed=7, **ATTN["verify"])
    b.bounds()
    sel = (4, 1, 1)
    good, _ = b.run()
    good_s, _ = b.run("sparse", sel=sel)
    bit, spoil = BAD[name]
    spoil(b)
    others = torch.tensor([t for t in range(b.M) if not b.cu[4] <= t < b.cu[5]], device="cuda")
    for call, ref in (("attn", good), ("sparse", good_s)):
        b.err.zero_()
        out, _ = b.run(call, sel=sel if call == "sparse" else None)
        torch.cuda.synchronize()
        note(f"{name} {call}: err {int(b.err.item())}")
        if call == "attn" or bit == L.DERR_CAPACITY:
            assert int(b.err.item()) == bit
        assert torch.equal(out[others], ref[others])


def test_bad_row_counts():
    """A request with more rows than max_block, decreasing cu and rows past max_rows: its bit, and no access outside."""
    need_gpu()
    b = Batch(seed=8, **ATTN["verify"])
    b.run(cfg=b.cfg(max_block=15))
    assert int(b.err.item()) == L.DERR_CAPACITY
    for i, x in ((3, 0), (9, 2 ** 30), (5, -5)):
        b = Batch(seed=8, **ATTN["verify"])
        b.dcu[i] = x
        b.run()
        torch.cuda.synchronize()
        assert int(b.err.item()) & L.DERR_CAPACITY


SHARED = {
    # whole batch, prefix a multiple of the page and not, longer and shorter than what follows
    "all": (dict(n_q=8, n_kv=2, hd=128, page=16, d=[1] * 9, ctx=[320, 321, 330, 352, 400, 320, 500, 336, 900]), [(0, 9, 320)]),
    "odd": (dict(n_q=8, n_kv=2, hd=64, page=32, d=[1, 2, 0, 3, 1], ctx=[205, 231, 207, 205, 300]), [(0, 5, 205)]),
    # groups with requests outside of them, one of a single request, an empty prefix
    "groups": (dict(n_q=9, n_kv=3, hd=64, page=16, d=[2, 1, 5, 1, 0, 3, 1, 4], ctx=[64, 70, 99, 33, 200, 129, 150, 40]),
               [(0, 3, 64), (3, 4, 33), (4, 7, 129), (7, 8, 0)]),
    # many rows a group: several tiles, several pieces of the prefix
    "tiles": (dict(n_q=16, n_kv=2, hd=128, page=64, d=[8, 1, 16, 4, 16, 2, 9], ctx=[700, 701, 760, 1000, 700, 710, 705]),
              [(0, 3, 640), (3, 7, 700)]),
    # more groups than a wave has lanes, some of them empty
    "many_groups": (dict(n_q=4, n_kv=2, hd=64, page=16, d=[1, 2] * 75, ctx=[40, 33] * 75),
                    [(3 + 10 * i + lo, 3 + 10 * i + hi, P) for i in range(14)
                     for lo, hi, P in ((0, 0, 5), (0, 1, 16), (1, 4, 33), (4, 6, 0), (6, 10, 17))]),
    "zero_own": (dict(n_q=4, n_kv=1, hd=128, page=16, d=[1, 1], ctx=[48, 48]), [(0, 2, 48)]),
    # room for many more rows than there are: prefixes cut by the largest piece
    "long": (dict(n_q=64, n_kv=8, hd=64, page=64, d=[1, 2], ctx=[4000, 3300], extra_rows=253), [(0, 1, 3999), (1, 2, 3073)]),
}


def _groups(b, groups):
    """Group descriptors: runs of consecutive requests from the first group's start; requests before the first or
    after the last run belong to none."""
    gcu = [groups[0][0]] + [g[1] for g in groups]
    return dev(np.array(gcu), torch.int32), dev(np.array([g[2] for g in groups]), torch.int32)


@pytest.mark.parametrize("name", list(SHARED))
def test_shared(name):
    need_gpu()
    shape, groups = SHARED[name]
    b = Batch(seed=9, prefix=groups, **shape)
    g = _groups(b, groups)
    out, ls = b.run("shared", groups=g)
    b.check(out, ls, b.oracle(), what=name)
    assert int(b.err.item()) == 0
    again, _ = b.run("shared", groups=g)
    assert torch.equal(out, again)


def test_shared_outside_groups():
    """Groups that leave out the first and the last requests."""
    need_gpu()
    b = Batch(n_q=8, n_kv=2, hd=128, page=16, d=[2, 1, 3, 1, 2], ctx=[90, 100, 101, 140, 7], seed=10, prefix=[(1, 4, 99)])
    g = (dev(np.array([1, 4]), torch.int32), dev(np.array([99]), torch.int32))
    out, ls = b.run("shared", groups=g)
    b.check(out, ls, b.oracle(), what="outside")


def test_shared_prefix_longer_than_a_context():
    need_gpu()
    b = Batch(n_q=8, n_kv=2, hd=128, page=16, d=[1, 1, 1], ctx=[64, 50, 64], seed=11, prefix=[(0, 3, 48)])
    out, ls = b.run("shared", groups=(dev(np.array([0, 3]), torch.int32), dev(np.array([60]), torch.int32)))
    torch.cuda.synchronize()
    assert int(b.err.item()) == L.DERR_GROUP
    for gcu, pre in (([0, 9], 10), ([2, 1], 10), ([-4, 2], 10), ([0, 3], 2 ** 31 - 1), ([0, 3], -7)):
        b.err.zero_()
        b.run("shared", groups=(dev(np.array(gcu), torch.int32), dev(np.array([pre]), torch.int32)))
        torch.cuda.synchronize()               # in bounds; the rows are unspecified


def test_shared_with_stale_and_later_rows():
    need_gpu()
    shape, groups = SHARED["groups"]
    b = Batch(seed=12, prefix=groups, stale=np.nan, **shape)
    out, ls = b.run("shared", groups=_groups(b, groups))
    b.check(out, ls, b.oracle(), what="shared stale")


SPARSE = {
    "decode": (dict(n_q=8, n_kv=2, hd=128, page=16, d=[1] * 8, ctx=[0, 15, 16, 127, 128, 500, 1500, 2999]), (8, 1, 2)),
    "verify": (dict(n_q=9, n_kv=3, hd=64, page=32, d=[3, 0, 1, 6], ctx=[400, 9, 1000, 30]), (5, 0, 1)),
    # blocks that cross a page; no pages but the forced ones; one page
    "cross": (dict(n_q=4, n_kv=2, hd=64, page=16, d=[20, 17], ctx=[310, 15]), (3, 1, 2)),
    "one": (dict(n_q=4, n_kv=1, hd=128, page=64, d=[2, 1], ctx=[200, 63]), (1, 0, 1)),
    # more pages than a workgroup has threads
    "many": (dict(n_q=4, n_kv=2, hd=64, page=16, d=[1, 2], ctx=[9000, 4200]), (40, 2, 3)),
    # more pages than one workgroup scores by itself, and than its threads keep in registers
    "long": (dict(n_q=2, n_kv=1, hd=64, page=16, d=[2, 1], ctx=[20000, 16600]), (24, 1, 2)),
    "longer": (dict(n_q=1, n_kv=1, hd=128, page=16, d=[1, 1], ctx=[70000, 900]), (100, 2, 1)),
    # more pages chosen than there are
    "all": (dict(n_q=8, n_kv=1, hd=64, page=16, d=[2, 1], ctx=[300, 20]), (64, 1, 1)),
    "group64": (dict(n_q=64, n_kv=1, hd=64, page=16, d=[1, 2], ctx=[200, 90]), (6, 1, 1)),
}


@pytest.mark.parametrize("name", list(SPARSE))
def test_sparse(name):
    need_gpu()
    shape, sel = SPARSE[name]
    b = Batch(seed=13, stale=None, **shape)
    b.bounds()
    blocks = torch.full((b.rows, b.n_kv, sel[0]), 9, dtype=torch.int32, device="cuda")
    out, ls = b.run("sparse", sel=sel, blocks=blocks)
    ref = op.paged_attn_sparse(b.q[: b.M], b.k, b.v, b.kmin, b.kmax, b.table, b.cu, b.ctx, b.page, *sel)
    torch.cuda.synchronize()
    bl = blocks.cpu().numpy()
    assert np.array_equal(bl[: b.M], ref["blocks"]) and (bl[b.M:] == 9).all()
    b.check(out, ls, ref, what=name)
    assert int(b.err.item()) == 0
    again, _ = b.run("sparse", sel=sel)
    assert torch.equal(out, again)


def test_sparse_ties_and_nan():
    """Equal bounds everywhere: the lowest pages win.  NaN bounds rank last, infinities first."""
    need_gpu()
    b = Batch(n_q=4, n_kv=2, hd=64, page=16, d=[1, 2], ctx=[5000, 700], seed=14)
    b.bounds()
    b.dkmin.fill_(-1.0)
    b.dkmax.fill_(1.0)
    sel = (10, 1, 2)
    blocks = torch.zeros(b.rows, b.n_kv, 10, dtype=torch.int32, device="cuda")
    b.run("sparse", sel=sel, blocks=blocks)
    bl = blocks.cpu().numpy()[: b.M]
    for t, p in ((0, 5000), (1, 700), (2, 701)):
        assert (bl[t] == list(range(8)) + [p // 16 - 1, p // 16]).all()
    for j in range(1, 9):
        b.dkmax[int(b.table[0, j]), 0] = float("nan")
    b.dkmax[int(b.table[0, 200]), 0] = 3e38
    b.run("sparse", sel=sel, blocks=blocks)
    bl = blocks.cpu().numpy()
    assert bl[0, 0].tolist() == [0] + list(range(9, 15)) + [200, 311, 312]
    assert bl[0, 1].tolist() == list(range(8)) + [311, 312]


def test_sparse_stale_slots():
    need_gpu()
    shape, sel = SPARSE["cross"]
    b = Batch(seed=15, stale=None, **shape)
    b.bounds()
    c = Batch(seed=15, stale=np.nan, **shape)
    c.bounds()
    out, _ = b.run("sparse", sel=sel)
    c.dkmin, c.dkmax = b.dkmin, b.dkmax
    got, _ = c.run("sparse", sel=sel)
    assert torch.equal(out[: b.M], got[: b.M])


APPEND = {
    "decode": dict(n_q=8, n_kv=2, hd=128, page=16, d=[1] * 6, ctx=[0, 15, 16, 31, 100, 7]),
    "verify": dict(n_q=9, n_kv=3, hd=64, page=32, d=[0, 4, 1, 33, 2], ctx=[5, 31, 0, 0, 62]),
    "prompt": dict(n_q=4, n_kv=1, hd=128, page=16, d=[150, 0, 70], ctx=[3, 8, 0]),
    "big_page": dict(n_q=2, n_kv=2, hd=64, page=256, d=[300, 1], ctx=[0, 255]),
}


def _append_case(b, dtype, seed, qkv=None):
    rng = np.random.default_rng(seed)
    nq, nkv = b.n_q * b.hd, b.n_kv * b.hd
    x = rng.standard_normal((b.rows, nq + 2 * nkv)).astype(np.float32) if qkv is None else qkv
    buf = torch.zeros(b.rows, nq + 2 * nkv + 8, dtype=dtype, device="cuda")
    buf[:, : nq + 2 * nkv] = torch.from_numpy(x).cuda()
    q, k, v = buf[:, :nq], buf[:, nq: nq + nkv], buf[:, nq + nkv: nq + 2 * nkv]
    req = np.pad(np.repeat(np.arange(b.B), b.d), (0, b.rows - b.M))
    pos = np.pad(np.concatenate([b.ctx[i] + np.arange(b.d[i]) for i in range(b.B)]), (0, b.rows - b.M))
    val = buf.double().cpu().numpy()
    split = lambda a, n: a.reshape(b.rows, n, b.hd)
    return q, k, v, pos, req, split(val[:, :nq], b.n_q), split(val[:, nq: nq + nkv], b.n_kv), split(val[:, nq + nkv: nq + 2 * nkv], b.n_kv)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("name", list(APPEND))
def test_append(name, dtype):
    """q and the keys within one rounding to bf16 of the oracle (2^-8 relative to the value, and the float32 rotation's
    2^-22 of the pair's size), values exactly rounded, every other slot bitwise as it was; bounds of the pages filled."""
    need_gpu()
    b = Batch(seed=16, **APPEND[name])
    b.bounds()
    q, k, v, pos, req, xq, xk, xv = _append_case(b, dtype, 17)
    k0, v0, lo0, hi0 = (x.clone() for x in (b.dk, b.dv, b.dkmin, b.dkmax))
    q_out = torch.full((b.rows, b.n_q, b.hd), 7.0, dtype=torch.bfloat16, device="cuda")
    L.paged_append(b.cfg(), b.pages(), b.B, b.dcu, dev(pos, torch.int32), dev(req, torch.int32), q, k, v, q_out, THETA, dev_err=b.err)
    torch.cuda.synchronize()
    assert int(b.err.item()) == 0
    M, half = b.M, b.hd // 2

    def near(got, x, ref):
        size = np.hypot(x[..., :half], x[..., half:])
        tol = 2.0 ** -8 * np.abs(ref) + 2.0 ** -21 * np.concatenate([size, size], -1)
        assert (np.abs(got - ref) <= tol).all(), np.abs(got - ref).max()

    near(q_out[:M].double().cpu().numpy(), xq[:M], op.rotate(xq[:M], pos[:M], THETA))
    assert (q_out[M:] == 7.0).all()
    kk, vv = b.dk.double().cpu().numpy(), b.dv.double().cpu().numpy()
    pg, sl = b.table[req[:M], pos[:M] // b.page], pos[:M] % b.page
    near(kk[pg, :, sl], xk[:M], op.rotate(xk[:M], pos[:M], THETA))
    assert np.array_equal(vv[pg, :, sl], bf(xv[:M]))
    touched = torch.zeros(b.dk.shape[0], b.page, dtype=torch.bool, device="cuda")
    touched[torch.from_numpy(pg).long().cuda(), torch.from_numpy(sl).long().cuda()] = True
    keep = ~touched[:, None, :, None].expand_as(b.dk)
    assert torch.equal(b.dk[keep], k0[keep]) and torch.equal(b.dv[keep], v0[keep])
    full = np.unique(pg[sl == b.page - 1])
    lo, hi = b.dkmin.double().cpu().numpy(), b.dkmax.double().cpu().numpy()
    assert np.array_equal(lo[full], kk[full].min(2)) and np.array_equal(hi[full], kk[full].max(2))
    rest = torch.tensor(sorted(set(range(len(lo))) - set(full.tolist())), device="cuda")
    assert torch.equal(b.dkmin[rest], lo0[rest]) and torch.equal(b.dkmax[rest], hi0[rest])
    # without queries and without bounds: the same pages
    k1, v1 = b.dk.clone(), b.dv.clone()
    b.dk.copy_(k0)
    b.dv.copy_(v0)
    b.dkmin = b.dkmax = None
    L.paged_append(b.cfg(), b.pages(), b.B, b.dcu, dev(pos, torch.int32), dev(req, torch.int32), None, k, v, None, THETA)
    assert torch.equal(b.dk, k1) and torch.equal(b.dv, v1)


def test_append_far_positions():
    need_gpu()
    pos = np.array([0, 1, 65535, 1000003, 2 ** 24 - 1])
    B, page = len(pos), 256
    cfg = L.paged_cfg(2, 1, 128, page, 2 ** 24, 1, B)
    table = torch.full((B, 2 ** 24 // page), -1, dtype=torch.int32, device="cuda")
    for i, p in enumerate(pos):
        table[i, p // page] = B - 1 - i
    k, v = (torch.zeros(B, 1, page, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x = np.random.default_rng(18).standard_normal((B, 4, 128)).astype(np.float32)
    xd = torch.from_numpy(x).cuda()
    q_out = torch.zeros(B, 2, 128, dtype=torch.bfloat16, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    L.paged_append(cfg, L.pages_desc(k, v, table), B, dev(np.arange(B + 1), torch.int32), dev(pos, torch.int32),
                   dev(np.arange(B), torch.int32), xd[:, :2].reshape(B, -1), xd[:, 2:3].reshape(B, -1), xd[:, 3:].reshape(B, -1),
                   q_out, 1e4, dev_err=err)
    torch.cuda.synchronize()
    ref = op.rotate(x.astype(np.float64), pos, 1e4)
    size = np.hypot(x[..., :64], x[..., 64:])
    tol = 2.0 ** -8 * np.abs(ref) + 2.0 ** -21 * np.concatenate([size, size], -1)
    got = np.concatenate([q_out.double().cpu().numpy(), np.stack([k[B - 1 - i, :, int(p) % page].double().cpu().numpy() for i, p in enumerate(pos)])], 1)
    assert int(err.item()) == 0 and (np.abs(got - ref[:, :3]) <= tol[:, :3]).all()


def test_append_bad_rows():
    """Rows of no request, past the table or on a bad page are left out, the others appended, queries rotated."""
    need_gpu()
    b = Batch(n_q=4, n_kv=2, hd=64, page=16, d=[1] * 6, ctx=[3, 20, 40, 40, 40, 40], seed=19)
    q, k, v, pos, req, xq, xk, xv = _append_case(b, torch.bfloat16, 20)
    good_k = b.dk.clone()
    q_out = torch.zeros(b.rows, 4, 64, dtype=torch.bfloat16, device="cuda")
    args = lambda: (b.cfg(), b.pages(), b.B, b.dcu, dev(pos, torch.int32), dev(req, torch.int32), q, k, v, q_out, THETA)
    for i, (spoil, bit) in enumerate([(lambda: req.__setitem__(2, 6), L.DERR_CAPACITY), (lambda: req.__setitem__(3, -1), L.DERR_CAPACITY),
                                      (lambda: pos.__setitem__(4, 10 ** 6), L.DERR_CAPACITY), (lambda: pos.__setitem__(5, -1), L.DERR_CAPACITY),
                                      (lambda: b.dtable.__setitem__((1, 1), 10 ** 6), L.DERR_PAGE)]):
        spoil()
        b.err.zero_()
        L.paged_append(*args(), dev_err=b.err)
        torch.cuda.synchronize()
        assert int(b.err.item()) & bit, i
    b.dk.copy_(good_k)
    L.paged_append(*args())
    torch.cuda.synchronize()
    changed = (b.dk != good_k).flatten(1).any(1).nonzero().flatten().tolist()
    assert changed == [int(b.table[0, 0])]


def test_offsets_past_32_bits():
    """A pool of more than 4 GiB for keys and as much for values: pages at its far end."""
    need_gpu()
    n_kv, page, hd = 8, 256, 128
    n_pages = (5 << 30) // (n_kv * page * hd * 2)
    rng = np.random.default_rng(21)
    k, v = (torch.zeros(n_pages, n_kv, page, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ids = np.array([[n_pages - 1, 3, n_pages - 7], [n_pages - 2, n_pages // 2, 5]])
    kk, vv = bf(rng.standard_normal((6, n_kv, page, hd))), bf(rng.standard_normal((6, n_kv, page, hd)))
    at = torch.from_numpy(ids.reshape(-1)).cuda()
    k[at], v[at] = dev(kk), dev(vv)
    d, ctx = np.array([2, 1]), np.array([700, 600])
    cu = np.array([0, 2, 3], dtype=np.int32)
    q = bf(rng.standard_normal((3, 32, hd)))
    small = np.arange(6).reshape(2, 3)
    cfg = L.paged_cfg(32, n_kv, hd, page, 768, 2, 3)
    out, lse = torch.zeros(3, 32, hd, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, 32, device="cuda")
    ws = L.workspace(L.paged_workspace_bytes("attn", cfg, 2))
    pages = L.pages_desc(k, v, dev(ids, torch.int32))
    dcu, dctx = dev(cu, torch.int32), dev(ctx, torch.int32)
    # append three new keys there first
    x = rng.standard_normal((3, 48 * hd)).astype(np.float32)
    xd = torch.from_numpy(x).cuda()
    pos, req = np.array([700, 701, 600]), np.array([0, 0, 1])
    L.paged_append(cfg, pages, 2, dcu, dev(pos, torch.int32), dev(req, torch.int32), None, xd[:, 32 * hd: 40 * hd], xd[:, 40 * hd:],
                   None, THETA)
    x = x.astype(np.float64).reshape(3, 48, hd)
    for t in range(3):
        pg, s = small[req[t], pos[t] // page], pos[t] % page
        kk[pg, :, s], vv[pg, :, s] = bf(op.rotate(x[t: t + 1, 32:40], pos[t: t + 1], THETA)[0]), bf(x[t, 40:])
    L.paged_attn(cfg, pages, 2, dev(q), dcu, dctx, out, ws, lse=lse)
    ref = op.paged_attn(q, kk, vv, small, cu, ctx, page)
    torch.cuda.synchronize()
    # a key may round to the other neighbour than the oracle's where the float32 rotation lies next to the middle
    tol = ref["mag"] * (2 * 2.0 ** -8 * 1.01 + 2.0 ** -8 + (3 * 2.0 ** -17) * (1 + ref["big"][:, :, None]))
    assert (np.abs(out.double().cpu().numpy() - ref["out"]) <= tol).all()


def test_serving_steps():
    """A layer's cache over several steps as an engine uses it: a prompt in pieces, decoding, a verified block of which
    some drafts are rejected and written over, then sparse decoding; each step's rows against the oracle's cache."""
    need_gpu()
    n_q, n_kv, hd, page, B = 8, 2, 64, 16, 3
    rng = np.random.default_rng(22)
    ld = 20
    table = rng.permutation(B * ld + 1)[: B * ld].reshape(B, ld).astype(np.int32)
    k, v = (torch.full((B * ld + 1, n_kv, page, hd), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kmin, kmax = (torch.zeros(B * ld + 1, n_kv, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pages = L.pages_desc(k, v, dev(table, torch.int32), kmin, kmax)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    keep = []
    ctx = np.zeros(B, dtype=np.int64)
    sel = (5, 1, 2)
    for step, (d, back) in enumerate([([40, 70, 3], 0), ([60, 0, 90], 0), ([1, 1, 1], 0), ([6, 6, 4], 3), ([6, 6, 4], 0), ([1, 1, 1], 0)]):
        d = np.array(d)
        M = int(d.sum())
        cu = np.concatenate([[0], np.cumsum(d)]).astype(np.int32)
        req = np.repeat(np.arange(B), d)
        pos = np.concatenate([ctx[i] + np.arange(d[i]) for i in range(B)])
        x = torch.from_numpy(rng.standard_normal((M, (n_q + 2 * n_kv) * hd)).astype(np.float32)).cuda().bfloat16()
        cfg = L.paged_cfg(n_q, n_kv, hd, page, ld * page, int(d.max()), M)
        q_out = torch.zeros(M, n_q, hd, dtype=torch.bfloat16, device="cuda")
        out, lse = torch.zeros_like(q_out), torch.zeros(M, n_q, device="cuda")
        dcu, dctx = dev(cu, torch.int32), dev(ctx, torch.int32)
        L.paged_append(cfg, pages, B, dcu, dev(pos, torch.int32), dev(req, torch.int32), x[:, : n_q * hd], x[:, n_q * hd: (n_q + n_kv) * hd],
                       x[:, (n_q + n_kv) * hd:], q_out, THETA, dev_err=err)
        blocks = None
        if step < 5:
            L.paged_attn(cfg, pages, B, q_out, dcu, dctx, out, L.workspace(L.paged_workspace_bytes("attn", cfg, B)), lse=lse, dev_err=err)
        else:
            blocks = torch.zeros(M, n_kv, sel[0], dtype=torch.int32, device="cuda")
            L.paged_attn_sparse(cfg, pages, B, q_out, dcu, dctx, out, L.workspace(L.paged_workspace_bytes("sparse", cfg, B, sel[0])),
                                *sel, blocks=blocks, lse=lse, dev_err=err)
        torch.cuda.synchronize()
        kk, vv, qq = (t.double().cpu().numpy() for t in (k, v, q_out))
        if blocks is None:
            ref = op.paged_attn(qq, kk, vv, table, cu, ctx, page)
        else:
            with np.errstate(invalid="ignore"):
                ref = op.paged_attn_sparse(qq, kk, vv, kk.min(2), kk.max(2), table, cu, ctx, page, *sel)
            assert np.array_equal(blocks.cpu().numpy(), ref["blocks"])
        tol = ref["mag"] * (2 * 2.0 ** -8 * 1.01 + (3 * 2.0 ** -17) * (1 + ref["big"][:, :, None]))
        assert (np.abs(out.double().cpu().numpy() - ref["out"]) <= tol).all(), step
        assert int(err.item()) == 0
        ctx = ctx + d - np.minimum(back, d)


def test_captured_graphs():
    """append and the three attention calls captured once, replayed on new inputs, contexts and row counts with the
    program's own work between the replays; two graphs with workspaces of their own."""
    need_gpu()
    b = Batch(n_q=8, n_kv=2, hd=128, page=16, d=[3, 1, 4, 2], ctx=[130, 145, 300, 129], seed=23, prefix=[(0, 4, 128)], slack=2)
    b.bounds()
    cfg, sel = b.cfg(max_ctx=320, max_block=4), (6, 1, 2)
    g = (dev(np.array([0, 4]), torch.int32), dev(np.array([128]), torch.int32))
    q, k, v, pos, req, *_ = _append_case(b, torch.bfloat16, 24)
    dpos, dreq = dev(pos, torch.int32), dev(req, torch.int32)
    q_out = torch.zeros(b.rows, 8, 128, dtype=torch.bfloat16, device="cuda")
    outs = [torch.zeros_like(q_out) for _ in range(3)]
    wss = [L.workspace(L.paged_workspace_bytes(c, cfg, b.B, sel[0])) for c in ("attn", "shared", "sparse")]
    pages = b.pages()

    def step(stream=None):
        L.paged_append(cfg, pages, b.B, b.dcu, dpos, dreq, q, k, v, q_out, THETA, dev_err=b.err)
        a = lambda i: (cfg, pages, b.B, q_out, b.dcu, b.dctx, outs[i], wss[i])
        L.paged_attn(*a(0), dev_err=b.err)
        L.paged_attn_shared(*a(1), *g, dev_err=b.err)
        L.paged_attn_sparse(*a(2), *sel, dev_err=b.err)

    step()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            step()
        graphs.append(gr)
    rng = np.random.default_rng(25)
    for it in range(6):
        d = rng.integers(0, 5, size=4)
        cu = np.concatenate([[0], np.cumsum(d)]).astype(np.int32)
        ctx = np.array([128, 140, 290, 128]) + rng.integers(0, 8, size=4)
        M = int(cu[-1])
        if M > b.rows:
            continue
        npos = np.pad(np.concatenate([ctx[i] + np.arange(d[i]) for i in range(4)]), (0, b.rows - M))
        b.dcu.copy_(torch.from_numpy(cu))
        b.dctx.copy_(torch.from_numpy(ctx.astype(np.int32)))
        dpos.copy_(torch.from_numpy(npos.astype(np.int32)))
        dreq.copy_(torch.from_numpy(np.pad(np.repeat(np.arange(4), d), (0, b.rows - M)).astype(np.int32)))
        q.copy_(torch.randn_like(q.float()).bfloat16())
        for x in outs:
            x.zero_()
        graphs[it % 2].replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in outs]
        for x in outs:
            x.zero_()
        step()
        torch.cuda.synchronize()
        for x, y in zip(got, outs):
            assert torch.equal(x[:M], y[:M]) and (x[M:] == 0).all()
    assert int(b.err.item()) == 0


def test_two_streams():
    """The same call on two side streams at once, with workspaces of their own."""
    need_gpu()
    b = Batch(seed=26, **ATTN["verify"])
    want, _ = b.run()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    cfg = b.cfg()
    wss = [L.workspace(L.paged_workspace_bytes("attn", cfg, b.B)) for _ in range(2)]
    outs = [b.outputs()[0] for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, ws, o in zip(streams, wss, outs):
            L.paged_attn(cfg, b.pages(), b.B, b.dq, b.dcu, b.dctx, o, ws, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


@pytest.mark.parametrize("cid", [2, 4])
def test_selected_rows_of_the_step(cid):
    """dcut_select's packed rows as the rows of a paged layer: heads of the repository's layers, kept blocks of a step."""
    need_gpu()
    c = wl.CONFIGS[cid]
    ly = c.layer
    B, D = 6, 15
    rng = np.random.default_rng(27)
    ctx = rng.integers(100, 400, size=B)
    sel = L.select_outputs(B, D, 1)
    conf = dev(rng.random((B, D)).astype(np.float32) ** 0.2, torch.float32)
    L.select(B, D, conf, dev(rng.integers(0, 99, (B, D + 1)), torch.int32), dev(ctx, torch.int32), [30], [1.0], sel)
    torch.cuda.synchronize()
    cu = sel["cu"].cpu().numpy()
    b = Batch(ly.n_q, ly.n_kv, ly.head_dim, 32, np.diff(cu), ctx, seed=28, extra_rows=B * (D + 1) - int(cu[-1]))
    q, k, v, *_ = _append_case(b, torch.bfloat16, 29)
    cfg = b.cfg(max_block=D + 1, max_ctx=int(ctx.max()) + D + 1)
    q_out, _ = b.outputs()
    L.paged_append(cfg, b.pages(), B, sel["cu"], sel["packed_pos"], sel["packed_req"], q, k, v, q_out, ly.rope_theta, dev_err=b.err)
    out, ls = b.outputs()
    L.paged_attn(cfg, b.pages(), B, q_out, sel["cu"], b.dctx, out, L.workspace(L.paged_workspace_bytes("attn", cfg, B)), lse=ls, dev_err=b.err)
    torch.cuda.synchronize()
    b.q, b.k, b.v = (x.double().cpu().numpy() for x in (q_out, b.dk, b.dv))
    b.check(out, ls, b.oracle(), what=c.name)


def _keep(b, d2):
    """The batch with only the first d2[i] new rows of each request kept: queries packed again, cu, old and new row
    numbers."""
    cu2 = np.concatenate([[0], np.cumsum(d2)]).astype(np.int32)
    old = np.concatenate([np.arange(b.cu[i], b.cu[i] + d2[i]) for i in range(b.B)])
    q2 = b.dq.clone()
    q2[: len(old)] = b.dq[torch.from_numpy(old).cuda()]
    b.dq = q2
    b.dcu.copy_(torch.from_numpy(cu2))
    return torch.from_numpy(old).cuda(), torch.arange(len(old), device="cuda")


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n_q,kept", [(2, 100), (2, 70), (2, 130), (8, 41), (8, 30)])
def test_wide_rows_do_not_depend_on_the_rows_kept(hd, n_q, kept):
    """160 rows a request against fewer: waves partly filled, and steps of keys that only the request's later rows see.
    The rows that stay are bitwise what they were."""
    need_gpu()
    ctx = [90, 0, 31, 64, 104, 127]
    b = Batch(n_q=n_q, n_kv=2, hd=hd, page=16, d=[160] * len(ctx), ctx=ctx, seed=31)
    cfg = b.cfg()
    out, ls = b.run(cfg=cfg)
    old, new = _keep(b, [kept] * b.B)
    out2, ls2 = b.run(cfg=cfg)
    torch.cuda.synchronize()
    assert torch.equal(out[old], out2[new]) and torch.equal(ls[old], ls2[new])


@pytest.mark.parametrize("value", [np.inf, -np.inf, 2.0 ** 60])
@pytest.mark.parametrize("name", ["wide", "prompt", "prompt64", "verify"])
def test_one_channel_of_a_later_key_never_reaches_earlier_rows(name, value):
    """One channel of the last row's key is infinite or far above the others, so that its scores are, not NaN: earlier
    rows are bitwise what they were."""
    need_gpu()
    b = Batch(seed=32, **ATTN[name])
    out, ls = b.run()
    rows = []
    for i in range(b.B):
        if b.d[i]:
            p = int(b.ctx[i] + b.d[i] - 1)
            b.dk[int(b.table[i, p // b.page]), :, p % b.page, 5] = value
            rows += list(range(b.cu[i], b.cu[i + 1] - 1))
    got, gls = b.run()
    torch.cuda.synchronize()
    rows = torch.tensor(rows, device="cuda")
    assert torch.equal(out[rows], got[rows]) and torch.equal(ls[rows], gls[rows])


@pytest.mark.parametrize("hd", [64, 128])
def test_shared_rows_do_not_depend_on_a_members_queries(hd):
    """One member's queries are scaled by 2^34 (its scores pass 2^31): the others' rows are bitwise what they were."""
    need_gpu()
    groups = [(0, 4, 200)]
    b = Batch(n_q=4, n_kv=2, hd=hd, page=16, d=[3, 40, 1, 5], ctx=[210, 240, 200, 330], seed=33, prefix=groups)
    g = _groups(b, groups)
    out, ls = b.run("shared", groups=g)
    b.dq[b.cu[2]: b.cu[3]] *= 2.0 ** 34
    got, gls = b.run("shared", groups=g)
    torch.cuda.synchronize()
    others = torch.tensor([t for t in range(b.M) if not b.cu[2] <= t < b.cu[3]], device="cuda")
    assert torch.equal(out[others], got[others]) and torch.equal(ls[others], gls[others])


@pytest.mark.parametrize("page,P,d", [(16, 16, 1), (16, 48, 1), (16, 50, 2), (16, 16, 40), (16, 48, 40), (32, 32, 40), (32, 96, 17)])
def test_shared_reads_prefixes_through_the_first_member_only(page, P, d):
    """The prefix's columns of the other members' tables are unset: right rows and no fault, whatever the prefix's place
    within a step of keys."""
    need_gpu()
    groups = [(0, 3, P)]
    b = Batch(n_q=8, n_kv=2, hd=64, page=page, d=[1, d, 2], ctx=[P + 5, P, P + 70], seed=34, prefix=groups)
    ref = b.oracle()
    b.dtable[1:, : P // page] = -1
    out, ls = b.run("shared", groups=_groups(b, groups))
    b.check(out, ls, ref, what=f"page {page} prefix {P}")
    assert int(b.err.item()) == 0


@pytest.mark.parametrize("end", [9, 2 ** 31 - 1, -3])
def test_append_row_counts_outside_the_bounds(end):
    """cu[B] above max_rows, or negative: its bit; the rows up to max_rows are appended, no others are touched."""
    need_gpu()
    b = Batch(n_q=4, n_kv=2, hd=64, page=16, d=[1] * 9, ctx=[3, 20, 40, 15, 31, 7, 0, 16, 2], seed=35)
    b.bounds()
    q, k, v, pos, req, *_ = _append_case(b, torch.bfloat16, 36)
    k0 = b.dk.clone()
    q_out = torch.full((b.rows, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    b.dcu[b.B] = end
    L.paged_append(b.cfg(max_rows=6), b.pages(), b.B, b.dcu, dev(pos, torch.int32), dev(req, torch.int32), q, k, v, q_out, THETA,
                   dev_err=b.err)
    torch.cuda.synchronize()
    live = 6 if end > 0 else 0
    assert int(b.err.item()) == L.DERR_CAPACITY
    assert (q_out[live:] == 7.0).all() and (q_out[:live] != 7.0).any(-1).all()
    changed = (b.dk != k0).flatten(1).any(1).nonzero().flatten().tolist()
    assert sorted(changed) == sorted(int(b.table[i, b.ctx[i] // 16]) for i in range(live))


def test_sparse_and_shared_bad_row_counts():
    """Requests whose rows lie past max_rows, or that end before they start: their bit, other rows bitwise unchanged."""
    need_gpu()
    sel = (4, 1, 1)
    for call in ("sparse", "shared"):
        b = Batch(n_q=4, n_kv=2, hd=64, page=16, d=[6, 5], ctx=[200, 300], seed=37, prefix=[(0, 2, 160)])
        b.bounds()
        cfg = b.cfg(max_rows=6)
        kw = dict(cfg=cfg, sel=sel) if call == "sparse" else dict(cfg=cfg, groups=_groups(b, [(0, 2, 160)]))
        b.dcu.copy_(torch.tensor([0, 6, 6]))
        want, _ = b.run(call, **kw)
        assert int(b.err.item()) == 0
        for cu in ([0, 6, 11], [0, 6, 2 ** 31 - 1], [0, 6, 4]):
            b.err.zero_()
            b.dcu.copy_(torch.tensor(cu))
            got, _ = b.run(call, **kw)
            torch.cuda.synchronize()
            note(f"{call} cu {cu}: err {int(b.err.item())}")
            assert int(b.err.item()) == L.DERR_CAPACITY
            if call == "sparse" and cu[2] > 6:
                assert torch.equal(want[:6], got[:6])
            assert (got[6:] == 7.0).all()


@pytest.mark.parametrize("shape,sel", [(dict(n_q=8, n_kv=2, hd=128, page=16, d=[1, 2], ctx=[1500, 700]), (8, 1, 2)),
                                       (dict(n_q=2, n_kv=1, hd=64, page=16, d=[1, 1], ctx=[300, 20000]), (8, 1, 2))])
@pytest.mark.parametrize("entry", [-1, 2 ** 30])
def test_sparse_reports_pages_that_are_not_chosen(shape, sel, entry):
    """A bad table entry among the pages that a row may choose from: its bit, wherever its score would have put it."""
    need_gpu()
    b = Batch(seed=38, **shape)
    b.bounds()
    blocks = torch.zeros(b.rows, b.n_kv, sel[0], dtype=torch.int32, device="cuda")
    want, _ = b.run("sparse", sel=sel, blocks=blocks)
    assert int(b.err.item()) == 0
    i = b.B - 1
    last = b.M - 1
    rows = list(range(b.cu[i], b.cu[i + 1]))
    chosen = set(blocks[rows].flatten().tolist())
    page0 = int((b.dtable[i] == 0).nonzero()) if bool((b.dtable[i] == 0).any()) else -1
    free = [j for j in range(2, int(b.ctx[i]) // b.page - 2) if j not in chosen and j != page0]
    for j in (free[0], free[len(free) // 2], free[-1]):
        b.err.zero_()
        good = int(b.dtable[i, j])
        # the entry takes the place of a page whose bounds nobody prefers
        b.dtable[i, j] = entry
        b.dkmin[0], b.dkmax[0] = 0.0, -1e30
        got, _ = b.run("sparse", sel=sel)
        torch.cuda.synchronize()
        assert int(b.err.item()) == L.DERR_PAGE, j
        others = torch.tensor([t for t in range(b.M) if t not in rows], device="cuda")
        assert torch.isfinite(got[others].float()).all()
        b.dtable[i, j] = good


def test_sparse_nan_queries():
    """A NaN in a query makes every score of its row and kv head NaN: all pages tie, the lowest are read.  Other rows and
    kv heads choose as before."""
    need_gpu()
    for shape, sel in ((dict(n_q=8, n_kv=2, hd=128, page=16, d=[1, 2], ctx=[1500, 700]), (8, 1, 2)),
                       (dict(n_q=4, n_kv=2, hd=64, page=16, d=[1], ctx=[20000]), (8, 0, 1))):
        b = Batch(seed=39, **shape)
        b.bounds()
        b.q[0, 1, 7] = np.nan
        b.dq[0, b.hd + 7] = float("nan")
        blocks = torch.zeros(b.rows, b.n_kv, sel[0], dtype=torch.int32, device="cuda")
        out, _ = b.run("sparse", sel=sel, blocks=blocks)
        want = op.paged_attn_sparse(b.q[: b.M], b.k, b.v, b.kmin, b.kmax, b.table, b.cu, b.ctx, b.page, *sel)["blocks"]
        bl = blocks.cpu().numpy()[: b.M]
        assert bl[0, 0].tolist() == list(range(sel[0] - sel[2])) + [b.ctx[0] // 16 - j for j in reversed(range(sel[2]))]
        assert np.array_equal(bl, want)
        o = out.float()
        assert torch.isnan(o[0, 1]).all() and torch.isfinite(o[0, 0]).all() and torch.isfinite(o[1: b.M]).all()


@pytest.mark.parametrize("max_rows", [64, 60000])
def test_bad_row_counts_in_tiles(max_rows):
    """A request that ends before it starts, in a launch of several tiles a request, listed longest first or not: its bit,
    though no tile is its own."""
    need_gpu()
    b = Batch(n_q=8, n_kv=2, hd=64, page=16, d=[40, 2, 1], ctx=[100, 30, 7], seed=40, extra_rows=max_rows - 43)
    b.dcu.copy_(torch.tensor([0, 40, 20, 20]))
    b.run(lse=False)
    torch.cuda.synchronize()
    assert int(b.err.item()) == L.DERR_CAPACITY


# Launches of more work items than are dispatched as they come (1024: requests' tiles x kv heads x pieces), whose items
# are listed longest first.
PLANNED = {
    # 64 requests x 2 kv heads x up to 11 pieces of 128 keys
    "decode": dict(n_q=8, n_kv=2, hd=128, page=16, d=[1] * 64, ctx=[(j * j * 37) % 1300 for j in range(64)]),
    "verify": dict(n_q=8, n_kv=2, hd=64, page=32, d=[j % 9 for j in range(64)], ctx=[(j * 211) % 1300 for j in range(64)]),
    # room for 20000 rows: 161 tiles of 128 (row, head) pairs x 8 kv heads, few of them with rows
    "prompt": dict(n_q=8, n_kv=8, hd=64, page=16, d=[150, 0, 1, 97, 200], ctx=[0, 3, 500, 63, 10], extra_rows=20000 - 448),
    # room for 10000 rows of 16 heads in groups of 4: 317 tiles x 4 kv heads
    "groups": dict(n_q=16, n_kv=4, hd=128, page=64, d=[33, 1, 40, 0, 3], ctx=[100, 900, 0, 5, 301], extra_rows=10000 - 77),
}


@pytest.mark.parametrize("name", list(PLANNED))
def test_attn_listed_longest_first(name):
    need_gpu()
    b = Batch(seed=41, **PLANNED[name])
    out, ls = b.run()
    b.check(out, ls, b.oracle(), what=name)
    assert int(b.err.item()) == 0
    again, ls2 = b.run()
    assert torch.equal(out, again) and torch.equal(ls, ls2)


def test_attn_pieces_of_2048_keys():
    """As many (request, kv head) pairs as work items are aimed at: a request's pieces are cut at 2048 keys, here up to 69
    of them, more than the merge takes at a time."""
    need_gpu()
    ctx = [140000, 5000, 2046, 2047, 2048, 4095, 4096] + [j % 40 for j in range(1529)]
    b = Batch(n_q=2, n_kv=1, hd=64, page=64, d=[1] * len(ctx), ctx=ctx, seed=42)
    out, ls = b.run()
    b.check(out, ls, b.oracle(), what="pieces")
    assert int(b.err.item()) == 0


@pytest.mark.parametrize("name", ["decode", "verify", "wide", "group64", "prompt", "prompt64"])
def test_bounds_far_above_the_batch(name):
    """One launch serves every batch within its bounds: contexts, blocks and row counts far below them."""
    need_gpu()
    b = Batch(seed=43, extra_rows=700, **ATTN[name])
    for kw in (dict(max_ctx=100000), dict(max_block=64 if b.max_block < 64 else 1000, max_ctx=70000)):
        out, ls = b.run(cfg=b.cfg(**kw))
        b.check(out, ls, b.oracle(), what=f"{name} {kw}")
        assert int(b.err.item()) == 0


@pytest.mark.parametrize("name,listed", [("wide", False), ("prompt", False), ("prompt", True), ("prompt64", False), ("prompt64", True)])
def test_bad_device_data_in_tiles(name, listed):
    """A fault of one request sets its bit and leaves the other requests' rows bitwise unchanged: wide tiles, dispatched as
    they come and listed longest first."""
    need_gpu()
    shape = ATTN[name]
    i = 2
    spoils = [(L.DERR_PAGE, lambda b: b.dtable.__setitem__((i, 0), -1)),
              (L.DERR_PAGE, lambda b: b.dtable.__setitem__((i, int(b.ctx[i] + b.d[i] - 1) // b.page), b.k.shape[0])),
              (L.DERR_CAPACITY, lambda b: b.dctx.__setitem__(i, -1)),
              (L.DERR_CAPACITY, lambda b: b.dctx.__setitem__(i, 2 ** 31 - 1))]
    for bit, spoil in spoils:
        b = Batch(seed=44, extra_rows=40000 if listed else 3, **shape)
        want, _ = b.run()
        assert int(b.err.item()) == 0
        spoil(b)
        got, _ = b.run()
        torch.cuda.synchronize()
        others = torch.tensor([t for t in range(b.M) if not b.cu[i] <= t < b.cu[i + 1]], device="cuda")
        assert int(b.err.item()) == bit
        assert torch.equal(want[others], got[others]) and (got[b.M:] == 7.0).all()


@pytest.mark.parametrize("name,call", [("verify", "attn"), ("wide", "attn"), ("prompt64", "attn"), ("verify", "sparse"), ("tiles", "shared"),
                                       ("groups", "shared")])
def test_rows_without_a_finite_score(name, call):
    """Every score of some rows is minus infinity: they give 0 and a log sum of minus infinity, the other rows what they
    gave."""
    need_gpu()
    shape, groups = SHARED[name] if call == "shared" else (ATTN[name], ())
    b = Batch(seed=45, prefix=groups, **shape)
    q = b.dq.view(b.rows, b.n_q, b.hd)
    q[:, :, 7] = 0.0                               # the channel in which the rows below differ from the others
    b.k[..., 7] = bf(np.array(-1e38))
    b.dk[..., 7] = -1e38
    b.bounds()
    kw = dict(groups=_groups(b, groups)) if call == "shared" else dict(sel=(4, 1, 1)) if call == "sparse" else {}
    want, wls = b.run(call, **kw)
    rows = torch.tensor([t for t in range(b.M) if t % 3 == 1], device="cuda")
    others = torch.tensor([t for t in range(b.M) if t % 3 != 1], device="cuda")
    q[rows, :, 7] = 1e38
    out, ls = b.run(call, **kw)
    torch.cuda.synchronize()
    assert (out[rows] == 0).all() and torch.isneginf(ls[rows]).all()
    assert torch.equal(out[others], want[others]) and torch.equal(ls[others], wls[others])
    assert torch.isfinite(wls[: b.M]).all() and int(b.err.item()) == 0


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("heads", [dict(n_q=4, n_kv=2, hd=64), dict(n_q=12, n_kv=2, hd=128), dict(n_q=64, n_kv=1, hd=64)])
def test_every_page_size(page, heads):
    """Each page size in every call, streamed and wide, with contexts and a prefix that end within a page."""
    need_gpu()
    P = 300
    for d in ([1, 2, 0, 1], [40, 1, 33, 2]):
        b = Batch(page=page, d=d, ctx=[P + 5, P + 260, P, P + 31], seed=46, prefix=[(0, 3, P)], **heads)
        b.bounds()
        ref = b.oracle()
        out, ls = b.run()
        b.check(out, ls, ref, what=f"page {page}")
        g = (dev(np.array([0, 3]), torch.int32), dev(np.array([P]), torch.int32))
        out, ls = b.run("shared", groups=g)
        b.check(out, ls, ref, what=f"page {page} shared")
        sel = (2, 0, 1)
        blocks = torch.zeros(b.rows, b.n_kv, sel[0], dtype=torch.int32, device="cuda")
        out, ls = b.run("sparse", sel=sel, blocks=blocks)
        ref = op.paged_attn_sparse(b.q[: b.M], b.k, b.v, b.kmin, b.kmax, b.table, b.cu, b.ctx, b.page, *sel)
        assert np.array_equal(blocks.cpu().numpy()[: b.M], ref["blocks"])
        b.check(out, ls, ref, what=f"page {page} sparse")
        assert int(b.err.item()) == 0


@pytest.mark.parametrize("call,shape", [("attn", dict(n_q=8, n_kv=2, hd=128, page=16, d=[2, 1, 3, 1], ctx=[300, 700, 500, 900])),
                                        ("attn", dict(n_q=8, n_kv=2, hd=64, page=16, d=[2, 40, 3, 1], ctx=[300, 700, 500, 900])),
                                        ("shared", dict(n_q=8, n_kv=2, hd=64, page=16, d=[2, 1, 3, 1], ctx=[300, 700, 500, 900])),
                                        ("sparse", dict(n_q=8, n_kv=2, hd=64, page=16, d=[2, 1, 3, 1], ctx=[300, 700, 500, 900]))])
def test_a_run_of_requests(call, shape):
    """The requests from the second on in a call of their own, their rows numbered as in the whole batch (cu starts above
    0): their rows are right, the first request's are neither read nor written."""
    need_gpu()
    b = Batch(seed=47, prefix=[(1, 4, 480)] if call == "shared" else (), **shape)
    b.bounds()
    sel = (30, 1, 1)
    ref = (op.paged_attn_sparse(b.q[: b.M], b.k, b.v, b.kmin, b.kmax, b.table, b.cu, b.ctx, b.page, *sel) if call == "sparse"
           else b.oracle())
    b.dq[: int(b.d[0])] = float("nan")
    b.dcu, b.dctx, b.dtable, b.B = b.dcu[1:], b.dctx[1:], b.dtable[1:], 3
    kw = dict(sel=sel) if call == "sparse" else dict(groups=_groups(b, [(0, 3, 480)])) if call == "shared" else {}
    out, ls = b.run(call, **kw)
    b.check(out, ls, ref, rows=np.arange(int(b.d[0]), b.M), what=call)
    n = int(b.d[0])
    assert (out[:n] == 7.0).all() and (ls[:n] == 7.0).all() and int(b.err.item()) == 0


def test_host_tensors_are_refused():
    """A tensor on the host beside a cache on the GPU: refused by name, nothing is launched."""
    need_gpu()
    b = Batch(seed=48, **ATTN["verify"])
    b.bounds()
    out, ls = b.outputs()
    ws = L.workspace(L.paged_workspace_bytes("attn", b.cfg(), b.B))
    good = dict(q=b.dq, cu=b.dcu, ctx_len=b.dctx, out=out, ws=ws, lse=ls, dev_err=b.err)
    for name in good:
        t = {**good, name: good[name].cpu()}
        with pytest.raises(L.DcutError, match=f"dcut_paged_attn, {name}:"):
            L.paged_attn(b.cfg(), b.pages(), b.B, t["q"], t["cu"], t["ctx_len"], t["out"], t["ws"], lse=t["lse"], dev_err=t["dev_err"])
    with pytest.raises(L.DcutError, match="pages_desc, device"):
        L.pages_desc(b.dk, b.dv, b.dtable.cpu())
    assert (out == 7.0).all() and int(b.err.item()) == 0
