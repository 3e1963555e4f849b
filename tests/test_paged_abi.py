"""The paged cache's entry points without a GPU: refusals before any launch, scratch sizes; its oracle's closed forms."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import paged as op
from paper_2607_14647_amd import lib as L

FAKE = C.c_void_p(0x1000)            # never dereferenced: validation fails first
GOOD = dict(n_q=8, n_kv=2, head_dim=128, page=16, max_ctx=1000, max_block=4, max_rows=16)


def _cfg(**kw):
    return L.PagedCfg(*[{**GOOD, **kw}[n] for n, _ in L.PagedCfg._fields_])


def _pages(**kw):
    d = dict(k=0x1000, v=0x1000, table=0x1000, n_pages=4, table_ld=4, kmin=0x1000, kmax=0x1000)
    d.update(kw)
    return L.Pages(*[d[n] for n, _ in L.Pages._fields_])


def _attn(cfg, pages=None, B=4, q=FAKE, ldq=1024, cu=FAKE, ctx=FAKE, out=FAKE, ws=None, wsb=0):
    pages = _pages() if pages is None else pages
    return L.lib().dcut_paged_attn(C.byref(cfg), C.byref(pages), B, q, ldq, cu, ctx, out, None, None, ws, wsb, None)


def _shared(cfg, n_groups=1, gcu=FAKE, pre=FAKE, ws=None, wsb=0, B=4):
    return L.lib().dcut_paged_attn_shared(C.byref(cfg), C.byref(_pages()), B, FAKE, 1024, FAKE, FAKE, n_groups, gcu, pre,
                                          FAKE, None, None, ws, wsb, None)


def _sparse(cfg, n_sel=8, n_sink=1, n_local=1, pages=None, ws=None, wsb=0):
    pages = _pages() if pages is None else pages
    return L.lib().dcut_paged_attn_sparse(C.byref(cfg), C.byref(pages), 4, FAKE, 1024, FAKE, FAKE, n_sel, n_sink, n_local,
                                          None, FAKE, None, None, ws, wsb, None)


def _append(cfg, pages=None, typ=L.BF16, q=FAKE, ldq=1024, k=FAKE, ldk=256, v=FAKE, ldv=256, theta=1e4, q_out=FAKE, pos=FAKE):
    pages = _pages() if pages is None else pages
    return L.lib().dcut_paged_append(C.byref(cfg), C.byref(pages), 4, FAKE, pos, FAKE, typ, q, ldq, k, ldk, v, ldv, theta,
                                     q_out, None, None)


BAD_CFG = [(dict(n_q=0), L.EINVAL), (dict(n_q=7), L.EINVAL), (dict(n_kv=0), L.EINVAL), (dict(head_dim=0), L.EINVAL),
           (dict(page=0), L.EINVAL), (dict(max_ctx=0), L.EINVAL), (dict(max_block=0), L.EINVAL), (dict(max_rows=0), L.EINVAL),
           (dict(max_block=1001), L.EINVAL), (dict(head_dim=96), L.EUNSUPPORTED), (dict(page=24), L.EUNSUPPORTED),
           (dict(page=8), L.EUNSUPPORTED), (dict(page=512), L.EUNSUPPORTED), (dict(n_q=130, n_kv=2), L.EUNSUPPORTED),
           (dict(max_rows=(1 << 17) + 1), L.EUNSUPPORTED), (dict(max_ctx=(1 << 24) + 1), L.EUNSUPPORTED),
           (dict(n_q=1024, n_kv=16, head_dim=64, max_rows=(1 << 16) + 1), L.EUNSUPPORTED)]


@pytest.mark.parametrize("kw,want", BAD_CFG)
def test_configurations_are_refused(kw, want):
    cfg = _cfg(**kw)
    ld = 1 << 16                       # wide enough for every head count here
    assert _attn(cfg, ldq=ld) == want
    assert L.lib().dcut_paged_attn_shared(C.byref(cfg), C.byref(_pages()), 4, FAKE, ld, FAKE, FAKE, 1, FAKE, FAKE, FAKE, None,
                                          None, None, 0, None) == want
    assert L.lib().dcut_paged_attn_sparse(C.byref(cfg), C.byref(_pages()), 4, FAKE, ld, FAKE, FAKE, 8, 1, 1, None, FAKE, None,
                                          None, None, 0, None) == want
    assert _append(cfg, ldq=ld, ldk=ld, ldv=ld) == want
    with pytest.raises(L.DcutError):
        L.paged_workspace_bytes("attn", cfg, 4)


def test_arguments_are_refused():
    c = _cfg()
    assert _attn(c, B=0) == L.EINVAL and _attn(c, B=4097) == L.EINVAL
    assert _attn(c, q=None) == L.EINVAL and _attn(c, cu=None) == L.EINVAL and _attn(c, ctx=None) == L.EINVAL
    assert _attn(c, out=None) == L.EINVAL
    assert _attn(c, q=C.c_void_p(0x1008)) == L.EINVAL and _attn(c, out=C.c_void_p(0x1008)) == L.EINVAL
    assert _attn(c, ldq=1023) == L.EINVAL and _attn(c, ldq=1028) == L.EINVAL
    for bad in (dict(k=None), dict(v=None), dict(table=None), dict(n_pages=0), dict(table_ld=0), dict(k=0x1008)):
        assert _attn(c, pages=_pages(**bad)) == L.EINVAL
        assert _append(c, pages=_pages(**bad)) == L.EINVAL
        assert _sparse(c, pages=_pages(**bad)) == L.EINVAL
    assert _shared(c, n_groups=0) == L.EINVAL and _shared(c, n_groups=5) == L.EINVAL
    assert _shared(c, gcu=None) == L.EINVAL and _shared(c, pre=None) == L.EINVAL
    assert _sparse(c, n_sel=0) == L.EINVAL and _sparse(c, n_local=0) == L.EINVAL and _sparse(c, n_sink=-1) == L.EINVAL
    assert _sparse(c, n_sel=2, n_sink=1, n_local=2) == L.EINVAL
    assert _sparse(c, n_sel=4097) == L.EUNSUPPORTED
    assert _sparse(c, pages=_pages(kmin=None)) == L.EINVAL and _sparse(c, pages=_pages(kmax=0x1008)) == L.EINVAL
    assert _append(c, typ=2) == L.EINVAL and _append(c, theta=0.0) == L.EINVAL and _append(c, theta=float("inf")) == L.EINVAL
    assert _append(c, q=None) == L.EINVAL and _append(c, q_out=None) == L.EINVAL and _append(c, k=None) == L.EINVAL
    assert _append(c, ldk=255) == L.EINVAL and _append(c, ldv=260) == L.EINVAL and _append(c, ldq=1020) == L.EINVAL
    assert _append(c, pos=None) == L.EINVAL and _append(c, pages=_pages(kmin=None)) == L.EINVAL
    assert _append(c, v=C.c_void_p(0x1002)) == L.EINVAL


def test_workspaces_are_checked():
    c = _cfg()
    for call, which, run in (("attn", 0, _attn), ("shared", 1, _shared), ("sparse", 2, _sparse)):
        n = L.paged_workspace_bytes(call, c, 4, 8)
        assert n > 0 and n % 256 == 0
        assert run(c) == L.EWORKSPACE
        assert run(c, ws=FAKE, wsb=n - 1) == L.EWORKSPACE
        assert run(c, ws=C.c_void_p(0x1010), wsb=n) == L.EWORKSPACE
    assert L.lib().dcut_paged_workspace_bytes(3, C.byref(c), 4, 8) == 2 ** 64 - 1
    assert L.lib().dcut_paged_workspace_bytes(2, C.byref(c), 4, 0) == 2 ** 64 - 1
    # the partial sums do not grow without bound with the context: at most one per 2048 keys
    # once a request has more than its share of pieces
    big = _cfg(max_ctx=1 << 20, max_rows=512, n_q=32, n_kv=8)
    # (132 float32 each), and a work order of one 16-byte entry per request and piece
    assert L.paged_workspace_bytes("attn", big, 512) <= 512 * 32 * 512 * 132 * 4 + 512 * 512 * 16 + 4096


def test_launches_of_too_many_work_items_are_refused():
    ws = C.c_void_p(0x1000)
    many = _cfg(n_q=1024, n_kv=1024, max_ctx=1 << 24, max_rows=4096, max_block=1)
    args = dict(q=FAKE, ldq=1 << 17, ws=ws, wsb=2 ** 63, B=4096)
    assert _attn(many, **args) == L.EUNSUPPORTED
    assert L.lib().dcut_paged_workspace_bytes(0, C.byref(many), 4096, 0) == 2 ** 64 - 1
    assert L.lib().dcut_paged_workspace_bytes(1, C.byref(many), 4096, 0) == 2 ** 64 - 1
    assert L.lib().dcut_paged_attn_shared(C.byref(many), C.byref(_pages()), 4096, FAKE, 1 << 17, FAKE, FAKE, 1, FAKE, FAKE, FAKE,
                                          None, None, ws, 2 ** 63, None) == L.EUNSUPPORTED
    rows = _cfg(n_q=512, n_kv=512, max_rows=1 << 16)
    assert L.lib().dcut_paged_workspace_bytes(2, C.byref(rows), 4, 8) == 2 ** 64 - 1
    assert L.lib().dcut_paged_attn_sparse(C.byref(rows), C.byref(_pages()), 4, FAKE, 1 << 17, FAKE, FAKE, 8, 1, 1, None, FAKE,
                                          None, None, ws, 2 ** 63, None) == L.EUNSUPPORTED
    decode = _cfg(n_q=4, n_kv=1, max_ctx=1 << 22, max_rows=4096, max_block=1)
    assert L.paged_workspace_bytes("attn", decode, 4096) > 0


def test_the_binding_refuses_what_a_pointer_cannot_say():
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    table = torch.zeros(4, 8, dtype=torch.int32)
    L.pages_desc(k, k, table[:, :5])
    for bad in (dict(k=k[:, :1]), dict(v=k[:2]), dict(table=table.t()), dict(kmin=k.transpose(0, 1)[0])):
        with pytest.raises(L.DcutError):
            L.pages_desc(**{**dict(k=k, v=k, table=table), **bad})
    x, c = torch.zeros(4, 128), _cfg(head_dim=64)
    pages = L.pages_desc(k, k, table)
    for q, kk, v in ((None, x, x.bfloat16()), (x.bfloat16(), x, x), (None, x.double(), x.double())):
        with pytest.raises(L.DcutError):
            L.paged_append(c, pages, 4, table, table, table, q, kk, v, q, 1e4)
    with pytest.raises(L.DcutError):
        L.paged_attn_shared(c, pages, 4, x, table, table, x, x, table[0, :3], table[0, :3])


def test_oracle_closed_forms():
    """Equal keys give the mean of the values; a key far above the others gives its value; rotation keeps lengths and
    turns position p by p times position 1's angle."""
    rng = np.random.default_rng(3)
    q, v = rng.standard_normal((4, 64)), rng.standard_normal((2, 7, 64))
    out, lse, _, _ = op.attend(q, np.zeros((2, 7, 64)), v)
    assert np.allclose(out, np.repeat(v.mean(1), 2, 0)) and np.allclose(lse, np.log(7))
    k = np.zeros((2, 7, 64))
    k[:, 3] = 0
    k[0, 3], k[1, 3] = 1e4 * q[:2].sum(0), 1e4 * q[2:].sum(0)
    out, _, _, _ = op.attend(q, k, v)
    for h in range(4):
        if (q[h] * (q[:2] if h < 2 else q[2:]).sum(0)).sum() > 1:
            assert np.allclose(out[h], v[h // 2, 3])
    x = rng.standard_normal((3, 2, 64))
    r1, r5 = op.rotate(x, np.array([1, 1, 1]), 1e4), op.rotate(x, np.array([5, 5, 5]), 1e4)
    assert np.allclose((r1 ** 2).sum(-1), (x ** 2).sum(-1))
    for _ in range(4):
        r1 = op.rotate(r1, np.array([1, 1, 1]), 1e4)
    assert np.allclose(r1, r5)
    # the score bounds the group's summed scores with every key of the page
    kk = rng.standard_normal((5, 16, 64))
    qs = rng.standard_normal((3, 64))
    score = np.maximum(qs, 0).sum(0) @ kk.max(1).T + np.minimum(qs, 0).sum(0) @ kk.min(1).T
    assert ((kk @ qs.sum(0)).max(1) <= score).all()
    assert op.select_pages(qs, kk.min(1), kk.max(1), 3, 1, 1) == sorted({0, 4, 1 + int(np.argmax(score[1:4]))})


# The calls below get as far as the check that is tried, or to a refusal of tensors that are not on a GPU: nothing is launched.

def _tensors(**kw):
    """A cache of 2 kv heads, pages of 16, head_dim 64, and the arguments of a batch of 4 with 6 rows, 4 query heads."""
    t = dict(k=torch.zeros(8, 2, 16, 64, dtype=torch.bfloat16), v=torch.zeros(8, 2, 16, 64, dtype=torch.bfloat16),
             table=torch.zeros(4, 5, dtype=torch.int32), kmin=torch.zeros(8, 2, 64, dtype=torch.bfloat16),
             kmax=torch.zeros(8, 2, 64, dtype=torch.bfloat16), q=torch.zeros(6, 4, 64, dtype=torch.bfloat16),
             cu=torch.zeros(5, dtype=torch.int32), ctx=torch.zeros(4, dtype=torch.int32), pos=torch.zeros(6, dtype=torch.int32),
             req=torch.zeros(6, dtype=torch.int32), nk=torch.zeros(6, 128, dtype=torch.bfloat16),
             nv=torch.zeros(6, 128, dtype=torch.bfloat16), out=torch.zeros(6, 4, 64, dtype=torch.bfloat16), lse=torch.zeros(6, 4),
             err=torch.zeros(1, dtype=torch.int32), ws=torch.zeros(1 << 20, dtype=torch.uint8),
             gcu=torch.zeros(2, dtype=torch.int32), pre=torch.zeros(1, dtype=torch.int32), blocks=torch.zeros(6, 2, 3, dtype=torch.int32))
    t.update(kw)
    return t


CALLS = {
    "append": lambda c, p, t: L.paged_append(c, p, 4, t["cu"], t["pos"], t["req"], t["q"], t["nk"], t["nv"], t["out"], 1e4, dev_err=t["err"]),
    "attn": lambda c, p, t: L.paged_attn(c, p, 4, t["q"], t["cu"], t["ctx"], t["out"], t["ws"], lse=t["lse"], dev_err=t["err"]),
    "attn_shared": lambda c, p, t: L.paged_attn_shared(c, p, 4, t["q"], t["cu"], t["ctx"], t["out"], t["ws"], t["gcu"], t["pre"],
                                                       lse=t["lse"], dev_err=t["err"]),
    "attn_sparse": lambda c, p, t: L.paged_attn_sparse(c, p, 4, t["q"], t["cu"], t["ctx"], t["out"], t["ws"], 3, 1, 1, blocks=t["blocks"],
                                                       lse=t["lse"], dev_err=t["err"]),
}


def _small_cfg(**kw):
    return _cfg(**{**dict(n_q=4, n_kv=2, head_dim=64, page=16, max_ctx=80, max_block=2, max_rows=6), **kw})


def _refused(call, why, cfg=None, **kw):
    t = _tensors(**kw)
    pages = L.pages_desc(t["k"], t["v"], t["table"], t["kmin"], t["kmax"])
    with pytest.raises(L.DcutError, match=f"dcut_paged_{call}, {why}:"):
        CALLS[call](_small_cfg() if cfg is None else cfg, pages, t)


def test_pools_of_other_types_and_shapes_are_refused():
    good = _tensors()
    desc = lambda **kw: L.pages_desc(*[{**good, **kw}[n] for n in ("k", "v", "table", "kmin", "kmax")])
    desc()
    desc(kmin=None, kmax=None)
    desc(**{n: good[n].view(torch.int16) for n in ("k", "v", "kmin", "kmax")})
    for bad in (dict(k=good["k"].half(), v=good["v"].half()), dict(v=good["v"].half()), dict(k=good["k"].float(), v=good["v"].float()),
                dict(k=good["k"][0], v=good["v"][0]), dict(kmin=good["kmin"].float()), dict(kmax=good["kmax"][:7]),
                dict(kmin=good["kmin"].flatten(1)), dict(table=good["table"].long()), dict(table=good["table"][0])):
        with pytest.raises(L.DcutError):
            desc(**bad)


@pytest.mark.parametrize("call", list(CALLS))
def test_pools_that_do_not_match_the_configuration_are_refused(call):
    for kw in (dict(page=32), dict(n_kv=1), dict(n_kv=4), dict(head_dim=128)):
        _refused(call, "pool", cfg=_small_cfg(**kw))


@pytest.mark.parametrize("call", list(CALLS))
def test_tables_that_end_before_the_batch_does_are_refused(call):
    """Fewer rows than requests; a view of fewer columns than its row stride, where max_ctx reaches into the others."""
    wide = torch.zeros(4, 9, dtype=torch.int32)
    _refused(call, "table", table=wide[:3])
    for view in (wide[:, :4], wide[:, 5:]):
        _refused(call, "table", table=view)                             # max_ctx 80: five columns
        assert L.pages_desc(_tensors()["k"], _tensors()["v"], view).max_ctx == 64
    # a row of its own has no stride to go by
    one = L.pages_desc(_tensors()["k"], _tensors()["v"], wide[1:2, 2:6])
    assert (one.table_ld, one.max_ctx) == (4, None)
    # nor has a single column: one page a request
    assert L.pages_desc(_tensors()["k"], _tensors()["v"], torch.zeros(1, 4, dtype=torch.int32).t()).table_ld == 1


WRONG = dict(cu=[lambda x: x.long(), lambda x: x[:4], lambda x: x.repeat(2)[::2]], ctx=[lambda x: x.long(), lambda x: x[:3]],
             pos=[lambda x: x.long(), lambda x: x.repeat(2)[::2]], req=[lambda x: x.long()],
             q=[lambda x: x.float(), lambda x: x.half(), lambda x: x[..., :32], lambda x: x[:, :3], lambda x: x.transpose(1, 2),
                lambda x: x.transpose(1, 2).contiguous().transpose(1, 2), lambda x: torch.cat([x, x], 2)[..., ::2], lambda x: x.flatten()],
             nk=[lambda x: x[:, :64], lambda x: torch.cat([x, x], 1)[:, ::2]], nv=[lambda x: x[:, :64], lambda x: x.t().contiguous().t()],
             out=[lambda x: x.float(), lambda x: x.repeat(1, 2, 1)[:, :4]], lse=[lambda x: x.bfloat16(), lambda x: x.repeat(1, 2)[:, :4]],
             err=[lambda x: x.long()], ws=[lambda x: x[::2]], gcu=[lambda x: x.long()], pre=[lambda x: x.long()],
             blocks=[lambda x: x.long(), lambda x: x.transpose(1, 2)])
NAMES = dict(cu="cu", ctx="ctx_len", pos="packed_pos", req="packed_req", nk="k", nv="v", out="out", err="dev_err", gcu="group_cu",
             pre="prefix_len")
USED = dict(append=("cu", "pos", "req", "q", "nk", "nv", "out", "err"), attn=("q", "cu", "ctx", "out", "lse", "err", "ws"))
USED["attn_shared"], USED["attn_sparse"] = USED["attn"] + ("gcu", "pre"), USED["attn"] + ("blocks",)


@pytest.mark.parametrize("call", list(CALLS))
def test_tensors_of_other_types_and_strides_are_refused(call):
    """A wrong element type, elements that do not follow each other, too few of them: refused by name."""
    good = _tensors()
    for name in USED[call]:
        why = "q_out" if (call, name) == ("append", "out") else NAMES.get(name, name)
        for wrong in WRONG[name]:
            bad = wrong(good[name])
            if call == "append" and name == "q" and bad.dtype is not torch.bfloat16:
                continue                   # of another type than k and v, refused as before
            _refused(call, why, **{name: bad})


@pytest.mark.parametrize("call", list(CALLS))
def test_rows_may_lie_apart(call):
    """Views of a fused projection, further dimensions, a single row of any stride: nothing is left to refuse but the
    device, on which the cache has to be."""
    x = torch.zeros(6, 512 + 8, dtype=torch.bfloat16)
    raw = lambda t: t.view(torch.int16)
    for kw in ({}, dict(q=x[:, :256], nk=x[:, 256:384], nv=x[:, 384:512]), dict(q=x[:, :256].view(6, 2, 2, 64)),
               dict(q=torch.zeros(4, 1, 64, dtype=torch.bfloat16).transpose(0, 1)),
               dict(q=raw(x)[:, :256], nk=raw(x)[:, 256:384], nv=raw(x)[:, 384:512], out=raw(_tensors()["out"]))):
        _refused(call, "device", **kw)
    wide = torch.zeros(4, 9, dtype=torch.int32)
    _refused(call, "device", cfg=_small_cfg(max_ctx=64), table=wide[:, :4])


@pytest.mark.parametrize("theta", [-1, -1.0, np.float32(-1), np.float64(-1), torch.tensor(-1.0)])
def test_rotation_bases_of_any_number_type(theta, monkeypatch):
    """They reach the library, which refuses this one by its value."""
    monkeypatch.setattr(L, "_stream_on", lambda *a: None)
    t = _tensors()
    pages = L.pages_desc(t["k"], t["v"], t["table"], t["kmin"], t["kmax"])
    with pytest.raises(L.DcutError, match="dcut_paged_append:"):
        L.paged_append(_small_cfg(), pages, 4, t["cu"], t["pos"], t["req"], t["q"], t["nk"], t["nv"], t["out"], theta)


@pytest.mark.parametrize("call", list(CALLS))
def test_a_table_without_columns_is_refused(call):
    _refused(call, "table", table=torch.zeros(4, 9, dtype=torch.int32)[:, :0])
