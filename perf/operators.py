"""Measured cases of the paged key/value cache: appending with rotation, and the attention that reads it.

Four operators over one cache of pages, each in its plain form (elementary torch operations in 32 bits)
and through the library's calls:

  append   rotate the new queries and keys by position, write keys and values into the pages of their
           requests, and the channel bounds of every page that gets full
  attn     causal grouped-query attention of each request's new rows over its pages: one row a request
           (decoding), a kept block of drafts (verification), a prompt
  shared   the same for requests that start with the same pages, which are read once for all of them
  sparse   the same over n_sel pages a query, chosen by an upper bound of its scores in each page

The cache is [n_pages][n_kv][page][head_dim]; request i's key j lies in page table[i][j // page], slot
j % page.  Pages are handed out in random order, as after some time of serving; table entries that no
request uses hold -1, free pages and the tails of last pages hold stale values.
"""
import math

import numpy as np
import torch

own = False

THETA = 500000.0
Q_STD = 1.5           # scores of a few units, so that a softmax has both heavy and light keys

# the heads of the repository's layers: its dense and its MoE configuration, and the tiny one
DENSE = dict(n_q=32, n_kv=8, head_dim=128)
MOE = dict(n_q=32, n_kv=4, head_dim=128)
TINY = dict(n_q=4, n_kv=2, head_dim=64)
# generic ones for drawn cases: no sharing, one key head for all, groups of 3, 5 and 7
HEADS = [DENSE, DENSE, MOE, TINY, dict(n_q=32, n_kv=8, head_dim=64), dict(n_q=16, n_kv=2, head_dim=128),
         dict(n_q=8, n_kv=8, head_dim=64), dict(n_q=8, n_kv=1, head_dim=128), dict(n_q=9, n_kv=3, head_dim=64),
         dict(n_q=40, n_kv=8, head_dim=128), dict(n_q=14, n_kv=2, head_dim=64)]


def _case(name, op, heads, B, page, rows, ctx, log=False, **more):
    """rows: (least, most) new rows of a request; ctx: (least, most) keys it has before them, of its own."""
    c = dict(op=op, B=B, page=page, d_lo=rows[0], d_hi=rows[1], ctx_lo=ctx[0], ctx_hi=ctx[1], ctx_log=log)
    c.update(heads)
    c.update(more)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # one decoding step of a batch of 64: 64 new rows, nothing but latency
        _case("append_decode_b64", "append", DENSE, 64, 16, (1, 1), (256, 1024), bounds=False, dtype="bf16"),
        # a batch of prompt pieces of odd lengths: 7 thousand rows, page bounds kept for the sparse reader
        _case("append_prompt_b8", "append", DENSE, 8, 64, (700, 1100), (0, 2000), bounds=True, dtype="bf16"),
        # one request served alone
        _case("attn_decode_b1", "attn", DENSE, 1, 16, (1, 1), (1900, 2100)),
        # decoding of a ragged batch of 128, contexts 512 to 8192
        _case("attn_decode_b128", "attn", DENSE, 128, 16, (1, 1), (512, 8191), log=True),
        # verification of blocks of which 1 to 8 rows were kept, the batch-64 contexts of the benchmark; as in
        # every case, the calls are bounded by the longest block of each request
        _case("attn_verify_b64", "attn", DENSE, 64, 32, (1, 8), (2048, 4096)),
        # groups of 7 query heads, 64 wide, short ragged contexts down to none
        _case("attn_verify_odd", "attn", dict(n_q=14, n_kv=2, head_dim=64), 33, 16, (0, 5), (0, 700)),
        # prompts in pieces of about 2000 rows on contexts of up to 2000: matrix products bound
        _case("attn_prompt_b4", "attn", DENSE, 4, 64, (1900, 2100), (0, 2000)),
        # 32 answers to one prompt of 8000 tokens
        _case("shared_decode_b32", "shared", DENSE, 32, 16, (1, 1), (16, 400), groups=1, pre_lo=8000, pre_hi=8000),
        # verification under three prompts of different lengths
        _case("shared_verify_b96", "shared", MOE, 96, 64, (1, 8), (100, 900), groups=3, pre_lo=2000, pre_hi=6000),
        # one request with a long context: 32 of some 500 pages a query
        _case("sparse_decode_b1", "sparse", DENSE, 1, 64, (1, 1), (30000, 33000), n_sel=32, n_sink=1, n_local=2),
        # decoding of a batch with contexts of 16 to 64 thousand
        _case("sparse_decode_b16", "sparse", DENSE, 16, 64, (1, 1), (16384, 65536), n_sel=32, n_sink=1, n_local=2),
        # verification, small pages
        _case("sparse_verify_b24", "sparse", MOE, 24, 32, (1, 6), (4000, 20000), n_sel=48, n_sink=1, n_local=3),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "attn", "attn", "attn", "shared", "sparse"])
    h = rng.choice(HEADS)
    page = rng.choice([16, 16, 32, 64, 128])
    key = h["n_kv"] * h["head_dim"] * 4                      # bytes of a key and its value
    if op == "append":
        B = _log_int(rng, 1, 256)
        hi = _log_int(rng, 1, min(1100, 6000 // B)) if rng.random() < 0.6 else 1
        return _case("", op, h, B, page, (rng.randint(0, 1) if hi > 1 else 1, hi), (0, _log_int(rng, 1, min(4000, 100000 // B))),
                     bounds=rng.random() < 0.5, dtype=rng.choice(["bf16", "bf16", "f32"]))
    if op == "attn" and rng.random() < 0.3:                  # prompts
        hi = _log_int(rng, 65, 2100)
        B = _log_int(rng, 1, max(1, 8000 // hi))
        return _case("", op, h, B, page, (_log_int(rng, 1, hi), hi), (0, _log_int(rng, 1, 2000)))
    d = rng.choice([1, 1, 1, rng.randint(2, 8), rng.randint(2, 16), rng.randint(2, 33)])
    if op == "sparse":
        B = _log_int(rng, 1, 48)
        page = rng.choice([16, 32, 64, 64])
        d = min(d, 16)
        hi = _log_int(rng, 100, max(200, min(65536, int(1.2e9 / key / B))))
        return _case("", op, h, B, page, (1, d), (_log_int(rng, 1, hi), hi), n_sel=_log_int(rng, 4, max(5, min(64, int(2.5e9 / (B * d * page * key))))),
                     n_sink=rng.randint(0, 2), n_local=rng.randint(1, 2))
    B = _log_int(rng, 1, 128)
    if op == "shared":
        pre = _log_int(rng, 16, 12000)
        return _case("", op, h, B, page, (1, d), (0, _log_int(rng, 1, 1000)), groups=rng.randint(1, min(4, B)),
                     pre_lo=_log_int(rng, 1, pre), pre_hi=pre)
    hi = _log_int(rng, 16, max(64, min(16000, int(1.2e9 / key / B))))
    return _case("", op, h, B, page, (rng.randint(0, 1) if d > 1 else 1, d), (_log_int(rng, 1, hi), hi), log=rng.random() < 0.5)


# ------------------------------------------------------------------ inputs

def _layout(case, seed):
    """Host arrays: new rows and context of each request, prefix and range of each group, page tables."""
    rng = np.random.default_rng([int(seed), 29])
    B, page = case["B"], case["page"]
    d = rng.integers(case["d_lo"], case["d_hi"] + 1, size=B)
    d[rng.integers(B)] = case["d_hi"]                        # the launch bound is met
    lo, hi = case["ctx_lo"], case["ctx_hi"]
    if case["ctx_log"]:
        ctx = np.rint(np.exp(rng.uniform(math.log(max(lo, 1)), math.log(max(hi, 1)), size=B))).astype(np.int64)
    else:
        ctx = rng.integers(lo, hi + 1, size=B)
    NG = case.get("groups", 0)
    gcu = np.concatenate([[0], np.sort(rng.choice(np.arange(1, B), NG - 1, replace=False)), [B]]) if NG else np.array([0, B])
    pre = rng.integers(case["pre_lo"], case["pre_hi"] + 1, size=NG) if NG else np.zeros(1, dtype=np.int64)
    group = np.repeat(np.arange(len(pre)), np.diff(gcu))
    ctx = ctx + pre[group]
    need = -(-(ctx + d) // page)                             # pages a request's table lists
    full = pre // page                                       # pages wholly of the prefix are shared, a last one copied
    total = int(full.sum() + (need - full[group]).sum())
    if case["op"] == "append":                               # whose pool is an output: of one size for all seeds
        total = B * -(-(hi + case["d_hi"]) // page)
    ids = rng.permutation(total + 3)                         # a few free pages
    ld = int(max(1, -(-(int((ctx + d).max())) // page)))
    table = np.full((B, ld), -1, dtype=np.int32)
    at = int(full.sum())
    starts = np.concatenate([[0], np.cumsum(full)])
    for i in range(B):
        g = group[i]
        own_pages = int(need[i] - full[g])
        table[i, : full[g]] = ids[starts[g]: starts[g] + full[g]]
        table[i, full[g]: need[i]] = ids[at: at + own_pages]
        at += own_pages
    return dict(d=d.astype(np.int64), ctx=ctx.astype(np.int64), table=table, n_pages=total + 3, gcu=gcu, pre=pre, group=group, full=full)


def _gen(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 64 + tag)
    return g


def _normal(seed, tag, shape, std, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=_gen(seed, tag))


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def prepare(case, seed):
    lay = _layout(case, seed)
    B, page, n_q, n_kv, hd, op = case["B"], case["page"], case["n_q"], case["n_kv"], case["head_dim"], case["op"]
    d, ctx, table = lay["d"], lay["ctx"], lay["table"]
    K = int(d.sum())
    rows = B * case["d_hi"]
    cu = np.concatenate([[0], np.cumsum(d)])
    req = np.repeat(np.arange(B), d)
    pos = ctx[req] + np.arange(K) - cu[req]
    st = dict(case=case, B=B, rows=rows, d_max=int(d.max()), L_max=int((ctx + d).max()), cu=_i32(cu), ctx=_i32(ctx),
              table=_i32(table), req=_i32(np.pad(req, (0, rows - K))), pos=_i32(np.pad(pos, (0, rows - K))),
              err=torch.zeros(1, dtype=torch.int32, device="cuda"))
    pool = (lay["n_pages"], n_kv, page, hd)
    st["k"], st["v"] = _normal(seed, 1, pool, 1.0), _normal(seed, 2, pool, 1.0)
    if op == "sparse":                                       # keys that stay near each other within a page
        st["k"].mul_(0.7).add_(_normal(seed, 3, (lay["n_pages"], n_kv, 1, hd), 0.7))
    if op == "shared":                                       # where a page is partly shared, each request has its copy
        first = _i32(lay["gcu"][:-1])[_i32(lay["group"]).long()].long()
        n = _i32(lay["pre"])[_i32(lay["group"]).long()].long()
        last = torch.minimum(n // page, torch.full_like(n, table.shape[1] - 1))[:, None]
        src, dst = st["table"][first].gather(1, last)[:, 0].long(), st["table"].gather(1, last)[:, 0].long()
        part = (torch.arange(page, device="cuda")[None] < (n % page)[:, None])[:, None, :, None] & (src != dst)[:, None, None, None]
        ok = (n % page > 0) & (src >= 0) & (dst >= 0)
        src, dst, part = src[ok], dst[ok], part[ok]
        for x in (st["k"], st["v"]):
            x[dst] = torch.where(part, x[src], x[dst])
        st["gcu"], st["pre"] = _i32(lay["gcu"]), _i32(lay["pre"])
    if op == "sparse" or case.get("bounds"):
        st["kmin"], st["kmax"] = st["k"].amin(2), st["k"].amax(2)
    dt = torch.float32 if case.get("dtype") == "f32" else torch.bfloat16
    if op == "append":                                       # one fused projection's rows: q, k and v are views of it
        st["qkv"] = _normal(seed, 4, (rows, (n_q + 2 * n_kv) * hd), Q_STD, dt)
        st["out"] = torch.zeros(rows, n_q, hd, dtype=torch.bfloat16, device="cuda")
    else:
        st["q"] = _normal(seed, 4, (rows, n_q, hd), Q_STD)
        st["out"] = torch.zeros(rows, n_q, hd, dtype=torch.bfloat16, device="cuda")
        st["lse"] = torch.zeros(rows, n_q, dtype=torch.float32, device="cuda")
        if op == "sparse":
            st["blocks"] = torch.zeros(rows, n_kv, case["n_sel"], dtype=torch.int32, device="cuda")
    return st


# ------------------------------------------------------------------ the library's calls

def _handles(st):
    """What a program that serves with the library keeps from step to step: descriptors and the workspace."""
    from paper_2607_14647_amd import lib as L
    c = st["case"]
    st["L"] = L
    st["cfg"] = L.paged_cfg(c["n_q"], c["n_kv"], c["head_dim"], c["page"], max_ctx=max(1, st["L_max"]), max_block=st["d_max"],
                            max_rows=st["rows"])
    st["pages"] = L.pages_desc(st["k"], st["v"], st["table"], st.get("kmin"), st.get("kmax"))
    if c["op"] != "append":
        st["ws"] = L.workspace(L.paged_workspace_bytes(c["op"], st["cfg"], st["B"], c.get("n_sel", 0)))


def _run_own(st):
    if "L" not in st:
        _handles(st)
    L, c, B = st["L"], st["case"], st["B"]
    if c["op"] == "append":
        nq, nkv = c["n_q"] * c["head_dim"], c["n_kv"] * c["head_dim"]
        q, k, v = st["qkv"].split([nq, nkv, nkv], dim=1)
        L.paged_append(st["cfg"], st["pages"], B, st["cu"], st["pos"], st["req"], q, k, v, st["out"], THETA, dev_err=st["err"])
        return
    args = (st["cfg"], st["pages"], B, st["q"], st["cu"], st["ctx"], st["out"], st["ws"])
    if c["op"] == "attn":
        L.paged_attn(*args, lse=st["lse"], dev_err=st["err"])
    elif c["op"] == "shared":
        L.paged_attn_shared(*args, st["gcu"], st["pre"], lse=st["lse"], dev_err=st["err"])
    else:
        L.paged_attn_sparse(*args, c["n_sel"], c["n_sink"], c["n_local"], blocks=st["blocks"], lse=st["lse"], dev_err=st["err"])


# ------------------------------------------------------------------ plain forms

def _padded(st):
    """[B][d_max] row numbers (rows past a request's own: the extra row `rows`), whether each is one, its position."""
    cu, d_max = st["cu"].long(), st["d_max"]
    k = torch.arange(d_max, device="cuda")
    ok = k < (cu[1:] - cu[:-1])[:, None]
    return torch.where(ok, cu[:-1, None] + k, st["rows"]), ok, st["ctx"].long()[:, None] + k


def _queries(st, idx):
    """Queries as [B][n_kv][d_max][group][head_dim] float32, zero where there is no row."""
    c = st["case"]
    q = torch.cat([st["q"].float(), torch.zeros(1, c["n_q"], c["head_dim"], device="cuda")])[idx]
    return q.view(c["B"], -1, c["n_kv"], c["n_q"] // c["n_kv"], c["head_dim"]).permute(0, 2, 1, 3, 4)


def _back(st, idx, x, like):
    """[B][n_kv][d_max][group][...] to the packed rows; rows of no request stay as they are in `like` (zero)."""
    x = x.permute(0, 2, 1, 3, *range(4, x.dim())).flatten(2, 3)
    out = torch.zeros(st["rows"] + 1, *like.shape[1:], dtype=like.dtype, device="cuda")
    out[idx.reshape(-1)] = x.flatten(0, 1).to(like.dtype)
    return out[: st["rows"]]


def _softmax_rows(s, v):
    """Softmax of scores s [..][R][N] (minus infinity where masked; rows may be empty) times v [..][N][hd], and the rows' log sums."""
    m = s.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    p = torch.exp(s - m)
    l = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(l > 0, l, torch.ones_like(l)), (m + torch.log(l)).squeeze(-1)


def _plain_attn(st):
    c = st["case"]
    idx, ok, pos = _padded(st)
    G, hd, n_kv = c["n_q"] // c["n_kv"], c["head_dim"], c["n_kv"]
    table = st["table"].long().clamp(min=0)
    gather = lambda x: x[table].permute(0, 2, 1, 3, 4).flatten(2, 3).float()          # [B][n_kv][keys][hd]
    q = _queries(st, idx)
    k = gather(st["k"])
    s = torch.matmul(q.flatten(2, 3), k.transpose(2, 3)) * (1.0 / math.sqrt(hd))
    del k
    seen = torch.arange(s.shape[-1], device="cuda") <= pos[:, :, None]                # [B][d_max][keys]
    s = s.view(*q.shape[:4], -1).masked_fill(~seen[:, None, :, None], -math.inf).flatten(2, 3)
    v = gather(st["v"])                                                               # stale slots are finite
    o, lse = _softmax_rows(s, v)
    shape = q.shape[:4]
    return dict(out=_back(st, idx, o.view(*shape, hd), st["out"]), lse=_back(st, idx, lse.view(shape), st["lse"]))


def _plain_sparse(st):
    c = st["case"]
    idx, ok, pos = _padded(st)
    B, page, n_kv, hd, n_sel = c["B"], c["page"], c["n_kv"], c["head_dim"], c["n_sel"]
    table = st["table"].long().clamp(min=0)
    q = _queries(st, idx)
    # upper bounds of the group's summed scores, in 64 bits: they decide which pages are read
    a, b = q.double().clamp(min=0).sum(3), q.double().clamp(max=0).sum(3)             # [B][n_kv][d_max][hd]
    bound = lambda x: x[table].permute(0, 2, 3, 1).double()                           # [B][n_kv][hd][pages]
    s = torch.matmul(a, bound(st["kmax"])) + torch.matmul(b, bound(st["kmin"]))       # [B][n_kv][d_max][pages]
    j = torch.arange(s.shape[-1], device="cuda")
    last = (pos // page)[:, None, :, None]
    s = torch.where(torch.isnan(s), -1.7e308, s).clamp(min=-1.7e308)
    s = s.masked_fill((j < c["n_sink"]) | (j > last - c["n_local"]), math.inf).masked_fill(j > last, -math.inf)
    top = torch.sort(s, dim=-1, descending=True, stable=True)[1][..., :n_sel]
    if top.shape[-1] < n_sel:
        top = torch.cat([top, torch.full((*top.shape[:-1], n_sel - top.shape[-1]), s.shape[-1], device="cuda")], -1)
    top = torch.sort(torch.where(top <= last, top, s.shape[-1]), dim=-1)[0]           # ascending, unused ones at the end
    used = top < s.shape[-1]
    phys = torch.gather(table[:, None, None].expand(-1, n_kv, q.shape[2], -1), -1, top.clamp(max=s.shape[-1] - 1))
    head = torch.arange(n_kv, device="cuda")[None, :, None, None]
    k = st["k"][phys, head].flatten(3, 4).float()                                     # [B][n_kv][d_max][n_sel page][hd]
    sc = torch.matmul(q, k.transpose(3, 4)) * (1.0 / math.sqrt(hd))
    del k
    at = top[..., None] * page + torch.arange(page, device="cuda")
    seen = (used[..., None] & (at <= pos[:, None, :, None, None])).flatten(3)
    o, lse = _softmax_rows(sc.masked_fill(~seen[:, :, :, None], -math.inf), st["v"][phys, head].flatten(3, 4).float())
    blocks = torch.zeros(st["rows"] + 1, n_kv, n_sel, dtype=torch.int32, device="cuda")
    blocks[idx.reshape(-1)] = torch.where(used, top, -1).to(torch.int32).permute(0, 2, 1, 3).flatten(0, 1)
    return dict(out=_back(st, idx, o, st["out"]), lse=_back(st, idx, lse, st["lse"]), blocks=blocks[: st["rows"]])


def _plain_append(st):
    c = st["case"]
    n_q, n_kv, hd, page = c["n_q"], c["n_kv"], c["head_dim"], c["page"]
    half = hd // 2
    live = torch.arange(st["rows"], device="cuda") < st["cu"][-1]
    pos, req = st["pos"][live].long(), st["req"][live].long()
    freq = THETA ** (-2.0 * torch.arange(half, dtype=torch.float64, device="cuda") / hd)
    ang = pos.double()[:, None] * freq                       # 64 bits: far positions turn many times
    cos, sin = ang.cos().float()[:, None], ang.sin().float()[:, None]
    x = st["qkv"][live].float().view(-1, n_q + 2 * n_kv, hd)
    x1, x2 = x[:, : n_q + n_kv, :half], x[:, : n_q + n_kv, half:]
    r = torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin], -1).bfloat16()
    pg = st["table"].long()[req, pos // page]
    st["out"][live] = r[:, :n_q]
    st["k"][pg, :, pos % page] = r[:, n_q:]
    st["v"][pg, :, pos % page] = x[:, n_q + n_kv:].bfloat16()
    if c["bounds"]:
        full = pg[pos % page == page - 1]
        st["kmin"][full], st["kmax"][full] = st["k"][full].amin(2), st["k"][full].amax(2)


def run(st):
    """One pass.  Rows past the last request's are never written and stay zero."""
    op = st["case"]["op"]
    if own:
        _run_own(st)
    elif op == "append":
        _plain_append(st)
    else:
        return _plain_sparse(st) if op == "sparse" else _plain_attn(st)
    return {n: st[n] for n in (("out", "k", "v", "kmin", "kmax") if op == "append" else ("out", "lse", "blocks")) if n in st}


# ------------------------------------------------------------------ definition in 64 bits

def _exact_rows(q, k, v, n):
    """q [n_q][hd] of one row over its first n keys k, v [n_kv][n][hd]: outputs [n_q][hd] and log sums [n_q]."""
    n_q, hd = q.shape
    G = n_q // k.shape[0]
    s = (k.repeat_interleave(G, 0)[:, :n] * q[:, None]).sum(2) / math.sqrt(hd)
    lse = torch.logsumexp(s, 1)
    return (torch.exp(s - lse[:, None])[:, :, None] * v.repeat_interleave(G, 0)[:, :n]).sum(1), lse


def _exact_prompt(q, k, v, L):
    """The rows of one prompt at once, a head at a time: row r sees keys 0 .. L + r."""
    d, n_q, hd = q.shape
    G = n_q // k.shape[0]
    hidden = torch.arange(L + d, device="cuda")[None] > L + torch.arange(d, device="cuda")[:, None]
    out, lse = torch.empty(d, n_q, hd, dtype=torch.float64, device="cuda"), torch.empty(d, n_q, dtype=torch.float64, device="cuda")
    for h in range(n_q):
        s = (q[:, h] @ k[h // G].T / math.sqrt(hd)).masked_fill(hidden, -math.inf)
        lse[:, h] = torch.logsumexp(s, 1)
        out[:, h] = torch.exp(s - lse[:, h, None]) @ v[h // G]
    return out, lse


def exact(case, seed):
    st = prepare(case, seed)
    lay = _layout(case, seed)
    n_q, n_kv, hd, page, op = case["n_q"], case["n_kv"], case["head_dim"], case["page"], case["op"]
    d, ctx, table = lay["d"].tolist(), lay["ctx"].tolist(), st["table"].long()
    f64 = dict(dtype=torch.float64, device="cuda")
    if op == "append":
        K, V = st["k"].double(), st["v"].double()
        x = st["qkv"].double().view(-1, n_q + 2 * n_kv, hd)
        z = torch.complex(x[..., : hd // 2], x[..., hd // 2:])
        turn = torch.exp(-math.log(THETA) * torch.arange(hd // 2, **f64) * 2.0 / hd)
        z = z * torch.polar(torch.ones(1, **f64), st["pos"].double()[:, None] * turn)[:, None]
        r = torch.cat([z.real, z.imag], -1)
        r[sum(d):] = 0
        out = dict(out=r[:, :n_q].contiguous(), k=K, v=V)
        if case["bounds"]:
            out["kmin"], out["kmax"] = st["kmin"].double(), st["kmax"].double()
        t = 0
        for i in range(case["B"]):
            p = torch.arange(ctx[i], ctx[i] + d[i], device="cuda")
            pg = table[i][p // page]
            K[pg, :, p % page], V[pg, :, p % page] = r[t: t + d[i], n_q: n_q + n_kv], x[t: t + d[i], n_q + n_kv:]
            t += d[i]
            if case["bounds"]:
                for j in range(ctx[i] // page, (ctx[i] + d[i]) // page):
                    out["kmin"][table[i, j]], out["kmax"][table[i, j]] = K[table[i, j]].min(1)[0], K[table[i, j]].max(1)[0]
        return out
    out = torch.zeros(st["rows"], n_q, hd, **f64)
    lse = torch.zeros(st["rows"], n_q, **f64)
    if op == "sparse":                                       # row by row from the list that the definition gives
        blocks = torch.zeros(st["rows"], n_kv, case["n_sel"], dtype=torch.int32, device="cuda")
        if sum(d) * n_kv > 2000:
            return None
        G, t = n_q // n_kv, 0
        for i in range(case["B"]):
            lo, hi = st["kmin"][table[i]].double(), st["kmax"][table[i]].double()     # [pages][n_kv][hd]
            for r in range(d[i]):
                p = ctx[i] + r
                n = p // page + 1
                q = st["q"][t].double().view(n_kv, G, hd)
                best = torch.maximum(q[None] * lo[:n, :, None], q[None] * hi[:n, :, None]).sum((2, 3)).cpu().numpy()
                for g in range(n_kv):
                    must = [j for j in range(n) if j < case["n_sink"] or j >= n - case["n_local"]]
                    rest = [j for j in sorted(range(n), key=lambda j: (-best[j, g], j)) if j not in set(must)]
                    pick = sorted((must + rest)[: case["n_sel"]])
                    blocks[t, g] = torch.tensor(pick + [-1] * (case["n_sel"] - len(pick)), dtype=torch.int32)
                    pg = table[i][torch.tensor(pick, device="cuda")]
                    m = (len(pick) - 1) * page + p % page + 1
                    o, l = _exact_rows(q[g], st["k"][pg, g].reshape(1, -1, hd).double(), st["v"][pg, g].reshape(1, -1, hd).double(), m)
                    out[t, g * G: g * G + G], lse[t, g * G: g * G + G] = o, l
                t += 1
        return dict(out=out, lse=lse, blocks=blocks)
    t = 0
    for i in range(case["B"]):
        n = ctx[i] + d[i]
        if d[i]:
            pg = table[i][: -(-n // page)]
            k, v = (x[pg].transpose(0, 1).reshape(n_kv, -1, hd)[:, :n].double() for x in (st["k"], st["v"]))
            out[t: t + d[i]], lse[t: t + d[i]] = _exact_prompt(st["q"][t: t + d[i]].double(), k, v, ctx[i])
        t += d[i]
    return dict(out=out, lse=lse)


# ------------------------------------------------------------------ work

def work(case):
    """Bytes and operations a pass cannot do without, at the mean of the case's ranges: each key and value that a
    request (or, shared, a group) sees once, queries in and outputs out, the products of the seen pairs."""
    B, n_q, n_kv, hd, page = case["B"], case["n_q"], case["n_kv"], case["head_dim"], case["page"]
    d = (case["d_lo"] + case["d_hi"]) / 2
    lo, hi = max(case["ctx_lo"], 1), max(case["ctx_hi"], 1)
    ctx = (hi - lo) / math.log(hi / lo) if case["ctx_log"] and hi > lo else (case["ctx_lo"] + case["ctx_hi"]) / 2
    rows = B * d
    key = 4 * n_kv * hd
    if case["op"] == "append":
        size = 4 if case["dtype"] == "f32" else 2
        full = rows / page if case["bounds"] else 0.0
        old = min(B * min(ctx, page / 2), full * page) if case["bounds"] else 0.0      # earlier keys of pages that get full
        return dict(bytes=rows * (n_q + 2 * n_kv) * hd * (size + 2) + (old * 2 + full * 4) * n_kv * hd, flops=rows * (n_q + n_kv) * hd * 3.0)
    io = rows * n_q * (4 * hd + 4)
    if case["op"] == "sparse":
        pages = (ctx + d) / page + 1
        n = min(case["n_sel"], pages) * page
        return dict(bytes=B * pages * key + rows * n * key + io + rows * n_kv * case["n_sel"] * 4,
                    flops=rows * (4.0 * n_q * hd * n + 4.0 * n_kv * hd * pages))
    pre = (case["pre_lo"] + case["pre_hi"]) / 2 if case["op"] == "shared" else 0.0
    keys = B * (ctx + d) + case.get("groups", 0) * pre
    return dict(bytes=keys * key + io, flops=4.0 * n_q * hd * rows * (pre + ctx + (d + 1) / 2))
