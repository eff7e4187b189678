"""Operators of a decode step over a cache of pages, through the framework's
kernel-level entry points (paper_2503_17707_amd.binding) and in plain form:

  append     new rows of keys and values into the pages of their sequences
  attention  one new token per sequence over its pages
  select     the best continuations over beams and vocabulary
  fork       pages of reordered beams: shared, copied on write, grown, freed

A pool holds pages [n_pages, 2 (k, v), kv heads, page_size, head_dim]; it is laid
out head by head ("heads": a page holds each head's tokens in a row) or as the
framework's own cache rows ("rows": a page holds tokens, each [k | v] of all heads).

Widths are those of the shapes this repository serves (32 heads of 64, 32 and 40
of 128, vocabulary 50272, prompts up to 2048) and, for grouped heads and long
caches, generic ones.  Inputs are drawn from the seed alone.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DT = {"bf16": (torch.bfloat16, 0), "f16": (torch.float16, 1)}
EOS, PAD = 2, 1


def listed():
    return [
        # one decode token of one sequence into the cache: the smallest call
        dict(name="append_token", op="append", dtype="f16", S=1, T=1, ragged=False, Hkv=32, hd=64, ps=16,
             layout="rows"),
        # one decode step of a full server batch, some sequences finished
        dict(name="append_step", op="append", dtype="bf16", S=256, T=1, ragged=True, Hkv=8, hd=128, ps=16,
             layout="heads"),
        # prompts of many lengths admitted together, their keys and values kept
        dict(name="append_prompts", op="append", dtype="f16", S=16, T=2048, ragged=True, Hkv=40, hd=128, ps=16,
             layout="rows"),
        # the first tokens after a short prompt: latency counts
        dict(name="attn_short", op="attention", dtype="f16", S=1, H=32, Hkv=32, hd=64, n=513, ragged=False, window=0,
             ps=16, layout="rows"),
        # a server's decode step of one layer, sequences of all lengths
        dict(name="attn_batch", op="attention", dtype="f16", S=32, H=40, Hkv=40, hd=128, n=2048, ragged=True, window=0,
             ps=16, layout="rows"),
        # grouped heads over longer contexts, each sequence at its own length
        dict(name="attn_grouped", op="attention", dtype="bf16", S=48, H=64, Hkv=8, hd=128, n=16384, ragged=True,
             window=0, ps=64, layout="heads"),
        # one very long context: few rows, the length is what can be shared out
        dict(name="attn_long", op="attention", dtype="bf16", S=1, H=32, Hkv=8, hd=128, n=131071, ragged=False, window=0,
             ps=16, layout="heads"),
        # beam search of one prompt, as it is read while it is written
        dict(name="select_one", op="select", B=1, W=4, V=50272),
        # beam search of a batch
        dict(name="select_batch", op="select", B=32, W=8, V=50272),
        # wide beams over a large vocabulary
        dict(name="select_wide", op="select", B=4, W=32, V=128256),
        # reordering after one step of four beams
        dict(name="fork_step", op="fork", dtype="f16", B=1, W=4, L=24, Hkv=32, hd=64, ps=16, n=512, layout="rows"),
        # reordering of a batch of beams, half a page copied for most of them
        dict(name="fork_batch", op="fork", dtype="f16", B=32, W=8, L=24, Hkv=32, hd=64, ps=16, n=300, layout="rows"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999)))))))


def draw(rng):
    op = rng.choice(["append", "attention", "attention", "attention", "select", "fork"])
    layout = rng.choice(["rows", "heads"])
    dtype = rng.choice(["f16", "bf16"])
    hd = rng.choice([64, 128])
    ps = rng.choice([8, 16, 16, 20, 32, 64, 128])
    if op == "append":
        Hkv = rng.choice([1, 2, 4, 8, 12, 32, 40])
        S = _log_int(rng, 1, 256)
        T = _log_int(rng, 1, max(1, min(2048, 50_000_000 // (S * Hkv * hd))))
        return dict(op=op, dtype=dtype, S=S, T=T, ragged=rng.random() < 0.7, Hkv=Hkv, hd=hd, ps=ps, layout=layout)
    if op == "attention":
        H, Hkv = rng.choice([(32, 32), (40, 40), (12, 12), (32, 8), (64, 8), (16, 2), (71, 1), (24, 4)])
        S = _log_int(rng, 1, 64)
        n = _log_int(rng, 1, max(1, min(131072, 110_000_000 // (S * Hkv * hd))))
        window = _log_int(rng, 1, 4096) if rng.random() < 0.2 else 0
        return dict(op=op, dtype=dtype, S=S, H=H, Hkv=Hkv, hd=hd, n=n, ragged=rng.random() < 0.7, window=window, ps=ps,
                    layout=layout)
    if op == "select":
        W = rng.choice([1, 2, 3, 4, 5, 8, 12, 16, 32])
        V = _log_int(rng, 40, 160_000)
        return dict(op=op, B=_log_int(rng, 1, max(1, min(64, 12_000_000 // (W * V)))), W=W, V=V)
    W = rng.choice([1, 2, 3, 4, 6, 8, 16])
    Hkv = rng.choice([2, 8, 12, 32])
    L = rng.choice([1, 6, 12, 24])
    n = _log_int(rng, 1, 2048)
    token = L * 2 * Hkv * hd * 2  # bytes of a token in all layers
    pages = max(1, 2_500_000_000 // (token * ps))
    B = _log_int(rng, 1, max(1, min(32, pages // (-(-n // ps) + 4 * W + 2))))
    n = max(1, min(n, (pages // B - 4 * W - 2) * ps))
    return dict(op=op, dtype=dtype, B=B, W=W, L=L, Hkv=Hkv, hd=hd, ps=ps, n=n, layout=layout)


# ---- inputs -------------------------------------------------------------------


def _pool(g, dt, lead, Hkv, ps, hd, layout):
    """Pages [*lead, 2, Hkv, ps, hd] of N(0, 1) values."""
    if layout == "heads":
        return torch.randn((*lead, 2, Hkv, ps, hd), generator=g, device=DEV, dtype=dt)
    p = torch.randn((*lead, ps, 2, Hkv, hd), generator=g, device=DEV, dtype=dt)
    k = len(lead)
    return p.permute(*range(k), k + 1, k + 2, k, k + 3)


def _spread(S, n, ragged):
    """Lengths of S sequences, the longest n; ragged: even over their logarithm."""
    if not ragged:
        return np.full(S, n, np.int32)
    return np.minimum(np.exp(np.arange(1, S + 1) / S * math.log(n + 0.999)).astype(np.int32), n)


def _tables(rs, lens, ps, n_pages, width):
    """Page tables of sequences of `lens` tokens on pages in no order; -1 past the end."""
    need = -(-lens.astype(np.int64) // ps)
    t = np.full((len(lens), width), -1, np.int32)
    t[np.arange(width)[None, :] < need[:, None]] = rs.permutation(n_pages)[: int(need.sum())]
    return t


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rs = np.random.RandomState(seed % (1 << 32))
    return {"append": _prepare_append, "attention": _prepare_attention, "select": _prepare_select,
            "fork": _prepare_fork}[case["op"]](case, g, rs)


def _prepare_append(c, g, rs):
    dt, code = DT[c["dtype"]]
    S, T, Hkv, hd, ps = c["S"], c["T"], c["Hkv"], c["hd"], c["ps"]
    if T == 1:  # a decode step: one row per sequence, a finished sequence adds none
        count = (rs.uniform(size=S) < (0.9 if c["ragged"] else 2.0)).astype(np.int32)
        start = rs.randint(0, 600, S).astype(np.int32)
        n_pages = S * (-(-600 // ps))
    else:
        count = rs.permutation(_spread(S, T, c["ragged"]))
        start = np.zeros(S, np.int32)
        n_pages = int((-(-count // ps)).sum()) + 3
    tables = _tables(rs, start + count, ps, n_pages, -(-max(600, T) // ps) + 1)
    # rows of a fused q, k, v projection; sequences one after another
    N = int(count.sum()) if T > 1 else S
    row0 = np.concatenate([[0], np.cumsum(count)[:-1]]).astype(np.int32) if T > 1 else np.arange(S, dtype=np.int32)
    qkv = torch.randn((N, 3 * Hkv * hd), generator=g, device=DEV, dtype=dt)
    k, v = (qkv[:, i * Hkv * hd:(i + 1) * Hkv * hd].unflatten(1, (Hkv, hd)) for i in (1, 2))
    return dict(op="append", code=code, k=k, v=v, pool=_pool(g, dt, (n_pages,), Hkv, ps, hd, c["layout"]), T=T,
                tables=_dev(tables), start=_dev(start), lens=_dev(start + count), row0=_dev(row0))


def _prepare_attention(c, g, rs):
    dt, code = DT[c["dtype"]]
    S, H, Hkv, hd, ps = c["S"], c["H"], c["Hkv"], c["hd"], c["ps"]
    lens = rs.permutation(_spread(S, c["n"], c["ragged"]))
    n_pages = int((-(-lens // ps)).sum()) + 1
    tables = _tables(rs, lens, ps, n_pages, -(-c["n"] // ps) + 2)
    pool = _pool(g, dt, (n_pages,), Hkv, ps, hd, c["layout"])
    q = torch.randn((S, H, hd), generator=g, device=DEV, dtype=torch.float32)
    # the workspace is sized as a serving program would for its largest batch
    # (one fp32 row of hd + 2 per head and piece of a sequence), once
    return dict(op="attention", code=code, q=(q * 1.5).to(dt), pool=pool, tables=_dev(tables), lens=_dev(lens),
                scale=hd ** -0.5, window=c["window"], out=torch.empty((S, H, hd), device=DEV, dtype=dt),
                ws=torch.empty(64 << 20, device=DEV, dtype=torch.uint8))


def _prepare_select(c, g, rs):
    B, W, V = c["B"], c["W"], c["V"]
    logits = torch.randn((B * W, V), generator=g, device=DEV, dtype=torch.float32) * 2.5
    logits[:, torch.randint(0, V, (max(1, V // 200),), generator=g, device=DEV)] = -math.inf  # banned tokens
    logits[:, EOS] = logits[:, 3 * V // 4] + 3.0
    # hypotheses close to one another; about one in ten has ended
    scores = -np.sort(rs.uniform(5, 8, (B, W)).astype(np.float32), axis=1)
    alive = (rs.uniform(size=(B, W)) < 0.9).astype(np.int32)
    out = [torch.empty((B, W), device=DEV, dtype=t) for t in (torch.float32, torch.int32, torch.int32, torch.int32)]
    return dict(op="select", logits=logits, scores=_dev(scores), alive=_dev(alive), out=out,
                ws=torch.empty(16 << 20, device=DEV, dtype=torch.uint8))


def _prepare_fork(c, g, rs):
    dt, code = DT[c["dtype"]]
    B, W, L, Hkv, hd, ps, n = c["B"], c["W"], c["L"], c["Hkv"], c["hd"], c["ps"], c["n"]
    R = B * W
    lens = np.repeat(rs.permutation(_spread(B, n, True)), W)
    need = -(-lens.astype(np.int64) // ps)
    private = np.minimum(need, rs.randint(0, 3, R) + (lens % ps != 0))  # pages since the beams parted
    width = int(need.max()) + 2
    n_pages = int(need[::W].sum()) + 3 * R + R + 8
    order = rs.permutation(n_pages).astype(np.int32)
    tables = np.full((R, width), -1, np.int32)
    at = 0
    for b in range(B):
        shared = order[at:at + need[b * W]]
        at += len(shared)
        for r in range(b * W, (b + 1) * W):
            tables[r, :need[r]] = shared
            if private[r]:
                tables[r, need[r] - private[r]:need[r]] = order[at:at + private[r]]
                at += private[r]
    refs = np.bincount(tables[tables >= 0], minlength=n_pages).astype(np.int32)
    refs[tables[::2 * W, 0]] += 1  # first pages that a prompt cache keeps too
    parents = (np.repeat(np.arange(B) * W, W) + rs.randint(0, W, R)).astype(np.int32)
    grow = (rs.uniform(size=R) < 0.9).astype(np.int32)
    i32 = dict(device=DEV, dtype=torch.int32)
    return dict(op="fork", code=code, pool=_pool(g, dt, (L, n_pages), Hkv, ps, hd, c["layout"]), parents=_dev(parents),
                tables=_dev(tables), lens=_dev(lens.astype(np.int32)), refs=_dev(refs), grow=_dev(grow),
                out_tables=torch.empty((R, width), **i32), out_start=torch.empty(R, **i32),
                out_lens=torch.empty(R, **i32), out_refs=torch.empty(n_pages, **i32), short=torch.empty(2, **i32),
                ws=torch.empty(16 << 20, device=DEV, dtype=torch.uint8))


# ---- one pass -----------------------------------------------------------------


def run(state):
    if own:
        return _own(state)
    return {"append": _plain_append, "attention": _plain_attention, "select": _plain_select,
            "fork": _plain_fork}[state["op"]](state)


def _own(s):
    from paper_2503_17707_amd import binding as pb

    if s["op"] == "append":
        pb.op_kv_append(s["code"], s["k"], s["v"], s["pool"], s["tables"], s["start"], s["lens"], row0=s["row0"],
                        max_rows=s["T"])
        return s["pool"]
    if s["op"] == "attention":
        pb.op_paged_attention(s["code"], s["q"], s["pool"], s["tables"], s["lens"], s["out"], scale=s["scale"],
                              window=s["window"], workspace=s["ws"])
        return s["out"]
    if s["op"] == "select":
        pb.op_beam_select(s["logits"], s["scores"], s["alive"], *s["out"], eos=EOS, pad=PAD, workspace=s["ws"])
        return s["out"]
    pb.op_page_fork(s["code"], s["pool"], s["parents"], s["tables"], s["lens"], s["refs"], s["grow"], s["out_tables"],
                    s["out_start"], s["out_lens"], s["out_refs"], s["short"], workspace=s["ws"])
    return [s["out_tables"], s["out_start"], s["out_lens"], s["out_refs"], s["short"], s["pool"]]


def _plain_append(s):
    pool, tables, start, lens, row0 = s["pool"], s["tables"], s["start"], s["lens"], s["row0"]
    n_pages, ps = pool.shape[0], pool.shape[3]
    i = torch.arange(s["T"], device=DEV)
    x = start[:, None] + i
    col = torch.div(x, ps, rounding_mode="floor")
    page = tables.gather(1, col.clamp(max=tables.shape[1] - 1))
    keep = (x < lens[:, None]) & (col < tables.shape[1]) & (page >= 0) & (page < n_pages)
    rows = (row0[:, None] + i)[keep]
    page, t = page[keep].long(), (x % ps)[keep]
    pool[page, 0, :, t] = s["k"][rows]
    pool[page, 1, :, t] = s["v"][rows]
    return pool


def _plain_attention(s):
    q, pool, tables, lens = s["q"], s["pool"], s["tables"].long(), s["lens"]
    S, H, hd = q.shape
    Hkv, ps = pool.shape[2], pool.shape[3]
    kv = pool[tables.clamp(min=0)]  # [S, width, 2, Hkv, ps, hd]
    k, v = (kv[:, :, i].permute(0, 2, 1, 3, 4).reshape(S, Hkv, -1, hd).float() for i in (0, 1))
    x = torch.arange(k.shape[2], device=DEV)
    inside = x < lens[:, None]
    if s["window"]:
        inside &= x >= lens[:, None] - s["window"]
    a = torch.matmul(q.float().view(S, Hkv, H // Hkv, hd), k.transpose(2, 3)) * s["scale"]
    a = a.masked_fill(~inside[:, None, None], -math.inf)
    e = torch.exp(a - a.amax(-1, keepdim=True))
    v = v.masked_fill(~inside[:, None, :, None], 0.0)
    o = torch.matmul(e, v) / e.sum(-1, keepdim=True)
    return o.view(S, H, hd).to(q.dtype)


def _plain_select(s):
    # in 64 bits: candidates of different beams can lie closer than 32 bits tell
    logits, scores, alive = s["logits"].double(), s["scores"].double(), s["alive"] != 0
    B, W = scores.shape
    V = logits.shape[1]
    m = logits.amax(-1, keepdim=True)
    lp = logits - m - torch.log(torch.exp(logits - m).sum(-1, keepdim=True))
    # an ended hypothesis goes on as itself
    ended = torch.where(torch.arange(V, device=DEV) == PAD, 0.0, -math.inf).double()
    x = torch.where(alive.view(-1, 1), lp, ended)
    x = (x.view(B, W, V) + scores[:, :, None]).view(B, W * V)
    # the W largest, ties to the lowest index
    last = torch.topk(x, W, dim=1).values[:, -1:]
    above = x > last
    at = x == last
    keep = above | (at & (torch.cumsum(at, 1) <= W - above.sum(1, keepdim=True)))
    place = torch.where(keep, torch.cumsum(keep, 1) - 1, W)
    index = torch.zeros((B, W + 1), device=DEV, dtype=torch.long)
    index.scatter_(1, place, torch.arange(W * V, device=DEV).expand(B, -1))
    index = index[:, :W]
    value, order = torch.sort(x.gather(1, index), dim=1, descending=True, stable=True)
    index = index.gather(1, order)
    beam = torch.div(index, V, rounding_mode="floor")
    token = index % V
    row = beam + torch.arange(B, device=DEV)[:, None] * W
    still = alive.gather(1, beam) & (token != EOS)
    dead = value == -math.inf  # fewer candidates than places
    return [value.float(), torch.where(dead, PAD, token).int(), torch.where(dead, -1, row).int(), (still & ~dead).int()]


def _plain_fork(s):
    pool, tables, refs = s["pool"], s["tables"].long(), s["refs"].long()
    n_pages, ps = pool.shape[1], pool.shape[4]
    width = tables.shape[1]
    cols = torch.arange(width, device=DEV)
    one = torch.ones((), device=DEV, dtype=torch.long)

    def add(refs, pages, what):  # `what` added to the count of every page named
        at = torch.where(pages < 0, n_pages, pages).reshape(-1)
        return torch.cat([refs, refs.new_zeros(1)]).index_add(0, at, what.expand_as(pages).reshape(-1))[:-1]

    held = tables.masked_fill(cols >= ((s["lens"] + ps - 1) // ps)[:, None], -1)
    there = s["parents"] >= 0
    parent = s["parents"].long().clamp(min=0)
    start = torch.where(there, s["lens"][parent].long(), 0)
    new = held[parent].masked_fill(~there[:, None], -1)
    refs = add(add(refs, held, -one), new, one)
    # a row that grows past its table does not grow
    wide = there & (start + s["grow"] > width * ps)
    grow = torch.where(there & ~wide, s["grow"], 0).long()
    # a growing row needs its last, partly filled page to itself: the lowest one
    # keeps it if every reference is a growing row's, the others take a copy
    n = (start + ps - 1) // ps
    last = new.gather(1, (n - 1).clamp(min=0)[:, None])[:, 0]
    last = torch.where((grow > 0) & (start % ps != 0), last, -1)
    movers = add(torch.zeros_like(refs), last, one)
    rows = torch.arange(len(new), device=DEV)
    first = torch.full((n_pages + 1,), len(new), device=DEV)
    first = first.scatter_reduce(0, torch.where(last < 0, n_pages, last), rows, "amin")
    at = last.clamp(min=0)
    copies = (last >= 0) & ((refs[at] > movers[at]) | (rows != first[at]))
    # free pages in ascending order to rows in ascending order, or to none
    need = (start + grow + ps - 1) // ps - n + copies
    missing = (need.sum() - (add(refs, torch.where(copies, last, -1), -one) == 0).sum()).clamp(min=0)
    enough = missing == 0
    copies, need, grow = copies & enough, need * enough, grow * enough
    refs = add(refs, torch.where(copies, last, -1), -one)
    free = refs == 0
    frees = torch.zeros(n_pages + 1, device=DEV, dtype=torch.long)
    frees = frees.scatter(0, torch.where(free, torch.cumsum(free, 0) - 1, n_pages), torch.arange(n_pages, device=DEV))
    k = cols - (n - copies.long())[:, None]
    fresh = (k >= 0) & (k < need[:, None])
    given = frees[((torch.cumsum(need, 0) - need)[:, None] + k).clamp(0, n_pages - 1)]
    refs = add(refs, torch.where(fresh, given, -1), one)
    out = torch.where(fresh, given, new)
    # the tokens in the pages that are copied, in every layer
    c = copies.nonzero()[:, 0]
    src, dst = last[c], out.gather(1, (n - 1).clamp(min=0)[:, None])[c, 0]
    inside = torch.arange(ps, device=DEV) < (start[c] % ps)[:, None]
    pool[:, dst] = torch.where(inside[None, :, None, None, :, None], pool[:, src], pool[:, dst])
    short = torch.stack([missing, wide.sum()])
    return [out.int(), start.int(), (start + grow).int(), refs.int(), short.int(), pool]


# ---- what a pass cannot do without -----------------------------------------------


def work(case):
    c = case
    if c["op"] == "append":
        rows = int(_spread(c["S"], c["T"], c["ragged"]).sum())
        return {"bytes": 2 * rows * 2 * c["Hkv"] * c["hd"] * 2, "flops": 0}
    if c["op"] == "attention":
        keys = _spread(c["S"], c["n"], c["ragged"]).astype(np.int64)
        keys = int((np.minimum(keys, c["window"]) if c["window"] else keys).sum())
        return {"bytes": 2 * keys * 2 * c["Hkv"] * c["hd"] + 2 * 2 * c["S"] * c["H"] * c["hd"],
                "flops": 4 * keys * c["H"] * c["hd"]}
    if c["op"] == "select":
        return {"bytes": 4 * c["B"] * c["W"] * c["V"], "flops": 4 * c["B"] * c["W"] * c["V"]}
    # tables and counts once in and out; of W rows that choose among W parents
    # W (1 - 1/W)^W parents go unchosen: as many others share theirs and copy the
    # tokens of half a page in every layer (nine in ten rows grow)
    R, W = c["B"] * c["W"], c["W"]
    tables = 2 * 4 * (R * (-(-c["n"] // c["ps"]) + 2) + R)
    copies = 0.9 * R * (1 - 1 / W) ** W
    return {"bytes": tables + copies * 2 * (c["ps"] / 2) * 2 * c["Hkv"] * c["hd"] * 2 * c["L"], "flops": 0}


# ---- the definition in 64 bits ---------------------------------------------------


def exact(case, seed):
    if case["op"] not in ("attention", "select"):
        return None  # values are moved there, none is computed
    s = prepare(case, seed)
    return _exact_attention(s) if case["op"] == "attention" else _exact_select(s)


def _exact_attention(s):
    """One head of one sequence after another, over its own tokens alone."""
    q, pool, tables, lens = s["q"], s["pool"], s["tables"].tolist(), s["lens"].tolist()
    S, H, hd = q.shape
    Hkv, ps = pool.shape[2], pool.shape[3]
    out = torch.zeros((S, H, hd), device=DEV, dtype=torch.float64)
    for b in range(S):
        lo = max(0, lens[b] - s["window"]) if s["window"] else 0
        pages = torch.tensor(tables[b][lo // ps:-(-lens[b] // ps)], device=DEV)
        skip = lo - lo // ps * ps
        for h in range(Hkv):
            kv = pool[pages, :, h].transpose(0, 1).reshape(2, -1, hd)[:, skip:skip + lens[b] - lo].double()
            qh = q[b, h * (H // Hkv):(h + 1) * (H // Hkv)].double()
            p = torch.softmax((qh @ kv[0].t().contiguous()) * s["scale"], 1)
            out[b, h * (H // Hkv):(h + 1) * (H // Hkv)] = p @ kv[1]
    return out


def _exact_select(s):
    """Rows reduced to their own best tokens first, on the host."""
    B, W = s["scores"].shape
    scores, alive = s["scores"].double().cpu().numpy(), s["alive"].cpu().numpy()
    got = [np.zeros((B, W)), *(np.zeros((B, W), np.int32) for _ in range(3))]
    for b in range(B):
        found = []
        for w in range(W):
            row = b * W + w
            if not alive[b, w]:
                found.append((-scores[b, w], w, PAD))
                continue
            x = s["logits"][row].cpu().numpy().astype(np.float64)
            x[:] -= np.logaddexp.reduce(x)
            edge = np.partition(x, -min(W, len(x)))[-min(W, len(x))]
            best = [v for v in np.flatnonzero(x >= edge) if x[v] > -np.inf]
            found += [(-(scores[b, w] + x[v]), w, int(v)) for v in best]
        found = sorted(found)[:W]
        for i in range(W):
            score, w, v = found[i] if i < len(found) else (np.inf, -1 - b * W, PAD)
            got[0][b, i], got[1][b, i], got[2][b, i] = -score, v, b * W + w
            got[3][b, i] = i < len(found) and alive[b, w] and v != EOS
    return [torch.from_numpy(x) for x in got]
