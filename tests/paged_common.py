"""Inputs of the paged-cache tests and their plain implementations: float64 for
what is computed, loops over rows and tokens for what is moved."""
import math

import numpy as np
import torch

CODE = {"f16": 1, "bf16": 0}
DT = {"f16": torch.float16, "bf16": torch.bfloat16}
# half a step of the type, relative to the value
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def make_pool(seed, kind, lead, Hkv, ps, hd, layout, device="cuda"):
    """Pool [*lead, 2, Hkv, ps, hd]: "heads" contiguous, "rows" pages of [k | v] rows,
    "gaps" heads of pages with unused elements between tokens, heads and pages."""
    g = torch.Generator().manual_seed(seed)
    dt = DT[kind]
    k = len(lead)
    if layout == "heads":
        return torch.randn((*lead, 2, Hkv, ps, hd), generator=g).to(dt).to(device)
    if layout == "rows":
        p = torch.randn((*lead, ps, 2, Hkv, hd), generator=g).to(dt).to(device)
        return p.permute(*range(k), k + 1, k + 2, k, k + 3)
    p = torch.randn((*lead[:-1], lead[-1] + 1, 2, Hkv + 1, ps + 1, hd + 8), generator=g).to(dt).to(device)
    return p.narrow(k - 1, 0, lead[-1]).narrow(k + 1, 1, Hkv).narrow(k + 2, 0, ps).narrow(k + 3, 8, hd)


def make_tables(rs, lens, ps, n_pages, width):
    """Pages in no order for sequences of `lens` tokens; -1 past the end."""
    order = list(rs.permutation(n_pages))
    t = np.full((len(lens), width), -1, np.int32)
    for s, n in enumerate(lens):
        for i in range(-(-int(n) // ps)):
            t[s, i] = order.pop()
    return t


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def tokens_of(pool, ids, lo, hi, ps):
    """Keys and values [2, Hkv, hi - lo, hd] of tokens lo .. hi-1."""
    return torch.stack([pool[int(ids[x // ps]), :, :, x % ps] for x in range(lo, hi)], dim=2)


def attention64(q, pool, tables, lens, ps, scale, window):
    """(out, tolerance per element) in float64; q [S, H, hd], tables on the host.

    Tolerance, with u half a step of the storage type and V the largest |value|
    attended to: the probabilities enter the product with V rounded (each by a
    factor 1 + d, |d| <= u) and their sum holds the same rounded ones, so out moves
    by at most u max |V - out| <= 2 u V; a score's fp32 error ds (dot product of
    hd terms and its scaling: (hd + 4) 2^-24 sum |q k| scale, twice where a scaled
    q is rounded) moves a probability by a factor e^(+-ds): 4 ds V; fp32 sums over
    n tokens: 2 n 2^-24 V; then one rounding to the type, u |out| (and half its
    smallest step)."""
    kind = "f16" if q.dtype == torch.float16 else "bf16"
    u = HALF_STEP[kind]
    S, H, hd = q.shape
    Hkv = pool.shape[2]
    out = torch.zeros((S, H, hd), dtype=torch.float64)
    tol = torch.zeros((S, H, hd), dtype=torch.float64)
    qd, pd = q.double().cpu(), pool.cpu()
    for s in range(S):
        n = int(lens[s])
        lo = max(0, n - window) if window else 0
        if n <= 0:
            continue
        kv = tokens_of(pd, tables[s], lo, n, ps).double()
        for h in range(H):
            k, v = kv[0, h // (H // Hkv)], kv[1, h // (H // Hkv)]
            a = (k @ qd[s, h]) * scale
            p = torch.softmax(a, 0)
            out[s, h] = p @ v
            ds = 2 * (hd + 4) * 2.0 ** -24 * float((k.abs() @ qd[s, h].abs()).max()) * abs(scale)
            V = float(v.abs().max())
            tol[s, h] = V * (2 * u + 4 * ds + 2 * (n - lo) * 2.0 ** -24) + u * out[s, h].abs() + 2.0 ** -25
    return out, tol


def select64(logits, scores, alive, eos, pad):
    """Beam selection of float64 candidates, one by one."""
    B, W = scores.shape
    V = logits.shape[1]
    outs = [np.full((B, W), -np.inf), np.full((B, W), pad, np.int32), np.full((B, W), -1, np.int32),
            np.zeros((B, W), np.int32)]
    for b in range(B):
        found = []
        for w in range(W):
            own = float(scores[b, w])
            if not math.isfinite(own):
                continue
            if not alive[b, w]:
                found.append((-own, w * V + pad, w, pad, 0))
                continue
            x = logits[b * W + w].astype(np.float64)
            x = np.where(np.isnan(x), -np.inf, np.minimum(x, np.finfo(np.float32).max))
            m = x.max()
            if m == -np.inf:
                continue
            lp = own + ((x - m) - math.log(np.exp(x - m).sum()))
            best = np.lexsort((np.arange(V), -lp))[:W]
            found += [(-lp[v], w * V + int(v), w, int(v), int(v != eos)) for v in best if lp[v] > -np.inf]
        for i, (neg, _, w, v, live) in enumerate(sorted(found)[:W]):
            outs[0][b, i], outs[1][b, i], outs[2][b, i], outs[3][b, i] = -neg, v, b * W + w, live
    return outs


def append_plain(pool, k, v, tables, start, lens, row0, max_rows, ps):
    """The pool after an append, token by token (a copy, on the host)."""
    out, k, v = pool.cpu().clone(), k.cpu(), v.cpu()
    for s in range(len(start)):
        if start[s] < 0:
            continue
        for i in range(min(int(lens[s]) - int(start[s]), max_rows)):
            x = int(start[s]) + i
            row = (int(row0[s]) if row0 is not None else s * max_rows) + i
            if x // ps >= tables.shape[1] or not 0 <= row < len(k):
                continue
            page = int(tables[s, x // ps])
            if 0 <= page < len(out):
                out[page, 0, :, x % ps] = k[row]
                out[page, 1, :, x % ps] = v[row]
    return out


def fork_plain(pools, parents, tables, lens, refs, grow, ps):
    """The fork, row by row: (tables, start, lens, refs, short, pools), on the host."""
    pools = pools.cpu().clone()
    n_pages, width = len(refs), tables.shape[1]
    refs = refs.astype(np.int64).copy()
    R = len(parents)
    lens = np.clip(lens, 0, width * ps)
    pages = [-(-int(n) // ps) for n in lens]
    good = lambda p: p if 0 <= p < n_pages else -1  # noqa: E731
    rows, start, g, wide = [], [], [], 0
    for r in range(len(lens)):
        for i in range(pages[r]):
            if good(tables[r, i]) >= 0:
                refs[tables[r, i]] -= 1
    for r in range(R):
        p = int(parents[r])
        there = 0 <= p < len(lens)
        rows.append([good(int(x)) for x in tables[p, :pages[p]]] if there else [])
        start.append(int(lens[p]) if there else 0)
        more = max(int(grow[r]), 0) if there else 0
        if start[r] + more > width * ps:
            wide, more = wide + 1, 0
        g.append(more)
        for x in rows[r]:
            if x >= 0:
                refs[x] += 1
    last = [rows[r][-1] if g[r] > 0 and start[r] % ps else -1 for r in range(R)]
    copies = []
    for r in range(R):
        others = refs[last[r]] - last.count(last[r]) if last[r] >= 0 else 0
        copies.append(last[r] >= 0 and (others > 0 or last.index(last[r]) != r))
    need = [-(-(start[r] + g[r]) // ps) - len(rows[r]) + copies[r] for r in range(R)]
    free = [i for i in range(n_pages) if refs[i] == 0]
    missing = max(0, sum(need) - len(free))
    if missing:
        g, need, copies = [0] * R, [0] * R, [False] * R
    out = np.full((R, width), -1, np.int32)
    for r in range(R):
        if copies[r]:
            refs[last[r]] -= 1
            dst = free.pop(0)
            pools[:, dst, :, :, :start[r] % ps] = pools[:, last[r], :, :, :start[r] % ps]
            rows[r][-1] = dst
            refs[dst] += 1
            need[r] -= 1
        for _ in range(need[r]):
            rows[r].append(free.pop(0))
            refs[rows[r][-1]] += 1
        out[r, :len(rows[r])] = rows[r]
    start = np.array(start, np.int32)
    return out, start, start + np.array(g, np.int32), refs.astype(np.int32), np.array([missing, wide], np.int32), pools
