"""Attention of one new token over a paged cache against float64: lengths from none
to thousands, pages of every kind of size, head groups, layouts, windows, and
what a table may hold outside the tokens attended to."""
import numpy as np
import pytest

from gpu_common import log

pytestmark = pytest.mark.gpu


def _run(kind, H, Hkv, hd, ps, layout, lens, window=0, seed=0, scale=None, ws="own", width=None, ld_extra=0):
    import torch

    from paged_common import CODE, DT, attention64, dev, make_pool, make_tables
    from paper_2503_17707_amd import binding as pb

    log("paged attention", kind, H, Hkv, hd, ps, layout, lens, window, ws)
    rs = np.random.RandomState(seed)
    S = len(lens)
    lens = np.array(lens, np.int32)
    n_pages = int(sum(-(-max(int(n), 0) // ps) for n in lens)) + 2
    width = width or max(1, -(-int(max(lens)) // ps))
    tables = make_tables(rs, np.maximum(lens, 0), ps, n_pages, width)
    pool = make_pool(seed, kind, (n_pages,), Hkv, ps, hd, layout)
    for s in range(S):  # what follows a sequence's last token, and unused pages, is NaN
        if lens[s] > 0 and lens[s] % ps:
            pool[int(tables[s, (lens[s] - 1) // ps]), :, :, lens[s] % ps:] = float("nan")
    for p in set(range(n_pages)) - set(tables.ravel().tolist()):
        pool[p] = float("nan")
    g = torch.Generator().manual_seed(seed + 1)
    rows = (torch.randn((S, H * hd + ld_extra), generator=g) * 2).to(DT[kind]).cuda()
    q = rows[:, :H * hd].unflatten(1, (H, hd))
    scale = hd ** -0.5 if scale is None else scale
    full = torch.full((S + 2, H * hd + ld_extra), 7.0, dtype=DT[kind], device="cuda")
    out = full[1:S + 1, :H * hd].unflatten(1, (H, hd))
    work = None
    if ws == "own":
        need = pb.paged_attention_workspace(S, H, pool, width)
        work = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
    elif ws == "small":
        work = torch.full((5000,), 255, dtype=torch.uint8, device="cuda")
    pb.op_paged_attention(CODE[kind], q, pool, dev(tables), dev(lens), out, scale=scale, window=window, workspace=work)
    ref, tol = attention64(q, pool, tables, lens, ps, scale, window)
    err = (out.double().cpu() - ref).abs()
    worst = float((err / tol.clamp(min=1e-300)).max())
    log("  worst error / tolerance %.3f" % worst)
    assert torch.all(err <= tol), "worst error / tolerance %.3f" % worst
    # rows before the first and behind the last sequence, and between rows, are untouched
    assert torch.all(full[0] == 7) and torch.all(full[S + 1] == 7) and torch.all(full[:, H * hd:] == 7)
    return out


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("layout", ["rows", "heads", "gaps"])
def test_lengths(kind, hd, layout):
    _run(kind, 4, 4, hd, 16, layout, [1, 0, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 255, 257, 511, 513])


@pytest.mark.parametrize("ps", [1, 2, 3, 7, 8, 20, 48, 64, 100, 128, 333, 4096])
@pytest.mark.parametrize("hd", [64, 128])
def test_page_sizes(ps, hd):
    _run("f16", 2, 2, hd, ps, "heads", [1, 99, 333, 700, 64], width=max(1, -(-700 // ps)) + 3)


@pytest.mark.parametrize("H,Hkv", [(1, 1), (2, 1), (3, 1), (8, 2), (16, 1), (17, 1), (24, 4), (33, 1), (40, 8), (71, 1),
                                   (130, 2)])
@pytest.mark.parametrize("kind,hd", [("bf16", 128), ("f16", 64)])
def test_head_groups(kind, hd, H, Hkv):
    _run(kind, H, Hkv, hd, 16, "rows", [1, 37, 300, 1025], ld_extra=40)


@pytest.mark.parametrize("window", [1, 2, 16, 31, 100, 1000])
@pytest.mark.parametrize("ps", [1, 16, 20])
def test_windows(window, ps):
    _run("bf16", 4, 2, 64, ps, "heads", [0, 1, 2, 16, 33, 100, 101, 700], window=window)


@pytest.mark.parametrize("ws", ["own", "small", None])
@pytest.mark.parametrize("lens", [[5000], [4097, 1, 0, 900], [2048] * 3])
@pytest.mark.parametrize("kind,H,Hkv,hd", [("f16", 4, 4, 64), ("bf16", 8, 1, 128)])
def test_long_sequences_in_pieces(kind, H, Hkv, hd, lens, ws):
    _run(kind, H, Hkv, hd, 16, "rows", lens, ws=ws)


@pytest.mark.parametrize("S", [70, 300, 1100])
def test_many_sequences(S):
    rs = np.random.RandomState(S)
    lens = rs.randint(0, 90, S)
    lens[S // 2] = 1500
    _run("f16", 2, 1, 64, 16, "heads", lens.tolist())


@pytest.mark.parametrize("kind,H,hd,ps,n,window,layout,ws", [
    ("f16", 16, 128, 16, 5000, 0, "rows", True),     # pieces
    ("f16", 16, 128, 1, 5000, 0, "heads", True),     # pieces of more pages than are held at a time
    ("bf16", 16, 64, 1, 1500, 0, "rows", False),     # whole, eight waves
    ("f16", 1, 64, 1, 700, 0, "gaps", False),        # whole, four waves
    ("bf16", 32, 128, 20, 3001, 0, "heads", True),   # two operands of queries, pieces
    ("f16", 32, 64, 1, 1300, 0, "rows", False),      # two operands, whole
    ("bf16", 16, 128, 16, 4000, 1111, "rows", True),
    ("f16", 40, 64, 7, 2100, 900, "heads", False),
])
def test_every_token_counts_once(kind, H, hd, ps, n, window, layout, ws):
    """A query per token whose key it shares with one other token alone: the output is the mean
    of their two values, and would show either of them left out or taken twice."""
    import torch

    from paged_common import CODE, DT, HALF_STEP, dev, make_pool, make_tables
    from paper_2503_17707_amd import binding as pb

    log("paged attention token by token", kind, H, hd, ps, n, window)
    g = torch.Generator().manual_seed(n)
    lo = n - window if window else 0
    half = (n - lo) // 2
    keys = (torch.randint(0, 2, (n, hd), generator=g) * 2 - 1).double()
    keys[lo + half:lo + 2 * half] = keys[lo:lo + half]
    values = torch.randn((n, hd), generator=g).to(DT[kind])
    pages = -(-n // ps)
    tables = make_tables(np.random.RandomState(n), [n], ps, pages, pages)
    pool = make_pool(1, kind, (pages,), 1, ps, hd, layout)
    pool.fill_(float("nan"))
    x = torch.arange(n)
    at = torch.from_numpy(tables[0]).long()[x // ps].cuda(), (x % ps).cuda()
    pool[at[0], 0, 0, at[1]] = keys.to(DT[kind]).cuda()
    pool[at[0], 1, 0, at[1]] = values.cuda()
    S = -(-2 * half // H)
    who = lo + torch.arange(S * H) % (2 * half)  # the token that a query asks for
    q = keys[who].to(DT[kind]).view(S, H, hd).cuda()
    out = torch.empty_like(q)
    work = None
    if ws:
        work = torch.full((pb.paged_attention_workspace(S, H, pool, pages),), 255, dtype=torch.uint8, device="cuda")
        assert work.numel() > 0
    pb.op_paged_attention(CODE[kind], q, pool, dev(np.repeat(tables, S, 0)), dev(np.full(S, n, np.int32)), out, window=window,
                          workspace=work)
    k, v = keys[lo:].cuda(), values[lo:].double().cuda()
    p = torch.softmax(keys[who].cuda() @ k.t().contiguous(), 1)
    ref = p @ v
    # scores are whole numbers up to hd: their factor to base two and its product round, equal
    # ones alike; parts of probabilities, sums and the output as elsewhere
    u, V = HALF_STEP[kind], float(v.abs().max())
    tol = V * (4 * u * u + 4 * 5 * hd * 2.0 ** -24 + 2 * len(v) * 2.0 ** -24) + u * ref.abs() + 2.0 ** -25
    mine = p.gather(1, (who - lo).cuda()[:, None])
    gap = mine * (v[who - lo] - ref)  # over 1 -+ mine: what a token left out or taken twice changes
    assert torch.all((gap.abs() / (1 + mine) > 4 * tol).any(1))
    err = (out.view(-1, hd).double() - ref).abs()
    log("  worst error / tolerance %.3f" % float((err / tol).max()))
    assert torch.all(err <= tol)


@pytest.mark.parametrize("S,H,Hkv,hd,window", [(128, 4, 2, 128, 0), (129, 4, 2, 128, 0), (200, 2, 2, 64, 0), (1500, 1, 1, 64, 0), (1024, 2, 1, 128, 0),
                                               (300, 2, 1, 64, 2100)])
def test_many_sequences_in_pieces(S, H, Hkv, hd, window):
    """Sequences of none to thousands of tokens in wide tables, where the cut is listed first and not."""
    rs = np.random.RandomState(S)
    lens = rs.randint(0, 24, S)
    lens[[3, S // 2, S - 2]] = [4999, 2500, 129]
    lens[[5, S - 1]] = [-7, 1600]
    _run("f16", H, Hkv, hd, 16, "heads", lens.tolist(), window=window, width=400)


def test_many_long_sequences_and_one_past_its_table():
    import torch

    from paged_common import attention64, dev, make_pool
    from paper_2503_17707_amd import binding as pb

    log("paged attention many long")
    S, ps, hd, pages = 140, 16, 64, 256
    rs = np.random.RandomState(0)
    lens = rs.randint(1, 4097, S).astype(np.int32)
    lens[7] = 4097
    pool = make_pool(0, "f16", (pages,), 1, ps, hd, "heads")
    tables = np.stack([rs.permutation(pages) for _ in range(S)]).astype(np.int32)  # pages in common
    tables[9, :] = -1
    q = torch.randn((S, 2, hd), generator=torch.Generator().manual_seed(1)).half().cuda()
    ws = torch.full((pb.paged_attention_workspace(S, 2, pool, pages),), 255, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    pb.op_paged_attention(1, q, pool, dev(tables), dev(lens), out, scale=0.125, workspace=ws)
    bad = torch.isnan(out).flatten(1)
    assert bad[[7, 9]].all() and not bad[[i for i in range(S) if i not in (7, 9)]].any()
    some = [0, 1, 8, 10, 63, 64, 65, 100, 139]
    ref, tol = attention64(q[some], pool, tables[some], lens[some], ps, 0.125, 0)
    assert torch.all((out[some].double().cpu() - ref).abs() <= tol)
    plain = torch.empty_like(q)  # no sequence in pieces
    pb.op_paged_attention(1, q, pool, dev(tables), dev(lens), plain, scale=0.125)
    rest = [i for i in range(S) if i not in (7, 9)]
    assert (out[rest].float() - plain[rest].float()).abs().max() < 2e-3


def test_peaked_and_flat_scores():
    # large scores: one key takes all; scale 0: the mean of the values
    _run("f16", 4, 4, 64, 16, "heads", [700, 65], scale=3.0)
    _run("f16", 4, 4, 64, 16, "heads", [700, 65], scale=0.0)
    _run("bf16", 4, 4, 128, 16, "heads", [700, 65], scale=-0.3)


@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("kind,hd", [("f16", 64), ("bf16", 128)])
def test_scores_far_from_zero_in_many_pieces(kind, hd, sign):
    """Scores near sign * 600 in sequences cut in many ways, the cut not a multiple of a tile."""
    import torch

    from paged_common import CODE, DT, attention64, dev, make_pool, make_tables
    from paper_2503_17707_amd import binding as pb

    log("paged attention far scores", kind, hd, sign)
    rs = np.random.RandomState(4)
    lens = np.concatenate([rs.randint(1, 6000, 30), [5999, 2049, 129, 1]]).astype(np.int32)
    ps, width = 16, 380
    n_pages = int((-(-lens // ps)).sum())
    tables = make_tables(rs, lens, ps, n_pages, width)
    pool = make_pool(5, kind, (n_pages,), 2, ps, hd, "heads")
    pool[:, 0, :, :, 0] = sign * 60.0
    q = torch.randn((len(lens), 4, hd), device="cuda").to(DT[kind])
    q[..., 0] = 10.0
    for rows in (len(lens), 7):
        out = torch.empty_like(q[:rows])
        ws = torch.full((pb.paged_attention_workspace(rows, 4, pool, width),), 255, dtype=torch.uint8, device="cuda")
        assert ws.numel() > 0
        pb.op_paged_attention(CODE[kind], q[:rows], pool, dev(tables[:rows]), dev(lens[:rows]), out, workspace=ws)
        ref, tol = attention64(q[:rows], pool, tables[:rows], lens[:rows], ps, 1.0, 0)
        assert torch.all((out.double().cpu() - ref).abs() <= tol)


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("n", [40, 5000])
def test_scores_of_millions(kind, n):
    """Two keys tie far above the others, at scores where fp32 steps are whole numbers: the
    output is the mean of their values, exactly."""
    import torch

    from paged_common import CODE, DT, dev
    from paper_2503_17707_amd import binding as pb

    hd, ps = 64, 16
    pages = -(-n // ps)
    pool = torch.zeros((pages, 2, 1, ps, hd), dtype=DT[kind], device="cuda")
    pool[:, 1] = 100.0
    for x, v in ((3, 1.0), (n - 2, 2.0)):
        pool[x // ps, 0, 0, x % ps, 0] = 2.0 ** 13
        pool[x // ps, 1, 0, x % ps] = v
    q = torch.zeros((1, 1, hd), dtype=DT[kind], device="cuda")
    tables, lens = dev(np.arange(pages, dtype=np.int32)[None]), dev(np.array([n], np.int32))
    ws = torch.full((pb.paged_attention_workspace(1, 1, pool, pages) + 16,), 255, dtype=torch.uint8, device="cuda")
    for e in (8, 10, 11, 12, 13, 14, 15):
        for scale in (1.0, 0.8, 8.0):
            log("paged attention scores of millions", kind, n, e, scale)
            q[..., 0] = 2.0 ** e
            out = torch.full_like(q, float("nan"))
            pb.op_paged_attention(CODE[kind], q, pool, tables, lens, out, scale=scale, workspace=ws)
            assert torch.all(out == 1.5), (e, scale, out[0, 0, :4].tolist())


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("H,hd", [(1, 64), (3, 128), (20, 128)])
def test_probabilities_are_not_rounded_to_the_type(kind, H, hd):
    """Half the keys weigh 1, half e^a, and their values cancel but for their own rounding: a
    probability that is rounded to the storage type shows, by up to half a step."""
    import torch

    from paged_common import CODE, DT, HALF_STEP, attention64, dev
    from paper_2503_17707_amd import binding as pb

    log("paged attention probabilities", kind, H, hd)
    S, n, ps = 40, 64, 16
    a = -torch.linspace(0.02, 1.0, S).to(DT[kind])
    pool = torch.zeros((S, n // ps, 2, 1, ps, hd), dtype=DT[kind])
    pool[:, :, 0, :, 1::2, 0] = a[:, None, None, None]
    pool[:, :, 1, :, 0::2] = 1.0
    pool[:, :, 1, :, 1::2] = -torch.exp(-a.double()).to(DT[kind])[:, None, None, None, None]
    pool = pool.flatten(0, 1).cuda()
    q = torch.zeros((S, H, hd), dtype=DT[kind], device="cuda")
    q[..., 0] = 1.0
    tables, lens = np.arange(S * n // ps, dtype=np.int32).reshape(S, -1), np.full(S, n, np.int32)
    out = torch.empty_like(q)
    pb.op_paged_attention(CODE[kind], q, pool, dev(tables), dev(lens), out)
    ref, _ = attention64(q, pool, tables, lens, ps, 1.0, 0)
    # |a| <= 1: the factor to base two, its product and the exponential are off by 5 2^-24 of a
    # probability, its parts by 2 u^2; both in numerator and sum; fp32 sums over n tokens
    u = HALF_STEP[kind]
    tol = 2.75 * (4 * u * u + (20 + 2 * n) * 2.0 ** -24) + u * ref.abs() + 2.0 ** -25
    err = (out.double().cpu() - ref).abs()
    log("  worst error / tolerance %.3f" % float((err / tol).max()))
    assert torch.all(err <= tol)


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("H,n", [(2, 500), (2, 5000), (20, 5000)])
def test_other_dimensions_beside_an_infinite_value(kind, H, n):
    import torch

    from paged_common import CODE, DT, attention64, dev, make_pool
    from paper_2503_17707_amd import binding as pb

    log("paged attention beside infinities", kind, H, n)
    ps, hd = 16, 64
    pages = -(-n // ps)
    pool = make_pool(3, kind, (pages,), 1, ps, hd, "heads")
    for x, j, v in ((n // 2, 5, float("inf")), (n - 1, 20, -float("inf"))):
        pool[x // ps, 1, 0, x % ps, j] = v
    q = torch.randn((1, H, hd), generator=torch.Generator().manual_seed(4)).to(DT[kind]).cuda()
    out, tables = torch.empty_like(q), np.arange(pages, dtype=np.int32)[None]
    ws = torch.full((pb.paged_attention_workspace(1, H, pool, pages) + 16,), 255, dtype=torch.uint8, device="cuda")
    pb.op_paged_attention(CODE[kind], q, pool, dev(tables), dev(np.array([n], np.int32)), out, scale=0.1, workspace=ws)
    assert torch.all(out[..., 5] == float("inf")) and torch.all(out[..., 20] == -float("inf"))
    pool[pool.isinf()] = 0
    ref, tol = attention64(q, pool, tables, [n], ps, 0.1, 0)
    keep = [j for j in range(hd) if j not in (5, 20)]
    assert torch.all(((out.double().cpu() - ref).abs() <= tol)[..., keep])


def test_many_small_probabilities_beside_a_large_one():
    """One key far above 20000 others that weigh 2^-18 each: together 7 percent."""
    import torch

    from paged_common import attention64, dev
    from paper_2503_17707_amd import binding as pb

    n, hd, ps = 20000, 64, 16
    log("paged attention small probabilities")
    pool = torch.zeros((n // ps, 2, 1, ps, hd), dtype=torch.float16, device="cuda")
    pool[:, 1] = 1.0
    pool[0, 0, 0, 0, 0] = 18 * 0.6931471805599453
    pool[0, 1, 0, 0] = -1.0
    q = torch.zeros((1, 1, hd), dtype=torch.float16, device="cuda")
    q[..., 0] = 1.0
    tables = np.arange(n // ps, dtype=np.int32)[None]
    out = torch.empty_like(q)
    ws = torch.empty(pb.paged_attention_workspace(1, 1, pool, n // ps) + 16, dtype=torch.uint8, device="cuda")
    pb.op_paged_attention(1, q, pool, dev(tables), dev(np.array([n], np.int32)), out, workspace=ws)
    ref, tol = attention64(q, pool, tables, [n], ps, 1.0, 0)
    assert torch.all((out.double().cpu() - ref).abs() <= tol)


@pytest.mark.parametrize("window", [500, 641, 1024, 1500, 4000])
@pytest.mark.parametrize("H,Hkv,hd", [(8, 2, 64), (8, 2, 128), (24, 1, 128), (40, 1, 64)])
def test_windows_of_long_sequences(window, H, Hkv, hd):
    """Whole and cut by what the window leaves, whatever the tables hold."""
    _run("bf16", H, Hkv, hd, 16, "rows", [0, 1, 499, 1500, 3001, 5000], window=window, width=400)


@pytest.mark.parametrize("window", [0, 40])
def test_bad_pages_give_nan_only_where_they_are_attended_to(window):
    import torch

    from paged_common import dev, make_pool, make_tables
    from paper_2503_17707_amd import binding as pb

    log("paged attention bad pages", window)
    ps, hd, H = 16, 64, 2
    lens = np.array([100, 100, 100, 100, 100, 90, -5], np.int32)
    tables = make_tables(np.random.RandomState(1), np.clip(lens, 0, 96), ps, 50, 6)
    tables[:5, 5] = [59, 58, 57, 56, 55]
    tables = np.concatenate([tables, np.full((7, 1), -1, np.int32)], 1)
    tables[:5, 6] = [50, 51, 52, 53, 54]
    tables[1, 6], tables[2, 5], tables[3, 0], tables[4, 2] = -1, 60, -7, 1 << 30
    pool = make_pool(1, "f16", (60,), H, ps, hd, "heads")
    q = torch.randn((7, H, hd), device="cuda").half()
    out = torch.empty_like(q)
    pb.op_paged_attention(1, q, pool, dev(tables), dev(lens), out, window=window)
    nan = torch.isnan(out.flatten(1)).all(1).tolist()
    fine = torch.isfinite(out.flatten(1)).all(1).tolist()
    in_reach = not window  # pages 0 and 2 (tokens 0-15, 32-47) lie before the last 40 tokens
    assert nan == [False, True, True, in_reach, in_reach, False, False]
    assert fine == [not x for x in nan]
    assert torch.all(out[6] == 0)
    # lens past the table's width
    lens[5] = 7 * ps + 1
    pb.op_paged_attention(1, q, pool, dev(tables), dev(lens), out, window=window)
    assert torch.isnan(out[5]).all()


def test_values_that_are_not_finite_come_through():
    """An infinite value at a token attended to reaches the output as the formula has it."""
    import torch

    from paged_common import dev, make_pool
    from paper_2503_17707_amd import binding as pb

    log("paged attention infinities")
    pool = make_pool(3, "bf16", (4,), 1, 16, 64, "heads")
    pool[1, 1, 0, 3, 5] = float("inf")
    pool[2, 1, 0, 2, 9] = float("nan")
    pool[3, 1, 0, 11, 20] = -float("inf")  # the last token, in the middle of a tile
    q = torch.randn((1, 1, 64), device="cuda").bfloat16()
    out = torch.empty_like(q)
    pb.op_paged_attention(0, q, pool, dev(np.array([[0, 1, 2, 3]], np.int32)), dev(np.array([60], np.int32)), out, scale=0.1)
    assert out[0, 0, 5] == float("inf") and torch.isnan(out[0, 0, 9])
    assert out[0, 0, 20] == -float("inf")
    keep = [i for i in range(64) if i not in (5, 9, 20)]
    assert torch.isfinite(out[0, 0, keep]).all()


def test_pool_past_32_bit_offsets():
    """Pages more than 2^32 bytes (and 2^31 elements) into a pool."""
    import torch

    from paged_common import attention64, dev
    from paper_2503_17707_amd import binding as pb

    log("paged attention large pool")
    ps, hd, H = 16, 128, 2
    n_pages = (5 << 30) // (2 * H * ps * hd * 2)
    pool = torch.empty((n_pages, 2, H, ps, hd), dtype=torch.float16, device="cuda")
    far = [n_pages - 1, 3, n_pages - 2, n_pages // 2 + 7]
    g = torch.Generator(device="cuda").manual_seed(5)
    for p in far:
        pool[p] = torch.randn(pool[p].shape, generator=g, device="cuda").half()
    tables = np.array([far], np.int32)
    k = torch.randn((1, H, hd), generator=g, device="cuda").half()
    pb.op_kv_append(1, k, k, pool, dev(tables), dev(np.array([60], np.int32)), dev(np.array([61], np.int32)))
    assert torch.equal(pool[far[3], 0, :, 12], k[0]) and torch.equal(pool[far[3], 1, :, 12], k[0])
    q = torch.randn((1, H, hd), generator=g, device="cuda").half()
    out = torch.empty_like(q)
    pb.op_paged_attention(1, q, pool, dev(tables), dev(np.array([61], np.int32)), out, scale=0.1)
    near = torch.stack([pool[p] for p in far])
    ref, tol = attention64(q, near, np.arange(4, dtype=np.int32)[None], [61], ps, 0.1, 0)
    assert torch.all((out.double().cpu() - ref).abs() <= tol)
