"""Pages of a cache: rows appended, and pages shared, copied on write, handed out
and freed, against plain loops; bit for bit, the untouched bytes too."""
import numpy as np
import pytest

from gpu_common import log

pytestmark = pytest.mark.gpu


def _append(kind, Hkv, hd, ps, layout, start, lens, row0=None, max_rows=None, tables=None, n_pages=None, seed=0,
            rows=None):
    import torch

    from paged_common import CODE, DT, append_plain, dev, make_pool, make_tables
    from paper_2503_17707_amd import binding as pb

    log("append", kind, Hkv, hd, ps, layout, start[:6], lens[:6], max_rows)
    start, lens = np.array(start, np.int32), np.array(lens, np.int32)
    S = len(start)
    rs = np.random.RandomState(seed)
    if n_pages is None:
        n_pages = int(sum(-(-max(int(n), 0) // ps) for n in lens)) + 2
    if tables is None:
        tables = make_tables(rs, np.maximum(lens, 0), ps, n_pages, max(1, -(-int(lens.max()) // ps)))
    count = np.maximum(lens - start, 0)
    if rows is None:
        rows = S * max_rows if row0 is None else int(max(np.add(row0, count)))
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn((rows, 3 * Hkv * hd), generator=g).to(DT[kind]).cuda()
    k, v = (qkv[:, i * Hkv * hd:(i + 1) * Hkv * hd].unflatten(1, (Hkv, hd)) for i in (1, 2))
    pool = make_pool(seed + 1, kind, (n_pages,), Hkv, ps, hd, layout)
    want = append_plain(pool, k, v, tables, start, lens, row0, max_rows if max_rows is not None else rows, ps)
    whole = pool if pool._base is None else pool._base
    before = whole.clone()
    pb.op_kv_append(CODE[kind], k, v, pool, dev(tables), dev(start), dev(lens),
                    row0=None if row0 is None else dev(np.array(row0, np.int32)), max_rows=max_rows)
    assert torch.equal(pool.cpu(), want)
    # the bytes between tokens, heads and pages too
    inside = torch.zeros_like(whole, dtype=torch.bool)
    view = inside.as_strided(pool.shape, pool.stride(), pool.storage_offset())
    view.fill_(True)
    assert torch.equal(whole[~inside], before[~inside])


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("layout", ["rows", "heads", "gaps"])
@pytest.mark.parametrize("Hkv,hd,ps", [(1, 64, 16), (3, 128, 5), (32, 64, 16), (40, 128, 20)])
def test_append_one_token_each(kind, layout, Hkv, hd, ps):
    start = [0, 4, 15, 16, 37, 7]
    _append(kind, Hkv, hd, ps, layout, start, [1, 5, 16, 16, 38, 8], max_rows=1)  # the fourth adds none


@pytest.mark.parametrize("layout", ["rows", "heads"])
@pytest.mark.parametrize("Hkv,hd", [(2, 64), (40, 128)])
def test_append_prompts(layout, Hkv, hd):
    # ragged, packed one after another, some onto what their pages hold already
    lens = [1, 200, 33, 16, 47]
    start = [0, 0, 30, 16, 3]
    count = np.subtract(lens, start)
    row0 = np.concatenate([[0], np.cumsum(count)[:-1]])
    _append("bf16", Hkv, hd, 16, layout, start, lens, row0=row0.tolist(), max_rows=200)
    # a padded batch; and max_rows cutting longer sequences off
    _append("f16", Hkv, hd, 16, layout, [0, 0, 5], [33, 7, 5], max_rows=33)
    _append("f16", Hkv, hd, 16, layout, [0, 2, 5], [33, 7, 5], max_rows=9)


def test_append_with_a_bound_far_above_the_rows():
    # max_rows left at the number of rows: many blocks' worth for each of many sequences
    rs = np.random.RandomState(1)
    count = rs.randint(0, 40, 700)
    row0 = np.concatenate([[0], np.cumsum(count)[:-1]])
    _append("f16", 1, 64, 16, "heads", np.zeros(700), count, row0=row0.tolist())
    _append("bf16", 2, 128, 16, "rows", [0, 3], [9000, 5], max_rows=9000)


@pytest.mark.parametrize("Hkv,hd", [(1, 64), (32, 64), (40, 128)])
def test_append_without_a_bound(Hkv, hd):
    # the largest max_rows there is: as many rows as lens and start say
    _append("f16", Hkv, hd, 16, "rows", [0, 3, 7], [70, 3, 47], row0=[0, 70, 70], max_rows=2 ** 31 - 1)


def test_append_skips_what_has_no_place():
    tables = np.array([[0, -1, 2], [3, 9, 5], [6, 7, 8], [1, -3, 1 << 30]], np.int32)
    # holes, ids past the pool, past the width, a negative start, rows outside k and v
    _append("f16", 2, 64, 4, "heads", [0, 0, 0, 0], [12, 12, 15, 12], row0=[0, 3, 8, 12], max_rows=15, tables=tables,
            n_pages=9, rows=20)
    _append("f16", 2, 64, 4, "heads", [-1, 0, 2, 1], [12, 12, 1, -4], row0=[0, -3, 8, 12], max_rows=15, tables=tables,
            n_pages=9, rows=20)


def _fork(kind, L, Hkv, hd, ps, layout, parents, tables, lens, refs, grow, seed=0, twice=True):
    import torch

    from paged_common import CODE, dev, fork_plain, make_pool
    from paper_2503_17707_amd import binding as pb

    log("fork", kind, L, Hkv, hd, ps, layout, len(lens), "->", len(parents))
    parents, lens, refs, grow = (np.array(x, np.int32) for x in (parents, lens, refs, grow))
    tables = np.array(tables, np.int32)
    n_pages, width, R = len(refs), tables.shape[1], len(parents)
    pools = make_pool(seed, kind, (L, n_pages), Hkv, ps, hd, layout)
    want = fork_plain(pools, parents, tables, lens, refs, grow, ps)
    i32 = dict(dtype=torch.int32, device="cuda")
    outs = [torch.full(s, 77, **i32) for s in ((R, width), (R,), (R,), (n_pages,), (2,))]
    ws = torch.full((pb.page_fork_workspace(R, n_pages),), 255, dtype=torch.uint8, device="cuda")
    ins = [dev(x) for x in (parents, tables, lens, refs, grow)]
    for _ in range(2 if twice else 1):  # inputs are kept: the same call gives the same again
        pb.op_page_fork(CODE[kind], pools, *ins, *outs, ws)
        for name, got, ref in zip(("tables", "start", "lens", "refs", "short"), outs, want):
            assert np.array_equal(got.cpu().numpy(), ref), name
        assert torch.equal(pools.cpu(), want[5])
    return want


def _state(rs, B, W, ps, n_max, spare, foreign=0.3):
    """Beams of B prompts that share prefixes: tables, lens, refs."""
    R = B * W
    lens = np.repeat(rs.randint(1, n_max + 1, B), W)
    need = -(-lens // ps)
    private = np.minimum(need, rs.randint(0, 3, R) + (lens % ps != 0))
    n_pages = int(need[::W].sum() + private.sum()) + spare
    order = rs.permutation(n_pages).tolist()
    tables = np.full((R, int(need.max()) + 2), -1, np.int32)
    for b in range(B):
        shared = [order.pop() for _ in range(need[b * W])]
        for r in range(b * W, (b + 1) * W):
            tables[r, :need[r]] = shared
            for i in range(private[r]):
                tables[r, need[r] - 1 - i] = order.pop()
    refs = np.bincount(tables[tables >= 0], minlength=n_pages)
    refs[rs.rand(n_pages) < foreign] += 1  # held by others too, used or not
    return tables, lens, refs


@pytest.mark.parametrize("kind,L,Hkv,hd,layout", [("f16", 1, 1, 64, "heads"), ("bf16", 3, 2, 128, "rows"),
                                                  ("f16", 2, 5, 64, "gaps")])
@pytest.mark.parametrize("B,W,ps,n_max", [(1, 1, 16, 40), (1, 4, 16, 100), (3, 5, 7, 60), (8, 8, 16, 300), (2, 3, 1, 20)])
def test_fork_of_beams(kind, L, Hkv, hd, layout, B, W, ps, n_max):
    rs = np.random.RandomState(B * 100 + W)
    for seed in range(3):
        tables, lens, refs = _state(rs, B, W, ps, n_max, 3 * B * W + 9)
        R = B * W
        parents = np.repeat(np.arange(B) * W, W) + rs.randint(0, W, R)
        parents[rs.rand(R) < 0.1] = -1
        grow = np.where(rs.rand(R) < 0.8, rs.choice([1, 1, 1, 2, ps + 1]), 0)
        _fork(kind, L, Hkv, hd, ps, layout, parents, tables, lens, refs, grow, seed=seed)


@pytest.mark.parametrize("B,W,ps,n_max", [(1, 4, 16, 100), (3, 5, 7, 60), (8, 8, 4, 100)])
def test_fork_in_a_pool_of_many_pages(B, W, ps, n_max):
    """The same forks with more pages than one block's LDS counts."""
    rs = np.random.RandomState(B + W)
    for seed in range(3):
        tables, lens, refs = _state(rs, B, W, ps, n_max, 3 * B * W + 9)
        R = B * W
        parents = np.repeat(np.arange(B) * W, W) + rs.randint(0, W, R)
        parents[rs.rand(R) < 0.1] = -1
        grow = np.where(rs.rand(R) < 0.8, rs.choice([1, 1, 2, 3 * ps]), 0)
        used = np.ones(9000, refs.dtype)
        a = _fork("f16", 2, 1, 64, ps, "heads", parents, tables, lens, refs, grow, seed=seed)
        b = _fork("f16", 2, 1, 64, ps, "heads", parents, tables, lens, np.concatenate([refs, used]), grow, seed=seed)
        for x, y in zip(a[:3], b[:3]):
            assert np.array_equal(x, y)
        few = np.where(np.cumsum(refs == 0) > 3, np.maximum(refs, 1), refs)  # three free pages are left
        _fork("f16", 1, 1, 64, ps, "heads", parents, tables, lens, few, grow, seed=seed)
        _fork("f16", 1, 1, 64, ps, "heads", parents, tables, lens, np.concatenate([few, used]), grow, seed=seed)


@pytest.mark.parametrize("R_in,R_out", [(1, 7), (3, 12), (9, 2), (1500, 1300)])
def test_fork_to_another_number_of_rows(R_in, R_out):
    rs = np.random.RandomState(R_in)
    tables, lens, refs = _state(rs, R_in, 1, 16, 50, 2 * R_out + 7)
    _fork("f16", 2, 1, 64, 16, "heads", rs.randint(0, R_in, R_out), tables, lens, refs, rs.randint(0, 3, R_out), twice=False)


def test_fork_hands_out_prompts_and_frees_rows():
    # empty rows gain pages for prompts of several lengths, ascending
    want = _fork("f16", 1, 1, 64, 4, "heads", [0, 1, 2], np.full((3, 5), -1), [0, 0, 0], [0, 1, 0, 0, 2, 0, 0, 0, 0, 0, 0],
                 [9, 0, 20])
    assert want[0][0].tolist() == [0, 2, 3, -1, -1] and want[0][2].tolist() == [5, 6, 7, 8, 9]
    # dropping rows gives their pages back, and the same call hands them out
    want = _fork("f16", 1, 1, 64, 4, "heads", [-1, 1, 9], [[0, 1], [2, -1], [3, -1]], [8, 4, 2], [1, 1, 1, 1], [3, 4, 5])
    assert want[0].tolist() == [[-1, -1], [2, 0], [-1, -1]] and want[3].tolist() == [1, 0, 1, 0]


def test_fork_keeps_a_page_for_its_last_writer_only():
    # rows 0, 1 and 2 of parent 0 inside page 1: all grow: row 0 keeps it, two copies
    want = _fork("f16", 2, 1, 64, 4, "heads", [0, 0, 0], [[0, 1, -1]], [6], [1, 1, 0, 0, 0], [1, 1, 1])
    assert want[0].tolist() == [[0, 1, -1], [0, 2, -1], [0, 3, -1]] and want[3].tolist() == [3, 1, 1, 1, 0]
    # row 0 does not grow and goes on reading it: the others both copy
    want = _fork("f16", 2, 1, 64, 4, "heads", [0, 0, 0], [[0, 1, -1]], [6], [1, 1, 0, 0, 0], [0, 1, 1])
    assert want[0].tolist() == [[0, 1, -1], [0, 2, -1], [0, 3, -1]]
    # someone else's reference: nobody writes to it
    want = _fork("f16", 2, 1, 64, 4, "heads", [0, 0], [[0, 1, -1]], [6], [1, 2, 0, 0, 0], [1, 1])
    assert want[0].tolist() == [[0, 2, -1], [0, 3, -1]] and want[3].tolist() == [2, 1, 1, 1, 0]


def test_fork_without_enough_pages_or_width():
    # a row that would pass its table stays, the others grow and copy
    want = _fork("f16", 1, 1, 64, 4, "heads", [1, 1, 0], [[0, 1], [2, 3]], [6, 5], [1, 1, 1, 1, 0, 1, 1], [1, 1, 3])
    assert want[4].tolist() == [0, 1] and want[2].tolist() == [6, 6, 6]
    # one page missing: no row grows or copies, the reordering stands
    want = _fork("f16", 1, 1, 64, 4, "heads", [1, 1, 0], [[0, 1], [2, 3]], [6, 5], [1, 1, 1, 1, 1, 1, 1], [1, 1, 2])
    assert want[4].tolist() == [1, 0] and want[2].tolist() == [5, 5, 6]
    # rows past their table stay as they are, the others grow
    want = _fork("f16", 1, 1, 64, 4, "heads", [0, 1], [[0, 1], [2, 3]], [8, 5], [1, 1, 1, 1, 0], [1, 3])
    assert want[4].tolist() == [0, 1] and want[2].tolist() == [8, 8]
    want = _fork("f16", 1, 1, 64, 4, "heads", [0, 1], [[0, 1], [2, 3]], [99, -5], [1, 1, 0, 0, 0], [2 ** 31 - 1, 2])
    assert want[4].tolist() == [0, 1] and want[1].tolist() == [8, 0]
    # entries that are no page are passed over
    _fork("f16", 1, 1, 64, 4, "heads", [0, 1, 0], [[0, 7, -1], [-3, 2, -1]], [6, 5], [1, 0, 1, 0, 0, 0, 0], [1, 1, 1])


def test_fork_of_nothing():
    _fork("f16", 1, 1, 64, 4, "heads", [0], np.zeros((0, 3)), [], [0, 2], [5])
    _fork("f16", 1, 1, 64, 4, "heads", [], [[0, -1]], [3], [1, 0], [])


@pytest.mark.parametrize("n_pages", [2730, 2731, 8191, 8192, 8193])
@pytest.mark.parametrize("R", [6, 511])
def test_fork_where_pools_no_longer_fit_one_block(n_pages, R):
    """Pools around the sizes where one block counts their pages in more LDS, and no longer does:
    references and free pages to the last one, rows near the most that block takes too."""
    rs = np.random.RandomState(n_pages + R)
    width, ps = 16384 // 512, 8
    lens = rs.randint(1, 20, R) if R > 100 else rs.randint(1, width * ps - 9, R)
    need = -(-lens // ps)
    pages = n_pages - 1 - rs.permutation(min(n_pages, 2000))  # of the far end, the last one among them
    rs.shuffle(pages)
    tables = np.full((R, width), -1)
    free = list(pages)
    for r in range(R):
        tables[r, :need[r]] = [free.pop() for _ in range(need[r])]
    refs = np.bincount(tables[tables >= 0], minlength=n_pages)
    refs[: n_pages // 2] = 1  # held by others
    parents = np.sort(rs.randint(0, R, R))
    _fork("f16", 1, 1, 64, ps, "heads", parents, tables, lens, refs, rs.randint(0, 3, R), seed=R)


def test_fork_over_many_pages():
    """Free pages far into a large pool, most of it in use."""
    rs = np.random.RandomState(3)
    refs = np.ones(50000, np.int32)
    refs[[77, 1023, 1024, 20000, 49998, 49999]] = 0
    tables = np.full((2, 4), -1)
    tables[0, 0], tables[1, :2] = 5, [9, 10]
    _fork("f16", 1, 1, 64, 8, "heads", [0, 1, 0, 1], tables, [3, 16], refs, [1, 1, 9, 8], seed=int(rs.randint(9)))
