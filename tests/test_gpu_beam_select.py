"""Beam selection against float64 candidates: widths, vocabularies, ties, banned
and undefined logits, ended and empty hypotheses."""
import numpy as np
import pytest

from gpu_common import log

pytestmark = pytest.mark.gpu

INF = float("inf")


def _run(logits, scores, alive, eos=2, pad=1, pitch=0, in_place=False, rows_apart=True):
    import torch

    from paged_common import select64
    from paper_2503_17707_amd import binding as pb

    logits = np.asarray(logits, np.float32)
    scores, alive = np.asarray(scores, np.float32), np.asarray(alive, np.int32)
    (B, W), V = scores.shape, logits.shape[1]
    log("beam select B=%d W=%d V=%d" % (B, W, V))
    want = select64(logits, scores, alive, eos, pad)
    lg = torch.full((B * W, V + pitch), float("nan"), device="cuda")
    lg[:, :V] = torch.from_numpy(logits)
    sc, al = torch.from_numpy(scores).cuda(), torch.from_numpy(alive).cuda()
    out = [sc if in_place else torch.full((B, W), 9.0, device="cuda"),
           *(torch.full((B, W), 9, dtype=torch.int32, device="cuda") for _ in range(2)),
           al if in_place else torch.full((B, W), 9, dtype=torch.int32, device="cuda")]
    ws = torch.full((pb.beam_select_workspace(B, W, V),), 255, dtype=torch.uint8, device="cuda")
    pb.op_beam_select(lg[:, :V], sc, al, *out, eos=eos, pad=pad, workspace=ws)
    for name, got, ref in zip(("tokens", "parents", "alive"), out[1:], want[1:]):
        if not rows_apart:
            break
        assert np.array_equal(got.cpu().numpy(), ref), (name, got.cpu().numpy(), ref)
    got = out[0].double().cpu().numpy()
    # fp32 sums of positive terms, each within (|l - m| log2 e + 4) 2^-24 of its
    # exponential where exponents, their products and the chunks' weights are rounded;
    # terms of l - m < -40 weigh under 2^-57 each; the logarithm's fraction is off by
    # up to 2 2^-24: the log sum is off by less than 64 2^-24 + V 2^-57, and the
    # sums of up to V / 64 terms per thread by at most another V / 64 2^-24 (V 2^-24 for
    # the shortest blocks); then one rounding of the score
    tol = (64 + min(V, 4096)) * 2.0 ** -24 + np.abs(want[0]) * 2.0 ** -24
    with np.errstate(invalid="ignore"):
        assert np.all((got == want[0]) | (np.abs(got - want[0]) <= tol))
    if not rows_apart:
        # Rows whose scores differ by less than the bound may come in either order: each choice
        # is as good as the one at its place, and the best tokens of its row, lowest first.
        tokens, parents = out[1].cpu().numpy(), out[2].cpu().numpy()
        x = logits.astype(np.float64)
        lse = x.max(1) + np.log(np.exp(x - x.max(1, keepdims=True)).sum(1))
        for b in range(B):
            taken = {}
            for j in range(W):
                r, t = parents[b, j], tokens[b, j]
                assert abs(scores[b, r - b * W] + x[r, t] - lse[r] - want[0][b, j]) <= tol[b, j]
                taken.setdefault(int(r), []).append(int(t))
            for r, ts in taken.items():
                assert ts == np.argsort(-x[r], kind="stable")[: len(ts)].tolist()
    return want


def _random(rs, B, W, V, sd=3.0):
    logits = rs.randn(B * W, V).astype(np.float32) * sd
    logits[:, rs.randint(0, V, max(1, V // 50))] = -INF
    scores = np.sort(-rs.uniform(2, 9, (B, W)), axis=1)[:, ::-1].astype(np.float32)
    return logits, scores, (rs.rand(B, W) < 0.85).astype(np.int32)


@pytest.mark.parametrize("W", [1, 2, 3, 4, 5, 8, 13, 16, 31, 32])
@pytest.mark.parametrize("B,V", [(1, 50272), (2, 1000), (3, 257)])
def test_widths(B, W, V):
    _run(*_random(np.random.RandomState(W), B, W, V))


@pytest.mark.parametrize("V", [3, 4, 5, 63, 64, 65, 255, 1023, 1024, 1025, 4095, 4097, 8191, 8193, 32000, 65537, 128256,
                               262147, 1 << 20])
def test_vocabularies(V):
    rs = np.random.RandomState(V)
    _run(*_random(rs, 2, 4, V))
    _run(*_random(rs, 1, 7, V), pitch=V % 3 + 1)  # rows that are not 16-byte aligned


@pytest.mark.parametrize("B", [17, 200, 700])
def test_many_prompts(B):
    _run(*_random(np.random.RandomState(B), B, 3, 501))


def test_more_places_than_candidates():
    rs = np.random.RandomState(4)
    for V, W in ((3, 8), (5, 32), (4, 3)):
        logits, scores, alive = _random(rs, 2, W, V)
        logits[0] = -INF
        logits[W:, 1:] = -INF
        _run(logits, scores, alive)
        _run(logits, scores, np.zeros_like(alive))


@pytest.mark.parametrize("W,V", [(4, 100), (8, 5000), (32, 50272)])
def test_ties_go_to_the_lowest_index(W, V):
    rs = np.random.RandomState(W)
    scores, alive = np.full((2, W), -1.5, np.float32), np.ones((2, W), np.int32)
    # all equal; few values; the same row for all beams
    _run(np.zeros((2 * W, V)), scores, alive)
    row = rs.randint(0, 3, V).astype(np.float32)
    _run(np.tile(row, (2 * W, 1)), scores, alive)
    _run(np.tile(row[::-1], (2 * W, 1)), scores, alive, eos=-1)
    # descending and ascending rows: the best in one place of the row
    _run(np.tile(np.linspace(5, -5, V), (2 * W, 1)), scores, alive)
    _run(np.tile(np.linspace(-5, 5, V), (2 * W, 1)), scores, alive)
    # all the best side by side, and one in each of W far places
    x = np.zeros((2 * W, V)); x[:, V // 2:V // 2 + 2 * W] = 4 + rs.rand(2 * W, 2 * W)
    _run(x, scores, alive)


def test_first_step_and_ended_hypotheses():
    rs = np.random.RandomState(6)
    W, V = 4, 900
    logits, scores, alive = _random(rs, 3, W, V)
    alive[:] = 1
    scores[:, 1:] = -INF
    scores[:, 0] = 0
    _run(logits, scores, alive)
    scores[1] = [np.nan, INF, -INF, -3]
    want = _run(logits, scores, alive)
    assert set(want[2][1]) == {W + 3}
    # ended ones compete with their own score; all ended
    scores[:] = np.sort(-rs.uniform(1, 4, (3, W)), axis=1)[:, ::-1]
    alive[0], alive[1, 1:] = 0, 0
    want = _run(logits, scores, alive, in_place=True)
    assert want[3][0].tolist() == [0] * W and want[2][0].tolist() == [0, 1, 2, 3]


def test_end_token_and_pad():
    rs = np.random.RandomState(7)
    logits, scores, alive = _random(rs, 2, 4, 300)
    logits[:, 299] = 30.0  # the end token is the best everywhere
    alive[:] = 1
    want = _run(logits, scores, alive, eos=299, pad=0)
    assert not want[3][:, 0].any()
    want = _run(logits, scores, alive, eos=-1, pad=299)
    assert want[3].all()


def test_logits_that_are_not_finite():
    rs = np.random.RandomState(8)
    logits, scores, alive = _random(rs, 2, 5, 2000)
    alive[:] = 1
    logits[:, ::3] = np.nan
    logits[1] = np.nan
    logits[2] = -INF
    logits[3, 700] = INF
    logits[4, [5, 6, 1999]] = INF
    logits[5] = INF
    logits[6, 10] = 3.4e38
    _run(logits, scores, alive)


def test_large_logits_and_scores():
    rs = np.random.RandomState(9)
    logits, scores, alive = _random(rs, 2, 4, 5000, sd=200.0)
    _run(logits, scores, alive)
    _run(logits * 1e30, scores, alive)
    _run(logits + 1e4, scores * 1000, alive)


@pytest.mark.parametrize("W", [7, 11, 12, 16, 20, 32])
@pytest.mark.parametrize("V", [33, 500, 954, 3000, 6245])
@pytest.mark.parametrize("spread", [0.0, 1e-3, 1.0])
def test_few_lists_of_many_entries(W, V, spread):
    """Rows about as good as each other: most of their entries reach the W-th best row's
    best, up to W x W of them, with equal ones among them or all equal."""
    rs = np.random.RandomState(W)
    logits, scores, alive = _random(rs, 5, W, V)
    alive[:] = 1
    scores[:] = -3 + spread * rs.randn(5, W)
    scores[1, ::2] = scores[1, 0]
    logits[2 * W : 3 * W] = logits[2 * W]                      # rows alike
    logits[3 * W : 4 * W] = np.round(logits[3 * W : 4 * W])    # few values
    logits[4 * W :] = 0.5
    _run(logits, scores, alive)


@pytest.mark.parametrize("W,V", [(1, 70000), (4, 60000), (8, 30000), (11, 20000), (12, 20000), (32, 60000), (16, 300000)])
@pytest.mark.parametrize("kind", ["equal", "low", "plateau", "steps"])
def test_crowds_of_equal_logits(W, V, kind):
    """Equal logits in every chunk of every row, of hypotheses with equal scores and not."""
    rs = np.random.RandomState(W)
    logits, scores, alive = _random(rs, 2, W, V)
    alive[:] = 1
    scores[0] = -4.0
    if kind == "equal":
        logits[:] = 0.25
    elif kind == "low":  # less is allowed than is asked for
        logits[:, rs.permutation(V)[3:]] = np.finfo(np.float32).min
    elif kind == "plateau":  # a few hundred equal best ones among others
        logits[:, rs.permutation(V)[: min(V, 400)]] = 20.0
        logits[0, V // 2 : V // 2 + 1000] = 20.0
    else:
        logits[:] = np.floor(np.arange(V) / 700.0) % 5
    # On the plateau rows of one score are not apart: their log sums are 20 + log(400 + s), where s
    # = sum e^(x - 20) over the others is some V e^(4.5 - 20) = V 1.9e-7, so they differ by parts
    # of s / 400 = V 4.6e-10 (3e-5 of 60000 logits) while the bound is over 64 2^-24 + 4096 2^-24
    # = 2.5e-4.
    _run(logits, scores, alive, rows_apart=kind != "plateau")


@pytest.mark.parametrize("far", [2.0 ** 21, 3.5e6, 2.0 ** 22, 5e6, 2.0 ** 23, 3e7])
@pytest.mark.parametrize("V", [37, 1024, 40000])
def test_logits_of_millions(far, V):
    """The whole number that exponents are taken relative to: at the end of its range, on
    both sides, in every logit or beside masked and ordinary ones."""
    rs = np.random.RandomState(11)
    for sign in (-1, 1):
        logits, scores, alive = _random(rs, 2, 4, V)
        alive[:] = 1
        near = np.isfinite(logits)
        logits[near] = sign * far
        logits[near] += np.float32(0.5) * rs.randint(-8, 9, near.sum()).astype(np.float32)
        logits[1, rs.rand(V) < 0.9] = np.finfo(np.float32).min
        logits[2, rs.rand(V) < 0.5] = -8e6
        logits[3, : V // 2] = rs.randn(V // 2)
        logits[4, V // 2:] = np.nan
        logits[5, V // 3] = INF
        logits[6, V // 3:] = -INF
        _run(logits, scores, alive)


@pytest.mark.parametrize("R,V", [(1, 255), (1, 257), (1, 1023), (1, 1024), (1, 1025), (3, 4097), (600, 8191), (600, 8192),
                                 (600, 8193), (300, 16385), (70, 50271), (70, 50273), (1, 131071)])
def test_every_logit_is_in_the_log_sum(R, V):
    """Log sums to the 2^-18 that are promised, where a logit left out or taken twice weighs more."""
    import torch

    from paper_2503_17707_amd import binding as pb

    log("beam select log sums", R, V)
    assert 1 / V > 1.5 * 2.0 ** -18  # of equal logits
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn((R, V), generator=g, device="cuda")
    x[0::3] = x[0::3, :1] * 3  # equal ones
    x[1::3] = 5 + 1e-3 * x[1::3]  # and nearly
    x[2::3] *= 3
    best, ref = x.double().max(1).values, torch.logsumexp(x.double(), 1)
    own = (ref - best).float().view(R, 1)  # leaves what the log sum is off by
    i32 = dict(dtype=torch.int32, device="cuda")
    out = [torch.empty((R, 1), device="cuda"), *(torch.empty((R, 1), **i32) for _ in range(3))]
    ws = torch.full((pb.beam_select_workspace(R, 1, V),), 255, dtype=torch.uint8, device="cuda")
    pb.op_beam_select(x, own, torch.ones((R, 1), **i32), *out, eos=-1, pad=0, workspace=ws)
    want = own[:, 0].double() + (best - ref)
    err = (out[0][:, 0].double() - want).abs()
    log("  worst error %.2e" % float(err.max()))
    assert torch.all(err <= 2.0 ** -18 + want.abs() * 2.0 ** -24)


def test_scores_below_the_lowest_float_are_none():
    import torch

    from paper_2503_17707_amd import binding as pb

    logits = torch.full((4, 9), -3e38, device="cuda")
    logits[:, 5] = 3e38  # the others' scores are -6e38
    scores = torch.tensor([[-1.0, -2.0], [-3.0, float("-inf")]], device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    alive = torch.ones((2, 2), **i32)
    out = [torch.empty((2, 2), device="cuda"), *(torch.empty((2, 2), **i32) for _ in range(3))]
    ws = torch.empty(pb.beam_select_workspace(2, 2, 9), dtype=torch.uint8, device="cuda")
    pb.op_beam_select(logits, scores, alive, *out, eos=2, pad=1, workspace=ws)
    assert out[0].tolist() == [[-1.0, -2.0], [-3.0, -INF]]
    assert [o.tolist() for o in out[1:]] == [[[5, 5], [5, 1]], [[0, 1], [2, -1]], [[1, 1], [1, 0]]]


def test_masks_of_the_lowest_float():
    """Tokens masked with the type's lowest value are the last candidates, not none."""
    rs = np.random.RandomState(10)
    low = np.finfo(np.float32).min
    logits, scores, alive = _random(rs, 3, 4, 700)
    alive[:] = 1
    logits[:, 3:] = low
    logits[4:8] = low
    _run(logits, scores, alive)
    _run(np.where(rs.rand(12, 700) < 0.5, low, -INF), scores, alive)
