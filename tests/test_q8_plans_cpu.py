"""The rule of sizes of the 8-bit product, asked on the host: which products the GPU tests have to hold."""
import pytest


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    import q8_plans

    path = q8_plans.host_program(tmp_path_factory.mktemp("q8_plans"))
    if path is None:
        pytest.skip("hipcc not available")
    return path


def _rows(cases):
    return [of[:5] + (of[5] + (1 << 30), of[6] + (1 << 30), of[7]) for of in cases]


def test_cases_are_the_launches_that_they_are_named_by(exe):
    import q8_plans as P

    got = P.plans(exe, _rows([of for _, _, of in P.CASES]))
    wrong = [(name, how, of, P.label(of[2], plan)) for (name, how, of), plan in zip(P.CASES, got) if P.label(of[2], plan) != (name, how)]
    assert not wrong


def test_cases_hold_every_launch_that_a_sample_reaches(exe):
    import q8_plans as P

    rows = P.sample(7, 400_000)
    got = P.plans(exe, rows)
    reached = {P.label(K, plan): (K, tuple(plan)) for K, plan in zip(rows[:, 2].tolist(), got.tolist())}
    missing = set(reached) - {(name, how) for name, how, _ in P.CASES}
    assert not missing
    assert len(reached) > 100  # (a sample that reaches little shows little)


def test_ranges_hold_every_step_of_a_launch_once(exe):
    """Whole tiles and split ones are all tiles; a range has a step at least, the last one the rest; the sums fit
    the workspace that was given."""
    import numpy as np
    import q8_plans as P

    rows = P.sample(8, 200_000)
    got = P.plans(exe, rows)
    M, N, K, room = (rows[:, i] for i in (0, 1, 2, 7))
    shape, splits, tail, full, kt, phases, _, need = (got[:, i] for i in range(8))
    bm, bn = (np.array([t[i] for t in P.TILES])[shape] for i in (0, 1))
    step = np.array([k[1] for k in P.KERNELS])[shape]
    assert ((full + tail) == -(-M // bm) * -(-N // bn)).all()
    assert ((tail > 0) == (splits > 1)).all() and (full >= 0).all()
    cut = splits > 1
    whole = K // step
    assert ((splits - 1) * kt < whole)[cut].all() and (splits * kt >= whole)[cut].all()
    assert ((tail * splits * bm * bn * 4) <= np.minimum(need, room))[cut].all()
    assert np.isin(phases, (1, 16)).all()
    few = np.array([k[0].startswith("few") for k in P.KERNELS])[shape]
    assert (M <= 16)[few].all() and not cut[few].any()
    assert (K >= 128)[shape >= 8].all()  # two stages of their ring are filled without asking


def test_a_workspace_for_the_most_tokens_serves_fewer(exe):
    """pb_op_gemm_q8_workspace(M, N, K) holds the sums of every call of up to M tokens, on rows of any stride."""
    import numpy as np
    import q8_plans as P

    from paper_2503_17707_amd import binding as pb

    rows = P.sample(9, 60_000)
    rows = np.concatenate([rows, [(m, n, k, k, k, 1 << 30, (1 << 30) + 16, 0) for n, k in ((5120, 5120), (2048, 8192), (4096, 16384))
                                  for m in range(1, 2049)]])  # weights off lines
    rng = np.random.default_rng(1)
    most = np.where(rng.integers(0, 2, len(rows)) == 0, rows[:, 0], rows[:, 0] + rng.integers(0, 4096, len(rows)))
    asked = np.array([pb.gemm_q8_workspace(int(m), int(r[1]), int(r[2])) for m, r in zip(most, rows)])
    assert (asked >= 0).all() and (asked <= P.ASKED).all() and not (asked % 16).any()
    rows[:, 7] = 1 << 40
    free = P.plans(exe, rows)
    over = (free[:, 7] > asked).nonzero()[0]
    assert not len(over), (len(over), rows[over[:3]].tolist(), most[over[:3]], asked[over[:3]], free[over[:3]].tolist())
    rows[:, 7] = asked
    assert (P.plans(exe, rows) == free).all()
