"""Every kernel of the 8-bit product in every way that its rule launches one, against float64
(test_q8_plans_cpu.py: that these are the launches)."""
import pytest

import q8_plans
from gpu_common import log

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,how,of", q8_plans.CASES, ids=lambda v: v if isinstance(v, str) else "")
def test_launch(name, how, of):
    """Sums are exact, and scaled as the kernels scale them: every bit is known."""
    import torch

    from paper_2503_17707_amd import binding as pb

    M, N, K, ldx, ldw, x, w, room = of
    log("gemm", name, how, of)
    g = torch.Generator("cuda").manual_seed(M + N + K)

    def rows(n, ld, at):
        buf = torch.randint(-128, 128, (at + n * ld,), generator=g, device="cuda", dtype=torch.int8)
        v = buf[at:].view(n, ld)[:, :K]
        assert v.data_ptr() % 128 == at
        return v

    X, W = rows(M, ldx, x), rows(N, ldw, w)
    sx = torch.rand(M, generator=g, device="cuda") + 0.5
    sw = torch.rand(N, generator=g, device="cuda") + 0.5
    ws = torch.full((room // 16 * 16,), 0x7f, dtype=torch.uint8, device="cuda") if room else None
    R = torch.full((M, N + 1), 77.0, device="cuda")
    C = torch.full((M, N + 1), 77.0, device="cuda", dtype=torch.float16)
    pb.op_gemm_q8(1, 3, X, sx, W, sw, None, R=R[:, :N], workspace=ws)
    pb.op_gemm_q8(1, 0, X, sx * 2.0 ** -18, W, sw, None, C=C[:, :N], qscale=0.5, qcols=N // 2, workspace=ws)
    want = torch.empty(M, N, device="cuda")
    for n in range(0, N, 4096):  # (below 2^53; rounded once)
        want[:, n:n + 4096] = (X.double() @ W[n:n + 4096].double().t()).float()
    want *= sx[:, None]
    want *= sw
    assert torch.equal(R[:, :N], want) and bool((R[:, N] == 77).all())
    want *= 2.0 ** -18
    want[:, :N // 2] *= 0.5
    assert torch.equal(C[:, :N], want.half()) and bool((C[:, N] == 77).all())
