"""Products of 8-bit rows (pb_op_gemm_q8) against float64."""
import math

import pytest

from gpu_common import log

pytestmark = pytest.mark.gpu


def _case(M, N, K, seed=0, kind="f16", bias=True):
    import torch

    from q8_common import DT, numbers8

    g = torch.Generator().manual_seed(seed)
    return dict(X=numbers8(g, M, K), W=numbers8(g, N, K), sx=torch.rand(M, generator=g) * 0.02 + 0.01,
                sw=torch.rand(N, generator=g) * 0.01 / math.sqrt(K) + 1e-4,
                bias=torch.randn(N, generator=g).to(DT[kind]) if bias else None, old=torch.randn(M, N, generator=g) * 3)


def _run(c, epi, kind="f16", pad=(0, 0, 0), ws=None, qscale=0.125, qcols=0, fill=77):
    """The product on rows with `pad` more columns in X, W and the output; checks what lies around it."""
    import torch

    from paper_2503_17707_amd import binding as pb
    from q8_common import CODE, DT, strided, untouched

    M, K = c["X"].shape
    N = c["W"].shape[0]
    X = strided(c["X"].cuda(), K + pad[0])[0]
    W = strided(c["W"].cuda(), K + pad[1])[0]
    out, buf = strided(c["old"].to(DT[kind] if epi < 2 else torch.float32).cuda(), N + pad[2], pad[2] // 2)
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    log("gemm", kind, M, N, K, "epi", epi, pad, "ws", 0 if ws is None else ws.numel())
    pb.op_gemm_q8(CODE[kind], epi, X, dev(c["sx"]), W, dev(c["sw"]), dev(c["bias"]), C=out if epi < 2 else None,
                  R=out if epi >= 2 else None, qscale=qscale, qcols=qcols, workspace=ws)
    torch.cuda.synchronize()
    assert untouched(buf, N, pad[2] // 2)
    return out.cpu()


def _check(c, got, epi, kind="f16", qscale=0.125, qcols=0):
    from q8_common import DT, gemm64

    want, tol = gemm64(c["X"], c["sx"], c["W"], c["sw"], c["bias"], epi, qscale, qcols, c["old"], DT[kind])
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), (float((off - tol).max()), int((off > tol).sum()))


def _ws(M, N, K):
    """The workspace that the product asks for, holding what is no sum."""
    import torch

    from paper_2503_17707_amd import binding as pb

    n = pb.gemm_q8_workspace(M, N, K)
    return torch.full((max(n, 16),), 0x7f, dtype=torch.uint8, device="cuda")


SIZES = [(1, 1, 16), (1, 64, 64), (1, 6144, 2048), (1, 5, 4080), (2, 2048, 8192), (3, 129, 112), (4, 768, 768), (5, 4999, 560),
         (8, 2048, 2048), (9, 100, 5104), (15, 300, 16), (16, 512, 8192), (17, 1000, 1008), (24, 4096, 1024), (31, 63, 4096),
         (33, 257, 2048), (48, 2000, 512), (64, 512, 5120), (65, 65, 80), (100, 1030, 1040), (127, 640, 2048),
         (130, 5120, 1280), (200, 384, 9216), (257, 515, 528), (333, 1280, 5120), (512, 512, 512), (700, 999, 1008),
         (1000, 2050, 272), (1511, 777, 640), (2048, 1024, 256), (4100, 520, 144), (3, 50272, 128)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_sizes(M, N, K):
    import torch

    kind = ("f16", "bf16")[(M + N) % 2]
    c = _case(M, N, K, seed=M * 31 + N, kind=kind)
    qcols = N // 3
    ws = _ws(M, N, K)
    got = _run(c, 0, kind, qcols=qcols, ws=ws)
    _check(c, got, 0, kind, qcols=qcols)
    # the workspace decides nothing but time
    assert torch.equal(got, _run(c, 0, kind, qcols=qcols))
    for epi in (1, 2, 3):
        got = _run(c, epi, kind, ws=ws)
        _check(c, got, epi, kind)


# Small products that the rule of sizes gives to each kernel: whole tiles, all tiles split, the
# last round's split; K in whole steps and with a rest.
KERNELS = [
    (1, 12373, 256), (13, 15858, 64), (1, 32, 256), (1, 32, 64), (1, 12100, 768), (1, 12199, 640), (16, 4096, 5104),  # up to 16 tokens
    (1, 44, 9984), (1, 32, 7552), (1, 16552, 7392), (17, 32, 256), (19, 35, 80),  # 32 x 32
    (1, 677, 8192), (1, 637, 8320), (1, 18401, 7680), (1, 16437, 8064), (1, 13857, 768), (1, 12713, 896),  # 32 x 64
    (67, 36, 11520), (76, 47, 9520), (48, 17268, 8704), (1, 19002, 7856), (78, 33, 256), (67, 36, 64),  # 64 x 64
    (11, 49, 5760), (68, 32, 2240), (68, 32, 128), (20, 16566, 64),  # 64 x 128
    (597, 32, 2048), (523, 32, 2608), (76, 18124, 3760), (589, 36, 256), (520, 35, 160),  # 128 x 64
    (616, 32, 1408), (549, 40, 1936), (648, 5403, 2816), (493, 8400, 1888), (593, 33, 128), (555, 32, 80),  # 128 x 128
    (1054, 1222, 8320), (863, 1775, 9632), (970, 8278, 14208), (135, 22328, 128), (132, 22859, 160),  # 128 x 256
    (142, 6242, 10240), (134, 7007, 8784), (1294, 12451, 2176), (566, 27430, 1472), (283, 23145, 128),
    (306, 26156, 144),  # 192 x 256
    (227, 8456, 9600), (229, 5384, 10704), (983, 16718, 1664), (683, 21867, 1616), (402, 22195, 128),
    (400, 26092, 144),  # 256 x 256
    (1, 13185, 2048), (1, 12146, 2176), (386, 4785, 6656), (88, 16863, 5328), (143, 6423, 9312), (566, 31211, 5504),
    (556, 22808, 2224), (403, 8506, 6784), (198, 22556, 3872),
    (1, 754, 12032), (1, 918, 8320), (97, 19052, 12288), (639, 35, 1920), (1337, 86, 30288), (177, 16833, 3088), (1278, 1036, 12864),
    (392, 5836, 10880), (452, 5855, 7744), (1169, 13350, 2816), (500, 5888, 7744), (1169, 13312, 2816),
    (88, 47, 8336), (1, 18285, 24624), (248, 8249, 6800), (111, 19495, 10272), (377, 11177, 2480), (2662, 6290, 2128),
    (152, 5752, 10304), (528, 27648, 2768), (231, 10660, 12048),
    # weight rows a multiple of 4 KB apart: columns of tiles that start at other places of K
    (20, 1000, 4096), (40, 600, 8192), (64, 2100, 12288), (100, 5000, 4096), (128, 20000, 4096), (90, 520, 16384),
]


# bytes / 16 before X's and W's first row and between their rows; lines are 8 of them
OFF = [(0, 1, 0, 1), (1, 0, 0, 0), (0, 0, 7, 0), (3, 2, 5, 4), (7, 7, 1, 3), (4, 5, 2, 6), (2, 4, 6, 2), (5, 6, 3, 7)]


@pytest.mark.parametrize("M,N,K", [(40, 700, 512), (50, 6144, 1280), (200, 640, 128), (200, 1000, 144), (150, 2000, 1664), (333, 1280, 5120),
                                   (260, 8192, 4096), (500, 520, 256), (900, 2048, 1920), (1511, 4999, 400), (1100, 5000, 128),
                                   (1500, 5000, 272), (1000, 1300, 9216)])
@pytest.mark.parametrize("off", OFF, ids=str)
def test_rows_off_lines(M, N, K, off):
    """Rows that start anywhere in a line of 128 bytes: sums are exact, so every bit is that of packed rows."""
    import torch

    from paper_2503_17707_amd import binding as pb

    log("gemm off lines", M, N, K, off)
    g = torch.Generator("cuda").manual_seed(M + N + K)

    def rows(n, before, between):
        ld = (K + 127) // 128 * 128 + 16 * between
        buf = torch.randint(-128, 128, (16 * before + n * ld,), generator=g, device="cuda").to(torch.int8)
        return buf[16 * before:].view(n, ld)[:, :K]

    X, W = rows(M, off[0], off[1]), rows(N, off[2], off[3])
    sx = torch.rand(M, generator=g, device="cuda") + 0.5
    sw = torch.rand(N, generator=g, device="cuda") + 0.5
    n64 = (X.double() @ W.double().t()).float()  # exact sums, rounded once, as the kernels round them
    want = n64 * sx[:, None] * sw[None]
    for ws in (_ws(M, N, K), None):
        R = torch.zeros(M, N, device="cuda")
        pb.op_gemm_q8(1, 3, X, sx, W, sw, None, R=R, workspace=ws)
        assert torch.equal(R, want)


@pytest.mark.parametrize("M,N,K", KERNELS)
def test_every_kernel(M, N, K):
    import torch

    from paper_2503_17707_amd import binding as pb
    from q8_common import gemm64

    log("gemm", M, N, K)
    g = torch.Generator("cuda").manual_seed(M + N + K)
    draw = lambda *of: torch.randint(-128, 128, of, generator=g, device="cuda").to(torch.int8)  # noqa: E731
    X, W = draw(M, K), draw(N, K)
    sx = torch.rand(M, generator=g, device="cuda") * 0.02 + 0.01
    sw = torch.rand(N, generator=g, device="cuda") * 0.01 / math.sqrt(K) + 1e-4
    bias = torch.randn(N, generator=g, device="cuda").half()
    old = torch.randn(M, N, generator=g, device="cuda")
    R = old.clone()
    pb.op_gemm_q8(1, 2, X, sx, W, sw, bias, R=R, workspace=_ws(M, N, K))
    want, tol = gemm64(X, sx, W, sw, bias, 2, 1.0, 0, old, torch.float16)
    assert bool(((R.double() - want).abs() <= tol).all())
    C = torch.zeros(M, N, dtype=torch.float16, device="cuda")
    pb.op_gemm_q8(1, 1, X, sx, W, sw, bias, C=C, workspace=_ws(M, N, K))
    want, tol = gemm64(X, sx, W, sw, bias, 1, 1.0, 0, old, torch.float16)
    assert bool(((C.double() - want).abs() <= tol).all())
    bias = bias.bfloat16()
    C = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
    pb.op_gemm_q8(0, 0, X, sx, W, sw, bias, C=C, qscale=0.3, qcols=N // 2 + 1, workspace=_ws(M, N, K))
    want, tol = gemm64(X, sx, W, sw, bias, 0, 0.3, N // 2 + 1, old, torch.bfloat16)
    assert bool(((C.double() - want).abs() <= tol).all())
    pb.op_gemm_q8(0, 3, X, sx, W, sw, None, R=R, workspace=_ws(M, N, K))
    want, tol = gemm64(X, sx, W, sw, None, 3, 1.0, 0, old, torch.bfloat16)
    assert bool(((R.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("M,N,K", [(1, 300, 2048), (7, 130, 1040), (40, 515, 2064), (150, 260, 528), (600, 600, 320),
                                   (2100, 300, 96)])
@pytest.mark.parametrize("pad", [(16, 48, 8), (112, 16, 1), (4096, 32, 3), (32, 4096, 31)], ids=str)
def test_strides(M, N, K, pad):
    c = _case(M, N, K, seed=7, bias=M != 7)
    for epi, kind in ((0, "bf16"), (2, "f16"), (1, "f16"), (3, "bf16")):
        c["bias"] = None if c["bias"] is None else c["bias"].to(dtype={"f16": c["old"].half().dtype, "bf16": c["old"].bfloat16().dtype}[kind])
        _check(c, _run(c, epi, kind, pad, ws=_ws(M, N, K), qcols=N), epi, kind, qcols=N)


def test_rows_are_the_same_in_every_batch():
    """The kernels and splits differ with the sizes, the bits do not."""
    import torch

    M, N, K = 700, 1536, 4096
    c = _case(M, N, K, seed=3)
    whole = _run(c, 2, ws=_ws(M, N, K))
    for lo, n in ((0, 1), (5, 2), (9, 4), (20, 8), (30, 16), (50, 24), (77, 60), (100, 100), (300, 256)):
        part = dict(c, X=c["X"][lo:lo + n], sx=c["sx"][lo:lo + n], old=c["old"][lo:lo + n])
        for ws in (None, _ws(n, N, K)):
            assert torch.equal(_run(part, 2, ws=ws), whole[lo:lo + n]), (lo, n)
    some = dict(c, W=c["W"][:130], sw=c["sw"][:130], bias=c["bias"][:130], old=c["old"][:, :130])
    assert torch.equal(_run(some, 2, ws=_ws(M, 130, K)), whole[:, :130])


def test_workspaces_of_every_size():
    import torch

    for M, N, K in ((1, 512, 8192), (20, 640, 8192), (120, 520, 8192), (300, 512, 16384)):
        c = _case(M, N, K, seed=11)
        want = _run(c, 3)
        _check(c, want, 3)
        for n in (16, 4 * M * N - 16, 4 * M * N, 8 * M * N, 12 * M * N + 16, 32 * M * N, 64 << 20):
            ws = torch.full((n // 16 * 16,), 0x7f, dtype=torch.uint8, device="cuda")
            assert torch.equal(_run(c, 3, ws=ws), want), (M, N, K, n)


@pytest.mark.parametrize("M", [1, 6, 20, 100, 300, 1100])
def test_the_largest_sums(M):
    """-128 times -128 over the longest K, and 127 times -128: no sum passes 32 bits."""
    import torch

    N, K = 70, 131056
    c = _case(M, N, 16, seed=1)
    c["X"], c["W"] = torch.full((M, K), -128, dtype=torch.int8), torch.full((N, K), -128, dtype=torch.int8)
    c["W"][33:] = 127
    c["sx"], c["sw"] = torch.full((M,), 1.0), torch.full((N,), 2.0 ** -20)
    for ws in (None, _ws(M, N, K)):
        got = _run(c, 3, ws=ws)
        want = torch.where(torch.arange(N) < 33, 16384.0 * K, -16256.0 * K) * 2.0 ** -20
        off = (got.double() - want.double() - c["bias"].double()).abs()
        assert bool((off <= 2.0 ** -24 * 3.1 * want.abs().double()).all())


@pytest.mark.parametrize("M", [2, 30, 200, 1300])
def test_scales_that_are_no_numbers(M):
    """NaN, infinite, zero and negative scales stay in their row and column; ReLU keeps NaN."""
    import torch

    N, K = 150, 256
    c = _case(M, N, K, seed=2)
    clean = _run(c, 1)
    c["sx"][1] = math.nan
    c["sw"][140] = math.nan
    c["sw"][7] = 0.0
    got = _run(c, 1, ws=_ws(M, N, K))
    assert bool(torch.isnan(got[1]).all()) and bool(torch.isnan(got[:, 140]).all())
    assert torch.equal(got[0, 7], c["bias"][7].clamp(min=0))
    keep = torch.ones(M, N, dtype=torch.bool)
    keep[1], keep[:, 140], keep[:, 7] = False, False, False
    assert torch.equal(got[keep], clean[keep])


def test_qcols_at_every_place():
    c = _case(5, 70, 64, seed=9)
    for qcols in (-1, 0, 1, 3, 4, 62, 69, 70, 1000):
        _check(c, _run(c, 0, qcols=qcols), 0, qcols=qcols)


def test_weights_past_four_gigabytes():
    import torch

    from paper_2503_17707_amd import binding as pb

    N, K = 70000, 65536  # 4.6 GB
    W = torch.zeros(N, K, dtype=torch.int8, device="cuda")
    W[-2:] = 3
    for M in (1, 30, 200):
        X = torch.ones(M, K, dtype=torch.int8, device="cuda")
        R = torch.zeros(M, N, device="cuda")
        log("gemm of 4.6 GB", M)
        pb.op_gemm_q8(1, 3, X, torch.ones(M, device="cuda"), W, torch.ones(N, device="cuda"), R=R)
        assert bool((R[:, -2:] == 3.0 * K).all()) and not bool(R[:, :-2].any())


def test_outputs_past_four_gigabytes():
    import torch

    from paper_2503_17707_amd import binding as pb

    M, N, K = 22000, 50272, 16  # 4.4 GB of fp32
    X = torch.zeros(M, K, dtype=torch.int8, device="cuda")
    X[-1] = 2
    W = torch.ones(N, K, dtype=torch.int8, device="cuda")
    R = torch.full((M, N), 7.0, device="cuda")
    log("gemm of 4.4 GB of output")
    pb.op_gemm_q8(1, 3, X, torch.ones(M, device="cuda"), W, torch.ones(N, device="cuda"), R=R)
    assert bool((R[-1] == 32.0).all()) and not bool(R[:-1].any())
