"""8-bit linear layers without a GPU: every refusal of the C entry points and of the
wrappers, and the workspace sizes."""
import ctypes

import pytest

A = [0x100000000 * (i + 1) for i in range(12)]  # operands far from one another; no refused call follows them


def _norm(pb, dtype=1, layer=0, x=A[0], ld_x=64, f32=0, delta=A[1], ld_delta=64, sum=A[2], ld_sum=64, g=A[3], b=A[4],
          eps=1e-5, out=A[5], ld_out=64, q=A[6], ld_q=64, scale=A[7], rows=4, d=64):
    return pb.lib().pb_op_norm_q8(dtype, layer, x, ld_x, f32, delta, ld_delta, sum, ld_sum, g, b, eps, out, ld_out, q,
                                  ld_q, scale, rows, d, None)


def _quant(pb, dtype=1, x=A[0], ld_x=64, f32=0, q=A[1], ld_q=64, scale=A[2], rows=4, cols=64):
    return pb.lib().pb_op_quant_q8(dtype, x, ld_x, f32, q, ld_q, scale, rows, cols, None)


def _gemm(pb, dtype=1, epi=0, X=A[0], ldx=64, sx=A[1], W=A[2], ldw=64, sw=A[3], bias=A[4], C=A[5], R=A[6], ldo=32, M=4, N=32,
          K=64, qscale=1.0, qcols=0, ws=A[7], ws_bytes=1 << 16):
    return pb.lib().pb_op_gemm_q8(dtype, epi, X, ldx, sx, W, ldw, sw, bias, C, R, ldo, M, N, K, qscale, qcols, ws, ws_bytes,
                                  None)


def _refused(pb, rc, name, what):
    assert rc == pb.PB_EINVAL, what
    assert pb.lib().pb_last_error().decode().startswith(name), what


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(dtype=-1), dict(x=None), dict(x=A[0] + 1), dict(x=A[0] + 2, f32=1), dict(ld_x=63),
                                 dict(ld_x=1 << 41), dict(ld_x=1 << 39, rows=1 << 29), dict(ld_q=1 << 38, rows=1 << 30),
                                 dict(delta=A[1] + 1), dict(ld_delta=10), dict(delta=None), dict(sum=A[2] + 1),
                                 dict(ld_sum=-64), dict(g=None), dict(g=A[3] + 1), dict(b=A[4] + 1), dict(eps=-1e-5),
                                 dict(eps=float("nan")), dict(eps=float("inf")), dict(out=A[5] + 1), dict(ld_out=63),
                                 dict(out=None, q=None, scale=None), dict(q=None), dict(scale=None), dict(scale=A[7] + 2),
                                 dict(ld_q=63), dict(rows=-1), dict(rows=(1 << 30) + 1), dict(d=0), dict(d=16385, ld_x=1 << 15)], ids=str)
def test_norm_refusals(bad):
    from paper_2503_17707_amd import binding as pb

    _refused(pb, _norm(pb, **bad), "pb_op_norm_q8", bad)


@pytest.mark.parametrize("bad", [dict(sum=A[0], ld_sum=128), dict(sum=A[0] + 2), dict(sum=A[1]), dict(out=A[0]), dict(out=A[1] + 64),
                                 dict(out=A[2]), dict(q=A[2] + 10), dict(q=A[0] + 500), dict(scale=A[6] + 252),
                                 dict(scale=A[3] + 124), dict(out=A[4]), dict(q=A[5] - 200)], ids=str)
def test_norm_outputs_that_overlap(bad):
    from paper_2503_17707_amd import binding as pb

    _refused(pb, _norm(pb, **bad), "pb_op_norm_q8", bad)
    assert "overlap" in pb.lib().pb_last_error().decode()


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(x=None), dict(x=A[0] + 1), dict(x=A[0] + 2, f32=1), dict(ld_x=63), dict(q=None),
                                 dict(ld_q=1), dict(scale=None), dict(scale=A[2] + 1), dict(rows=-2), dict(cols=0),
                                 dict(cols=(1 << 24) + 1, ld_x=1 << 25, ld_q=1 << 25), dict(rows=(1 << 30) + 1), dict(q=A[0] + 100), dict(scale=A[0]),
                                 dict(ld_x=1 << 36, rows=1 << 30),
                                 dict(scale=A[1] + 4)], ids=str)
def test_quant_refusals(bad):
    from paper_2503_17707_amd import binding as pb

    _refused(pb, _quant(pb, **bad), "pb_op_quant_q8", bad)


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(epi=-1), dict(epi=4), dict(X=None), dict(X=A[0] + 8), dict(ldx=72), dict(ldx=48),
                                 dict(ldx=(1 << 23) + 16), dict(W=None), dict(W=A[2] + 4), dict(ldw=56), dict(ldw=40),
                                 dict(ldw=1 << 24), dict(sx=None), dict(sx=A[1] + 2), dict(sw=None), dict(sw=A[3] + 1),
                                 dict(bias=A[4] + 1), dict(C=None), dict(C=A[5] + 1), dict(epi=2, R=None),
                                 dict(epi=3, R=A[6] + 2), dict(ldo=31), dict(epi=2, ldo=8), dict(M=-1), dict(N=0), dict(K=0),
                                 dict(K=63), dict(K=72, ldx=80, ldw=80), dict(K=131072, ldx=131072, ldw=131072),
                                 dict(M=1 << 30, N=1 << 20, ldo=1 << 20), dict(M=1 << 24, ldo=1 << 39), dict(ws=A[7] + 4)], ids=str)
def test_gemm_refusals(bad):
    from paper_2503_17707_amd import binding as pb

    _refused(pb, _gemm(pb, **bad), "pb_op_gemm_q8", bad)


@pytest.mark.parametrize("bad", [dict(C=A[0]), dict(C=A[0] + 255), dict(C=A[2] + 32 * 64 - 2), dict(C=A[1] + 14), dict(C=A[3]),
                                 dict(C=A[4] + 62), dict(epi=2, R=A[0]), dict(ws=A[0]), dict(ws=A[5]), dict(ws=A[2] - 64),
                                 dict(epi=3, ws=A[6] + 16)], ids=lambda b: str({k: hex(v) for k, v in b.items()}))
def test_gemm_overlaps(bad):
    from paper_2503_17707_amd import binding as pb

    if "C" in bad and bad["C"] % 2:
        bad = dict(C=bad["C"] - 1)
    _refused(pb, _gemm(pb, **bad), "pb_op_gemm_q8", bad)
    assert "overlap" in pb.lib().pb_last_error().decode()


def test_nothing_to_do_is_no_error():
    from paper_2503_17707_amd import binding as pb

    assert _norm(pb, rows=0, x=None) == 0 and _quant(pb, rows=0, q=None) == 0 and _gemm(pb, M=0, X=None) == 0


def test_workspace_sizes():
    from paper_2503_17707_amd import binding as pb

    f = pb.lib().pb_op_gemm_q8_workspace
    for M, N, K in ((0, 64, 64), (4, 0, 64), (4, 64, 0), (4, 64, 40), (4, 64, 131072), (1 << 30, 1 << 30, 64), (-1, 64, 64)):
        assert f(M, N, K) == 0
    for M, N, K in ((1, 64, 8192), (24, 2048, 8192), (333, 5120, 20480), (4096, 36864, 9216)):
        n = f(M, N, K)
        assert n % 16 == 0 and n <= 64 * 4 * M * N + (64 << 20)


def test_wrappers_refuse_what_the_library_cannot_see():
    import torch

    from paper_2503_17707_amd import binding as pb

    def refused(f, *a, **kw):
        with pytest.raises(pb.PbError) as e:
            f(*a, **kw)
        assert e.value.code == pb.PB_EINVAL

    x, g = torch.zeros(3, 64), torch.zeros(64, dtype=torch.float16)
    q, s = torch.zeros(3, 64, dtype=torch.int8), torch.zeros(3)
    h = x.half()
    refused(pb.op_norm_q8, 1, x, g, q, s)  # on the host
    refused(pb.op_norm_q8, 1, x.double(), g, q, s)
    refused(pb.op_norm_q8, 0, h, g, q, s)
    refused(pb.op_norm_q8, 1, x, g.float(), q, s)
    refused(pb.op_norm_q8, 1, x[0], g, q, s)
    refused(pb.op_norm_q8, 1, x, g, q.to(torch.uint8), s)
    refused(pb.op_norm_q8, 1, x, g, q, s.half())
    refused(pb.op_norm_q8, 1, x, g, q, None)
    refused(pb.op_norm_q8, 1, x, g, q, s, delta=h, sum=h)
    refused(pb.op_quant_q8, 1, h, q, s)
    refused(pb.op_quant_q8, 0, h, q, s)
    refused(pb.op_quant_q8, 2, h, q, s)
    refused(pb.op_quant_q8, 1, h.to_sparse(), q, s)
    refused(pb.op_quant_q8, 1, h, q, s.to_sparse())
    for bad in (("f16", h, q, s), (None, h, q, s), (1.5, h, q, s)):
        with pytest.raises(TypeError):
            pb.op_quant_q8(*bad)
    with pytest.raises(TypeError):
        pb.op_norm_q8(1, h, g, q, s, eps="small")
    with pytest.raises(TypeError):
        pb.op_gemm_q8(1, 2, q, s, q, s, R=torch.zeros(3, 3), qcols=None)
    refused(pb.op_quant_q8, 1, h, q[:, :32], s)
    refused(pb.op_quant_q8, 1, h, q, s[:2])
    refused(pb.op_gemm_q8, 1, 0, q, s, q, s, C=torch.zeros(3, 3, dtype=torch.float16))
    refused(pb.op_gemm_q8, 1, 0, q, s, q, s, C=torch.zeros(3, 3))
    refused(pb.op_gemm_q8, 1, 2, q, s, q[:, :32], s, R=torch.zeros(3, 3))
    refused(pb.op_gemm_q8, 1, 2, q.t(), s, q, s, R=torch.zeros(3, 3))
    refused(pb.op_gemm_q8, 1, 2, q, s, q, s[:2], R=torch.zeros(3, 3))
    refused(pb.op_gemm_q8, 1, 2, q[0], s, q, s, R=torch.zeros(3, 3))
    assert ctypes.sizeof(ctypes.c_void_p) == 8
