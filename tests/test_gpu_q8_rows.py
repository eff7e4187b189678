"""Norms and rows in 8 bits (pb_op_norm_q8, pb_op_quant_q8) against float64."""
import math

import pytest

from gpu_common import log

pytestmark = pytest.mark.gpu


def _out_tolerance(y, err, dt):
    """y is formed in 64 bits (both sides within err), rounded to fp32 (2^-24 of it, or half of fp32's smallest step)
    and from there to the type (half a step, or half its smallest one): at most err (1 + half) + (half + 2^-24 (1 + half))
    |y| + both halves of smallest steps."""
    from q8_common import HALF

    half, least = HALF[dt]
    return 2 * err + (half + 2.0 ** -24 * (1 + half)) * y.abs() + least + 2.0 ** -149


def _norm(kind, rows, d, f32, layer, delta, out, bias, seed=0, eps=1e-5, pad=(0, 0, 0, 0, 0), x=None, in_place=False):
    """One call on rows with `pad` more columns in x, delta, sum, out, q; every output checked."""
    import torch

    from paper_2503_17707_amd import binding as pb
    from q8_common import CODE, DT, check_rows8, norm64, strided, untouched

    g = torch.Generator().manual_seed(seed)
    dt = DT[kind]
    st = torch.float32 if f32 else dt
    x = (torch.randn(rows, d, generator=g) * 3 + 0.5).to(st) if x is None else x.to(st)
    dl = torch.randn(rows, d, generator=g).to(dt) if delta else None
    gain = (1 + 0.2 * torch.randn(d, generator=g)).to(dt)
    b = (0.3 * torch.randn(d, generator=g)).to(dt) if bias else None
    xv, xb = strided(x.cuda(), d + pad[0], pad[0] // 2)
    dv = strided(dl.cuda(), d + pad[1], pad[1] // 2)[0] if delta else None
    blank = lambda t, k: strided(torch.zeros(rows, d, dtype=t, device="cuda"), d + pad[k], pad[k] // 2)  # noqa: E731
    sv, sb = (xv, xb) if in_place else blank(st, 2) if delta else (None, None)
    ov, ob = blank(dt, 3) if out else (None, None)
    qv, qb = blank(torch.int8, 4)
    scale = torch.full((rows,), -1.0, device="cuda")
    log("norm", kind, rows, d, f32, layer, delta, out, bias, pad)
    pb.op_norm_q8(CODE[kind], xv, gain.cuda(), qv, scale, delta=dv, sum=sv, b=None if b is None else b.cuda(), out=ov,
                  layer=layer, eps=eps)
    torch.cuda.synchronize()
    s = (x.float() + dl.float()).to(st) if delta else x
    if delta:
        assert torch.equal(sv.cpu(), s) and untouched(sb, d, pad[0 if in_place else 2] // 2)
    if not in_place:
        assert torch.equal(xv.cpu(), x)
    y, err = norm64(s, gain, b, layer, eps)
    check_rows8(qv, scale, y, err, (kind, rows, d))
    assert untouched(qb, d, pad[4] // 2)
    if out:  # formed in fp32, then rounded to the type
        assert bool(((ov.cpu().double() - y).abs() <= _out_tolerance(y, err, dt)).all())
        assert untouched(ob, d, pad[3] // 2)
    return qv.clone(), scale


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 2), (5, 7), (2, 48), (9, 64), (7, 255), (4, 256), (6, 513), (5, 1000), (3, 1025),
                                    (2, 2048), (5, 2049), (3, 4091), (2, 4096), (2, 5120), (3, 8191), (2, 9216), (2, 12289),
                                    (1, 16384), (2, 16383)])
def test_norm(kind, f32, rows, d):
    _norm(kind, rows, d, f32, layer=False, delta=True, out=False, bias=False, seed=d)
    if d > 1:
        _norm(kind, rows, d, f32, layer=True, delta=True, out=True, bias=True, seed=d + 1)
    _norm(kind, rows, d, f32, layer=False, delta=False, out=True, bias=True, seed=d + 2)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("pad", [(16, 16, 16, 16, 16), (1, 3, 5, 7, 9), (2, 4, 6, 2, 3), (8, 1, 8, 1, 8)], ids=str)
def test_norm_of_strided_rows(f32, pad):
    for d in (40, 777, 2052):
        _norm("f16", 6, d, f32, layer=True, delta=True, out=True, bias=True, pad=pad, seed=sum(pad))


def test_norm_in_place_and_more_rows_than_blocks():
    q0, s0 = _norm("bf16", 70, 300, True, False, True, False, False, seed=5)
    q1, s1 = _norm("bf16", 70, 300, True, False, True, False, False, seed=5, in_place=True)
    assert bool((q0 == q1).all()) and bool((s0 == s1).all())
    q2, s2 = _norm("bf16", 70, 300, True, False, True, False, False, seed=5, in_place=True, pad=(4, 0, 0, 0, 4))
    assert bool((q0 == q2).all()) and bool((s0 == s2).all())
    _norm("f16", 3000, 33, False, True, True, True, True, seed=6)
    # rows that blocks walk over, the next one loaded ahead
    for rows, d, f32, bias in ((600, 9000, True, True), (513, 9000, True, False), (530, 9216, False, True), (257, 16384, False, False)):
        for layer in (False, True):
            q0, s0 = _norm("f16", rows, d, f32, layer, True, False, bias, seed=rows)
        q1, s1 = _norm("f16", rows, d, f32, layer, True, True, bias, seed=rows, in_place=True)
        assert bool((q0 == q1).all()) and bool((s0 == s1).all())
        _norm("bf16", rows, d, f32, layer, False, False, bias, seed=rows, pad=(8, 0, 0, 0, 1))


def test_norm_without_quantization_and_with_large_offsets():
    import torch

    from paper_2503_17707_amd import binding as pb
    from q8_common import norm64

    g = torch.Generator().manual_seed(3)
    x = torch.randn(4, 500, generator=g) * 1e-3 + 1e4  # a mean far above the spread
    gain = torch.ones(500, dtype=torch.float16)
    out = torch.zeros(4, 500, dtype=torch.float16, device="cuda")
    pb.op_norm_q8(1, x.cuda(), gain.cuda(), out=out, layer=True)
    y, err = norm64(x, gain, None, True, 1e-5)
    assert bool(((out.cpu().double() - y).abs() <= _out_tolerance(y, err, torch.float16)).all())


@pytest.mark.parametrize("d", [3, 70, 777, 2048, 5003, 9216])
def test_layer_norm_of_rows_of_one_value(d):
    """Their mean is the value: sums of d equal fp32 values are exact in 64 bits (24 + 14 bits), the division rounds to it."""
    import torch

    from paper_2503_17707_amd import binding as pb

    values = torch.tensor([2.5, -0.1, 1e-3, 65000.0, 1 / 3, 1e30, -7e-20])
    for st in (torch.float32, torch.bfloat16):
        x = values[:, None].expand(-1, d).to(st).cuda().contiguous()
        gain = torch.ones(d, dtype=torch.bfloat16, device="cuda")
        q, scale = torch.full((7, d), 5, dtype=torch.int8, device="cuda"), torch.ones(7, device="cuda")
        out = torch.ones(7, d, dtype=torch.bfloat16, device="cuda")
        for b in (None, torch.zeros_like(gain)):
            pb.op_norm_q8(0, x, gain, q, scale, b=b, out=out, layer=True)
            assert bool((scale == 0).all()) and bool((q == 0).all()) and bool((out == 0).all())


@pytest.mark.parametrize("f32", [False, True])
def test_norm_of_special_rows(f32):
    """Zeros, one value, huge and tiny rows, NaN and infinity: each row by itself."""
    import torch

    from paper_2503_17707_amd import binding as pb

    d = 70
    g = torch.Generator().manual_seed(1)
    x = torch.randn(9, d, generator=g)
    x[0] = 0
    x[1] = 0
    x[1, 69] = 3.0
    x[2, 5] = math.nan
    x[3, 69] = math.inf
    x[4, 0] = -math.inf
    x[5] *= 1e30 if f32 else 1e38
    x[6] *= 1e-38
    x[7] = 2.5
    st = torch.float32 if f32 else torch.bfloat16
    gain = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    q, scale = torch.full((9, d), 5, dtype=torch.int8, device="cuda"), torch.zeros(9, device="cuda")
    out = torch.zeros(9, d, dtype=torch.bfloat16, device="cuda")
    x = x.to(st)
    for layer in (False, True):
        pb.op_norm_q8(0, x.cuda(), gain, q, scale, out=out, layer=layer, eps=0.0 if not layer else 1e-5)
        s, qq = scale.cpu(), q.cpu()
        bad = [2, 3, 4] + ([] if layer else [0])  # RMS without eps: a row of zeros has no norm
        for r in range(9):
            if r in bad:
                assert math.isnan(s[r]) and bool((qq[r] == 0).all())
            elif (layer and r in (0, 7)):
                assert s[r] == 0 and bool((qq[r] == 0).all())
            else:
                assert s[r] > 0 and int(qq[r].abs().max()) == 127, r
        if not layer:
            assert int(qq[1, 69]) == 127 and int(qq[1].abs().sum()) == 127
            assert bool((qq[7] == 127).all())
            assert bool(torch.isfinite(out[5].float()).all())  # squares of 1e38 do not pass 64 bits


def test_a_gain_that_is_no_number():
    import torch

    from paper_2503_17707_amd import binding as pb

    x = torch.randn(3, 100).cuda()
    for bad in (math.nan, math.inf):
        g = torch.ones(100, dtype=torch.float16, device="cuda")
        g[99] = bad
        x[1, 99] = 0.0
        q, scale = torch.ones(3, 100, dtype=torch.int8, device="cuda"), torch.zeros(3, device="cuda")
        pb.op_norm_q8(1, x, g, q, scale)
        assert bool(torch.isnan(scale).all()) and bool((q == 0).all())


def _quant(kind, x, pad=(0, 0)):
    import torch

    from paper_2503_17707_amd import binding as pb
    from q8_common import CODE, check_rows8, strided, untouched

    rows, cols = x.shape
    xv = strided(x.cuda(), cols + pad[0], pad[0] // 2)[0]
    qv, qb = strided(torch.zeros(rows, cols, dtype=torch.int8, device="cuda"), cols + pad[1], pad[1] // 2)
    scale = torch.full((rows,), -1.0, device="cuda")
    log("quant", kind, x.dtype, rows, cols, pad)
    pb.op_quant_q8(CODE[kind], xv, qv, scale)
    torch.cuda.synchronize()
    y = x.double()
    check_rows8(qv, scale, y, torch.zeros_like(y), (kind, rows, cols))
    assert untouched(qb, cols, pad[1] // 2)
    return qv.cpu(), scale.cpu()


@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 3), (4, 64), (3, 257), (9, 500), (2, 1025), (3, 2048), (2, 4100), (2, 8192),
                                       (3, 16383), (2, 20480), (1, 36864), (2, 40001), (1, 65535), (2, 65544), (1, 70001),
                                       (1, 200000)])
def test_quant(kind, rows, cols):
    import torch

    from q8_common import DT

    g = torch.Generator().manual_seed(cols)
    x = torch.randn(rows, cols, generator=g).to(DT.get(kind, torch.float32))
    _quant("f16" if kind == "f32" else kind, x)
    _quant("f16" if kind == "f32" else kind, x[:, :min(cols, 3001)], pad=(3, 5))


@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
def test_quant_ties_go_to_even(kind):
    import torch

    from q8_common import DT

    for unit in (1.0, 3.0, 5.0, 0.375):  # scales of one and of several bits: (k + 1/2) unit is a number of the type
        k = torch.arange(-15, 16) + 0.5
        row = torch.cat([k * unit, torch.tensor([127.0 * unit])])[None]
        x = row.to(DT.get(kind, torch.float32))
        if not torch.equal(x.double(), row.double()):
            continue  # 127 units or a tie are no number of this type
        q, scale = _quant("bf16" if kind == "bf16" else "f16", x)
        assert float(scale[0]) == unit
        assert torch.equal(q[0, :31].double(), k.double().round())


def test_quant_of_special_rows():
    import torch

    from paper_2503_17707_amd import binding as pb

    x = torch.randn(8, 333)
    x[0] = 0
    x[1, 332] = math.nan
    x[2, 0] = math.inf
    x[3] *= 1e38 / x[3].abs().max() * 3
    x[4] = 0
    x[4, 7] = 127 * 2.0 ** -127  # its scale would be subnormal
    x[5] = 0
    x[5, 7] = -127 * 2.0 ** -126
    x[6] = -1e-45
    x[7] = -3.0
    q, scale = torch.ones(8, 333, dtype=torch.int8, device="cuda"), torch.zeros(8, device="cuda")
    pb.op_quant_q8(1, x.cuda(), q, scale)
    s, q = scale.cpu(), q.cpu()
    assert s[0] == 0 and bool((q[0] == 0).all())
    for r in (1, 2):
        assert math.isnan(s[r]) and bool((q[r] == 0).all())
    assert math.isfinite(s[3]) and int(q[3].abs().max()) == 127
    assert s[4] == 0 and bool((q[4] == 0).all())
    assert s[5] == 2.0 ** -126 and int(q[5, 7]) == -127 and int(q[5].abs().sum()) == 127
    assert s[6] == 0 and bool((q[6] == 0).all())
    assert bool((q[7] == -127).all())


def test_rows_past_four_gigabytes():
    """The last rows of a matrix of more than 2^32 bytes."""
    import torch

    from paper_2503_17707_amd import binding as pb
    from q8_common import check_rows8

    rows, cols = 36000, 65536  # 4.7 GB in, 2.4 GB out
    x = torch.zeros(rows, cols, dtype=torch.float16, device="cuda")
    x[-3:] = torch.randn(3, cols, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).half()
    q, scale = torch.ones(rows, cols, dtype=torch.int8, device="cuda"), torch.ones(rows, device="cuda")
    pb.op_quant_q8(1, x, q, scale)
    y = x[-3:].double().cpu()
    check_rows8(q[-3:], scale[-3:], y, torch.zeros_like(y))
    assert bool((scale[:-3] == 0).all()) and not bool(q[:-3].any())


def test_another_stream():
    import torch

    from paper_2503_17707_amd import binding as pb
    from q8_common import check_rows8

    s = torch.cuda.Stream()
    x = torch.randn(50, 3000).half()
    xd = torch.empty(50, 3000, dtype=torch.float16, device="cuda")
    q, scale = torch.zeros(50, 3000, dtype=torch.int8, device="cuda"), torch.zeros(50, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        xd.copy_(x)
        pb.op_quant_q8(1, xd, q, scale)  # the current stream
    pb.op_quant_q8(1, xd, q, scale, stream=s)  # a stream that is given
    s.synchronize()
    check_rows8(q, scale, x.double(), torch.zeros(50, 3000, dtype=torch.float64))
