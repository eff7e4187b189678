"""8-bit norms and rows where numbers are none: NaN, infinities, overflow and zeros in rows, gains and biases, through every kernel
of pb_op_norm_q8 (few lanes a row, a wave, a block, blocks that walk over rows with the next one loaded ahead) and of
pb_op_quant_q8; good rows between bad ones are those of a call without any, bit for bit."""
import math

import pytest

from gpu_common import log

pytestmark = pytest.mark.gpu

# 16 bits: 1 element, 16 / 32 / 64 lanes a row, blocks of one piece, of two loaded ahead; fp32: up to 64 lanes with one and
# two pieces, blocks of two, of three loaded ahead (4100 .. 12288), of four
WIDTHS = [3, 70, 250, 500, 600, 4093, 4100, 5003, 6147, 9216, 12291, 16384]
ROWS = 1100  # a block of the kernels that load ahead takes 3 to 5 of them


def _inputs(d, f32, seed):
    import torch

    g = torch.Generator().manual_seed(seed)
    st = torch.float32 if f32 else torch.float16
    x = (torch.randn(ROWS, d, generator=g) * 2 + 0.5).to(st)
    delta = torch.randn(ROWS, d, generator=g).half()
    gain = (1 + 0.2 * torch.randn(d, generator=g)).half()
    b = (0.3 * torch.randn(d, generator=g)).half()
    return g, x, delta, gain, b


def _call(x, delta, gain, b, layer, want_q=True):
    import torch

    from paper_2503_17707_amd import binding as pb

    rows, d = x.shape
    q = torch.full((rows, d), 5, dtype=torch.int8, device="cuda") if want_q else None
    scale = torch.full((rows,), -1.0, device="cuda") if want_q else None
    out = torch.zeros(rows, d, dtype=torch.float16, device="cuda")
    total = torch.zeros_like(x, device="cuda")
    pb.op_norm_q8(1, x.cuda(), gain.cuda(), q, scale, delta=delta.cuda(), sum=total, b=None if b is None else b.cuda(), out=out,
                  layer=layer)
    return q, scale, out, total


def _same(a, b):
    """Equal bits, NaN where NaN is."""
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("layer", [False, True])
def test_bad_rows_between_good_ones(d, f32, bias, layer):
    import torch

    from q8_common import check_rows8, norm64

    g, x, delta, gain, b = _inputs(d, f32, d + layer)
    b = b if bias else None
    log("special rows", d, f32, bias, layer)
    clean = _call(x, delta, gain, b, layer)
    kinds = torch.where(torch.rand(ROWS, generator=g) < 0.3, torch.randint(1, 9, (ROWS,), generator=g), 0)
    kinds[:9] = torch.arange(9)
    at = torch.randint(0, d, (ROWS,), generator=g)
    at[::3] = d - 1  # in the last piece, cut short or moved back
    at[1::3] = 0
    x, delta = x.clone(), delta.clone()
    none = []  # rows that have no norm
    for r, kind in enumerate(kinds.tolist()):
        i = int(at[r])
        if kind in (1, 2, 3):
            x[r, i] = (math.nan, math.inf, -math.inf)[kind - 1]
        elif kind == 4:
            delta[r, i] = math.nan
        elif kind == 5:
            x[r, i], delta[r, i] = math.inf, -math.inf
        elif kind == 6:  # past the largest number of the stream, or of 16 bits
            x[r, i], delta[r, i] = (3.4e38 if f32 else 65504.0), 65504.0
        elif kind == 7:
            x[r], delta[r] = 0, 0
        elif kind == 8:
            x[r] *= 1e30 if f32 else 1e4
        if 1 <= kind <= 5 or (kind in (6, 8) and not bool(torch.isfinite((x[r].float() + delta[r].float()).to(x.dtype)).all())):
            none.append(r)
    q, scale, out, total = _call(x, delta, gain, b, layer)
    total64 = (x.float() + delta.float()).to(x.dtype)
    assert _same(total.cpu(), total64)
    assert bool(scale[none].isnan().all()) and not bool(q[none].any())
    assert not bool(scale[[r for r in range(ROWS) if r not in set(none)]].isnan().any())
    good = (kinds == 0).nonzero()[:, 0]
    for got, want in zip((q, scale, out, total), clean):
        assert torch.equal(got[good.cuda()], want[good.cuda()])
    # rows of zeros, huge ones and what is left of the largest: against float64
    odd = [r for r in range(ROWS) if kinds[r] >= 6 and r not in set(none)][:20]
    y, err = norm64(total64[odd], gain, b, layer, 1e-5)
    check_rows8(q[odd], scale[odd], y, err, (d, f32, bias, layer))
    zero = [r for r in range(ROWS) if kinds[r] == 7]
    if not bias:
        assert not bool(scale[zero].any()) and not bool(q[zero].any())
    # the norm in 16 bits of rows with an infinity or NaN: the formula's NaN and infinities
    some = none[:20]
    y = norm64(total64[some], gain, b, layer, 1e-5)[0]
    got = out[some].cpu()
    assert torch.equal(got.isnan(), y.isnan())
    # without 8 bits: the same norm
    assert _same(_call(x, delta, gain, b, layer, want_q=False)[2], out)


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("f32", [False, True])
def test_gains_and_biases_that_are_no_numbers(d, f32):
    """No row has 8 bits then, neither a block's first nor those that it walks to."""
    import torch

    _, x, delta, gain, b = _inputs(d, f32, 3 * d)
    log("special gains", d, f32)
    x, delta = x.cuda(), delta.cuda()
    x[::7] = 0  # (zero times infinity is none either)
    delta[::7] = 0
    for i in sorted({0, d // 2, d - 1}):
        for value in (math.nan, math.inf, -math.inf):
            for layer in (False, True):
                bad_gain, bad_b = gain.clone(), b.clone()
                bad_gain[i], bad_b[i] = value, value
                for of in ((bad_gain, None), (bad_gain, b), (gain, bad_b)):
                    q, scale, out, _ = _call(x, delta, *of, layer)
                    assert bool(scale.isnan().all()) and not bool(q.any()), (i, value, layer)
                    assert not bool(torch.isfinite(out[:, i]).any())


@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("cols", [3, 70, 250, 500, 1000, 2000, 5000, 7000, 13000, 30000, 50000, 70001])
def test_quantized_rows_between_bad_ones(kind, cols):
    import torch

    from paper_2503_17707_amd import binding as pb
    from q8_common import DT

    rows = 60
    g = torch.Generator().manual_seed(cols)
    x = torch.randn(rows, cols, generator=g).to(DT.get(kind, torch.float32))
    log("special quant", kind, cols)

    def call(x):
        q, s = torch.full((rows, cols), 5, dtype=torch.int8, device="cuda"), torch.full((rows,), -1.0, device="cuda")
        pb.op_quant_q8(0 if kind == "bf16" else 1, x.cuda(), q, s)
        return q, s

    clean = call(x)
    bad = torch.arange(0, rows, 3)
    at = torch.randint(0, cols, (rows,), generator=g)
    at[::2] = cols - 1
    for r in bad.tolist():
        x[r, at[r]] = (math.nan, math.inf, -math.inf)[r // 3 % 3]
    q, s = call(x)
    assert bool(s[bad.cuda()].isnan().all()) and not bool(q[bad.cuda()].any())
    good = torch.tensor([r for r in range(rows) if r % 3]).cuda()
    assert torch.equal(q[good], clean[0][good]) and torch.equal(s[good], clean[1][good])


def test_more_rows_than_a_launch_has_blocks():
    """Blocks walk on to a second row past 2^18 of them."""
    import torch

    from paper_2503_17707_amd import binding as pb

    rows, cut = (1 << 18) + 300, 1 << 18
    g = torch.Generator("cuda").manual_seed(1)
    for d in (520, 1100):
        x = torch.randn(rows, d, generator=g, device="cuda", dtype=torch.float16)
        x[1, 3] = math.inf
        x[cut + 2, d - 1] = math.nan
        gain, b = (torch.randn(d, generator=g, device="cuda", dtype=torch.float16) for _ in range(2))

        def calls(x):
            got = []
            for layer, bias in ((True, b), (False, None)):
                q, s = torch.full(x.shape, 5, dtype=torch.int8, device="cuda"), torch.full((len(x),), -1.0, device="cuda")
                pb.op_norm_q8(1, x, gain, q, s, b=bias, layer=layer)
                got += [q, s]
            q, s = torch.full(x.shape, 5, dtype=torch.int8, device="cuda"), torch.full((len(x),), -1.0, device="cuda")
            pb.op_quant_q8(1, x, q, s)
            return got + [q, s]

        log("rows past the blocks of a launch", d)
        whole, head, tail = calls(x), calls(x[:cut]), calls(x[cut:])
        for w, h, t in zip(whole, head, tail):
            assert _same(w[:cut], h) and _same(w[cut:], t)
        assert bool(whole[1][[1, cut + 2]].isnan().all()) and int(whole[1].isnan().sum()) == 2
