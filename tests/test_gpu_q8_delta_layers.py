"""8-bit layers whose o and fc2 outputs go to the stream in the next norm (delta, RMS and layer norm, the sum in place), in 32- and
16-bit streams: every norm against float64, the whole pass recorded and replayed."""
import pytest

from gpu_common import log
from test_gpu_q8_layers import Decoder

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,f32,layer_norm", [("f16", True, False), ("bf16", True, True), ("bf16", False, False), ("f16", False, True)])
def test_layers_that_add_in_the_norm(kind, f32, layer_norm):
    import torch

    from q8_common import check_rows8, norm64

    B, T, d, H, F = 2, 45, 256, 4, 1040
    log("8-bit layers with deltas", kind, f32, layer_norm)
    m = Decoder(kind, B * T, 3, d, H, F, 64, seed=5)
    x = torch.zeros(B * T, d, device="cuda", dtype=torch.float32 if f32 else m.dt)
    delta = torch.zeros(B * T, d, device="cuda", dtype=m.dt)
    start = torch.randn(B * T, d, generator=torch.Generator().manual_seed(2)).cuda().to(x.dtype)

    def norm(gains, add, look):
        before = x.clone() if look else None
        gain, b = gains[0], gains[1] if layer_norm else None
        m.pb.op_norm_q8(m.code, x, gain, m.q8, m.s8, delta=delta if add else None, sum=x if add else None, b=b, layer=layer_norm)
        if look:
            want = (before.float() + delta.float()).to(x.dtype) if add else before
            assert torch.equal(x, want)
            c = lambda t: None if t is None else t.cpu()  # noqa: E731
            check_rows8(m.q8, m.s8, *norm64(x.cpu(), c(gain), c(b), layer_norm, 1e-5), (kind, f32, layer_norm))

    def product(q, w):  # bias, no scaled columns: the output as it is
        m.pb.op_gemm_q8(m.code, 0, q, m.s8, w["w"], w["s"], w["b"], C=delta, workspace=m.ws)

    def run(look=False):
        for l, w in enumerate(m.layers):
            norm(w["n1"], l > 0, look)
            m.product(0, m.q8, w["qkv"], C=m.qkv)
            m.pb.op_attention(m.code, m.qkv, m.att, B, T, H, m.hd)
            m.quant(m.att, m.q8)
            product(m.q8, w["o"])
            norm(w["n2"], True, look)
            m.product(1, m.q8, w["fc1"], C=m.hid)
            m.quant(m.hid, m.h8)
            product(m.h8, w["fc2"])
        norm(m.nf, True, look)

    def outputs():
        torch.cuda.synchronize()
        return [t.clone() for t in (x, m.q8, m.s8)]

    x.copy_(start)
    run(look=True)
    want = outputs()
    assert bool(torch.isfinite(want[2]).all()) and bool((want[2] > 0).all())
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
        run()
    for k in range(4):
        x.copy_(start)
        m.ws.fill_(k)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(outputs(), want)), k
        x.copy_(start * 0.5)  # eager work between the replays
        run()
        torch.cuda.synchronize()
