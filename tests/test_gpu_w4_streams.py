"""A description of 4-bit weights made under one stream of torch's and used under another, whose caller orders nothing but the tensors of its own."""
import pytest

from test_gpu_w4 import Projection, activations, engine

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 300])
def test_described_under_a_late_stream(kind, N):
    import torch
    eng = engine(kind)
    p = Projection(eng, N, 1024, 128)
    t, _ = activations(eng, 5, 1024)
    scales = p.w4.scales.contiguous()
    want = eng.op_gemm_w4(t, p.w4).clone()
    big = torch.zeros(1 << 26, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(20):
            big.add_(1)                      # keeps this stream busy
        late = eng.w4(p.w4.codes, scales, 1024)
    got = eng.op_gemm_w4(t, late)
    assert torch.equal(got, want)
    torch.cuda.synchronize()
    assert torch.equal(late.scales, scales)


def test_described_under_the_compute_stream_and_in_a_captured_step():
    import torch
    eng = engine("bf16")
    p = Projection(eng, 300, 1024, 128)
    t, _ = activations(eng, 5, 1024)
    scales = p.w4.scales.contiguous()
    want = eng.op_gemm_w4(t, p.w4).clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(eng.compute_stream):
        got = eng.op_gemm_w4(t, eng.w4(p.w4.codes, scales, 1024))
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        inside = eng.w4(p.w4.codes, scales, 1024)
        eng.op_gemm_w4(t, inside, out=out)
    for factor in (1, 2, 4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eng.op_gemm_w4(t, eng.w4(p.w4.codes, scales, 1024))) and torch.equal(out, want * factor)
        scales.mul_(2)
