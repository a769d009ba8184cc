"""Scales of 4-bit weights as the C ABI takes them: beginning at any element, of either sign; each form of the products' kernels."""
import ctypes

import numpy as np
import pytest

from test_gpu_w4 import Projection, activations, engine, wide_loss

pytestmark = pytest.mark.gpu
#: (type, rows, outputs, inputs): four rows at a time, ranges, tiles, many rows in tiles of 64 and of 128, float32 tiles
FORMS = [("bf16", 1, 70, 712), ("bf16", 3, 4099, 8200), ("bf16", 40, 8201, 712), ("bf16", 70, 12001, 424), ("bf16", 513, 8201, 264), ("f32", 1, 70, 712), ("f32", 20, 70, 712),
         ("f32", 300, 701, 424)]


@pytest.mark.parametrize("kind,M,N,K", FORMS)
@pytest.mark.parametrize("group", [32, 128])
def test_scales_at_any_element_and_of_either_sign(kind, M, N, K, group):
    import torch
    import paper_2410_03065_amd as cake
    eng = engine(kind)
    rng = np.random.default_rng([M, N, K])
    p = Projection(eng, N, K, group, scales=rng.choice([-1, 1], (N, -(-K // group))) * rng.uniform(0.01, 0.03, (N, -(-K // group))))
    t, a = activations(eng, M, K)
    whole = eng.op_gemm_w4(t, p.w4).clone()
    p.scales, signed = np.abs(p.scales), p.scales                # the bounds are of magnitudes
    off = np.abs(whole.double().cpu().numpy() - a @ p.values.T)
    assert (off <= p.bound(a, kind) + (wide_loss(p, a) if M > 64 else 0)).all()
    by_group = p.w4.scales.t()
    assert by_group.is_contiguous() and torch.equal(p.w4.scales.double().cpu(), torch.from_numpy(signed).double())
    for begin in (1, 3, 5):
        room = torch.zeros(by_group.numel() + 8, dtype=eng.tdtype, device="cuda")
        room[begin:begin + by_group.numel()] = by_group.reshape(-1)
        w = cake.W4.from_buffer_copy(p.w4)
        w.scales_at = room.data_ptr() + begin * room.element_size()
        out = torch.empty((M, N), device="cuda")
        torch.cuda.synchronize()
        assert eng.lib.cake_op_gemm_w4(eng.ctx, t.data_ptr(), ctypes.byref(w), out.data_ptr(), M) == cake.OK
        torch.cuda.synchronize()
        assert torch.equal(out, whole)
