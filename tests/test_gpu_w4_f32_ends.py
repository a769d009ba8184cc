"""Products with 4-bit weights of float32 models at the ends of the range: infinities as in plain products, numbers that no bfloat16 reaches, the largest
activations whose groups are added up without loss, the smallest; each form of the kernels."""
import numpy as np
import pytest

from test_gpu_w4 import Projection, activations, engine

pytestmark = pytest.mark.gpu
#: rows and outputs of: a row alone, four at a time, tiles of 32
FORMS = [(1, 70), (2, 70), (40, 90), (70, 3001), (300, 700)]


@pytest.mark.parametrize("M,N", FORMS)
@pytest.mark.parametrize("value", [np.inf, -np.inf])
def test_an_infinity_is_one_of_its_code_s_sign(M, N, value):
    import torch
    eng = engine("f32")
    p = Projection(eng, N, 296, 64)
    t, _ = activations(eng, M, 296)
    clean = eng.op_gemm_w4(t, p.w4).clone()
    m = M - 1
    t[m, 133] = value
    got = eng.op_gemm_w4(t, p.w4)
    assert torch.equal(got[:m], clean[:m])
    with np.errstate(invalid="ignore"):
        np.testing.assert_array_equal(got[m].cpu().numpy(), (value * p.values[:, 133]).astype(np.float32))      # NaN where the code is 0
    t[m, 150] = -value                         # the same group: codes of equal sign cancel
    got, c, d = eng.op_gemm_w4(t, p.w4)[m].cpu().numpy(), p.values[:, 133], p.values[:, 150]
    np.testing.assert_array_equal(np.isnan(got), c * d >= 0)
    assert (got[c * d < 0] == np.float32(value) * np.sign(c[c * d < 0])).all()


@pytest.mark.parametrize("M,N", FORMS)
def test_a_finite_number_that_no_bfloat16_reaches(M, N):
    """The largest float32: 16 times a code of it is infinite, and nothing where the code is 0."""
    import torch
    eng = engine("f32")
    p = Projection(eng, N, 296, 64)
    t, _ = activations(eng, M, 296)
    m, most = M - 1, np.finfo(np.float32).max
    t[m, 133] = 0
    without = eng.op_gemm_w4(t, p.w4).clone()
    for value in (most, -most):
        t[m, 133] = float(value)
        got = eng.op_gemm_w4(t, p.w4)
        assert torch.equal(got[:m], without[:m])
        c, row = p.values[:, 133], got[m].cpu().numpy()
        np.testing.assert_array_equal(row[c != 0], np.inf * np.sign(value * c[c != 0]))
        np.testing.assert_array_equal(row[c == 0], without[m].cpu().numpy()[c == 0])


@pytest.mark.parametrize("M,N", FORMS)
@pytest.mark.parametrize("group", [32, 128])
def test_the_largest_and_the_smallest_activations(M, N, group):
    """Up to 2^113 a group of 128 inputs and codes of 8 stays finite: 128 * 16 * 8 * 2^113 = 2^127.  At 2^-100 the third term still has all of its bits (to 2^-124);
    at 2^-125 what lies below 2^-133 is gone: at most 2^-134 of each activation, times 8 times the scale."""
    import torch
    eng, K, rng = engine("f32"), 520, np.random.default_rng([M, N, group])
    for big, lost in ((112, 0.0), (-100, 0.0), (-125, 2.0 ** -134)):
        scales = (2.0 ** (-60 if big > 0 else 60) * rng.uniform(1, 2, (N, -(-K // group)))).astype(np.float32)
        p = Projection(eng, N, K, group, scales=scales)
        a = (rng.uniform(1, 2, (M, K)) * rng.choice([-1, 1], (M, K)) * 2.0 ** big).astype(np.float32)
        t = torch.from_numpy(a).cuda()
        a = a.astype(np.float64)
        off = np.abs(eng.op_gemm_w4(t, p.w4).double().cpu().numpy() - a @ p.values.T)
        assert (off <= p.bound(a, "f32") + lost * 8 * group * scales.astype(np.float64).sum(axis=1)).all(), big
