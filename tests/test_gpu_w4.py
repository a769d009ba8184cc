"""cake_op_pack_w4 and the cake_op_gemm_w4 products against the definition in 64 bits: sizes from one row and one output on, inputs that
end inside a step and inside a group, every group size, form and type; special values, memory beside the operands, streams, graphs, refusals."""
import ctypes

import numpy as np
import pytest

from oracle import serving
from q8_helpers import engine as small_engine

pytestmark = pytest.mark.gpu
_engines = {}


def engine(kind, **kw):
    if kw:
        return small_engine(4, 2, 64, kind, **kw)
    if kind not in _engines:
        _engines[kind] = small_engine(4, 2, 64, kind)
    return _engines[kind]


class Projection:
    """Random codes (from -8 to 7, where asked) and scales, in rows whose padding holds anything."""

    def __init__(self, eng, N, K, group, seed=0, scales=None):
        import torch
        rng = np.random.default_rng([N, K, group, seed])
        self.K, self.group = K, group
        codes = np.clip(np.rint(rng.standard_normal((N, (K + 31) // 32 * 32)) * 3), -8, 7)
        codes[:, K:] = rng.integers(-8, 8, codes[:, K:].shape)
        self.raw = serving.two_a_byte(codes)
        self.scales = serving.round_to(0.02 * np.exp(0.5 * rng.standard_normal((N, -(-K // group)))) if scales is None else scales, eng.shape.dtype)
        self.values = serving.w4_values(self.raw, self.scales, K, group)
        self.w4 = eng.w4(torch.from_numpy(self.raw).cuda(), torch.from_numpy(self.scales).cuda().to(eng.tdtype), K, group)

    def magnitudes(self, a):
        """(sum of |a| |w|, 32 times the sum of |a| times the scales) of each result."""
        n_groups = self.scales.shape[1]
        padded = np.zeros((len(a), n_groups * self.group))
        padded[:, :self.K] = np.abs(a)
        return np.abs(a) @ np.abs(self.values).T, 32 * padded.reshape(len(a), n_groups, -1).sum(axis=2) @ np.abs(self.scales.astype(np.float64)).T

    def bound(self, a, kind):
        """A product of 32 inputs adds at most 8 roundings to the sum it is added to (its products are exact and added up in fours at least);
        within a group sums stay below 32 times the activations' magnitudes (a code enters as 24 + c), over two products of 32 inputs for
        each (three times that for float32, whose activations are three terms and lose at most 2^-24); outside, one rounding
        a group and one for each of up to 16 parts."""
        total, inside = self.magnitudes(a)
        terms = 3 if kind == "f32" else 1
        return 2.0 ** -24 * (8 * 2 * (self.group // 32) * terms * inside + (self.scales.shape[1] + 16 + terms) * total) + 1e-37


def activations(eng, M, K, seed=0):
    import torch
    rng = np.random.default_rng([M, K, seed, 3])
    a = (rng.standard_normal((M, K)) * np.exp(0.5 * rng.standard_normal((1, K)))).astype(np.float32)
    t = torch.from_numpy(a).cuda().to(eng.tdtype)
    return t, t.double().cpu().numpy()


def check_plain(kind, M, N, K, group, seed=0):
    import torch
    eng = engine(kind)
    p = Projection(eng, N, K, group, seed)
    t, a = activations(eng, M, K, seed)
    room = torch.full((M + 2, N), 77.0, device="cuda")
    got = eng.op_gemm_w4(t, p.w4, out=room[1:M + 1])
    assert (room[0] == 77).all() and (room[M + 1] == 77).all()
    want, got = a @ p.values.T, got.double().cpu().numpy()
    off = np.abs(got - want)
    assert (off <= p.bound(a, kind)).all(), (off / p.bound(a, kind)).max()
    if M * N >= 64:
        # independent roundings: about 16 in a group (float32: 48), each of 2^-25 of a sum of 24 sqrt(group) activations, against codes that add up
        # to 3 sqrt(group): 8 sqrt(16) 2^-25 = 1e-6 (sqrt(3) times that) of what the result's terms add up to as squares; twice that for the rms of 64 or more
        size = np.sqrt(a ** 2 @ (p.values ** 2).T)
        assert np.sqrt((off ** 2).mean()) <= (2e-6 if kind == "bf16" else 3.5e-6) * np.sqrt((size ** 2).mean())
    return got


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 31, 33, 64, 65, 127, 130, 257])
def test_rows(kind, group, M):
    check_plain(kind, M, 70, 712, group)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("K", [8, 16, 24, 32, 40, 64, 88, 120, 128, 136, 160, 192, 256, 504, 520, 1016, 2048, 4104])
def test_inputs(kind, group, K):
    check_plain(kind, 3, 50, K, group)
    check_plain(kind, 40, 33, K, group)


@pytest.mark.parametrize("K", [8, 136, 1016, 1024])
@pytest.mark.parametrize("M", [130, 300])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_inputs_of_many_rows(group, M, K):
    check_plain("bf16", M, 300, K, group)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 2, 3, 15, 16, 17, 31, 33, 63, 65, 127, 129, 255, 257, 515, 1030])
def test_outputs(kind, N):
    check_plain(kind, 1, N, 384, 128)
    check_plain(kind, 20, N, 384, 64)
    check_plain(kind, 150, N, 384, 128)


@pytest.mark.parametrize("M,N,K,group", [(1, 14336, 4096, 128), (1, 4096, 14336, 128), (16, 6144, 4096, 64), (33, 4096, 14336, 64), (64, 4096, 4096, 32),
                                         (100, 12288, 4096, 128), (512, 4096, 4096, 128), (1024, 1280, 5120, 128), (1025, 700, 11008, 64)])
def test_projections_of_real_models(M, N, K, group):
    check_plain("bf16", M, N, K, group)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K,group", [(1, 688, 256, 128), (1, 17, 40, 32), (5, 100, 712, 64), (33, 258, 512, 128), (140, 300, 1024, 128), (300, 257, 264, 32)])
def test_residual_and_swiglu(kind, M, N, K, group):
    import torch
    eng = engine(kind)
    gate, up = Projection(eng, N, K, group, 1, None), Projection(eng, N, K, group, 2)
    t, a = activations(eng, M, K)
    x = torch.randn((M, N), device="cuda", generator=torch.Generator("cuda").manual_seed(M))
    before = x.double().cpu().numpy()
    got = eng.op_gemm_w4_residual(t, gate.w4, x)
    assert got is x
    want = before + a @ gate.values.T
    assert (np.abs(x.double().cpu().numpy() - want) <= gate.bound(a, kind) + 2.0 ** -24 * (np.abs(want) + np.abs(before))).all()
    out = eng.op_gemm_w4_swiglu(t, gate.w4, up.w4)
    assert out.dtype is eng.tdtype
    g, u = a @ gate.values.T, a @ up.values.T
    want, dg, du = serving.silu_product(g, u), gate.bound(a, kind), up.bound(a, kind)
    half = 2.0 ** -8 if kind == "bf16" else 2.0 ** -24
    # the slope of silu is at most 1.1; its exponential, sum and quotient, and the product: float32, a few units each
    bound = half * np.abs(want) + 1.1 * dg * (np.abs(u) + du) + np.abs(g) * du + 2.0 ** -20 * np.abs(want) * (1 + np.abs(g) / 16) + 1e-37
    off = np.abs(out.double().cpu().numpy() - want)
    assert (off <= bound).all(), (off / bound).max()


def test_every_code_and_its_place():
    """One input at a time: column k of the result is code (n, k) itself."""
    import torch
    for kind in ("bf16", "f32"):
        for group in (32, 64, 128):
            eng = engine(kind)
            K, N = 264, 48
            p = Projection(eng, N, K, group, scales=np.ones((N, -(-K // group)), np.float32))
            got = eng.op_gemm_w4(torch.eye(K, device="cuda").to(eng.tdtype), p.w4).cpu().numpy()
            np.testing.assert_array_equal(got, p.values.T.astype(np.float32))
            assert p.values.min() == -8 and p.values.max() == 7


@pytest.mark.parametrize("M", [1, 20, 200])
def test_activations_of_one_sign_and_large_outliers(M):
    """The offset of the codes must leave the result: sums of it are far larger than what remains."""
    import torch
    eng = engine("bf16")
    p = Projection(eng, 90, 2048, 128)
    a = np.abs(np.random.default_rng(M).standard_normal((M, 2048))).astype(np.float32) + 3
    a[:, 17] = 5000
    t = torch.from_numpy(a).cuda().to(torch.bfloat16)
    a = t.double().cpu().numpy()
    off = np.abs(eng.op_gemm_w4(t, p.w4).double().cpu().numpy() - a @ p.values.T)
    assert (off <= p.bound(a, "bf16")).all()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("M", [2, 40, 150])
def test_values_that_are_not_finite_stay_with_their_row_or_output(kind, M):
    import torch
    eng = engine(kind)
    p = Projection(eng, 70, 300 // 8 * 8, 64)
    t, a = activations(eng, M, p.K)
    clean = eng.op_gemm_w4(t, p.w4).clone()
    t[1, 5] = float("nan")
    got = eng.op_gemm_w4(t, p.w4)
    rest = torch.arange(M, device="cuda") != 1
    assert torch.isnan(got[1]).all() and torch.equal(got[rest], clean[rest])
    t[1, 5] = float("inf")
    got = eng.op_gemm_w4(t, p.w4)
    assert not torch.isfinite(got[1]).any() and torch.equal(got[rest], clean[rest])
    t[1, 5] = 0
    clean = eng.op_gemm_w4(t, p.w4).clone()
    p.w4.scales[33, 2] = float("nan")
    got = eng.op_gemm_w4(t, p.w4)
    others = torch.arange(70, device="cuda") != 33
    assert torch.isnan(got[:, 33]).all() and torch.equal(got[:, others], clean[:, others])
    p.w4.scales[33] = 0
    assert (eng.op_gemm_w4(t, p.w4)[:, 33] == 0).all()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("M", [1, 37, 129, 200])
def test_a_row_does_not_depend_on_those_beside_it_and_runs_repeat(kind, M):
    import torch
    eng = engine(kind)
    p = Projection(eng, 130, 1160, 128)
    t, _ = activations(eng, M, p.K)
    first = eng.op_gemm_w4(t, p.w4).clone()
    for _ in range(3):
        assert torch.equal(eng.op_gemm_w4(t, p.w4), first)
    t[:M // 2] = 9.0
    assert torch.equal(eng.op_gemm_w4(t, p.w4)[M // 2:], first[M // 2:])


# ---------------------------------------------------------------------------------------------- choices between kernels
def wide_loss(p, a):
    """What many rows may lose more (a scale and an activation each rounded to a multiple of 2^-24 in units that put the largest of its output
    at 2^10 or more, the largest of its row at 2^14 or more): codes are at most 8."""
    most_a, most_s = np.abs(a).max(axis=1, keepdims=True), p.scales.astype(np.float64).max(axis=1)
    return 2.0 ** -35 * 8 * np.abs(a).sum(axis=1, keepdims=True) * most_s + 2.0 ** -39 * most_a * np.abs(p.values).sum(axis=1)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", [(65, 12301, 264), (80, 10001, 1000), (129, 6208, 136), (128, 30000, 40), (300, 2667, 712), (513, 8200, 200), (512, 8192, 1024), (1030, 4100, 72), (65, 12308, 4104)])
def test_many_rows(group, M, N, K):
    """At least 800 000 results: weights in half precision; 64 and 128 rows a workgroup, one to four tiles wide, inputs in one range and in several."""
    check_plain("bf16", M, N, K, group)


@pytest.mark.parametrize("form", ["residual", "swiglu"])
@pytest.mark.parametrize("M,N,K,group", [(65, 6200, 264, 32), (70, 12309, 5000, 128), (128, 33000, 72, 64), (513, 9001, 200, 128), (520, 17000, 136, 64)])
def test_many_rows_residual_and_swiglu(form, M, N, K, group):
    import torch
    eng = engine("bf16")
    gate, up = Projection(eng, N, K, group, 1), Projection(eng, N, K, group, 2)
    t, a = activations(eng, M, K)
    if form == "residual":
        x = torch.randn((M, N), device="cuda", generator=torch.Generator("cuda").manual_seed(M))
        before = x.double().cpu().numpy()
        want = before + a @ gate.values.T
        got = eng.op_gemm_w4_residual(t, gate.w4, x).double().cpu().numpy()
        assert (np.abs(got - want) <= gate.bound(a, "bf16") + 2.0 ** -24 * (np.abs(want) + np.abs(before))).all()
        return
    g, u = a @ gate.values.T, a @ up.values.T
    want, dg, du = serving.silu_product(g, u), gate.bound(a, "bf16"), up.bound(a, "bf16")
    # as in test_residual_and_swiglu
    bound = 2.0 ** -8 * np.abs(want) + 1.1 * dg * (np.abs(u) + du) + np.abs(g) * du + 2.0 ** -20 * np.abs(want) * (1 + np.abs(g) / 16) + 1e-37
    assert (np.abs(eng.op_gemm_w4_swiglu(t, gate.w4, up.w4).double().cpu().numpy() - want) <= bound).all()


@pytest.mark.parametrize("M,N", [(3, 70), (40, 90), (70, 12000), (520, 9000)])
def test_scales_and_activations_of_very_different_size(M, N):
    """Scales over 2^40 within an output, outputs over 2^60, activations over 2^40 within a row, rows over 2^60; an output and a row of zeros."""
    import torch
    eng, K, group = engine("bf16"), 520, 64
    rng = np.random.default_rng([M, N])
    scales = 2.0 ** (rng.integers(-40, 1, (N, 9)) + rng.integers(-40, 21, (N, 1)))
    scales[N // 2] = 0
    p = Projection(eng, N, K, group, scales=scales.astype(np.float32))
    a = rng.standard_normal((M, K)) * 2.0 ** (rng.integers(-40, 1, (M, K)) + rng.integers(-20, 41, (M, 1)))
    a[M // 2] = 0
    t = torch.from_numpy(a.astype(np.float32)).cuda().to(torch.bfloat16)
    a = t.double().cpu().numpy()
    off = np.abs(eng.op_gemm_w4(t, p.w4).double().cpu().numpy() - a @ p.values.T)
    assert (off <= p.bound(a, "bf16") + (wide_loss(p, a) if M > 64 else 0)).all()


def test_many_rows_at_the_ends_of_the_range():
    """Activations of 2^100 against scales of 2^-90, of 2^-110 against 2^100, of 2^-120 against 2^-20: results in the middle and below the range."""
    import torch
    eng, M, N, K = engine("bf16"), 66, 12200, 136
    rng = np.random.default_rng(8)
    for big_a, big_s in ((100, -90), (-110, 100), (-120, -20), (-131, 100), (100, -131)):
        p = Projection(eng, N, K, 128, scales=(2.0 ** big_s * rng.uniform(1, 2, (N, 2))).astype(np.float32))
        t = torch.from_numpy((rng.standard_normal((M, K)) * 2.0 ** big_a).astype(np.float32)).cuda().to(torch.bfloat16)
        a = t.double().cpu().numpy()
        off = np.abs(eng.op_gemm_w4(t, p.w4).double().cpu().numpy() - a @ p.values.T)
        assert (off <= p.bound(a, "bf16") + wide_loss(p, a)).all(), (big_a, big_s)


@pytest.mark.parametrize("M,N", [(70, 12000), (520, 9000)])
def test_many_rows_values_that_are_not_finite(M, N):
    import torch
    eng = engine("bf16")
    p = Projection(eng, N, 296, 64)
    t, _ = activations(eng, M, 296)
    clean = eng.op_gemm_w4(t, p.w4).clone()
    t[1, 5], t[M - 1, 295] = float("nan"), float("inf")
    p.w4.scales[33, 2], p.w4.scales[N - 1, 0] = float("nan"), float("inf")
    got = eng.op_gemm_w4(t, p.w4)
    rows, outputs = torch.ones(M, dtype=torch.bool, device="cuda"), torch.ones(N, dtype=torch.bool, device="cuda")
    rows[[1, M - 1]], outputs[[33, N - 1]] = False, False
    assert not torch.isfinite(got[~rows]).any() and not torch.isfinite(got[:, ~outputs]).any()
    assert torch.equal(got[rows][:, outputs], clean[rows][:, outputs])


@pytest.mark.parametrize("M,N,K,group", [(2, 3000, 16392, 128), (1, 4112, 20000, 32), (40, 200, 9000, 64), (40, 8200, 4096, 128), (9, 10000, 2056, 32)])
def test_few_rows_of_long_inputs_and_many_outputs(M, N, K, group):
    """Activations in several parts through LDS; inputs in ranges; four, eight and sixteen waves."""
    check_plain("bf16", M, N, K, group)


def check_swiglu(eng, M, N, K, group):
    gate, up = Projection(eng, N, K, group, 1), Projection(eng, N, K, group, 2)
    t, a = activations(eng, M, K)
    g, u = a @ gate.values.T, a @ up.values.T
    want, dg, du = serving.silu_product(g, u), gate.bound(a, "bf16"), up.bound(a, "bf16")
    # as in test_residual_and_swiglu
    bound = 2.0 ** -8 * np.abs(want) + 1.1 * dg * (np.abs(u) + du) + np.abs(g) * du + 2.0 ** -20 * np.abs(want) * (1 + np.abs(g) / 16) + 1e-37
    assert (np.abs(eng.op_gemm_w4_swiglu(t, gate.w4, up.w4).double().cpu().numpy() - want) <= bound).all()


@pytest.mark.parametrize("M,N,K,group", [(1, 1000, 16400, 128), (2, 1000, 8200, 64), (4, 2048, 8192, 32), (3, 2049, 8192, 128), (1, 8200, 1032, 128), (16, 300, 9000, 32)])
def test_few_rows_gate_and_up(M, N, K, group):
    """Four, eight and sixteen waves, the last with all of a workgroup's LDS."""
    check_swiglu(engine("bf16"), M, N, K, group)


@pytest.mark.parametrize("form", ["plain", "swiglu"])
def test_many_rows_of_long_inputs(form):
    """More inputs than the pass before the product keeps in registers, and ranges of them."""
    eng = small_engine(32, 2, 64, "bf16")                      # a larger workspace
    if form == "swiglu":
        check_swiglu(eng, 300, 1400, 17000, 128)
        return
    p = Projection(eng, 2700, 17000, 64)
    t, a = activations(eng, 300, 17000)
    off = np.abs(eng.op_gemm_w4(t, p.w4).double().cpu().numpy() - a @ p.values.T)
    assert (off <= p.bound(a, "bf16")).all()


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", [(17, 10007, 136), (97, 1999, 264), (100, 2000, 520), (101, 2001, 8), (733, 300, 128), (257, 801, 1016), (32, 12345, 48), (64, 4096, 1032), (1024, 688, 256)])
def test_many_rows_in_float32(group, M, N, K):
    """Both sides of where tiles of 32 rows begin."""
    check_plain("f32", M, N, K, group)


@pytest.mark.parametrize("M,N,K,group", [(100, 1003, 264, 32), (257, 688, 256, 64), (130, 2049, 136, 128), (65, 1600, 1032, 32)])
def test_many_rows_in_float32_residual_and_swiglu(M, N, K, group):
    test_residual_and_swiglu("f32", M, N, K, group)


@pytest.mark.parametrize("M,N", [(70, 3001), (300, 700)])
def test_many_rows_in_float32_values_that_are_not_finite(M, N):
    import torch
    eng = engine("f32")
    p = Projection(eng, N, 296, 64)
    t, _ = activations(eng, M, 296)
    clean = eng.op_gemm_w4(t, p.w4).clone()
    t[1, 5], t[M - 1, 295] = float("nan"), float("inf")
    p.w4.scales[33, 2], p.w4.scales[N - 1, 0] = float("nan"), float("inf")
    got = eng.op_gemm_w4(t, p.w4)
    rows, outputs = torch.ones(M, dtype=torch.bool, device="cuda"), torch.ones(N, dtype=torch.bool, device="cuda")
    rows[[1, M - 1]], outputs[[33, N - 1]] = False, False
    assert not torch.isfinite(got[~rows]).any() and not torch.isfinite(got[:, ~outputs]).any()
    assert torch.equal(got[rows][:, outputs], clean[rows][:, outputs])


@pytest.mark.parametrize("N,K", [(1, 136), (5, 24)])
def test_a_description_keeps_its_scales(N, K):
    """One output, or one group: a layout in which the transposed scales are the scales themselves."""
    import torch
    eng = engine("bf16")
    codes = torch.full((N, (K + 31) // 32 * 16), 0x11, dtype=torch.uint8, device="cuda")
    scales = torch.ones((N, -(-K // 32)), dtype=torch.bfloat16, device="cuda")
    w, a = eng.w4(codes, scales, K, 32), torch.ones((2, K), dtype=torch.bfloat16, device="cuda")
    scales.zero_()
    assert (eng.op_gemm_w4(a, w) == K).all()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_the_most_rows(kind):
    import torch
    eng = engine(kind)
    M, N, K = 2 ** 20, 3, 8
    p = Projection(eng, N, K, 32)
    t = torch.randn((M, K), device="cuda").to(eng.tdtype)
    a = t.double().cpu().numpy()
    got = eng.op_gemm_w4(t, p.w4).double().cpu().numpy()
    assert (np.abs(got - a @ p.values.T) <= p.bound(a, kind)).all()
    out = eng.op_gemm_w4_swiglu(t, p.w4, p.w4).double().cpu().numpy()
    y = a @ p.values.T
    want = serving.silu_product(y, y)
    assert (np.abs(out - want) <= (2.0 ** -8 if kind == "bf16" else 2.0 ** -20) * (1 + np.abs(y)) * np.abs(want) + 4 * p.bound(a, kind) * (1 + np.abs(y))).all()


def test_a_small_workspace():
    """A context whose workspace holds neither the activations of many rows nor several parts of the result."""
    import torch
    eng = small_engine(4, 2, 64, "bf16")
    for M, N, K in ((70, 11500, 16400), (600, 2000, 4096), (64, 8200, 4096)):
        p = Projection(eng, N, K, 128)
        t, a = activations(eng, M, K)
        off = np.abs(eng.op_gemm_w4(t, p.w4).double().cpu().numpy() - a @ p.values.T)
        assert (off <= p.bound(a, "bf16")).all()


# ---------------------------------------------------------------------------------------------- packing
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("N,K,group", [(1, 8, 32), (3, 40, 32), (17, 128, 128), (5, 688, 32), (70, 712, 64), (130, 1000, 128), (1000, 256, 64), (257, 4096, 128)])
def test_packing(kind, N, K, group):
    import torch
    eng = engine(kind)
    rng = np.random.default_rng([N, K])
    w = rng.standard_normal((N, K)) * 0.02 * np.exp(rng.standard_normal((N, 1)))
    w[0, :min(K, group)] = 0
    t = torch.from_numpy(w.astype(np.float32)).cuda().to(eng.tdtype)
    packed, values = eng.pack_w4(t, group=group, want_values=True)
    raw, scales, want = serving.pack_w4(t.float().cpu().numpy(), group, kind)
    np.testing.assert_array_equal(packed.scales.float().cpu().numpy(), scales)
    np.testing.assert_array_equal(packed.codes.cpu().numpy(), raw)
    half = 2.0 ** -8 if kind == "bf16" else 2.0 ** -24
    assert (np.abs(values.double().cpu().numpy() - want) <= half * np.abs(want)).all()
    again = eng.pack_w4(t, group=group)
    assert torch.equal(again.codes, packed.codes) and torch.equal(again.scales, packed.scales)
    # what the codes stand for is within half a step (and the scale's own rounding) of the weights
    step = np.repeat(scales.astype(np.float64), group, axis=1)[:, :K]
    assert (np.abs(want - t.double().cpu().numpy()) <= step * (0.5 + 7 * half + 1e-6)).all()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_packing_quotients_between_two_codes_and_special_values(kind):
    """Weights at and beside the middle between two codes; groups of zeros, of the smallest numbers, with infinities and NaN."""
    import torch
    eng = engine(kind)
    rng = np.random.default_rng(5)
    w = np.zeros((40, 64), np.float32)
    for n in range(40):
        s = serving.round_to(np.float32(rng.uniform(0.001, 9)), kind)
        w[n] = serving.round_to((rng.integers(-6, 7, 64) + 0.5).astype(np.float32) * s, kind)
        w[n] = np.nextafter(w[n], rng.choice([-9, 0, 9], 64)).astype(np.float32) if kind == "f32" else w[n]
        w[n, 0], w[n, 32] = 7 * s, -7 * s
    w[1], w[2, :32], w[3, 40], w[4, 3], w[5, 63] = 0, 1e-44 if kind == "f32" else 1e-39, np.inf, np.nan, -np.inf
    t = torch.from_numpy(w).cuda().to(eng.tdtype)
    packed, values = eng.pack_w4(t, group=32, want_values=True)
    raw, scales, want = serving.pack_w4(t.float().cpu().numpy(), 32, kind)
    got_scales = packed.scales.float().cpu().numpy()
    np.testing.assert_array_equal(got_scales, scales)
    seen = ~np.isnan(np.repeat(scales, 32, axis=1))               # codes under a NaN scale mean nothing
    np.testing.assert_array_equal(np.where(seen, serving.one_each(packed.codes.cpu().numpy()), 0), np.where(seen, serving.one_each(raw), 0))
    np.testing.assert_array_equal(np.isnan(values.float().cpu().numpy()), ~seen)


def test_a_packed_projection_multiplies():
    import torch
    eng = engine("bf16")
    w = (torch.randn((200, 712), device="cuda") * 0.02).to(torch.bfloat16)
    packed, _ = eng.pack_w4(w, group=64, want_values=True)
    t, a = activations(eng, 9, 712)
    _, scales, values = serving.pack_w4(w.float().cpu().numpy(), 64, "bf16")
    got = eng.op_gemm_w4(t, packed).double().cpu().numpy()
    p = Projection(eng, 200, 712, 64)
    p.scales, p.values = scales, values
    assert (np.abs(got - a @ values.T) <= p.bound(a, "bf16")).all()


# ---------------------------------------------------------------------------------------------- streams, graphs, refusals
def test_on_another_stream():
    import torch
    eng = engine("bf16")
    p = Projection(eng, 300, 1024, 128)
    t, _ = activations(eng, 20, 1024)
    want = eng.op_gemm_w4(t, p.w4).clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        big = torch.zeros(1 << 26, device="cuda")
        for _ in range(10):
            big.add_(1)                      # keeps this stream busy: the operand below is late
        late = t + big[0].bfloat16() - 10
        got = eng.op_gemm_w4(late, p.w4) + 0
        packed = eng.pack_w4(late, group=32)
        codes = packed.codes + 0
    side.synchronize()
    assert torch.equal(got, eng.op_gemm_w4(late, p.w4)) and torch.equal(codes, eng.pack_w4(late, group=32).codes)
    own = engine("bf16", compute_stream=torch.cuda.current_stream())
    assert torch.equal(own.op_gemm_w4(t, Projection(own, 300, 1024, 128).w4), want)


@pytest.mark.parametrize("M", [1, 48, 200])
def test_graph_replays_beside_eager_calls(M):
    import torch
    eng = engine("bf16")
    gate, up, down = Projection(eng, 512, 1024, 128, 1), Projection(eng, 512, 1024, 128, 2), Projection(eng, 1024, 512, 64, 3)
    t, _ = activations(eng, M, 1024)
    x, y = torch.zeros((M, 1024), device="cuda"), torch.zeros((M, 1024), device="cuda")

    def step(x):
        return eng.op_gemm_w4_residual(eng.op_gemm_w4_swiglu(t, gate.w4, up.w4), down.w4, x)
    step(y.clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(x)
    x.zero_()
    for seed in range(4):
        t.copy_(activations(eng, M, 1024, seed)[0])
        graph.replay()
        torch.cuda.synchronize()
        step(y)
        assert torch.equal(x, y)


def test_two_graphs_of_one_context_in_turn():
    import torch
    eng, made = engine("bf16"), []
    for M, N, K in ((1, 256, 8192), (40, 300, 4096), (130, 140, 2048), (66, 12160, 520), (70, 12000, 392)):
        p = Projection(eng, N, K, 128)
        t, _ = activations(eng, M, K)
        out = eng.op_gemm_w4(t, p.w4)
        want = out.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            eng.op_gemm_w4(t, p.w4, out=out)
        made.append((graph, out, want, p, t))
    for _ in range(3):
        for graph, out, want, _, _ in made:
            out.zero_()
            graph.replay()
            assert torch.equal(out, want)


def test_refusals():
    import torch
    import paper_2410_03065_amd as cake
    eng = engine("bf16")
    p = Projection(eng, 48, 136, 64)
    t, _ = activations(eng, 4, 136)
    out, x = eng.op_gemm_w4(t, p.w4), torch.zeros((4, 48), device="cuda")

    def refused(f):
        with pytest.raises(cake.CakeError) as e:
            f()
        assert e.value.code == cake.E_INVAL
    for bad in (t.float(), t[:, :128].contiguous(), t[:, ::2], t.cpu(), t[0], t.t()):
        refused(lambda: eng.op_gemm_w4(bad, p.w4))
        refused(lambda: eng.op_gemm_w4_residual(bad, p.w4, x))
        refused(lambda: eng.op_gemm_w4_swiglu(bad, p.w4, p.w4))
    refused(lambda: eng.op_gemm_w4(t, p.w4, out=out.bfloat16()))
    refused(lambda: eng.op_gemm_w4(t, p.w4, out=out[:3]))
    refused(lambda: eng.op_gemm_w4_residual(t, p.w4, x.double()))
    refused(lambda: eng.op_gemm_w4_swiglu(t, p.w4, Projection(eng, 49, 136, 64).w4))
    refused(lambda: eng.op_gemm_w4_swiglu(t, p.w4, Projection(eng, 48, 136, 32).w4))
    refused(lambda: engine("f32").op_gemm_w4(t.float(), p.w4))
    codes, scales = p.w4.codes, p.w4.scales.contiguous()
    for args in ((codes[:, :64], scales, 136, 64), (codes, scales[:, :2], 136, 64), (codes, scales.float(), 136, 64), (codes, scales, 136, 48), (codes, scales, 130, 64),
                 (codes, scales, 0, 64), (codes.int(), scales, 136, 64), (codes.cpu(), scales, 136, 64), (codes[:0], scales[:0], 136, 64), (codes[0], scales, 136, 64)):
        refused(lambda: eng.w4(*args))
    for w, group in ((t.float(), 64), (t[:, :130], 64), (t, 16), (t[0], 64), (t[:0], 64), (t.cpu(), 64), (t[:, ::2], 64)):
        refused(lambda: eng.pack_w4(w, group=group))
    for field, value in (("n", 0), ("n", -1), ("n", 2 ** 31 - 1), ("k", 0), ("k", 12), ("k", 2 ** 31 - 8), ("group", 0), ("group", 256), ("codes_at", None),
                         ("codes_at", codes.data_ptr() + 8), ("scales_at", None), ("scales_at", scales.data_ptr() + 1)):
        bad = cake.W4.from_buffer_copy(p.w4)
        setattr(bad, field, value)
        assert eng.lib.cake_op_gemm_w4(eng.ctx, t.data_ptr(), ctypes.byref(bad), out.data_ptr(), 4) == cake.E_INVAL, field
        assert eng.lib.cake_op_gemm_w4_swiglu(eng.ctx, t.data_ptr(), ctypes.byref(p.w4), ctypes.byref(bad), out.data_ptr(), 4) == cake.E_INVAL, field
    good = ctypes.byref(p.w4)
    for args in ((None, good, out.data_ptr(), 4), (t.data_ptr(), None, out.data_ptr(), 4), (t.data_ptr(), good, None, 4), (t.data_ptr() + 2, good, out.data_ptr(), 4),
                 (t.data_ptr(), good, out.data_ptr() + 2, 4), (t.data_ptr(), good, out.data_ptr(), -1), (t.data_ptr(), good, out.data_ptr(), 2 ** 20 + 1)):
        assert eng.lib.cake_op_gemm_w4(eng.ctx, *args) == cake.E_INVAL
        assert eng.lib.cake_op_gemm_w4_residual(eng.ctx, *args) == cake.E_INVAL
    for args in ((None, codes.data_ptr(), scales.data_ptr(), None, 4, 136, 64), (t.data_ptr(), None, scales.data_ptr(), None, 4, 136, 64),
                 (t.data_ptr(), codes.data_ptr(), None, None, 4, 136, 64), (t.data_ptr(), codes.data_ptr(), scales.data_ptr(), t.data_ptr() + 8, 4, 136, 64),
                 (t.data_ptr(), codes.data_ptr(), scales.data_ptr(), None, 0, 136, 64), (t.data_ptr(), codes.data_ptr(), scales.data_ptr(), None, 4, 12, 64),
                 (t.data_ptr(), codes.data_ptr(), scales.data_ptr(), None, 4, 136, 16), (t.data_ptr() + 4, codes.data_ptr(), scales.data_ptr(), None, 4, 136, 64)):
        assert eng.lib.cake_op_pack_w4(eng.ctx, *args) == cake.E_INVAL


def test_no_rows():
    import torch
    eng = engine("bf16")
    p = Projection(eng, 48, 136, 64)
    none = torch.empty((0, 136), dtype=torch.bfloat16, device="cuda")
    assert eng.op_gemm_w4(none, p.w4).shape == (0, 48) and eng.op_gemm_w4_swiglu(none, p.w4, p.w4).shape == (0, 48)
