"""Products with 4-bit weights, many rows: every number of steps of 128 inputs that the last turn of the kernel's loop can hold, in tiles of 64 and of
128 rows, undivided and in ranges, all forms; the same bits again, and whatever the other rows hold."""
import numpy as np
import pytest

from q8_helpers import engine as small_engine
from test_gpu_w4 import Projection, activations, check_plain, check_swiglu, engine

pytestmark = pytest.mark.gpu
ROWS = [(70, 12000), (513, 8200)]                  # tiles of 64 rows (four steps a turn), of 128 (two)


@pytest.mark.parametrize("M,N", ROWS)
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11])
def test_steps(M, N, steps):
    check_plain("bf16", M, N, 128 * steps, 128, steps)
    check_plain("bf16", M, N, 128 * steps - 40, 64, steps)


@pytest.mark.parametrize("M,N", [(70, 6100), (513, 9001)])
@pytest.mark.parametrize("steps", [1, 2, 3, 5, 6, 7, 11])
def test_steps_gate_and_up(M, N, steps):
    check_swiglu(engine("bf16"), M, N, 128 * steps - 8, 32)


@pytest.mark.parametrize("steps", [49, 51, 53, 55, 57, 59])
@pytest.mark.parametrize("form", ["plain", "swiglu"])
def test_steps_of_ranges(form, steps):
    """Two ranges of 24 to 30 steps."""
    eng = small_engine(32, 2, 64, "bf16")          # a larger workspace
    if form == "swiglu":
        check_swiglu(eng, 300, 1400, 128 * steps, 128)
        return
    p = Projection(eng, 2700, 128 * steps, 128, steps)
    t, a = activations(eng, 300, 128 * steps, steps)
    off = np.abs(eng.op_gemm_w4(t, p.w4).double().cpu().numpy() - a @ p.values.T)
    assert (off <= p.bound(a, "bf16")).all()


@pytest.mark.parametrize("form", ["plain", "residual", "swiglu"])
@pytest.mark.parametrize("M,N", ROWS)
@pytest.mark.parametrize("steps", [1, 2, 3, 5, 6, 7, 11])
def test_the_same_bits_again_and_beside_other_rows(form, M, N, steps):
    import torch
    eng = engine("bf16")
    p, up = Projection(eng, N, 128 * steps, 128, 1), Projection(eng, N, 128 * steps, 128, 2)
    t, _ = activations(eng, M, 128 * steps, steps)

    def run():
        if form == "residual":
            return eng.op_gemm_w4_residual(t, p.w4, torch.ones((M, N), device="cuda"))
        return eng.op_gemm_w4(t, p.w4) if form == "plain" else eng.op_gemm_w4_swiglu(t, p.w4, up.w4)
    first = run()
    for _ in range(5):
        assert torch.equal(run(), first)
    t[:M // 2] = -3.0
    assert torch.equal(run()[M // 2:], first[M // 2:])


@pytest.mark.parametrize("kind,M", [("bf16", 262140), ("bf16", 262141), ("f32", 199996), ("f32", 199997)])
def test_the_most_rows_four_at_a_time(kind, M):
    """One output: the last number of rows that goes four at a time (65535 fours of bf16 models, as many as a grid takes), and the next."""
    check_plain(kind, M, 1, 8, 32)
