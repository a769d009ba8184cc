"""cake_op_sample against the definition in 64 bits: every filter alone and together, ties, masked and infinite logits, flat and
peaked rows, single rows and many, settings out of range, graphs."""
import numpy as np
import pytest

from oracle import serving
from q8_helpers import engine

pytestmark = pytest.mark.gpu
_engine = []


def eng():
    if not _engine:
        _engine.append(engine(4, 4, 64, "bf16"))
    return _engine[0]


def check(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, device_logits=None):
    import torch
    logits = np.asarray(logits, np.float32)
    rows = len(logits)
    f = lambda a, t: None if a is None else torch.from_numpy(np.broadcast_to(np.asarray(a, t), (rows,)).copy()).cuda()  # noqa: E731
    given = [f(temperature, np.float32), f(top_k, np.int32), f(top_p, np.float32), f(min_p, np.float32)]
    d = torch.from_numpy(logits).cuda() if device_logits is None else device_logits
    tokens, logprobs = eng().op_sample(d, f(u, np.float32), *given)
    host = [None if a is None else a.cpu().numpy() for a in given]
    want, want_lp = serving.sample(logits, np.broadcast_to(np.asarray(u, np.float32), (rows,)), *host)
    np.testing.assert_array_equal(tokens.cpu().numpy(), want)
    lp = logprobs.double().cpu().numpy()
    fine = np.isfinite(want_lp)
    np.testing.assert_array_equal(lp[~fine], want_lp[~fine])
    # one rounding to float32 of a number computed in 64 bits; weights are whole multiples of 2^-44, so a sum of n is off by n 2^-45
    assert (np.abs(lp[fine] - want_lp[fine]) <= 2.0 ** -24 * np.abs(want_lp[fine]) + 1e-7).all()
    return want


def rows_of(rows, vocab, seed=0, spread=2.2):
    rng = np.random.default_rng([seed, rows, vocab])
    x = rng.standard_normal((rows, vocab)) * spread
    for r in range(rows):
        x[r, rng.integers(0, vocab, 12)] += rng.uniform(2, 10, 12)
    return x.astype(np.float32), rng.random(rows).astype(np.float32) * np.float32(1 - 2.0 ** -24), rng


@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (5, 63), (4, 64), (7, 1000), (1, 2049), (300, 517), (2, 32000), (5, 50001), (3, 128256), (1, 524288)])
def test_each_filter(rows, vocab):
    x, u, rng = rows_of(rows, vocab)
    check(x, u)
    check(x, u, temperature=rng.uniform(0.3, 2, rows))
    check(x, u, top_k=rng.integers(1, 60, rows))
    check(x, u, top_p=rng.uniform(0.1, 0.99, rows))
    check(x, u, min_p=rng.uniform(0.001, 0.5, rows))
    check(x, u, 0.8, rng.integers(1, 300, rows), rng.uniform(0.5, 0.99, rows), rng.uniform(0.001, 0.1, rows))


def test_many_random_numbers_on_one_row():
    """The chosen tokens over a grid of u: every border between two tokens is met from both sides."""
    x, _, _ = rows_of(1, 300, seed=3)
    x = np.repeat(x, 4096, axis=0)
    u = (np.arange(4096) + 0.5) / 4096
    for settings, least in (((0.9, 40, 0.9), 2), ((3.0, 100, 0.95), 50), ((2.0,), 100)):
        got = check(x, u, *settings)
        assert len(set(got)) >= least and (np.diff(got) >= 0).all()


@pytest.mark.parametrize("spread", [0.0, 1e-6, 0.05, 1.0])
@pytest.mark.parametrize("vocab", [900, 9000, 70001])
def test_flat_rows_whose_last_bin_is_long(spread, vocab):
    rng = np.random.default_rng([vocab, int(spread * 1e6)])
    x = (rng.standard_normal((3, vocab)) * spread).astype(np.float32)
    u = rng.random(3)
    check(x, u, top_p=[0.3, 0.5, 0.9])
    check(x, u, top_k=[1, vocab // 2, vocab - 1])
    check(x, u, top_k=[vocab // 3, 600, vocab], top_p=[0.7, 0.11, 0.4])
    check(x, u, top_k=[vocab // 3, 600, vocab], top_p=[0.999, 0.01, 0.4], min_p=0.9)


@pytest.mark.parametrize("vocab", [40000])
def test_long_front_with_the_two_filters_in_different_bins(vocab):
    x, u, _ = rows_of(4, vocab, spread=1.0)
    check(x, u, top_k=[20000, 9000, 30000, 5000], top_p=[0.5, 0.99, 0.2, 0.9])


def test_ties_go_by_id():
    x = np.zeros((4, 3000), np.float32)
    x[:, 1500:] = -0.0                            # the same number
    x[1, 7] = x[1, 2900] = 3
    for u in (0.0, 0.3, 0.999):
        check(x, u, top_k=[1, 2, 5, 2000])
        check(x, u, top_p=[0.0005, 0.01, 0.5, 0.75])
        check(x, u, temperature=0.0)
    x[2, :10] = np.nextafter(np.float32(0), np.float32(1))
    check(x, 0.5, top_k=[3, 3, 3, 3])


def test_masked_rows():
    low = np.finfo(np.float32).min
    x, u, _ = rows_of(9, 5000)
    x[0] = -np.inf
    x[1] = np.nan
    x[2, 100:] = -np.inf
    x[3, 1:] = low
    x[4] = low
    x[5, :4000] = np.nan
    x[6, 17] = np.inf
    x[7, [5, 4000]] = np.inf
    x[8] = -np.inf
    x[8, 4999] = -3e38
    for more in ({}, dict(top_k=20), dict(top_p=0.7), dict(min_p=0.01), dict(top_k=30, top_p=0.8, min_p=0.02), dict(temperature=0.0),
                 dict(temperature=1e-30), dict(temperature=1e30, top_p=0.9)):
        check(x, u, **more)


def test_settings_out_of_range():
    x, u, _ = rows_of(6, 2000)
    nan, inf = float("nan"), float("inf")
    check(x, u, temperature=[nan, -1.0, 0.0, inf, 1e-38, 3e38])
    check(x, u, top_k=[-5, 0, 2000, 2 ** 31 - 1, -2 ** 31, 1])
    check(x, u, top_p=[nan, 1.5, 0.0, -1.0, inf, 1e-30])
    check(x, u, min_p=[nan, 1.5, 0.0, -1.0, inf, 1.0])
    check(x, [nan, 0.0, 1.0, 1.0, 0.0, 0.5], top_p=[1.0, 1.0, 1.0, 0.9, 0.9, 0.9])
    check(x, 1.0)


def test_rows_apart_and_rows_off_16_bytes():
    import torch
    x, u, _ = rows_of(5, 1003)
    wide = torch.full((5, 1111), 1e9, device="cuda")
    wide[:, 3:1006] = torch.from_numpy(x).cuda()
    check(x, u, 0.9, 50, 0.9, 0.01, device_logits=wide[:, 3:1006])
    check(x[:1], u[:1], device_logits=wide[:1, 3:1006])


def test_a_row_does_not_depend_on_its_batch():
    import torch
    x, u, rng = rows_of(600, 3001)
    d, t = torch.from_numpy(x).cuda(), lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    k, p = rng.integers(0, 99, 600).astype(np.int32), rng.uniform(0.3, 1.1, 600).astype(np.float32)
    many, lp = eng().op_sample(d, t(u), top_k=t(k), top_p=t(p))
    for r in (0, 299, 599):
        one, lp1 = eng().op_sample(d[r:r + 1], t(u[r:r + 1]), top_k=t(k[r:r + 1]), top_p=t(p[r:r + 1]))
        assert int(one) == int(many[r]) and float(lp1) == float(lp[r])


def test_graph_replays():
    import torch
    x, u, _ = rows_of(4, 20000)
    d, du = torch.from_numpy(x).cuda(), torch.from_numpy(u).cuda()
    k, p = torch.tensor([0, 40, 0, 5000], dtype=torch.int32).cuda(), torch.tensor([1.0, 0.9, 0.95, 0.9]).cuda()
    eng().op_sample(d, du, top_k=k, top_p=p)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = eng().op_sample(d, du, top_k=k, top_p=p)
    for seed in range(4):
        x, u, _ = rows_of(4, 20000, seed)
        d.copy_(torch.from_numpy(x)), du.copy_(torch.from_numpy(u))
        graph.replay()
        again = [t.clone() for t in got]
        want = check(x, u, top_k=k.cpu().numpy(), top_p=p.cpu().numpy())
        np.testing.assert_array_equal(again[0].cpu().numpy(), want)


def test_refusals():
    import torch
    import paper_2410_03065_amd as cake
    d, u = torch.zeros((2, 100), device="cuda"), torch.zeros(2, device="cuda")
    for bad in (d.double(), d[0], d.t(), d.cpu(), d.expand(2, 100)[:, ::2], torch.zeros((1, 100), device="cuda").expand(2, 100)):
        with pytest.raises(cake.CakeError):
            eng().op_sample(bad, u)
    for kw in (dict(temperature=u[:1]), dict(top_k=u), dict(top_p=u.double()), dict(min_p=u.cpu())):
        with pytest.raises(cake.CakeError):
            eng().op_sample(d, u, **kw)
    e, t = eng(), torch.zeros(2, dtype=torch.int32, device="cuda")
    call = lambda *a: e.lib.cake_op_sample(e.ctx, *a)  # noqa: E731
    ok = [d.data_ptr(), 100, 2, 100, None, None, None, None, u.data_ptr(), t.data_ptr(), None]
    assert call(*ok) == cake.OK
    for i, v in ((0, None), (1, 99), (2, -1), (3, 0), (3, 2 ** 19 + 1), (8, None), (9, None)):
        assert call(*[v if j == i else a for j, a in enumerate(ok)]) == cake.E_INVAL, i
    assert call(*[0 if j == 2 else a for j, a in enumerate(ok)]) == cake.OK


# Vocabularies on both sides of what one workgroup holds, and long ones, whose rows many workgroups share.
@pytest.mark.parametrize("vocab", [2047, 32767, 32768, 32769, 40001])
def test_around_the_longest_row_of_one_workgroup(vocab):
    x, u, rng = rows_of(3, vocab)
    check(x, u, 1.3)
    check(x, u, 0.8, rng.integers(1, 300, 3), rng.uniform(0.5, 0.99, 3), rng.uniform(0.001, 0.1, 3))
    check(x, u, top_k=[vocab // 2, 700, vocab - 1], top_p=[0.97, 0.5, 0.9])
    for at in (0, vocab - 1):                     # the first and the last id
        y = np.full((1, vocab), -np.inf, np.float32)
        y[0, at] = -5.0
        assert check(y, 0.7, top_k=3, top_p=0.5)[0] == at


@pytest.mark.parametrize("vocab", [33000])
def test_masks_ties_and_settings_of_long_rows(vocab):
    low = np.finfo(np.float32).min
    x, u, _ = rows_of(9, vocab)
    x[0] = -np.inf
    x[1] = np.nan
    x[2, 100:] = -np.inf
    x[3, 1:] = low
    x[4] = low
    x[5, :30000] = np.nan
    x[6, 17] = np.inf
    x[7, [5, 31000]] = np.inf
    x[8] = 0.0
    x[8, 7:] = -0.0
    for more in ({}, dict(top_k=20), dict(top_k=9000, top_p=0.6), dict(top_p=0.7), dict(min_p=0.01), dict(top_k=30, top_p=0.8, min_p=0.02),
                 dict(temperature=0.0), dict(temperature=1e-30), dict(temperature=1e30, top_p=0.9)):
        check(x, u, **more)


@pytest.mark.parametrize("vocab", [3000, 40000])
def test_logits_and_temperatures_at_the_ends_of_the_range(vocab):
    """Logits whose difference passes float32's largest number, and differences that only a tiny temperature tells apart."""
    x, u, rng = rows_of(3, vocab)
    for settings in (dict(), dict(top_k=40), dict(top_p=0.9), dict(top_k=100, top_p=0.8, min_p=0.01)):
        check(x * np.float32(1.7e37), u, temperature=2e37, **settings)
        check(x * np.float32(1e-38), u, temperature=1e-38, **settings)
        check(x * np.float32(1e-40), u, temperature=1e-40, **settings)


def test_graph_replays_of_long_rows():
    import torch
    x, u, _ = rows_of(4, 40000)
    d, du = torch.from_numpy(x).cuda(), torch.from_numpy(u).cuda()
    k, p = torch.tensor([0, 40, 0, 5000], dtype=torch.int32).cuda(), torch.tensor([1.0, 0.9, 0.95, 0.9]).cuda()
    graph = torch.cuda.CUDAGraph()
    eng().op_sample(d, du, top_k=k, top_p=p)
    with torch.cuda.graph(graph):
        got = eng().op_sample(d, du, top_k=k, top_p=p)
    for seed in range(4):
        x, u, _ = rows_of(4, 40000, seed)
        d.copy_(torch.from_numpy(x)), du.copy_(torch.from_numpy(u))
        graph.replay()
        again = got[0].clone()
        np.testing.assert_array_equal(again.cpu().numpy(), check(x, u, top_k=k.cpu().numpy(), top_p=p.cpu().numpy()))
