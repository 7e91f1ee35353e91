"""GPU parity of spd_rmsnorm against the fp64 oracle.

Bars.  h = bf16(x + residual) is one rounding of an exact sum: equal.  y: a thread's sum of up to 32 squares, six shuffles and up to 16
waves' parts are at most 60 roundings of positive fp32 sums, half of which reaches the square root; root, quotient and two products add
a few: below 40 2^-24 < 2^-18 relative.  The bf16 form rounds once more, by at most 2^-8 relative; the 8-bit form's codes and scales are those of
y (1 +- 2^-18)."""
import numpy as np
import pytest
import torch

from oracle import mx
from paper_2504_19867_amd import semipd as S
from gpu_util import DEV
from mx_util import E4M3, assert_quantised, bf16_tensor, mx_values, normal

pytestmark = pytest.mark.gpu
PRE, DEC = S.SPD_PHASE_PREFILL, S.SPD_PHASE_DECODE
DELTA, EPS = 2.0 ** -18, 1e-5


@pytest.fixture(scope="module")
def ctx():
    c = S.Context(0)
    yield c
    c.close()


def _bytes(T, hidden):
    """codes and scales with room behind, which has to stay as it is"""
    return (torch.full((T * hidden + 64,), 0x55, dtype=torch.uint8, device=DEV), torch.full((T * hidden // 32 + 64,), 0x55, dtype=torch.uint8, device=DEV))


def _run(ctx, phase, x, r, w, mx8, eps=EPS):
    T, hidden = x.shape
    tx, tw, tr = bf16_tensor(x), bf16_tensor(w), None if r is None else bf16_tensor(r)
    if mx8:
        out, scales = _bytes(T, hidden)
    else:
        out, scales = torch.full((T * hidden + 8,), 7.0, dtype=torch.bfloat16, device=DEV), None
    torch.cuda.synchronize()
    ctx.rmsnorm(phase, tx, tr, tw, eps, out, T, hidden, out_scales=scales)
    ctx.phase_sync(phase)
    y, h = mx.rmsnorm(x, r, w, eps)
    if tr is not None:
        assert np.array_equal(tr.double().cpu().numpy(), h)
    if mx8:
        assert (out[T * hidden:] == 0x55).all() and (scales[T * hidden // 32:] == 0x55).all()
        got, b = mx_values(out[:T * hidden], scales[:T * hidden // 32], T, hidden)
        assert_quantised(got, b, y, DELTA)
    else:
        assert (out[T * hidden:] == 7.0).all()
        got = out[:T * hidden].double().cpu().numpy().reshape(T, hidden)
        assert (np.abs(got - y) <= (2.0 ** -8 + DELTA) * np.abs(y)).all()
    assert np.array_equal(tx.double().cpu().numpy(), x)
    return got


@pytest.mark.parametrize("T, hidden", [(1, 8), (3, 24), (2, 512), (5, 520), (1, 2048), (7, 2056), (4, 4096), (2, 4104), (3, 8192), (1, 8200), (2, 16384),
                                       (1, 16392), (1, 32768), (300, 1000), (2050, 128)])
@pytest.mark.parametrize("residual", [False, True])
def test_bf16(ctx, T, hidden, residual):
    rng = np.random.default_rng(T + hidden)
    _run(ctx, DEC, normal(rng, T, hidden, spread=6), normal(rng, T, hidden, spread=6) if residual else None, normal(rng, hidden), False)


@pytest.mark.parametrize("T, hidden", [(1, 128), (3, 256), (2, 512), (5, 640), (1, 2048), (7, 2176), (4, 4096), (2, 4224), (3, 8192), (1, 8320), (2, 16384),
                                       (1, 16512), (1, 32768), (301, 1024), (2050, 128)])
@pytest.mark.parametrize("residual", [False, True])
def test_mx(ctx, T, hidden, residual):
    rng = np.random.default_rng(T + hidden)
    _run(ctx, PRE, normal(rng, T, hidden, spread=6), normal(rng, T, hidden, spread=6) if residual else None, normal(rng, hidden, spread=0), True)


@pytest.mark.parametrize("mx8", [False, True])
def test_rows_of_zeros_and_far_magnitudes(ctx, mx8):
    rng = np.random.default_rng(9)
    x = normal(rng, 6, 256)
    x[0] = 0
    x[1] *= 2.0 ** 40
    x[2] *= 2.0 ** -40                                 # far below sqrt(eps)
    x[3, :128] = 0
    x[4, 32:64] *= 2.0 ** -30
    w = normal(rng, 256)
    w[200:] = 0
    got = _run(ctx, DEC, x, None, w, mx8)
    assert (got[0] == 0).all() and (got[:, 200:] == 0).all()


def test_what_is_not_finite_stays_in_its_row(ctx):
    rng = np.random.default_rng(10)
    x, w = normal(rng, 4, 256), normal(rng, 256)
    clean, _ = mx.rmsnorm(x, None, w, EPS)
    for bad in (np.inf, np.nan):
        y = x.copy()
        y[1, 77] = bad
        t, tw = bf16_tensor(y), bf16_tensor(w)
        codes, scales = _bytes(4, 256)
        out = torch.empty(4, 256, dtype=torch.bfloat16, device=DEV)
        torch.cuda.synchronize()
        ctx.rmsnorm(DEC, t, None, tw, EPS, codes, 4, 256, out_scales=scales)
        ctx.rmsnorm(DEC, t, None, tw, EPS, out, 4, 256)
        ctx.phase_sync(DEC)
        got, b = mx_values(codes[:1024], scales[:32], 4, 256)
        keep = [0, 2, 3]
        assert_quantised(got[keep], b[keep], clean[keep], DELTA)
        o = out.double().cpu().numpy()
        assert np.isnan(got[1, 77]) and np.isnan(o[1, 77]) and np.isfinite(o[keep]).all()
        assert (np.isnan(o[1]).all() if np.isnan(bad) else (np.delete(o[1], 77) == 0).all())


@pytest.mark.parametrize("mx8", [False, True])
def test_weights_that_are_not_finite_stay_in_their_column(ctx, mx8):
    """h w / rms as it is: infinite by the signs of h and w, NaN where h is 0; in 8 bits NaN, and the other entries of the block as if it were not there."""
    rng = np.random.default_rng(13)
    T, hidden = 40, 256
    x, w = normal(rng, T, hidden), normal(rng, hidden)
    bad = {5: np.inf, 40: -np.inf, 41: np.inf, 100: np.nan, 255: -np.inf}
    x[3, 5] = x[7, 255] = 0
    clean = w.copy()
    clean[list(bad)] = 0
    for col, value in bad.items():
        w[col] = value
    tx, tw = bf16_tensor(x), bf16_tensor(w)
    out, scales = _bytes(T, hidden) if mx8 else (torch.zeros(T, hidden, dtype=torch.bfloat16, device=DEV), None)
    torch.cuda.synchronize()
    ctx.rmsnorm(DEC, tx, None, tw, EPS, out, T, hidden, out_scales=scales)
    ctx.phase_sync(DEC)
    with np.errstate(invalid="ignore"):
        lost = x[:, list(bad)] * w[list(bad)]            # (the root is finite and positive)
    y, _ = mx.rmsnorm(x, None, clean, EPS)
    if mx8:
        got, b = mx_values(out[:T * hidden], scales[:T * hidden // 32], T, hidden)
        assert np.isnan(got[:, list(bad)]).all()
        got[:, list(bad)] = 0
        assert_quantised(got, b, y, DELTA)
    else:
        got = out.double().cpu().numpy()
        np.testing.assert_array_equal(got[:, list(bad)], lost)
        got[:, list(bad)] = 0
        assert (np.abs(got - y) <= (2.0 ** -8 + DELTA) * np.abs(y)).all()


@pytest.mark.parametrize("mx8", [False, True])
@pytest.mark.parametrize("seed", [0, 1, 2])
def test_sums_whose_last_bits_decide(ctx, seed, mx8):
    """One large entry and thousands whose squares a sum in 24 bits next to it would round.  eps makes the root 64, so that y = h w / 64 is exact and many
    entries lie halfway between two codes (or bf16 values): all go to the even one."""
    rng = np.random.default_rng(seed)
    hidden = 4096
    x = rng.integers(112, 128, (1, hidden)) / 16 * rng.choice([-1.0, 1.0], (1, hidden))
    x[0, rng.integers(hidden)] = 4064
    eps = 4096 - (x * x).mean()
    assert eps > 0 and eps == np.float32(eps)
    for w in (np.full(hidden, 64.0), rng.integers(128, 256, hidden) / 4):
        y, _ = mx.rmsnorm(x, None, w, eps)
        assert np.array_equal(y, x * w / 64)
        tx, tw = bf16_tensor(x), bf16_tensor(w)
        out, scales = _bytes(1, hidden) if mx8 else (torch.zeros(1, hidden, dtype=torch.bfloat16, device=DEV), None)
        torch.cuda.synchronize()
        ctx.rmsnorm(PRE, tx, None, tw, eps, out, 1, hidden, out_scales=scales)
        ctx.phase_sync(PRE)
        if mx8:
            got, b = mx_values(out[:hidden], scales[:hidden // 32], 1, hidden)
            want, wb = mx.quantise(y, mx.E4M3)
            assert np.array_equal(b, wb) and np.array_equal(got, want), (got != want).sum()
        else:
            got, want = out.double().cpu().numpy(), mx.to_bf16(y)
            assert np.array_equal(got, want), (got != want).sum()


def test_codes_of_y_rounded_to_fp32(ctx):
    """The 8-bit form's y is off by one rounding to fp32 (2^-24) and next to nothing else, whatever the row's length."""
    rng = np.random.default_rng(14)
    for T, hidden in ((400, 4096), (60, 16384), (700, 384)):
        x, r, w = normal(rng, T, hidden, spread=6), normal(rng, T, hidden, spread=6), normal(rng, hidden)
        tx, tr, tw = bf16_tensor(x), bf16_tensor(r), bf16_tensor(w)
        out, scales = _bytes(T, hidden)
        torch.cuda.synchronize()
        ctx.rmsnorm(PRE, tx, tr, tw, EPS, out, T, hidden, out_scales=scales)
        ctx.phase_sync(PRE)
        got, b = mx_values(out[:T * hidden], scales[:T * hidden // 32], T, hidden)
        assert_quantised(got, b, mx.rmsnorm(x, r, w, float(np.float32(EPS)))[0], 2.0 ** -24 + 2.0 ** -38)


@pytest.mark.parametrize("mx8", [False, True])
def test_magnitudes_whose_squares_pass_fp32(ctx, mx8):
    rng = np.random.default_rng(15)
    x, w = normal(rng, 4, 512), normal(rng, 512)
    x *= np.array([2.0 ** 70, 2.0 ** 120, 2.0 ** -90, 2.0 ** 63])[:, None]
    got = _run(ctx, DEC, x, None, w, mx8)
    assert (got[[0, 1, 3]].any(1)).all()
    assert (_run(ctx, DEC, x[2:3], None, w, mx8, eps=2.0 ** -148) != 0).any()         # below fp32's range


def test_a_row_of_infinite_root(ctx):
    """Whatever is finite in it weighs nothing, also where entry times weight passes fp32's range."""
    x, w = np.zeros((1, 128)), np.ones(128)
    x[0, 3], x[0, 9], w[9], x[0, 20] = np.inf, 2.0 ** 127, 2.0 ** 100, 5
    tx, tw = bf16_tensor(x), bf16_tensor(w)
    out = torch.empty_like(tx)
    torch.cuda.synchronize()
    ctx.rmsnorm(DEC, tx, None, tw, EPS, out, 1, 128)
    ctx.phase_sync(DEC)
    o = out.double().cpu().numpy()[0]
    assert np.isnan(o[3]) and (np.delete(o, 3) == 0).all()


def test_in_place_and_without_rows(ctx):
    rng = np.random.default_rng(11)
    x, w = normal(rng, 9, 1032), normal(rng, 1032)
    t, tw = bf16_tensor(x), bf16_tensor(w)
    torch.cuda.synchronize()
    ctx.rmsnorm(PRE, t, None, tw, EPS, t, 9, 1032)
    ctx.rmsnorm(PRE, None, None, None, EPS, None, 0, 1032)
    ctx.phase_sync(PRE)
    y, _ = mx.rmsnorm(x, None, w, EPS)
    assert (np.abs(t.double().cpu().numpy() - y) <= (2.0 ** -8 + DELTA) * np.abs(y)).all()


def test_captured_and_replayed(ctx):
    """A graph of both forms, replayed with eager calls between: what the eager call gives, every time."""
    rng = np.random.default_rng(12)
    T, hidden = 33, 1024
    w = bf16_tensor(normal(rng, hidden))
    x = torch.empty(T, hidden, dtype=torch.bfloat16, device=DEV)
    out, codes, scales = torch.empty_like(x), *(t[:n] for t, n in zip(_bytes(T, hidden), (T * hidden, T * hidden // 32)))
    c = S.Context(0)
    stream = torch.cuda.ExternalStream(c.phase_stream(DEC))
    calls = lambda: (c.rmsnorm(DEC, x, None, w, EPS, out, T, hidden), c.rmsnorm(DEC, x, None, w, EPS, codes, T, hidden, out_scales=scales))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        calls()
    for seed in range(4):
        x.copy_(bf16_tensor(normal(np.random.default_rng(seed), T, hidden)))
        torch.cuda.synchronize()
        calls()
        c.phase_sync(DEC)
        want = [t.clone() for t in (out, codes, scales)]
        for t in (out.view(torch.uint8), codes, scales):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (out, codes, scales)))
    c.close()


def test_more_rows_than_a_launch_takes(ctx):
    """Short rows, more than 2^21 of them, and entries beyond 2^32: rows by the first and last launch."""
    for T, hidden in ((2 ** 22 + 3, 8), (2 ** 21 + 1, 2056)):
        gen = torch.Generator(device=DEV).manual_seed(hidden)
        x = torch.empty(T, hidden, dtype=torch.bfloat16, device=DEV).normal_(generator=gen)
        out, w = torch.zeros_like(x), torch.full((hidden,), 1.5, dtype=torch.bfloat16, device=DEV)
        torch.cuda.synchronize()
        ctx.rmsnorm(DEC, x, None, w, EPS, out, T, hidden)
        ctx.phase_sync(DEC)
        for rows in (slice(0, 5), slice(2 ** 21 - 2, 2 ** 21 + 2), slice(T - 5, T)):
            h = x[rows].double().cpu().numpy()
            y, _ = mx.rmsnorm(h, None, np.full(hidden, 1.5), EPS)
            assert (np.abs(out[rows].double().cpu().numpy() - y) <= (2.0 ** -8 + DELTA) * np.abs(y)).all()


def test_codes_beyond_4gib(ctx):
    T, hidden = 2 ** 19 + 77, 8320
    gen = torch.Generator(device=DEV).manual_seed(1)
    x = torch.empty(T, hidden, dtype=torch.bfloat16, device=DEV).normal_(generator=gen)
    w = torch.full((hidden,), 1.5, dtype=torch.bfloat16, device=DEV)
    out, scales = torch.zeros(T, hidden, dtype=torch.uint8, device=DEV), torch.zeros(hidden // 128, T, 4, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    ctx.rmsnorm(DEC, x, None, w, EPS, out, T, hidden, out_scales=scales)
    ctx.phase_sync(DEC)
    for rows in (slice(0, 3), slice(T - 3, T)):
        y, _ = mx.rmsnorm(x[rows].double().cpu().numpy(), None, np.full(hidden, 1.5), EPS)
        assert_quantised(*mx_values(out[rows].contiguous(), scales[:, rows].contiguous(), 3, hidden), y, DELTA)
