"""GPU parity of the gated FFN's first step over MXFP4 weights and MXFP8 rows (spd_ffn_pack_gate_up_mx, spd_ffn_unpack_gate_up_mx,
spd_ffn_gate_up_mx) against the fp64 oracle, and of the chain norm -> FFN.

Bars.  Quantisation is one rounding of exact quotients: equal.  Product: silu(g) u is rounded once, 2^-8 relative at most.  Before that a
matrix instruction adds products.  Of eight neighbours it cuts each, towards zero, to a multiple of q = 2^(e - 13), e the largest sum of a pair's exponents
(test_what_the_matrix_instruction_cuts).  2^e is at most twice the largest product m of the eight: exponents alone make at most the product, but for E2M1's 0.5,
which counts as 2^0; and where the pair that makes e has an E4M3 code below the normal ones, all that is cut has too (a product is a multiple of 2^(its sum
of exponents - 4), so is cut only if e is 10 more than that, and E2M1's exponents span 2), which E4M3's exponents do not allow.  So with Q = 2^(floor(log2 2m) - 13), a
multiple of q, a product loses at most |x w| mod Q: dg = sum (|x w| mod Q).  The sums of eight it adds to an fp32 sum, keeping 2^-20 of the largest,
and rounds that: 2^-13 sum over the steps of 128 entries of max |x w| more.  The result is then off by 1.1 |u| dg + |silu(g)| du; exponential and reciprocal
add 2^-20 |y|."""
import numpy as np
import pytest
import torch

from oracle import ffn as F
from oracle import mx
from paper_2504_19867_amd import semipd as S
from gpu_util import DEV
from mx_util import assert_quantised, bf16_tensor, mx_tensors, mx_values, normal

pytestmark = pytest.mark.gpu
PRE, DEC = S.SPD_PHASE_PREFILL, S.SPD_PHASE_DECODE


@pytest.fixture(scope="module")
def ctx():
    c = S.Context(0)
    yield c
    c.close()


def _pack(ctx, phase, wg, wu):
    I, K = wg.shape
    n = S.ffn_mx_bytes(K, I)
    w = torch.full((n + 256,), 0x5A, dtype=torch.uint8, device=DEV)
    tg, tu = bf16_tensor(wg), bf16_tensor(wu)
    torch.cuda.synchronize()
    ctx.ffn_pack_gate_up_mx(phase, tg, tu, w, K, I)
    ctx.phase_sync(phase)
    assert (w[n:] == 0x5A).all()
    return w


def _unpack(ctx, phase, w, K, I):
    back = [torch.full((I, K), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    torch.cuda.synchronize()
    ctx.ffn_unpack_gate_up_mx(phase, w, *back, K, I)
    ctx.phase_sync(phase)
    return [t.double().cpu().numpy() for t in back]


def _weights(rng, I, K):
    return normal(rng, I, K, spread=2) * 2.0 ** -3, normal(rng, I, K, spread=2) * 2.0 ** -3


def _rows(rng, T, K, spread=2):
    return mx.quantise(normal(rng, T, K, spread=spread), mx.E4M3)


def _bar(x, wg, wu, y, g, u):
    def off(w):
        m = np.zeros((x.shape[0], w.shape[0]))
        for t in range(x.shape[0]):
            p = np.abs(x[t] * w).reshape(w.shape[0], -1, 8)
            most = p.max(-1)
            Q = np.exp2(np.floor(np.log2(np.maximum(2 * most, 2.0 ** -900))) - 13)[..., None]
            p /= Q
            m[t] = ((p - np.floor(p)) * Q).sum((1, 2)) + 2.0 ** -13 * most.reshape(w.shape[0], -1, 16).max(-1).sum(-1)
        return m
    s = g / (1 + np.exp(-g))
    return (2.0 ** -8 + 2.0 ** -20) * np.abs(y) + 1.1 * np.abs(u) * off(wg) + np.abs(s) * off(wu)


def _check(got, x, wg, wu):
    y = F.gate_up(x, wg, wu)
    assert got.shape == y.shape and np.isfinite(got).all()
    err, bar = np.abs(got - y), _bar(x, wg, wu, y, x @ wg.T, x @ wu.T)
    assert (err <= bar).all(), f"{(err > bar).sum()} entries beyond the bar, worst {(err / bar).max():.3g} of it"


def _run(ctx, phase, codes, scales, w, T, K, I, offset=0):
    flat = torch.full(((T + 1) * I + offset,), 7.0, dtype=torch.bfloat16, device=DEV)
    out = flat[offset:]
    torch.cuda.synchronize()
    ctx.ffn_gate_up_mx(phase, codes, scales, w, out, T, K, I)
    ctx.phase_sync(phase)
    assert (flat[:offset] == 7.0).all() and (out[T * I:] == 7.0).all()
    return out[:T * I].double().cpu().numpy().reshape(T, I)


@pytest.mark.parametrize("I, K", [(128, 128), (256, 384), (640, 256), (128, 1152)])
def test_pack_and_unpack_are_the_oracles_quantisation(ctx, I, K):
    rng = np.random.default_rng(I + K)
    wg, wu = _weights(rng, I, K)
    wg[0] = 0
    wg[1, :32] *= 2.0 ** 100
    wu[2, 32:64] *= 2.0 ** -100
    wu[3, :8] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -6]      # every tie, under scale 1
    wu[3, 8:32] = 0
    back = _unpack(ctx, DEC, _pack(ctx, DEC, wg, wu), K, I)
    for got, want in zip(back, (wg, wu)):
        assert np.array_equal(got, mx.quantise(want, mx.E2M1)[0])
    again = _unpack(ctx, PRE, _pack(ctx, PRE, *back), K, I)     # what a packed weight stands for packs to itself
    assert all(np.array_equal(a, b) for a, b in zip(back, again))


@pytest.mark.parametrize("T", [16, 100, 200])
def test_what_the_matrix_instruction_cuts(ctx, T):
    """Two large products that cancel, and a small one: whole where it is none of their eight neighbours, else a multiple of 2^-13 of the exponents' sum."""
    K, I = 128, 128
    wg, wu, x = np.zeros((I, K)), np.zeros((I, K)), np.zeros((T, K))
    x[:, 0], wg[:, 0] = 4, 6                                     # g = 24: silu(g) is 24 to 2^-34
    x[:, 17:19], wu[:, 17], wu[:, 18] = 448, 6, -6               # exponents 8 and 2: multiples of 2^-3
    at = np.array([1, 16, 20, 23, 24, 40, 100])[np.arange(T) % 7]
    small = np.array([2.0 ** -9, 2.0 ** -4, 0.125, 0.1875, 0.3125, 0.4375])[np.arange(T) % 6]
    x[np.arange(T), at] = small
    wu[:, [1, 16, 20, 23, 24, 40, 100]] = 1
    got = _run(ctx, DEC, *mx_tensors(x, np.full((T, 4), 127)), _pack(ctx, DEC, wg, wu), T, K, I)
    near = (at >= 16) & (at < 24)
    want = 24 * np.where(near, np.floor(small * 8) / 8, small)
    assert (np.abs(got - want[:, None]) <= 2.0 ** -8 * want[:, None]).all()


TOKENS = [1, 2, 15, 16, 17, 31, 33, 64, 65, 100, 128, 129, 200, 256, 257, 300]


@pytest.mark.parametrize("T", TOKENS)
@pytest.mark.parametrize("I, K", [(128, 128), (384, 256), (256, 1152)])
def test_product(ctx, T, I, K):
    rng = np.random.default_rng(1000 * T + I + K)
    wg, wu = _weights(rng, I, K)
    w = _pack(ctx, DEC, wg, wu)
    x, b = _rows(rng, T, K)
    got = _run(ctx, DEC if T < 100 else PRE, *mx_tensors(x, b), w, T, K, I)
    _check(got, x, mx.quantise(wg, mx.E2M1)[0], mx.quantise(wu, mx.E2M1)[0])


@pytest.mark.parametrize("cus", [32, 64, 160, 224])
@pytest.mark.parametrize("T, I, K", [(1, 1408, 512), (40, 1408, 640), (128, 2816, 256), (70, 3584, 384), (520, 1408, 256)])
def test_shares_of_the_chip(ctx, cus, T, I, K):
    """Launch shapes go by the phase's compute units."""
    c = S.Context(0)
    total = c.device_info()[0]
    c.set_partition(cus, total - cus)
    rng = np.random.default_rng(cus + T)
    wg, wu = _weights(rng, I, K)
    w = _pack(c, PRE, wg, wu)
    x, b = _rows(rng, T, K)
    q = [mx.quantise(v, mx.E2M1)[0] for v in (wg, wu)]
    for phase in (PRE, DEC):
        got = _run(c, phase, *mx_tensors(x, b), w, T, K, I)
        pick = sorted({0, T // 2, T - 1})
        _check(got[pick], x[pick], *q)
    c.close()


@pytest.mark.parametrize("T, I, K", [(256, 2048, 128), (257, 2048, 384), (300, 2048, 128), (512, 2048, 640), (700, 2048, 128), (2100, 1408, 256),
                                     (640, 896, 1152), (1000, 512, 128)])
def test_tiles_of_many_tokens(T, I, K):
    """On 32 compute units: tiles of 128 and of 256 tokens, one and several per workgroup, the last one with one token, some and all."""
    c = S.Context(0)
    c.set_partition(c.device_info()[0] - 32, 32)
    rng = np.random.default_rng(I + T)
    wg, wu = _weights(rng, I, K)
    w = _pack(c, DEC, wg, wu)
    x, b = _rows(rng, T, K)
    got = _run(c, DEC, *mx_tensors(x, b), w, T, K, I)
    pick = sorted({*range(0, T, 61), 127, 128, T - 2, T - 1})
    _check(got[pick], x[pick], *(mx.quantise(v, mx.E2M1)[0] for v in (wg, wu)))
    c.close()


@pytest.mark.parametrize("T", [3, 20, 50, 100])
@pytest.mark.parametrize("I", [128, 1408, 2048, 2560, 2816, 3584, 4096, 4224])
def test_units_per_workgroup(T, I):
    """On 32 compute units: workgroups of two to eight units of 16 outputs, whole and not; slices that divide evenly over waves and rings and not."""
    c = S.Context(0)
    c.set_partition(c.device_info()[0] - 32, 32)
    rng = np.random.default_rng(I + T)
    for K in (128, 896, 1152):
        wg, wu = _weights(rng, I, K)
        w = _pack(c, DEC, wg, wu)
        x, b = _rows(rng, T, K)
        got = _run(c, DEC, *mx_tensors(x, b), w, T, K, I)
        pick = sorted({0, T // 2, T - 1})
        _check(got[pick], x[pick], *(mx.quantise(v, mx.E2M1)[0] for v in (wg, wu)))
    c.close()


@pytest.mark.parametrize("T", [1, 48, 300])
def test_model_shape(ctx, T):
    """hidden 4096, inter 14336: sampled outputs of all tokens"""
    K, I = 4096, 14336
    gen = torch.Generator(device=DEV)
    gen.manual_seed(T)
    w = [torch.randn(I, K, generator=gen, device=DEV).mul_(K ** -0.5).to(torch.bfloat16) for _ in range(2)]
    packed = torch.empty(S.ffn_mx_bytes(K, I), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    ctx.ffn_pack_gate_up_mx(DEC, *w, packed, K, I)
    x, b = _rows(np.random.default_rng(T), T, K)
    got = _run(ctx, DEC, *mx_tensors(x, b), packed, T, K, I)
    cols = np.random.default_rng(1).choice(I, 40, replace=False)
    q = [mx.quantise(t[cols].double().cpu().numpy(), mx.E2M1)[0] for t in w]
    _check(got[:, cols], x, *q)


def test_alignment_of_out_and_scales(ctx):
    """out starts on any entry, the scales on any word"""
    T, K, I = 37, 256, 256
    rng = np.random.default_rng(5)
    wg, wu = _weights(rng, I, K)
    w = _pack(ctx, DEC, wg, wu)
    x, b = _rows(rng, T, K)
    codes, scales = mx_tensors(x, b)
    want = _run(ctx, DEC, codes, scales, w, T, K, I)
    moved = torch.empty(scales.numel() + 4, dtype=torch.uint8, device=DEV)
    moved[4:] = scales.flatten()
    for offset in (1, 3, 4):
        assert np.array_equal(_run(ctx, DEC, codes, moved[4:], w, T, K, I, offset), want)
    for T2 in (150, 300):
        x2, b2 = _rows(rng, T2, K)
        c2, s2 = mx_tensors(x2, b2)
        assert np.array_equal(_run(ctx, DEC, c2, s2, w, T2, K, I, 1), _run(ctx, DEC, c2, s2, w, T2, K, I))


def test_a_tokens_result_does_not_depend_on_its_batch_neighbours(ctx):
    """The same row among others of the same batch size: the same bits, whatever its neighbours hold."""
    T, K, I = 50, 512, 256
    rng = np.random.default_rng(6)
    w = _pack(ctx, DEC, *_weights(rng, I, K))
    x, b = _rows(rng, T, K)
    first = _run(ctx, DEC, *mx_tensors(x, b), w, T, K, I)
    y, c = _rows(rng, T, K)
    y[20], c[20] = x[20], b[20]
    assert np.array_equal(_run(ctx, DEC, *mx_tensors(y, c), w, T, K, I)[20], first[20])


@pytest.mark.parametrize("T", [3, 70, 300])
def test_nan_stays_in_its_row_and_its_column(ctx, T):
    K, I = 256, 256
    rng = np.random.default_rng(7)
    wg, wu = _weights(rng, I, K)
    wu[100, 40] = np.inf                                # the block of 32 around it becomes NaN
    w = _pack(ctx, DEC, wg, wu)
    back = _unpack(ctx, DEC, w, K, I)
    assert np.isnan(back[1][100, 32:64]).all() and np.isfinite(np.delete(back[1], 100, 0)).all() and np.isfinite(back[1][100, 64:]).all()
    x, b = _rows(rng, T, K)
    codes, scales = mx_tensors(x, b)
    raw = codes.view(torch.uint8)
    raw[T - 1, 200] = 0x7F
    out = torch.empty(T, I, dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    ctx.ffn_gate_up_mx(DEC, codes, scales, w, out, T, K, I)
    ctx.phase_sync(DEC)
    got = out.double().cpu().numpy()
    assert np.isnan(got[T - 1]).all() and np.isnan(got[:, 100]).all()
    q = [mx.quantise(np.delete(v, 100, 0), mx.E2M1)[0] for v in (wg, wu)]
    _check(np.delete(got, 100, 1)[:T - 1], x[:T - 1], *q)


@pytest.mark.parametrize("T", [1, 77, 400])
def test_norm_then_ffn(ctx, T):
    """The two calls as a layer makes them, on one stream: the FFN on the codes that the norm wrote."""
    K, I = 512, 384
    rng = np.random.default_rng(T)
    x, r, weight = normal(rng, T, K, spread=2), normal(rng, T, K, spread=2), normal(rng, K)
    wg, wu = _weights(rng, I, K)
    w = _pack(ctx, PRE, wg, wu)
    tx, tr, tw = bf16_tensor(x), bf16_tensor(r), bf16_tensor(weight)
    codes, scales = torch.empty(T, K, dtype=torch.uint8, device=DEV), torch.empty(K // 128, T, 4, dtype=torch.uint8, device=DEV)
    out = torch.empty(T, I, dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    ctx.rmsnorm(PRE, tx, tr, tw, 1e-5, codes, T, K, out_scales=scales)
    ctx.ffn_gate_up_mx(PRE, codes, scales, w, out, T, K, I)
    ctx.phase_sync(PRE)
    values, b = mx_values(codes, scales, T, K)
    assert_quantised(values, b, mx.rmsnorm(x, r, weight, 1e-5)[0], 2.0 ** -18)
    _check(out.double().cpu().numpy(), values, *(mx.quantise(v, mx.E2M1)[0] for v in (wg, wu)))


@pytest.mark.parametrize("T", [5, 90, 300])
def test_captured_and_replayed(T):
    K, I = 384, 512
    rng = np.random.default_rng(T)
    c = S.Context(0)
    w = _pack(c, DEC, *_weights(rng, I, K))
    codes, scales = (t.clone() for t in mx_tensors(*_rows(rng, T, K)))
    out = torch.empty(T, I, dtype=torch.bfloat16, device=DEV)
    stream = torch.cuda.ExternalStream(c.phase_stream(DEC))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        c.ffn_gate_up_mx(DEC, codes, scales, w, out, T, K, I)
    for seed in range(3):
        x = mx_tensors(*_rows(np.random.default_rng(seed), T, K))
        codes.view(torch.uint8).copy_(x[0].view(torch.uint8))
        scales.copy_(x[1])
        torch.cuda.synchronize()
        c.ffn_gate_up_mx(DEC, codes, scales, w, out, T, K, I)
        c.phase_sync(DEC)
        want = out.clone()
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    c.close()


def _codes(T, K, seed):
    """rows of random finite codes, under scales about 1, and their values"""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randint(0, 0x70, (T, K), generator=gen, device=DEV, dtype=torch.uint8)
    x += 128 * torch.randint(0, 2, (T, K), generator=gen, device=DEV, dtype=torch.uint8)
    return x, torch.randint(118, 124, (K // 128, T, 4), generator=gen, device=DEV, dtype=torch.uint8)


def test_rows_and_outputs_beyond_4gib(ctx):
    rng = np.random.default_rng(2)
    for K, I, T in ((8192, 128, 2 ** 19 + 300), (128, 2048, 2 ** 20 + 140)):
        wg, wu = _weights(rng, I, K)
        w = _pack(ctx, PRE, wg, wu)
        x, scales = _codes(T, K, 3)
        out = torch.zeros(T, I, dtype=torch.bfloat16, device=DEV)
        torch.cuda.synchronize()
        ctx.ffn_gate_up_mx(PRE, x, scales, w, out, T, K, I)
        ctx.phase_sync(PRE)
        for rows in (slice(0, 2), slice(T - 3, T)):
            n = rows.stop - rows.start
            v, _ = mx_values(x[rows].contiguous(), scales[:, rows].contiguous(), n, K)
            _check(out[rows].double().cpu().numpy(), v, mx.quantise(wg, mx.E2M1)[0], mx.quantise(wu, mx.E2M1)[0])
        del x, scales, out


def test_weights_beyond_4gib(ctx):
    K, I = 8192, 516096
    gen = torch.Generator(device=DEV).manual_seed(4)
    wg, wu = (torch.empty(I, K, dtype=torch.bfloat16, device=DEV).normal_(0, K ** -0.5, generator=gen) for _ in range(2))
    n = S.ffn_mx_bytes(K, I)
    w = torch.zeros(n, dtype=torch.uint8, device=DEV)
    assert n > 2 ** 32
    torch.cuda.synchronize()
    ctx.ffn_pack_gate_up_mx(PRE, wg, wu, w, K, I)
    ctx.phase_sync(PRE)
    ends = [0, 1, I - 130, I - 1]
    want = [mx.quantise(t[ends].double().cpu().numpy(), mx.E2M1)[0] for t in (wg, wu)]
    for t in (wg, wu):
        t.zero_()
    torch.cuda.synchronize()
    ctx.ffn_unpack_gate_up_mx(PRE, w, wg, wu, K, I)
    ctx.phase_sync(PRE)
    assert all(np.array_equal(t[ends].double().cpu().numpy(), q) for t, q in zip((wg, wu), want))
    del wg, wu
    for T in (2, 130):
        x, scales = _codes(T, K, T)
        out = torch.zeros(T, I, dtype=torch.bfloat16, device=DEV)
        torch.cuda.synchronize()
        ctx.ffn_gate_up_mx(DEC, x, scales, w, out, T, K, I)
        ctx.phase_sync(DEC)
        _check(out[:2, ends].double().cpu().numpy(), mx_values(x, scales, T, K)[0][:2], *want)
