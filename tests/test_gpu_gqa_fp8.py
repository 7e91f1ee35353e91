"""GPU parity of GQA pools in 8 bits (pool kind SPD_KV_GQA_FP8) against the fp64 oracle.

Pages.  Scales are powers of two and codes one rounding of exact quotients: gathered rows equal the oracle's, bit for bit.

Attention.  The kernels' products are those of the cached values (exact in bf16) with bf16 queries, summed in fp32.  Weights are rounded to bf16 ahead of
the second product: by 2^-8 of a weight at most, so by 2^-8 A of the result, A = sum p |v|; where the sum of weights is taken over the rounded ones
(prefill) by twice that.  A score of magnitude s is off by less than (D + 4) 2^-24 of the sum of its products' magnitudes, S = scale sum |q k|, a weight by
2 (D + 4) 2^-24 S relative: 2^-15 S with D = 128.  The output is rounded once, by 2^-8 of it."""
import numpy as np
import pytest
import torch

from oracle import mx
from paper_2504_19867_amd import semipd as S
from gpu_util import DEV
from mx_util import bf16_tensor, normal

pytestmark = pytest.mark.gpu
PRE, DEC = S.SPD_PHASE_PREFILL, S.SPD_PHASE_DECODE


class Pool8:
    """A pool in 8 bits beside the oracle's rows of its requests."""

    def __init__(self, Hkv, D, P=16, pages=400, ctx=None):
        self.Hkv, self.D, self.P = Hkv, D, P
        self.ctx = ctx or S.Context(0)
        self.own = ctx is None
        nbytes = S.pool_bytes(S.SPD_KV_GQA_FP8, P, Hkv, D, D, pages)
        self.mem = torch.full((nbytes,), 0xFF, dtype=torch.uint8, device=DEV)     # codes of NaN, scales of NaN
        self.pool = S.Pool(self.ctx, self.mem, nbytes, S.SPD_KV_GQA_FP8, P, Hkv, D, D, pages)
        self.k, self.v = {}, {}
        torch.cuda.synchronize()

    def note(self, rid, start, k, v):
        for side, rows in ((self.k, k), (self.v, v)):
            side.setdefault(rid, mx.Cache8(self.Hkv, self.D)).write(start, rows)

    def write(self, rid, start, k, v, phase=DEC):
        self.pool.kv_reserve(rid, start + len(k))
        tk, tv = bf16_tensor(k), bf16_tensor(v)
        torch.cuda.synchronize()
        self.pool.kv_write(phase, rid, start, len(k), tk, tv)
        self.ctx.phase_sync(phase)
        self.note(rid, start, k, v)

    def gather(self, rid, n, phase=DEC):
        out = [torch.full((n + 1, self.Hkv, self.D), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        torch.cuda.synchronize()
        self.pool.kv_gather(phase, rid, n, *out)
        self.ctx.phase_sync(phase)
        assert all((t[n] == 7.0).all() for t in out)
        return [t[:n].double().cpu().numpy() for t in out]

    def assert_rows(self, rid, phase=DEC):
        want = self.k[rid].rows, self.v[rid].rows
        for got, w in zip(self.gather(rid, len(want[0]), phase), want):
            np.testing.assert_array_equal(got, w)

    def close(self):
        self.pool.close()
        if self.own:
            self.ctx.close()


def attention(q, k, v, scale, first=None):
    """(out, bar) of rows q [n, H, D] over k, v [m, Hkv, D]; row i sees first + i + 1 keys (None: all)"""
    n, H, D = q.shape
    G = H // k.shape[1]
    out, A, Smax = np.empty((n, H, D)), np.empty((n, H, D)), np.empty((n, H, 1))
    for h in range(H):
        kk, vv = k[:, h // G], v[:, h // G]
        s = scale * q[:, h] @ kk.T
        mag = scale * np.abs(q[:, h]) @ np.abs(kk).T
        if first is not None:
            hide = np.arange(len(k))[None] > first + np.arange(n)[:, None]
            s[hide], mag[hide] = -np.inf, 0
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        out[:, h], A[:, h], Smax[:, h] = p @ vv, p @ np.abs(vv), mag.max(-1, keepdims=True)
    weight = 2.0 ** -8 if first is None else 2.0 ** -7
    return out, (weight + 2.0 ** -15 * Smax) * A + 2.0 ** -8 * np.abs(out) + 1e-30


def assert_close(got, want_bar, what=""):
    want, bar = want_bar
    err = np.abs(got - want)
    assert got.shape == want.shape and (err <= bar).all(), f"{what}: worst {np.nanmax(err / bar):.3g} of the bar, {np.isnan(got).sum()} NaN"


def _rows(rng, n, Hkv, D, spread=1.5):
    return normal(rng, n, Hkv, D, spread=spread), normal(rng, n, Hkv, D, spread=spread)


def _decode(p, ids, lens, q, scale, k=None, v=None, rope=None, noalloc=False):
    B, H, D = q.shape
    tq, out = bf16_tensor(q), torch.full((B + 1, H, D), 7.0, dtype=torch.bfloat16, device=DEV)
    tk, tv = (None, None) if k is None else (bf16_tensor(k), bf16_tensor(v))
    torch.cuda.synchronize()
    batch = p.pool.make_decode_batch(ids, lens, tq, out, H, scale, tk, tv, rope)
    (p.pool.decode_step_noalloc_batch if noalloc else p.pool.decode_step_batch)(batch)
    p.ctx.phase_sync(DEC)
    assert (out[B] == 7.0).all()
    for t, x in ((tq, q), (tk, k), (tv, v)):
        assert t is None or np.array_equal(t.double().cpu().numpy(), x)
    return out[:B].double().cpu().numpy()


def _check_decode(p, ids, lens, q, scale, got, what=""):
    for i, (rid, n) in enumerate(zip(ids, lens)):
        assert_close(got[i:i + 1], attention(q[i:i + 1], p.k[rid].rows[:n], p.v[rid].rows[:n], scale), f"{what} request {i} of {n} tokens")


# ----------------------------------------------------------------------------------------- rows
@pytest.mark.parametrize("Hkv, D, P", [(1, 64, 16), (2, 128, 16), (3, 64, 32), (5, 128, 48), (8, 128, 16), (9, 128, 64)])
@pytest.mark.parametrize("phase", [PRE, DEC])
def test_rows_come_back_as_the_oracle_rounds_them(Hkv, D, P, phase):
    p = Pool8(Hkv, D, P)
    rng = np.random.default_rng(Hkv * D + P)
    for rid, cuts in enumerate(([1], [16], [37], [15, 16, 17, 18, 200], [5, 9, 30, 31, 32, 97], [160])):
        start = 0
        for cut in cuts:
            p.write(rid, start, *_rows(rng, cut - start, Hkv, D, spread=8), phase=phase)
            start = cut
        p.assert_rows(rid, phase)
    p.close()


def test_scales_far_apart_and_zeros():
    """Each head's keys and values go by their own scale; a block of zeros takes any scale that comes."""
    p = Pool8(4, 64)
    rng = np.random.default_rng(1)
    k, v = _rows(rng, 40, 4, 64)
    k[:, 1] = 0
    k[:, 2] *= 2.0 ** 100
    v[:, 3] *= 2.0 ** -100
    v[:16] = 0
    p.write(1, 0, k[:35], v[:35])
    p.write(1, 35, k[35:] * 2.0 ** 12, v[35:] * 2.0 ** -12)        # the scale grows, and does not shrink
    p.assert_rows(1)
    p.write(2, 0, k[:3] * 0, v[:3] * 0)
    p.write(2, 3, k[3:20] * 2.0 ** -20, v[3:20])
    p.assert_rows(2)
    p.close()


def test_a_block_written_again_from_its_start_forgets_its_scale():
    p = Pool8(2, 128)
    rng = np.random.default_rng(2)
    k, v = _rows(rng, 32, 2, 128)
    p.write(1, 0, k * 2.0 ** 9, v * 2.0 ** 9)
    p.write(1, 16, k[:5], v[:5])
    p.assert_rows(1)
    p.write(1, 0, k[:7], v[:7])
    assert len(p.k[1].rows) == 7
    p.assert_rows(1)
    p.write(1, 3, k[:2] * 4, v[:2])
    p.assert_rows(1)
    p.close()


def test_what_is_not_finite_is_nan_and_alone():
    p = Pool8(2, 64)
    rng = np.random.default_rng(3)
    k, v = _rows(rng, 20, 2, 64)
    clean = mx.Cache8(2, 64)
    clean.write(0, np.where(np.arange(64) == 9, 0, k))
    bad = k.copy()
    bad[:, :, 9] = 0
    bad[4, 1, 9], bad[18, 0, 9] = np.inf, np.nan
    p.pool.kv_reserve(1, 20)
    tk, tv = bf16_tensor(bad), bf16_tensor(v)
    torch.cuda.synchronize()
    p.pool.kv_write(DEC, 1, 0, 20, tk, tv)
    p.ctx.phase_sync(DEC)
    got = p.gather(1, 20)[0]
    want = clean.rows.copy()
    want[4, 1, 9] = want[18, 0, 9] = np.nan
    np.testing.assert_array_equal(got, want)
    p.close()


# ----------------------------------------------------------------------------------------- decode
@pytest.mark.parametrize("H, Hkv, D, P", [(8, 8, 64, 16), (32, 8, 128, 16), (64, 8, 128, 16), (6, 2, 128, 32), (14, 2, 64, 48), (16, 1, 128, 64), (3, 3, 128, 16)])
def test_decode(H, Hkv, D, P):
    p = Pool8(Hkv, D, P, pages=900)
    rng = np.random.default_rng(H + D)
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 64, 129, 200, 333, 1025, 2600]
    for rid, n in enumerate(lens):
        p.write(rid, 0, *_rows(rng, n, Hkv, D))
    q = normal(rng, len(lens), H, D)
    ids = list(range(len(lens)))
    got = _decode(p, ids, lens, q, D ** -0.5)
    _check_decode(p, ids, lens, q, D ** -0.5, got)
    assert np.array_equal(_decode(p, ids, lens, q, D ** -0.5), got)
    assert np.array_equal(_decode(p, ids, lens, q, D ** -0.5, noalloc=True), got)
    p.close()


def test_decode_of_part_of_what_is_cached():
    """A context that ends inside a block: what lies behind it, not finite or large, weighs nothing."""
    p = Pool8(2, 128)
    rng = np.random.default_rng(4)
    k, v = _rows(rng, 60, 2, 128)
    kb, vb = k.copy(), v.copy()
    kb[45:48], vb[45:48] = np.nan, np.nan
    kb[48:], vb[48:] = np.inf, np.nan
    p.pool.kv_reserve(1, 60)
    tk, tv = bf16_tensor(kb), bf16_tensor(vb)
    torch.cuda.synchronize()
    p.pool.kv_write(DEC, 1, 0, 60, tk, tv)
    p.ctx.phase_sync(DEC)
    p.note(1, 0, k[:45], v[:45])
    for n in (45, 33, 32, 1):
        q = normal(rng, 1, 8, 128)
        _check_decode(p, [1], [n], q, 128 ** -0.5, _decode(p, [1], [n], q, 128 ** -0.5))
    p.close()


@pytest.mark.parametrize("Hkv, D, P", [(2, 128, 16), (8, 64, 32)])
@pytest.mark.parametrize("noalloc", [False, True])
def test_decode_with_append(Hkv, D, P, noalloc):
    """Forty iterations: blocks and pages begin and end on the way, scales grow."""
    p = Pool8(Hkv, D, P)
    rng = np.random.default_rng(D + P)
    H, lens, ids = 4 * Hkv, [0, 1, 14, 31, 100], [5, 6, 7, 8, 9]
    for rid, n in zip(ids, lens):
        if n:
            p.write(rid, 0, *_rows(rng, n, Hkv, D))
    for it in range(40):
        lens = [n + 1 for n in lens]
        k, v = _rows(rng, len(ids), Hkv, D, spread=4)
        q = normal(rng, len(ids), H, D)
        got = _decode(p, ids, lens, q, D ** -0.5, k, v, noalloc=noalloc)
        for i, (rid, n) in enumerate(zip(ids, lens)):
            p.note(rid, n - 1, k[i:i + 1], v[i:i + 1])
        _check_decode(p, ids, lens, q, D ** -0.5, got, f"iteration {it}")
        if it % 13 == 0 or it == 39:
            for rid in ids:
                p.assert_rows(rid)
    # the same token at the same place again: nothing changes
    before = [p.gather(rid, n) for rid, n in zip(ids, lens)]
    again = _decode(p, ids, lens, q, D ** -0.5, k, v, noalloc=noalloc)
    assert np.array_equal(again, got)
    for rid, n, b in zip(ids, lens, before):
        assert all(np.array_equal(x, y) for x, y in zip(p.gather(rid, n), b))
    p.close()


def _rope_rows(ctx, cfg, rows, positions):
    """rows [n, heads, D] as spd_rope_qk turns them"""
    t = bf16_tensor(rows)
    torch.cuda.synchronize()
    ctx.rope_qk(DEC, cfg, positions, t, rows.shape[1], None, 0, rows.shape[2])
    ctx.phase_sync(DEC)
    return t.double().cpu().numpy()


ROPES = [dict(rotary_dim=128), dict(rotary_dim=64, rotary_offset=24), dict(rotary_dim=96, interleaved=True), dict(rotary_dim=128, factor=8.0)]


@pytest.mark.parametrize("rope", ROPES)
@pytest.mark.parametrize("many", [False, True])
def test_decode_rotates_and_appends(rope, many):
    """RoPE inside the step, by the attention launch and (many short contexts on a small share) by the launch ahead of it."""
    H, Hkv, D = 16, 4, 128
    ctx = S.Context(0)
    if many:
        total = ctx.device_info()[0]
        ctx.set_partition(total - 32, 32)
    p = Pool8(Hkv, D, pages=1200, ctx=ctx)
    cfg = S.rope_config(**rope)
    rng = np.random.default_rng(rope["rotary_dim"] + many)
    lens = [int(n) for n in rng.integers(1, 50, 300)] if many else [1, 5, 16, 17, 33, 300]
    ids = list(range(10, 10 + len(lens)))
    for rid, n in zip(ids, lens):
        if n > 1:
            p.write(rid, 0, *_rows(rng, n - 1, Hkv, D))
    k, v = _rows(rng, len(ids), Hkv, D, spread=3)
    q = normal(rng, len(ids), H, D)
    got = _decode(p, ids, lens, q, D ** -0.5, k, v, rope=cfg)
    pos = [n - 1 for n in lens]
    qr, kr = _rope_rows(ctx, cfg, q, pos), _rope_rows(ctx, cfg, k, pos)
    for i, (rid, n) in enumerate(zip(ids, lens)):
        p.note(rid, n - 1, kr[i:i + 1], v[i:i + 1])
    _check_decode(p, ids, lens, qr, D ** -0.5, got)
    for rid in ids[::17] if many else ids:
        p.assert_rows(rid)
    assert np.array_equal(_decode(p, ids, lens, q, D ** -0.5, k, v, rope=cfg, noalloc=True), got)
    p.close()
    ctx.close()


@pytest.mark.parametrize("cus", [32, 128, 256])
@pytest.mark.parametrize("lens", [[9000], [4500, 130, 2300], [700] * 24])
def test_long_contexts_are_split_and_merged(cus, lens):
    H, Hkv, D = 8, 2, 128
    ctx = S.Context(0)
    total = ctx.device_info()[0]
    ctx.set_partition(total if cus == total else total - cus, cus)
    p = Pool8(Hkv, D, pages=1500, ctx=ctx)
    rng = np.random.default_rng(cus + len(lens))
    ids = list(range(len(lens)))
    for rid, n in zip(ids, lens):
        p.write(rid, 0, *_rows(rng, n - 1, Hkv, D))
    k, v = _rows(rng, len(ids), Hkv, D)
    q = normal(rng, len(ids), H, D)
    got = _decode(p, ids, lens, q, D ** -0.5, k, v)
    for i, (rid, n) in enumerate(zip(ids, lens)):
        p.note(rid, n - 1, k[i:i + 1], v[i:i + 1])
    pick = ids[::7]
    _check_decode(p, pick, [lens[i] for i in pick], q[pick], D ** -0.5, got[pick])
    p.close()
    ctx.close()


def test_scores_that_climb_along_the_context():
    """Keys whose scores rise by hundreds: earlier weights vanish, nothing overflows."""
    p = Pool8(1, 128)
    rng = np.random.default_rng(8)
    n = 700
    k, v = _rows(rng, n, 1, 128, spread=0)
    k += np.rint(np.linspace(-40, 40, n))[:, None, None]
    k, q = mx.to_bf16(k), mx.to_bf16(np.abs(rng.normal(size=(1, 4, 128))))
    p.write(1, 0, k, v)
    _check_decode(p, [1], [n], q, 0.2, _decode(p, [1], [n], q, 0.2))
    p.close()


# ----------------------------------------------------------------------------------------- prefill
def _prefill(p, ids, lens, prefixes, H, rng, rope=None, spread=1.0):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    q = normal(rng, cu[-1], H, p.D)
    k, v = _rows(rng, cu[-1], p.Hkv, p.D, spread=spread)
    tq, tk, tv = bf16_tensor(q), bf16_tensor(k), bf16_tensor(v)
    out = torch.full((cu[-1] + 1, H, p.D), 7.0, dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    p.pool.prefill_step(ids, cu, tq, tk, tv, out, H, p.Hkv, p.D, p.D, p.D ** -0.5, prefix_lens=prefixes, rope=rope)
    p.ctx.phase_sync(PRE)
    assert (out[cu[-1]] == 7.0).all()
    pos = [pre + i for n, pre in zip(lens, prefixes or [0] * len(lens)) for i in range(n)]
    if rope is not None:
        q, k = _rope_rows(p.ctx, rope, q, pos), _rope_rows(p.ctx, rope, k, pos)
    for t, x in ((tq, q), (tk, k), (tv, v)):
        assert np.array_equal(t.double().cpu().numpy(), x)
    got = out[:cu[-1]].double().cpu().numpy()
    for r, (rid, n, pre) in enumerate(zip(ids, lens, prefixes or [0] * len(lens))):
        a, b = cu[r], cu[r + 1]
        kk, vv = k[a:b], v[a:b]
        if pre:
            kk, vv = np.concatenate([p.k[rid].rows[:pre], kk]), np.concatenate([p.v[rid].rows[:pre], vv])
        assert_close(got[a:b], attention(q[a:b], kk, vv, p.D ** -0.5, first=pre), f"request {r}: {n} rows behind {pre}")
        p.note(rid, pre, k[a:b], v[a:b])
        p.assert_rows(rid, PRE)
    return got


@pytest.mark.parametrize("H, Hkv, D, P", [(8, 8, 64, 16), (32, 8, 128, 16), (6, 2, 128, 32), (4, 1, 64, 16)])
@pytest.mark.parametrize("rope", [None, dict(), dict(interleaved=True)])
def test_prefill_and_chunks(H, Hkv, D, P, rope):
    """Whole prompts, then their next pieces, whose prefixes end inside blocks, at blocks' ends and at nothing; then a decode step over what the
    prefill phase wrote."""
    p = Pool8(Hkv, D, P, pages=600)
    cfg = None if rope is None else S.rope_config(rotary_dim=D, **rope)
    rng = np.random.default_rng(H * D + P)
    _prefill(p, [1, 2, 3, 4], [1, 37, 160, 300], None, H, rng, cfg)
    _prefill(p, [1, 2, 3, 4, 5], [1, 100, 16, 77, 50], [1, 37, 160, 300, 0], H, rng, cfg)
    _prefill(p, [5, 1, 3], [3, 140, 1], [50, 2, 176], H, rng, cfg, spread=4)
    p.ctx.phase_wait_for(DEC, PRE)
    ids, lens = [1, 2, 3, 4, 5], [142, 137, 177, 377, 53]
    q = normal(rng, 5, H, D)
    _check_decode(p, ids, lens, q, D ** -0.5, _decode(p, ids, lens, q, D ** -0.5))
    p.close()


def test_a_piece_over_what_was_decoded_and_a_piece_again():
    """Pieces, decode iterations and pieces in turn on one request; a piece given again from an earlier position replaces what lay there."""
    p = Pool8(2, 128)
    rng = np.random.default_rng(11)
    _prefill(p, [1], [90], None, 8, rng)
    n = 90
    for _ in range(9):
        n += 1
        k, v = _rows(rng, 1, 2, 128, spread=4)
        _decode(p, [1], [n], normal(rng, 1, 8, 128), 128 ** -0.5, k, v)
        p.note(1, n - 1, k, v)
    _prefill(p, [1], [30], [99], 8, rng)
    _prefill(p, [1], [10], [70], 8, rng)
    assert len(p.k[1].rows) == 80
    q = normal(rng, 1, 8, 128)
    _check_decode(p, [1], [80], q, 128 ** -0.5, _decode(p, [1], [80], q, 128 ** -0.5))
    p.close()


def test_whole_prompts_are_what_a_bf16_pool_gives():
    """Attention over a step's own rows does not go through the pages: the same bits."""
    H, Hkv, D, lens = 32, 8, 128, [300, 1, 77]
    rng = np.random.default_rng(12)
    T = sum(lens)
    q, (k, v) = normal(rng, T, H, D), _rows(rng, T, Hkv, D)
    cu = np.cumsum([0] + lens).tolist()
    outs = []
    for kind in (S.SPD_KV_GQA, S.SPD_KV_GQA_FP8):
        ctx = S.Context(0)
        nbytes = S.pool_bytes(kind, 16, Hkv, D, D, 64)
        pool = S.Pool(ctx, torch.empty(nbytes, dtype=torch.uint8, device=DEV), nbytes, kind, 16, Hkv, D, D, 64)
        out = torch.empty(T, H, D, dtype=torch.bfloat16, device=DEV)
        tq, tk, tv = bf16_tensor(q), bf16_tensor(k), bf16_tensor(v)
        torch.cuda.synchronize()
        pool.prefill_step([1, 2, 3], cu, tq, tk, tv, out, H, Hkv, D, D, D ** -0.5, rope=S.rope_config(rotary_dim=D))
        ctx.phase_sync(PRE)
        outs.append((out, tq, tk))
        pool.close()
        ctx.close()
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("Hkv, D", [(8, 128), (9, 64)])
def test_two_heads_per_wave_and_a_piece_that_begins_inside_a_block(Hkv, D):
    """More tiles than a small share has workgroups for, so that a wave takes two heads in turn: rows ahead of the piece are re-coded and, behind a
    cached prefix, handed out by both."""
    ctx = S.Context(0)
    total = ctx.device_info()[0]
    p = Pool8(Hkv, D, pages=400, ctx=ctx)
    rng = np.random.default_rng(Hkv)
    ctx.set_partition(total - 32, 32)
    for rid, kept, grow in ((1, 7, 2.0 ** 6), (2, 15, 2.0 ** -9), (3, 1, 2.0 ** 40)):
        p.write(rid, 0, *_rows(rng, kept, Hkv, D))
        p.write(rid, kept, *(r * grow for r in _rows(rng, 1100, Hkv, D)))
        p.assert_rows(rid)
    ctx.set_partition(32, total - 32)
    _prefill(p, [4, 5], [39, 30], None, Hkv, rng)
    _prefill(p, [4, 5], [1100, 70], [39, 30], Hkv, rng, spread=4)
    _prefill(p, [4], [1050], [1139], Hkv, rng, S.rope_config(rotary_dim=D))
    p.close()
    ctx.close()


# ----------------------------------------------------------------------------------------- large pools, graphs, both phases
def test_a_waves_pages_change_windows():
    """Chunks of more than 256 tiles, whose page numbers a wave holds in several goes; every number of steps behind the first 32, to the pipeline's depth."""
    H, Hkv, D = 32, 32, 64
    ctx = S.Context(0)
    ctx.set_partition(ctx.device_info()[0] - 32, 32)
    p = Pool8(Hkv, D, P=48, pages=900, ctx=ctx)
    rng = np.random.default_rng(16)
    lens = [4097, 4225, 4353, 4500, 8200, 9000]
    for rid, n in enumerate(lens):
        p.write(rid, 0, *_rows(rng, n - 1, Hkv, D))
    for rid, n in enumerate(lens):
        k, v = _rows(rng, 1, Hkv, D)
        q = normal(rng, 1, H, D)
        got = _decode(p, [rid], [n], q, D ** -0.5, k, v)
        p.note(rid, n - 1, k, v)
        _check_decode(p, [rid], [n], q, D ** -0.5, got)
    p.close()
    ctx.close()


def test_rows_beyond_4gib():
    """A prefix whose bf16 rows take more than 4 GiB for the keys: written, gathered, and attended to by a piece that begins inside a block."""
    H, Hkv, D, n, m = 8, 8, 128, 2 ** 21 + 1003, 5
    ctx = S.Context(0)
    nbytes = S.pool_bytes(S.SPD_KV_GQA_FP8, 1024, Hkv, D, D, 2051)
    mem = torch.full((nbytes,), 0xFF, dtype=torch.uint8, device=DEV)
    pool = S.Pool(ctx, mem, nbytes, S.SPD_KV_GQA_FP8, 1024, Hkv, D, D, 2051)
    gen = torch.Generator(device=DEV).manual_seed(17)
    k, v = (torch.empty(n, Hkv, D, dtype=torch.bfloat16, device=DEV).normal_(generator=gen) for _ in range(2))
    pool.kv_reserve(1, n)
    torch.cuda.synchronize()
    pool.kv_write(PRE, 1, 0, n, k, v)
    ctx.phase_sync(PRE)
    rows = [torch.zeros_like(k) for _ in range(2)]
    torch.cuda.synchronize()
    pool.kv_gather(PRE, 1, n, *rows)
    ctx.phase_sync(PRE)
    for got, given in zip(rows, (k, v)):
        for begin, end in ((0, 40), (n - n % 16 - 32, n)):
            cache = mx.Cache8(Hkv, D)
            cache.write(0, given[begin:end].double().cpu().numpy())
            np.testing.assert_array_equal(got[begin:end].double().cpu().numpy(), cache.rows)
    del k, v
    rng = np.random.default_rng(18)
    q, kn, vn = normal(rng, m, H, D), *_rows(rng, m, Hkv, D)
    tq, tk, tv = (bf16_tensor(t) for t in (q, kn, vn))
    out = torch.zeros(m, H, D, dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    pool.prefill_step([1], [0, m], tq, tk, tv, out, H, Hkv, D, D, D ** -0.5, prefix_lens=[n])
    ctx.phase_sync(PRE)
    got = out.double().cpu().numpy()
    hide = torch.arange(n + m, device=DEV)[None] > n + torch.arange(m, device=DEV)[:, None]
    for h in range(H):                                   # `attention`, on the GPU
        kk, vv = (torch.cat([r[:, h], t[:, h]]).double() for r, t in zip(rows, (tk, tv)))
        qh = tq[:, h].double()
        s = D ** -0.5 * qh @ kk.T.contiguous()
        s[hide] = -torch.inf
        weights = torch.softmax(s, -1)
        mag = (D ** -0.5 * qh.abs() @ kk.abs().T.contiguous()).amax(-1, keepdim=True)
        want, A = weights @ vv, weights @ vv.abs()
        bar = (2.0 ** -7 + 2.0 ** -15 * mag) * A + 2.0 ** -8 * want.abs()
        assert_close(got[:, h], (want.cpu().numpy(), bar.cpu().numpy()), f"head {h}")
    pool.close()
    ctx.close()


def test_pages_beyond_4gib():
    Hkv, D, P = 8, 128, 16
    page_bytes = S.pool_bytes(S.SPD_KV_GQA_FP8, P, Hkv, D, D, 1)
    low = -(-(1 << 32) // page_bytes)
    p = Pool8(Hkv, D, P, pages=low + 200)
    p.pool.kv_reserve(99, low * P)                       # holds every page that begins below 4 GiB
    rng = np.random.default_rng(13)
    _prefill(p, [1, 2], [130, 33], None, 8, rng)
    _prefill(p, [1, 2], [20, 60], [130, 33], 8, rng)
    assert min(p.pool.kv_block_table(1) + p.pool.kv_block_table(2)) >= low
    lens = [151, 94]
    k, v = _rows(rng, 2, Hkv, D)
    q = normal(rng, 2, 8, D)
    p.ctx.phase_wait_for(DEC, PRE)
    got = _decode(p, [1, 2], lens, q, D ** -0.5, k, v)
    for i in range(2):
        p.note(i + 1, lens[i] - 1, k[i:i + 1], v[i:i + 1])
        p.assert_rows(i + 1)
    _check_decode(p, [1, 2], lens, q, D ** -0.5, got)
    p.close()


def test_captured_and_replayed():
    """A decode step without allocation in a graph: every replay appends and attends to what is there by then; chunked prefill is refused."""
    p = Pool8(2, 128)
    rng = np.random.default_rng(14)
    lens, ids = [40, 300], [1, 2]
    for rid, n in zip(ids, lens):
        p.write(rid, 0, *_rows(rng, n - 1, 2, 128))
    q, k, v = (torch.empty(2, h, 128, dtype=torch.bfloat16, device=DEV) for h in (8, 2, 2))
    out = torch.empty_like(q)
    batch = p.pool.make_decode_batch(ids, lens, q, out, 8, 128 ** -0.5, k, v)
    stream = torch.cuda.ExternalStream(p.ctx.phase_stream(DEC))
    graph = torch.cuda.CUDAGraph()
    p.ctx.phase_sync(DEC)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        p.pool.decode_step_noalloc_batch(batch)
    for it in range(4):
        qn, (kn, vn) = normal(rng, 2, 8, 128), _rows(rng, 2, 2, 128, spread=3)
        for t, x in ((q, qn), (k, kn), (v, vn)):
            t.copy_(bf16_tensor(x))
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, rid in enumerate(ids):
            p.note(rid, lens[i] - 1, kn[i:i + 1], vn[i:i + 1])
            p.assert_rows(rid)
        _check_decode(p, ids, lens, qn, 128 ** -0.5, out.double().cpu().numpy(), f"replay {it}")
    tables = [p.pool.kv_block_table(r) for r in ids], p.pool.stats()
    pre = torch.cuda.ExternalStream(p.ctx.phase_stream(PRE))
    other = torch.cuda.CUDAGraph()
    p.ctx.phase_sync(PRE)
    rows = torch.zeros(4, 2, 128, dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.graph(other, stream=pre):
        with pytest.raises(S.SpdError) as e:
            p.pool.prefill_step([1], [0, 4], rows, rows, rows, rows, 2, 2, 128, 128, 1.0, prefix_lens=[40])
        p.ctx.rmsnorm(PRE, rows, None, q, 1e-5, rows, 1, 256)                   # (a graph wants a node)
    assert e.value.status == S.SPD_ESTATE
    assert ([p.pool.kv_block_table(r) for r in ids], p.pool.stats()) == tables
    torch.cuda.synchronize()
    p.close()


def test_both_phases_at_once():
    """A chunked step on one half of the chip while decode iterations run on the other: what each gives alone."""
    H, Hkv, D = 16, 4, 128
    ctx = S.Context(0)
    total = ctx.device_info()[0]
    ctx.set_partition(total // 2, total // 2)
    p = Pool8(Hkv, D, pages=1200, ctx=ctx)
    rng = np.random.default_rng(15)
    _prefill(p, [1, 2], [500, 333], None, H, rng)
    lens, ids = [600, 37, 1200], [11, 12, 13]
    for rid, n in zip(ids, lens):
        p.write(rid, 0, *_rows(rng, n, Hkv, D))
    q = normal(rng, 3, H, D)
    tq, out = bf16_tensor(q), torch.empty(3, H, D, dtype=torch.bfloat16, device=DEV)
    worker = p.pool.decode_worker_start([p.pool.make_decode_batch(ids, lens, tq, out, H, D ** -0.5)])
    try:
        _prefill(p, [1, 2], [200, 150], [500, 333], H, rng)
    finally:
        p.pool.decode_worker_stop(worker)
    ctx.phase_sync(DEC)
    _check_decode(p, ids, lens, q, D ** -0.5, out.double().cpu().numpy())
    p.close()
    ctx.close()
