"""What the norm and the FFN over MXFP4 weights refuse, through the C ABI, no GPU: addresses are never touched."""
import pytest

from paper_2504_19867_amd import semipd as S

A = 4096


@pytest.fixture()
def ctx():
    c = S.Context(-1)
    yield c
    c.close()


def _norm(ctx, phase=1, x=A, r=2 * A, w=3 * A, eps=1e-5, out=4 * A, scales=5 * A, T=4, hidden=256):
    return S.lib.spd_rmsnorm(ctx.h if ctx else None, phase, x, r, w, eps, out, scales, T, hidden)


def test_norm(ctx):
    assert _norm(ctx) == S.SPD_ESTATE and _norm(ctx, r=None) == S.SPD_ESTATE and _norm(ctx, scales=None, hidden=8) == S.SPD_ESTATE
    assert _norm(ctx, out=A, scales=None) == S.SPD_ESTATE                        # in place
    assert _norm(None) == S.SPD_EINVAL
    bad = [dict(phase=2), dict(phase=-1), dict(T=-1), dict(hidden=0), dict(hidden=-128), dict(hidden=200), dict(hidden=12, scales=None), dict(hidden=32896),
           dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=None), dict(w=None), dict(out=None),
           dict(x=A + 8), dict(r=A + 8), dict(w=A + 8), dict(out=A + 8), dict(scales=A + 2), dict(r=A), dict(r=4 * A),
           dict(out=A), dict(out=A + 2032, scales=None), dict(out=A - 16, scales=None), dict(r=A + 2032), dict(r=3 * A - 16), dict(out=2 * A + 16), dict(out=3 * A + 496),
           dict(scales=A), dict(scales=2 * A + 2044), dict(scales=3 * A + 508), dict(scales=4 * A + 1020)]
    for b in bad:
        assert _norm(ctx, **b) == S.SPD_EINVAL, b


def test_ffn(ctx):
    def call(phase=1, x=A, xs=2 * A, w=32 * A, out=4 * A, T=4, hidden=256, inter=128):
        return S.lib.spd_ffn_gate_up_mx(ctx.h, phase, x, xs, w, out, T, hidden, inter)
    assert call() == S.SPD_ESTATE and call(out=4 * A + 2) == S.SPD_ESTATE and call(xs=A + 4) == S.SPD_ESTATE
    assert S.lib.spd_ffn_gate_up_mx(None, 1, A, A, A, A, 4, 256, 128) == S.SPD_EINVAL
    for b in (dict(phase=2), dict(T=-1), dict(hidden=64), dict(hidden=0), dict(inter=64), dict(inter=-128), dict(hidden=1 << 24), dict(x=None), dict(xs=None),
              dict(w=None), dict(out=None), dict(x=A + 8), dict(w=A + 8), dict(xs=A + 2), dict(out=A + 1), dict(out=A), dict(out=A + 1022), dict(out=2 * A - 1022), dict(out=2 * A + 30),
              dict(out=32 * A + 2 * 17408 - 2), dict(out=32 * A - 1022)):
        assert call(**b) == S.SPD_EINVAL, b


def test_pack_and_unpack(ctx):
    gate, up, w = A, 32 * A, 64 * A                                              # 32768, 32768 and 17408 bytes
    for fn, order in ((S.lib.spd_ffn_pack_gate_up_mx, (0, 1, 2)), (S.lib.spd_ffn_unpack_gate_up_mx, (2, 0, 1))):
        def call(gate=gate, up=up, w=w, phase=0, hidden=128, inter=128, h=ctx.h):
            at = (gate, up, w)
            return fn(h, phase, *(at[i] for i in order), hidden, inter)
        assert call() == S.SPD_ESTATE and call(up=gate + 32768) == S.SPD_ESTATE and call(w=up + 32768) == S.SPD_ESTATE
        assert (call(up=gate) == S.SPD_ESTATE) == (order[0] == 0)                # both read, or both written
        for b in (dict(h=None), dict(phase=2), dict(gate=None), dict(up=None), dict(w=None), dict(gate=A + 8), dict(up=A + 8), dict(w=A + 8), dict(hidden=96),
                  dict(inter=192), dict(hidden=0), dict(w=gate + 32752), dict(w=up), dict(w=up - 17392)):
            assert call(**b) == S.SPD_EINVAL, b


def test_bytes():
    assert S.ffn_mx_bytes(128, 128) == 17408 and S.ffn_mx_bytes(4096, 14336) == 2 * 4096 * 14336 * 17 // 32
    for hidden, inter in ((0, 128), (128, 0), (130, 128), (128, 130), (-128, 128)):
        with pytest.raises(S.SpdError):
            S.ffn_mx_bytes(hidden, inter)
    assert S.lib.spd_ffn_mx_bytes(128, 128, None) == S.SPD_EINVAL


def test_no_rows_overlap_nothing(ctx):
    """Without tokens an output of no bytes may point anywhere, into the weights too."""
    assert S.lib.spd_rmsnorm(ctx.h, 1, A, None, 3 * A, 1e-5, 3 * A + 16, None, 0, 256) == S.SPD_ESTATE
    assert S.lib.spd_rmsnorm(ctx.h, 1, A, 3 * A + 32, 3 * A, 1e-5, 4 * A, 3 * A + 16, 0, 256) == S.SPD_ESTATE
    assert S.lib.spd_ffn_gate_up_mx(ctx.h, 1, A, A, 2 * A, 2 * A + 16, 0, 256, 128) == S.SPD_ESTATE
