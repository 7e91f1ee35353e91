"""GQA pools in 8 bits through the C ABI, no GPU: geometry, allocation, what is refused."""
import pytest

from paper_2504_19867_amd import semipd as S

A = 4096


def test_bytes():
    # 16 tokens x 8 heads x 2 x 128 codes, 8 x 2 scales in a line of 128 bytes
    assert S.pool_bytes(S.SPD_KV_GQA_FP8, 16, 8, 128, 128, 10) == 10 * (32768 + 128)
    assert S.pool_bytes(S.SPD_KV_GQA_FP8, 64, 3, 64, 64, 1) == 64 * 3 * 128 + 128
    assert S.pool_bytes(S.SPD_KV_GQA_FP8, 1024, 2, 64, 64, 1) == 1024 * 2 * 128 + 256
    for bad in ((15, 8, 128, 128, 4), (16, 8, 96, 96, 4), (16, 8, 128, 64, 4), (16, 0, 128, 128, 4), (16, 8, 128, 128, 0), (2048, 8, 128, 128, 4)):
        with pytest.raises(S.SpdError):
            S.pool_bytes(S.SPD_KV_GQA_FP8, *bad)
    with pytest.raises(S.SpdError):
        S.pool_bytes(4, 16, 8, 128, 128, 4)


def test_host_only_pool():
    ctx = S.Context(-1)
    pool = S.Pool(ctx, None, 0, S.SPD_KV_GQA_FP8, 16, 2, 64, 64, 8)
    pool.kv_reserve(1, 40)
    assert pool.kv_block_table(1) == [0, 1, 2] and pool.stats()[:3] == (8, 5, 1)

    def status(fn, *args, **kw):
        with pytest.raises(S.SpdError) as e:
            fn(*args, **kw)
        return e.value.status
    assert status(pool.kv_write, 1, 1, 0, 4, A, None) == S.SPD_EINVAL                 # values are wanted
    assert status(pool.kv_write, 1, 1, 0, 4, A, A + 8) == S.SPD_EINVAL
    assert status(pool.kv_write, 1, 1, -1, 4, A, A) == S.SPD_EINVAL
    assert status(pool.kv_write, 1, 1, 0, 4, A, A) == S.SPD_ESTATE                    # no GPU
    assert status(pool.kv_gather, 1, 1, 4, A, A) == S.SPD_ESTATE
    step = dict(n_q_heads=4, n_kv_heads=2, dim_qk=64, dim_v=64, scale=1.0)
    assert status(pool.prefill_step, [1], [0, 4], A, A, A, A, **step) == S.SPD_ESTATE
    assert status(pool.prefill_step, [1], [0, 4], A, A, A, A, **step, prefix_lens=[-1]) in (S.SPD_EINVAL, S.SPD_ESTATE)
    assert status(pool.prefill_step, [1], [0, 4], A, A, A, A, **step, latent=A) == S.SPD_EINVAL
    assert status(pool.prefill_step, [1], [0, 4], A, A, A, A, **dict(step, dim_qk=128)) == S.SPD_EINVAL
    assert status(pool.prefill_step, [1], [0, 4], A, A, A, A, **step, rope=S.rope_config(rotary_dim=128)) == S.SPD_EINVAL
    assert status(pool.decode_step, [1], [4], A, A, 4, 1.0) == S.SPD_ESTATE
    assert status(pool.decode_step, [1], [4], A, A, 4, 1.0, k_new=A) == S.SPD_EINVAL
    assert status(pool.decode_step, [1], [4], A, A, 34, 1.0) == S.SPD_EINVAL          # 17 heads per KV head
    assert status(pool.decode_step, [1, 1], [4, 4], A, A, 4, 1.0, k_new=A, v_new=A) == S.SPD_EINVAL
    pool.kv_free(1)
    pool.close()
    ctx.close()
