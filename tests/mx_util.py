"""Helpers of the tests of 8- and 4-bit forms: values of codes and scales, and the bars."""
import numpy as np
import torch

from oracle import mx
from gpu_util import DEV

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def bf16_tensor(values: np.ndarray) -> torch.Tensor:
    """fp64 values that bf16 holds exactly, on the GPU"""
    t = torch.from_numpy(np.ascontiguousarray(values)).to(torch.bfloat16)
    assert np.array_equal(t.double().numpy(), values, equal_nan=True)
    return t.to(DEV)


def normal(rng, *shape, spread: float = 0.0) -> np.ndarray:
    """bf16 values N(0, 1), each row times a power of two up to 2^+-spread"""
    x = mx.to_bf16(rng.normal(size=shape))
    return x * np.exp2(np.rint(rng.uniform(-spread, spread, shape[:-1] + (1,))))


def mx_values(codes: torch.Tensor, scales: torch.Tensor, T: int, hidden: int):
    """(values [T, hidden], scale bytes [T, hidden / 32]) of E4M3 codes and their [hidden / 128][T][4] scale bytes"""
    b = scales.cpu().view(torch.uint8).numpy().reshape(hidden // 128, T, 4).transpose(1, 0, 2).reshape(T, hidden // 32).astype(np.int64)
    v = codes.cpu().view(E4M3).double().numpy().reshape(T, hidden // 32, 32) * np.exp2(b - 127.0)[..., None]
    return v.reshape(T, hidden), b


def mx_tensors(values: np.ndarray, b: np.ndarray):
    """codes and scales as the library takes them, of values [T, hidden] that E4M3 holds exactly under the bytes b [T, hidden / 32]"""
    T, hidden = values.shape
    y = (values.reshape(T, -1, 32) / np.exp2(b - 127.0)[..., None]).reshape(T, hidden)
    codes = torch.from_numpy(y).float().to(E4M3)
    assert np.array_equal(codes.double().numpy(), y, equal_nan=True)
    scales = torch.from_numpy(np.ascontiguousarray(b.astype(np.uint8).reshape(T, hidden // 128, 4).transpose(1, 0, 2)))
    return codes.to(DEV), scales.to(DEV)


def assert_quantised(got: np.ndarray, b: np.ndarray, y: np.ndarray, delta: float):
    """`got` and its scale bytes are a quantisation of y known to a relative delta: the scale that y (1 +- delta) asks for, and
    codes between those of y (1 - delta) and y (1 + delta)."""
    blocks = y.reshape(y.shape[0], -1, 32)
    amax = np.abs(blocks).max(-1)
    lo, hi = mx.scale_byte(amax * (1 - delta), mx.E4M3), mx.scale_byte(amax * (1 + delta), mx.E4M3)
    assert ((b >= lo) & (b <= hi)).all(), (b - lo).min()
    s = np.exp2(b - 127.0)[..., None]
    ends = [mx.nearest(np.clip(np.abs(blocks) * (1 + d) / s, 0, 448), mx.E4M3) * s for d in (-delta, delta)]
    g = got.reshape(blocks.shape)
    assert ((np.abs(g) >= ends[0]) & (np.abs(g) <= ends[1]) & ((g == 0) | (np.sign(g) == np.sign(blocks)))).all()
