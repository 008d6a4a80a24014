"""Plain 64-bit references of the operators around the linear layers, and the 8-bit copy's format written out in numpy."""
import math

import numpy as np
import torch

from paper_2509_25149_b200 import binding as B

ACTS = {"none": B.ACT_NONE, "relu2": B.ACT_RELU2, "silu": B.ACT_SILU, "gelu": B.ACT_GELU}


def f64(t):
    return t.detach().cpu().double().numpy()


def e4m3_value(code):
    s, e, m = code >> 7, (code >> 3) & 15, code & 7
    v = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
    return -v if s else v


E4M3 = np.array([e4m3_value(c) if (c & 127) != 127 else np.nan for c in range(256)])
GRID = E4M3[:127]  # 0 .. 448, ascending


def nearest_codes(v):
    """E4M3 codes of values within +-448, to nearest, ties to the even code."""
    a = np.abs(v)
    hi = np.clip(np.searchsorted(GRID, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = GRID[hi] - a, a - GRID[lo]
    code = np.where(up < down, hi, np.where(up > down, lo, np.where(hi % 2 == 0, hi, lo)))
    return (code + np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def scale_exponent(amax):
    """Smallest E >= -127 with amax <= 448 * 2^E (comparisons of binary64 numbers only)."""
    E = np.full(amax.shape, -127, dtype=np.int64)
    for e in range(-126, 129):
        E = np.where(amax > 448.0 * 2.0 ** (e - 1), e, E)
    return E


def copy8(x):
    """codes [rows, cols], scale bytes [rows, blocks] of a float64 array."""
    rows, cols = x.shape
    nb = (cols + 31) // 32
    p = np.zeros((rows, nb * 32))
    p[:, :cols] = x
    b = p.reshape(rows, nb, 32)
    E = scale_exponent(np.abs(b).max(2))
    codes = nearest_codes(b / 2.0 ** E[:, :, None].astype(np.float64)).reshape(rows, nb * 32)[:, :cols]
    return codes, (E + 127).astype(np.uint8)


def decode8(codes, scales):
    s = 2.0 ** (scales.astype(np.float64) - 127)
    return E4M3[codes] * np.repeat(s, 32, axis=1)[:, :codes.shape[1]]


def copy_on_gpu(x):
    """An MXFP8 copy of a float64 array, made here."""
    codes, scales = copy8(x)
    t = B.alloc_tensor(x.shape[0], x.shape[1], format=B.FORMAT_MXFP8)
    t.codes.copy_(torch.from_numpy(codes))
    t.scales.copy_(torch.from_numpy(scales))
    return t


def act64(z, act):
    with np.errstate(over="ignore"):
        if act == "relu2":
            return np.maximum(z, 0) ** 2
        if act == "silu":
            return z / (1 + np.exp(-z))
        if act == "gelu":
            return z / (1 + np.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def slope64(z, act):
    with np.errstate(over="ignore"):
        if act == "relu2":
            return 2 * np.maximum(z, 0)
        if act == "silu":
            s = 1 / (1 + np.exp(-z))
            return s + z * s * (1 - s)
        if act == "gelu":
            k = 2 * math.sqrt(2 / math.pi)
            s = 1 / (1 + np.exp(-k * (z + 0.044715 * z ** 3)))
            return s + z * s * (1 - s) * k * (1 + 3 * 0.044715 * z * z)
    return np.ones_like(z)


def guarded(rows, cols, dtype, ld=None, fill=None):
    """A [rows x cols] view into a larger buffer, 16-byte aligned, rows `ld` apart; and a check that the rest is untouched."""
    ld = cols if ld is None else ld
    unit = 16 // torch.empty(0, dtype=dtype).element_size()
    mark = 77 if not dtype.is_floating_point else 77.0
    flat = torch.full((unit + rows * ld + 64,), mark, dtype=dtype, device="cuda")
    view = flat[unit:unit + rows * ld].view(rows, ld)[:, :cols]
    inside = torch.zeros_like(flat, dtype=torch.bool)
    inside[unit:unit + rows * ld].view(rows, ld)[:, :cols] = True
    if fill is not None:
        view.copy_(fill)
    return view, lambda: bool((flat[~inside] == mark).all())


def guarded_copy(rows, cols):
    codes, a = guarded(rows, cols, torch.uint8)
    nb = (cols + 31) // 32
    scales, b = guarded(rows, nb, torch.uint8)
    return B.NVFP4Tensor(codes, scales, None, rows, cols, B.SF_LINEAR, B.FORMAT_MXFP8), lambda: a() and b()


def assert_within(got, want, tol, what):
    err = np.abs(got - want)
    bad = ~(err <= tol)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(bad, err / np.maximum(tol, 1e-300), -1)), err.shape)
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} off, worst at {i}: got {got[i]}, want {want[i]}, tolerance {tol[i] if np.ndim(tol) else tol}")
