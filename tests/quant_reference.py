"""Plain fp64 counterparts of the 4-bit matrices: rounding to them, their values, products with them."""
import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
VALUES = np.concatenate([E2M1, -E2M1])
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def bf16(x):
    """x (fp32) rounded to bf16, ties to even; NaN stays."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return np.where(np.isnan(x), np.float32(np.nan), (((u + 0x7FFF + (u >> 16 & 1)) >> 16 << 16) & 0xFFFFFFFF).astype(np.uint32).view(np.float32))


def quantize(w, group):
    """(code indexes [N][K], scales [N][groups]) of fp32 weights."""
    w = np.asarray(w, np.float32)
    N, K = w.shape
    groups = -(-K // group)
    codes, scales = np.zeros((N, K), np.uint8), np.zeros((N, groups), np.float32)
    for n in range(N):
        for g in range(groups):
            x = w[n, g * group:(g + 1) * group]
            if not np.isfinite(x).all():
                scales[n, g] = np.nan
                continue
            s = bf16(np.abs(x).max() / np.float32(6))
            scales[n, g] = s
            if s == 0:
                continue
            q = np.abs(x.astype(np.float64)) / float(s)
            best = np.argmin(np.abs(q[:, None] - E2M1) + 1e-9 * (np.arange(8) % 2), 1)      # ties to the even code
            codes[n, g * group:(g + 1) * group] = best + 8 * np.signbit(x)
    return codes, scales


def pack_rows(codes):
    """Two codes a byte, the lower column in the low four bits."""
    N, K = codes.shape
    c = np.zeros((N, K + K % 2), np.uint8)
    c[:, :K] = codes
    return c[:, ::2] | c[:, 1::2] << 4


def values(codes, scales, group):
    return VALUES[codes] * np.repeat(np.asarray(scales, np.float64), group, 1)[:, :codes.shape[1]]


def linear(x, w, group, dtype, y_dtype):
    """(y, tolerance): products are exact; a group's sum has at most `group` terms (thrice as many for an fp32 x) and a
    scaling, then come the groups and the eight waves, each one fp32 operation of at most 2^-23 of what it has summed;
    then the result's rounding."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        y = x @ w.T
        size = np.abs(x) @ np.abs(w.T)
        terms = min(group, x.shape[1]) * (1 if dtype == "bf16" else 3) + 1 + -(-x.shape[1] // group) + 8
        tol = 2.0 ** -23 * terms * size
        return y, tol + HALF_STEP[y_dtype] * (np.abs(y) + tol) + 1e-38
