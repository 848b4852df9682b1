"""Microscaled 4-bit floating point and log probabilities from their definitions, in numpy and 64 bits."""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def blocks_of(k):
    return (k + 31) // 32


def quantize(x):
    """x [M][K] (any float type) -> (codes uint8 [M][16 * blocks], scale bytes uint8 [M][blocks])."""
    x = np.asarray(x, np.float64)
    m, k = x.shape
    nb = blocks_of(k)
    b = np.zeros((m, nb * 32))
    b[:, :k] = x
    b = b.reshape(m, nb, 32)
    bad = ~np.isfinite(b).all(axis=2)
    b = np.where(bad[..., None], 0.0, b)
    top = np.abs(b).max(axis=2)
    exponent = np.frexp(top)[1].astype(np.int64) - 1                 # floor(log2)
    byte = np.where(top > 0, np.maximum(exponent + 125, 0), 0)
    q = np.abs(b) * np.exp2(127.0 - byte)[..., None]
    # nearest of the grid; of two as near the even code; beyond 6 it is 6
    dist = np.abs(q[..., None] - GRID) + (np.arange(8) & 1) * 1e-9   # quotients at a tie are exact, others are further apart
    code = np.argmin(dist, axis=-1).astype(np.uint8)
    tie_free = np.sort(np.abs(q[..., None] - GRID), axis=-1)
    assert np.all((tie_free[..., 0] == tie_free[..., 1]) | (tie_free[..., 1] - tie_free[..., 0] > 2e-9) | (q > 6)), "tie margin"
    code |= (np.signbit(b).astype(np.uint8) << 3)
    byte = np.where(bad, 255, byte).astype(np.uint8)
    code = np.where(bad[..., None], 0, code).reshape(m, nb * 16, 2)
    return (code[..., 0] | (code[..., 1] << 4)).astype(np.uint8), byte


def values(codes, scale_bytes, k):
    """What the form stands for, fp64 [M][k]."""
    m = codes.shape[0]
    c = np.stack((codes & 15, codes >> 4), axis=-1).reshape(m, -1)
    v = np.where(c & 8, -1.0, 1.0) * GRID[c & 7]
    s = np.where(scale_bytes == 255, np.nan, np.exp2(scale_bytes.astype(np.float64) - 127))
    return (v.reshape(m, -1, 32) * s[..., None]).reshape(m, -1)[:, :k]


def scale_offsets(m, k):
    """Where the scale of (row, block) is in the tiles: int64 [m][blocks]."""
    r, b = np.arange(m, dtype=np.int64)[:, None], np.arange(blocks_of(k), dtype=np.int64)[None, :]
    return (r // 128 * ((k + 127) // 128) + b // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + b % 4


def tile_scales(scale_bytes, k, fill=0):
    """[m][blocks] bytes -> the tiles as one array; places of no row hold `fill`, blocks behind k hold 0."""
    m = scale_bytes.shape[0]
    kt = (k + 127) // 128
    full = np.zeros((m, kt * 4), np.uint8)
    full[:, :scale_bytes.shape[1]] = scale_bytes
    out = np.full((m + 127) // 128 * 512 * kt, fill, np.uint8)
    out[scale_offsets(m, kt * 128)] = full
    return out


def conv1x1(xv, wv, bias, relu):
    """(y, S): fp64 result of [M][K] x [N][K] values and the sum of the magnitudes that an output's error is measured by."""
    y = xv @ wv.T
    s = np.abs(xv) @ np.abs(wv).T
    if bias is not None:
        y, s = y + np.asarray(bias, np.float64), s + np.abs(np.asarray(bias, np.float64))
    return (np.maximum(y, 0) if relu else y), s


def logprobs(x, targets, top):
    """(log probabilities of targets, entropy, top indexes, their log probabilities), fp64, of rows of logits."""
    x = np.asarray(x, np.float64)
    rows, v = x.shape
    with np.errstate(all="ignore"):
        m = x.max(axis=1, keepdims=True)
        lp = (x - m) - np.log(np.exp(x - m).sum(axis=1, keepdims=True))
        p = np.exp(lp)
        h = -np.where(p == 0, 0.0, p * lp).sum(axis=1)
    t = np.asarray(targets, np.int64).reshape(rows, -1)
    given = np.take_along_axis(lp, np.clip(t, 0, v - 1), axis=1)
    given = np.where(t < 0, 0.0, np.where(t >= v, np.nan, given))
    order = np.argsort(-np.where(np.isnan(x), -np.inf, x), axis=1, kind="stable")[:, :top]
    raw = np.take_along_axis(np.where(np.isnan(x), -np.inf, x), order, axis=1)
    with np.errstate(all="ignore"):
        best = (raw - m) - np.log(np.exp(x - m).sum(axis=1, keepdims=True))    # m + log(sum) would lose the sum next to a huge m
    return given, h, order, best
