"""Plain 64-bit references of 8-bit floating point weights: quantisation with a scale for every 128 x 128, the integers of codes (numpy only)."""
import numpy as np

from experts_ref import w8_unpack

# magnitudes of the codes 0 .. 126 (e4m3), 127 is not a number
E4M3 = np.array([m / 512 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127])
LARGEST = 3.4028234663852886e38


def blocks(n):
    return -(-n // 128)


def spread(scales, M, K):
    """a scale for every weight"""
    return np.repeat(np.repeat(scales, 128, -2)[..., :M, :], 128, -1)[..., :K]


def quantise(w, base, max_scale):
    """w float64 [experts][out_c][K] -> (codes, scales [E][ceil(out_c / 128)][ceil(K / 128)], the values they stand for)"""
    w = np.where(np.isnan(w), 0.0, np.clip(w, -LARGEST, LARGEST))
    E, M, K = w.shape
    wp = np.zeros((E, blocks(M) * 128, blocks(K) * 128))
    wp[:, :M, :K] = np.abs(w)
    a = wp.reshape(E, blocks(M), 128, blocks(K), 128).max((2, 4))
    S = np.clip(np.ceil(a / (448 * 2.0 ** base)), 1, max_scale).astype(np.int64)
    unit = spread(S, M, K) * 2.0 ** base
    q = np.minimum(np.abs(w) / unit, 448.0)
    code = np.zeros(q.shape, np.int64)
    mid = (E4M3[1:] + E4M3[:-1]) / 2
    lo = np.searchsorted(mid, q)                       # mid[lo - 1] < q <= mid[lo]
    tie = (lo < 126) & (q == mid[np.minimum(lo, 125)])
    code = lo + (tie & (lo % 2 == 1))                  # from an odd code up to the even one
    sign = np.signbit(w) & (code > 0)
    return code + 128 * sign, S, np.where(sign, -1, 1) * E4M3[code] * unit


def integers(codes, scales):
    """512 e4m3 S as Python integers (an object array); codes that are no numbers: 0"""
    mag = np.array([int(512 * v) for v in E4M3] + [0], object)
    E, M, K = codes.shape
    return mag[codes & 127] * np.where(codes & 128, -1, 1) * spread(scales, M, K).astype(object)


def unpack(buf, E, M, K):
    """prepared buffer (uint8) -> (codes [E][M][K], scales, everything else zero)"""
    tiles, n = -(-M // 32) * -(-K // 64) * 2048, blocks(M) * blocks(K)
    buf = buf.reshape(E, -1)
    assert buf.shape[1] == tiles + -(-4 * n // 16) * 16
    codes = w8_unpack(np.ascontiguousarray(buf[:, :tiles]).reshape(-1), E, M, K).view(np.uint8).astype(np.int64)
    rest = codes.copy()
    rest[:, :M, :K] = 0
    scales = np.ascontiguousarray(buf[:, tiles:tiles + 4 * n]).view(np.int32).astype(np.int64).reshape(E, blocks(M), blocks(K))
    return codes[:, :M, :K], scales, not rest.any()
