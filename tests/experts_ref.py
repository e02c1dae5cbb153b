"""Plain 64-bit references of the expert layers: quantisation to 4-bit floats, products by expert, weighted sums (numpy only)."""
import numpy as np

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def quantise(w, base, max_shift):
    """w float64 [experts][out_c][K] -> (magnitude codes with bit 3 the sign, shift per 32 weights, the values they stand for)"""
    w = np.where(np.isnan(w), 0.0, np.clip(w, -3.4028234663852886e38, 3.4028234663852886e38))
    E, M, K = w.shape
    n = (K + 31) // 32
    wp = np.zeros((E, M, n * 32))
    wp[:, :, :K] = w
    wp = wp.reshape(E, M, n, 32)
    amax = np.abs(wp).max(-1)
    e = np.frexp(amax)[1] - 3                                   # amax = f 2^(e'), f in [1/2, 1)
    e = np.where(amax > 0, e, base)
    e = np.clip(np.clip(e, None, base + max_shift), base, None)
    a = np.abs(wp) / np.exp2(e.astype(np.float64))[..., None]
    mid = (E2M1[1:] + E2M1[:-1]) / 2
    m = np.zeros(a.shape, np.int64)
    for i, t in enumerate(mid):                                 # from code i to i + 1: ties go to the even one
        m += (a > t) | ((a == t) & (i % 2 == 1))
    sign = np.signbit(wp) & (m > 0)
    values = np.where(sign, -1, 1) * E2M1[m] * np.exp2(e.astype(np.float64))[..., None]
    flat = lambda t: t.reshape(E, M, n * 32)[:, :, :K]
    return flat(m + 8 * sign), e - base, flat(values)


def mx4_integers(codes, shifts):
    """-> Python integers as an object array: 2 * e2m1 * 2^shift"""
    mag = np.array([0, 1, 2, 3, 4, 6, 8, 12], object)[codes & 7] * np.where(codes & 8, -1, 1)
    two = np.array([1 << s for s in range(256)], object)[shifts]
    return mag * np.repeat(two, 32, axis=-1)[:, :, :codes.shape[2]]


def mx4_unpack(buf, E, M, K):
    """prepared buffer -> (codes [E][M][K], shifts [E][M][ceil(K / 32)], everything else zero)"""
    mt, kt = -(-M // 32), -(-K // 64)
    t = buf.reshape(E, mt, kt, 1088)
    by = t[..., :1024].reshape(E, mt, kt, 32, 32)
    codes = np.concatenate([by & 15, by >> 4], axis=-1).transpose(0, 1, 3, 2, 4).reshape(E, mt * 32, kt * 64)
    shifts = t[..., 1024:].reshape(E, mt, kt, 32, 2).transpose(0, 1, 3, 2, 4).reshape(E, mt * 32, kt * 2)
    rest = codes.copy()
    rest[:, :M, :K] = 0
    return codes[:, :M, :K], shifts[:, :M, :(K + 31) // 32], not rest.any()


def w8_unpack(buf, E, M, K):
    mt, kt = -(-M // 32), -(-K // 64)
    t = buf.view(np.int8).reshape(E, mt, kt, 32, 4, 16)
    out = np.zeros((E, mt, kt, 32, 4, 16), np.int8)
    for r in range(32):
        for q in range(4):
            out[:, :, :, r, q] = t[:, :, :, r, q ^ (r // 2 % 4) ^ (r // 8 % 2)]
    return out.reshape(E, mt, kt, 32, 64).transpose(0, 1, 3, 2, 4).reshape(E, mt * 32, kt * 64)


def experts(x, W, route, top_k, p, bias=None, one=None):
    """x [T][K][lam]; W integer [E][M][K] (object or int); route [n] -> [n][M][lam]"""
    n, M = len(route), W.shape[1]
    wp = (W % p).astype(np.int64)
    out = np.zeros((n, M, x.shape[2]), np.int64)
    for r, e in enumerate(route):
        if 0 <= e < W.shape[0]:
            # float64 holds the sums: residues below 127, K below 2^39
            y = np.rint(wp[e].astype(np.float64) @ x[r // top_k].astype(np.float64)).astype(np.int64)
            if bias is not None:
                y += (bias[e].astype(np.int64) % p)[:, None] * one.astype(np.int64)[None, :]
            out[r] = y % p
    return out


def combine(x, gates, p):
    """x [T][top_k][V][lam], gates [T][top_k] -> [T][V][lam]"""
    return (x.astype(np.int64) * (gates.astype(np.int64) % p)[:, :, None, None]).sum(1) % p
