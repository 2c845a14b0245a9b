"""The microscaled 4-bit formats in 64 bits, from their definition (numpy; no code of the package): every rounding is a search over the
representable values, a tie goes to the even code."""
import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def e4m3_values():
    """the positive E4M3 values, by code 1 .. 126"""
    c = np.arange(1, 127)
    e, m = c >> 3, c & 7
    return np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))


def nearest(y, grid, first_code):
    """index into `grid` (ascending, codes from first_code) of the value nearest to y, ties to the even code, saturating"""
    hi = np.clip(np.searchsorted(grid, y), 0, len(grid) - 1)
    lo = np.maximum(hi - 1, 0)
    dl, dh = np.abs(y - grid[lo]), np.abs(grid[hi] - y)
    return np.where((dl < dh) | ((dl == dh) & ((lo + first_code) % 2 == 0)), lo, hi)


def quantize(x, nv, ceil_rule=False, top=np.inf):
    """x [R, K] float64 -> codes [R, K], scale codes [R, blocks], factors [R]; a NaN's block: scale code 255 / 127"""
    x = np.clip(np.asarray(x, np.float64), -top, top)                  # (a NaN stays)
    R, K = x.shape
    n = 16 if nv else 32
    b = np.zeros((R, -(-K // n) * n))
    b[:, :K] = x
    b = b.reshape(R, -1, n)
    bad = np.isnan(b).any(-1)
    mag = np.abs(b)
    a = np.where(bad, 0.0, np.max(np.nan_to_num(mag), -1))
    if nv:
        row = np.max(np.where(np.isnan(x), 0.0, np.abs(x)), -1, initial=0.0)
        factor = np.array([2.0 ** next(t for t in range(-126, 200) if r <= 2688 * 2.0 ** t) if r > 0 else 1.0 for r in row])
        grid = e4m3_values()
        want = a / (6 * factor[:, None])
        code = np.where(a > 0, nearest(want, grid, 1) + 1, 0)
        s = np.where(code > 0, grid[np.maximum(code, 1) - 1], 0.0) * factor[:, None]
        code = np.where(bad, 127, code)
    else:
        factor = np.ones(R)
        f, e = np.frexp(a)                                              # a = f 2^e, f in [0.5, 1)
        E = e - 3 + (f > 0.75) if ceil_rule else e - 3
        E = np.clip(np.where(a > 0, E, -127), -127, 127)
        s = np.ldexp(1.0, E)
        code = np.where(bad, 255, E + 127)
    q = nearest(np.nan_to_num(mag) / np.where(s > 0, s, 1.0)[..., None], E2M1, 0)
    q = np.where((s > 0)[..., None], q, 0) | (np.signbit(b).astype(np.int64) << 3)
    return q.reshape(R, -1)[:, :K].astype(np.uint8), code.astype(np.uint8), factor


def values(codes, scales, factor, nv):
    """float64 values of codes [R, K] (one each), scale codes and factors"""
    v = E2M1[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    if nv:
        s = np.concatenate([[0.0], e4m3_values(), [np.nan]])[scales & 127]
        return v * np.repeat(s, 16, 1)[:, :codes.shape[1]] * np.asarray(factor, np.float64)[:, None]
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return v * np.repeat(s, 32, 1)[:, :codes.shape[1]]


def pack(codes):
    """one code each -> two to a byte, the lower index in the low nibble"""
    if codes.shape[-1] % 2:
        codes = np.concatenate([codes, np.zeros_like(codes[..., :1])], -1)
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def unpack(b, K):
    return np.stack([b & 15, b >> 4], -1).reshape(b.shape[:-1] + (-1,))[..., :K]
